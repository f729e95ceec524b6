// Host side of the K/V store operators of include/h2o.h: argument checks, how a call is cut into blocks, launches.
// Nothing is allocated on the device; a call's parts go through the caller's scratch.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "store_plan.cuh"

namespace {

using namespace h2o;

int check_store(const h2o_store_config_t* c) {
  if (!c || !c->k || !c->v) return H2O_ERR_INVALID_ARG;
  if (c->n_heads < 1 || c->rows < 1 || c->device < 0 || c->row_stride < 0) return H2O_ERR_INVALID_ARG;
  if (c->format != H2O_F32 && c->format != H2O_BF16 && c->format != H2O_KV8) return H2O_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return H2O_ERR_UNSUPPORTED;
  if (c->rows > INT32_MAX || c->n_heads > 65535) return H2O_ERR_UNSUPPORTED;
  if (misaligned(c->k, 16) || misaligned(c->v, 16)) return H2O_ERR_INVALID_ARG;
  const int64_t dense = (int64_t)c->n_heads * c->head_dim;
  if (c->format == H2O_KV8) {
    if (!c->k_scale || !c->v_scale) return H2O_ERR_INVALID_ARG;
    if (c->row_stride != 0) return H2O_ERR_INVALID_ARG;
    if (c->rows * c->n_heads > INT32_MAX) return H2O_ERR_UNSUPPORTED;  // rows of all heads are counted in 32 bits
  } else {
    if (c->row_stride != 0 && (c->row_stride < dense || c->row_stride % 8 != 0)) return H2O_ERR_INVALID_ARG;
    if (c->row_stride > (1ll << 36)) return H2O_ERR_UNSUPPORTED;
  }
  return H2O_OK;
}

int check_rows(const h2o_store_t* store, const void* k, const void* v, int dtype, int64_t n, int64_t& stride,
               const int64_t* rows, int64_t first_row) {
  if (!store) return H2O_ERR_INVALID_ARG;
  const h2o_store_config_t& c = store->cfg;
  if (c.format != H2O_KV8) return H2O_ERR_UNSUPPORTED;
  if (n < 0 || stride < 0) return H2O_ERR_INVALID_ARG;
  if (dtype != H2O_F32 && dtype != H2O_BF16) return H2O_ERR_UNSUPPORTED;
  if (n == 0) return H2O_OK;
  if (!k || !v || misaligned(k, 16) || misaligned(v, 16) || misaligned(rows, 8)) return H2O_ERR_INVALID_ARG;
  const int64_t dense = (int64_t)c.n_heads * c.head_dim;
  if (stride == 0) stride = dense;
  if (stride < dense || stride % 8 != 0) return H2O_ERR_INVALID_ARG;
  if (!rows && (first_row < 0 || first_row > c.rows - n)) return H2O_ERR_INVALID_ARG;
  if (n > INT32_MAX) return H2O_ERR_UNSUPPORTED;
  return H2O_OK;
}

int check_queries(const h2o_store_t* store, const h2o_queries_t* q) {
  if (!store || !q) return H2O_ERR_INVALID_ARG;
  if (q->batch < 0 || q->q_rows < 0 || q->max_q < 0 || q->q_stride < 0 || q->out_stride < 0) return H2O_ERR_INVALID_ARG;
  if (q->query_group < 1 || q->query_group > kMaxGroup) return q->query_group < 1 ? H2O_ERR_INVALID_ARG : H2O_ERR_UNSUPPORTED;
  if (std::isnan(q->softmax_scale) || std::isinf(base2(q->softmax_scale))) return H2O_ERR_INVALID_ARG;
  const h2o_store_config_t& c = store->cfg;
  if (q->dtype != H2O_F32 && q->dtype != H2O_BF16) return H2O_ERR_UNSUPPORTED;
  if (c.format != H2O_KV8 && q->dtype != c.format) return H2O_ERR_UNSUPPORTED;
  if (q->batch > 65535 || q->q_rows > INT32_MAX) return H2O_ERR_UNSUPPORTED;
  if ((int64_t)c.n_heads * q->query_group > 65535) return H2O_ERR_UNSUPPORTED;
  if (!q->cu_q && (q->q_rows < q->batch || q->max_q > 1)) return H2O_ERR_INVALID_ARG;
  const int64_t dense = (int64_t)c.n_heads * q->query_group * c.head_dim;
  for (int64_t s : {q->q_stride, q->out_stride})
    if (s != 0 && (s < dense || s % 8 != 0)) return H2O_ERR_INVALID_ARG;
  if (misaligned(q->cu_q, 4)) return H2O_ERR_INVALID_ARG;
  return H2O_OK;
}
int check_ranges(const h2o_ranges_t* r) {
  if (!r || r->max_length < 0) return H2O_ERR_INVALID_ARG;
  if (!r->begin || !r->length || misaligned(r->begin, 8) || misaligned(r->length, 4)) return H2O_ERR_INVALID_ARG;
  return H2O_OK;
}

// What a call launches and how much scratch it needs.
struct Plan {
  h2o::AttendView a;
  Kernel kernel[2];   // per part
  int tile[2];        // query rows of a block, per part
  size_t scratch;     // bytes of scratch
  size_t lse_offset;  // of the partial log-sums in it
  int rc;
};

// More query rows than this (of one K/V head) run on the tcgen05 kernel, 256 to a block; up to it the mma.sync kernel,
// which reads each key once as well and has less to set up.  One sequence of 16384 rows, mma.sync against tcgen05 (us):
// bfloat16, 8 heads of 128, 16 query rows 30 / 26, 20 rows 36 / 26; 32 heads 61 / 65 and 69 / 65; 16 heads of 64: 28 / 37
// and 37 / 37.  8-bit, 8 heads of 128, 32 query rows 26 / 28; 32 heads 61 / 73.
int few_rows(int format) { return format == H2O_KV8 ? 32 : 16; }

// Prefix and own rows together up to this many keys: each sequence's blocks read the prefix again (from the second-level
// cache) rather than leave chunks for a joining kernel.  Device time of a call, joined / walked, prefix 300, up to 60 own
// rows, 4 sequences, 8 heads of 128: 7.8 / 6.2 us, 8-bit 8.5 / 8.2; 660 keys: 6.6 / 7.4; and a launch less, 15 / 12 us a call.
// Up to two blocks to an SM: prefix 400, 16 heads, 16 sequences: 11.7 / 8.4; 32 sequences, 8-bit: 16.4 / 17.7.
constexpr int kWalkKeys = 512;

Plan make_plan(const h2o_store_t* store, const h2o_queries_t* q, const h2o_ranges_t* prefix, int n_groups,
               const int32_t* cu_group, int max_group, const h2o_ranges_t* own) {
  Plan pl;
  std::memset(&pl, 0, sizeof(pl));
  const h2o_store_config_t& c = store->cfg;
  const int sms = h2o::sm_count(c.device);
  h2o::AttendView& a = pl.a;
  a.q = q->q;
  a.out = q->out;
  a.lse = q->lse;
  a.heads = c.n_heads;
  a.group = q->query_group;
  a.dim = c.head_dim;
  const int64_t dense = (int64_t)a.heads * a.group * a.dim;
  a.q_stride = q->q_stride ? q->q_stride : dense;
  a.out_stride = q->out_stride ? q->out_stride : dense;
  a.q_rows = q->q_rows;
  a.cu_q = q->cu_q;
  a.cu_group = cu_group;
  a.batch = q->batch;
  a.n_groups = n_groups;
  a.max_q = std::min<int64_t>(q->max_q, q->q_rows);
  a.max_group = std::min(max_group, q->batch);
  const float scale = q->softmax_scale > 0.f ? q->softmax_scale : 1.0f / std::sqrt((float)a.dim);
  a.scale2 = base2(scale);
  a.k = c.k;
  a.v = c.v;
  a.k_scale = c.k_scale;
  a.v_scale = c.v_scale;
  a.rows = c.rows;
  a.row_stride = c.row_stride;
  a.status = c.status;
  a.polls = store->polls;
  int n = 0;
  for (int k = 0; k < 2; ++k) {
    const h2o_ranges_t* r = k == 0 ? prefix : own;
    if (!r) continue;
    h2o::AttendPart& p = a.part[n];
    p.begin = r->begin;
    p.length = r->length;
    p.max_length = (int)std::min<int64_t>(r->max_length, c.rows);
    p.grouped = prefix && k == 0;
    p.causal = prefix && k == 1;
    p.problems = p.grouped ? n_groups : a.batch;
    const int64_t rows = std::min<int64_t>((p.grouped ? (int64_t)a.max_group * a.max_q : a.max_q), a.q_rows) * a.group;
    if (q->dtype == H2O_F32) {
      pl.kernel[n] = Kernel::Fma;
      pl.tile[n] = h2o::attend_fma_row_tile(rows);
    } else if (rows <= few_rows(c.format)) {
      pl.kernel[n] = Kernel::Mma;
      pl.tile[n] = h2o::attend_mma_row_tile(rows);
    } else {
      pl.kernel[n] = c.format == H2O_BF16 && p.max_length <= kShortKeys ? Kernel::Tc1 : Kernel::Tc2;
      pl.tile[n] = pl.kernel[n] == Kernel::Tc1 ? 128 : 256;
    }
    p.row_tiles = (int)((rows + pl.tile[n] - 1) / pl.tile[n]);
    const int64_t units = (int64_t)p.row_tiles * a.heads * p.problems;
    split_part(p, p.max_length, units, sms, pl.kernel[n], pl.tile[n], c.format, a.dim, 128, !p.grouped);
    if (units * p.splits > INT32_MAX) pl.rc = H2O_ERR_UNSUPPORTED;
    p.slot0 = n == 0 ? 0 : a.part[0].splits;
    ++n;
  }
  a.n_parts = n;
  if (n == 2 && pl.kernel[0] == Kernel::Mma && pl.kernel[1] == Kernel::Mma && pl.tile[1] == 8 &&
      (int64_t)a.part[0].max_length + a.part[1].max_length <= kWalkKeys &&
      (int64_t)a.part[1].problems * a.part[1].row_tiles * a.heads <= 2 * sms) {
    a.walk = 1;
    a.part[1].splits = 1;
    a.part[1].chunk = std::max(1, a.part[1].max_length);
    return pl;
  }
  // The second part's kernel, where it is one of its own, starts before the first one's has ended: neither needs the
  // other's results until the end.  Prompts' own rows, unsplit, then join what the first part left themselves (32 prompts
  // of up to 200 tokens: 415 -> 348 us); single tokens' blocks are many and short, and leave that to the joining kernel.
  a.early = n == 2 && is_tc(pl.kernel[0]);
  a.finish = a.early && a.part[1].splits == 1 && is_tc(pl.kernel[1]);
  const int64_t slots = (int64_t)a.part[0].splits + (n == 2 && !a.finish ? a.part[1].splits : 0);
  if (slots > 1 || a.finish) {
    a.slots = (int)slots;
    const size_t rows = (size_t)slots * a.q_rows * a.heads * a.group;
    pl.lse_offset = align_up(rows * a.dim * sizeof(float));
    pl.scratch = pl.lse_offset + align_up(rows * sizeof(float));
  }
  return pl;
}

int run_plan(const h2o_store_t* store, const h2o_queries_t* q, Plan& pl, void* scratch, size_t scratch_bytes, void* stream) {
  if (pl.rc != H2O_OK) return pl.rc;
  if (pl.scratch > 0) {
    if (!scratch || scratch_bytes < pl.scratch || misaligned(scratch, kAlign)) return H2O_ERR_WORKSPACE;
    pl.a.part_out = static_cast<float*>(scratch);
    pl.a.part_lse = reinterpret_cast<float*>(static_cast<char*>(scratch) + pl.lse_offset);
  }
  DeviceGuard guard(store->cfg.device);
  if (!guard.ok) return H2O_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  const int format = store->cfg.format;
  const bool both = pl.a.n_parts == 2 && !pl.a.walk && pl.kernel[0] == Kernel::Mma && pl.kernel[1] == Kernel::Mma;
  for (int k = 0; k < (both || pl.a.walk ? 1 : pl.a.n_parts) && e == cudaSuccess; ++k) {
    if (pl.kernel[k] == Kernel::Fma) e = h2o::launch_attend_fma(pl.a, k, pl.tile[k], format, st);
    else if (pl.kernel[k] == Kernel::Tc2) e = h2o::launch_attend_tc(pl.a, k, 2, format, store->two_k, store->two_v, st);
    else if (pl.kernel[k] == Kernel::Tc1) e = h2o::launch_attend_tc(pl.a, k, 1, format, store->one_k, store->one_v, st);
    else e = h2o::launch_attend_mma(pl.a, k, both, pl.tile, format, store->few_k, store->few_v, st);
  }
  if (e == cudaSuccess && pl.scratch > 0 && !pl.a.finish) e = h2o::launch_attend_join(pl.a, q->dtype, st);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return H2O_ERR_CUDA;
  }
  return H2O_OK;
}

int check_cross(const h2o_store_t* store, const h2o_queries_t* q, const h2o_ranges_t* r) {
  int rc = check_queries(store, q);
  if (rc == H2O_OK && !nothing_to_do(q)) rc = check_ranges(r);
  return rc;
}
int check_prefix(const h2o_store_t* store, const h2o_queries_t* q, const h2o_ranges_t* prefix, int n_groups,
                 const int32_t* cu_group, int max_group, const h2o_ranges_t* own) {
  int rc = check_queries(store, q);
  if (rc != H2O_OK || nothing_to_do(q)) return rc;
  rc = check_ranges(prefix);
  if (rc == H2O_OK) rc = check_ranges(own);
  if (rc != H2O_OK) return rc;
  if (n_groups < 1 || max_group < 1 || misaligned(cu_group, 4)) return H2O_ERR_INVALID_ARG;
  if (!cu_group && (n_groups != 1 || max_group < q->batch)) return H2O_ERR_INVALID_ARG;
  if (n_groups > 65535) return H2O_ERR_UNSUPPORTED;
  return H2O_OK;
}

}  // namespace

extern "C" {

int h2o_store_create(h2o_store_t** out, const h2o_store_config_t* cfg) {
  if (!out) return H2O_ERR_INVALID_ARG;
  const int rc = check_store(cfg);
  if (rc != H2O_OK) return rc;
  int ndev = 0, major = 0;
  if (cudaGetDeviceCount(&ndev) != cudaSuccess) {
    cudaGetLastError();
    return H2O_ERR_CUDA;
  }
  if (cfg->device >= ndev) return H2O_ERR_INVALID_ARG;
  if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, cfg->device) != cudaSuccess) return H2O_ERR_CUDA;
  if (major != 10) return H2O_ERR_UNSUPPORTED;  // the kernels are built for sm_100a only
  h2o_store* s = new (std::nothrow) h2o_store();
  if (!s) return H2O_ERR_INVALID_ARG;
  s->cfg = *cfg;
  s->polls = h2o::kStorePolls;
  if (s->cfg.row_stride == 0) s->cfg.row_stride = (int64_t)cfg->n_heads * cfg->head_dim;
  // the kernels for bfloat16 queries read the rows by TMA
  if (cfg->format != H2O_F32) {
    struct {
      unsigned char* map;
      const void* base;
      int box;
    } const maps[6] = {{s->few_k, cfg->k, h2o::kFewBoxRows},
                       {s->few_v, cfg->v, h2o::kFewBoxRows},
                       {s->one_k, cfg->k, h2o::attend_tc_box_rows(cfg->format, cfg->head_dim, 1)},
                       {s->one_v, cfg->v, h2o::attend_tc_box_rows(cfg->format, cfg->head_dim, 1)},
                       {s->two_k, cfg->k, h2o::attend_tc_box_rows(cfg->format, cfg->head_dim, 2)},
                       {s->two_v, cfg->v, h2o::attend_tc_box_rows(cfg->format, cfg->head_dim, 2)}};
    for (const auto& m : maps)
      if (!h2o::make_store_map(reinterpret_cast<CUtensorMap_st*>(m.map), s->cfg, m.base, m.box)) {
        delete s;
        return H2O_ERR_CUDA;
      }
  }
  *out = s;
  return H2O_OK;
}

int h2o_store_destroy(h2o_store_t* store) {
  delete store;
  return H2O_OK;
}

int h2o_debug_store_set_polls(h2o_store_t* store, int32_t polls) {
  if (!store) return H2O_ERR_INVALID_ARG;
  store->polls = polls < 0 ? h2o::kStorePolls : std::min((uint32_t)polls, h2o::kStorePolls);
  return H2O_OK;
}

int h2o_store_write(h2o_store_t* store, const void* k, const void* v, int32_t dtype, int64_t n_tokens, int64_t stride,
                    const int64_t* rows, int64_t first_row, void* stream) {
  const int rc = check_rows(store, k, v, dtype, n_tokens, stride, rows, first_row);
  if (rc != H2O_OK || n_tokens == 0) return rc;
  DeviceGuard guard(store->cfg.device);
  if (!guard.ok) return H2O_ERR_CUDA;
  if (h2o::launch_store_write(store->cfg, k, v, dtype, stride, n_tokens, rows, first_row, static_cast<cudaStream_t>(stream)) != cudaSuccess) {
    cudaGetLastError();
    return H2O_ERR_CUDA;
  }
  return H2O_OK;
}

int h2o_store_read(h2o_store_t* store, void* k, void* v, int32_t dtype, int64_t n_tokens, int64_t stride,
                   const int64_t* rows, int64_t first_row, void* stream) {
  const int rc = check_rows(store, k, v, dtype, n_tokens, stride, rows, first_row);
  if (rc != H2O_OK || n_tokens == 0) return rc;
  DeviceGuard guard(store->cfg.device);
  if (!guard.ok) return H2O_ERR_CUDA;
  if (h2o::launch_store_read(store->cfg, k, v, dtype, stride, n_tokens, rows, first_row, static_cast<cudaStream_t>(stream)) != cudaSuccess) {
    cudaGetLastError();
    return H2O_ERR_CUDA;
  }
  return H2O_OK;
}

size_t h2o_cross_scratch_bytes(const h2o_store_t* store, const h2o_queries_t* queries, const h2o_ranges_t* ranges) {
  if (check_cross(store, queries, ranges) != H2O_OK || nothing_to_do(queries)) return 0;
  return make_plan(store, queries, nullptr, 0, nullptr, 0, ranges).scratch;
}

int h2o_cross_attend(h2o_store_t* store, const h2o_queries_t* queries, const h2o_ranges_t* ranges, void* scratch,
                     size_t scratch_bytes, void* stream) {
  int rc = check_cross(store, queries, ranges);
  if (rc != H2O_OK || nothing_to_do(queries)) return rc;
  rc = check_pointers(queries);
  if (rc != H2O_OK) return rc;
  Plan pl = make_plan(store, queries, nullptr, 0, nullptr, 0, ranges);
  return run_plan(store, queries, pl, scratch, scratch_bytes, stream);
}

size_t h2o_prefix_scratch_bytes(const h2o_store_t* store, const h2o_queries_t* queries, const h2o_ranges_t* prefix,
                                int32_t n_groups, const int32_t* cu_group, int32_t max_group, const h2o_ranges_t* own) {
  if (check_prefix(store, queries, prefix, n_groups, cu_group, max_group, own) != H2O_OK || nothing_to_do(queries)) return 0;
  return make_plan(store, queries, prefix, n_groups, cu_group, max_group, own).scratch;
}

int h2o_prefix_attend(h2o_store_t* store, const h2o_queries_t* queries, const h2o_ranges_t* prefix, int32_t n_groups,
                      const int32_t* cu_group, int32_t max_group, const h2o_ranges_t* own, void* scratch,
                      size_t scratch_bytes, void* stream) {
  int rc = check_prefix(store, queries, prefix, n_groups, cu_group, max_group, own);
  if (rc != H2O_OK || nothing_to_do(queries)) return rc;
  rc = check_pointers(queries);
  if (rc != H2O_OK) return rc;
  Plan pl = make_plan(store, queries, prefix, n_groups, cu_group, max_group, own);
  return run_plan(store, queries, pl, scratch, scratch_bytes, stream);
}

}  // extern "C"
