// Host side of the paged K/V cache and of rotary positions (h2o_pages_*, h2o_rotate of include/h2o.h): argument checks, how a
// call is cut into blocks, launches.  Nothing is allocated on the device; a call's parts go through the caller's scratch.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <numeric>

#include "pages.cuh"
#include "store_plan.cuh"

namespace {

using namespace h2o;

constexpr int kMaxAxes = 8, kMaxHeadDim = 512, kMaxPageSize = 65536;
constexpr int64_t kMaxStride = 1ll << 36;
constexpr int kMaxRows = INT32_MAX - 4096;  // of a sequence (tiles of them are counted in 32 bits)

int check_pages(const h2o_pages_config_t* c) {
  if (!c || !c->k || !c->v) return H2O_ERR_INVALID_ARG;
  if (c->n_heads < 1 || c->n_pages < 1 || c->page_size < 1 || c->device < 0) return H2O_ERR_INVALID_ARG;
  if (c->format != H2O_F32 && c->format != H2O_BF16) return H2O_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return H2O_ERR_UNSUPPORTED;
  if (c->page_size % 8 != 0 || c->page_size > kMaxPageSize || c->n_heads > 65535) return H2O_ERR_UNSUPPORTED;
  if (misaligned(c->k, 16) || misaligned(c->v, 16)) return H2O_ERR_INVALID_ARG;
  const int64_t s[3] = {c->page_stride, c->row_stride, c->head_stride};
  if (s[0] == 0 && s[1] == 0 && s[2] == 0) return H2O_OK;
  for (int64_t x : s) {
    if (x < c->head_dim || x % 8 != 0) return H2O_ERR_INVALID_ARG;
    if (x > kMaxStride) return H2O_ERR_UNSUPPORTED;
  }
  return H2O_OK;
}

int check_rotary(const h2o_rotary_t* r, int head_dim) {
  if (!r || !r->frequency || misaligned(r->frequency, 8)) return H2O_ERR_INVALID_ARG;
  if (r->rotary_dim < 2 || r->rotary_dim > head_dim || r->rotary_dim % 2 != 0) return H2O_ERR_INVALID_ARG;
  if (r->axes < 1 || r->device < 0 || (r->pairs != 0 && r->pairs != 1)) return H2O_ERR_INVALID_ARG;
  return r->axes > kMaxAxes ? H2O_ERR_UNSUPPORTED : H2O_OK;
}

// A stride between tokens of rows of `dense` elements, filled in.
bool bad_stride(int64_t& s, int64_t dense) {
  if (s == 0) s = dense;
  return s < dense || s % 8 != 0;
}

Turn turn_of(const h2o_rotary_t* r, const int64_t* positions, int64_t stride, int64_t n_tokens, int inverse) {
  Turn t = {};
  if (!r) return t;
  t.frequency = r->frequency;
  t.axis = r->axis;
  t.positions = positions;
  t.position_stride = stride ? stride : n_tokens;
  t.half = r->rotary_dim / 2;
  t.axes = r->axes;
  t.halves = r->pairs == 0;
  t.inverse = inverse;
  return t;
}

int check_sequences(const h2o_sequences_t* s) {
  if (!s || s->max_length < 0 || s->max_pages < 0 || s->table_stride < 0) return H2O_ERR_INVALID_ARG;
  if (!s->length || misaligned(s->length, 4) || misaligned(s->table, 4) || (!s->table && s->max_pages > 0)) return H2O_ERR_INVALID_ARG;
  if (s->table_stride != 0 && s->table_stride < s->max_pages) return H2O_ERR_INVALID_ARG;
  return s->table_stride > kMaxStride ? H2O_ERR_UNSUPPORTED : H2O_OK;
}

int check_queries(const h2o_pages_t* pages, const h2o_queries_t* q) {
  if (!pages || !q) return H2O_ERR_INVALID_ARG;
  if (q->batch < 0 || q->q_rows < 0 || q->max_q < 0 || q->q_stride < 0 || q->out_stride < 0) return H2O_ERR_INVALID_ARG;
  if (q->query_group < 1) return H2O_ERR_INVALID_ARG;
  if (std::isnan(q->softmax_scale) || std::isinf(base2(q->softmax_scale))) return H2O_ERR_INVALID_ARG;
  const h2o_pages_config_t& c = pages->cfg;
  if (q->dtype != c.format || q->query_group > kMaxGroup) return H2O_ERR_UNSUPPORTED;
  if (q->batch > 65535 || q->q_rows > INT32_MAX) return H2O_ERR_UNSUPPORTED;
  if ((int64_t)c.n_heads * q->query_group > 65535) return H2O_ERR_UNSUPPORTED;
  if (!q->cu_q && (q->q_rows < q->batch || q->max_q > 1)) return H2O_ERR_INVALID_ARG;
  const int64_t dense = (int64_t)c.n_heads * q->query_group * c.head_dim;
  for (int64_t s : {q->q_stride, q->out_stride})
    if (s != 0 && (s < dense || s % 8 != 0)) return H2O_ERR_INVALID_ARG;
  return misaligned(q->cu_q, 4) ? H2O_ERR_INVALID_ARG : H2O_OK;
}
int check_attend(const h2o_pages_t* pages, const h2o_queries_t* q, const h2o_sequences_t* s, int window, int sinks) {
  int rc = check_queries(pages, q);
  if (rc != H2O_OK) return rc;
  if (window < 0 || sinks < 0) return H2O_ERR_INVALID_ARG;
  return nothing_to_do(q) ? H2O_OK : check_sequences(s);
}

// What a call launches and how much scratch it needs.
struct Plan {
  AttendView a;
  Kernel kernel;
  int tile;           // query rows of a block
  size_t scratch;     // bytes of scratch
  size_t lse_offset;  // of the partial log-sums in it
  int rc;
};

// More query rows than this (of one K/V head) run on the tcgen05 kernel: as for the K/V store.
constexpr int kFewRows = 16;

// Splits the keys of a prompt between the items of the tcgen05 kernel, `rows` query rows in each.  Costs in keys of one block, of
// which two share an SM and take 64 in a microsecond: an item costs its keys and 4 us more, the last ones to finish leave a
// quarter of an item's time unused; chunks cost the joining kernel's start and their rows' trip through memory and back.
void split_prompt(AttendPart& p, int64_t units, int64_t rows, int dim, int sms) {
  const int64_t len = std::max(1, p.most_keys), num = p.problems > 1 ? 2 : 3, room = 2 * sms, fixed = 256, step = 128;
  int64_t best = -1;
  for (int64_t n = 1; n <= kMaxSplits && (n == 1 || units * n <= 16 * room); ++n) {
    const int64_t chunk = ((len + n - 1) / n + step - 1) / step * step;
    const int64_t splits = (len + chunk - 1) / chunk, one = std::min(chunk, len) + fixed;
    int64_t cost = std::max(one, (units * len * num / 3 + units * splits * num / 3 * fixed) / room) + one / 4;
    if (splits > 1) cost += 200 + units * splits * num / 3 * rows * dim * 8 * 64 / 6400000;
    if (best < 0 || cost < best) {
      best = cost;
      p.chunk = (int)chunk;
      p.splits = (int)splits;
    }
    if (chunk == step) break;
  }
}

// Few units of few query rows: the blocks should all run at once.  split_part's costs lead to more chunks than that, and the blocks
// that find no place at first then run alone at the end: with heads of 128, of which two blocks fit an SM, 20000 keys of 8 heads
// take 24.1 us in 296 blocks and 32.1 in 384; of 32 heads 54.4 in 256 and 72.2 in 320.  With heads of 64 three fit (32 heads, 20000
// keys: 34.3 us in 384 blocks, 43.2 in 512).  A few places stay free, as each chunk costs the joining kernel about 0.1 us: 1.5
// blocks to an SM where two fit, 2 where three fit, there up to 32 chunks.  Of several sequences only the longest length is known;
// the lengths are taken to lie evenly between a third of it and it (two thirds on average), and a window to cut what is longer:
// `share` is what such a sequence has of the keys of the longest.  Without / with this, in us (bf16, K and V from memory, replayed
// from a graph): heads of 128: one sequence of 8 heads, 5000 keys 19.3 / 13.3, 20000 31.4 / 23.7, 33000 40.1 / 31.7; 4 of up to
// 20000 51.5 / 43.2; 4 with a window of 4000 23.9 / 18.8, of 10000 37.0 / 32.8; with 16 query heads to each of 8, 20000 keys 38.2 / 27.8;
// heads of 64: 8 heads, 5000 14.8 / 11.6; 32 heads, 20000 42.8 / 34.8; 4 of up to 20000 29.2 / 29.4, of up to 33000 50.0 / 41.  Of 294
// calls measured, seven lose 3 to 6 % (32 heads of 64 with 16 query heads each, 5000 keys: 17.9 / 19.0; a window of 1020, 8 sequences
// of 4 heads: 10.6 / 11.1); the mean gains 9 %.
void bound_chunks(AttendPart& p, int64_t units, int sms, int blocks_per_sm) {
  double share = 1.0;
  if (p.problems > 1) {
    const double longest = std::max(1, p.max_length), shortest = longest / 3, keys = std::max(1, p.most_keys);
    if (keys > shortest) share -= (keys - shortest) * (keys - shortest) / (2 * (longest - shortest) * keys);
  }
  const double per_sm = sms / (units * share), up = share == 1.0 ? 0.999 : 0.5;  // (lengths that are known: as many chunks as cover it)
  int64_t most = (int64_t)(1.5 * per_sm + up);
  if (blocks_per_sm > 2) most = std::max(most, std::min<int64_t>(32, (int64_t)(2 * per_sm + up)));
  if (p.splits > most) {
    p.chunk = (int)(((p.most_keys + most - 1) / most + 127) / 128 * 128);
    p.splits = (p.most_keys + p.chunk - 1) / p.chunk;
  }
}

Plan make_plan(const h2o_pages_t* pages, const h2o_queries_t* q, const h2o_sequences_t* s, int window, int sinks) {
  Plan pl;
  std::memset(&pl, 0, sizeof(pl));
  const h2o_pages_config_t& c = pages->cfg;
  AttendView& a = pl.a;
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
  a.batch = q->batch;
  a.n_groups = a.max_group = 1;
  a.max_q = (int)std::min<int64_t>(q->max_q, q->q_rows);
  a.scale2 = base2(q->softmax_scale > 0.f ? q->softmax_scale : 1.0f / std::sqrt((float)a.dim));
  a.k = c.k;
  a.v = c.v;
  a.rows = kMaxRows;
  a.row_stride = c.row_stride;
  a.status = c.status;
  a.polls = pages->polls;
  a.n_parts = 1;
  AttendPart& p = a.part[0];
  p.length = s->length;
  p.max_length = (int)std::min({(int64_t)s->max_length, (int64_t)s->max_pages * c.page_size, (int64_t)kMaxRows});
  p.causal = 1;
  p.problems = a.batch;
  Paging& g = a.pages;
  g.table = s->max_pages > 0 ? s->table : s->length;  // (without a single page no entry is read)
  g.stride = s->table_stride ? s->table_stride : s->max_pages;
  g.page_stride = c.page_stride;
  g.head_stride = c.head_stride;
  g.n_pages = c.n_pages;
  g.page_size = c.page_size;
  g.shift = (c.page_size & (c.page_size - 1)) == 0 ? (int)std::log2((double)c.page_size) : -1;
  g.window = window;
  g.sinks = sinks;
  const int64_t rows = (int64_t)a.max_q * a.group;
  if (c.format == H2O_F32) {
    pl.kernel = Kernel::Fma;
    pl.tile = attend_fma_row_tile(rows);
  } else {
    pl.kernel = rows <= kFewRows ? Kernel::Mma : Kernel::Tc1;
    pl.tile = rows <= kFewRows ? attend_mma_row_tile(rows) : 128;
  }
  g.box = pl.kernel == Kernel::Fma ? 8 : pl.kernel == Kernel::Mma ? pages->few_box : pages->many_box;
  // the most keys a tile of query rows walks over: sinks in whole tiles (of 64 keys at most), the window, as far as the tile's tokens
  // lie apart, and down to the box the window starts in
  p.most_keys = p.max_length;
  if (window > 0) {
    const int64_t span = std::min<int64_t>(a.max_q - 1, (pl.tile + a.group - 2) / a.group);
    const int64_t head = ((int64_t)std::min(sinks, p.max_length) + 63) / 64 * 64;
    p.most_keys = (int)std::min<int64_t>(p.max_length, head + window + span + g.box);
  }
  p.row_tiles = (int)((rows + pl.tile - 1) / pl.tile);
  const int64_t units = (int64_t)p.row_tiles * a.heads * p.problems;
  if (pl.kernel == Kernel::Tc1) split_prompt(p, units, std::min<int64_t>(rows, pl.tile), a.dim, sm_count(c.device));
  else split_part(p, p.most_keys, units, sm_count(c.device), pl.kernel, pl.tile, c.format, a.dim, 128, true);
  if (pl.kernel == Kernel::Mma && 4 * units <= sm_count(c.device)) bound_chunks(p, units, sm_count(c.device), attend_mma_paged_blocks_per_sm(a.dim, pl.tile));
  if (units * p.splits > INT32_MAX) pl.rc = H2O_ERR_UNSUPPORTED;
  if (p.splits > 1) {
    a.slots = p.splits;
    const size_t n = (size_t)p.splits * a.q_rows * a.heads * a.group;
    pl.lse_offset = align_up(n * a.dim * sizeof(float));
    pl.scratch = pl.lse_offset + align_up(n * sizeof(float));
  }
  return pl;
}

int launched(cudaError_t e) {
  if (e == cudaSuccess) return H2O_OK;
  cudaGetLastError();
  return H2O_ERR_CUDA;
}

}  // namespace

extern "C" {

int h2o_rotate(const h2o_rotary_t* rotary, const void* x, void* out, int32_t dtype, int64_t n_tokens, int32_t n_heads,
               int32_t head_dim, int64_t x_stride, int64_t out_stride, const int64_t* positions, int64_t position_stride,
               int32_t inverse, void* stream) {
  if (n_tokens < 0 || n_heads < 1 || head_dim < 1 || x_stride < 0 || out_stride < 0 || position_stride < 0) return H2O_ERR_INVALID_ARG;
  if (head_dim % 8 != 0 || head_dim > kMaxHeadDim || n_heads > 65535) return H2O_ERR_UNSUPPORTED;
  const int rc = check_rotary(rotary, head_dim);
  if (rc != H2O_OK) return rc;
  if (dtype != H2O_F32 && dtype != H2O_BF16) return H2O_ERR_UNSUPPORTED;
  if (n_tokens > INT32_MAX || position_stride > kMaxStride) return H2O_ERR_UNSUPPORTED;
  if (n_tokens == 0) return H2O_OK;
  if (!x || !out || !positions || misaligned(x, 16) || misaligned(out, 16) || misaligned(positions, 8)) return H2O_ERR_INVALID_ARG;
  const int64_t dense = (int64_t)n_heads * head_dim;
  if (bad_stride(x_stride, dense) || bad_stride(out_stride, dense)) return H2O_ERR_INVALID_ARG;
  if (position_stride != 0 && position_stride < n_tokens) return H2O_ERR_INVALID_ARG;
  if (x == out && x_stride != out_stride && n_tokens > 1) return H2O_ERR_INVALID_ARG;
  MoveArgs a = {};
  a.q = x;
  a.q_out = out;
  a.q_stride = x_stride;
  a.q_out_stride = out_stride;
  a.n_tokens = n_tokens;
  a.q_heads = n_heads;
  a.dim = head_dim;
  a.q_turn = 1;
  a.turn = turn_of(rotary, positions, position_stride, n_tokens, inverse != 0);
  a.status = rotary->status;
  DeviceGuard guard(rotary->device);
  if (!guard.ok) return H2O_ERR_CUDA;
  return launched(launch_move(a, dtype, static_cast<cudaStream_t>(stream)));
}

int h2o_pages_create(h2o_pages_t** out, const h2o_pages_config_t* cfg) {
  if (!out) return H2O_ERR_INVALID_ARG;
  const int rc = check_pages(cfg);
  if (rc != H2O_OK) return rc;
  int ndev = 0, major = 0;
  if (cudaGetDeviceCount(&ndev) != cudaSuccess) {
    cudaGetLastError();
    return H2O_ERR_CUDA;
  }
  if (cfg->device >= ndev) return H2O_ERR_INVALID_ARG;
  if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, cfg->device) != cudaSuccess) return H2O_ERR_CUDA;
  if (major != 10) return H2O_ERR_UNSUPPORTED;  // the kernels are built for sm_100a only
  h2o_pages* p = new (std::nothrow) h2o_pages();
  if (!p) return H2O_ERR_INVALID_ARG;
  p->cfg = *cfg;
  p->polls = kStorePolls;
  if (cfg->page_stride == 0) {
    p->cfg.head_stride = cfg->head_dim;
    p->cfg.row_stride = (int64_t)cfg->n_heads * cfg->head_dim;
    p->cfg.page_stride = p->cfg.row_stride * cfg->page_size;
  }
  if (cfg->format == H2O_BF16) {  // the kernels for bfloat16 read the pages by TMA
    p->few_box = std::gcd(cfg->page_size, kFewBoxRows);
    p->many_box = std::gcd(cfg->page_size, pages_tc_tile_keys());
    struct {
      unsigned char* map;
      const void* base;
      int box;
      bool whole;
    } const maps[4] = {{p->few_k, cfg->k, p->few_box, p->few_box == kFewBoxRows},
                       {p->few_v, cfg->v, p->few_box, p->few_box == kFewBoxRows},
                       {p->many_k, cfg->k, p->many_box, p->many_box == pages_tc_tile_keys()},
                       {p->many_v, cfg->v, p->many_box, true}};
    for (const auto& m : maps)
      if (!make_page_map(reinterpret_cast<CUtensorMap_st*>(m.map), p->cfg, m.base, m.box, m.whole)) {
        delete p;
        return H2O_ERR_CUDA;
      }
  }
  *out = p;
  return H2O_OK;
}

int h2o_pages_destroy(h2o_pages_t* pages) {
  delete pages;
  return H2O_OK;
}

int h2o_debug_pages_set_polls(h2o_pages_t* pages, int32_t polls) {
  if (!pages) return H2O_ERR_INVALID_ARG;
  pages->polls = polls < 0 ? kStorePolls : std::min((uint32_t)polls, kStorePolls);
  return H2O_OK;
}

int h2o_pages_append(h2o_pages_t* pages, const h2o_tokens_t* tokens, const h2o_sequences_t* sequences, const h2o_rotary_t* rotary,
                     void* stream) {
  if (!pages || !tokens) return H2O_ERR_INVALID_ARG;
  const h2o_pages_config_t& c = pages->cfg;
  h2o_tokens_t t = *tokens;
  if (t.n_tokens < 0 || t.batch < 0 || t.kv_stride < 0 || t.q_stride < 0 || t.q_out_stride < 0 || t.position_stride < 0) return H2O_ERR_INVALID_ARG;
  if (t.q && t.query_group < 1) return H2O_ERR_INVALID_ARG;
  if (t.n_tokens > INT32_MAX || t.batch > 65535 || t.position_stride > kMaxStride) return H2O_ERR_UNSUPPORTED;
  if (t.q && (int64_t)c.n_heads * t.query_group > 65535) return H2O_ERR_UNSUPPORTED;
  if (rotary) {
    const int rc = check_rotary(rotary, c.head_dim);
    if (rc != H2O_OK) return rc;
    if (rotary->device != c.device) return H2O_ERR_INVALID_ARG;
  }
  if (t.n_tokens == 0 || t.batch == 0) return H2O_OK;
  const int rc = check_sequences(sequences);
  if (rc != H2O_OK) return rc;
  if (!t.k || !t.v || misaligned(t.k, 16) || misaligned(t.v, 16) || misaligned(t.cu, 4) || misaligned(t.positions, 8)) return H2O_ERR_INVALID_ARG;
  if (!t.cu && t.n_tokens < t.batch) return H2O_ERR_INVALID_ARG;
  if (bad_stride(t.kv_stride, (int64_t)c.n_heads * c.head_dim)) return H2O_ERR_INVALID_ARG;
  if (t.position_stride != 0 && t.position_stride < t.n_tokens) return H2O_ERR_INVALID_ARG;
  MoveArgs a = {};
  if (t.q) {
    if (!t.q_out || misaligned(t.q, 16) || misaligned(t.q_out, 16)) return H2O_ERR_INVALID_ARG;
    const int64_t dense = (int64_t)c.n_heads * t.query_group * c.head_dim;
    if (bad_stride(t.q_stride, dense) || bad_stride(t.q_out_stride, dense)) return H2O_ERR_INVALID_ARG;
    if (t.q == t.q_out && t.q_stride != t.q_out_stride && t.n_tokens > 1) return H2O_ERR_INVALID_ARG;
    a.q = t.q;
    a.q_out = t.q_out;
    a.q_stride = t.q_stride;
    a.q_out_stride = t.q_out_stride;
    a.q_heads = c.n_heads * t.query_group;
  }
  a.k = t.k;
  a.v = t.v;
  a.kv_stride = t.kv_stride;
  a.n_tokens = t.n_tokens;
  a.kv_heads = c.n_heads;
  a.dim = c.head_dim;
  a.q_turn = a.k_turn = rotary != nullptr;
  a.turn = turn_of(rotary, t.positions, t.position_stride, t.n_tokens, 0);
  a.pk = c.k;
  a.pv = c.v;
  a.page_stride = c.page_stride;
  a.row_stride = c.row_stride;
  a.head_stride = c.head_stride;
  a.table = sequences->table;
  a.table_stride = sequences->table_stride ? sequences->table_stride : sequences->max_pages;
  a.length = sequences->length;
  a.cu = t.cu;
  a.n_pages = c.n_pages;
  a.page_size = c.page_size;
  a.max_pages = sequences->max_pages;
  a.max_length = sequences->max_length;
  a.batch = t.batch;
  a.status = c.status;
  DeviceGuard guard(c.device);
  if (!guard.ok) return H2O_ERR_CUDA;
  return launched(launch_move(a, c.format, static_cast<cudaStream_t>(stream)));
}

size_t h2o_pages_scratch_bytes(const h2o_pages_t* pages, const h2o_queries_t* queries, const h2o_sequences_t* sequences,
                               int32_t window, int32_t sinks) {
  if (check_attend(pages, queries, sequences, window, sinks) != H2O_OK || nothing_to_do(queries)) return 0;
  return make_plan(pages, queries, sequences, window, sinks).scratch;
}

int h2o_pages_attend(h2o_pages_t* pages, const h2o_queries_t* queries, const h2o_sequences_t* sequences, int32_t window,
                     int32_t sinks, void* scratch, size_t scratch_bytes, void* stream) {
  int rc = check_attend(pages, queries, sequences, window, sinks);
  if (rc != H2O_OK || nothing_to_do(queries)) return rc;
  rc = check_pointers(queries);
  if (rc != H2O_OK) return rc;
  Plan pl = make_plan(pages, queries, sequences, window, sinks);
  if (pl.rc != H2O_OK) return pl.rc;
  if (pl.scratch > 0) {
    if (!scratch || scratch_bytes < pl.scratch || misaligned(scratch, kAlign)) return H2O_ERR_WORKSPACE;
    pl.a.part_out = static_cast<float*>(scratch);
    pl.a.part_lse = reinterpret_cast<float*>(static_cast<char*>(scratch) + pl.lse_offset);
  }
  DeviceGuard guard(pages->cfg.device);
  if (!guard.ok) return H2O_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (pl.kernel == Kernel::Fma) e = launch_attend_fma(pl.a, 0, pl.tile, H2O_F32, st);
  else if (pl.kernel == Kernel::Mma) e = launch_attend_mma_paged(pl.a, pl.tile, pages->few_k, pages->few_v, st);
  else e = launch_pages_tc(pl.a, pages->many_k, pages->many_v, st);
  if (e == cudaSuccess && pl.scratch > 0) e = launch_attend_join(pl.a, pages->cfg.format, st);
  return launched(e);
}

}  // extern "C"
