// Host side of the paged K/V cache and of rotary positions (h2o_pages_*, h2o_rotate of include/h2o.h): argument checks, how a
// call is cut into blocks, launches.  Nothing is allocated on the device; a call's parts go through the caller's scratch.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "pages.cuh"

namespace {

constexpr int kMaxGroup = 32, kMaxAxes = 8, kMaxHeadDim = 512, kMaxPageSize = 65536;
constexpr int64_t kMaxStride = 1ll << 36;

bool misaligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }

struct DeviceGuard {
  int prev = -1;
  bool ok = false, changed = false;
  explicit DeviceGuard(int dev) {
    if (cudaGetDevice(&prev) != cudaSuccess) return;
    ok = prev == dev || cudaSetDevice(dev) == cudaSuccess;
    changed = ok && prev != dev;
  }
  ~DeviceGuard() {
    if (changed) cudaSetDevice(prev);
  }
};

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

h2o::Turn turn_of(const h2o_rotary_t* r, const int64_t* positions, int64_t stride, int64_t n_tokens, int inverse) {
  h2o::Turn t = {};
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

// The softmax scale for logits in base 2.
float base2(float scale) { return (float)((double)scale * 1.4426950408889634074); }

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
bool nothing_to_do(const h2o_queries_t* q) { return q->batch == 0 || q->q_rows == 0 || q->max_q == 0; }
int check_pointers(const h2o_queries_t* q) {
  if (!q->q || !q->out || misaligned(q->q, 16) || misaligned(q->out, 16) || misaligned(q->lse, 4)) return H2O_ERR_INVALID_ARG;
  return q->q == q->out ? H2O_ERR_INVALID_ARG : H2O_OK;
}
int check_attend(const h2o_pages_t* pages, const h2o_queries_t* q, const h2o_sequences_t* s, int window, int sinks) {
  int rc = check_queries(pages, q);
  if (rc != H2O_OK) return rc;
  if (window < 0 || sinks < 0) return H2O_ERR_INVALID_ARG;
  return nothing_to_do(q) ? H2O_OK : check_sequences(s);
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
  h2o::MoveArgs a = {};
  a.q = x;
  a.q_out = out;
  a.q_stride = x_stride;
  a.q_out_stride = out_stride;
  a.n_tokens = n_tokens;
  a.q_heads = n_heads;
  a.dim = head_dim;
  a.q_turn = 1;
  a.turn = turn_of(rotary, positions, position_stride, n_tokens, inverse != 0);
  DeviceGuard guard(rotary->device);
  if (!guard.ok) return H2O_ERR_CUDA;
  return launched(h2o::launch_move(a, dtype, static_cast<cudaStream_t>(stream)));
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
  p->polls = h2o::kStorePolls;
  if (cfg->page_stride == 0) {
    p->cfg.head_stride = cfg->head_dim;
    p->cfg.row_stride = (int64_t)cfg->n_heads * cfg->head_dim;
    p->cfg.page_stride = p->cfg.row_stride * cfg->page_size;
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
  pages->polls = polls < 0 ? h2o::kStorePolls : std::min((uint32_t)polls, h2o::kStorePolls);
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
  h2o::MoveArgs a = {};
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
  return launched(h2o::launch_move(a, c.format, static_cast<cudaStream_t>(stream)));
}

size_t h2o_pages_scratch_bytes(const h2o_pages_t* pages, const h2o_queries_t* queries, const h2o_sequences_t* sequences,
                               int32_t window, int32_t sinks) {
  if (check_attend(pages, queries, sequences, window, sinks) != H2O_OK || nothing_to_do(queries)) return 0;
  return 0;
}

int h2o_pages_attend(h2o_pages_t* pages, const h2o_queries_t* queries, const h2o_sequences_t* sequences, int32_t window,
                     int32_t sinks, void* scratch, size_t scratch_bytes, void* stream) {
  int rc = check_attend(pages, queries, sequences, window, sinks);
  if (rc != H2O_OK || nothing_to_do(queries)) return rc;
  rc = check_pointers(queries);
  if (rc != H2O_OK) return rc;
  const h2o_pages_config_t& c = pages->cfg;
  const h2o_queries_t* q = queries;
  h2o::PagesAttend p = {};
  h2o::AttendView& a = p.a;
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
  a.max_q = std::min<int64_t>(q->max_q, q->q_rows);
  a.scale2 = base2(q->softmax_scale > 0.f ? q->softmax_scale : 1.0f / std::sqrt((float)a.dim));
  a.k = c.k;
  a.v = c.v;
  a.status = c.status;
  a.part[0].length = sequences->length;
  a.part[0].max_length = (int)std::min<int64_t>(sequences->max_length, (int64_t)sequences->max_pages * c.page_size);
  p.table = sequences->table;
  p.table_stride = sequences->table_stride ? sequences->table_stride : sequences->max_pages;
  p.page_stride = c.page_stride;
  p.row_stride = c.row_stride;
  p.head_stride = c.head_stride;
  p.n_pages = c.n_pages;
  p.page_size = c.page_size;
  p.max_pages = sequences->max_pages;
  p.window = window;
  p.sinks = sinks;
  DeviceGuard guard(c.device);
  if (!guard.ok) return H2O_ERR_CUDA;
  return launched(h2o::launch_pages_attend_simple(p, c.format, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
