// Internal declarations of the K/V store operators (h2o_store_*, h2o_cross_attend, h2o_prefix_attend).
//
// A store is caller-owned K and V rows that many queries read and nothing evicts.  An attention call is one or two
// PARTS: a part is a list of problems, each a range of query tokens against a range of store rows; the keys of a
// problem can be split into chunks whose results are joined afterwards (each chunk leaves its normalised output and
// the logarithm of its sum of exponentials).
//   cross attention    one part: a problem per sequence
//   shared prefix      part 0: a problem per group of sequences (all their query tokens against the group's prefix),
//                      part 1: a problem per sequence against its own rows, causal
#pragma once
#include "h2o_internal.cuh"

// The handle: host memory only.
struct h2o_store {
  h2o_store_config_t cfg;  // strides filled in
  uint32_t polls;          // of a wait before it gives up
  // tensor maps of the rows (opaque here): boxes for few query rows, and for many in blocks of one and of two groups
  alignas(64) unsigned char few_k[128], few_v[128], one_k[128], one_v[128], two_k[128], two_v[128];
};

namespace h2o {

constexpr int kMaxSplits = 64;  // of a part's keys
// Polls of a wait before it gives up (tens of milliseconds; what is waited for takes microseconds), and of the waits for a
// block's own copies and products that end a block that has given up.
constexpr uint32_t kStorePolls = 1u << 22;

struct AttendPart {
  const int64_t* begin;    // dev [problems]: first store row
  const int32_t* length;   // dev [problems]: rows
  int max_length;          // upper bound of the lengths (longer ones are cut)
  int problems;            // sequences, or groups of sequences
  int grouped;             // 1: a problem is a group (its token range comes from cu_group)
  int causal;              // 1: query i of n sees all rows but the last n - 1 - i
  int chunk, splits;       // keys per split, splits per problem (of the longest)
  int row_tiles;           // tiles of query rows per problem (of the longest)
  int slot0;               // first partial slot of this part
};

struct AttendView {
  const void* q;
  void* out;
  float* lse;              // nullable
  int64_t q_stride, out_stride, q_rows;  // elements between tokens; tokens
  const int32_t* cu_q;     // dev [batch + 1], or null: token b belongs to sequence b
  const int32_t* cu_group; // dev [n_groups + 1], or null: one group of all sequences
  int batch, n_groups, max_q, max_group;
  int heads, group, dim;   // K/V heads, query heads per K/V head
  float scale2;            // softmax scale times log2(e)
  const void *k, *v;
  const uint8_t *k_scale, *v_scale;  // 8-bit rows only
  int64_t rows, row_stride;
  float *part_out, *part_lse;  // [slots][q_rows][heads * group](dim), null when nothing goes through them
  int slots;
  // early: part 1's kernel is launched to start before part 0's has ended.  finish (with early): part 1, unsplit, writes the
  // results, joined with what part 0 left; otherwise every part leaves its chunks for the joining kernel, or there is one
  // unsplit part that writes the results.
  int early, finish;
  int walk;  // 1: part 1's blocks take the prefix as well, and nothing else is launched (few rows of the mma.sync kernel)
  int32_t* status;
  uint32_t polls;  // of a wait before it gives up
  int n_parts;
  AttendPart part[2];
};

// A problem's query tokens and store rows, cut to what the caller allowed for, so that no index leaves its array
// whatever the device arrays hold.
struct Problem {
  int64_t t0, row0;  // first query token, first store row
  int nt, len;       // tokens, rows
};
__device__ __forceinline__ int64_t clamp64(int64_t x, int64_t lo, int64_t hi) { return x < lo ? lo : (x > hi ? hi : x); }
__device__ __forceinline__ int64_t first_token(const AttendView& a, int seq) {
  return clamp64(a.cu_q ? (int64_t)a.cu_q[seq] : (int64_t)seq, 0, a.q_rows);
}
__device__ __forceinline__ Problem locate(const AttendView& a, const AttendPart& p, int i) {
  int s0 = i, s1 = i + 1;
  int64_t most = a.max_q;
  if (p.grouped) {
    s0 = a.cu_group ? max(0, min(a.cu_group[i], a.batch)) : 0;
    s1 = a.cu_group ? max(s0, min(a.cu_group[i + 1], a.batch)) : a.batch;
    s1 = min(s1, s0 + a.max_group);
    most *= a.max_group;
  }
  Problem r;
  r.t0 = first_token(a, s0);
  r.nt = (int)clamp64(first_token(a, s1) - r.t0, 0, most);
  r.row0 = clamp64(p.begin[i], 0, a.rows);
  r.len = (int)clamp64(p.length[i], 0, min((int64_t)p.max_length, a.rows - r.row0));
  return r;
}
// In the checked build: may these be used?  (Elsewhere always.)
__device__ __forceinline__ bool token_ok(const AttendView& a, int64_t token, int hq) {
  return H2O_IN_RANGE(token, a.q_rows, a.status) && H2O_IN_RANGE(hq, a.heads * a.group, a.status);
}
__device__ __forceinline__ bool row_ok(const AttendView& a, int head, int64_t row) {
  return H2O_IN_RANGE(row, a.rows, a.status) && H2O_IN_RANGE(head, a.heads, a.status);
}
__device__ __forceinline__ bool partial_ok(const AttendView& a, int64_t at) {
  return H2O_IN_RANGE(at, a.slots * a.q_rows * a.heads * a.group, a.status);
}
// Rows of a problem that its query token `i` sees.
__device__ __forceinline__ int seen_rows(const AttendPart& p, const Problem& r, int i) {
  return p.causal ? max(0, r.len - (r.nt - 1 - i)) : r.len;
}

// The group of a sequence: the last one that starts at or before it.
__device__ __forceinline__ int group_of(const AttendView& a, int seq) {
  if (!a.cu_group) return 0;
  int lo = 0, hi = a.n_groups;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.cu_group[mid] <= seq) lo = mid;
    else hi = mid;
  }
  return lo;
}

// What part 0 left for the query tokens of one sequence (a.finish): its chunks' results, joined with part 1's own.
struct Prefix {
  int used;         // chunks
  int64_t t0, t1;   // tokens that part 0 has worked on: others are left as they were
  __device__ __forceinline__ int64_t at(const AttendView& a, int s, int64_t token, int hq) const {
    return ((int64_t)(a.part[0].slot0 + s) * a.q_rows + token) * a.heads * a.group + hq;
  }
};
__device__ __forceinline__ Prefix prefix_of(const AttendView& a, int seq) {
  const Problem pr = locate(a, a.part[0], group_of(a, seq));
  return Prefix{(pr.len + a.part[0].chunk - 1) / a.part[0].chunk, pr.t0, pr.t0 + pr.nt};
}
// The largest of the chunks' logarithms and `top`; then the sum of the chunks' weights relative to it.
__device__ __forceinline__ float prefix_top(const AttendView& a, const Prefix& f, int64_t token, int hq, float top) {
  for (int s = 0; s < f.used; ++s)
    if (partial_ok(a, f.at(a, s, token, hq))) top = fmaxf(top, a.part_lse[f.at(a, s, token, hq)]);
  return top;
}
__device__ __forceinline__ float prefix_sum(const AttendView& a, const Prefix& f, int64_t token, int hq, float top) {
  float sum = 0.f;
  for (int s = 0; s < f.used; ++s)
    if (partial_ok(a, f.at(a, s, token, hq))) sum += exp2f(a.part_lse[f.at(a, s, token, hq)] - top);
  return sum;
}
// Waits until the kernels before this one have ended (nothing to wait for in an ordinary launch).
__device__ __forceinline__ void wait_for_earlier() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// What one thread block works on: row tile fastest, then head, split, problem.
struct BlockWork {
  int problem, head, split, row_tile;
};
__device__ __forceinline__ BlockWork block_work(const AttendView& a, const AttendPart& p, unsigned idx) {
  BlockWork w;
  w.row_tile = idx % p.row_tiles;
  idx /= p.row_tiles;
  w.head = idx % a.heads;
  idx /= a.heads;
  w.split = idx % p.splits;
  w.problem = idx / p.splits;
  return w;
}
inline int64_t part_blocks(const AttendView& a, const AttendPart& p) {
  return (int64_t)p.row_tiles * a.heads * p.splits * p.problems;
}

// The value of a scale byte (a biased exponent).  Only bytes 112 .. 134 are ever written here; others, in rows nobody has
// written or of a caller's own, are cut to that range, where every code times the scale is an f16 number.
__device__ __forceinline__ float kv8_scale(uint32_t byte) { return __uint_as_float(min(max(byte, 112u), 134u) << 23); }

// Softmax scale (times log2(e)) times the power of two of an f16 query row.  Kept a normal number: a factor of 0 would make
// NaN of a hidden key's -infinity, an infinite one of a logit of 0.  (Below the smallest one every logit is 0 up to 2^-100.)
__device__ __forceinline__ float f16_row_factor(float scale2, int e2) {
  return fminf(fmaxf(scale2 * __uint_as_float((uint32_t)(127 + e2) << 23), 1.17549435e-38f), 3.40282347e38f);
}

// Launches `kernel`, `early`: it may start before the kernel in front of it has ended.
template <typename... Args>
cudaError_t launch_kernel(void (*kernel)(Args...), dim3 grid, int threads, int smem, cudaStream_t stream, bool early, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = early ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// Launchers.
cudaError_t launch_store_write(const h2o_store_config_t& c, const void* k, const void* v, int dtype, int64_t stride,
                               int64_t n, const int64_t* rows, int64_t first_row, cudaStream_t stream);
cudaError_t launch_store_read(const h2o_store_config_t& c, void* k, void* v, int dtype, int64_t stride, int64_t n,
                              const int64_t* rows, int64_t first_row, cudaStream_t stream);
int attend_fma_row_tile(int64_t rows);
cudaError_t launch_attend_fma(const AttendView& a, int part, int tile, int format, cudaStream_t stream);
constexpr int kFewBoxRows = 32;  // rows of a box of the store's tensor maps
bool make_store_map(CUtensorMap_st* map, const h2o_store_config_t& c, const void* base, int box_rows);
int attend_mma_row_tile(int64_t rows);
int attend_mma_blocks_per_sm(int format, int tile);
// part `first`, or (both) parts 0 and 1 in one launch, or (a.walk) part 1 with the prefix
cudaError_t launch_attend_mma(const AttendView& a, int first, bool both, const int* tile, int format, const void* map_k,
                              const void* map_v, cudaStream_t stream);
int attend_tc_box_rows(int format, int dim, int groups);
// `groups` of 128 query rows to a block
cudaError_t launch_attend_tc(const AttendView& a, int part, int groups, int format, const void* map_k, const void* map_v,
                             cudaStream_t stream);
cudaError_t launch_attend_join(const AttendView& a, int q_dtype, cudaStream_t stream);

}  // namespace h2o
