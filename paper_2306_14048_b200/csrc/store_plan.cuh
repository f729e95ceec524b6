// Host-side pieces that the K/V store and the paged cache share: small checks, and how a part's keys are split into chunks.
#pragma once
#include <algorithm>

#include "store.cuh"

namespace h2o {

constexpr size_t kAlign = 256;
constexpr int kMaxGroup = 32;

inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
inline bool misaligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }

struct DeviceGuard {
  int prev = -1;
  bool ok = false;
  explicit DeviceGuard(int dev) {
    if (cudaGetDevice(&prev) != cudaSuccess) return;
    ok = prev == dev || cudaSetDevice(dev) == cudaSuccess;
    changed = ok && prev != dev;
  }
  ~DeviceGuard() {
    if (changed) cudaSetDevice(prev);
  }
  bool changed = false;
};

// The softmax scale for logits in base 2.
inline float base2(float scale) { return (float)((double)scale * 1.4426950408889634074); }

inline bool nothing_to_do(const h2o_queries_t* q) { return q->batch == 0 || q->q_rows == 0 || q->max_q == 0; }
inline int check_pointers(const h2o_queries_t* q) {
  if (!q->q || !q->out || misaligned(q->q, 16) || misaligned(q->out, 16) || misaligned(q->lse, 4)) return H2O_ERR_INVALID_ARG;
  if (q->q == q->out) return H2O_ERR_INVALID_ARG;
  return H2O_OK;
}

enum class Kernel { Fma, Mma, Tc1, Tc2 };  // (tcgen05: one or two groups of 128 rows to a block)
inline bool is_tc(Kernel k) { return k == Kernel::Tc1 || k == Kernel::Tc2; }

// Up to this many keys in a range the tcgen05 kernel takes 128 rows to a block, two blocks to an SM, so that one's start
// and end run beside the other's tiles (bfloat16; the 8-bit kernel's shared memory holds one).  Own rows of 64 prompts of up
// to 200 tokens behind a shared prefix: 117 -> 89 us; beside it, 515 keys for 32 heads of 131 tokens: 100 -> 108.
constexpr int kShortKeys = 512;

// Splits the `keys` of a part: `units` blocks per split, `room` blocks that run at once.  Costs in keys of one block: a block
// costs its keys and `fixed` more (start, merge, its result's trip through memory), the joining kernel twice as much;
// a block that has its SM to itself is taken to run twice as fast, and the last blocks to finish to leave a quarter of a
// block's time unused.  Only the longest length is known here: the lengths of a batch's sequences (`ragged`) are taken
// to average two thirds of it.  Chunks are multiples of `step` keys, what a block takes at a time.
inline void split_part(AttendPart& p, int keys, int64_t units, int sms, Kernel kernel, int tile, int format, int dim, int64_t step, bool ragged) {
  // Fixed costs: about 3 us at a block's share of the memory's 6.4 TB/s; of the tcgen05 kernel 8 us at 80 keys in 1 us, of
  // the FMA kernel 2 us at 64 keys in 3.5.
  const int key_bytes = 2 * dim * (format == H2O_KV8 ? 1 : format == H2O_BF16 ? 2 : 4);
  const bool tiles = kernel == Kernel::Fma && tile >= 16;
  const int per_sm = kernel == Kernel::Tc2 ? 1 : kernel == Kernel::Tc1 || tiles ? 2 : kernel == Kernel::Fma ? 4 : attend_mma_blocks_per_sm(format, tile);
  const int64_t room = (int64_t)sms * per_sm;
  const int64_t fixed = is_tc(kernel) ? 640 : tiles ? 36 : 19200000 / (room * key_bytes);
  if (tiles) step = 64;
  const int64_t len = std::max(1, keys), num = ragged ? 2 : 3;
  int64_t best = -1;
  for (int64_t n = 1; n <= kMaxSplits && (n == 1 || units * n <= 16 * room); ++n) {
    const int64_t chunk = ((len + n - 1) / n + step - 1) / step * step;
    const int64_t splits = (len + chunk - 1) / chunk;
    const int64_t one = std::min(chunk, len) + fixed;
    const int64_t blocks = std::max(units, units * splits * num / 3);
    int64_t cost = std::max(one / 2, (units * len * num / 3 + blocks * fixed) / room) + one / 4;
    if (splits > 1) cost += 2 * fixed;
    if (best < 0 || cost < best) {
      best = cost;
      p.chunk = (int)chunk;
      p.splits = (int)splits;
    }
    if (chunk == step) break;
  }
}

}  // namespace h2o
