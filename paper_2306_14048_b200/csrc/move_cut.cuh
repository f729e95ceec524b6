// How a launch of the rotating kernel is cut into blocks, and which head and channels an item of a block is: plain arithmetic,
// the same on the host (where a test goes over every item) and on the device.
#pragma once
#include <cstdint>

#ifdef __CUDACC__
#define H2O_BOTH __host__ __device__ __forceinline__
#else
#define H2O_BOTH inline
#endif

namespace h2o {

constexpr int kMoveThreads = 128;
constexpr int kMaxHalf = 256;  // pairs of a head (head_dim up to 512), or of a block's tokens together
constexpr int kMaxTokens = 8;  // of a block

// x / d for small numbers, by multiplication: the upper half of x * (2^32 / d + 1) (exact as long as x * d < 2^32).  The factor of
// d = 1 does not fit 32 bits: it is 0, and the mask lets x through.
struct Divisor {
  uint32_t factor, mask;
};
inline Divisor divisor(int d) { return d > 1 ? Divisor{(uint32_t)((1ull << 32) / (uint32_t)d) + 1, 0u} : Divisor{0u, ~0u}; }
H2O_BOTH int quotient(int x, Divisor d) {
#ifdef __CUDA_ARCH__
  return (int)(__umulhi((uint32_t)x, d.factor) + ((uint32_t)x & d.mask));
#else
  return (int)(((uint64_t)(uint32_t)x * d.factor >> 32) + ((uint32_t)x & d.mask));
#endif
}

// `tokens` to a block, which share its threads and their sines; `items` of a token, `per` of them to a head.
struct MoveCut {
  int tokens, per, items;
  Divisor by_per, by_items;  // (by_items of one token to a block: 0, whatever is divided)
  // Item i of a block: which of its tokens, which head of that, which of the head's items.
  H2O_BOTH void split(int i, int& token, int& head, int& c) const {
    token = quotient(i, by_items);
    i -= token * items;
    head = quotient(i, by_per);
    c = i - head * per;
  }
};

// Cuts a launch for `heads` heads of each of n_tokens tokens.  `parts`: blocks that share the items of the same tokens.
inline MoveCut move_cut(int64_t n_tokens, int heads, int per, int half, int sms, int64_t& parts) {
  MoveCut cut;
  cut.per = per;
  cut.items = heads * per;
  // Few tokens: blocks enough that a thread has one item.  Many: each token's sines computed once, several tokens to a block as long
  // as that leaves a thread up to four items.
  const int64_t most = (cut.items + kMoveThreads - 1) / kMoveThreads;
  cut.tokens = 1;
  parts = most;
  if (n_tokens * most > 8 * sms) {
    parts = (cut.items + 8 * kMoveThreads - 1) / (8 * kMoveThreads);
    int fit = kMaxTokens;
    if (4 * kMoveThreads / cut.items < fit) fit = 4 * kMoveThreads / cut.items;
    if (half > 0 && kMaxHalf / half < fit) fit = kMaxHalf / half;
    if (fit > 1) cut.tokens = fit;
  }
  cut.by_per = divisor(cut.per);
  cut.by_items = cut.tokens > 1 ? divisor(cut.items) : Divisor{0u, 0u};
  return cut;
}

}  // namespace h2o
