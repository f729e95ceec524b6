// Rotary positions, and new tokens' K and V on their way into a paged cache (h2o_rotate, h2o_pages_append).
//
// A pair of channels (a, b) at position p with frequency f turns by t = p f:  a' = a cos t - b sin t,  b' = b cos t + a sin t.
// p f is a product in 64 bits, reduced to turns: t / 2 pi minus the nearest integer, at most half a turn, becomes fp32 and
// goes to sincospif.  (In fp32 the angle of position 1e6 would be off by 0.06.)  A block computes the sines and cosines of
// its tokens once, into shared memory, and all heads use them; so the kernel is bound by memory: every value read once,
// written once.  Products are fp32, rounded to the type once.
// Appending 15121 tokens, 32 query and 32 K/V heads of 128, bfloat16: 122-125 us, 5.9-6.1 TB/s (a plain copy of as many bytes 6.3);
// 7785 tokens in float32 124 us, 6.2 TB/s.  Rotating 9001 tokens of 32 heads 31 us, 4.7 TB/s (a copy 27; here each block has a chain of its
// own, positions, sines, products, and an SM sees few of them in so short a launch), neighbouring pairs 35; float32 50 us, 5.9 TB/s.
// 64 tokens of a step: 2.9 us on the device.
#include <algorithm>

#include "move_cut.cuh"
#include "pages.cuh"

namespace h2o {

namespace {

constexpr int kThreads = kMoveThreads;
constexpr int kAhead = 2;      // items a thread has under way

// 16 bytes of a head's channels, as they lie in memory and as numbers.
template <typename T>
struct Chunk {
  static constexpr int N = 16 / sizeof(T);
  uint4 raw;
  __device__ __forceinline__ void load(const T* p) { raw = __ldcs(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<uint4*>(p) = raw; }
  __device__ __forceinline__ void numbers(float (&f)[N]) const {
    if constexpr (N == 8) {
      Vec16<__nv_bfloat16>::unpack(raw, f);
    } else {
      f[0] = __uint_as_float(raw.x); f[1] = __uint_as_float(raw.y); f[2] = __uint_as_float(raw.z); f[3] = __uint_as_float(raw.w);
    }
  }
  __device__ __forceinline__ void set(const float (&f)[N]) {
    if constexpr (N == 8) {
      raw.x = Vec16<__nv_bfloat16>::pack2(f[0], f[1]); raw.y = Vec16<__nv_bfloat16>::pack2(f[2], f[3]);
      raw.z = Vec16<__nv_bfloat16>::pack2(f[4], f[5]); raw.w = Vec16<__nv_bfloat16>::pack2(f[6], f[7]);
    } else {
      raw = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
  }
};

__device__ __forceinline__ float2 turn_of(float2 x, float2 cs) {
  return make_float2(fmaf(x.x, cs.x, -(x.y * cs.y)), fmaf(x.y, cs.x, x.x * cs.y));
}

// The last s with cu[s] <= t, found by a whole warp 32 entries at a time; -1 if t lies in no sequence.
__device__ __forceinline__ int sequence_of(const int32_t* cu, int batch, int64_t t, int32_t* status) {
  const int lane = threadIdx.x & 31;
  int lo = 0, n = batch;
  while (n > 0) {
    const int step = (n + 31) / 32, at = lo + lane * step;
    const unsigned below = __ballot_sync(0xffffffffu, lane * step < n && H2O_IN_RANGE(at, batch, status) && cu[at] <= t);
    const int c = __popc(below);
    if (c == 0) return -1;
    lo += (c - 1) * step;
    if (step == 1) break;
    n = min(step, n - (c - 1) * step);
  }
  return H2O_IN_RANGE(lo, batch, status) && cu[lo] <= t && t < cu[lo + 1] ? lo : -1;
}

// How the channels of a head are shared out to threads.  An item is what a thread moves at once:
//   Halves      two chunks, one in each half of the rotated channels (or two of those that are not)
//   Neighbours  two chunks in a row
//   Single      one pair of channels, or two of those that are not rotated: heads, or halves, that are not whole chunks.  Loads of 2 or
//               4 bytes, none of them ahead: 9001 tokens of 32 heads, bfloat16, 96 channels of which 24 rotate 59 us (1.9 TB/s), 80 of
//               which 20 50 us.
enum class Kind { Halves, Neighbours, Single };

// An item: where it comes from, where it goes (null: nowhere), which of its channels, and whether it is rotated; whether there is
// such an item (known only in the checked build, elsewhere always).
template <typename T>
struct Piece {
  const T* from;
  T* to;
  int x0, x1, pair, turns;  // first pair's angle, pairs from it on that are rotated (Neighbours)
  bool turn, ok;
};

constexpr int64_t kNoPage = -1, kNoSequence = -2;

template <typename T, Kind KIND>
__global__ void __launch_bounds__(kThreads) move_kernel(const __grid_constant__ MoveArgs a, const __grid_constant__ MoveCut cut) {
  constexpr int N = Chunk<T>::N;
  __shared__ float2 cs[kMaxHalf];
  __shared__ int64_t place[kMaxTokens], rows[kMaxTokens];  // of K and V of each token in the pages; its row
  const int64_t t0 = (int64_t)blockIdx.x * cut.tokens;
  const int here = (int)min((int64_t)cut.tokens, a.n_tokens - t0), half = a.turn.half;
  const int turned = half / N;  // items of a head with a rotation (Halves)
  const int items = cut.items * here;
  auto piece = [&](int i, bool to) {  // (to: where it goes is known by now)
    Piece<T> p;
    int k, head, c;
    cut.split(i, k, head, c);
    p.ok = H2O_IN_RANGE(k, here, a.status) && H2O_IN_RANGE(head, a.q_heads + 2 * a.kv_heads, a.status) && H2O_IN_RANGE(c, cut.per, a.status);
    const int64_t t = t0 + k;
    const int64_t at = a.kv_heads > 0 && to && p.ok ? place[k] : kNoPage;
    if (head < a.q_heads) {
      p.from = static_cast<const T*>(a.q) + t * a.q_stride + (int64_t)head * a.dim;
      p.to = at == kNoSequence ? nullptr : static_cast<T*>(a.q_out) + t * a.q_out_stride + (int64_t)head * a.dim;
      p.turn = a.q_turn;
    } else {
      head -= a.q_heads;
      const bool is_v = head >= a.kv_heads;
      if (is_v) head -= a.kv_heads;
      p.from = static_cast<const T*>(is_v ? a.v : a.k) + t * a.kv_stride + (int64_t)head * a.dim;
      p.to = at < 0 ? nullptr : static_cast<T*>(is_v ? a.pv : a.pk) + at + head * a.head_stride;
      p.turn = !is_v && a.k_turn;
    }
    if constexpr (KIND == Kind::Single) {
      const bool apart = a.turn.halves && c < half;
      p.x0 = apart ? c : 2 * c;
      p.x1 = apart ? c + half : 2 * c + 1;
      p.pair = k * half + c;
      p.turn = p.turn && c < half;
      p.ok = p.ok && H2O_IN_RANGE(max(p.x0, p.x1), a.dim, a.status) && (!p.turn || H2O_IN_RANGE(p.pair, half * here, a.status));
    } else {
      const bool apart = KIND == Kind::Halves && c < turned;
      p.x0 = apart ? c * N : 2 * c * N;
      p.x1 = apart ? c * N + half : p.x0 + N;
      p.pair = k * half + (apart ? c * N : p.x0 / 2);
      p.turns = half - (apart ? c * N : p.x0 / 2);
      p.turn = p.turn && (KIND == Kind::Halves ? apart : p.turns > 0);
      p.ok = p.ok && H2O_IN_RANGE(p.x1 + N - 1, a.dim, a.status) &&
             (!p.turn || H2O_IN_RANGE(p.pair + (KIND == Kind::Halves ? N : min(N, p.turns)) - 1, half * here, a.status));
    }
    if (!p.ok) {
      p.to = nullptr;
      p.turn = false;
    }
    return p;
  };
  // ---- the first items' values are asked for before anything is known about the token ----
  const int first = blockIdx.y * kThreads + threadIdx.x, stride = gridDim.y * kThreads;
  Chunk<T> u[kAhead], w[kAhead];
  if constexpr (KIND != Kind::Single) {
#pragma unroll
    for (int n = 0; n < kAhead; ++n)
      if (first + n * stride < items) {
        const Piece<T> p = piece(first + n * stride, false);
        if (!p.ok) continue;
        u[n].load(p.from + p.x0);
        w[n].load(p.from + p.x1);
      }
  }
  // ---- the tokens' sequences and rows ----
  if (a.kv_heads > 0) {
    for (int k = threadIdx.x >> 5; k < here; k += kThreads / 32) {
      const int64_t t = t0 + k;
      const int s = a.cu ? sequence_of(a.cu, a.batch, t, a.status) : t < a.batch ? (int)t : -1;
      int64_t row = 0, at = kNoSequence;
      if (s >= 0) {
        row = (int64_t)a.length[s] - (a.cu ? (int64_t)a.cu[s + 1] - t : 1);
        at = kNoPage;
        if (row >= 0 && row < a.max_length && row / a.page_size < a.max_pages) {
          const int x = (int)row, in = x / a.page_size;
          const int page = H2O_IN_RANGE(s, a.batch, a.status) && H2O_IN_RANGE(in, a.max_pages, a.status) ? a.table[s * a.table_stride + in] : -1;
          if (page >= 0 && page < a.n_pages) at = page * a.page_stride + x % a.page_size * a.row_stride;
        }
      }
      if ((threadIdx.x & 31) == 0) {
        place[k] = at;
        rows[k] = row;
      }
    }
    __syncthreads();
  }
  // ---- sines and cosines ----
  for (int i = threadIdx.x; i < half * here; i += kThreads) {
    const int k = here == 1 ? 0 : i / half, pair = i - k * half;
    if (!(H2O_IN_RANGE(k, here, a.status) && H2O_IN_RANGE(pair, half, a.status) && H2O_IN_RANGE(i, kMaxHalf, a.status))) continue;
    int64_t p;
    if (a.turn.positions) p = a.turn.positions[(a.turn.axis ? min((int)a.turn.axis[pair], a.turn.axes - 1) : 0) * a.turn.position_stride + t0 + k];
    else p = rows[k];
    double turns = (double)p * a.turn.frequency[pair] * 0.15915494309189533577;  // 1 / 2 pi
    turns -= rint(turns);
    float s, c;
    sincospif(2.f * (float)turns, &s, &c);
    cs[i] = make_float2(c, a.turn.inverse ? -s : s);
  }
  __syncthreads();
  // ---- the heads ----
  if constexpr (KIND == Kind::Single) {
    for (int i = first; i < items; i += stride) {
      const Piece<T> p = piece(i, true);
      if (!p.to) continue;
      float2 x = make_float2((float)p.from[p.x0], (float)p.from[p.x1]);
      if (p.turn) x = turn_of(x, cs[p.pair]);
      p.to[p.x0] = (T)x.x;
      p.to[p.x1] = (T)x.y;
    }
  } else {
    for (int at = first; at < items; at += kAhead * stride) {
#pragma unroll
      for (int n = 0; n < kAhead; ++n) {
        const int i = at + n * stride;
        if (i >= items) break;
        const Piece<T> p = piece(i, true);
        if (p.turn) {
          float f[N], g[N];
          u[n].numbers(f);
          w[n].numbers(g);
          if constexpr (KIND == Kind::Halves) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
              const float2 y = turn_of(make_float2(f[e], g[e]), cs[p.pair + e]);
              f[e] = y.x;
              g[e] = y.y;
            }
          } else {
#pragma unroll
            for (int e = 0; e < N; e += 2) {
              if (e / 2 < p.turns) {
                const float2 y = turn_of(make_float2(f[e], f[e + 1]), cs[p.pair + e / 2]);
                f[e] = y.x;
                f[e + 1] = y.y;
              }
              if (N / 2 + e / 2 < p.turns) {
                const float2 y = turn_of(make_float2(g[e], g[e + 1]), cs[p.pair + N / 2 + e / 2]);
                g[e] = y.x;
                g[e + 1] = y.y;
              }
            }
          }
          u[n].set(f);
          w[n].set(g);
        }
        if (p.to) {
          u[n].store(p.to + p.x0);
          w[n].store(p.to + p.x1);
        }
        if (i + kAhead * stride < items) {
          const Piece<T> next = piece(i + kAhead * stride, false);
          if (!next.ok) continue;
          u[n].load(next.from + next.x0);
          w[n].load(next.from + next.x1);
        }
      }
    }
  }
}

template <typename T>
cudaError_t launch(const MoveArgs& a, cudaStream_t stream) {
  constexpr int N = Chunk<T>::N;
  // pairs of chunks need a head of whole pairs of chunks and, for halves, rotated channels of whole pairs
  const bool chunks = a.dim % (2 * N) == 0;
  const Kind kind = !chunks || (a.turn.halves && a.turn.half % N != 0) ? Kind::Single : a.turn.halves ? Kind::Halves : Kind::Neighbours;
  const int per = kind == Kind::Single ? a.dim / 2 : a.dim / (2 * N);
  int64_t parts;
  const MoveCut cut = move_cut(a.n_tokens, a.q_heads + 2 * a.kv_heads, per, a.turn.half, sm_count(), parts);
  const dim3 grid((unsigned)((a.n_tokens + cut.tokens - 1) / cut.tokens), (unsigned)std::min<int64_t>(65535, parts));
  if (kind == Kind::Halves) move_kernel<T, Kind::Halves><<<grid, kThreads, 0, stream>>>(a, cut);
  else if (kind == Kind::Neighbours) move_kernel<T, Kind::Neighbours><<<grid, kThreads, 0, stream>>>(a, cut);
  else move_kernel<T, Kind::Single><<<grid, kThreads, 0, stream>>>(a, cut);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_move(const MoveArgs& a, int dtype, cudaStream_t stream) {
  return dtype == H2O_F32 ? launch<float>(a, stream) : launch<__nv_bfloat16>(a, stream);
}

}  // namespace h2o
