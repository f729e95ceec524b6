// Rotary positions, and new tokens' K and V on their way into a paged cache (h2o_rotate, h2o_pages_append).
//
// A pair of channels (a, b) at position p with frequency f turns by t = p f:  a' = a cos t - b sin t,  b' = b cos t + a sin t.
// p f is a product in 64 bits, reduced to turns: t / 2 pi minus the nearest integer, at most half a turn, becomes fp32 and
// goes to sincospif.  (In fp32 the angle of position 1e6 would be off by 0.06.)  A block computes the sines and cosines of
// its token once, into shared memory, and all heads use them; so the kernel is bound by memory: every value read once,
// written once.  Products are fp32, rounded to the type once.
#include "pages.cuh"

namespace h2o {

namespace {

constexpr int kThreads = 128;
constexpr int kMaxHalf = 256;  // pairs of a head (head_dim up to 512)

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
__device__ __forceinline__ int sequence_of(const int32_t* cu, int batch, int64_t t) {
  const int lane = threadIdx.x & 31;
  int lo = 0, n = batch;
  while (n > 0) {
    const int step = (n + 31) / 32, at = lo + lane * step;
    const unsigned below = __ballot_sync(0xffffffffu, lane * step < n && cu[at] <= t);
    const int c = __popc(below);
    if (c == 0) return -1;
    lo += (c - 1) * step;
    if (step == 1) break;
    n = min(step, n - (c - 1) * step);
  }
  return cu[lo] <= t && t < cu[lo + 1] ? lo : -1;
}

// How the channels of a head are shared out to threads.  An item is what a thread moves at once:
//   Halves      two chunks, one in each half of the rotated channels (or two of those that are not)
//   Neighbours  two chunks in a row
//   Single      one pair of channels, or two of those that are not rotated
enum class Kind { Halves, Neighbours, Single };

template <typename T, Kind KIND>
__global__ void __launch_bounds__(kThreads) move_kernel(const __grid_constant__ MoveArgs a) {
  constexpr int N = Chunk<T>::N;
  __shared__ float2 cs[kMaxHalf];
  const int64_t t = blockIdx.x;
  const int half = a.turn.half;
  // ---- the token's sequence and row ----
  int64_t row = 0;
  T *to_k = nullptr, *to_v = nullptr;
  if (a.kv_heads > 0) {
    int s = a.cu ? sequence_of(a.cu, a.batch, t) : t < a.batch ? (int)t : -1;
    if (s < 0) return;  // (the whole block: the token belongs to no sequence)
    row = (int64_t)a.length[s] - (a.cu ? (int64_t)a.cu[s + 1] - t : 1);
    if (row >= 0 && row < a.max_length && row / a.page_size < a.max_pages) {
      const int x = (int)row;
      const int page = a.table[s * a.table_stride + x / a.page_size];
      if (page >= 0 && page < a.n_pages && H2O_IN_RANGE(page, a.n_pages, a.status)) {
        const int64_t at = page * a.page_stride + x % a.page_size * a.row_stride;
        to_k = static_cast<T*>(a.pk) + at;
        to_v = static_cast<T*>(a.pv) + at;
      }
    }
  }
  // ---- sines and cosines ----
  for (int i = threadIdx.x; i < half; i += kThreads) {
    int64_t p = row;
    if (a.turn.positions) p = a.turn.positions[(a.turn.axis ? min((int)a.turn.axis[i], a.turn.axes - 1) : 0) * a.turn.position_stride + t];
    double turns = (double)p * a.turn.frequency[i] * 0.15915494309189533577;  // 1 / 2 pi
    turns -= rint(turns);
    float s, c;
    sincospif(2.f * (float)turns, &s, &c);
    cs[i] = make_float2(c, a.turn.inverse ? -s : s);
  }
  __syncthreads();
  // ---- the heads ----
  const int per = KIND == Kind::Single ? a.dim / 2 : a.dim / (2 * N);  // items of a head
  const int turned = half / N;                                         // of them with a rotation (Halves)
  const int items = (a.q_heads + 2 * a.kv_heads) * per;
  for (int i = blockIdx.y * kThreads + threadIdx.x; i < items; i += gridDim.y * kThreads) {
    int head = i / per;
    const int c = i - head * per;
    const T* from;
    T* to;
    bool turn;
    if (head < a.q_heads) {
      from = static_cast<const T*>(a.q) + t * a.q_stride + (int64_t)head * a.dim;
      to = static_cast<T*>(a.q_out) + t * a.q_out_stride + (int64_t)head * a.dim;
      turn = a.q_turn;
    } else {
      head -= a.q_heads;
      const bool is_v = head >= a.kv_heads;
      if (is_v) head -= a.kv_heads;
      from = static_cast<const T*>(is_v ? a.v : a.k) + t * a.kv_stride + (int64_t)head * a.dim;
      to = is_v ? to_v : to_k;
      if (!to) continue;
      to += head * a.head_stride;
      turn = !is_v && a.k_turn;
    }
    if constexpr (KIND == Kind::Single) {
      const bool apart = a.turn.halves && c < half;
      const int x0 = apart ? c : 2 * c, x1 = apart ? c + half : 2 * c + 1;
      turn = turn && c < half;
      float2 x = make_float2((float)from[x0], (float)from[x1]);
      if (turn) x = turn_of(x, cs[c]);
      to[x0] = (T)x.x;
      to[x1] = (T)x.y;
    } else {
      const int x0 = KIND == Kind::Halves && c < turned ? c * N : 2 * c * N;
      const int x1 = KIND == Kind::Halves && c < turned ? c * N + half : x0 + N;
      Chunk<T> u, w;
      u.load(from + x0);
      w.load(from + x1);
      if (turn && (KIND == Kind::Halves ? c < turned : x0 < 2 * half)) {
        float f[N], g[N];
        u.numbers(f);
        w.numbers(g);
        if constexpr (KIND == Kind::Halves) {
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const float2 y = turn_of(make_float2(f[e], g[e]), cs[c * N + e]);
            f[e] = y.x;
            g[e] = y.y;
          }
        } else {
#pragma unroll
          for (int e = 0; e < N; e += 2) {
            const int i0 = (x0 + e) / 2, i1 = (x1 + e) / 2;
            if (i0 < half) {
              const float2 y = turn_of(make_float2(f[e], f[e + 1]), cs[i0]);
              f[e] = y.x;
              f[e + 1] = y.y;
            }
            if (i1 < half) {
              const float2 y = turn_of(make_float2(g[e], g[e + 1]), cs[i1]);
              g[e] = y.x;
              g[e + 1] = y.y;
            }
          }
        }
        u.set(f);
        w.set(g);
      }
      u.store(to + x0);
      w.store(to + x1);
    }
  }
}

template <typename T>
cudaError_t launch(const MoveArgs& a, cudaStream_t stream) {
  constexpr int N = Chunk<T>::N;
  // pairs of chunks need a head of whole pairs of chunks and, for halves, rotated channels of whole pairs
  const bool chunks = a.dim % (2 * N) == 0;
  const Kind kind = !chunks || (a.turn.halves && a.turn.half % N != 0) ? Kind::Single : a.turn.halves ? Kind::Halves : Kind::Neighbours;
  const int64_t items = (int64_t)(a.q_heads + 2 * a.kv_heads) * (kind == Kind::Single ? a.dim / 2 : a.dim / (2 * N));
  const dim3 grid((unsigned)a.n_tokens, (unsigned)((items + 4 * kThreads - 1) / (4 * kThreads)));
  if (kind == Kind::Halves) move_kernel<T, Kind::Halves><<<grid, kThreads, 0, stream>>>(a);
  else if (kind == Kind::Neighbours) move_kernel<T, Kind::Neighbours><<<grid, kThreads, 0, stream>>>(a);
  else move_kernel<T, Kind::Single><<<grid, kThreads, 0, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_move(const MoveArgs& a, int dtype, cudaStream_t stream) {
  return dtype == H2O_F32 ? launch<float>(a, stream) : launch<__nv_bfloat16>(a, stream);
}

}  // namespace h2o
