// K/V store in 8-bit floating point: rows quantised as they are written, and read back.
//
// A row of a head (head_dim channels of one token) becomes e4m3 codes and one power of two:
//   a = max |x| over the row's finite values
//   e = the smallest integer in [-15, 7] with a <= 448 * 2^e        (448 = the largest e4m3 value)
//   code = e4m3(min(max(x * 2^-e, -448), 448)), nearest, ties to even; NaN stays NaN
//   scale byte = e + 127
// The multiplication by a power of two is exact, so the code is decided by one rounding, the same in every precision.
// e4m3 keeps its own exponent per element, so a scale per row serves as well as one per small group of channels; the
// range of e makes every code * 2^e (4 significant bits, 2^-24 .. 57344) exactly a bf16, f16 and f32 number, which is
// what the attention kernels multiply.
#include <cuda_fp8.h>

#include "store.cuh"

namespace h2o {

namespace {

// Exponent e of a row whose largest finite magnitude is `a`: with a = m * 2^k, 1 <= m < 2, 448 = 1.75 * 2^8.
__device__ __forceinline__ int kv8_exponent(float a) {
  const uint32_t b = __float_as_uint(a);
  const int k = (int)(b >> 23) - 127;  // (zero and subnormals: far below the range, cut to -15)
  const int e = k - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
  return max(-15, min(7, e));
}

// 16 consecutive channels of an input row, as they lie in memory (few registers while the loads are under way) and as
// numbers; and of an output row.  Inputs are read once: a streaming load leaves the second-level cache to the store's rows.
template <typename T>
struct Raw16 {
  uint4 v[sizeof(T)];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) v[i] = __ldcs(reinterpret_cast<const uint4*>(p) + i);
  }
};
__device__ __forceinline__ void numbers(const Raw16<__nv_bfloat16>& r, float (&f)[16]) {
  float lo[8], hi[8];
  Vec16<__nv_bfloat16>::unpack(r.v[0], lo);
  Vec16<__nv_bfloat16>::unpack(r.v[1], hi);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    f[i] = lo[i];
    f[8 + i] = hi[i];
  }
}
__device__ __forceinline__ void numbers(const Raw16<float>& r, float (&f)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[4 * i] = __uint_as_float(r.v[i].x); f[4 * i + 1] = __uint_as_float(r.v[i].y);
    f[4 * i + 2] = __uint_as_float(r.v[i].z); f[4 * i + 3] = __uint_as_float(r.v[i].w);
  }
}
__device__ __forceinline__ void store16(__nv_bfloat16* p, const float (&f)[16]) {
  float lo[8], hi[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    lo[i] = f[i];
    hi[i] = f[8 + i];
  }
  Vec16<__nv_bfloat16>::store(p, lo);
  Vec16<__nv_bfloat16>::store(p + 8, hi);
}
__device__ __forceinline__ void store16(float* p, const float (&f)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) *reinterpret_cast<float4*>(p + 4 * i) = make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
}

struct RowsArgs {
  uint8_t *k8, *v8, *ks, *vs;
  void *k, *v;
  const int64_t* rows;
  int64_t first_row, stride, capacity;
  int n, heads;
  int32_t* status;
};

constexpr int kRowThreads = 256;

// Bound by memory.  A thread has 16 channels of one head (blockIdx.x, threadIdx.x) and TOKENS tokens in a row
// (blockIdx.y): a whole vector of codes, and the loads of all its tokens under way together.  K for z = 0, V for z = 1.
template <typename T, int D, int TOKENS, bool WRITE>
__global__ void __launch_bounds__(kRowThreads) store_rows_kernel(RowsArgs a) {
  constexpr int kLanes = D / 16;  // neighbouring threads of a head's row
  const int column = blockIdx.x * kRowThreads + threadIdx.x;
  if (column >= a.heads * kLanes) return;  // (whole groups of kLanes threads)
  const int head = column / kLanes, lane = column % kLanes;
  const int first = blockIdx.y * TOKENS;
  T* const x = static_cast<T*>(blockIdx.z ? a.v : a.k) + (int64_t)column * 16;
  uint8_t* const codes = (blockIdx.z ? a.v8 : a.k8) + (int64_t)head * a.capacity * D + lane * 16;
  uint8_t* const scales = (blockIdx.z ? a.vs : a.ks) + (int64_t)head * a.capacity;
  int64_t row[TOKENS];
#pragma unroll
  for (int i = 0; i < TOKENS; ++i) {
    const int token = first + i;
    row[i] = token >= a.n ? -1 : a.rows ? a.rows[token] : a.first_row + token;
    if (row[i] >= a.capacity) row[i] = -1;
    if (row[i] >= 0 && !(H2O_IN_RANGE(row[i], a.capacity, a.status) && H2O_IN_RANGE(head, a.heads, a.status) &&
                         H2O_IN_RANGE(column * 16 + 15, a.stride, a.status)))
      row[i] = -1;
  }
  if constexpr (WRITE) {
    Raw16<T> raw[TOKENS];
#pragma unroll
    for (int i = 0; i < TOKENS; ++i)
      if (first + i < a.n) raw[i].load(x + (first + i) * a.stride);  // (not waiting for the row's number)
    const unsigned mask = ((1u << kLanes) - 1u) << ((threadIdx.x & 31) / kLanes * kLanes);  // this row's threads
#pragma unroll
    for (int i = 0; i < TOKENS; ++i) {
      if (row[i] < 0) continue;  // (the same for all threads of a row)
      float f[16], m = 0.f;
      numbers(raw[i], f);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float b = fabsf(f[e]);
        m = b < INFINITY ? fmaxf(m, b) : m;  // (false for NaN)
      }
#pragma unroll
      for (int o = kLanes / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(mask, m, o));
      const int e2 = kv8_exponent(m);
      const float inv = __uint_as_float((uint32_t)(127 - e2) << 23);
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float* g = &f[4 * e];
        const __nv_fp8x2_storage_t lo = __nv_cvt_float2_to_fp8x2(make_float2(g[0] * inv, g[1] * inv), __NV_SATFINITE, __NV_E4M3);
        const __nv_fp8x2_storage_t hi = __nv_cvt_float2_to_fp8x2(make_float2(g[2] * inv, g[3] * inv), __NV_SATFINITE, __NV_E4M3);
        w[e] = (uint32_t)lo | ((uint32_t)hi << 16);
      }
      *reinterpret_cast<uint4*>(codes + row[i] * D) = make_uint4(w[0], w[1], w[2], w[3]);
      if (lane == 0) scales[row[i]] = (uint8_t)(e2 + 127);
    }
  } else {
    uint4 w[TOKENS];
    uint32_t byte[TOKENS];
#pragma unroll
    for (int i = 0; i < TOKENS; ++i)
      if (row[i] >= 0) {
        w[i] = *reinterpret_cast<const uint4*>(codes + row[i] * D);
        byte[i] = scales[row[i]];
      }
#pragma unroll
    for (int i = 0; i < TOKENS; ++i) {
      if (row[i] < 0) continue;
      const float s = kv8_scale(byte[i]);
      const uint32_t words[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
      float f[16];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t pair = (words[e >> 1] >> (16 * (e & 1))) & 0xffffu;
        const float2 g = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)pair, __NV_E4M3)));
        f[2 * e] = g.x * s;
        f[2 * e + 1] = g.y * s;
      }
      store16(x + (first + i) * a.stride, f);
    }
  }
}

template <typename T, int D, bool WRITE>
cudaError_t launch_tokens(const RowsArgs& a, cudaStream_t stream) {
  const unsigned columns = (unsigned)(((int64_t)a.heads * (D / 16) + kRowThreads - 1) / kRowThreads);
  // Several tokens to a thread where there are blocks enough all the same.  16391 tokens, 32 heads of 128, bfloat16:
  // written to consecutive rows 71.2 us with one, 67.3 with two, 65.6 with four (6.2 TB/s; scattered rows 77); read
  // back 70.1 / 69.4 / 72.5.
  constexpr int kMany = WRITE && sizeof(T) == 2 ? 4 : 2;
  if ((int64_t)columns * 2 * a.n / kMany >= 8 * sm_count())
    store_rows_kernel<T, D, kMany, WRITE><<<dim3(columns, (unsigned)((a.n + kMany - 1) / kMany), 2), kRowThreads, 0, stream>>>(a);
  else
    store_rows_kernel<T, D, 1, WRITE><<<dim3(columns, (unsigned)a.n, 2), kRowThreads, 0, stream>>>(a);
  return cudaGetLastError();
}

template <bool WRITE>
cudaError_t launch_rows(const h2o_store_config_t& c, void* k, void* v, int dtype, int64_t stride, int64_t n,
                        const int64_t* rows, int64_t first_row, cudaStream_t stream) {
  RowsArgs a;
  a.k8 = static_cast<uint8_t*>(c.k);
  a.v8 = static_cast<uint8_t*>(c.v);
  a.ks = c.k_scale;
  a.vs = c.v_scale;
  a.rows = rows;
  a.stride = stride;
  a.capacity = c.rows;
  a.heads = c.n_heads;
  a.status = c.status;
  const int64_t elem = dtype == H2O_F32 ? 4 : 2;
  constexpr int64_t kMost = 65535;  // tokens of a launch (the grid's second dimension)
  for (int64_t at = 0; at < n; at += kMost) {
    a.n = (int)(n - at < kMost ? n - at : kMost);
    a.k = static_cast<char*>(k) + at * stride * elem;
    a.v = static_cast<char*>(v) + at * stride * elem;
    a.rows = rows ? rows + at : nullptr;
    a.first_row = first_row + at;
    const cudaError_t e = dtype == H2O_F32
                              ? (c.head_dim == 128 ? launch_tokens<float, 128, WRITE>(a, stream) : launch_tokens<float, 64, WRITE>(a, stream))
                              : (c.head_dim == 128 ? launch_tokens<__nv_bfloat16, 128, WRITE>(a, stream)
                                                   : launch_tokens<__nv_bfloat16, 64, WRITE>(a, stream));
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace

cudaError_t launch_store_write(const h2o_store_config_t& c, const void* k, const void* v, int dtype, int64_t stride,
                               int64_t n, const int64_t* rows, int64_t first_row, cudaStream_t stream) {
  return launch_rows<true>(c, const_cast<void*>(k), const_cast<void*>(v), dtype, stride, n, rows, first_row, stream);
}
cudaError_t launch_store_read(const h2o_store_config_t& c, void* k, void* v, int dtype, int64_t stride, int64_t n,
                              const int64_t* rows, int64_t first_row, cudaStream_t stream) {
  return launch_rows<false>(c, k, v, dtype, stride, n, rows, first_row, stream);
}

}  // namespace h2o
