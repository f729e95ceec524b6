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

constexpr float kE4m3Max = 448.f;

// Exponent e of a row whose largest finite magnitude is `a`: with a = m * 2^k, 1 <= m < 2, 448 = 1.75 * 2^8.
__device__ __forceinline__ int kv8_exponent(float a) {
  const uint32_t b = __float_as_uint(a);
  const int k = (int)(b >> 23) - 127;  // (zero and subnormals: far below the range, cut to -15)
  const int e = k - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
  return max(-15, min(7, e));
}

template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&f)[8]);
template <>
__device__ __forceinline__ void load8<__nv_bfloat16>(const __nv_bfloat16* p, float (&f)[8]) {
  Vec16<__nv_bfloat16>::load(p, f);
}
template <>
__device__ __forceinline__ void load8<float>(const float* p, float (&f)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
  f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&f)[8]);
template <>
__device__ __forceinline__ void store8<__nv_bfloat16>(__nv_bfloat16* p, const float (&f)[8]) {
  Vec16<__nv_bfloat16>::store(p, f);
}
template <>
__device__ __forceinline__ void store8<float>(float* p, const float (&f)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
}

struct RowsArgs {
  uint8_t *k8, *v8, *ks, *vs;
  void *k, *v;
  const int64_t* rows;
  int64_t first_row, n, stride, capacity;
  int heads;
};

// D / 8 neighbouring threads take one row of one head (8 channels each): K for z = 0, V for z = 1.
template <typename T, int D, bool WRITE>
__global__ void __launch_bounds__(256) store_rows_kernel(RowsArgs a) {
  constexpr int kLanes = D / 8;
  const int64_t item = ((int64_t)blockIdx.x * 256 + threadIdx.x) / kLanes;  // token * heads + head
  const int lane = threadIdx.x % kLanes;
  if (item >= a.n * a.heads) return;  // (whole groups of kLanes threads)
  const int64_t token = item / a.heads;
  const int head = (int)(item - token * a.heads);
  const int64_t row = a.rows ? a.rows[token] : a.first_row + token;
  if (row < 0 || row >= a.capacity) return;
  T* x = static_cast<T*>(blockIdx.z ? a.v : a.k) + token * a.stride + (int64_t)head * D + lane * 8;
  uint8_t* codes = (blockIdx.z ? a.v8 : a.k8) + ((int64_t)head * a.capacity + row) * D + lane * 8;
  uint8_t* scale = (blockIdx.z ? a.vs : a.ks) + (int64_t)head * a.capacity + row;
  float f[8];
  if constexpr (WRITE) {
    load8<T>(x, f);
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float b = fabsf(f[i]);
      m = b < INFINITY ? fmaxf(m, b) : m;  // (false for NaN)
    }
    const unsigned mask = (kLanes == 16 ? 0xffffu : 0xffu) << ((threadIdx.x & 31) / kLanes * kLanes);  // this row's threads
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(mask, m, o));
    const int e = kv8_exponent(m);
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const __nv_fp8x2_storage_t lo = __nv_cvt_float2_to_fp8x2(make_float2(f[4 * i] * inv, f[4 * i + 1] * inv), __NV_SATFINITE, __NV_E4M3);
      const __nv_fp8x2_storage_t hi = __nv_cvt_float2_to_fp8x2(make_float2(f[4 * i + 2] * inv, f[4 * i + 3] * inv), __NV_SATFINITE, __NV_E4M3);
      w[i] = (uint32_t)lo | ((uint32_t)hi << 16);
    }
    *reinterpret_cast<uint2*>(codes) = make_uint2(w[0], w[1]);
    if (lane == 0) *scale = (uint8_t)(e + 127);
  } else {
    const uint2 w = *reinterpret_cast<const uint2*>(codes);
    const float s = kv8_scale(*scale);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t pair = ((i < 2 ? w.x : w.y) >> (16 * (i & 1))) & 0xffffu;
      const __half2 h = __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)pair, __NV_E4M3));
      const float2 g = __half22float2(h);
      f[2 * i] = g.x * s;
      f[2 * i + 1] = g.y * s;
    }
    store8<T>(x, f);
  }
}

template <bool WRITE>
cudaError_t launch_rows(const h2o_store_config_t& c, void* k, void* v, int dtype, int64_t stride, int64_t n,
                        const int64_t* rows, int64_t first_row, cudaStream_t stream) {
  RowsArgs a;
  a.k8 = static_cast<uint8_t*>(c.k);
  a.v8 = static_cast<uint8_t*>(c.v);
  a.ks = c.k_scale;
  a.vs = c.v_scale;
  a.k = k;
  a.v = v;
  a.rows = rows;
  a.first_row = first_row;
  a.n = n;
  a.stride = stride;
  a.capacity = c.rows;
  a.heads = c.n_heads;
  const int64_t threads = n * c.n_heads * (c.head_dim / 8);
  const dim3 grid((unsigned)((threads + 255) / 256), 1, 2);
  if (dtype == H2O_F32) {
    if (c.head_dim == 128) store_rows_kernel<float, 128, WRITE><<<grid, 256, 0, stream>>>(a);
    else store_rows_kernel<float, 64, WRITE><<<grid, 256, 0, stream>>>(a);
  } else {
    if (c.head_dim == 128) store_rows_kernel<__nv_bfloat16, 128, WRITE><<<grid, 256, 0, stream>>>(a);
    else store_rows_kernel<__nv_bfloat16, 64, WRITE><<<grid, 256, 0, stream>>>(a);
  }
  return cudaGetLastError();
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
