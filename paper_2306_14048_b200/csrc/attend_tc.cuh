// Device pieces that the tcgen05 attention kernels share: bounded waits, exponentials, tensor-memory loads and stores, operand
// addresses.
#pragma once
#include <cuda.h>

#include "sm100_ptx.cuh"

namespace h2o {
namespace tc {

using namespace ptx;

// Up to `polls` polls, or until another wait of the block has given up.
__device__ __forceinline__ bool wait_or_abort(uint64_t* bar, uint32_t parity, volatile int* abort_flag, uint32_t polls) {
  for (uint32_t it = 0; it < polls; ++it) {
    if (mbar_try_wait(bar, parity)) return true;
    if ((it & 1023u) == 1023u && *abort_flag) return false;
  }
  *abort_flag = 1;
  return false;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// exp2 of two values on the FMA pipe: nearest integer by the 1.5 * 2^23 trick, degree-5 polynomial of 2^f on
// [-0.5, 0.5] (1.8e-7 relative, as good as ex2.approx), times 2^n put together with integer arithmetic.  Below -126.5,
// -infinity (a key that is not seen) included: 0, as the exponent field of 2^-127 is; NaN stays NaN; above kPolyMax the
// result means nothing.
constexpr float kPolyMax = 100.f;
__device__ __forceinline__ float max_or_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 ex2_fma2(float2 x) {
  x.x = max_or_nan(x.x, -127.f);
  x.y = max_or_nan(x.y, -127.f);
  const float2 t = __fadd2_rn(x, make_float2(12582912.f, 12582912.f));
  const float2 n = __fadd2_rn(t, make_float2(-12582912.f, -12582912.f));
  const float2 f = __ffma2_rn(n, make_float2(-1.f, -1.f), x);
  float2 p = make_float2(0.0013280353741720319f, 0.0013280353741720319f);
  p = __ffma2_rn(p, f, make_float2(0.009675574488937855f, 0.009675574488937855f));
  p = __ffma2_rn(p, f, make_float2(0.05550701171159744f, 0.05550701171159744f));
  p = __ffma2_rn(p, f, make_float2(0.24022118747234344f, 0.24022118747234344f));
  p = __ffma2_rn(p, f, make_float2(0.6931470036506653f, 0.6931470036506653f));
  p = __ffma2_rn(p, f, make_float2(1.0000001192092896f, 1.0000001192092896f));
  return __fmul2_rn(p, make_float2(__uint_as_float((__float_as_uint(t.x) << 23) + 0x3f800000u),
                                   __uint_as_float((__float_as_uint(t.y) << 23) + 0x3f800000u)));
}

// 32-byte global load: a whole sector, where neighbouring threads read rows far apart (the address is 32-byte aligned)
__device__ __forceinline__ void ld_global_256(const float* p, float4& a, float4& b) {
  asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=f"(a.x), "=f"(a.y), "=f"(a.z), "=f"(a.w), "=f"(b.x), "=f"(b.y), "=f"(b.z), "=f"(b.w)
               : "l"(p)
               : "memory");
}
// N consecutive columns of the warp's 32 lanes from / to registers
__device__ __forceinline__ void tmem_st8(uint32_t addr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(addr), "r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
template <int N>
__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t (&r)[N]) {
#pragma unroll
  for (int i = 0; i + 32 <= N; i += 32) tmem_ld32(addr + i, *reinterpret_cast<uint32_t(*)[32]>(&r[i]));
  if constexpr (N % 32 != 0) tmem_ld16(addr + N / 32 * 32, *reinterpret_cast<uint32_t(*)[16]>(&r[N / 32 * 32]));
}
// Waits for loads under way into r; no use of r moves ahead of it.
template <int N>
__device__ __forceinline__ void tmem_wait_ld_of(uint32_t (&r)[N]) {
  tmem_wait_ld();
#pragma unroll
  for (int i = 0; i < N; i += 8)
    asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7]));
}
template <int N>
__device__ __forceinline__ void tmem_store(uint32_t addr, const uint32_t (&r)[N]) {
  static_assert(N % 32 == 0 || N % 32 == 8 || N % 32 == 16, "");
  if constexpr (N % 32 == 8) tmem_st8(addr + N / 32 * 32, &r[N / 32 * 32]);
#pragma unroll
  for (int i = 0; i + 32 <= N; i += 32) tmem_st32(addr + i, *reinterpret_cast<const uint32_t(*)[32]>(&r[i]));
  if constexpr (N % 32 == 16) tmem_st16(addr + N / 32 * 32, *reinterpret_cast<const uint32_t(*)[16]>(&r[N / 32 * 32]));
}

// 16-byte chunk `c` of row `r` of a 16-bit operand tile: halves of 64 channels, each [rows][128 bytes] swizzled.
__device__ __forceinline__ uint32_t operand_addr(uint32_t tile, int rows, int r, int c) {
  return tile + (c >> 3) * (rows * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4);
}
__device__ __forceinline__ void st_shared16(uint32_t addr, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

}  // namespace tc
}  // namespace h2o
