// Attention over a K/V store for many query rows (prompts, a prefix shared by many sequences): tcgen05 with the
// accumulators in tensor memory; bfloat16 queries, bfloat16 or 8-bit rows, head_dim 64 or 128.
//
// A block takes up to 256 query rows (query tokens times the query heads of one K/V head) as two groups of 128, A and
// B, which share every tile of 128 keys.  Per group g and key tile j:
//   S_g(j) = Q_g K_j^T     M 128, N 128: with fewer keys per instruction the operands' shared-memory reads bind
//   P_g(j) = exp2(S - m)   written over S_g as 16-bit values (tensor memory holds O and S of both groups: all 512
//                          columns, so S is not double-buffered: while one group computes exponentials the tensor
//                          cores work for the other)
//   O_g   += P_g(j) V_j    P is the tensor-memory operand, V the MN-major shared-memory operand
// Roles: warp 0 TMA, warps 1 and 2 issue the matrix instructions of A and B (A's also clears what lies behind the range
// in its last V tile: 0 * NaN must not reach the sums), warp 3 tensor memory, warps 4..7 and 8..11 the softmax of A
// and B, one thread per row; with 8-bit rows warps 12..15 turn code tiles into f16 tiles.
// The reference maximum follows lazily (O is rescaled when a logit exceeds it by 8, base 2).  The commit behind
// S_g(j) covers P V(j - 1) too, so a softmax thread that sees S_g(j) may rescale O without another wait.
//
// Rounding: P is one bf16 (8-bit rows: one f16).  Its error, 2^-9 relative per key and of either sign, averages over
// the keys to about that of the output's own rounding; a second product for the remainder would cost half as much tensor
// time again.  Row sums are fp32 sums of the unrounded values.
// Part of the exponentials runs on the FMA pipe (ex2_fma2): the special-function unit alone would need as long as
// both products together (16 a clock for 128 x 128 x 2).
#include <cuda.h>
#include <cuda_fp16.h>

#include "sm100_ptx.cuh"
#include "store.cuh"

namespace h2o {

namespace {

using namespace ptx;

constexpr int kM = 128, kN = 128;  // rows of a group, keys of a tile
constexpr int kMaxSlots = 5, kRawSlots = 2;
constexpr float kRescale = 8.f;
__host__ __device__ constexpr int threads(int fmt) { return fmt == H2O_KV8 ? 512 : 384; }
__host__ __device__ constexpr int tile_bytes(int d) { return kN * d * 2; }
__host__ __device__ constexpr int slots(int fmt, int d) { return d == 64 ? 5 : fmt == H2O_KV8 ? 4 : 5; }
__host__ __device__ constexpr int smem_bytes(int fmt, int d) {
  return (2 + slots(fmt, d)) * tile_bytes(d) + (fmt == H2O_KV8 ? kRawSlots * kN * d : 0) + 1024;
}
// registers of a thread: the block starts with regs_start() each; the softmax warps take what the others give back
__host__ __device__ constexpr int regs_softmax(int fmt) { return fmt == H2O_KV8 ? 176 : 216; }
__host__ __device__ constexpr int regs_other(int fmt) { return fmt == H2O_KV8 ? 80 : 72; }

struct Shared {
  uint64_t q_full[2];
  uint64_t kv_full[kMaxSlots], kv_empty[kMaxSlots];
  uint64_t raw_full[kRawSlots], raw_empty[kRawSlots];
  uint64_t s_full[2], p_full[2], o_final[2];
  uint64_t tail;  // the last V tile has been cleared behind the range
  uint32_t tmem_base;
  int abort_flag;
  float row_factor[2 * kM];
  __half scale[2][kN];  // 8-bit rows: the powers of two of the tile being converted
};

__device__ __forceinline__ bool wait_or_abort(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
  for (uint32_t it = 0; it < kSpinLimit; ++it) {
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
// [-0.5, 0.5] (1.8e-7 relative, as good as ex2.approx), exponent added with integer arithmetic.  Below -126: ~1e-38.
__device__ __forceinline__ float2 ex2_fma2(float2 x) {
  x.x = fmaxf(x.x, -126.f);
  x.y = fmaxf(x.y, -126.f);
  const float2 t = __fadd2_rn(x, make_float2(12582912.f, 12582912.f));
  const float2 n = __fadd2_rn(t, make_float2(-12582912.f, -12582912.f));
  const float2 f = __ffma2_rn(n, make_float2(-1.f, -1.f), x);
  float2 p = make_float2(0.0013280353741720319f, 0.0013280353741720319f);
  p = __ffma2_rn(p, f, make_float2(0.009675574488937855f, 0.009675574488937855f));
  p = __ffma2_rn(p, f, make_float2(0.05550701171159744f, 0.05550701171159744f));
  p = __ffma2_rn(p, f, make_float2(0.24022118747234344f, 0.24022118747234344f));
  p = __ffma2_rn(p, f, make_float2(0.6931470036506653f, 0.6931470036506653f));
  p = __ffma2_rn(p, f, make_float2(1.0000001192092896f, 1.0000001192092896f));
  return make_float2(__uint_as_float(__float_as_uint(p.x) + (__float_as_uint(t.x) << 23)),
                     __uint_as_float(__float_as_uint(p.y) + (__float_as_uint(t.y) << 23)));
}

// Barrier of the four converting warps that tells each of them whether all are well.
__device__ __forceinline__ bool together(bool ok) {
  uint32_t all;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "barrier.cta.red.and.aligned.pred q, 2, 128, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(all)
      : "r"(ok ? 1u : 0u)
      : "memory");
  return all != 0;
}

// 16-byte chunk `c` of row `r` of a 16-bit operand tile: halves of 64 channels, each [rows][128 bytes] swizzled.
__device__ __forceinline__ uint32_t operand_addr(uint32_t tile, int rows, int r, int c) {
  return tile + (c >> 3) * (rows * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4);
}
__device__ __forceinline__ void st_shared16(uint32_t addr, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t codes_to_f16(uint32_t pair, __half2 scale) {  // two e4m3 codes times a power of two
  uint32_t r;
  asm("{\n\t.reg .b16 h;\n\tcvt.u16.u32 h, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, h;\n\t}" : "=r"(r) : "r"(pair));
  const __half2 h = __hmul2(*reinterpret_cast<const __half2*>(&r), scale);
  return *reinterpret_cast<const uint32_t*>(&h);
}

template <int FMT, int D>
__global__ void __launch_bounds__(threads(FMT), 1)
attend_tc_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                 const __grid_constant__ AttendView a, int part_index) {
  constexpr bool kF16 = FMT == H2O_KV8;
  constexpr int kTile = tile_bytes(D), kSlots = slots(FMT, D), kRaw = kN * D;
  constexpr uint32_t kColO = 0, kColS = 256;  // O_g at 128 g, S_g / P_g at 256 + 128 g
  extern __shared__ unsigned char dyn_raw[];
  __shared__ Shared sh;
  unsigned char* dyn = dyn_raw + ((1024u - (smem_u32(dyn_raw) & 1023u)) & 1023u);
  unsigned char* q_tiles = dyn;
  unsigned char* ring = dyn + 2 * kTile;
  unsigned char* raw = ring + kSlots * kTile;

  const AttendPart& part = a.part[part_index];
  const BlockWork w = block_work(a, part, blockIdx.x);
  const Problem pr = locate(a, part, w.problem);
  const int rows = pr.nt * a.group, r0 = w.row_tile * (2 * kM);
  if (r0 >= rows) return;
  const int n_rows = min(2 * kM, rows - r0);
  const int key0 = w.split * part.chunk;
  const bool direct = a.part_out == nullptr;
  if (!direct && key0 >= pr.len) return;  // (the join kernel does not read it)
  const int last_seen = seen_rows(part, pr, (r0 + n_rows - 1) / a.group);
  const int key1 = min(last_seen, key0 + part.chunk);
  const int nt = max(0, (key1 - key0 + kN - 1) / kN);
  const int n_groups = n_rows > kM ? 2 : 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int g = 0; g < 2; ++g) {
      mbar_init(&sh.q_full[g], 4);
      mbar_init(&sh.s_full[g], 1);
      mbar_init(&sh.p_full[g], 4);
      mbar_init(&sh.o_final[g], 1);
    }
    for (int i = 0; i < kSlots; ++i) {
      mbar_init(&sh.kv_full[i], kF16 ? 4 : 1);
      mbar_init(&sh.kv_empty[i], n_groups);
    }
    for (int i = 0; i < kRawSlots; ++i) {
      mbar_init(&sh.raw_full[i], 1);
      mbar_init(&sh.raw_empty[i], 4);
    }
    mbar_init(&sh.tail, 1);
    sh.abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == 3) tmem_alloc(&sh.tmem_base, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem_base;
  volatile int* abort_flag = &sh.abort_flag;

  if (warp < 4 || warp >= 12) {
    setmaxnreg_dec<regs_other(FMT)>();
    if (warp == 0) {
      // ---- TMA: K_0, V_0, K_1, V_1, ... (16-bit rows: into the operand ring; 8-bit rows: into the code ring) ----
      if (lane == 0) {
        constexpr int kS = kF16 ? kRawSlots : kSlots;
        constexpr uint32_t bytes = kF16 ? kRaw : kTile;
        uint64_t* full = kF16 ? sh.raw_full : sh.kv_full;
        uint64_t* empty = kF16 ? sh.raw_empty : sh.kv_empty;
        int slot = 0;
        uint32_t phase = 1;
        bool ok = true;
        for (int r = 0; r < 2 * nt; ++r) {
          ok = wait_or_abort(&empty[slot], phase, abort_flag);
          if (!ok) break;
          mbar_expect_tx(&full[slot], bytes);
          tma_load_tile((kF16 ? raw : ring) + slot * bytes, (r & 1) ? &map_v : &map_k, w.head, (int)pr.row0 + key0 + (r >> 1) * kN, &full[slot]);
          if (++slot == kS) {
            slot = 0;
            phase ^= 1;
          }
        }
      }
    } else if (warp < 3 && warp <= n_groups) {
      // ---- matrix instructions of group g (the whole warp walks, one elected lane issues) ----
      constexpr uint32_t fmt = kF16 ? kFmtF16 : kFmtBF16;
      constexpr uint32_t idesc_s = instr_desc_f16(kM, kN, fmt, fmt, false, false);
      constexpr uint32_t idesc_o = instr_desc_f16(kM, D, fmt, fmt, false, true);
      const int g = warp - 1;
      const uint32_t d_s = tmem + kColS + 128u * g, d_o = tmem + kColO + 128u * g;
      const uint64_t dq = smem_desc_sw128(smem_u32(q_tiles + g * kTile), 16, 1024);
      bool ok = nt == 0 || wait_or_abort(&sh.q_full[g], 0, abort_flag);
      int slot = 0;
      uint32_t phase = 0;
      auto next = [&] {
        if (++slot == kSlots) {
          slot = 0;
          phase ^= 1;
        }
      };
      for (int j = -1; j < nt; ++j) {
        if (j >= 0) {  // O += P(j) V_j
          ok = ok && wait_or_abort(&sh.kv_full[slot], phase, abort_flag);
          if (!kF16 && j == nt - 1) {
            // the range's last V tile: zeros behind it, by group A's warp
            if (g == 0) {
              const int there = key1 - key0 - j * kN;
              const uint32_t tile = smem_u32(ring + slot * kTile);
              ok = __all_sync(0xffffffffu, ok) != 0;
              if (ok) {
                for (int i = lane; i < (kN - there) * (D / 8); i += 32)
                  st_shared16(operand_addr(tile, kN, there + i / (D / 8), i % (D / 8)), make_uint4(0, 0, 0, 0));
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.tail);
              }
            }
            ok = ok && wait_or_abort(&sh.tail, 0, abort_flag);
          }
          ok = ok && wait_or_abort(&sh.p_full[g], (uint32_t)j & 1u, abort_flag);
          ok = __all_sync(0xffffffffu, ok) != 0;
          if (!ok) break;
          tc_fence_after();
          const uint64_t dv = smem_desc_sw128(smem_u32(ring + slot * kTile), kTile / 2, 1024);
          if (elect_one()) {
            if (j == 0) mma_ts_lohi<false>(d_o, d_s, desc_lo(dv), desc_hi(dv), idesc_o);
            else mma_ts_lohi<true>(d_o, d_s, desc_lo(dv), desc_hi(dv), idesc_o);
#pragma unroll
            for (int ks = 1; ks < kN / 16; ++ks)
              mma_ts_lohi<true>(d_o, d_s + 8u * ks, desc_lo(dv) + ((2048u * ks) >> 4), desc_hi(dv), idesc_o);
            mma_commit(&sh.kv_empty[slot]);
            if (j == nt - 1) mma_commit(&sh.o_final[g]);
          }
          __syncwarp();
          next();
        }
        if (j + 1 < nt) {  // S(j + 1) = Q K_{j+1}^T, over P(j): one thread's instructions run in order
          ok = ok && wait_or_abort(&sh.kv_full[slot], phase, abort_flag);
          ok = __all_sync(0xffffffffu, ok) != 0;
          if (!ok) break;
          tc_fence_after();
          const uint64_t dk = smem_desc_sw128(smem_u32(ring + slot * kTile), 16, 1024);
          if (elect_one()) {
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
              const uint32_t off = ((uint32_t)(ks >> 2) * (kN * 128) + (uint32_t)(ks & 3) * 32u) >> 4;
              if (ks == 0) mma_ss_lohi<false>(d_s, desc_lo(dq), desc_hi(dq), desc_lo(dk), desc_hi(dk), idesc_s);
              else mma_ss_lohi<true>(d_s, desc_lo(dq) + off, desc_hi(dq), desc_lo(dk) + off, desc_hi(dk), idesc_s);
            }
            mma_commit(&sh.s_full[g]);
            mma_commit(&sh.kv_empty[slot]);
          }
          __syncwarp();
          next();
        }
      }
    } else if (kF16 && warp >= 12) {
      // ---- code tiles to f16 tiles: thread t takes chunk t % (D / 16) of every (2048 / D)-th row ----
      constexpr int kChunks = D / 16, kStride = 128 / kChunks;
      const int t = threadIdx.x - 384, c = t % kChunks;
      const int64_t base = (int64_t)w.head * a.rows + pr.row0;
      auto fetch = [&](int r) {
        const int key = key0 + (r >> 1) * kN + t;
        return key < key1 ? (uint32_t)((r & 1) ? a.v_scale : a.k_scale)[base + key] : 127u;
      };
      uint32_t byte = nt > 0 ? fetch(0) : 0;
      int slot = 0;
      uint32_t phase = 1;
      for (int r = 0; r < 2 * nt; ++r) {
        const int rs = r % kRawSlots;
        sh.scale[r & 1][t] = __float2half_rn(kv8_scale(byte));
        if (r + 1 < 2 * nt) byte = fetch(r + 1);
        bool ok = wait_or_abort(&sh.raw_full[rs], (uint32_t)(r / kRawSlots) & 1u, abort_flag);
        ok = ok && wait_or_abort(&sh.kv_empty[slot], phase, abort_flag);
        ok = together(ok);  // (also publishes the scales; one answer for the four warps, so that none waits for another)
        if (ok) {
          const uint32_t src = smem_u32(raw + rs * kRaw), dst = smem_u32(ring + slot * kTile);
          const int there = min(kN, key1 - key0 - (r >> 1) * kN);
#pragma unroll 4
          for (int i = 0; i < kN / kStride; ++i) {
            const int row = t / kChunks + i * kStride;
            const uint32_t at = D == 128 ? src + row * 128 + ((c ^ (row & 7)) << 4) : src + row * 64 + ((c ^ ((row >> 1) & 3)) << 4);
            uint32_t x[4];
            asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(at) : "memory");
            const __half2 f = __half2half2(sh.scale[r & 1][row]);
            uint4 y[2];
            y[0] = make_uint4(codes_to_f16(x[0] & 0xffffu, f), codes_to_f16(x[0] >> 16, f), codes_to_f16(x[1] & 0xffffu, f), codes_to_f16(x[1] >> 16, f));
            y[1] = make_uint4(codes_to_f16(x[2] & 0xffffu, f), codes_to_f16(x[2] >> 16, f), codes_to_f16(x[3] & 0xffffu, f), codes_to_f16(x[3] >> 16, f));
            if (row >= there) y[0] = y[1] = make_uint4(0, 0, 0, 0);  // behind the range
            const int first = (c >> 2) & 1;  // (lanes of the two halves start with different chunks: no bank conflict)
            st_shared16(operand_addr(dst, kN, row, 2 * c + first), first ? y[1] : y[0]);
            st_shared16(operand_addr(dst, kN, row, 2 * c + 1 - first), first ? y[0] : y[1]);
          }
          fence_proxy_async();
        }
        __syncwarp();
        if (!ok) break;
        if (lane == 0) {
          mbar_arrive(&sh.raw_empty[rs]);
          mbar_arrive(&sh.kv_full[slot]);
        }
        if (++slot == kSlots) {
          slot = 0;
          phase ^= 1;
        }
      }
    }
  } else {
    setmaxnreg_inc<regs_softmax(FMT)>();
    const int g = (warp - 4) >> 2, quarter = warp & 3;
    if (g < n_groups) {
      // ---- the group's query rows into shared memory: D / 8 lanes a row ----
      {
        constexpr int kLanes = D / 8, kPer = 32 / kLanes;
        const int c = lane % kLanes;
        const uint32_t tile = smem_u32(q_tiles + g * kTile);
#pragma unroll 4
        for (int i = 0; i < 32 / kPer; ++i) {
          const int rt = quarter * 32 + i * kPer + lane / kLanes, r = g * kM + rt;
          uint4 x = make_uint4(0, 0, 0, 0);
          if (r < n_rows) {
            const int tok = (r0 + r) / a.group, hq = w.head * a.group + (r0 + r) - tok * a.group;
            x = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.q) + (pr.t0 + tok) * a.q_stride + (int64_t)hq * D + c * 8);
          }
          if constexpr (kF16) {
            float f[8];
            Vec16<__nv_bfloat16>::unpack(x, f);
            float big = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) big = fabsf(f[e]) < INFINITY ? fmaxf(big, fabsf(f[e])) : big;
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
            const int e2 = max(-100, min(126, (int)(__float_as_uint(big) >> 23) - 127));
            const float down = __uint_as_float((uint32_t)(127 - e2) << 23);
            x = make_uint4(pack_half2(f[0] * down, f[1] * down), pack_half2(f[2] * down, f[3] * down),
                           pack_half2(f[4] * down, f[5] * down), pack_half2(f[6] * down, f[7] * down));
            if (c == 0) sh.row_factor[r] = a.scale2 * __uint_as_float((uint32_t)(127 + e2) << 23);
          }
          st_shared16(operand_addr(tile, kM, rt, c), x);
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.q_full[g]);
      }
      // ---- softmax, one thread per row ----
      const int rt = quarter * 32 + lane, r = g * kM + rt;
      const int tok = (r0 + r) / a.group;
      const int seen = min(key1, r < n_rows ? seen_rows(part, pr, tok) : key1);
      const int all_seen = part.causal ? min(key1, seen_rows(part, pr, (r0 + g * kM) / a.group)) : key1;
      const float factor = kF16 ? sh.row_factor[r] : a.scale2;
      const uint32_t lane_addr = (uint32_t)(quarter * 32) << 16;
      const uint32_t t_s = tmem + kColS + 128u * g + lane_addr, t_o = tmem + kColO + 128u * g + lane_addr;
      float m = -INFINITY;
      float2 l2 = make_float2(0.f, 0.f);
      bool ok = true;
      for (int j = 0; j < nt; ++j) {
        ok = __all_sync(0xffffffffu, wait_or_abort(&sh.s_full[g], (uint32_t)j & 1u, abort_flag));
        if (!ok) break;
        tc_fence_after();
        uint32_t s[4][32];
#pragma unroll
        for (int i = 0; i < 4; ++i) tmem_ld32(t_s + 32u * i, s[i]);
        tmem_wait_ld();
        const int key = key0 + j * kN;
        if (key + kN > all_seen) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (key + 32 * i + e >= seen) s[i][e] = 0xff800000u;
        }
        float top4[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          top4[i] = __uint_as_float(s[i][0]);
#pragma unroll
          for (int e = 1; e + 1 < 32; e += 2) top4[i] = max3(top4[i], __uint_as_float(s[i][e]), __uint_as_float(s[i][e + 1]));
          top4[i] = fmaxf(top4[i], __uint_as_float(s[i][31]));
        }
        // (the factor is positive: the maximum commutes with it)
        const float top = fmaxf(max3(top4[0], top4[1], top4[2]), top4[3]) * factor;
        const bool grows = top > m + kRescale;
        if (__any_sync(0xffffffffu, grows)) {
          const float mn = grows ? top : m;
          const float alpha = mn == -INFINITY ? 1.f : ex2(m - mn);
          l2 = __fmul2_rn(l2, make_float2(alpha, alpha));
          m = mn;
          if (j > 0) {
#pragma unroll
            for (int cc = 0; cc < D / 32; ++cc) {
              uint32_t o[32];
              tmem_ld32(t_o + 32u * cc, o);
              tmem_wait_ld();
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
              tmem_st32(t_o + 32u * cc, o);
            }
          }
        }
        const float neg = m == -INFINITY ? 0.f : -m;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint32_t pw[32];  // 64 keys, two to a column
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            const uint32_t(&src)[32] = s[2 * i + (e >> 4)];
            const int at = 2 * (e & 15);
            const float2 x = __ffma2_rn(make_float2(__uint_as_float(src[at]), __uint_as_float(src[at + 1])),
                                        make_float2(factor, factor), make_float2(neg, neg));
            const float2 p = (e & 3) == 3 ? ex2_fma2(x) : make_float2(ex2(x.x), ex2(x.y));
            l2 = __fadd2_rn(l2, p);
            pw[e] = kF16 ? pack_half2(p.x, p.y) : Vec16<__nv_bfloat16>::pack2(p.x, p.y);
          }
          tmem_st32(t_s + 32u * i, pw);
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.p_full[g]);
      }
      // ---- result ----
      if (ok && nt > 0) ok = __all_sync(0xffffffffu, wait_or_abort(&sh.o_final[g], 0, abort_flag));
      if (ok) {
        tc_fence_after();
        const float sum = l2.x + l2.y;
        const bool none = sum == 0.f || m == -INFINITY;
        const float inv = none ? 0.f : 1.f / sum;
        const float lse2 = none ? -INFINITY : m + log2f(sum);
        const int64_t token = pr.t0 + tok;
        const int hq = w.head * a.group + (r0 + r) - tok * a.group;
        const int64_t at = ((int64_t)(part.slot0 + w.split) * a.q_rows + token) * a.heads * a.group + hq;
        __nv_bfloat16* to = static_cast<__nv_bfloat16*>(a.out) + token * a.out_stride + (int64_t)hq * D;
        const bool wide = ((reinterpret_cast<uintptr_t>(a.out) | (uintptr_t)(a.out_stride * 2)) & 31u) == 0;
#pragma unroll
        for (int cc = 0; cc < D / 32; ++cc) {
          uint32_t o[32];
          if (nt > 0) {
            tmem_ld32(t_o + 32u * cc, o);
            tmem_wait_ld();
          }
          if (r >= n_rows) continue;
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = none ? 0u : __float_as_uint(__uint_as_float(o[e]) * inv);
          if (direct) {
            uint32_t x[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = Vec16<__nv_bfloat16>::pack2(__uint_as_float(o[2 * e]), __uint_as_float(o[2 * e + 1]));
            if (wide) {
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                uint32_t v[8];
#pragma unroll
                for (int b = 0; b < 8; ++b) v[b] = x[8 * e + b];
                st_global_256(to + cc * 32 + e * 16, v);
              }
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e)
                *reinterpret_cast<uint4*>(to + cc * 32 + e * 8) = make_uint4(x[4 * e], x[4 * e + 1], x[4 * e + 2], x[4 * e + 3]);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              uint32_t v[8];
#pragma unroll
              for (int b = 0; b < 8; ++b) v[b] = o[8 * e + b];
              st_global_256(a.part_out + at * D + cc * 32 + e * 8, v);
            }
          }
        }
        if (r < n_rows) {
          if (!direct) a.part_lse[at] = lse2;
          else if (a.lse) a.lse[token * a.heads * a.group + hq] = lse2 * 0.6931471805599453f;
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && sh.abort_flag && a.status) atomicCAS(a.status, 0, H2O_ERR_TIMEOUT);
  if (warp == 3) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <int FMT, int D>
cudaError_t launch(const AttendView& a, int part, const CUtensorMap& k, const CUtensorMap& v, cudaStream_t stream) {
  constexpr int smem = smem_bytes(FMT, D);
  static unsigned long long flags = 0;
  const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(attend_tc_kernel<FMT, D>), smem, &flags);
  if (e != cudaSuccess) return e;
  attend_tc_kernel<FMT, D><<<(unsigned)part_blocks(a, a.part[part]), threads(FMT), smem, stream>>>(k, v, a, part);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attend_tc(const AttendView& a, int part, int format, const void* map_k, const void* map_v, cudaStream_t st) {
  const CUtensorMap& k = *static_cast<const CUtensorMap*>(map_k);
  const CUtensorMap& v = *static_cast<const CUtensorMap*>(map_v);
  if (format == H2O_KV8) return a.dim == 128 ? launch<H2O_KV8, 128>(a, part, k, v, st) : launch<H2O_KV8, 64>(a, part, k, v, st);
  return a.dim == 128 ? launch<H2O_BF16, 128>(a, part, k, v, st) : launch<H2O_BF16, 64>(a, part, k, v, st);
}

}  // namespace h2o
