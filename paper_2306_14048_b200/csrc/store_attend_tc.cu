// Attention over a K/V store for many query rows (prompts, a prefix shared by many sequences): tcgen05 with the
// accumulators in tensor memory; bfloat16 queries, bfloat16 or 8-bit rows, head_dim 64 or 128.
//
// A block takes up to 256 query rows (query tokens times the query heads of one K/V head) as two groups of 128, A and
// B, which share every key tile (80 keys for head_dim 128, 96 or 64 for 64); up to 128 rows are given to both groups, which
// then take the tiles in turn and join their results at the end.  Per group g and key tile j:
//   S_g(j) = Q_g K_j^T     into tensor memory, from there into the softmax threads' registers, which frees S_g at once:
//                          S_g(j + 1) runs while the exponentials of tile j are computed
//   P_g(j) = exp2(S - m)   16-bit, into tensor memory of its own
//   O_g   += P_g(j) V_j    P is the tensor-memory operand, V the MN-major shared-memory operand
// The tile size is what tensor memory holds of O (2 x 128 columns), S (2 x 80) and P (2 x 40).  With S and P in one place
// and tiles of 128 keys the chain S - exponentials - P V of a group is serial: 3700 cycles per tile of both groups for
// 2048 of tensor work.  4 x 2048 queries against 4096 keys, 32 heads: 593 us that way, 505 us this way when it was
// first built, 469 us now (1170 TFLOP/s) before the power limit lowers the clock and 530 to 550 us (1000 to 1040) after.
// Tiles of 64 keys with S prefetched into registers and P in two buffers took 650 us, two threads to a row 725 us.
// Roles: warp 0 TMA; warps 1 and 2 issue S of A and B (they also clear what lies behind the range in its last V tile:
// 0 * NaN must not reach the sums); warp 3 issues P V of both and owns tensor memory; warps 4..7 and 8..11 are the softmax
// of A and B, one thread per row; with 8-bit rows warps 12..15 and 16..19 turn code tiles of K and of V into f16 tiles.
// A wait on a barrier costs 300 to 400 cycles here even when it is complete (it queues behind the exponentials), so the
// issuers have few: K and V of a tile arrive on one barrier, and P V waits for P alone, which comes after S and so after
// the tile.  Their loops run on values the compiler knows to be uniform (constant tensor-memory addresses, counts from a
// shuffle): 575 -> 550 us.
// The reference m of a row is the maximum of its first tile (8-bit rows: 7 less).  Later tiles compute their exponentials
// against it without looking for a maximum: only when a tile's sum comes out large (kLargeSum) the tile is done again with
// the new maximum and O is rescaled.  A value far above the reference costs no precision in floating point, only range.
//
// Rounding: P is one bf16 (8-bit rows: one f16).  Its error, up to 2^-8 relative per key and of either sign, averages over
// the keys to about that of the output's own rounding, which is up to 2^-8 as well; a second product for the remainder would
// cost half as much tensor time again.  Row sums are fp32 sums of the unrounded values.
#include <cuda.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "attend_tc.cuh"
#include "store.cuh"

namespace h2o {

namespace {

using namespace ptx;
using namespace tc;

constexpr int kM = 128;  // rows of a group
// G: groups of a block, 2, or 1 (bfloat16 rows only: half the block, two of them on an SM).
// (8-bit rows of 64 channels: what fits the softmax threads' 144 registers; one group: what fits half an SM's shared memory)
__host__ __device__ constexpr int tile_keys(int fmt, int d, int g) { return g == 1 ? 64 : d == 128 ? 80 : fmt == H2O_KV8 ? 64 : 96; }
__host__ __device__ constexpr int threads(int fmt, int g) { return fmt == H2O_KV8 ? 640 : 128 + 128 * g; }
__host__ __device__ constexpr int tile_bytes(int fmt, int d, int g) { return tile_keys(fmt, d, g) * d * 2; }
// Ring of stages, K and V of a tile in each.  Two groups that take tiles in turn use an even number where TMA fills the
// stages: a warp that waits for a tile then has seen the stage's tile before, so a parity cannot be mistaken for an older
// one.  (Converted tiles complete in order, so a warp that has seen its last tile may count on all before it.)
__host__ __device__ constexpr int stages(int fmt, int d, int g) { return g == 1 ? (d == 64 ? 4 : 2) : d == 64 ? 6 : fmt == H2O_KV8 ? 3 : 4; }
__host__ __device__ constexpr int turn_stages(int fmt, int d, int g) { return fmt == H2O_KV8 ? stages(fmt, d, g) : stages(fmt, d, g) & ~1; }
constexpr int kMaxStages = 6, kRawStages = 2;  // (a stage of the code ring also holds K and V)
__host__ __device__ constexpr int smem_bytes(int fmt, int d, int g) {
  return g * kM * d * 2 + 2 * stages(fmt, d, g) * tile_bytes(fmt, d, g) + (fmt == H2O_KV8 ? 2 * kRawStages * tile_keys(fmt, d, g) * d : 0) + 1024;
}
// Registers of a thread: the softmax warps take what the others give back.  8-bit: 640 threads start with 96 each =
// 256 x 144 + 384 x 64; bfloat16: 384 start with 168 = 256 x 216 + 128 x 72; one group: 256 with 128 = 128 x 176 + 128 x 80.
__host__ __device__ constexpr int regs_softmax(int fmt, int g) { return fmt == H2O_KV8 ? 144 : g == 1 ? 176 : 216; }
__host__ __device__ constexpr int regs_other(int fmt, int g) { return fmt == H2O_KV8 ? 64 : g == 1 ? 80 : 72; }
// Every kPolyEvery-th pair of exponentials runs on the FMA pipe.  4 x 2048 queries against 4096 keys, 32 heads: none 482,
// one in sixteen 484, one in eight 469, one in four 490 us (before the power limit lowers the clock).
constexpr int kPolyEvery = 8;

struct Shared {
  uint64_t q_full[2];
  uint64_t kv_full[kMaxStages], kv_empty[kMaxStages];
  uint64_t raw_full[kRawStages], raw_empty[kRawStages];
  uint64_t s_full[2], s_read[2];   // S is complete / in the softmax threads' registers
  uint64_t p_full[2], p_empty[2];  // P is complete / used, and O includes it
  uint64_t o_final[2];
  uint64_t tail;  // the last V tile has been cleared behind the range
  uint64_t ended;  // of a block that gives up: the products of warps 1 to 3 have ended
  uint32_t tmem_base;
  int abort_flag;
  int loads;  // tiles that TMA has been asked for
  float row_factor[2 * kM];  // 8-bit rows: softmax scale times the query row's power of two
  __half scale[2][2][96];    // 8-bit rows: the powers of two of K and V of the tile being converted
};

constexpr float kRescale = 8.f;
// A tile whose sum against the old reference exceeds this is done again against its own maximum: inside f16's range (largest
// 65504) for the 8-bit rows; for bfloat16 rows so that O, which is divided by its sum at the end, holds values up to 2^100.
template <int FMT>
constexpr float kLargeSumOf = FMT == H2O_KV8 ? 32768.f : 1048576.f;
// How far (base 2) the reference lies below the maximum it was taken from.  In f16 whatever is below 2^-25 becomes 0: with 2^7
// for the largest probability that is 2^-32 of it, so 2^20 such keys that go missing weigh 2^-12.  A first tile's sum
// (80 x 2^7) and what is done again (2^7 x 2^kRescale) stay below the limit.
template <int FMT>
constexpr float kHeadOf = FMT == H2O_KV8 ? 7.f : 0.f;

// Barrier of the eight softmax warps.
__device__ __forceinline__ void softmax_sync() { asm volatile("barrier.cta.sync 3, 256;" ::: "memory"); }
// Barrier of the four warps that convert K (kv = 0) or V (1), that tells each of them whether all are well.
__device__ __forceinline__ bool together(bool ok, int kv) {
  uint32_t all;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "barrier.cta.red.and.pred q, %2, 128, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(all)
      : "r"(ok ? 1u : 0u), "r"(1 + kv)
      : "memory");
  return all != 0;
}

__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// four e4m3 codes times a power of two
__device__ __forceinline__ void codes_to_f16(uint32_t word, __half2 scale, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(word));
  const __half2 x = __hmul2(*reinterpret_cast<const __half2*>(&lo), scale), y = __hmul2(*reinterpret_cast<const __half2*>(&hi), scale);
  lo = *reinterpret_cast<const uint32_t*>(&x);
  hi = *reinterpret_cast<const uint32_t*>(&y);
}

// FINISH: part 1 of a shared prefix, which joins what part 0 left (an instance of its own: the rest is 5 % faster without).
template <int FMT, int D, int G, bool FINISH>
__global__ void __launch_bounds__(threads(FMT, G), 3 - G)
attend_tc_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                 const __grid_constant__ AttendView a, int part_index) {
  constexpr bool kF16 = FMT == H2O_KV8;
  constexpr int kN = tile_keys(FMT, D, G), kTile = tile_bytes(FMT, D, G), kQTile = kM * D * 2, kStages = stages(FMT, D, G), kRaw = kN * D;
  constexpr float kLargeSum = kLargeSumOf<FMT>, kHead = kHeadOf<FMT>;
  // tensor memory: O, S (starts on multiples of 32 columns) and P (of 8) of the groups
  constexpr uint32_t kColO = 0, kStepO = D, kColS = G * D, kStepS = 96, kColP = kColS + kStepS * (G - 1) + kN, kStepP = kN / 2;
  constexpr uint32_t kCols = G == 2 ? 512 : 256;
  static_assert(kColP + G * kStepP <= kCols, "tensor memory");
  static_assert(smem_bytes(FMT, D, G) + sizeof(Shared) + (G == 1 ? 1024 : 0) <= (G == 1 ? 114 : 227) * 1024, "shared memory of a block");
  static_assert(G == 1 || kM * (D + 4) * 4 <= 2 * turn_stages(FMT, D, G) * kTile, "B's output fits the ring");
  extern __shared__ unsigned char dyn_raw[];
  __shared__ Shared sh;
  unsigned char* dyn = dyn_raw + ((1024u - (smem_u32(dyn_raw) & 1023u)) & 1023u);
  unsigned char* q_tiles = dyn;
  unsigned char* ring = dyn + G * kQTile;
  unsigned char* raw = ring + 2 * kStages * kTile;

  let_next_start();
  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  // what does not depend on the block's work, while the others look that up
  if (threadIdx.x == 0) {
    prefetch_tensormap(&map_k);
    prefetch_tensormap(&map_v);
    for (int g = 0; g < 2; ++g) {
      mbar_init(&sh.q_full[g], 4);
      mbar_init(&sh.s_full[g], 1);
      mbar_init(&sh.s_read[g], 4);
      mbar_init(&sh.p_full[g], 4);
      mbar_init(&sh.p_empty[g], 1);
      mbar_init(&sh.o_final[g], 1);
    }
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&sh.kv_full[i], kF16 ? 8 : 1);  // (eight converting warps)
      mbar_init(&sh.kv_empty[i], G);  // a product P V of each group
    }
    for (int i = 0; i < kRawStages; ++i) {
      mbar_init(&sh.raw_full[i], 1);
      mbar_init(&sh.raw_empty[i], 8);
    }
    mbar_init(&sh.tail, 1);
    mbar_init(&sh.ended, 3);
    sh.abort_flag = 0;
    fence_barrier_init();
  }
  const AttendPart& part = a.part[part_index];
  const BlockWork w = block_work(a, part, blockIdx.x);
  const Problem pr = locate(a, part, w.problem);
  const int rows = pr.nt * a.group, r0 = w.row_tile * (G * kM);
  // (a launch that started early does not end before the one in front of it, whatever its blocks have to do)
  if (a.early && part_index == 1 && blockIdx.x == 0) wait_for_earlier();
  if (r0 >= rows) return;
  const int n_rows = min(G * kM, rows - r0);
  const int key0 = w.split * part.chunk;
  const bool direct = a.part_out == nullptr || FINISH;
  if (!direct && key0 >= pr.len) return;  // (the join kernel does not read it)
  const int last_seen = seen_rows(part, pr, (r0 + n_rows - 1) / a.group);
  const int key1 = min(last_seen, key0 + part.chunk);
  // (the shuffle tells the compiler that the value is the same in all lanes: the issuing loops then stay in uniform registers)
  const int nt = __shfl_sync(0xffffffffu, max(0, (key1 - key0 + kN - 1) / kN), 0);
  const bool alt = G == 2 && __shfl_sync(0xffffffffu, n_rows, 0) <= kM;  // both groups on the same rows, tiles in turn
  const int n_stages = alt ? turn_stages(FMT, D, G) : kStages;
  // token and query head of row r of the block: (first + r) / group by a multiplication (exact: first + r < 2^9, group <= 32)
  const int tok0 = r0 / a.group, first_g = r0 - tok0 * a.group;
  const uint32_t magic = (65536u + a.group - 1) / a.group;
  auto split_row = [&](int r, int& tok, int& hq) {
    const int d = (int)((uint32_t)(first_g + r) * magic >> 16);
    tok = tok0 + d;
    hq = w.head * a.group + first_g + r - d * a.group;
  };
  // The query rows are asked for before the first tiles, into the softmax warps' registers: behind the tiles' traffic a trip
  // to memory takes microseconds.
  const bool softmax_warp = warp >= 4 && warp < 4 + 4 * G;
  const int grp = (warp >> 2) - 1, base = alt ? 0 : grp * kM;  // a softmax warp's group, and the group's first row in the block
  constexpr int kLanes = D / 8, kPer = 32 / kLanes;            // lanes to a query row, rows to a load
  uint4 qx[32 / kPer];
  auto load_query = [&] {
#pragma unroll
    for (int i = 0; i < 32 / kPer; ++i) {
      const int r = base + (warp & 3) * 32 + i * kPer + lane / kLanes;
      qx[i] = make_uint4(0, 0, 0, 0);
      if (r < n_rows) {
        int tok, hq;
        split_row(r, tok, hq);
        if (token_ok(a, pr.t0 + tok, hq))
          qx[i] = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.q) + (pr.t0 + tok) * a.q_stride + (int64_t)hq * D + lane % kLanes * 8);
      }
    }
  };
  const bool loads_query = softmax_warp && nt > 0 && base < n_rows && !(alt && grp == 1);
  if (loads_query) load_query();
  const int row0 = (int)pr.row0 + key0;
  auto load_tile = [&](int j, int slot) {  // K and V of tile j (16-bit rows: into a stage; 8-bit rows: into the code ring)
    uint64_t* full = kF16 ? &sh.raw_full[slot] : &sh.kv_full[slot];
    unsigned char* to = kF16 ? raw + 2 * slot * kRaw : ring + 2 * slot * kTile;
    mbar_expect_tx(full, kF16 ? 2 * kRaw : 2 * kTile);
    const int row = row_ok(a, w.head, row0 + j * kN) ? row0 + j * kN : 0;
    tma_load_tile(to, &map_k, w.head, row, full);
    tma_load_tile(to + (kF16 ? kRaw : kTile), &map_v, w.head, row, full);
  };
  const int n_load = kF16 ? kRawStages : n_stages;  // stages of the ring that TMA fills
  if (warp == 3) tmem_alloc(&sh.tmem_base, kCols);
  tc_fence_before();
  // (warp 0 has initialised the barriers and needs nothing of the others: its first copies start at once)
  if (warp == 0) asm volatile("barrier.cta.arrive 4, %0;" ::"n"(threads(FMT, G)) : "memory");
  else asm volatile("barrier.cta.sync 4, %0;" ::"n"(threads(FMT, G)) : "memory");
  tc_fence_after();
  // a block of two groups has all of tensor memory, which starts at 0: a constant keeps the operand addresses out of registers
  const uint32_t tmem = G == 2 ? 0u : __shfl_sync(0xffffffffu, sh.tmem_base, 0);
  if (G == 2 && warp == 3 && lane == 0 && sh.tmem_base != 0) sh.abort_flag = 1;
  volatile int* abort_flag = &sh.abort_flag;

  if (!softmax_warp) {
    setmaxnreg_dec<regs_other(FMT, G)>();
    if (warp == 0) {
      // ---- TMA ----
      if (lane == 0) {
        int slot = 0, j = 0;
        uint32_t phase = 1;
        for (; j < nt; ++j) {
          if (!wait_or_abort(kF16 ? &sh.raw_empty[slot] : &sh.kv_empty[slot], phase, abort_flag, a.polls)) break;
          load_tile(j, slot);
          if (++slot == n_load) {
            slot = 0;
            phase ^= 1;
          }
        }
        sh.loads = j;
      }
    } else if (warp < 1 + G) {
      // ---- S of group g (the whole warp walks, one elected lane issues) ----
      constexpr uint32_t fmt = kF16 ? kFmtF16 : kFmtBF16;
      constexpr uint32_t idesc = instr_desc_f16(kM, kN, fmt, fmt, false, false);
      const int g = warp - 1, first = alt ? g : 0, step = alt ? 2 : 1;
      const uint32_t d_s = tmem + kColS + kStepS * g;
      const uint64_t dq = smem_desc_sw128(smem_u32(q_tiles + (alt ? 0 : g) * kQTile), 16, 1024);
      bool ok = first >= nt || wait_or_abort(&sh.q_full[alt ? 0 : g], 0, abort_flag, a.polls);
      int slot = first;
      uint32_t phase = 0;
      for (int j = first, n = 0; j < nt; j += step, ++n) {
        if (slot >= n_stages) {
          slot -= n_stages;
          phase ^= 1;
        }
        ok = ok && wait_or_abort(&sh.kv_full[slot], phase, abort_flag, a.polls);
        if (n > 0) ok = ok && wait_or_abort(&sh.s_read[g], (uint32_t)(n - 1) & 1u, abort_flag, a.polls);
        ok = __all_sync(0xffffffffu, ok) != 0;
        if (!ok) break;
        tc_fence_after();
        if (!kF16 && j == nt - 1) {
          // the range's last V tile: zeros behind it, by group A's warp or the one that uses it
          if (alt || g == 0) {
            const int there = key1 - key0 - j * kN;
            const uint32_t tile = smem_u32(ring + (2 * slot + 1) * kTile);
            for (int x = lane; x < (kN - there) * (D / 8); x += 32)
              st_shared16(operand_addr(tile, kN, there + x / (D / 8), x % (D / 8)), make_uint4(0, 0, 0, 0));
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.tail);
          } else {
            ok = __all_sync(0xffffffffu, wait_or_abort(&sh.tail, 0, abort_flag, a.polls)) != 0;
            if (!ok) break;
          }
        }
        const uint64_t dk = smem_desc_sw128(smem_u32(ring + 2 * slot * kTile), 16, 1024);
        if (elect_one()) {
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks) {
            const uint32_t qoff = ((uint32_t)(ks >> 2) * (kM * 128) + (uint32_t)(ks & 3) * 32u) >> 4;
            const uint32_t koff = ((uint32_t)(ks >> 2) * (kN * 128) + (uint32_t)(ks & 3) * 32u) >> 4;
            if (ks == 0) mma_ss_lohi<false>(d_s, desc_lo(dq), desc_hi(dq), desc_lo(dk), desc_hi(dk), idesc);
            else mma_ss_lohi<true>(d_s, desc_lo(dq) + qoff, desc_hi(dq), desc_lo(dk) + koff, desc_hi(dk), idesc);
          }
          mma_commit(&sh.s_full[g]);
        }
        __syncwarp();
        slot += step;
      }
    } else if (warp == 3) {
      // ---- O += P V of both groups, in the order A(0), B(0), A(1), ... (tiles in turn: A(0), B(1), A(2), ...) ----
      constexpr uint32_t fmt = kF16 ? kFmtF16 : kFmtBF16;
      constexpr uint32_t idesc = instr_desc_f16(kM, D, fmt, fmt, false, true);
      bool ok = true;
      int slot = 0;
      for (int j = 0; j < nt && ok; ++j) {
        const int n = alt ? j >> 1 : j;  // the group's own count
        const uint64_t dv = smem_desc_sw128(smem_u32(ring + (2 * slot + 1) * kTile), kTile / 2, 1024);
        for (int g = alt ? j & 1 : 0; g < (alt ? (j & 1) + 1 : G); ++g) {
          ok = __all_sync(0xffffffffu, wait_or_abort(&sh.p_full[g], (uint32_t)n & 1u, abort_flag, a.polls)) != 0;
          if (!ok) break;
          tc_fence_after();
          const uint32_t d_o = tmem + kColO + kStepO * g, d_p = tmem + kColP + kStepP * g;
          if (elect_one()) {
            if (n == 0) mma_ts_lohi<false>(d_o, d_p, desc_lo(dv), desc_hi(dv), idesc);
            else mma_ts_lohi<true>(d_o, d_p, desc_lo(dv), desc_hi(dv), idesc);
#pragma unroll
            for (int ks = 1; ks < kN / 16; ++ks)
              mma_ts_lohi<true>(d_o, d_p + 8u * ks, desc_lo(dv) + ((2048u * ks) >> 4), desc_hi(dv), idesc);
            mma_commit(&sh.p_empty[g]);
            mma_commit(&sh.kv_empty[slot]);
            if (alt) mma_commit(&sh.kv_empty[slot]);  // (for the group that does not use the tile)
            if (j + (alt ? 2 : 1) >= nt) mma_commit(&sh.o_final[g]);
          }
          __syncwarp();
        }
        if (++slot == n_stages) slot = 0;
      }
    } else if (kF16 && warp >= 12) {
      // ---- code tiles to f16 tiles, four warps for K and four for V: a thread takes 16 codes at a time ----
      // (Two sets of four warps that take tiles in turn: 50.4 us against 47.3 for 16 sequences of 4 query heads behind a prefix of
      // 32768, 8 heads; a third stage of codes: no difference.)
      // Eight neighbouring threads take four chunks of two rows (rows of 128 codes: the low four of one, the high four of
      // the other), which keeps both the loads and the stores free of bank conflicts.
      const int kv = (warp - 12) >> 2, t = threadIdx.x - 384 - 128 * kv;
      const int64_t base = (int64_t)w.head * a.rows + pr.row0;
      const uint8_t* scales = kv ? a.v_scale : a.k_scale;
      // of the next two tiles, one row to a thread: behind the tiles' traffic a load takes longer than a tile
      auto fetch = [&](int j) {
        const int key = key0 + j * kN + t;
        return t < kN && key < key1 && row_ok(a, w.head, pr.row0 + key) ? (uint32_t)scales[base + key] : 127u;
      };
      uint32_t byte = fetch(0), byte_next = fetch(1);
      int slot = 0;
      uint32_t phase = 1;
      bool raw_there = false, slot_free = false;
      for (int j = 0; j < nt; ++j) {
        const int rs = j % kRawStages;
        if (t < kN) sh.scale[j & 1][kv][t] = __float2half_rn(kv8_scale(byte));
        byte = byte_next;
        byte_next = fetch(j + 2);
        bool ok = raw_there || wait_or_abort(&sh.raw_full[rs], (uint32_t)(j / kRawStages) & 1u, abort_flag, a.polls);
        ok = ok && (slot_free || wait_or_abort(&sh.kv_empty[slot], phase, abort_flag, a.polls));
        ok = together(ok, kv);  // (also publishes the scales; one answer for the four warps, so that none waits for another)
        if (ok) {
          // the next tile's waits, asked ahead (the conversion hides the answers' way)
          const int rn = (j + 1) % kRawStages, sn = slot + 1 == n_stages ? 0 : slot + 1;
          raw_there = j + 1 < nt && mbar_test_wait(&sh.raw_full[rn], (uint32_t)((j + 1) / kRawStages) & 1u);
          slot_free = mbar_test_wait(&sh.kv_empty[sn], sn == 0 ? phase ^ 1u : phase);
          const int there = key1 - key0 - j * kN;
          const uint32_t src = smem_u32(raw + (2 * rs + kv) * kRaw), dst = smem_u32(ring + (2 * slot + kv) * kTile);
#pragma unroll
          for (int i = 0; i < kN * D / 16 / 128; ++i) {
            int row, c;
            if constexpr (D == 128) {
              const int q = i * 16 + (t >> 3), odd = (t >> 2) & 1;  // pair of rows q / 2
              row = (q & ~1) + odd;
              c = (t & 3) + 4 * (odd ^ (q & 1));
            } else {
              row = i * 32 + (t >> 2);
              c = t & 3;
            }
            const uint32_t at = D == 128 ? src + row * 128 + ((c ^ (row & 7)) << 4) : src + row * 64 + ((c ^ ((row >> 1) & 3)) << 4);
            uint32_t x[4];
            asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(at) : "memory");
            const __half2 f = __half2half2(sh.scale[j & 1][kv][row]);
            uint4 lo, hi;
            codes_to_f16(x[0], f, lo.x, lo.y);
            codes_to_f16(x[1], f, lo.z, lo.w);
            codes_to_f16(x[2], f, hi.x, hi.y);
            codes_to_f16(x[3], f, hi.z, hi.w);
            if (there < kN && row >= there) lo = hi = make_uint4(0, 0, 0, 0);  // behind the range
            st_shared16(operand_addr(dst, kN, row, 2 * c), lo);
            st_shared16(operand_addr(dst, kN, row, 2 * c + 1), hi);
          }
          fence_proxy_async();
        }
        __syncwarp();
        if (!ok) break;
        if (lane == 0) {
          mbar_arrive(&sh.raw_empty[rs]);
          mbar_arrive(&sh.kv_full[slot]);
        }
        if (++slot == n_stages) {
          slot = 0;
          phase ^= 1;
        }
      }
    }
  } else {
    setmaxnreg_inc<regs_softmax(FMT, G)>();
    const int g = grp, quarter = warp & 3;
    if (base < n_rows) {
      if (loads_query) {
        const int c = lane % kLanes;
        const uint32_t tile = smem_u32(q_tiles + g * kQTile);
#pragma unroll
        for (int i = 0; i < 32 / kPer; ++i) {
          const int rt = quarter * 32 + i * kPer + lane / kLanes;
          if constexpr (kF16) {
            float f[8];
            Vec16<__nv_bfloat16>::unpack(qx[i], f);
            float big = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) big = fabsf(f[e]) < INFINITY ? fmaxf(big, fabsf(f[e])) : big;
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
            const int e2 = max(-100, min(126, (int)(__float_as_uint(big) >> 23) - 127));
            const float down = __uint_as_float((uint32_t)(127 - e2) << 23);
            qx[i] = make_uint4(pack_half2(f[0] * down, f[1] * down), pack_half2(f[2] * down, f[3] * down),
                               pack_half2(f[4] * down, f[5] * down), pack_half2(f[6] * down, f[7] * down));
            if (c == 0) sh.row_factor[base + rt] = f16_row_factor(a.scale2, e2);
          }
          st_shared16(operand_addr(tile, kM, rt, c), qx[i]);
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.q_full[g]);
      }
      // (both groups on the same rows, 8-bit: B takes the row factors that A's warps left)
      if (kF16 && alt) softmax_sync();

      // (looked up while the first tile is on its way)
      Prefix prefix{0, 0, 0};
      if constexpr (FINISH) prefix = prefix_of(a, w.problem);

      // ---- softmax ----
      const int rt = quarter * 32 + lane, r = base + rt;
      int tok, hq;
      split_row(r, tok, hq);
      const int seen = min(key1, r < n_rows ? seen_rows(part, pr, tok) : key1);
      const int all_seen = part.causal ? min(key1, seen_rows(part, pr, (r0 + base) / a.group)) : key1;
      const float factor = kF16 ? sh.row_factor[r] : a.scale2;
      const uint32_t lane_addr = (uint32_t)(quarter * 32) << 16;
      const uint32_t t_s = tmem + kColS + kStepS * g + lane_addr, t_o = tmem + kColO + kStepO * g + lane_addr;
      const uint32_t t_p = tmem + kColP + kStepP * g + lane_addr;
      const bool idle = base + quarter * 32 >= n_rows;
      float m = -INFINITY;
      float2 l2 = make_float2(0.f, 0.f);
      bool ok = true;
      const int first = alt ? g : 0, step = alt ? 2 : 1;
      using N0 = std::integral_constant<int, 0>;
      using N1 = std::integral_constant<int, kN * 3 / 8>;
      using N2 = std::integral_constant<int, kN / 2>;
      for (int j = first, n = 0; j < nt; j += step, ++n) {
        ok = __all_sync(0xffffffffu, wait_or_abort(&sh.s_full[g], (uint32_t)n & 1u, abort_flag, a.polls));
        if (!ok) break;
        if (idle) {  // none of the warp's rows exists: whatever P holds there goes into rows of O that nobody reads
          if (n > 0) ok = __all_sync(0xffffffffu, wait_or_abort(&sh.p_empty[g], (uint32_t)(n - 1) & 1u, abort_flag, a.polls));
          if (!ok) break;
          if (lane == 0) {
            mbar_arrive(&sh.s_read[g]);
            mbar_arrive(&sh.p_full[g]);
          }
          continue;
        }
        tc_fence_after();
        const int key = key0 + j * kN;
        uint32_t s[kN], p[kN / 2];
        tmem_load(t_s, s);
        tmem_wait_ld_of(s);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.s_read[g]);
        if (key + kN > all_seen) {
#pragma unroll
          for (int e = 0; e < kN; ++e)
            if (key + e >= seen) s[e] = 0xff800000u;
        }
        // two 16-bit probabilities to a word of p, words FROM .. TO - 1; returns their sum
        auto exponentials = [&](auto from, auto to) {
          const float neg = m == -INFINITY ? 0.f : -m;
          float2 sum = make_float2(0.f, 0.f);
          float top = -INFINITY;  // of the exponents ex2_fma2 gets
#pragma unroll
          for (int e = decltype(from)::value; e < decltype(to)::value; ++e) {
            const float2 x = __ffma2_rn(make_float2(__uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1])),
                                        make_float2(factor, factor), make_float2(neg, neg));
            const bool poly = e % kPolyEvery == kPolyEvery - 1;
            if (poly) top = max3(top, x.x, x.y);
            const float2 y = poly ? ex2_fma2(x) : make_float2(ex2(x.x), ex2(x.y));
            sum = __fadd2_rn(sum, y);
            p[e] = kF16 ? pack_half2(y.x, y.y) : Vec16<__nv_bfloat16>::pack2(y.x, y.y);
          }
          if (top > kPolyMax) sum.x = INFINITY;
          return sum;
        };
        float2 sum = make_float2(0.f, 0.f);
        bool again = true;  // (the first tile: its maximum first)
        if (n > 0) {
          sum = exponentials(N0{}, N1{});
          // Has P(j - 1) been used (and does O include it)?  Asked ahead: the last exponentials hide the answer's way.
          const bool used = mbar_test_wait(&sh.p_empty[g], (uint32_t)(n - 1) & 1u);
          sum = __fadd2_rn(sum, exponentials(N1{}, N2{}));
          if (!used) ok = wait_or_abort(&sh.p_empty[g], (uint32_t)(n - 1) & 1u, abort_flag, a.polls);
          again = m == -INFINITY || sum.x + sum.y > kLargeSum;
        }
        if (__any_sync(0xffffffffu, again || !ok)) {
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          float top = -INFINITY;
#pragma unroll
          for (int e = 0; e < kN; e += 2) top = max3(top, __uint_as_float(s[e]), __uint_as_float(s[e + 1]));
          top *= factor;  // (the factor is positive: the maximum commutes with it)
          const float mn = top - kHead > m + kRescale ? top - kHead : m;
          const float alpha = mn == -INFINITY ? 1.f : ex2(m - mn);
          l2 = __fmul2_rn(l2, make_float2(alpha, alpha));
          m = mn;
          if (n > 0) {
            tc_fence_after();
#pragma unroll
            for (int cc = 0; cc < D / 16; ++cc) {
              uint32_t o[16];
              tmem_ld16(t_o + 16u * cc, o);
              tmem_wait_ld_of(o);
#pragma unroll
              for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
              tmem_st16(t_o + 16u * cc, o);
            }
          }
          sum = exponentials(N0{}, N2{});
        }
        l2 = __fadd2_rn(l2, sum);
        tc_fence_after();
        tmem_store(t_p, p);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.p_full[g]);
      }
      // ---- result ----
      const float sum = l2.x + l2.y;
      bool none = !ok || sum == 0.f;  // no key seen (NaN is a result)
      const bool wrote = nt > first;  // the group has an O
      if (ok && wrote) ok = __all_sync(0xffffffffu, wait_or_abort(&sh.o_final[g], 0, abort_flag, a.polls));
      float* join = reinterpret_cast<float*>(q_tiles);  // [2][128]
      if (alt) {  // B leaves m, sum (over Q) and O (over the K/V ring: both groups are done with them), A joins them
        if (g == 1 && ok && nt > 0) ok = __all_sync(0xffffffffu, wait_or_abort(&sh.o_final[0], 0, abort_flag, a.polls));
        tc_fence_after();
        float* theirs = reinterpret_cast<float*>(ring) + rt * (D + 4);
        if (g == 1) {
          join[rt] = none ? -INFINITY : m;
          join[kM + rt] = none ? 0.f : sum;
#pragma unroll
          for (int cc = 0; cc < D / 32; ++cc) {
            uint32_t o[32];
            if (wrote) {
              tmem_ld32(t_o + 32u * cc, o);
              tmem_wait_ld_of(o);
            }
#pragma unroll
            for (int e = 0; e < 32; e += 4)
              *reinterpret_cast<uint4*>(theirs + cc * 32 + e) = none ? make_uint4(0, 0, 0, 0) : make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
          }
        }
        softmax_sync();
        ok = __all_sync(0xffffffffu, ok && !*abort_flag) != 0;  // (A's result needs B's)
      }
      if (ok && !(alt && g == 1)) {
        tc_fence_after();
        float mine_w = none ? 0.f : 1.f, their_w = 0.f, total = none ? 0.f : sum, top = none ? -INFINITY : m;
        const float* theirs = reinterpret_cast<const float*>(ring) + rt * (D + 4);
        if (alt) {
          const float mb = join[rt];
          top = fmaxf(top, mb);
          const float to = top == -INFINITY ? 0.f : top;
          mine_w = none ? 0.f : ex2(m - to);
          their_w = ex2(mb - to);
          total = mine_w * total + their_w * join[kM + rt];
        }
        const int64_t token = pr.t0 + tok;
        bool write = r < n_rows && token_ok(a, token, hq);
        if constexpr (FINISH) {
          wait_for_earlier();
          write = write && token >= prefix.t0 && token < prefix.t1;
          if (write) {
            const float mx = prefix_top(a, prefix, token, hq, top);
            const float scale = top == -INFINITY ? 0.f : ex2(top - mx);
            mine_w *= scale;
            their_w *= scale;
            total = total * scale + (mx == -INFINITY ? 0.f : prefix_sum(a, prefix, token, hq, mx));
            top = mx;
          }
        }
        none = total == 0.f;
        const float inv = none ? 0.f : 1.f / total;
        const float lse2 = none ? -INFINITY : top + log2f(total);
        const int64_t at = ((int64_t)(part.slot0 + w.split) * a.q_rows + token) * a.heads * a.group + hq;
        if (!direct) write = write && partial_ok(a, at);
        __nv_bfloat16* to = static_cast<__nv_bfloat16*>(a.out) + token * a.out_stride + (int64_t)hq * D;
        // part 0's first chunk (mostly the only one), 64 channels of it asked for at a time
        [[maybe_unused]] float4 first[FINISH ? 16 : 1];
        [[maybe_unused]] float first_w = 0.f;
        if constexpr (FINISH) {
#pragma unroll
          for (int i = 0; i < 16; ++i) first[i] = make_float4(0.f, 0.f, 0.f, 0.f);
          write = write && (prefix.used == 0 || partial_ok(a, prefix.at(a, prefix.used - 1, token, hq)));
          if (write && prefix.used > 0 && !none) first_w = exp2f(a.part_lse[prefix.at(a, 0, token, hq)] - top) * inv;
        }
        auto load_first = [&](int cc) {
          const float* from = a.part_out + prefix.at(a, 0, token, hq) * D + cc * 32;
#pragma unroll
          for (int i = 0; i < 16; i += 2) ld_global_256(from + 4 * i, first[i], first[i + 1]);
        };
        const bool wide = ((reinterpret_cast<uintptr_t>(a.out) | (uintptr_t)(a.out_stride * 2)) & 31u) == 0;
#pragma unroll
        for (int cc = 0; cc < D / 32; ++cc) {
          if constexpr (FINISH) {
            if (cc % 2 == 0 && write && prefix.used > 0) load_first(cc);
          }
          uint32_t o[32];
          if (wrote) {
            tmem_ld32(t_o + 32u * cc, o);
            tmem_wait_ld_of(o);
          }
          if (!write) continue;
          // (a weight of 0 belongs to an O that was never written)
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            const float4 y = alt ? *reinterpret_cast<const float4*>(theirs + cc * 32 + e) : make_float4(0.f, 0.f, 0.f, 0.f);
            const float ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int b = 0; b < 4; ++b) {
              const float x = mine_w == 0.f ? 0.f : mine_w * __uint_as_float(o[e + b]);
              o[e + b] = __float_as_uint((alt ? fmaf(their_w, ys[b], x) : x) * inv);
            }
          }
          if constexpr (FINISH) {  // part 0's chunks
            auto add = [&](int e, float wgt, const float4& v) {
              o[e] = __float_as_uint(fmaf(wgt, v.x, __uint_as_float(o[e])));
              o[e + 1] = __float_as_uint(fmaf(wgt, v.y, __uint_as_float(o[e + 1])));
              o[e + 2] = __float_as_uint(fmaf(wgt, v.z, __uint_as_float(o[e + 2])));
              o[e + 3] = __float_as_uint(fmaf(wgt, v.w, __uint_as_float(o[e + 3])));
            };
#pragma unroll
            for (int e = 0; e < 32; e += 4) add(e, first_w, first[(cc % 2) * 8 + e / 4]);
            for (int s = 1; s < prefix.used; ++s) {
              const int64_t from = prefix.at(a, s, token, hq);
              const float wgt = none ? 0.f : exp2f(a.part_lse[from] - top) * inv;
#pragma unroll
              for (int e = 0; e < 32; e += 4) add(e, wgt, *reinterpret_cast<const float4*>(a.part_out + from * D + cc * 32 + e));
            }
          }
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
        if (write) {
          if (!direct) a.part_lse[at] = lse2;
          else if (a.lse) a.lse[token * a.heads * a.group + hq] = lse2 * 0.6931471805599453f;
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (sh.abort_flag) {  // the block ends after its copies and products under way (each waited for with a limit)
    if (warp == 0) {
      for (int j = max(0, sh.loads - n_load); j < sh.loads; ++j) {
        uint64_t* full = kF16 ? &sh.raw_full[j % n_load] : &sh.kv_full[j % n_load];
        for (uint32_t it = 0; it < kStorePolls && !mbar_try_wait(full, (uint32_t)(j / n_load) & 1u); ++it) {}
      }
      if (lane == 0 && a.status) atomicCAS(a.status, 0, H2O_ERR_TIMEOUT);
    } else if (warp <= 3) {
      if (elect_one()) mma_commit(&sh.ended);
      __syncwarp();
      for (uint32_t it = 0; it < kStorePolls && !mbar_try_wait(&sh.ended, 0); ++it) {}
    }
    __syncthreads();
  }
  if (warp == 3) {
    tc_fence_after();
    tmem_dealloc(tmem, kCols);
  }
}

template <int FMT, int D, int G, bool FINISH>
cudaError_t launch_finish(const AttendView& a, int part, const CUtensorMap& k, const CUtensorMap& v, cudaStream_t stream) {
  constexpr int smem = smem_bytes(FMT, D, G);
  static unsigned long long flags = 0;
  const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(attend_tc_kernel<FMT, D, G, FINISH>), smem, &flags);
  if (e != cudaSuccess) return e;
  return launch_kernel(attend_tc_kernel<FMT, D, G, FINISH>, dim3((unsigned)part_blocks(a, a.part[part])), threads(FMT, G), smem, stream,
                       a.early != 0 && part == 1, k, v, a, part);
}
template <int FMT, int D, int G>
cudaError_t launch(const AttendView& a, int part, const CUtensorMap& k, const CUtensorMap& v, cudaStream_t st) {
  return a.finish && part == 1 ? launch_finish<FMT, D, G, true>(a, part, k, v, st) : launch_finish<FMT, D, G, false>(a, part, k, v, st);
}

}  // namespace

int attend_tc_box_rows(int format, int dim, int groups) { return tile_keys(format, dim, groups); }

cudaError_t launch_attend_tc(const AttendView& a, int part, int groups, int format, const void* map_k, const void* map_v, cudaStream_t st) {
  const CUtensorMap& k = *static_cast<const CUtensorMap*>(map_k);
  const CUtensorMap& v = *static_cast<const CUtensorMap*>(map_v);
  if (format == H2O_KV8) return a.dim == 128 ? launch<H2O_KV8, 128, 2>(a, part, k, v, st) : launch<H2O_KV8, 64, 2>(a, part, k, v, st);
  if (groups == 1) return a.dim == 128 ? launch<H2O_BF16, 128, 1>(a, part, k, v, st) : launch<H2O_BF16, 64, 1>(a, part, k, v, st);
  return a.dim == 128 ? launch<H2O_BF16, 128, 2>(a, part, k, v, st) : launch<H2O_BF16, 64, 2>(a, part, k, v, st);
}

}  // namespace h2o
