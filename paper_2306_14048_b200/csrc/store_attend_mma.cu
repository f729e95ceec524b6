// Attention over a K/V store for few query rows (a decoding step): bfloat16 queries, bfloat16 or 8-bit rows,
// head_dim 64 or 128.  Bound by reading K and V once.
//
// Rows here are query tokens times the query heads of one K/V head: one for a plain decoding step, the group for
// grouped heads, all sequences of a group for a shared prefix.  A block takes 8 NT of them and a chunk of the keys;
// its four warps take 32-key tiles of the chunk in turn, each with its own ring of K and V tiles that it fills by TMA
// and its own running maximum and sum, so nothing but the merge at the end synchronises the block.
//
// Both products have the keys and channels on the M side of mma.sync m16n8k16 and the few query rows on N = 8:
//   S^T (keys x rows)      = K Q^T        A = K tile
//   O^T (channels x rows) += V^T P^T      A = V tile, transposed as it is loaded
// With rows on M a single row would leave 15 of 16 lanes' work unused; on N it is 7 of 8, and the accumulator of a row
// is half as many registers.  P leaves S^T's accumulators transposed (movmatrix), with no trip through shared memory.
//
// The reference maximum (8-bit rows: 7 less) moves only when a logit exceeds it by 8 (base 2), which a warp vote finds: in
// steady state no shuffle and no rescaling.  Sums are kept per lane and added at the end.
//
// bfloat16 rows: P = bf16 hi + bf16 lo (two products), so that its rounding (2^-8) does not add to the output's.  hi lies
// below P, so lo is positive like P: a value of infinity in V then gives that infinity in both products (a lo of 0 or
// less would make them NaN together).  What is left out is below 2^-15 of P: hi leaves 2^-7, of which lo rounds 2^-8 away.
// 8-bit rows: e4m3 codes become f16 exactly and P is one f16 (11 bits).  K's power of two multiplies the score; V's
// multiplies the codes (exact in f16 by the format's range; in P it would push small probabilities into subnormals).
// The query rows become f16 by a power of two of their own that brings the largest value into [1, 2).  Which
// channel sits in which k-slot (which key row of V^T in which M row) is free as long as both operands agree: a lane
// takes 16 codes of a row with one load.
#include <cuda.h>
#include <cuda_fp16.h>

#include "sm100_ptx.cuh"
#include "store.cuh"

namespace h2o {

namespace {

using namespace ptx;

constexpr int kWarps = 4, kThreads = kWarps * 32;
constexpr int kKeys = kFewBoxRows;                  // keys of a tile
constexpr float kRescale = 8.f;
// 8-bit rows: how far (base 2) the reference lies below the maximum.  In f16 whatever is below 2^-25 becomes 0: with at least
// 2^7 for the largest probability that is 2^-32 of it, so 2^20 such keys that go missing weigh 2^-12.  The largest
// is 2^(7 + 8), inside f16's range.
constexpr float kHeadF16 = 7.f;
// Shared memory of a block's rings (KB), and blocks on an SM that its registers and the splitting of the keys count on (one
// more fits where the code takes fewer), for blocks of up to 8 nt rows.  bfloat16, one query row (64 sequences of up to 2048
// rows, 32 heads / 32 of 4096, 4 heads of 8 query heads / 64 behind a prefix of 8192): 96 KB and 2 blocks 193 / 37.8 / 88.6
// us, 64 and 2 195.5 / 35.3 / 86.2, 64 and 3 195.5 / 37.1 / 86.0.  8-bit rows, whose conversion wants warps (32 sequences of
// up to 4096, 8 heads of 4 / 64 of 2048, 32 heads of 64): 64 and 3 40.7 / 68.5, 48 and 3 39.8 / 62.3, 48 and 4 41 / 62.1.
__host__ __device__ constexpr int ring_kb(int fmt, int nt) { return nt > 1 ? 96 : fmt == H2O_KV8 ? 48 : 64; }
__host__ __device__ constexpr int blocks_per_sm(int fmt, int nt) { return nt == 1 && fmt == H2O_KV8 ? 3 : 2; }
constexpr int kMaxSlots = 8;

__host__ __device__ constexpr int row_bytes(int fmt, int d) { return fmt == H2O_KV8 ? d : 2 * d; }
__host__ __device__ constexpr int tile_bytes(int fmt, int d) { return kKeys * row_bytes(fmt, d); }
__host__ __device__ constexpr int ring_slots(int fmt, int d, int nt) {
  return ring_kb(fmt, nt) * 1024 / kWarps / tile_bytes(fmt, d) < kMaxSlots ? ring_kb(fmt, nt) * 1024 / kWarps / tile_bytes(fmt, d) : kMaxSlots;
}

__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity, uint32_t polls) {
  for (uint32_t it = 0; it < polls; ++it)
    if (mbar_try_wait(bar, parity)) return true;
  return false;
}

__device__ __forceinline__ void tma_4d(void* dst, const CUtensorMap* map, int c1, int c3, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::
          "r"(smem_u32(dst)),
      "l"(map), "r"(0), "r"(c1), "r"(0), "r"(c3), "r"(smem_u32(bar))
      : "memory");
}

template <bool F16>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (F16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldsm4_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ void codes_to_f16(uint32_t word, uint32_t& lo, uint32_t& hi) {  // four e4m3 codes
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(word));
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// The largest bf16 number below p (0 for 0), in the upper half of the word; NaN stays NaN.
__device__ __forceinline__ uint32_t below(float p) { return (max(__float_as_uint(p), 1u) - 1u) & 0xffff0000u; }
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

template <int NT>  // the kernel's larger number of n-tiles
struct Shared {
  uint64_t full[kWarps][kMaxSlots];
  float m[kWarps][8 * NT], l[kWarps][8 * NT];  // the warps' statistics, per row
  int gave_up;                          // a wait of some warp has
  float row_factor[8 * NT];                // softmax scale times log2(e) (times the row's power of two)
  float k_factor[kWarps][kKeys];       // 8-bit rows: K's power of two of each key of the warp's tile
  __half v_factor[kWarps][kKeys];
  uint2 q[NT][8][32];                   // query operand, [n-tile][k-step][lane]
};

// The address of 16-byte chunk `c` of row `r` of a tile, as TMA swizzles it (tiles are 1024-byte aligned).
// Rows of 256 bytes are two halves of 128 bytes, one after the other.
template <int FMT, int D>
__device__ __forceinline__ uint32_t chunk_addr(uint32_t tile, int r, int c) {
  if constexpr (row_bytes(FMT, D) == 64) return tile + r * 64 + ((c ^ ((r >> 1) & 3)) << 4);
  else if constexpr (row_bytes(FMT, D) == 128) return tile + r * 128 + ((c ^ (r & 7)) << 4);
  else return tile + (c >> 3) * (kKeys * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4);
}

// NTB: the kernel's larger number of n-tiles, which the ring is made for.  WALK: the block takes its sequence's prefix
// (part 0's range) and then its own rows, and writes the result: no chunks, no joining kernel.
template <int FMT, int D, int NT, int NTB, bool WALK>
__device__ __forceinline__ void attend(const AttendView& a, const CUtensorMap* map_k, const CUtensorMap* map_v,
                                       const AttendPart& part, unsigned block, unsigned char* ring, Shared<NTB>& sh) {
  constexpr bool kF16 = FMT == H2O_KV8;
  constexpr float kHead = kF16 ? kHeadF16 : 0.f;
  constexpr int kTile = tile_bytes(FMT, D), kSlots = ring_slots(FMT, D, NTB), kSteps = D / 16, kRows = 8 * NT;
  constexpr int kPitch = D + 4;  // floats per row of a warp's partial output
  static_assert(kRows * kPitch * 4 <= kSlots * kTile, "a warp's partial output fits its ring");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gl = lane >> 2, c4 = lane & 3;
  const BlockWork w = block_work(a, part, block);
  const Problem pr = locate(a, part, w.problem);
  const int rows = pr.nt * a.group, r0 = w.row_tile * kRows;
  if (r0 >= rows) return;
  const int n_rows = min(kRows, rows - r0);
  const int key0 = w.split * part.chunk;
  const bool direct = a.part_out == nullptr;
  if (!direct && key0 >= pr.len) return;  // (the join kernel does not read it)
  const int last_seen = seen_rows(part, pr, (r0 + n_rows - 1) / a.group);  // the tile's last row sees the most
  const int key1 = min(last_seen, key0 + part.chunk);
  const int first_seen = part.causal ? seen_rows(part, pr, r0 / a.group) : last_seen;

  [[maybe_unused]] Problem prefix{0, 0, 0, 0};
  if constexpr (WALK) prefix = locate(a, a.part[0], group_of(a, w.problem));
  const int pre = WALK ? prefix.len : 0, pre_tiles = (pre + kKeys - 1) / kKeys;

  // ---- this warp's tiles: warp + 4 j of the prefix's and then the chunk's ----
  const int n_tiles = pre_tiles + max(0, (key1 - key0 + kKeys - 1) / kKeys);
  const int mine = n_tiles > warp ? (n_tiles - warp + kWarps - 1) / kWarps : 0;
  unsigned char* my_ring = ring + warp * (kSlots * kTile);
  uint64_t* full = sh.full[warp];
  auto issue = [&](int i) {  // item i: K of tile i / 2, then its V; lane 0 only
    const int t = warp + kWarps * (i >> 1);
    int row = WALK && t < pre_tiles ? (int)prefix.row0 + t * kKeys : (int)pr.row0 + key0 + (t - pre_tiles) * kKeys;
    if (!row_ok(a, w.head, row)) row = 0;
    mbar_expect_tx(&full[i % kSlots], kTile);
    tma_4d(my_ring + (i % kSlots) * kTile, (i & 1) ? map_v : map_k, row, w.head, &full[i % kSlots]);
  };
  if (threadIdx.x == 0) sh.gave_up = 0;
  if (lane == 0) {
    for (int s = 0; s < kSlots; ++s) mbar_init(&full[s], 1);
    fence_barrier_init();
    for (int i = 0; i < min(kSlots, 2 * mine); ++i) issue(i);
  }
  __syncwarp();

  // ---- the query operand: lane (gl, c4) of n-tile nt holds row 8 nt + gl (the warps share the n-tiles) ----
  for (int nt = warp; nt < NT; nt += kWarps) {
    const int r = nt * 8 + gl;
    const bool there = r < n_rows && token_ok(a, pr.t0 + (r0 + r) / a.group, w.head * a.group + (r0 + r) % a.group);
    const int tok = there ? (r0 + r) / a.group : 0;
    const __nv_bfloat16* qr = static_cast<const __nv_bfloat16*>(a.q) + (pr.t0 + tok) * a.q_stride +
                              ((int64_t)w.head * a.group + (there ? r0 + r - tok * a.group : 0)) * D;
    if constexpr (!kF16) {
#pragma unroll
      for (int ks = 0; ks < kSteps; ++ks) {
        uint2 b = make_uint2(0, 0);
        if (there) {
          b.x = *reinterpret_cast<const uint32_t*>(qr + 16 * ks + 2 * c4);
          b.y = *reinterpret_cast<const uint32_t*>(qr + 16 * ks + 2 * c4 + 8);
        }
        sh.q[nt][ks][lane] = b;
      }
      if (c4 == 0) sh.row_factor[r] = a.scale2;
    } else {
      // k-step ks, slot pairs (2 c4, 2 c4 + 8): channels 4 (ks % 4) + {0, 1}, {2, 3} of the lane's 16-channel chunk
      uint2 raw[kSteps];
      float big = 0.f;
#pragma unroll
      for (int ks = 0; ks < kSteps; ++ks) {
        const int chunk = D == 128 ? 2 * c4 + (ks >> 2) : c4;
        raw[ks] = there ? *reinterpret_cast<const uint2*>(qr + 16 * chunk + 4 * (ks & 3)) : make_uint2(0, 0);
        const float f[4] = {__uint_as_float(raw[ks].x << 16), __uint_as_float(raw[ks].x & 0xffff0000u),
                            __uint_as_float(raw[ks].y << 16), __uint_as_float(raw[ks].y & 0xffff0000u)};
#pragma unroll
        for (int e = 0; e < 4; ++e) big = fabsf(f[e]) < INFINITY ? fmaxf(big, fabsf(f[e])) : big;
      }
      big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
      big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
      const int e2 = max(-100, min(126, (int)(__float_as_uint(big) >> 23) - 127));  // (zeros: any power will do)
      const float down = __uint_as_float((uint32_t)(127 - e2) << 23);
#pragma unroll
      for (int ks = 0; ks < kSteps; ++ks) {
        uint2 b;
        b.x = pack_half2(__uint_as_float(raw[ks].x << 16) * down, __uint_as_float(raw[ks].x & 0xffff0000u) * down);
        b.y = pack_half2(__uint_as_float(raw[ks].y << 16) * down, __uint_as_float(raw[ks].y & 0xffff0000u) * down);
        sh.q[nt][ks][lane] = b;
      }
      if (c4 == 0) sh.row_factor[r] = f16_row_factor(a.scale2, e2);
    }
  }
  __syncthreads();

  float factor[NT][2];
  int seen[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int r = nt * 8 + 2 * c4 + e;
      factor[nt][e] = sh.row_factor[r];
      seen[nt][e] = r < n_rows ? (part.causal ? seen_rows(part, pr, (r0 + r) / a.group) : last_seen) : last_seen;
    }
  uint2 qf[NT == 1 ? kSteps : 1];
  if constexpr (NT == 1) {
#pragma unroll
    for (int ks = 0; ks < kSteps; ++ks) qf[ks] = sh.q[0][ks][lane];
  }
  float m[NT][2], l[NT][2], o[kSteps][NT][4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m[nt][0] = m[nt][1] = -INFINITY;
    l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
    for (int ct = 0; ct < kSteps; ++ct)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[ct][nt][e] = 0.f;
  }
  // Items this lane would ask for; -1 - i once its wait for item i has given up.  Nothing is asked for from then on (lane 0
  // asks, and has seen every item before arrive), and the warp leaves the loop at the next vote: a vote for each wait costs
  // an 8-bit step as much again as this (39.4 us without, 40.0 and 40.3).
  int limit = 2 * mine;
  // 8-bit rows: the scale bytes of the warp's next tile, one key per lane
  uint32_t scale_k = 127, scale_v = 127;
  auto fetch_scales = [&](int j) {
    const int t = warp + kWarps * j;
    const bool in_prefix = WALK && t < pre_tiles;
    const int key = (in_prefix ? t : t - pre_tiles) * kKeys + (in_prefix ? 0 : key0) + lane;
    if (key < (in_prefix ? pre : key1) && row_ok(a, w.head, (in_prefix ? prefix.row0 : pr.row0) + key)) {
      const int64_t at = (int64_t)w.head * a.rows + (in_prefix ? prefix.row0 : pr.row0) + key;
      scale_k = a.k_scale[at];
      scale_v = a.v_scale[at];
    }
  };
  if constexpr (kF16) {
    if (mine > 0) fetch_scales(0);
  }

  int j = 0;
  for (; j < mine; ++j) {
    const int tile_no = warp + kWarps * j;
    const bool in_prefix = WALK && tile_no < pre_tiles;
    const int tile_key = in_prefix ? tile_no * kKeys : key0 + (tile_no - pre_tiles) * kKeys, end = in_prefix ? pre : key1;
    const int there = min(kKeys, end - tile_key);
    if constexpr (kF16) {
      sh.k_factor[warp][lane] = kv8_scale(scale_k);
      sh.v_factor[warp][lane] = __float2half_rn(kv8_scale(scale_v));
      if (j + 1 < mine) fetch_scales(j + 1);
      __syncwarp();
    }
    // ---- S^T = K Q^T ----
    float s[2][NT][4];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[mt][nt][e] = 0.f;
    {
      const int i = 2 * j, slot = i % kSlots;
      if (!wait(&full[slot], (uint32_t)(i / kSlots) & 1u, a.polls) && limit >= 0) limit = -1 - i;
      const uint32_t tile = smem_u32(my_ring + slot * kTile);
      if constexpr (!kF16) {
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) {
          uint32_t ka[2][4];
#pragma unroll
          for (int mt = 0; mt < 2; ++mt)
            ldsm4(ka[mt], chunk_addr<FMT, D>(tile, mt * 16 + (lane & 15), 2 * ks + (lane >> 4)));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            uint2 b;
            if constexpr (NT == 1) b = qf[ks];
            else b = sh.q[nt][ks][lane];
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) mma<false>(s[mt][nt], ka[mt], b.x, b.y);
          }
        }
      } else {
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {
          uint4 lo[2], hi[2];  // 16 codes of keys gl and gl + 8
#pragma unroll
          for (int mt = 0; mt < 2; ++mt) {
            const int chunk = D == 128 ? 2 * c4 + c : c4;
            const uint32_t at = chunk_addr<FMT, D>(tile, mt * 16 + gl, chunk);
            const uint32_t at8 = chunk_addr<FMT, D>(tile, mt * 16 + gl + 8, chunk);
            asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(lo[mt].x), "=r"(lo[mt].y), "=r"(lo[mt].z), "=r"(lo[mt].w) : "r"(at) : "memory");
            asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(hi[mt].x), "=r"(hi[mt].y), "=r"(hi[mt].z), "=r"(hi[mt].w) : "r"(at8) : "memory");
          }
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            uint32_t ka[2][4];
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
              const uint32_t wl = t == 0 ? lo[mt].x : t == 1 ? lo[mt].y : t == 2 ? lo[mt].z : lo[mt].w;
              const uint32_t wh = t == 0 ? hi[mt].x : t == 1 ? hi[mt].y : t == 2 ? hi[mt].z : hi[mt].w;
              codes_to_f16(wl, ka[mt][0], ka[mt][2]);
              codes_to_f16(wh, ka[mt][1], ka[mt][3]);
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              uint2 b;
              if constexpr (NT == 1) b = qf[4 * c + t];
              else b = sh.q[nt][4 * c + t][lane];
#pragma unroll
              for (int mt = 0; mt < 2; ++mt) mma<true>(s[mt][nt], ka[mt], b.x, b.y);
            }
          }
        }
      }
      __syncwarp();
      if (lane == 0 && i + kSlots < limit) issue(i + kSlots);
    }
    // ---- logits (base 2); lane: keys gl, gl + 8 (+ 16 mt), rows 2 c4, 2 c4 + 1 (+ 8 nt) ----
    const bool masked = tile_key + kKeys > (in_prefix ? pre : min(first_seen, key1));
    bool grows = false;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      float kf[2] = {1.f, 1.f};
      if constexpr (kF16) {
        kf[0] = sh.k_factor[warp][mt * 16 + gl];
        kf[1] = sh.k_factor[warp][mt * 16 + gl + 8];
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float x = s[mt][nt][e];
          if constexpr (kF16) x *= kf[e >> 1];
          x *= factor[nt][e & 1];
          if (masked) {
            const int key = tile_key + mt * 16 + gl + 8 * (e >> 1);
            if (key >= (in_prefix ? pre : min(seen[nt][e & 1], key1))) x = -INFINITY;
          }
          s[mt][nt][e] = x;
          grows |= x > m[nt][e & 1] + (kRescale + kHead);
        }
    }
    if (__any_sync(0xffffffffu, grows || limit < 0)) {
      if (__any_sync(0xffffffffu, limit < 0)) break;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float top = fmaxf(fmaxf(s[0][nt][e], s[0][nt][e + 2]), fmaxf(s[1][nt][e], s[1][nt][e + 2]));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
          const float mn = fmaxf(m[nt][e], top - kHead);
          const float alpha = mn == -INFINITY ? 1.f : ex2(m[nt][e] - mn);
          l[nt][e] *= alpha;
          m[nt][e] = mn;
#pragma unroll
          for (int ct = 0; ct < kSteps; ++ct) {
            o[ct][nt][e] *= alpha;
            o[ct][nt][e + 2] *= alpha;
          }
        }
    }
    // ---- P, as the B operand of the second product: keys on K, rows on N ----
    uint32_t ph[2][NT][2];
    [[maybe_unused]] uint32_t pl[2][NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float b0 = m[nt][0] == -INFINITY ? 0.f : m[nt][0], b1 = m[nt][1] == -INFINITY ? 0.f : m[nt][1];
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float p0 = ex2(s[mt][nt][2 * h] - b0), p1 = ex2(s[mt][nt][2 * h + 1] - b1);
          l[nt][0] += p0;
          l[nt][1] += p1;
          if constexpr (kF16) {
            ph[mt][nt][h] = transpose8x8(pack_half2(p0, p1));
          } else {
            const uint32_t h0 = below(p0), h1 = below(p1);
            ph[mt][nt][h] = transpose8x8(__byte_perm(h0, h1, 0x7632));
            pl[mt][nt][h] = transpose8x8(Vec16<__nv_bfloat16>::pack2(p0 - __uint_as_float(h0), p1 - __uint_as_float(h1)));
          }
        }
    }
    // ---- O^T += V^T P^T ----
    {
      const int i = 2 * j + 1, slot = i % kSlots;
      if (!wait(&full[slot], (uint32_t)(i / kSlots) & 1u, a.polls) && limit >= 0) limit = -1 - i;
      const uint32_t tile = smem_u32(my_ring + slot * kTile);
      if (there < kKeys) {
        // rows behind the range may hold anything, and 0 * NaN must not reach the sums
        for (int x = lane; x < (kKeys - there) * (row_bytes(FMT, D) / 16); x += 32) {
          const uint32_t at = chunk_addr<FMT, D>(tile, there + x / (row_bytes(FMT, D) / 16), x % (row_bytes(FMT, D) / 16));
          asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(at), "r"(0) : "memory");
        }
        __syncwarp();
      }
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        if constexpr (!kF16) {
#pragma unroll
          for (int ct = 0; ct < kSteps; ++ct) {
            uint32_t va[4];
            ldsm4_trans(va, chunk_addr<FMT, D>(tile, kt * 16 + (lane & 7) + ((lane >> 4) << 3), 2 * ct + ((lane >> 3) & 1)));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              mma<false>(o[ct][nt], va, ph[kt][nt][0], ph[kt][nt][1]);
              mma<false>(o[ct][nt], va, pl[kt][nt][0], pl[kt][nt][1]);
            }
          }
        } else {
          const __half2 f0 = *reinterpret_cast<const __half2*>(&sh.v_factor[warp][kt * 16 + 2 * c4]);
          const __half2 f1 = *reinterpret_cast<const __half2*>(&sh.v_factor[warp][kt * 16 + 2 * c4 + 8]);
#pragma unroll
          for (int cc = 0; cc < kSteps; cc += 2) {
            uint32_t x[4];  // (keys 0-7, keys 8-15) of channels 16 cc .., then of 16 (cc + 1) ..
            ldsm4_trans(x, chunk_addr<FMT, D>(tile, kt * 16 + (lane & 15), cc + (lane >> 4)));
#pragma unroll
            for (int q = 0; q < 2; ++q) {
              // a word holds keys 2 c4, 2 c4 + 1 of channels 2 gl, 2 gl + 1: M row gl is channel 2 gl, row gl + 8 the next
              uint32_t va[4];
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const uint32_t y = __byte_perm(x[2 * q + h], 0, 0x3120);
                uint32_t e0, e1;
                codes_to_f16(y, e0, e1);
                const __half2 g0 = __hmul2(*reinterpret_cast<const __half2*>(&e0), h ? f1 : f0);
                const __half2 g1 = __hmul2(*reinterpret_cast<const __half2*>(&e1), h ? f1 : f0);
                va[2 * h] = *reinterpret_cast<const uint32_t*>(&g0);
                va[2 * h + 1] = *reinterpret_cast<const uint32_t*>(&g1);
              }
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) mma<true>(o[cc + q][nt], va, ph[kt][nt][0], ph[kt][nt][1]);
            }
          }
        }
      }
      if (WALK && there < kKeys) fence_proxy_async();  // (the zeros come before the copy that may go over them)
      __syncwarp();
      if (lane == 0 && i + kSlots < limit) issue(i + kSlots);
    }
  }
  if (__any_sync(0xffffffffu, limit < 0)) {
    if (lane == 0) {  // the block does not end before the copies under way
      const int taken = limit < 0 ? -1 - limit : min(2 * mine, 2 * j + 1);
      for (int i = taken; i < min(2 * mine, taken + kSlots); ++i) wait(&full[i % kSlots], (uint32_t)(i / kSlots) & 1u, kStorePolls);
      sh.gave_up = 1;
      if (a.status) atomicCAS(a.status, 0, H2O_ERR_TIMEOUT);
    }
    __syncwarp();
  }

  // ---- the warps' results, joined through shared memory (each warp over its own ring) ----
  float* my_o = reinterpret_cast<float*>(my_ring);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float sum = l[nt][e];
      sum += __shfl_xor_sync(0xffffffffu, sum, 4);
      sum += __shfl_xor_sync(0xffffffffu, sum, 8);
      sum += __shfl_xor_sync(0xffffffffu, sum, 16);
      const int r = nt * 8 + 2 * c4 + e;
      if (gl == 0) {
        sh.m[warp][r] = m[nt][e];
        sh.l[warp][r] = sum;
      }
#pragma unroll
      for (int ct = 0; ct < kSteps; ++ct) {
        my_o[r * kPitch + ct * 16 + (kF16 ? 2 * gl : gl)] = o[ct][nt][e];
        my_o[r * kPitch + ct * 16 + (kF16 ? 2 * gl + 1 : gl + 8)] = o[ct][nt][e + 2];
      }
    }
  __syncthreads();
  if (sh.gave_up) return;  // (the same for the whole block)
  constexpr int kLanes = D / 4;  // threads of a row, four channels each
  for (int r = threadIdx.x / kLanes; r < n_rows; r += kThreads / kLanes) {
    const int c = (threadIdx.x % kLanes) * 4;
    const int tok = (r0 + r) / a.group;
    const int64_t token = pr.t0 + tok;
    const int hq = w.head * a.group + (r0 + r) - tok * a.group;
    if (WALK && (token < prefix.t0 || token >= prefix.t0 + prefix.nt)) continue;  // beyond what the caller allowed for
    if (!token_ok(a, token, hq)) continue;
    float top = -INFINITY;
#pragma unroll
    for (int x = 0; x < kWarps; ++x) top = fmaxf(top, sh.m[x][r]);
    const float base = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int x = 0; x < kWarps; ++x) {
      const float wgt = ex2(sh.m[x][r] - base);
      sum += wgt * sh.l[x][r];
      const float4 part_o = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(ring + x * (kSlots * kTile)) + r * kPitch + c);
      v.x = fmaf(wgt, part_o.x, v.x);
      v.y = fmaf(wgt, part_o.y, v.y);
      v.z = fmaf(wgt, part_o.z, v.z);
      v.w = fmaf(wgt, part_o.w, v.w);
    }
    const bool none = sum == 0.f;
    const float inv = none ? 0.f : 1.f / sum;
    const float lse2 = none ? -INFINITY : top + log2f(sum);
    if (direct) {
      uint2 word;
      word.x = Vec16<__nv_bfloat16>::pack2(v.x * inv, v.y * inv);
      word.y = Vec16<__nv_bfloat16>::pack2(v.z * inv, v.w * inv);
      *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + token * a.out_stride + (int64_t)hq * D + c) = word;
      if (a.lse && c == 0) a.lse[token * a.heads * a.group + hq] = lse2 * 0.6931471805599453f;
    } else {
      const int64_t at = ((int64_t)(part.slot0 + w.split) * a.q_rows + token) * a.heads * a.group + hq;
      if (!partial_ok(a, at)) continue;
      *reinterpret_cast<float4*>(a.part_out + at * D + c) = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
      if (c == 0) a.part_lse[at] = lse2;
    }
  }
}

// One launch for part `first` alone, with 8 NT0 rows to a block, or for parts 0 and 1 (a shared prefix: many rows and
// few), with 8 NT0 and 8 NT1.
template <int FMT, int D, int NT0, int NT1, bool WALK>
__global__ void __launch_bounds__(kThreads, blocks_per_sm(FMT, NT0))
attend_mma_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                  const __grid_constant__ AttendView a, int first, unsigned blocks0) {
  extern __shared__ unsigned char dyn[];
  __shared__ Shared<NT0> sh;
  unsigned char* ring = dyn + ((1024u - (smem_u32(dyn) & 1023u)) & 1023u);
  let_next_start();  // (the joining kernel waits for this one's end; others are launched to start after it)
  if (NT0 == NT1 || blockIdx.x < blocks0) {
    const bool second = blockIdx.x >= blocks0;
    attend<FMT, D, NT0, NT0, WALK>(a, &map_k, &map_v, a.part[second ? 1 : first], blockIdx.x - (second ? blocks0 : 0), ring, sh);
  } else {
    attend<FMT, D, NT1, NT0, false>(a, &map_k, &map_v, a.part[1], blockIdx.x - blocks0, ring, sh);
  }
  // a launch that started early does not end before the one in front of it, whatever its blocks have to do
  if (a.early && blockIdx.x == 0) wait_for_earlier();
}

template <int FMT, int D, int NT0, int NT1, bool WALK = false>
cudaError_t launch(const AttendView& a, int first, bool both, const CUtensorMap& map_k, const CUtensorMap& map_v, cudaStream_t stream) {
  constexpr int smem = kWarps * ring_slots(FMT, D, NT0) * tile_bytes(FMT, D) + 1024;
  static unsigned long long flags = 0;
  const void* f = reinterpret_cast<const void*>(attend_mma_kernel<FMT, D, NT0, NT1, WALK>);
  const cudaError_t e = ensure_dynamic_smem(f, smem, &flags);
  if (e != cudaSuccess) return e;
  const int64_t b0 = part_blocks(a, a.part[first]), b1 = both ? part_blocks(a, a.part[1]) : 0;
  return launch_kernel(attend_mma_kernel<FMT, D, NT0, NT1, WALK>, dim3((unsigned)(b0 + b1)), kThreads, smem, stream, a.early != 0, map_k, map_v, a,
                       first, (unsigned)b0);
}

template <int FMT, int D>
cudaError_t launch_rows(const AttendView& a, int first, bool both, const int* tile, const CUtensorMap& map_k, const CUtensorMap& map_v,
                        cudaStream_t st) {
  if (a.walk) return launch<FMT, D, 1, 1, true>(a, 1, false, map_k, map_v, st);
  const int t0 = tile[first], t1 = both ? tile[1] : t0;
  if (t0 == 8) return launch<FMT, D, 1, 1>(a, first, both, map_k, map_v, st);
  if (t0 == 16) return t1 == 8 ? launch<FMT, D, 2, 1>(a, first, both, map_k, map_v, st) : launch<FMT, D, 2, 2>(a, first, both, map_k, map_v, st);
  if constexpr (FMT == H2O_KV8) {  // (bfloat16 rows: more than 16 query rows run on the tcgen05 kernel)
    if (t1 == 8) return launch<FMT, D, 4, 1>(a, first, both, map_k, map_v, st);
    return t1 == 16 ? launch<FMT, D, 4, 2>(a, first, both, map_k, map_v, st) : launch<FMT, D, 4, 4>(a, first, both, map_k, map_v, st);
  }
  return cudaErrorInvalidValue;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

}  // namespace

int attend_mma_row_tile(int64_t rows) { return rows <= 8 ? 8 : rows <= 16 ? 16 : 32; }
int attend_mma_blocks_per_sm(int format, int tile) { return blocks_per_sm(format, tile / 8); }

// Rows of a store: {bytes or elements of up to 128 bytes, rows, pieces of a row, heads}; a box is `box_rows` rows of one
// head, swizzled over as many bytes as its inner extent.
bool make_store_map(CUtensorMap_st* map, const h2o_store_config_t& c, const void* base, int box_rows) {
  static EncodeTiledFn fn = nullptr;
  if (!fn) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      return false;
    fn = reinterpret_cast<EncodeTiledFn>(p);
  }
  const bool eight = c.format == H2O_KV8;
  const cuuint64_t inner = eight ? c.head_dim : 64, pieces = eight ? 1 : c.head_dim / 64;
  const cuuint64_t row = eight ? c.head_dim : c.row_stride * 2, head = eight ? c.rows * c.head_dim : c.head_dim * 2;
  const cuuint64_t dims[4] = {inner, (cuuint64_t)c.rows, pieces, (cuuint64_t)c.n_heads};
  const cuuint64_t strides[3] = {row, 128, head};
  const cuuint32_t box[4] = {(cuuint32_t)inner, (cuuint32_t)box_rows, (cuuint32_t)pieces, 1};
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  return fn(map, eight ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims,
            strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            eight && c.head_dim == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

cudaError_t launch_attend_mma(const AttendView& a, int first, bool both, const int* tile, int format, const void* map_k,
                              const void* map_v, cudaStream_t st) {
  const CUtensorMap& k = *static_cast<const CUtensorMap*>(map_k);
  const CUtensorMap& v = *static_cast<const CUtensorMap*>(map_v);
  if (format == H2O_KV8) return a.dim == 128 ? launch_rows<H2O_KV8, 128>(a, first, both, tile, k, v, st) : launch_rows<H2O_KV8, 64>(a, first, both, tile, k, v, st);
  return a.dim == 128 ? launch_rows<H2O_BF16, 128>(a, first, both, tile, k, v, st) : launch_rows<H2O_BF16, 64>(a, first, both, tile, k, v, st);
}

}  // namespace h2o
