// Attention over a paged cache for many query rows (prompts, pieces of prompts, windows): tcgen05 with the accumulators in
// tensor memory; bfloat16, head_dim 64 or 128.
//
// An item of work is up to 128 query rows (query tokens times the query heads of one K/V head) against the keys that they see,
// 64 at a time:
//   S(j) = Q K_j^T         into tensor memory, from there into the softmax threads' registers, which frees S at once
//   P(j) = exp2(S - m)     bf16, into tensor memory of its own
//   O   += P(j) V_j        P is the tensor-memory operand, V the MN-major shared-memory operand
// Two blocks share an SM, so that one's exponentials run beside the other's products.  A block goes on to further items until
// there are none: it takes over the place of a block of the grid that has not started (clusterlaunchcontrol), so that the
// hardware hands the work out in the grid's order and nobody counts.  The next item's keys and queries are on their way while
// the last tiles of an item are computed, and its first S while the item's result is written.
// Roles: warp 0 takes items and issues the copies of K, a box of a page to a lane; warp 2 copies query rows and V; warp 1 issues
// S, warp 3 issues P V, clears what nobody sees in a V tile (0 * NaN must not reach the sums) and owns tensor memory; warps
// 4..7 are the softmax, one thread per row.
// Bound by the softmax warps and the power limit.  A tile takes 1640 cycles with two blocks on the SM (1350 alone): 900 for the
// exponentials (450 of them the special function unit's), 330 to learn that S is there, 320 for loading, masking and storing;
// its products take 640 (S reads the queries from shared memory again for every 16 channels, 48 cycles of 32; the keys of a tile
// are as many as tensor memory holds beside O and P).  An item costs 4 to 5 us more: the last product, the result, the first
// tile's maximum.  Four prompts of up to 4096 tokens, 32 heads of 128, window 1020 and 4 sinks, pages of 64: 245-247 us, 745 TFLOP/s of
// what the mask leaves, for a few calls; back to back 290 us, 635, at the 1600 MHz that the power limit leaves after a second.  Steps, for a
// few calls: 360 with blocks of one item, two groups of rows and pairs of K and V in one ring; 310 with further items; 247 once no warp
// waited for a table entry where it read it; 245 with steps of 16 keys that nobody sees left out of the products.
// Tried: tiles of 80 keys (long ranges 3 % faster, windows 5 % slower); S of 128 keys at once with P over it (304 against 285 us
// under the power limit); more or fewer exponentials on the FMA pipe (one pair in 4: 266, in 16: 248).
// The reference m of a row is the maximum of its first tile.  Later tiles compute their exponentials against it without
// looking for a maximum: only when a tile's sum comes out large (kLargeSum) the tile is done again with the new maximum and O
// is rescaled.  A value far above the reference costs no precision in floating point, only range.
// Rounding: P is one bf16.  Its error, up to 2^-8 relative per key and of either sign, averages over the keys to about that of
// the output's own rounding, which is up to 2^-8 as well.  Row sums are fp32 sums of the unrounded values.
#include "attend_tc.cuh"
#include "pages.cuh"

namespace h2o {

namespace {

using namespace tc;

constexpr int kM = 128, kN = 64;  // rows and keys of a tile
constexpr int kThreads = 256;
constexpr int kItems = 2;  // ring of items, the one under way and the next
constexpr int kMostSkipped = 256;  // places in a row without work (1.5 us each)
// Rings of tiles of K and of V, what fits half an SM's shared memory beside the queries.  (K is done with a tile earlier than V: a
// ring of pairs would hold it as long.)
__host__ __device__ constexpr int tile_bytes(int d) { return kN * d * 2; }
__host__ __device__ constexpr int slots_k(int d) { return d == 128 ? 2 : 4; }
__host__ __device__ constexpr int slots_v(int d) { return d == 128 ? 3 : 4; }
constexpr int kMaxSlots = 5;
// Registers of a thread: 256 start with 128 each = 128 x 176 + 128 x 80.
constexpr int kRegsSoftmax = 176, kRegsOther = 80;
constexpr int kPolyEvery = 8;  // every so many pairs of exponentials one runs on the FMA pipe
constexpr float kRescale = 8.f;
constexpr float kLargeSum = 1048576.f;  // O, which is divided by its sum at the end, then holds values up to 2^100

// What a block works on; nt < 0: nothing any more.
struct Item {
  int nt;              // tiles of keys
  int head, split;
  int r0, n_rows;      // rows of the problem
  int problem, key0;   // first key of the chunk, as the block numbers them
  int tokens, len;     // of the problem
  int64_t t0;          // its first token
  Keys keys;
};

struct Shared {
  uint4 answer;  // to the request for another block's place
  uint64_t full[2][kMaxSlots], empty[2][kMaxSlots];  // K, V
  uint64_t item_full[kItems], item_empty[kItems];
  uint64_t answered;
  uint64_t q_full, q_empty;
  uint64_t s_full, s_read;   // S is complete / in the softmax threads' registers
  uint64_t p_full, p_empty;  // P is complete / used, and O includes it
  uint64_t o_final;
  uint64_t ended;  // of a block that gives up: the products of warps 1 and 3 have ended
  Item item[kItems];
  uint32_t tmem_base;
  int abort_flag;
};
__host__ __device__ constexpr int smem_bytes(int d) { return kM * d * 2 + (slots_k(d) + slots_v(d)) * tile_bytes(d) + (int)sizeof(Shared); }

// Asks for the place of a block that has not started.
__device__ __forceinline__ void request_place(uint4* answer, uint64_t* bar) {
  mbar_expect_tx(bar, 16);
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(smem_u32(answer)), "r"(smem_u32(bar))
               : "memory");
}
// The place (its block index), or -1: there is none any more.
__device__ __forceinline__ int place_of(const uint4* answer) {
  uint32_t there, x;
  asm volatile(
      "{\n\t.reg .b128 a;\n\t.reg .pred p;\n\t.reg .b32 y, z, w;\n\t"
      "ld.shared.b128 a, [%2];\n\t"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, a;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t"
      "mov.b32 %1, 0;\n\t"
      "@p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%1, y, z, w}, a;\n\t}"
      : "=r"(there), "=r"(x)
      : "r"(smem_u32(answer))
      : "memory");
  return there ? (int)x : -1;
}
// Steps of 16 keys of the tile that starts at `key`, up to the last one with a key that some row of the item sees.
__device__ __forceinline__ int steps_of(const AttendView& a, const Keys& k, int key) {
  int end = min(k.end - key, kN);
  if (key + kN <= k.from) end = min(end, a.pages.sinks - key);
  return max(1, (end + 15) >> 4);
}
// The lowest n bits, for any n.
__device__ __forceinline__ uint32_t bits_below(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}

// A lane's box of the tile that comes next, looked up a tile ahead of its copy.  (The entry is looked at only when the copy is
// issued: a use of it where it is read would wait for it, 400 cycles for each of K and V.)
struct Box {
  int entry, row;
  __device__ __forceinline__ void find(const AttendView& a, const Item& it, int j, int b) {
    const int x = it.keys.at(it.key0 + j * kN) + b * a.pages.box;
    row = x - page_index(a, x) * a.pages.page_size;
    entry = a.pages.n_pages;
    if (j < it.nt && b * a.pages.box < kN && !unseen(a, it.keys, x, a.pages.box) && page_rows_ok(a, it.head, row, a.pages.box))
      entry = table_entry(a, it.problem, x);
  }
};

template <int D>
__global__ void __launch_bounds__(kThreads, 2)
pages_tc_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ AttendView a) {
  constexpr int kTile = tile_bytes(D), kQTile = kM * D * 2, kSlotsK = slots_k(D), kSlotsV = slots_v(D), kHalves = D / 64;
  constexpr uint32_t kColO = 0, kColS = D, kColP = D + kN, kCols = 256;
  static_assert(kColP + kN / 2 <= kCols, "tensor memory");
  static_assert(smem_bytes(D) + 1024 <= 114 * 1024, "two blocks on an SM");
  extern __shared__ unsigned char dyn[];
  unsigned char* const q_tile = dyn;
  unsigned char* const ring_k = dyn + kQTile;
  unsigned char* const ring_v = ring_k + kSlotsK * kTile;
  Shared& sh = *reinterpret_cast<Shared*>(ring_v + kSlotsV * kTile);
  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    prefetch_tensormap(&map_k);
    prefetch_tensormap(&map_v);
    for (int i = 0; i < 2 * kMaxSlots; ++i) {
      mbar_init(&sh.full[0][i], 1);
      mbar_init(&sh.empty[0][i], 1);
    }
    for (int i = 0; i < kItems; ++i) {
      mbar_init(&sh.item_full[i], 1);
      mbar_init(&sh.item_empty[i], 7);  // all warps but warp 0
    }
    mbar_init(&sh.answered, 1);
    mbar_init(&sh.q_full, 1);
    mbar_init(&sh.q_empty, 1);
    mbar_init(&sh.s_full, 1);
    mbar_init(&sh.s_read, 4);
    mbar_init(&sh.p_full, 4);
    mbar_init(&sh.p_empty, 1);
    mbar_init(&sh.o_final, 1);
    mbar_init(&sh.ended, 2);
    // the operands' swizzle counts from multiples of 1024 bytes
    sh.abort_flag = (smem_u32(dyn) & 1023u) != 0;
    fence_barrier_init();
  }
  if (warp == 3) tmem_alloc(&sh.tmem_base, kCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, sh.tmem_base, 0);
  volatile int* const abort_flag = &sh.abort_flag;
  const AttendPart& part = a.part[0];
  const int box = a.pages.box, shift = 31 - __clz(box);  // 8, 16, 32 or 64
  auto wait = [&](uint64_t* bar, uint32_t parity) { return wait_or_abort(bar, parity & 1u, abort_flag, a.polls); };
  // all lanes of a warp
  auto wait_all = [&](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(bar, parity)) != 0; };
  // what a block that gives up has under way ends before it does
  auto settle = [&](uint64_t* bar, uint32_t parity) {
    for (uint32_t x = 0; x < kStorePolls && !mbar_try_wait(bar, parity & 1u); ++x) {}
  };
  // Item number n, by a whole warp; its fields are copied, so that its place is free again.
  auto next_item = [&](uint32_t n, Item& it) {
    if (!wait_all(&sh.item_full[n % kItems], n / kItems)) return false;
    it = sh.item[n % kItems];
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.item_empty[n % kItems]);
    return it.nt >= 0;
  };
  // token and query head of row r of an item: (first + r) / group by a multiplication (exact: first + r < 2^8, group <= 32)
  const uint32_t magic = (65536u + a.group - 1) / a.group;
  auto split_row = [&](const Item& it, int r, int& tok, int& hq) {
    const int tok0 = it.r0 / a.group, first = it.r0 - tok0 * a.group;
    const int d = (int)((uint32_t)(first + r) * magic >> 16);
    tok = tok0 + d;
    hq = it.head * a.group + first + r - d * a.group;
  };

  if (warp < 4) {
    setmaxnreg_dec<kRegsOther>();
    if (warp == 0) {
      // ---- items, and the copies of their K ----
      // A lane has a box of rows of a tile and half of its channels (one lane all of the tile, if that is one box).
      const int boxes = kN / box, copies = boxes == 1 ? 1 : boxes * kHalves;
      const int my_box = boxes == 1 ? lane : lane / kHalves, my_half = boxes == 1 ? 0 : lane % kHalves;
      uint32_t n = 0, tiles = 0, requests = 0;  // items published, tiles and places asked for
      bool ok = true, pending = false;
      Item it, next;
      // What a place stands for: row tiles last to first (the longest of a causal prompt first), then head, split, sequence.
      // False: no work.
      auto describe = [&](unsigned i) {
        const int row_tile = part.row_tiles - 1 - (int)(i % part.row_tiles);
        i /= part.row_tiles;
        next.head = (int)(i % a.heads);
        i /= a.heads;
        next.split = (int)(i % part.splits);
        next.problem = (int)(i / part.splits);
        const Problem pr = locate<true>(a, part, next.problem);
        next.r0 = row_tile * kM;
        next.n_rows = min(kM, pr.nt * a.group - next.r0);
        next.key0 = next.split * part.chunk;
        next.tokens = pr.nt;
        next.len = pr.len;
        next.t0 = pr.t0;
        if (next.n_rows <= 0 || (a.part_out != nullptr && next.key0 >= shared_keys<true>(part, pr))) return false;
        next.keys = keys_of<true>(a, seen_rows(part, pr, next.r0 / a.group), seen_rows(part, pr, (next.r0 + next.n_rows - 1) / a.group), kN);
        next.nt = max(0, (min(next.keys.count(), next.key0 + part.chunk) - next.key0 + kN - 1) / kN);
        return true;
      };
      auto publish = [&] {
        ok = ok && wait_all(&sh.item_empty[n % kItems], n / kItems + 1);
        if (ok && lane == 0) {
          sh.item[n % kItems] = next;
          mbar_arrive(&sh.item_full[n % kItems]);
        }
        __syncwarp();
        ++n;
      };
      auto request = [&] {
        if (lane == 0) request_place(&sh.answer, &sh.answered);
        __syncwarp();
        pending = true;
      };
      // The next item, or the end (nt < 0), found and published; after many places without work an item of no rows, so that nobody
      // waits for long.
      auto advance = [&](bool first) {
        next.nt = -1;
        int skipped = 0;
        for (bool found = first && describe(blockIdx.x); !found;) {
          if (!pending) request();
          ok = wait_all(&sh.answered, requests);
          if (!ok) return;
          pending = false;
          ++requests;
          const int place = place_of(&sh.answer);
          fence_proxy_async();  // (read before the next answer is written over it)
          __syncwarp();
          if (place < 0) {
            next.nt = -1;
            break;
          }
          found = describe((unsigned)place);
          if (!found && ++skipped == kMostSkipped) {
            next.nt = next.n_rows = 0;
            found = true;
          }
        }
        publish();
      };
      advance(true);
      while (ok && next.nt >= 0) {
        it = next;
        // The next place is asked for a few tiles before this item's last copies and taken two tiles before (not earlier: what a
        // block holds back nobody else can take).
        const int ask = max(0, it.nt - 4), take = max(0, it.nt - 2);
        Box next_box;
        next_box.find(a, it, 0, my_box);
        if (it.nt == 0) advance(false);
        for (int j = 0; j < it.nt && ok; ++j) {
          if (j == ask) request();
          const uint32_t at = tiles % kSlotsK;
          ok = wait_all(&sh.empty[0][at], tiles / kSlotsK + 1);
          if (!ok) break;
          if (lane == 0) mbar_expect_tx(&sh.full[0][at], kTile);
          __syncwarp();
          if (lane < copies)
            tma_page(smem_u32(ring_k + at * kTile) + my_half * (kN * 128) + my_box * box * 128, &map_k, next_box.row, my_half, it.head, page_in(a, next_box.entry),
                     &sh.full[0][at]);
          ++tiles;
          next_box.find(a, it, j + 1, my_box);
          if (j == take) advance(false);
        }
      }
      // of a block that gives up: nothing of its own is under way when it ends
      if (*abort_flag) {
        if (pending) settle(&sh.answered, requests);
        for (uint32_t t = tiles > kSlotsK ? tiles - kSlotsK : 0u; t < tiles; ++t) settle(&sh.full[0][t % kSlotsK], t / kSlotsK);
      }
    } else if (warp == 1) {
      // ---- S (the whole warp walks, one elected lane issues) ----
      constexpr uint32_t idesc_16 = instr_desc_f16(kM, 16, kFmtBF16, kFmtBF16, false, false);
      const uint64_t dq = smem_desc_sw128(smem_u32(q_tile), 16, 1024);
      const uint32_t d_s = tmem + kColS;
      uint32_t count = 0, queries = 0;  // tiles, items with tiles
      bool ok = true;
      Item it;
      for (uint32_t n = 0; ok && next_item(n, it); ++n) {
        const int nt = __shfl_sync(0xffffffffu, it.nt, 0);
        if (nt == 0) continue;
        ok = wait_all(&sh.q_full, queries++);
        for (int j = 0; j < nt && ok; ++j, ++count) {
          const uint32_t slot = count % kSlotsK;
          ok = wait_all(&sh.full[0][slot], count / kSlotsK);
          if (ok && count > 0) ok = wait_all(&sh.s_read, count - 1);
          if (!ok) break;
          tc_fence_after();
          const uint64_t dk = smem_desc_sw128(smem_u32(ring_k + slot * kTile), 16, 1024);
          // (as many columns as hold a key that somebody sees; the others keep what was there, and are masked)
          const uint32_t idesc = idesc_16 + ((uint32_t)(__shfl_sync(0xffffffffu, steps_of(a, it.keys, it.keys.at(it.key0 + j * kN)), 0) - 1) << 18);
          if (elect_one()) {
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
              const uint32_t qoff = ((uint32_t)(ks >> 2) * (kM * 128) + (uint32_t)(ks & 3) * 32u) >> 4;
              const uint32_t koff = ((uint32_t)(ks >> 2) * (kN * 128) + (uint32_t)(ks & 3) * 32u) >> 4;
              if (ks == 0) mma_ss_lohi<false>(d_s, desc_lo(dq), desc_hi(dq), desc_lo(dk), desc_hi(dk), idesc);
              else mma_ss_lohi<true>(d_s, desc_lo(dq) + qoff, desc_hi(dq), desc_lo(dk) + koff, desc_hi(dk), idesc);
            }
            mma_commit(&sh.s_full);
            mma_commit(&sh.empty[0][slot]);
            if (j == nt - 1) mma_commit(&sh.q_empty);
          }
          __syncwarp();
        }
      }
    } else if (warp == 2) {
      // ---- the items' query rows, as soon as the last S of the item before has been computed, and the copies of their V ----
      const int boxes = kN / box;
      uint32_t queries = 0, tiles = 0;  // items with keys, tiles
      bool ok = true;
      Item it;
      const uint32_t tile = smem_u32(q_tile);
      for (uint32_t n = 0; ok && next_item(n, it); ++n) {
        if (it.nt == 0) continue;
        Box next_box;
        next_box.find(a, it, 0, lane);
        if (queries > 0) ok = wait_all(&sh.q_empty, queries - 1);
        if (!ok) break;
        ++queries;
        constexpr int kLanes = D / 8, kPer = 32 / kLanes;  // lanes to a row, rows to a copy
        const int tok0 = it.r0 / a.group, first = it.r0 - tok0 * a.group, c = lane % kLanes;
        const __nv_bfloat16* const from = static_cast<const __nv_bfloat16*>(a.q) + (it.t0 + tok0) * a.q_stride + (int64_t)it.head * a.group * D + c * 8;
#pragma unroll 8
        for (int r = lane / kLanes; r < kM; r += kPer) {
          const uint32_t x = (uint32_t)(first + min(r, it.n_rows - 1)), tok = x * magic >> 16, g = x - tok * a.group;
          const bool there = r < it.n_rows && token_ok(a, it.t0 + tok0 + tok, it.head * a.group + (int)g);
          cp_async16(tile + (c >> 3) * (kM * 128) + r * 128 + (((c ^ r) & 7) << 4), from + (int64_t)tok * a.q_stride + g * D, there);
        }
        for (int j = 0; j < it.nt && ok; ++j) {
          const uint32_t at = tiles % kSlotsV;
          ok = wait_all(&sh.empty[1][at], tiles / kSlotsV + 1);
          if (ok) {
            if (lane == 0) mbar_expect_tx(&sh.full[1][at], kTile);
            __syncwarp();
            if (lane < boxes)
              tma_page(smem_u32(ring_v + at * kTile) + lane * box * (128 * kHalves), &map_v, next_box.row, 0, it.head, page_in(a, next_box.entry), &sh.full[1][at]);
            ++tiles;
            next_box.find(a, it, j + 1, lane);
          }
          if (j == 0) {  // (the first tile's V is asked for while the query rows are on their way)
            asm volatile("cp.async.wait_all;" ::: "memory");
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.q_full);
          }
        }
      }
      if (*abort_flag)
        for (uint32_t t = tiles > kSlotsV ? tiles - kSlotsV : 0u; t < tiles; ++t) settle(&sh.full[1][t % kSlotsV], t / kSlotsV);
    } else {
      // ---- O += P V ----
      constexpr uint32_t idesc = instr_desc_f16(kM, D, kFmtBF16, kFmtBF16, false, true);
      const uint32_t d_o = tmem + kColO, d_p = tmem + kColP;
      // V lies box after box, a box as halves of 64 channels; groups of 8 rows, 16 rows to a step
      const uint32_t group = box == 8 ? 1024u * kHalves : 1024u;
      uint32_t step[kN / 16];
#pragma unroll
      for (int ks = 0; ks < kN / 16; ++ks) step[ks] = (uint32_t)(ks * 16 / box * (box * 128 * kHalves) + ks * 16 % box * 128) >> 4;
      uint32_t count = 0;
      bool ok = true;
      Item it;
      for (uint32_t n = 0; ok && next_item(n, it); ++n) {
        const int nt = __shfl_sync(0xffffffffu, it.nt, 0);
        for (int j = 0; j < nt && ok; ++j, ++count) {
          const uint32_t slot = count % kSlotsV;
          ok = wait_all(&sh.full[1][slot], count / kSlotsV);
          if (!ok) break;
          const uint32_t tile = smem_u32(ring_v + slot * kTile);
          const int key = it.keys.at(it.key0 + j * kN), steps = __shfl_sync(0xffffffffu, steps_of(a, it.keys, key), 0);
          if (key + kN > it.keys.end || (key < it.keys.from && key + kN > a.pages.sinks)) {
            constexpr int kLanes = D / 8;  // lanes to a row
            const int c = lane % kLanes;
#pragma unroll 4
            for (int r = lane / kLanes; r < 16 * steps; r += 32 / kLanes)
              if (unseen(a, it.keys, key + r, 1))
                st_shared16(tile + (r >> shift) * (box * 128 * kHalves) + (c >> 3) * (box * 128) + (r & (box - 1)) * 128 + (((c ^ r) & 7) << 4),
                            make_uint4(0, 0, 0, 0));
            fence_proxy_async();
            __syncwarp();
          }
          ok = wait_all(&sh.p_full, count);
          if (!ok) break;
          tc_fence_after();
          const uint64_t dv = smem_desc_sw128(tile, (uint32_t)box * 128u, group);
          if (elect_one()) {
            if (j == 0) mma_ts_lohi<false>(d_o, d_p, desc_lo(dv), desc_hi(dv), idesc);
            else mma_ts_lohi<true>(d_o, d_p, desc_lo(dv), desc_hi(dv), idesc);
#pragma unroll
            for (int ks = 1; ks < kN / 16; ++ks)
              if (ks < steps) mma_ts_lohi<true>(d_o, d_p + 8u * ks, desc_lo(dv) + step[ks], desc_hi(dv), idesc);
            mma_commit(&sh.p_empty);
            mma_commit(&sh.empty[1][slot]);
            if (j == nt - 1) mma_commit(&sh.o_final);
          }
          __syncwarp();
        }
      }
    }
  } else {
    setmaxnreg_inc<kRegsSoftmax>();
    const int quarter = warp & 3, r = quarter * 32 + lane;
    const uint32_t lane_addr = (uint32_t)(quarter * 32) << 16;
    const uint32_t t_s = tmem + kColS + lane_addr, t_o = tmem + kColO + lane_addr, t_p = tmem + kColP + lane_addr;
    const bool wide = ((reinterpret_cast<uintptr_t>(a.out) | (uintptr_t)(a.out_stride * 2)) & 31u) == 0;
    uint32_t count = 0, done = 0;  // tiles, items with tiles
    bool ok = true;
    Item it;
    for (uint32_t n = 0; ok && next_item(n, it); ++n) {
      const int nt = __shfl_sync(0xffffffffu, it.nt, 0);
      int tok, hq;
      split_row(it, r, tok, hq);
      const Problem pr{it.t0, 0, it.tokens, it.len};
      // the first key that the row does not see; of the item's first row; the first key behind the sinks that the row sees; of the
      // item's last row
      const int seen = r < it.n_rows ? seen_rows(part, pr, tok) : it.keys.end, all_seen = seen_rows(part, pr, it.r0 / a.group);
      const int from = window_from(a, seen), last_from = window_from(a, it.keys.end);
      const bool idle = quarter * 32 >= it.n_rows;
      float m = -INFINITY;
      float2 l2 = make_float2(0.f, 0.f);
      for (int j = 0; j < nt; ++j, ++count) {
        ok = wait_all(&sh.s_full, count);
        if (!ok) break;
        if (idle) {  // none of the warp's rows exists: whatever P holds there goes into rows of O that nobody reads
          if (count > 0) ok = wait_all(&sh.p_empty, count - 1);
          if (!ok) break;
          if (lane == 0) {
            mbar_arrive(&sh.s_read);
            mbar_arrive(&sh.p_full);
          }
          continue;
        }
        tc_fence_after();
        const int key = it.keys.at(it.key0 + j * kN);
        uint32_t s[kN], p[kN / 2];
        tmem_load(t_s, s);
        tmem_wait_ld_of(s);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.s_read);
        if (key + kN > all_seen || (key < last_from && key + kN > a.pages.sinks)) {
#pragma unroll
          for (int w = 0; w < kN; w += 32) {
            const int x = key + w;
            const uint32_t visible = bits_below(seen - x) & ~(bits_below(from - x) & ~bits_below(a.pages.sinks - x));
#pragma unroll
            for (int e = 0; e < 32 && w + e < kN; ++e)
              if (!(visible & (1u << e))) s[w + e] = 0xff800000u;
          }
        }
        // two 16-bit probabilities to a word of p, words FROM .. TO - 1; returns their sum
        auto exponentials = [&](int first, int last) {
          const float neg = m == -INFINITY ? 0.f : -m;
          float2 sum = make_float2(0.f, 0.f);
          float top = -INFINITY;  // of the exponents ex2_fma2 gets
#pragma unroll
          for (int e = 0; e < kN / 2; ++e) {
            if (e < first || e >= last) continue;
            const float2 x = __ffma2_rn(make_float2(__uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1])), make_float2(a.scale2, a.scale2),
                                        make_float2(neg, neg));
            const bool poly = e % kPolyEvery == kPolyEvery - 1;
            if (poly) top = max3(top, x.x, x.y);
            const float2 y = poly ? ex2_fma2(x) : make_float2(ex2(x.x), ex2(x.y));
            sum = __fadd2_rn(sum, y);
            p[e] = Vec16<__nv_bfloat16>::pack2(y.x, y.y);
          }
          if (top > kPolyMax) sum.x = INFINITY;
          return sum;
        };
        float2 sum = make_float2(0.f, 0.f);
        bool again = true;  // (the first tile: its maximum first)
        // Has the P before been used (and does O include it)?  Asked ahead: the last exponentials hide the answer's way.
        bool used = count == 0;
        if (j > 0) {
          sum = exponentials(0, kN / 2 - 8);
          used = mbar_test_wait(&sh.p_empty, (count - 1) & 1u);
          sum = __fadd2_rn(sum, exponentials(kN / 2 - 8, kN / 2));
          again = m == -INFINITY || sum.x + sum.y > kLargeSum;
        }
        if (!used) ok = wait(&sh.p_empty, count - 1);
        if (__any_sync(0xffffffffu, again || !ok)) {
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          float top = -INFINITY;
#pragma unroll
          for (int e = 0; e < kN; e += 2) top = max3(top, __uint_as_float(s[e]), __uint_as_float(s[e + 1]));
          top *= a.scale2;  // (positive: the maximum commutes with it)
          const float mn = top > m + kRescale ? top : m;
          const float alpha = mn == -INFINITY ? 1.f : ex2(m - mn);
          l2 = __fmul2_rn(l2, make_float2(alpha, alpha));
          m = mn;
          if (j > 0) {
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
          sum = exponentials(0, kN / 2);
        }
        l2 = __fadd2_rn(l2, sum);
        tc_fence_after();
        tmem_store(t_p, p);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.p_full);
      }
      if (!ok) break;
      // ---- the item's result ----
      if (nt > 0) ok = wait_all(&sh.o_final, done++);
      if (!ok) break;
      tc_fence_after();
      const float total = l2.x + l2.y;
      const bool none = nt == 0 || total == 0.f;  // no key seen (NaN is a result)
      const float inv = none ? 0.f : 1.f / total;
      const float lse2 = none ? -INFINITY : m + log2f(total);
      const int64_t token = it.t0 + tok;
      const int64_t at = ((int64_t)(part.slot0 + it.split) * a.q_rows + token) * a.heads * a.group + hq;
      const bool direct = a.part_out == nullptr;
      const bool write = r < it.n_rows && token_ok(a, token, hq) && (direct || partial_ok(a, at));
      __nv_bfloat16* to = static_cast<__nv_bfloat16*>(a.out) + token * a.out_stride + (int64_t)hq * D;
#pragma unroll
      for (int cc = 0; cc < D / 32; ++cc) {
        uint32_t o[32];
        if (nt > 0) {
          tmem_ld32(t_o + 32u * cc, o);
          tmem_wait_ld_of(o);
        }
        if (!write) continue;
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
      // (the next item's first P, which lets O be written again, comes after these loads)
      tc_fence_before();
      if (write) {
        if (!direct) a.part_lse[at] = lse2;
        else if (a.lse) a.lse[token * a.heads * a.group + hq] = lse2 * 0.6931471805599453f;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (sh.abort_flag) {  // the block ends after its copies (warp 0, above) and products under way, waited for with a limit
    if (warp == 0 && lane == 0 && a.status) atomicCAS(a.status, 0, H2O_ERR_TIMEOUT);
    if (warp == 1 || warp == 3) {
      if (elect_one()) mma_commit(&sh.ended);
      __syncwarp();
      for (uint32_t x = 0; x < kStorePolls && !mbar_try_wait(&sh.ended, 0); ++x) {}
    }
    __syncthreads();
  }
  if (warp == 3) {
    tc_fence_after();
    tmem_dealloc(tmem, kCols);
  }
}

template <int D>
cudaError_t launch(const AttendView& a, const CUtensorMap& k, const CUtensorMap& v, cudaStream_t stream) {
  constexpr int smem = smem_bytes(D);
  static unsigned long long flags = 0;
  const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(pages_tc_kernel<D>), smem, &flags);
  if (e != cudaSuccess) return e;
  return launch_kernel(pages_tc_kernel<D>, dim3((unsigned)part_blocks(a, a.part[0])), kThreads, smem, stream, false, k, v, a);
}

}  // namespace

int pages_tc_tile_keys() { return kN; }

cudaError_t launch_pages_tc(const AttendView& a, const void* map_k, const void* map_v, cudaStream_t stream) {
  const CUtensorMap& k = *static_cast<const CUtensorMap*>(map_k);
  const CUtensorMap& v = *static_cast<const CUtensorMap*>(map_v);
  return a.dim == 128 ? launch<128>(a, k, v, stream) : launch<64>(a, k, v, stream);
}

}  // namespace h2o
