// Attention over a K/V store for float32 queries, on the fp32 FMA pipe (float32 or 8-bit rows, head_dim 64 and 128): a kernel
// for up to four query rows (a decoding step) and one for more.
//
// More: a block takes BM query rows (query tokens times the query heads of one K/V head) and walks over its keys 64 at a
// time: S = Q K^T by register tiles, softmax with the running maximum and sum of each row, O += P V.
// 256 threads as 16 x 16: thread (x, y) has rows y * RM .. + RM - 1, keys x + 16 j of a tile, output columns
// 4 x + 64 j .. + 3, so a row's statistics are shuffles within 16 lanes and its probabilities pass between them
// through shared memory without a block barrier.  K of the next tile is fetched (cp.async, float32 rows) during
// P V, V during the next S.  Bound by shared memory: 8 vector loads (32 wavefronts) feed 64 multiply-adds of a warp.
// 4 x 512 queries against 2048 keys each, 16 heads of 128 (34.4 GFLOP): 1106 us, 31 TFLOP/s; 8-bit rows 1315 us.
#include "store.cuh"

namespace h2o {

namespace {

constexpr int kThreads = 256, kBN = 64, kJ = kBN / 16;  // (tiles of 32 keys and three blocks on an SM: the same time)

__device__ __forceinline__ void cp_async16(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void store4(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }

// e4m3 -> float, by its bits: exponent and mantissa moved into place, times 2^120 (exact, subnormals included)
__device__ __forceinline__ float e4m3(uint32_t b) {
  const float f = __uint_as_float(((b & 0x80u) << 24) | ((b & 0x7fu) << 20)) * 1.329227995784916e36f;
  return (b & 0x7fu) == 0x7fu ? __uint_as_float(0x7fffffffu) : f;
}

template <int D, int BM>
struct Smem {
  float q[BM][D + 4];
  float k[kBN][D + 4];
  float v[kBN][D];
  float p[BM][kBN + 4];
};

// One tile of K or V (rows row0 .. row0 + n - 1 of one head; the rest of the tile zero: a key that no row sees may
// hold anything, and 0 * NaN must not reach the sums).
template <int FMT, int D, int PITCH>
__device__ __forceinline__ void load_tile(float* dst, const void* base, const uint8_t* scale, const AttendView& a, int head,
                                          int64_t row0, int n) {
  if constexpr (FMT == H2O_F32) {
    constexpr int kV = D / 4;
    for (int i = threadIdx.x; i < kBN * kV; i += kThreads) {
      const int r = i / kV, c = (i % kV) * 4;
      float* to = dst + r * PITCH + c;
      if (r < n && row_ok(a, head, row0 + r)) cp_async16(to, static_cast<const float*>(base) + (row0 + r) * a.row_stride + (int64_t)head * D + c);
      else *reinterpret_cast<float4*>(to) = make_float4(0.f, 0.f, 0.f, 0.f);
    }
  } else {
    constexpr int kV = D / 16;
    for (int i = threadIdx.x; i < kBN * kV; i += kThreads) {
      const int r = i / kV, c = (i % kV) * 16;
      uint4 w = make_uint4(0, 0, 0, 0);
      float s = 0.f;
      if (r < n && row_ok(a, head, row0 + r)) {
        const int64_t at = (int64_t)head * a.rows + row0 + r;
        w = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(base) + at * D + c);
        s = kv8_scale(scale[at]);
      }
      const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<float4*>(dst + r * PITCH + c + 4 * j) =
            make_float4(e4m3(words[j] & 255u) * s, e4m3((words[j] >> 8) & 255u) * s, e4m3((words[j] >> 16) & 255u) * s, e4m3(words[j] >> 24) * s);
    }
  }
  cp_commit();
}

template <int FMT, int D, int BM>
__global__ void __launch_bounds__(kThreads) attend_fma_kernel(const __grid_constant__ AttendView a, int part_index) {
  constexpr int RM = BM / 16, NC = D / 64;
  extern __shared__ __align__(16) unsigned char dyn[];
  Smem<D, BM>& sh = *reinterpret_cast<Smem<D, BM>*>(dyn);
  const AttendPart& part = a.part[part_index];
  const BlockWork w = block_work(a, part, blockIdx.x);
  const Problem pr = locate(a, part, w.problem);
  const int rows = pr.nt * a.group;
  const int r0 = w.row_tile * BM;
  if (r0 >= rows) return;
  const int n_rows = min(BM, rows - r0);
  const int key0 = w.split * part.chunk;
  // keys beyond what the tile's last row sees are never needed
  const int last_seen = seen_rows(part, pr, (r0 + n_rows - 1) / a.group);
  const int key1 = min(last_seen, key0 + part.chunk);
  const bool direct = a.part_out == nullptr;
  if (!direct && key0 >= pr.len) return;  // (the join kernel does not read it)
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4;

  // the query rows, zero behind the last one
  for (int i = threadIdx.x; i < BM * (D / 4); i += kThreads) {
    const int r = i / (D / 4), c = (i % (D / 4)) * 4;
    float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
    if (r < n_rows) {
      const int tok = (r0 + r) / a.group, g = (r0 + r) - tok * a.group;
      if (token_ok(a, pr.t0 + tok, w.head * a.group + g))
        f = *reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + (pr.t0 + tok) * a.q_stride + ((int64_t)w.head * a.group + g) * D + c);
    }
    *reinterpret_cast<float4*>(&sh.q[r][c]) = f;
  }
  int seen[RM];
#pragma unroll
  for (int i = 0; i < RM; ++i) {
    const int r = y * RM + i;
    seen[i] = r < n_rows ? seen_rows(part, pr, (r0 + r) / a.group) : 0;
  }
  float m[RM], l[RM];
  float4 o[RM][NC];
#pragma unroll
  for (int i = 0; i < RM; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int j = 0; j < NC; ++j) o[i][j] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  auto load_k = [&](int key) { load_tile<FMT, D, D + 4>(&sh.k[0][0], a.k, a.k_scale, a, w.head, pr.row0 + key, max(0, min(kBN, key1 - key))); };
  auto load_v = [&](int key) { load_tile<FMT, D, D>(&sh.v[0][0], a.v, a.v_scale, a, w.head, pr.row0 + key, max(0, min(kBN, key1 - key))); };
  if (key0 < key1) {
    load_k(key0);
    load_v(key0);
  }
  // A warp without rows only copies (32 sequences behind a prefix of 4096: 126 -> 102 us; full tiles 2 % slower).
  const bool works = (int)(threadIdx.x >> 5) * 2 * RM < n_rows;
  for (int key = key0; key < key1; key += kBN) {
    cp_wait<1>();  // K of this tile (V's copies may still be under way)
    __syncthreads();
    if (works) {
      float s[RM][kJ];
#pragma unroll
      for (int i = 0; i < RM; ++i)
#pragma unroll
        for (int j = 0; j < kJ; ++j) s[i][j] = 0.f;
#pragma unroll 4
      for (int c = 0; c < D; c += 4) {
        float4 kk[kJ];
#pragma unroll
        for (int j = 0; j < kJ; ++j) kk[j] = *reinterpret_cast<const float4*>(&sh.k[x + 16 * j][c]);
#pragma unroll
        for (int i = 0; i < RM; ++i) {
          const float4 qq = *reinterpret_cast<const float4*>(&sh.q[y * RM + i][c]);
#pragma unroll
          for (int j = 0; j < kJ; ++j) {
            s[i][j] = fmaf(qq.x, kk[j].x, s[i][j]);
            s[i][j] = fmaf(qq.y, kk[j].y, s[i][j]);
            s[i][j] = fmaf(qq.z, kk[j].z, s[i][j]);
            s[i][j] = fmaf(qq.w, kk[j].w, s[i][j]);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < RM; ++i) {
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < kJ; ++j) {
          const int kx = key + x + 16 * j;
          s[i][j] = kx < seen[i] && kx < key1 ? s[i][j] * a.scale2 : -INFINITY;
          top = fmaxf(top, s[i][j]);
        }
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        const float mn = fmaxf(m[i], top);
        const float base = mn == -INFINITY ? 0.f : mn;  // nothing seen so far: every exponential is 0
        const float alpha = exp2f(m[i] - base);
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < kJ; ++j) {
          const float p = exp2f(s[i][j] - base);
          sum += p;
          sh.p[y * RM + i][x + 16 * j] = p;
        }
        l[i] = l[i] * alpha + sum;
        m[i] = mn;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
          o[i][j].x *= alpha;
          o[i][j].y *= alpha;
          o[i][j].z *= alpha;
          o[i][j].w *= alpha;
        }
      }
    }
    cp_wait<0>();
    __syncthreads();  // V is there, K has been read
    if (key + kBN < key1) load_k(key + kBN);
    if (works) {
#pragma unroll 2
      for (int kk = 0; kk < kBN; kk += 4) {
        float4 pp[RM];
#pragma unroll
        for (int i = 0; i < RM; ++i) pp[i] = *reinterpret_cast<const float4*>(&sh.p[y * RM + i][kk]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
#pragma unroll
          for (int j = 0; j < NC; ++j) {
            const float4 vv = *reinterpret_cast<const float4*>(&sh.v[kk + e][4 * x + 64 * j]);
#pragma unroll
            for (int i = 0; i < RM; ++i) {
              const float p = e == 0 ? pp[i].x : e == 1 ? pp[i].y : e == 2 ? pp[i].z : pp[i].w;
              o[i][j].x = fmaf(p, vv.x, o[i][j].x);
              o[i][j].y = fmaf(p, vv.y, o[i][j].y);
              o[i][j].z = fmaf(p, vv.z, o[i][j].z);
              o[i][j].w = fmaf(p, vv.w, o[i][j].w);
            }
          }
        }
      }
    }
    __syncthreads();  // V has been read
    if (key + kBN < key1) load_v(key + kBN);
  }
#pragma unroll
  for (int i = 0; i < RM; ++i) {
    float sum = l[i];
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    const int r = y * RM + i;
    if (r >= n_rows) continue;
    const int tok = (r0 + r) / a.group;
    const int64_t token = pr.t0 + tok;
    const int hq = w.head * a.group + (r0 + r) - tok * a.group;
    if (!token_ok(a, token, hq)) continue;
    const bool none = sum == 0.f;
    const float inv = none ? 0.f : 1.f / sum;
    const float lse2 = none ? -INFINITY : m[i] + log2f(sum);
    if (direct) {
      float* to = static_cast<float*>(a.out) + token * a.out_stride + (int64_t)hq * D;
#pragma unroll
      for (int j = 0; j < NC; ++j)
        store4(to + 4 * x + 64 * j, make_float4(o[i][j].x * inv, o[i][j].y * inv, o[i][j].z * inv, o[i][j].w * inv));
      if (a.lse && x == 0) a.lse[token * a.heads * a.group + hq] = lse2 * 0.6931471805599453f;
    } else {
      const int64_t at = ((int64_t)(part.slot0 + w.split) * a.q_rows + token) * a.heads * a.group + hq;
      if (!partial_ok(a, at)) continue;
#pragma unroll
      for (int j = 0; j < NC; ++j)
        store4(a.part_out + at * D + 4 * x + 64 * j, make_float4(o[i][j].x * inv, o[i][j].y * inv, o[i][j].z * inv, o[i][j].w * inv));
      if (x == 0) a.part_lse[at] = lse2;
    }
  }
}

// Up to R query rows: bound by reading K and V once.  Four warps take 8 or 16 keys of the block's chunk in turn, straight
// from memory into registers: a lane has four channels of a key (D = 128: a warp one key to a load, D = 64: two).  The 8
// partial dot products of a lane become sums over the key's lanes by halving exchanges (9 or 8 shuffles instead of
// 8 x 5), which leaves every key's logit with a few lanes; the probabilities go back by one shuffle per key.  K and V of a
// step are asked for together, 16 vectors a lane: 16 warps keep 128 KB of an SM under way.
constexpr int kFewThreads = 128, kFewWarps = 4, kLoads = 8;

template <int FMT, int D>
__device__ __forceinline__ float4 load_row4(const void* base, const uint8_t* scale, const AttendView& a, int head, int64_t row, int c) {
  if (!row_ok(a, head, row)) return make_float4(0.f, 0.f, 0.f, 0.f);
  if constexpr (FMT == H2O_F32) {
    return __ldcs(reinterpret_cast<const float4*>(static_cast<const float*>(base) + row * a.row_stride + (int64_t)head * D + c));
  } else {
    const int64_t at = (int64_t)head * a.rows + row;
    const uint32_t w = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(base) + at * D + c);
    const float s = kv8_scale(scale[at]);
    return make_float4(e4m3(w & 255u) * s, e4m3((w >> 8) & 255u) * s, e4m3((w >> 16) & 255u) * s, e4m3(w >> 24) * s);
  }
}

template <int FMT, int D, int R>
__global__ void __launch_bounds__(kFewThreads) attend_few_kernel(const __grid_constant__ AttendView a, int part_index) {
  constexpr int kLanes = D / 4, kPer = 32 / kLanes, kKeys = kLoads * kPer;  // lanes of a key, keys of a load, of a step
  __shared__ float sh_m[kFewWarps][R], sh_l[kFewWarps][R];
  __shared__ __align__(16) float sh_o[kFewWarps][R][D];
  const AttendPart& part = a.part[part_index];
  const BlockWork w = block_work(a, part, blockIdx.x);
  const Problem pr = locate(a, part, w.problem);
  const int rows = pr.nt * a.group, r0 = w.row_tile * R;
  if (r0 >= rows) return;
  const int n_rows = min(R, rows - r0);
  const int key0 = w.split * part.chunk;
  const bool direct = a.part_out == nullptr;
  if (!direct && key0 >= pr.len) return;  // (the join kernel does not read it)
  const int key1 = min(seen_rows(part, pr, (r0 + n_rows - 1) / a.group), key0 + part.chunk);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int c = lane % kLanes * 4, sub = lane / kLanes;  // the lane's channels, its key of a load

  float4 q[R];
  int seen[R];
  float m[R], l[R];
  float4 o[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const bool there = r < n_rows;
    const int tok = there ? (r0 + r) / a.group : 0;
    const int64_t hq = (int64_t)w.head * a.group + (there ? r0 + r - tok * a.group : 0);
    q[r] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (token_ok(a, pr.t0 + tok, (int)hq))
      q[r] = *reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + (pr.t0 + tok) * a.q_stride + hq * D + c);
    seen[r] = there ? min(key1, seen_rows(part, pr, tok)) : 0;
    m[r] = -INFINITY;
    l[r] = 0.f;
    o[r] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  // the key of a step whose logit this lane ends up with (a few lanes the same one)
  const int mine = kPer == 1 ? lane >> 2 : 2 * ((lane >> 1) & 7) + (lane >> 4);
  for (int key = key0 + warp * kKeys; key < key1; key += kFewWarps * kKeys) {
    float4 kk[kLoads], vv[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int x = key + i * kPer + sub;
      const bool there = x < key1;  // (what lies behind the range may be anything)
      kk[i] = there ? load_row4<FMT, D>(a.k, a.k_scale, a, w.head, pr.row0 + x, c) : make_float4(0.f, 0.f, 0.f, 0.f);
      vv[i] = there ? load_row4<FMT, D>(a.v, a.v_scale, a, w.head, pr.row0 + x, c) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    float s[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float d[kLoads];
#pragma unroll
      for (int i = 0; i < kLoads; ++i) d[i] = fmaf(q[r].w, kk[i].w, fmaf(q[r].z, kk[i].z, fmaf(q[r].y, kk[i].y, q[r].x * kk[i].x)));
      // a lane keeps the half of its values that its bit names and gives the other half away
      int bit = kLanes / 2;
#pragma unroll
      for (int n = kLoads / 2; n > 0; n >>= 1, bit >>= 1) {
        const bool upper = (lane & bit) != 0;
#pragma unroll
        for (int i = 0; i < n; ++i) {
          const float give = upper ? d[i] : d[i + n], keep = upper ? d[i + n] : d[i];
          d[i] = keep + __shfl_xor_sync(0xffffffffu, give, bit);
        }
      }
#pragma unroll
      for (; bit > 0; bit >>= 1) d[0] += __shfl_xor_sync(0xffffffffu, d[0], bit);
      s[r] = key + mine < seen[r] ? d[0] * a.scale2 : -INFINITY;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (__any_sync(0xffffffffu, s[r] > m[r] + 8.f)) {  // the reference maximum follows lazily
        const float mn = fmaxf(m[r], warp_max(s[r]));
        const float alpha = mn == -INFINITY ? 1.f : exp2f(m[r] - mn);
        m[r] = mn;
        l[r] *= alpha;
        o[r].x *= alpha;
        o[r].y *= alpha;
        o[r].z *= alpha;
        o[r].w *= alpha;
      }
      const float p = exp2f(s[r] - (m[r] == -INFINITY ? 0.f : m[r]));
      l[r] += p;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const float pi = __shfl_sync(0xffffffffu, p, kPer == 1 ? 4 * i : 16 * sub + 2 * i);
        o[r].x = fmaf(pi, vv[i].x, o[r].x);
        o[r].y = fmaf(pi, vv[i].y, o[r].y);
        o[r].z = fmaf(pi, vv[i].z, o[r].z);
        o[r].w = fmaf(pi, vv[i].w, o[r].w);
      }
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const float sum = warp_sum(l[r]) * (kKeys / 32.f);  // (32 / kKeys lanes have counted each key)
    if (kPer == 2) {
      o[r].x += __shfl_xor_sync(0xffffffffu, o[r].x, 16);
      o[r].y += __shfl_xor_sync(0xffffffffu, o[r].y, 16);
      o[r].z += __shfl_xor_sync(0xffffffffu, o[r].z, 16);
      o[r].w += __shfl_xor_sync(0xffffffffu, o[r].w, 16);
    }
    if (sub == 0) store4(&sh_o[warp][r][c], o[r]);
    if (lane == 0) {
      sh_m[warp][r] = m[r];
      sh_l[warp][r] = sum;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n_rows * kLanes; i += kFewThreads) {
    const int r = i / kLanes, cc = i % kLanes * 4;
    float top = -INFINITY;
#pragma unroll
    for (int x = 0; x < kFewWarps; ++x) top = fmaxf(top, sh_m[x][r]);
    const float base = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int x = 0; x < kFewWarps; ++x) {
      const float wgt = exp2f(sh_m[x][r] - base);
      const float4 y = *reinterpret_cast<const float4*>(&sh_o[x][r][cc]);
      sum += wgt * sh_l[x][r];
      v.x = fmaf(wgt, y.x, v.x);
      v.y = fmaf(wgt, y.y, v.y);
      v.z = fmaf(wgt, y.z, v.z);
      v.w = fmaf(wgt, y.w, v.w);
    }
    const bool none = sum == 0.f;
    const float inv = none ? 0.f : 1.f / sum;
    const float lse2 = none ? -INFINITY : top + log2f(sum);
    v = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
    const int tok = (r0 + r) / a.group;
    const int64_t token = pr.t0 + tok;
    const int hq = w.head * a.group + (r0 + r) - tok * a.group;
    if (!token_ok(a, token, hq)) continue;
    if (direct) {
      store4(static_cast<float*>(a.out) + token * a.out_stride + (int64_t)hq * D + cc, v);
      if (a.lse && cc == 0) a.lse[token * a.heads * a.group + hq] = lse2 * 0.6931471805599453f;
    } else {
      const int64_t at = ((int64_t)(part.slot0 + w.split) * a.q_rows + token) * a.heads * a.group + hq;
      if (!partial_ok(a, at)) continue;
      store4(a.part_out + at * D + cc, v);
      if (cc == 0) a.part_lse[at] = lse2;
    }
  }
}

template <int FMT, int D, int R>
cudaError_t launch_few(const AttendView& a, int part, cudaStream_t stream) {
  attend_few_kernel<FMT, D, R><<<(unsigned)part_blocks(a, a.part[part]), kFewThreads, 0, stream>>>(a, part);
  return cudaGetLastError();
}
template <int FMT, int D, int BM>
cudaError_t launch(const AttendView& a, int part, cudaStream_t stream) {
  constexpr int smem = (int)sizeof(Smem<D, BM>);
  static unsigned long long flags = 0;
  const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(attend_fma_kernel<FMT, D, BM>), smem, &flags);
  if (e != cudaSuccess) return e;
  attend_fma_kernel<FMT, D, BM><<<(unsigned)part_blocks(a, a.part[part]), kThreads, smem, stream>>>(a, part);
  return cudaGetLastError();
}
template <int FMT, int D>
cudaError_t launch_shape(const AttendView& a, int part, int tile, cudaStream_t stream) {
  switch (tile) {
    case 1: return launch_few<FMT, D, 1>(a, part, stream);
    case 2: return launch_few<FMT, D, 2>(a, part, stream);
    case 4: return launch_few<FMT, D, 4>(a, part, stream);
    case 16: return launch<FMT, D, 16>(a, part, stream);
    default: return launch<FMT, D, 64>(a, part, stream);
  }
}

}  // namespace

// Rows of a tile for problems of up to `rows` rows: 1, 2 or 4 in the kernel for few; else 16 or 64 (fewer rows make more
// shared-memory loads per product: 131 query tokens, 515 keys, 16 heads ran in 24.4 us in tiles of 16, 22.7 in tiles of 64).
int attend_fma_row_tile(int64_t rows) { return rows <= 2 ? (int)rows : rows <= 4 ? 4 : rows <= 16 ? 16 : 64; }

cudaError_t launch_attend_fma(const AttendView& a, int part, int tile, int format, cudaStream_t stream) {
  if (format == H2O_F32) return a.dim == 128 ? launch_shape<H2O_F32, 128>(a, part, tile, stream) : launch_shape<H2O_F32, 64>(a, part, tile, stream);
  return a.dim == 128 ? launch_shape<H2O_KV8, 128>(a, part, tile, stream) : launch_shape<H2O_KV8, 64>(a, part, tile, stream);
}

}  // namespace h2o
