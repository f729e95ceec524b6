// Attention over a K/V store for float32 queries, on the fp32 FMA pipe (float32 or 8-bit rows, head_dim 64 and 128).
//
// A block takes BM query rows (query tokens times the query heads of one K/V head) and walks over its keys 64 at a
// time: S = Q K^T by register tiles, softmax with the running maximum and sum of each row, O += P V.
// 256 threads as 16 x 16: thread (x, y) has rows y * RM .. + RM - 1, keys x + 16 j of a tile, output columns
// 4 x + 64 j .. + 3, so a row's statistics are shuffles within 16 lanes and its probabilities pass between them
// through shared memory without a block barrier.  K of the next tile is fetched (cp.async, float32 rows) during
// P V, V during the next S.  Bound by shared memory: 8 vector loads (32 wavefronts) feed 64 multiply-adds of a warp.
// 4 x 512 queries against 2048 keys, 16 heads of 128: 630 us, 27 TFLOP/s.
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
      if (r < n) cp_async16(to, static_cast<const float*>(base) + (row0 + r) * a.row_stride + (int64_t)head * D + c);
      else *reinterpret_cast<float4*>(to) = make_float4(0.f, 0.f, 0.f, 0.f);
    }
  } else {
    constexpr int kV = D / 16;
    for (int i = threadIdx.x; i < kBN * kV; i += kThreads) {
      const int r = i / kV, c = (i % kV) * 16;
      uint4 w = make_uint4(0, 0, 0, 0);
      float s = 0.f;
      if (r < n) {
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
  for (int key = key0; key < key1; key += kBN) {
    cp_wait<1>();  // K of this tile (V's copies may still be under way)
    __syncthreads();
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
    cp_wait<0>();
    __syncthreads();  // V is there, K has been read
    if (key + kBN < key1) load_k(key + kBN);
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
#pragma unroll
      for (int j = 0; j < NC; ++j)
        store4(a.part_out + at * D + 4 * x + 64 * j, make_float4(o[i][j].x * inv, o[i][j].y * inv, o[i][j].z * inv, o[i][j].w * inv));
      if (x == 0) a.part_lse[at] = lse2;
    }
  }
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
template <int FMT>
cudaError_t launch_shape(const AttendView& a, int part, int tile, cudaStream_t stream) {
  if (a.dim == 128) return tile == 16 ? launch<FMT, 128, 16>(a, part, stream) : launch<FMT, 128, 64>(a, part, stream);
  return tile == 16 ? launch<FMT, 64, 16>(a, part, stream) : launch<FMT, 64, 64>(a, part, stream);
}

}  // namespace

// Rows of a tile for `problems` problems of up to `rows` rows: 64, whose products are bound by the FMA pipe, where that
// makes blocks enough to fill the device, else 16 (131 query tokens, 515 keys, 16 heads of two sequences: 22.8 -> 8.8 us).
int attend_fma_row_tile(int64_t rows, int64_t problems) { return (rows + 63) / 64 * problems < 2 * sm_count() ? 16 : 64; }

cudaError_t launch_attend_fma(const AttendView& a, int part, int tile, int format, cudaStream_t stream) {
  return format == H2O_F32 ? launch_shape<H2O_F32>(a, part, tile, stream) : launch_shape<H2O_KV8>(a, part, tile, stream);
}

}  // namespace h2o
