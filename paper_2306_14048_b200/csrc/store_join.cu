// Joins the chunks of split attention over a K/V store.
//
// A chunk i of a query row has left its normalised output o_i and the base-2 logarithm L_i of its sum of exponentials;
// the row's output is sum w_i o_i / sum w_i with w_i = 2^(L_i - max L), in the fixed order of the chunks.  One warp per
// row: the lanes read the logarithms of up to 32 chunks at once, then all of them take the same chunk, a few loads ahead.
#include "store.cuh"

namespace h2o {

namespace {

constexpr int kMaxSlots = 2 * kMaxSplits;  // two parts

template <typename T, int D>
__global__ void __launch_bounds__(256) attend_join_kernel(const __grid_constant__ AttendView a) {
  constexpr int kPer = D / 32;
  const int seq = blockIdx.y;
  const int lane = threadIdx.x & 31;
  const int hq_all = a.heads * a.group;
  const int64_t item = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int64_t t0 = first_token(a, seq);
  const int nt = (int)clamp64(first_token(a, seq + 1) - t0, 0, a.max_q);
  const int i = (int)(item / hq_all), hq = (int)(item - (int64_t)i * hq_all);
  bool live = i < nt;
  const int64_t token = t0 + i;
  // chunks of this row: for each part, the first and how many were written
  int slot[2] = {0, 0}, used[2] = {0, 0};
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (k >= a.n_parts || !live) break;
    const AttendPart& p = a.part[k];
    const int which = p.grouped ? group_of(a, seq) : seq;
    const Problem pr = locate(a, p, which);
    if (token < pr.t0 || token >= pr.t0 + pr.nt) live = false;  // beyond what the caller allowed for: left as it was
    slot[k] = p.slot0;
    used[k] = (pr.len + p.chunk - 1) / p.chunk;
  }
  // (Launched while the kernels that leave the chunks may still run: what does not depend on them is looked up before.  All
  // wait, so that this kernel never ends before them.)
  wait_for_earlier();
  if (!live || !token_ok(a, token, hq)) return;
  const int n = used[0] + used[1];
  const int64_t pitch = a.q_rows * hq_all, at = token * hq_all + hq;
  auto place = [&](int s) { return (int64_t)(s < used[0] ? slot[0] + s : slot[1] + s - used[0]) * pitch + at; };
  float lse[kMaxSlots / 32], top = -INFINITY;
#pragma unroll
  for (int k = 0; k < kMaxSlots / 32; ++k) {
    const int s = 32 * k + lane;
    lse[k] = s < n && partial_ok(a, place(s)) ? a.part_lse[place(s)] : -INFINITY;
    top = fmaxf(top, lse[k]);
  }
  top = warp_max(top);
  const float base = top == -INFINITY ? 0.f : top;
  float total = 0.f;
#pragma unroll
  for (int k = 0; k < kMaxSlots / 32; ++k) {
    lse[k] = exp2f(lse[k] - base);  // now the chunk's weight (0 for a chunk without a visible key, whose output is 0)
    total += lse[k];
  }
  total = warp_sum(total);
  float o[kPer];
#pragma unroll
  for (int e = 0; e < kPer; ++e) o[e] = 0.f;
#pragma unroll
  for (int k = 0; k < kMaxSlots / 32; ++k) {
    const int here = min(32, n - 32 * k);
#pragma unroll 4
    for (int s = 0; s < here; ++s) {
      const float w = __shfl_sync(0xffffffffu, lse[k], s);
      if (!partial_ok(a, place(32 * k + s))) continue;
      const float* from = a.part_out + place(32 * k + s) * D + lane * kPer;
      if constexpr (kPer == 4) {
        const float4 v = *reinterpret_cast<const float4*>(from);
        o[0] = fmaf(w, v.x, o[0]);
        o[1] = fmaf(w, v.y, o[1]);
        o[2] = fmaf(w, v.z, o[2]);
        o[3] = fmaf(w, v.w, o[3]);
      } else {
        const float2 v = *reinterpret_cast<const float2*>(from);
        o[0] = fmaf(w, v.x, o[0]);
        o[1] = fmaf(w, v.y, o[1]);
      }
    }
  }
  const float inv = total == 0.f ? 0.f : 1.f / total;
  T* to = static_cast<T*>(a.out) + token * a.out_stride + (int64_t)hq * D + lane * kPer;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int e = 0; e < kPer; ++e) to[e] = o[e] * inv;
  } else {
    uint32_t w[kPer / 2];
#pragma unroll
    for (int e = 0; e < kPer / 2; ++e) w[e] = Vec16<__nv_bfloat16>::pack2(o[2 * e] * inv, o[2 * e + 1] * inv);
    if constexpr (kPer == 4) *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(to) = w[0];
  }
  if (a.lse && lane == 0) a.lse[at] = total == 0.f ? -INFINITY : (top + log2f(total)) * 0.6931471805599453f;
}

template <typename T, int D>
cudaError_t launch(const AttendView& a, cudaStream_t stream) {
  const int64_t rows = (int64_t)a.max_q * a.heads * a.group;
  return launch_kernel(attend_join_kernel<T, D>, dim3((unsigned)((rows + 7) / 8), (unsigned)a.batch), 256, 0, stream, true, a);
}

}  // namespace

cudaError_t launch_attend_join(const AttendView& a, int q_dtype, cudaStream_t stream) {
  if (q_dtype == H2O_F32) return a.dim == 128 ? launch<float, 128>(a, stream) : launch<float, 64>(a, stream);
  return a.dim == 128 ? launch<__nv_bfloat16, 128>(a, stream) : launch<__nv_bfloat16, 64>(a, stream);
}

}  // namespace h2o
