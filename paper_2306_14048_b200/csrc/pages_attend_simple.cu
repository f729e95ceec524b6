// Attention over a paged K/V cache, the plain way: a warp has one query row and walks over the rows that it sees.
#include "pages.cuh"

namespace h2o {

namespace {

constexpr int kWarps = 4;

template <typename T, int D>
__global__ void __launch_bounds__(32 * kWarps) simple_kernel(const __grid_constant__ PagesAttend p) {
  constexpr int kPer = D / 32;
  const AttendView& a = p.a;
  const int lane = threadIdx.x & 31, seq = blockIdx.y;
  const int64_t item = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int hq_all = a.heads * a.group;
  const int64_t t0 = first_token(a, seq);
  const int nt = (int)clamp64(first_token(a, seq + 1) - t0, 0, a.max_q);
  const int i = (int)(item / hq_all), hq = (int)(item - (int64_t)i * hq_all), head = hq / a.group;
  if (i >= nt) return;
  const int64_t token = t0 + i;
  const int len = (int)clamp64(a.part[0].length[seq], 0, a.part[0].max_length);
  const int at = len - nt + i;
  float q[kPer], o[kPer], m = -INFINITY, l = 0.f;
  for (int e = 0; e < kPer; ++e) {
    q[e] = (float)static_cast<const T*>(a.q)[token * a.q_stride + (int64_t)hq * D + lane * kPer + e];
    o[e] = 0.f;
  }
  const int first = p.window > 0 ? max(0, at - p.window + 1) : 0;
  for (int x = 0; x <= at; ++x) {
    if (x >= p.sinks && x < first) x = first;
    const int page = p.table[seq * p.table_stride + x / p.page_size];
    float k[kPer], v[kPer], s = 0.f;
    for (int e = 0; e < kPer; ++e) {
      k[e] = v[e] = 0.f;
      if (page >= 0 && page < p.n_pages) {
        const int64_t from = page * p.page_stride + x % p.page_size * p.row_stride + head * p.head_stride + lane * kPer + e;
        k[e] = (float)static_cast<const T*>(a.k)[from];
        v[e] = (float)static_cast<const T*>(a.v)[from];
      }
      s = fmaf(q[e], k[e], s);
    }
    s = warp_sum(s) * a.scale2;
    const float mn = fmaxf(m, s), base = mn == -INFINITY ? 0.f : mn, alpha = exp2f(m - base), w = exp2f(s - base);
    l = l * alpha + w;
    m = mn;
    for (int e = 0; e < kPer; ++e) o[e] = fmaf(w, v[e], o[e] * alpha);
  }
  for (int e = 0; e < kPer; ++e)
    static_cast<T*>(a.out)[token * a.out_stride + (int64_t)hq * D + lane * kPer + e] = (T)(l == 0.f ? 0.f : o[e] / l);
  if (a.lse && lane == 0) a.lse[token * hq_all + hq] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

template <typename T, int D>
cudaError_t launch(const PagesAttend& p, cudaStream_t stream) {
  const int64_t rows = (int64_t)p.a.max_q * p.a.heads * p.a.group;
  simple_kernel<T, D><<<dim3((unsigned)((rows + kWarps - 1) / kWarps), (unsigned)p.a.batch), 32 * kWarps, 0, stream>>>(p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_pages_attend_simple(const PagesAttend& p, int dtype, cudaStream_t stream) {
  if (dtype == H2O_F32) return p.a.dim == 128 ? launch<float, 128>(p, stream) : launch<float, 64>(p, stream);
  return p.a.dim == 128 ? launch<__nv_bfloat16, 128>(p, stream) : launch<__nv_bfloat16, 64>(p, stream);
}

}  // namespace h2o
