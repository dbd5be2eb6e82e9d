// Probabilities of plain or fused rows: p_v = exp(z_v - m) / sum exp(z - m), z = l / T.
// A CTA takes a row: its largest value, its sum, then the probabilities.
#include <cuda_bf16.h>

#include "row_stream.cuh"

namespace dels {
namespace {

__device__ __forceinline__ void put(float* out, float x) { __stcs(out, x); }
__device__ __forceinline__ void put(uint16_t* out, float x) {
  __stcs(reinterpret_cast<unsigned short*>(out), __bfloat16_as_ushort(__float2bfloat16_rn(x)));
}

template <typename T, int F, bool VEC, typename O>
__global__ void __launch_bounds__(kStreamThreads) k_row_probs(const ProbsArgs a) {
  __shared__ float red[kStreamWarps];
  const int tid = threadIdx.x;
  const unsigned r = blockIdx.x;
  pdl_wait();
  if (tid == 0) pdl_trigger();
  const FusedRow<T, F, false> row(a.in, r);
  O* out = static_cast<O*>(a.out) + (long long)r * a.ld_out;
  const int V = a.in.V;
  float m = -INFINITY, nan = 0.f;
  for (int v = tid; v < V; v += kStreamThreads) {
    const float x = row.contracted(row.l_at(v), row.s_at(v), row.p_at(v));
    m = fmaxf(m, x);
    nan += x != x ? 1.f : 0.f;
  }
  m = warp_max(m);
  if ((tid & 31) == 0) red[tid >> 5] = m;
  __syncthreads();
  for (int i = 0; i < kStreamWarps; ++i) m = fmaxf(m, red[i]);
  float s = 0.f;
  for (int v = tid; v < V; v += kStreamThreads) {
    const float x = row.contracted(row.l_at(v), row.s_at(v), row.p_at(v));
    s += ex2_approx((x - m) * a.in.scale);
  }
  s = block_sum(s);
  const bool ok = block_sum(nan) == 0.f && m > -INFINITY && m < INFINITY && s > 0.f && s < INFINITY;
  if (!ok && tid == 0) raise_status(a.status, DELS_STATUS_NONFINITE);
  const float inv = ok ? 1.f / s : NAN;
  for (int v = tid; v < V; v += kStreamThreads) {
    const float x = row.contracted(row.l_at(v), row.s_at(v), row.p_at(v));
    put(out + v, ex2_approx((x - m) * a.in.scale) * inv);
  }
}

}  // namespace

cudaError_t launch_row_probs(const ProbsArgs& a, bool f32, bool fused, bool vec, cudaStream_t s) {
  return dispatch_rows(a.in, f32, fused, vec, [&](auto type, auto terms, auto v) {
    using T = typename decltype(type)::type;
    constexpr int F = decltype(terms)::value;
    constexpr bool VEC = decltype(v)::value;
    return a.out_f32 ? launch_pdl(k_row_probs<T, F, VEC, float>, dim3(a.in.rows), dim3(kStreamThreads), 0, s, a)
                     : launch_pdl(k_row_probs<T, F, VEC, uint16_t>, dim3(a.in.rows), dim3(kStreamThreads), 0, s, a);
  });
}

}  // namespace dels
