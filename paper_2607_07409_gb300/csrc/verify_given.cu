// Speculative sampling from given probabilities and uniforms. A CTA takes a request: its
// first warp finds the tokens kept, then all threads sum the weights that the bonus token
// is drawn from, each a run of columns, in float64; the thread whose run has the border
// walks it.
#include "dels_device.cuh"

namespace dels {
namespace {

constexpr int kGivenThreads = 256;

__device__ __forceinline__ float given_at(const GivenRows& g, long long i) {
  return g.f32 ? __ldg(static_cast<const float*>(g.p) + i) : bf16_to_f(__ldg(static_cast<const uint16_t*>(g.p) + i));
}
__device__ __forceinline__ bool is_probability(float x) { return x >= 0.f && x < INFINITY; }

// What request b keeps, and what its bonus token is drawn from.
struct Kept {
  int a;
  int token;           // the rejected one, or -1: all were kept
  int code;            // status bits
};
__device__ Kept count_kept(const VerifyGivenArgs& a, int b) {
  Kept k{0, -1, 0};
  const int len = a.lengths ? a.lengths[b] : a.n;
  const float last = a.uniforms[(long long)b * (a.n + 1) + a.n];
  if (len < 0 || len > a.n || !(last >= 0.f && last < 1.f)) {
    k.code = DELS_STATUS_BAD_VALUE;
    return k;
  }
  for (; k.a < len; ++k.a) {
    const int x = a.tokens[(long long)b * a.n + k.a];
    const float u = a.uniforms[(long long)b * (a.n + 1) + k.a];
    if (x < 0 || x >= a.V) k.code |= DELS_STATUS_BAD_TOKEN;
    if (!(u >= 0.f && u < 1.f)) k.code |= DELS_STATUS_BAD_VALUE;
    if (k.code) return k;
    const float p = given_at(a.target, b * a.target.ld_b + k.a * a.target.ld + x);
    const float q = a.draft.p ? given_at(a.draft, b * a.draft.ld_b + k.a * a.draft.ld + x) : 1.f;
    if (!is_probability(p) || !is_probability(q)) k.code = DELS_STATUS_NONFINITE;
    if (k.code) return k;
    if (!((double)u * (double)q < (double)p)) {
      k.token = x;
      return k;
    }
  }
  return k;
}

__global__ void __launch_bounds__(kGivenThreads) k_verify_given(const VerifyGivenArgs a) {
  __shared__ double sums[kGivenThreads];
  __shared__ Kept kept;
  __shared__ int bad;
  const int tid = threadIdx.x, b = blockIdx.x;
  pdl_wait();
  if (tid == 0) {
    pdl_trigger();
    kept = count_kept(a, b);
    bad = 0;
  }
  __syncthreads();
  const Kept k = kept;
  const long long p0 = b * a.target.ld_b + k.a * a.target.ld, q0 = b * a.draft.ld_b + k.a * a.draft.ld;
  const int run = (a.V + kGivenThreads - 1) / kGivenThreads;
  const int v0 = min(a.V, tid * run), v1 = min(a.V, v0 + run);
  bool rest = k.token >= 0;          // from max(0, p - q)
  const auto weight = [&](int v) {
    const double p = given_at(a.target, p0 + v);
    if (!rest) return p;
    if (!a.draft.p) return v == k.token ? 0.0 : p;
    return fmax(0.0, p - (double)given_at(a.draft, q0 + v));
  };
  int bonus = -1, code = k.code;
  if (!code) {
    for (int v = v0; v < v1; ++v)
      if (!is_probability(given_at(a.target, p0 + v)) ||
          (rest && a.draft.p && !is_probability(given_at(a.draft, q0 + v))))
        bad = 1;
    for (int pass = 0; pass < 2; ++pass) {
      double s = 0.0;
      for (int v = v0; v < v1; ++v) s += weight(v);
      __syncthreads();
      sums[tid] = s;
      __syncthreads();
      double total = 0.0, before = 0.0;
      for (int i = 0; i < kGivenThreads; ++i) {
        if (i == tid) before = total;
        total += sums[i];
      }
      if (bad || total > 0.0 || !rest) {
        if (bad || !(total > 0.0)) {
          code = DELS_STATUS_NONFINITE;
          break;
        }
        const double at = (double)a.uniforms[(long long)b * (a.n + 1) + a.n] * total;
        if (before <= at && before + s > at) {
          double c = before;
          for (int v = v0; v < v1; ++v) {
            const double w = weight(v);
            c += w;
            if (w > 0.0) bonus = v;
            if (c > at) break;
          }
          a.out_bonus[b] = bonus;
        }
        break;
      }
      rest = false;
    }
  }
  if (tid == 0) {
    a.out_accept[b] = k.a;
    if (code) {
      a.out_bonus[b] = -1;
      raise_status(a.status, code);
    }
  }
}

}  // namespace

cudaError_t launch_verify_given(const VerifyGivenArgs& a, cudaStream_t s) {
  return launch_pdl(k_verify_given, dim3(a.B), dim3(kGivenThreads), 0, s, a);
}

}  // namespace dels
