// Rows of (fused) vocabulary logits as the scoring and distillation kernels
// stream them: one cluster of 1 to 16 CTAs takes a row, every CTA a slice of its
// columns, every thread items of 8 columns; the slices' sums meet in distributed
// shared memory, so that a call is one launch without scratch in memory.
#pragma once

#include "dels_device.cuh"

namespace dels {

constexpr int kStreamThreads = 512;
constexpr int kStreamWarps = kStreamThreads / 32;
constexpr int kStreamStep = kStreamThreads * 8;    // columns of one item per thread
constexpr int kMaxCluster = 16;

__device__ __forceinline__ float row_elem(const float* p, long long i) { return __ldg(p + i); }
__device__ __forceinline__ float row_elem(const uint16_t* p, long long i) { return bf16_to_f(__ldg(p + i)); }

// 8 consecutive elements from a 16-byte aligned address (streamed: read once).
__device__ __forceinline__ void row_vec(const float* p, float (&x)[8]) {
  const float4 a = __ldcs(reinterpret_cast<const float4*>(p));
  const float4 b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void row_vec(const uint16_t* p, float (&x)[8]) {
  const uint4 w = __ldcs(reinterpret_cast<const uint4*>(p));
  x[0] = bf16lo(w.x); x[1] = bf16hi(w.x); x[2] = bf16lo(w.y); x[3] = bf16hi(w.y);
  x[4] = bf16lo(w.z); x[5] = bf16hi(w.z); x[6] = bf16lo(w.w); x[7] = bf16hi(w.w);
}

// One row of l = (l_L + alpha l_S) - beta l_P, rounded to float32 after every
// operation (no contraction), so that equal inputs order equally wherever they
// are evaluated; an absent term counts as zero. FUSED = false: l = l_L as stored.
template <typename T, bool FUSED>
struct FusedRow {
  const T* L;          // FUSED: may be null
  const T* S;          // FUSED only, may be null
  const float* P;      // FUSED only, may be null
  float a, b;

  __device__ __forceinline__ FusedRow(const StreamRows& in, long long row) {
    L = in.longp ? static_cast<const T*>(in.longp) + row * in.ld_long : nullptr;
    S = nullptr;
    P = nullptr;
    a = b = 1.f;
    if constexpr (FUSED) {
      const int j = (int)(row % in.n_weights);
      if (in.shortp) {
        S = static_cast<const T*>(in.shortp) + row * in.ld_short;
        if (in.alpha) a = __ldg(in.alpha + j);
      }
      if (in.prior) {
        P = in.prior;
        if (in.beta) b = __ldg(in.beta + j);
      }
    }
  }
  __device__ __forceinline__ float combine(float l, float s, float p) const {
    return FUSED ? __fsub_rn(__fadd_rn(l, __fmul_rn(a, s)), __fmul_rn(b, p)) : l;
  }
  __device__ __forceinline__ float s_at(int c) const { return FUSED && S ? row_elem(S, c) : 0.f; }
  __device__ __forceinline__ float p_at(int c) const { return FUSED && P ? __ldg(P + c) : 0.f; }
  __device__ __forceinline__ float at(int c) const {
    if constexpr (!FUSED) return row_elem(L, c);
    return combine(L ? row_elem(L, c) : 0.f, s_at(c), p_at(c));
  }
  // The terms of 8 columns. VEC: c .. c + 7 of 16-byte aligned rows; otherwise
  // c + i * kStreamThreads (a warp's lanes side by side). Columns from `end` on
  // (CHECK) read as l = -inf.
  template <bool VEC, bool CHECK>
  __device__ __forceinline__ void load(int c, int end, float (&l)[8], float (&s)[8], float (&p)[8]) const {
    if (VEC && (!CHECK || c + 8 <= end)) {
      if (!FUSED || L) row_vec(L + c, l);
      else
#pragma unroll
        for (int i = 0; i < 8; ++i) l[i] = 0.f;
      if constexpr (FUSED) {
        if (S) row_vec(S + c, s);
        else
#pragma unroll
          for (int i = 0; i < 8; ++i) s[i] = 0.f;
        if (P) {
          const float4 u = __ldg(reinterpret_cast<const float4*>(P + c));
          const float4 v = __ldg(reinterpret_cast<const float4*>(P + c) + 1);
          p[0] = u.x; p[1] = u.y; p[2] = u.z; p[3] = u.w; p[4] = v.x; p[5] = v.y; p[6] = v.z; p[7] = v.w;
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) p[i] = 0.f;
        }
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int k = VEC ? c + i : c + i * kStreamThreads;
      const bool in = !CHECK || k < end;
      l[i] = in ? (!FUSED || L ? row_elem(L, k) : 0.f) : -INFINITY;
      if constexpr (FUSED) {
        s[i] = in ? s_at(k) : 0.f;
        p[i] = in ? p_at(k) : 0.f;
      }
    }
  }
};

// First column of item `it` of thread t in a slice that starts at c0.
template <bool VEC>
__device__ __forceinline__ int item_col(int c0, int it, int t) {
  return VEC ? c0 + it * kStreamStep + t * 8 : c0 + it * kStreamStep + t;
}
// Column i of an item.
template <bool VEC>
__device__ __forceinline__ int elem_col(int c, int i) { return VEC ? c + i : c + i * kStreamThreads; }

// ---------------------------------------------------------------------------
// Running softmax sums. With t = (x - m) log2(e) / T, m the largest entry so far:
//   rest = sum 2^t without one entry that attains m (it is 1: held out, so that
//          ln(1 + rest) keeps its digits where one entry has nearly all mass),
//   w    = sum 2^t t over the same entries (both of one sign: the entropy
//          ln S - ln2 w / S has no cancellation).
// ---------------------------------------------------------------------------
struct SoftRec {
  float m, rest, w;
};
constexpr float kLowT = -1e30f;   // 2^t t is 0 from here on, -inf included

__device__ __forceinline__ SoftRec softrec_init() { return SoftRec{-INFINITY, 0.f, 0.f}; }

// b's sums relative to M >= b.m, its held-out entry among them unless it stays out.
__device__ __forceinline__ void softrec_add(SoftRec& r, const SoftRec& b, float M, float c, bool stays_out) {
  const float d = b.m == -INFINITY ? 0.f : fmaxf((b.m - M) * c, kLowT);
  const float f = b.m == -INFINITY ? (b.rest != b.rest ? NAN : 0.f) : ex2_approx(d);
  const float out = b.m == -INFINITY || stays_out ? 0.f : f;
  r.rest += f * b.rest + out;
  r.w += f * (b.w + d * b.rest) + out * d;
}
__device__ __forceinline__ SoftRec softrec_merge(const SoftRec& a, const SoftRec& b, float c) {
  SoftRec r{fmaxf(a.m, b.m), 0.f, 0.f};
  const bool a_out = a.m >= b.m;
  softrec_add(r, a, r.m, c, a_out);
  softrec_add(r, b, r.m, c, !a_out);
  return r;
}
__device__ __forceinline__ bool softrec_valid(const SoftRec& r) {
  return r.m > -INFINITY && r.m < INFINITY && r.rest >= 0.f && r.rest < INFINITY;
}

// One lane's sums under its warp's reference (the warp's largest entry so far),
// in which the lane that holds an entry equal to it keeps that entry out.
struct WarpSoft {
  float ref, off;      // the same in every lane; off = ref, or 0 while ref is -inf
  float rest, w;
  bool holds;
  __device__ __forceinline__ void init() {
    ref = -INFINITY;
    off = rest = w = 0.f;
    holds = false;
  }
  // A warp's new largest entry: the sums move to it. Returns the factor they
  // were scaled by (all lanes converged).
  __device__ __forceinline__ float move(float top, float c) {
    const float d = ref == -INFINITY ? 0.f : fmaxf((ref - top) * c, kLowT);
    const float f = ref == -INFINITY ? (rest != rest ? NAN : 0.f) : ex2_approx(d);
    w = f * (w + d * rest);
    rest *= f;
    if (holds) {
      rest += f;
      w += f * d;
    }
    holds = false;
    ref = off = top;
    return f;
  }
  // The warp's record (all lanes converged), in every lane.
  __device__ __forceinline__ SoftRec record() const {
    SoftRec r{ref, rest, w};
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      r.rest += __shfl_xor_sync(0xFFFFFFFFu, r.rest, d);
      r.w += __shfl_xor_sync(0xFFFFFFFFu, r.w, d);
    }
    return r;
  }
};

// Largest of 8 values (NaN ignored).
__device__ __forceinline__ float max8(const float (&x)[8]) {
  return fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
}

// Cluster barrier of C CTAs; one CTA alone takes its own barrier.
__device__ __forceinline__ void cluster_or_cta_sync(int C) {
  if (C > 1) cluster_sync_all();
  else __syncthreads();
}

}  // namespace dels
