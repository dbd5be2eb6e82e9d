// Rows of (fused) vocabulary logits as the scoring and distillation kernels
// stream them: one cluster of 1 to 8 CTAs takes a row, every CTA a slice of its
// columns, every thread items of 8 columns; the slices' sums meet in distributed
// shared memory, so that a call is one launch without scratch in memory.
#pragma once

#include <type_traits>

#include "dels_device.cuh"

namespace dels {

constexpr int kStreamThreads = 256;
constexpr int kStreamWarps = kStreamThreads / 32;
constexpr int kStreamStep = kStreamThreads * 8;    // columns of one item per thread
constexpr int kMaxCluster = 8;

// ---------------------------------------------------------------------------
// Pairs of float32 values for the packed arithmetic of sm_100 and later: one
// instruction for two roundings.
// ---------------------------------------------------------------------------
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair2(float lo, float hi) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ f32x2 both2(float x) { return pair2(x, x); }
__device__ __forceinline__ void split2(f32x2 v, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ float sum2(f32x2 v) {
  float lo, hi;
  split2(v, lo, hi);
  return lo + hi;
}

__device__ __forceinline__ float row_elem(const float* p, long long i) { return __ldg(p + i); }
__device__ __forceinline__ float row_elem(const uint16_t* p, long long i) { return bf16_to_f(__ldg(p + i)); }

// 8 elements as loaded: one 16-byte word of bf16, two of float32.
template <typename T>
struct Raw8 {
  static constexpr int W = sizeof(T) / 2;
  uint4 w[W];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int k = 0; k < W; ++k) w[k] = __ldcs(reinterpret_cast<const uint4*>(p) + k);
  }
  __device__ __forceinline__ void fill(float x) {
    const uint32_t b = __float_as_uint(x);         // 0 or -inf: exact in bf16
    const uint32_t v = sizeof(T) == 4 ? b : (b >> 16) * 0x00010001u;
#pragma unroll
    for (int k = 0; k < W; ++k) w[k] = make_uint4(v, v, v, v);
  }
  __device__ __forceinline__ void set(int i, float x) {      // x: an element of the type
    uint32_t* u = reinterpret_cast<uint32_t*>(w);
    if constexpr (sizeof(T) == 4) {
      u[i] = __float_as_uint(x);
    } else {
      const uint32_t h = __float_as_uint(x) >> 16;
      u[i >> 1] = i & 1 ? (u[i >> 1] & 0xFFFFu) | h << 16 : (u[i >> 1] & 0xFFFF0000u) | h;
    }
  }
  __device__ __forceinline__ void unpack(float (&x)[8]) const {
    if constexpr (sizeof(T) == 4) {
      x[0] = __uint_as_float(w[0].x); x[1] = __uint_as_float(w[0].y);
      x[2] = __uint_as_float(w[0].z); x[3] = __uint_as_float(w[0].w);
      x[4] = __uint_as_float(w[W - 1].x); x[5] = __uint_as_float(w[W - 1].y);
      x[6] = __uint_as_float(w[W - 1].z); x[7] = __uint_as_float(w[W - 1].w);
    } else {
      x[0] = bf16lo(w[0].x); x[1] = bf16hi(w[0].x); x[2] = bf16lo(w[0].y); x[3] = bf16hi(w[0].y);
      x[4] = bf16lo(w[0].z); x[5] = bf16hi(w[0].z); x[6] = bf16lo(w[0].w); x[7] = bf16hi(w[0].w);
    }
  }
};

// One row of l = (l_L + alpha l_S) - beta l_P, rounded to float32 after every
// operation, so that equal inputs order equally wherever they are evaluated; an
// absent term counts as zero. FUSED = false: l = l_L as stored.
//
// A thread takes items of 8 columns. VEC: the row's terms lie alike against
// 16-byte boundaries (rows of an odd vocabulary do, and lie differently from row
// to row): items are counted from the boundary at or before the row's start,
// `sh` elements before it, so that whole items are vector loads and only a row's
// first and last are not. Otherwise an item's columns are kStreamThreads apart (a
// warp's lanes side by side) and sh = 0. Positions below are columns + sh.
template <typename T, bool FUSED, bool VEC>
struct FusedRow {
  const T* L;          // at position 0; FUSED: may be null
  const T* S;          // FUSED only, may be null
  const float* P;      // FUSED only, may be null
  float a, b;
  float minus_zero;    // -0, from the launch: see values()
  int sh, end;         // positions sh .. end - 1 are the row

  __device__ __forceinline__ FusedRow(const StreamRows& in, long long row) {
    L = in.longp ? static_cast<const T*>(in.longp) + row * in.ld_long : nullptr;
    S = nullptr;
    P = nullptr;
    a = b = 1.f;
    minus_zero = in.minus_zero;
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
    sh = 0;
    if constexpr (VEC) {
      sh = (int)((reinterpret_cast<uintptr_t>(!FUSED || L ? L : S) & 15u) / sizeof(T));
      if (!FUSED || L) L -= sh;
      if (FUSED && S) S -= sh;
      if (FUSED && P) P -= sh;
    }
    end = sh + in.V;
  }
  __device__ __forceinline__ float combine(float l, float s, float p) const {
    return FUSED ? __fsub_rn(__fadd_rn(l, __fmul_rn(a, s)), __fmul_rn(b, p)) : l;
  }
  // by position
  __device__ __forceinline__ float l_at(int k) const { return !FUSED || L ? row_elem(L, k) : 0.f; }
  __device__ __forceinline__ float s_at(int k) const { return FUSED && S ? row_elem(S, k) : 0.f; }
  __device__ __forceinline__ float p_at(int k) const { return FUSED && P ? __ldg(P + k) : 0.f; }
  __device__ __forceinline__ float at(int k) const { return combine(l_at(k), s_at(k), p_at(k)); }
};

// First position of item `it` of thread t in a slice that starts at k0; position i of an item.
template <bool VEC>
__device__ __forceinline__ int item_pos(int k0, int it, int t) {
  return k0 + it * kStreamStep + (VEC ? t * 8 : t);
}
template <bool VEC>
__device__ __forceinline__ int elem_pos(int k, int i) { return VEC ? k + i : k + i * kStreamThreads; }

// One item's terms as loaded.
template <typename T, bool FUSED, bool VEC>
struct Item {
  Raw8<T> l;
  Raw8<T> s;           // FUSED only
  int k;               // its first position; -1: past the slice

  __device__ __forceinline__ void load_whole(const FusedRow<T, FUSED, VEC>& row, int pos) {
    k = pos;
    if constexpr (VEC) {
      if (!FUSED || row.L) l.load(row.L + pos);
      else l.fill(0.f);
      if constexpr (FUSED) {
        if (row.S) s.load(row.S + pos);
        else s.fill(0.f);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        l.set(i, row.l_at(elem_pos<VEC>(pos, i)));
        if constexpr (FUSED) s.set(i, row.s_at(elem_pos<VEC>(pos, i)));
      }
    }
  }
  // As far as its positions are in the row and before `stop`: -inf (l_S: 0) elsewhere.
  __device__ __forceinline__ void load(const FusedRow<T, FUSED, VEC>& row, int pos, int stop) {
    if (VEC && pos >= row.sh && pos + 8 <= stop) return load_whole(row, pos);
    k = pos;
    l.fill(-INFINITY);
    if constexpr (FUSED) s.fill(0.f);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int q = elem_pos<VEC>(pos, i);
      if (q >= row.sh && q < stop) {
        l.set(i, row.l_at(q));
        if constexpr (FUSED) s.set(i, row.s_at(q));
      }
    }
  }
  // The prior of its positions (CHECK: 0 outside the row and from `stop` on).
  template <bool CHECK>
  __device__ __forceinline__ void prior(const FusedRow<T, FUSED, VEC>& row, int stop, float (&p)[8]) const {
    if constexpr (!FUSED) return;
    if (!row.P) {
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = 0.f;
      return;
    }
    if constexpr (!VEC || CHECK) {
      if (!VEC || k < row.sh || k + 8 > stop) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int q = elem_pos<VEC>(k, i);
          p[i] = !CHECK || (q >= row.sh && q < stop) ? row.p_at(q) : 0.f;
        }
        return;
      }
    }
    if constexpr (VEC) {
      const int o = row.sh & 3;                    // the prior's own place against 16 bytes is -sh
      const float* base = row.P + k;
      if (o == 0) {
        const float4 u = __ldg(reinterpret_cast<const float4*>(base));
        const float4 v = __ldg(reinterpret_cast<const float4*>(base) + 1);
        p[0] = u.x; p[1] = u.y; p[2] = u.z; p[3] = u.w; p[4] = v.x; p[5] = v.y; p[6] = v.z; p[7] = v.w;
        return;
      }
      // the widest aligned loads of each place
      if (o == 2) {
        const float2 u = __ldg(reinterpret_cast<const float2*>(base));
        const float4 v = __ldg(reinterpret_cast<const float4*>(base + 2));
        const float2 w = __ldg(reinterpret_cast<const float2*>(base + 6));
        p[0] = u.x; p[1] = u.y; p[2] = v.x; p[3] = v.y; p[4] = v.z; p[5] = v.w; p[6] = w.x; p[7] = w.y;
      } else if (o == 1) {
        const float u = __ldg(base);
        const float4 v = __ldg(reinterpret_cast<const float4*>(base + 1));
        const float2 w = __ldg(reinterpret_cast<const float2*>(base + 5));
        const float z = __ldg(base + 7);
        p[0] = u; p[1] = v.x; p[2] = v.y; p[3] = v.z; p[4] = v.w; p[5] = w.x; p[6] = w.y; p[7] = z;
      } else {
        const float u = __ldg(base);
        const float2 v = __ldg(reinterpret_cast<const float2*>(base + 1));
        const float4 w = __ldg(reinterpret_cast<const float4*>(base + 3));
        const float z = __ldg(base + 7);
        p[0] = u; p[1] = v.x; p[2] = v.y; p[3] = w.x; p[4] = w.y; p[5] = w.z; p[6] = w.w; p[7] = z;
      }
    }
  }
  // Values of the 8 positions, and the l_S and l_P in them. The products are packed
  // fmas with an addend of -0 that only the launch knows: a packed product that
  // feeds a packed sum is contracted whatever its rounding modifier and the
  // compiler's flags (seen by comparing bits), and so is one with a constant -0.
  template <bool CHECK>
  __device__ __forceinline__ void values(const FusedRow<T, FUSED, VEC>& row, int stop, float (&x)[8], float (&sv)[8],
                                         float (&p)[8]) const {
    l.unpack(x);
    if constexpr (!FUSED) return;
    s.unpack(sv);
    prior<CHECK>(row, stop, p);
    const f32x2 a2 = both2(row.a), b2 = both2(-row.b);       // x - b p = x + (-b) p, both rounded alike
    const f32x2 z2 = both2(row.minus_zero);
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const f32x2 v = add2(add2(pair2(x[i], x[i + 1]), fma2(a2, pair2(sv[i], sv[i + 1]), z2)),
                           fma2(b2, pair2(p[i], p[i + 1]), z2));
      split2(v, x[i], x[i + 1]);
    }
  }
};

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
// The records of lanes 0 .. 7 of a warp merged (all lanes converged; lane i + 8 has
// lane i's), in every lane, in a fixed order.
__device__ __forceinline__ SoftRec softrec_merge8(const SoftRec& b, float c) {
  SoftRec r{warp_max(b.m), 0.f, 0.f};
  const unsigned who = __ballot_sync(0xFFFFFFFFu, b.m == r.m);
  softrec_add(r, b, r.m, c, (threadIdx.x & 7) == (unsigned)(__ffs(who) - 1));
#pragma unroll
  for (int d = 4; d > 0; d >>= 1) {
    r.rest += __shfl_xor_sync(0xFFFFFFFFu, r.rest, d);
    r.w += __shfl_xor_sync(0xFFFFFFFFu, r.w, d);
  }
  return r;
}
static_assert(kStreamWarps == 8 && kMaxCluster <= 8, "one record per lane of eight");
__device__ __forceinline__ bool softrec_valid(const SoftRec& r) {
  return r.m > -INFINITY && r.m < INFINITY && r.rest >= 0.f && r.rest < INFINITY;
}

// Largest of 8 values (NaN ignored).
__device__ __forceinline__ float max8(const float (&x)[8]) {
  return fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
}

// One lane's sums under its warp's reference (the warp's largest entry so far),
// in which the lane that holds an entry equal to it keeps that entry out. The sums
// are pairs: even and odd elements apart.
struct WarpSoft {
  float ref, off;      // the same in every lane; off = ref, or 0 while ref is -inf
  f32x2 rest, w;
  bool holds;
  __device__ __forceinline__ void init() {
    ref = -INFINITY;
    off = 0.f;
    rest = w = 0ull;
    holds = false;
  }
  // U items' values, all lanes converged; `vm`: the largest of the lane's.
  template <int U>
  __device__ __forceinline__ void push(float (&x)[U][8], float vm, float c) {
    if (__any_sync(0xFFFFFFFFu, vm > ref)) {
      const float top = warp_max(vm);
      const float d = ref == -INFINITY ? 0.f : fmaxf((ref - top) * c, kLowT);
      const float r1 = sum2(rest);
      const float f = ref == -INFINITY ? (r1 != r1 ? NAN : 0.f) : ex2_approx(d);
      w = pair2(f * (sum2(w) + d * r1) + (holds ? f * d : 0.f), 0.f);
      rest = pair2(f * r1 + (holds ? f : 0.f), 0.f);
      ref = off = top;
      const unsigned who = __ballot_sync(0xFFFFFFFFu, vm == top);
      holds = (int)(threadIdx.x & 31) == __ffs(who) - 1;
      bool out = holds;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (out && x[u][i] == top) {
            out = false;
            x[u][i] = -INFINITY;
          }
    }
    const f32x2 no = both2(-off), c2 = both2(c);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        float t0, t1;
        split2(mul2(add2(pair2(x[u][i], x[u][i + 1]), no), c2), t0, t1);
        const f32x2 e = pair2(ex2_approx(t0), ex2_approx(t1));
        rest = add2(rest, e);
        w = fma2(e, pair2(fmaxf(t0, kLowT), fmaxf(t1, kLowT)), w);
      }
  }
  // The warp's record (all lanes converged), in every lane.
  __device__ __forceinline__ SoftRec record() const {
    SoftRec r{ref, sum2(rest), sum2(w)};
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      r.rest += __shfl_xor_sync(0xFFFFFFFFu, r.rest, d);
      r.w += __shfl_xor_sync(0xFFFFFFFFu, r.w, d);
    }
    return r;
  }
};

// The items of a thread in positions k0 .. k1 - 1 of a row (a slice, at most the
// row's end), U at a time: f(items, checked) with checked = std::false_type where
// all of them are whole for every thread. U loads are in flight at once; what U
// leaves over, and a row's ends, go one by one.
template <int U, typename T, bool FUSED, bool VEC, typename F>
__device__ __forceinline__ void stream_items(const FusedRow<T, FUSED, VEC>& row, int k0, int k1, F&& f) {
  const int items = (k1 - k0 + kStreamStep - 1) / kStreamStep;
  const int whole = (k1 - k0) / kStreamStep;
  int it = 0;
  if (k0 < row.sh && items > 0) {                  // a row's first item may not be whole
    Item<T, FUSED, VEC> v[1];
    v[0].load(row, item_pos<VEC>(k0, 0, threadIdx.x), k1);
    f(v, std::true_type{});
    it = 1;
  }
  for (; it + U <= whole; it += U) {
    Item<T, FUSED, VEC> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u].load_whole(row, item_pos<VEC>(k0, it + u, threadIdx.x));
    f(v, std::false_type{});
  }
  for (; it < items; ++it) {
    const int pos = item_pos<VEC>(k0, it, threadIdx.x);
    if (!__any_sync(0xFFFFFFFFu, pos < k1)) break;
    Item<T, FUSED, VEC> v[1];
    v[0].load(row, pos, k1);
    f(v, std::true_type{});
  }
}

// The two halves of a cluster barrier (all threads of all its CTAs).
__device__ __forceinline__ void cluster_arrive_relaxed() {
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

}  // namespace dels
