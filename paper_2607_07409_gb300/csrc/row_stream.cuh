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
  __device__ __forceinline__ void load(const T* p, int half) {      // half: elements between the words
#pragma unroll
    for (int k = 0; k < W; ++k) w[k] = __ldcs(reinterpret_cast<const uint4*>(p + k * half));
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
// A thread takes items of 8 columns: consecutive ones of bf16 rows, two times four of
// float32 rows, 4 kStreamThreads apart (a warp's 16-byte loads are side by side
// either way). VEC: the row's terms lie alike against 16-byte boundaries (rows of an odd vocabulary do, and lie differently from row
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
      const unsigned j = (unsigned)row % (unsigned)in.n_weights;
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

// Distance from an item's first four positions to its other four.
template <typename T>
constexpr int kHalf = sizeof(T) == 4 ? 4 * kStreamThreads : 4;
// First position of item `it` of thread t in a slice that starts at k0; position i of an item.
template <typename T, bool VEC>
__device__ __forceinline__ int item_pos(int k0, int it, int t) {
  return k0 + it * kStreamStep + (VEC ? t * (sizeof(T) == 4 ? 4 : 8) : t);
}
template <typename T, bool VEC>
__device__ __forceinline__ int elem_pos(int k, int i) {
  return VEC ? k + (i < 4 ? i : kHalf<T> + i - 4) : k + i * kStreamThreads;
}
// Four floats of the prior, `o` past a 16-byte boundary.
__device__ __forceinline__ void prior4(const float* p, int o, float* x) {
  if (o == 0) {
    const float4 u = __ldg(reinterpret_cast<const float4*>(p));
    x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w;
  } else if (o == 2) {
    const float2 u = __ldg(reinterpret_cast<const float2*>(p)), v = __ldg(reinterpret_cast<const float2*>(p + 2));
    x[0] = u.x; x[1] = u.y; x[2] = v.x; x[3] = v.y;
  } else {
    const float2 u = __ldg(reinterpret_cast<const float2*>(p + 1));
    x[0] = __ldg(p); x[1] = u.x; x[2] = u.y; x[3] = __ldg(p + 3);
  }
}

// One item's terms as loaded.
template <typename T, bool FUSED, bool VEC>
struct Item {
  Raw8<T> l;
  Raw8<T> s;           // FUSED only
  int k;               // its first position
  float pr[8];         // its l_P, where the stream has loaded it (whole items of FUSED rows)

  __device__ __forceinline__ void load_whole(const FusedRow<T, FUSED, VEC>& row, int pos) {
    k = pos;
    if constexpr (VEC) {
      if (!FUSED || row.L) l.load(row.L + pos, kHalf<T>);
      else l.fill(0.f);
      if constexpr (FUSED) {
        if (row.S) s.load(row.S + pos, kHalf<T>);
        else s.fill(0.f);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        l.set(i, row.l_at(elem_pos<T, VEC>(pos, i)));
        if constexpr (FUSED) s.set(i, row.s_at(elem_pos<T, VEC>(pos, i)));
      }
    }
  }
  // As far as its positions are in the row and before `stop`: -inf (l_S: 0) elsewhere.
  __device__ __forceinline__ void load(const FusedRow<T, FUSED, VEC>& row, int pos, int stop) {
    if (VEC && pos >= row.sh && pos + kHalf<T> + 4 <= stop) return load_whole(row, pos);
    k = pos;
    l.fill(-INFINITY);
    if constexpr (FUSED) s.fill(0.f);
    if (pos >= stop) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int q = elem_pos<T, VEC>(pos, i);
      if (q >= row.sh && q < stop) {
        l.set(i, row.l_at(q));
        if constexpr (FUSED) s.set(i, row.s_at(q));
      }
    }
  }
  // The prior of the positions of an item at k (CHECK: 0 outside the row and from `stop` on).
  template <bool CHECK>
  __device__ __forceinline__ void prior(const FusedRow<T, FUSED, VEC>& row, int stop, float (&p)[8]) const {
    if constexpr (!FUSED) return;
    if (!row.P) {
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = 0.f;
      return;
    }
    if constexpr (!VEC || CHECK) {
      if (!VEC || k < row.sh || k + kHalf<T> + 4 > stop) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int q = elem_pos<T, VEC>(k, i);
          p[i] = !CHECK || (q >= row.sh && q < stop) ? row.p_at(q) : 0.f;
        }
        return;
      }
    }
    if constexpr (VEC) {                           // (the prior's own place against 16 bytes is -sh)
      prior4(row.P + k, -row.sh & 3, p);
      prior4(row.P + k + kHalf<T>, -row.sh & 3, p + 4);
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
    if constexpr (VEC && !CHECK) {
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = pr[i];
    } else {
      prior<CHECK>(row, stop, p);
    }
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

// Largest of 8 values (NaN ignored).
__device__ __forceinline__ float max8(const float (&x)[8]) {
  return fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
}

// ---------------------------------------------------------------------------
// Running softmax sums: exponentials as 2^z, z = (x - off) c - r, c = log2(e) / T.
// The reference is off = 0 with a whole number r near m c, m an entry met: z is
// then one fma, exact but for its own rounding (m c itself would be rounded, a
// common factor of 2^(|m c| 2^-24) in all of them), and a change of r scales sums by
// a power of two. Past kMaxRef, where a whole row is masked by values such as -1e9
// or the type's lowest, off = m and r = 0.
// ---------------------------------------------------------------------------
struct Ref {
  float off, r;
};
__device__ __forceinline__ Ref make_ref(float m, float c) {
  const float s = m * c;
  return past_ref_bound(s) ? Ref{m, 0.f} : Ref{0.f, rintf(s)};
}
__device__ __forceinline__ float ref_z(float x, const Ref& f, float c) { return fmaf(x - f.off, c, -f.r); }
constexpr float kLowT = -1e30f;   // 2^z z is 0 from here on, -inf included
// What sums relative to `from` are multiplied by, as a power of two, for `to`.
__device__ __forceinline__ float ref_shift(const Ref& from, const Ref& to, float c) {
  return fmaxf((from.off - to.off) * c + (from.r - to.r), kLowT);
}

// m: the largest entry; rest = sum 2^z without one entry that attains m (held out, so
// that ln S = z_m ln 2 + ln(1 + rest / 2^z_m) keeps its digits where one entry has
// nearly all mass); w = sum 2^z z over the same.
struct SoftRec {
  float m;
  Ref f;
  float rest, w;
};
__device__ __forceinline__ SoftRec softrec_init() { return SoftRec{-INFINITY, Ref{0.f, 0.f}, 0.f, 0.f}; }

// The records of lanes 0 .. 7 of a warp merged (all lanes converged; lane i + 8 has
// lane i's), in every lane, in a fixed order.
__device__ __forceinline__ SoftRec softrec_merge8(const SoftRec& b, float c) {
  SoftRec r;
  r.m = warp_max(b.m);
  const int top = __ffs(__ballot_sync(0xFFFFFFFFu, b.m == r.m)) - 1;
  r.f.off = __shfl_sync(0xFFFFFFFFu, b.f.off, top);
  r.f.r = __shfl_sync(0xFFFFFFFFu, b.f.r, top);
  const bool none = b.m == -INFINITY;              // (its rest is 0, or NaN where it met one)
  const float d = none ? 0.f : ref_shift(b.f, r.f, c), f = none ? 1.f : ex2_approx(d);
  r.rest = f * b.rest;
  r.w = f * (b.w + d * b.rest);
  if (!none && (int)(threadIdx.x & 7) != top) {      // another's largest goes in
    const float z = fmaxf(ref_z(b.m, r.f, c), kLowT), e = ex2_approx(z);
    r.rest += e;
    r.w += e * z;
  }
#pragma unroll
  for (int d2 = 4; d2 > 0; d2 >>= 1) {
    r.rest += __shfl_xor_sync(0xFFFFFFFFu, r.rest, d2);
    r.w += __shfl_xor_sync(0xFFFFFFFFu, r.w, d2);
  }
  return r;
}
static_assert(kStreamWarps == 8 && kMaxCluster <= 8, "one record per lane of eight");
__device__ __forceinline__ bool softrec_valid(const SoftRec& r) {
  return r.m > -INFINITY && r.m < INFINITY && r.rest >= 0.f && r.rest < INFINITY;
}

// One lane's sums under its warp's reference; `m` is the warp's largest entry so
// far, and the lane that met it first keeps it out of its sums. The sums are pairs:
// even and odd elements apart.
struct WarpSoft {
  float m;             // the same in every lane, as f
  Ref f;
  f32x2 rest, w;
  bool holds;
  __device__ __forceinline__ void init() {
    m = -INFINITY;
    f = Ref{0.f, 0.f};
    rest = w = 0ull;
    holds = false;
  }
  // A new largest entry `top` > m (all lanes converged): the one held so far goes
  // into the sums; whether this lane holds the new one (`vm`: its largest).
  __device__ __forceinline__ bool raise(float top, float vm, float c) {
    float r1 = sum2(rest), w1 = sum2(w);
    if (holds) {
      const float z = ref_z(m, f, c), e = ex2_approx(z);
      r1 += e;
      w1 += e * z;
    }
    if (m == -INFINITY || past_ref_bound(top * c) || f.off != 0.f || fmaf(top, c, -f.r) > 1.f) {
      const Ref to = make_ref(top, c);
      if (m > -INFINITY) {
        const float d = ref_shift(f, to, c), s = ex2_approx(d);
        w1 = s * (w1 + d * r1);
        r1 *= s;
      }
      f = to;
    }
    rest = pair2(r1, 0.f);
    w = pair2(w1, 0.f);
    m = top;
    const unsigned who = __ballot_sync(0xFFFFFFFFu, vm == top);
    return holds = (int)(threadIdx.x & 31) == __ffs(who) - 1;
  }
  // CLAMPED: no x is so low that 2^z z is not a number (x relative to f.off).
  template <bool CLAMPED>
  __device__ __forceinline__ void add(const float (&x)[8], float c) {
    const f32x2 c2 = both2(c), nr = both2(-f.r);
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const f32x2 z = fma2(pair2(x[i], x[i + 1]), c2, nr);
      float z0, z1;
      split2(z, z0, z1);
      const f32x2 e = pair2(ex2_approx(z0), ex2_approx(z1));
      rest = add2(rest, e);
      w = fma2(e, CLAMPED ? z : pair2(fmaxf(z0, kLowT), fmaxf(z1, kLowT)), w);
    }
  }
  // The warp's record (all lanes converged), in every lane.
  __device__ __forceinline__ SoftRec record() const {
    SoftRec r{m, f, sum2(rest), sum2(w)};
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      r.rest += __shfl_xor_sync(0xFFFFFFFFu, r.rest, d);
      r.w += __shfl_xor_sync(0xFFFFFFFFu, r.w, d);
    }
    return r;
  }
};

// 16 bytes from global to shared memory without a register between.
__device__ __forceinline__ void copy16(uint32_t smem, const void* gmem) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(gmem) : "memory");
}
__device__ __forceinline__ void copy16_l1(uint32_t smem, const void* gmem) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(gmem) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Shared memory that whole items are copied to ahead of their use, in 16-byte pieces:
// 8 logits are W of them, a fused item l_L's and l_S's. A piece belongs to one
// thread, which copies it, waits for it and reads it: no barrier. A warp's copies of a
// piece are 512 bytes side by side.
//
// Items come in groups of U; a ring has D groups. With R > 0 the first two pieces of
// every item have a place of their own that stays (32 bytes: the item's 8 values as
// float32 later), copied R groups ahead, and the ring has the others.
template <typename T, bool FUSED, int U_, int D_, int R_ = 0>
struct Copies {
  static constexpr int U = U_, D = D_, R = R_;
  static constexpr int W = Raw8<T>::W;
  static constexpr int kPieces = FUSED ? 2 * W : W;
  static constexpr int kStay = R > 0 ? 2 : 0;
  static constexpr int kRing = kPieces > kStay ? kPieces - kStay : 0;
  static constexpr int kPiece = 16 * kStreamThreads;             // one piece of all threads
  static constexpr int kRingBytes = D * U * kRing * kPiece;
  static constexpr int kItemBytes = kStay * kPiece;              // per item that stays
};

struct StreamPlan {
  int head;            // calls of the row's first item, which may not be whole: 0 or 1
  int groups;          // calls of U whole items
  int items;           // of a thread
  template <int U>
  __device__ __forceinline__ static StreamPlan of(int k0, int k1, int sh, bool vec) {
    StreamPlan p;
    p.items = (k1 - k0 + kStreamStep - 1) / kStreamStep;
    p.head = p.items > 0 && k0 < sh;
    p.groups = vec ? max(0, (k1 - k0) / kStreamStep - p.head) / U : 0;
    return p;
  }
  template <int U>
  __device__ __forceinline__ int calls() const { return head + groups + items - head - groups * U; }
  // First item of a call.
  template <int U>
  __device__ __forceinline__ int first(int call) const {
    const int g = call - head;
    return g <= 0 ? call : g < groups ? head + g * U : head + groups * U + (g - groups);
  }
};
// The items of a thread in positions k0 .. k1 - 1 of a row (a slice, at most the
// row's end). run() calls f(items, checked, call, it): checked = std::false_type where
// all of them are whole for every thread, `call` the number of the call, `it` the
// first one's number. With VEC whole items come U at a time, D - 1 such groups ahead in
// flight and the prior one group ahead in registers; what U leaves over, and a row's
// ends, go one by one. begin() starts the first copies; one that is not run is
// drained.
template <typename Cp, typename T, bool FUSED, bool VEC>
struct RowStream {
  static constexpr int U = Cp::U, D = Cp::D, R = Cp::R, W = Cp::W, PC = Cp::kPiece;
  const FusedRow<T, FUSED, VEC>& row;
  int k0, k1;
  uint8_t *ring, *stay;    // the calling thread's
  StreamPlan p;
  int slot_in = 0;

  __device__ __forceinline__ RowStream(const FusedRow<T, FUSED, VEC>& r, int from, int to, uint8_t* ring_, uint8_t* stay_)
      : row(r), k0(from), k1(to), ring(ring_ + threadIdx.x * 16), stay(stay_ + threadIdx.x * 16),
        p(StreamPlan::of<U>(from, to, r.sh, VEC)) {}
  // Piece k of item i of the groups, which is in place q of the ring.
  __device__ __forceinline__ uint8_t* place(int k, int i, int q) const {
    return k < Cp::kStay ? stay + (size_t)(p.head + i) * Cp::kItemBytes + k * PC
                         : ring + (q * Cp::kRing + k - Cp::kStay) * PC;
  }
  __device__ __forceinline__ void copy(int i, int q, int from, int to) const {
    const int at = item_pos<T, VEC>(k0, p.head + i, threadIdx.x);
#pragma unroll
    for (int k = 0; k < Cp::kPieces; ++k) {
      if (k < from || k >= to) continue;
      const uint32_t dst = smem_u32(place(k, i, q));
      if (k < W) {
        if (!FUSED || row.L) copy16(dst, row.L + at + k * kHalf<T>);
      } else {
        if (row.S) copy16(dst, row.S + at + (k - W) * kHalf<T>);
      }
    }
  }
  // What is copied when call g begins: the ring pieces of group g + D - 1 and those that
  // stay of group g + R - 1; one commit a call, empty at the end, so that at most
  // D - 1 later ones are in flight when group g is waited for.
  __device__ __forceinline__ void issue(int g) {
    if (Cp::kRing > 0 && g < p.groups) {
#pragma unroll
      for (int u = 0; u < U; ++u) copy(g * U + u, slot_in * U + u, Cp::kStay, Cp::kPieces);
      slot_in = slot_in + 1 == D ? 0 : slot_in + 1;
    }
  }
  __device__ __forceinline__ void issue_stay(int g) const {
    if (R > 0 && g < p.groups) {
#pragma unroll
      for (int u = 0; u < U; ++u) copy(g * U + u, 0, 0, Cp::kStay);
    }
  }
  __device__ __forceinline__ void begin() {
    if constexpr (VEC) {
#pragma unroll
      for (int d = 0; d < D - 1; ++d) {
        issue(d);
        if (d < R - 1) issue_stay(d);
        copies_commit();
      }
#pragma unroll 1
      for (int g = D - 1; g < R - 1; ++g) issue_stay(g);
    }
  }
  __device__ __forceinline__ void drain() const {
    if constexpr (VEC) copies_wait<0>();
  }
  __device__ __forceinline__ void prior_of(int g, float (&x)[U][8]) const {
    if constexpr (FUSED && VEC) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (row.P && g < p.groups) {
          const int at = item_pos<T, VEC>(k0, p.head + g * U + u, threadIdx.x);
          prior4(row.P + at, -row.sh & 3, x[u]);             // (its own place against 16 bytes is -sh)
          prior4(row.P + at + kHalf<T>, -row.sh & 3, x[u] + 4);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) x[u][i] = 0.f;
        }
      }
    }
  }
  template <typename F>
  __device__ __forceinline__ void run(F&& f) {
    int it = 0, call = 0;
    auto one = [&]() {
      Item<T, FUSED, VEC> v[1];
      v[0].load(row, item_pos<T, VEC>(k0, it, threadIdx.x), k1);
      f(v, std::true_type{}, call, it);
      ++it;
      ++call;
    };
    if constexpr (VEC) {
      float pn[U][8];
      prior_of(0, pn);
      if (p.head) one();
      int slot = 0;
#pragma unroll 1
      for (int g = 0; g < p.groups; ++g) {
        issue(g + D - 1);
        issue_stay(g + R - 1);
        copies_commit();
        copies_wait<D - 1>();
        Item<T, FUSED, VEC> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int i = g * U + u, q = slot * U + u;
          v[u].k = item_pos<T, VEC>(k0, p.head + i, threadIdx.x);
#pragma unroll
          for (int k = 0; k < W; ++k) {
            if (!FUSED || row.L) v[u].l.w[k] = *reinterpret_cast<const uint4*>(place(k, i, q));
            if constexpr (FUSED) {
              if (row.S) v[u].s.w[k] = *reinterpret_cast<const uint4*>(place(W + k, i, q));
            }
          }
          if (FUSED && !row.L) v[u].l.fill(0.f);
          if constexpr (FUSED) {
            if (!row.S) v[u].s.fill(0.f);
#pragma unroll
            for (int i2 = 0; i2 < 8; ++i2) v[u].pr[i2] = pn[u][i2];
          }
        }
        prior_of(g + 1, pn);
        f(v, std::false_type{}, call, it);
        it += U;
        ++call;
        slot = slot + 1 == D ? 0 : slot + 1;
      }
      copies_wait<0>();
    }
    while (it < p.items) one();
  }
};

// The two halves of a cluster barrier (all threads of all its CTAs).
__device__ __forceinline__ void cluster_arrive_relaxed() {
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

}  // namespace dels
