// Rows of (fused) vocabulary logits as the scoring and distillation kernels
// stream them: one cluster of 1 to 8 CTAs takes a row, every CTA a slice of its
// columns, every thread items of 8 columns; the slices' sums meet in distributed
// shared memory, so that a pass over the rows needs no scratch in memory and no second
// launch to join them.
//
// What bounds the stream: of float32 rows the bytes (5.7 TB/s of a copy's 6.8); of bf16
// rows the instructions of a column beside the latency that 24 warps an SM hide: 19.2
// of the fused loss, 8.5 of plain scoring, 20.8 of fused scoring, at 58 to 67 % of the
// issue slots. Hence packed pairs, whole items without tests, one reference for a warp,
// and copies that pass through shared memory without a register or a barrier.
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

// What a row has: l_L as stored; any of the fusion's terms (an absent one counts as
// zero); all of them.
enum { kPlain = 0, kSome = 1, kFull = 2 };
// Kernels of float32 rows with some of the terms, which test for each where it is used:
// one CTA less on an SM than the others, for the registers that this takes (with as
// many 1740 bytes of spills, now 320 and in the loss alone: 304 rows of 151936, l_L and
// l_S, loss 148, 92 us).
template <typename T, int F>
constexpr int kFewer = F == kSome && sizeof(T) == 4 ? 1 : 0;

// One row of l = (l_L + alpha l_S) - beta l_P: combine() rounds to float32 after every
// operation, so that equal inputs order equally wherever they are evaluated,
// contracted() after each of two fmas.
//
// A thread takes items of 8 columns: consecutive ones of bf16 rows, two times four of
// float32 rows, 4 kStreamThreads apart (a warp's 16-byte loads are side by side
// either way; 32 bytes a lane took twice the requests to L2). VEC: the row's terms lie
// alike against 16-byte boundaries (rows of an odd vocabulary do, and lie differently
// from row to row): items are counted from the boundary at or before the row's start,
// `sh` elements before it, so that whole items are vector loads and only a row's
// first and last are not. Otherwise an item's columns are kStreamThreads apart (a
// warp's lanes side by side) and sh = 0. Positions below are columns + sh.
template <typename T, int F, bool VEC>
struct FusedRow {
  const T* L;          // at position 0; kSome: may be null
  const T* S;          // F != kPlain; kSome: may be null
  const float* P;
  float a, b;
  float minus_zero;    // -0, from the launch: see values()
  int sh, end;         // positions sh .. end - 1 are the row

  __device__ __forceinline__ FusedRow(const StreamRows& in, long long row) {
    L = F != kSome || in.longp ? static_cast<const T*>(in.longp) + row * in.ld_long : nullptr;
    S = nullptr;
    P = nullptr;
    a = b = 1.f;
    minus_zero = in.minus_zero;
    if constexpr (F != kPlain) {
      const unsigned j = (unsigned)row % (unsigned)in.n_weights;
      if (F == kFull || in.shortp) {
        S = static_cast<const T*>(in.shortp) + row * in.ld_short;
        if (in.alpha) a = __ldg(in.alpha + j);
      }
      if (F == kFull || in.prior) {
        P = in.prior;
        if (in.beta) b = __ldg(in.beta + j);
      }
    }
    sh = 0;
    if constexpr (VEC) {
      sh = (int)((reinterpret_cast<uintptr_t>(has_l() ? L : S) & 15u) / sizeof(T));
      if (has_l()) L -= sh;
      if (has_s()) S -= sh;
      if (has_p()) P -= sh;
    }
    end = sh + in.V;
  }
  __device__ __forceinline__ bool has_l() const { return F != kSome || L; }
  __device__ __forceinline__ bool has_s() const { return F == kFull || (F == kSome && S); }
  __device__ __forceinline__ bool has_p() const { return F == kFull || (F == kSome && P); }
  __device__ __forceinline__ float combine(float l, float s, float p) const {
    return F ? __fsub_rn(__fadd_rn(l, __fmul_rn(a, s)), __fmul_rn(b, p)) : l;
  }
  // The same in two fmas, where no order of entries hangs on the last bit.
  __device__ __forceinline__ float contracted(float l, float s, float p) const {
    return F ? fmaf(-b, p, fmaf(a, s, l)) : l;
  }
  // by position
  __device__ __forceinline__ float l_at(int k) const { return has_l() ? row_elem(L, k) : 0.f; }
  __device__ __forceinline__ float s_at(int k) const { return has_s() ? row_elem(S, k) : 0.f; }
  __device__ __forceinline__ float p_at(int k) const { return has_p() ? __ldg(P + k) : 0.f; }
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
template <typename T, int F, bool VEC>
struct Item {
  Raw8<T> l;
  Raw8<T> s;           // F != kPlain
  int k;               // its first position

  // As far as its positions are in the row and before `stop`: l = -inf (l_S, l_P: 0)
  // elsewhere.
  __device__ __forceinline__ void load(const FusedRow<T, F, VEC>& row, int pos, int stop, float (&pr)[8]) {
    k = pos;
    l.fill(-INFINITY);
    if constexpr (F != kPlain) {
      s.fill(0.f);
#pragma unroll
      for (int i = 0; i < 8; ++i) pr[i] = 0.f;
    }
    if (pos >= stop) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int q = elem_pos<T, VEC>(pos, i);
      if (q >= row.sh && q < stop) {
        l.set(i, row.l_at(q));
        if constexpr (F != kPlain) {
          s.set(i, row.s_at(q));
          pr[i] = row.p_at(q);
        }
      }
    }
  }
  // A whole item, straight from memory.
  __device__ __forceinline__ void load_whole(const FusedRow<T, F, VEC>& row, int pos, float (&pr)[8]) {
    k = pos;
    if (row.has_l()) l.load(row.L + pos, kHalf<T>);
    else l.fill(0.f);
    if constexpr (F != kPlain) {
      if (row.has_s()) s.load(row.S + pos, kHalf<T>);
      else s.fill(0.f);
#pragma unroll
      for (int i = 0; i < 8; ++i) pr[i] = row.p_at(elem_pos<T, VEC>(pos, i));
    }
  }
  // Values of the 8 positions, and the l_S in them. Where they are rounded after every
  // operation the products are packed fmas with an addend of -0 that only the launch
  // knows: a packed product that feeds a packed sum is contracted whatever its rounding
  // modifier and the compiler's flags (seen by comparing bits), and so is one with a
  // constant -0.
  template <bool CONTRACT>
  __device__ __forceinline__ void values(const FusedRow<T, F, VEC>& row, const float (&pr)[8], float (&x)[8],
                                         float (&sv)[8]) const {
    l.unpack(x);
    if constexpr (F != kPlain) {
      s.unpack(sv);
      const f32x2 a2 = both2(row.a), b2 = both2(-row.b);     // x - b p = x + (-b) p, both rounded alike
      const f32x2 z2 = both2(row.minus_zero);
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const f32x2 lv = pair2(x[i], x[i + 1]), s2 = pair2(sv[i], sv[i + 1]), p2 = pair2(pr[i], pr[i + 1]);
        split2(CONTRACT ? fma2(b2, p2, fma2(a2, s2, lv)) : add2(add2(lv, fma2(a2, s2, z2)), fma2(b2, p2, z2)), x[i],
               x[i + 1]);
      }
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
// Items come in groups of U, D groups ahead, in a ring of D groups. With STAY the first
// two pieces of every item have a place of their own (32 bytes: what 8 values take as
// float32 later), and the ring has the others.
template <typename T, int F, int U_, int D_, bool STAY_ = false>
struct Copies {
  static constexpr int U = U_, D = D_;
  static constexpr bool STAY = STAY_;
  static constexpr int W = Raw8<T>::W;
  static constexpr int kPieces = F ? 2 * W : W;
  static constexpr int kStay = STAY ? 2 : 0;
  static constexpr int kRing = kPieces > kStay ? kPieces - kStay : 0;
  static constexpr int kPiece = 16 * kStreamThreads;             // one piece of all threads
  static constexpr int kRingBytes = D * U * kRing * kPiece;
  static constexpr int kItemBytes = kStay * kPiece;              // per item that stays
};

// The items of a thread in positions k0 .. k1 - 1 of a row (a slice, at most the
// row's end). begin() starts the first copies; run() calls whole(group) for groups of U
// items that are whole for every thread, which reads them with take() and their l_P
// with prior(), and ragged(item, l_P, it) for an item of the others (at a row's ends;
// all without VEC), loaded where it is used if it is not whole itself.
template <typename Cp, typename T, int F, bool VEC>
struct RowStream {
  static constexpr int U = Cp::U, D = Cp::D, W = Cp::W, PC = Cp::kPiece;
  static constexpr int kRingGroup = U * Cp::kRing * PC, kStayGroup = U * Cp::kItemBytes;
  FusedRow<T, F, VEC> row;
  const StreamRows& rows;  // to make `row` anew where it is rarely used: its pointers then take no registers on the way
  unsigned r;
  int k0, k1, items, groups;
  int lo, hi;              // groups lo .. hi - 1 are whole
  uint8_t *ring, *stay;    // the calling thread's
  const T *next_l, *next_s;// its first item of the next group to copy
  int next_group = 0;
  uint32_t in;             // the ring's place for it
  uint32_t in_stay;
  // while a group is processed
  const uint8_t *out, *out_stay;
  const float* p;          // l_P of its first item
  int pos;                 // its position

  __device__ __forceinline__ RowStream(const StreamRows& rows_, unsigned r_, int rank, uint8_t* ring_, uint8_t* stay_)
      : row(rows_, r_), rows(rows_), r(r_), ring(ring_ + threadIdx.x * 16), stay(stay_ + threadIdx.x * 16) {
    const long long first = (long long)rank * rows.slice_cols;
    k0 = (int)min(first, (long long)row.end);
    k1 = (int)min(first + rows.slice_cols, (long long)row.end);
    items = (k1 - k0 + kStreamStep - 1) / kStreamStep;
    groups = (items + U - 1) / U;
    lo = k0 < row.sh ? 1 : 0;
    hi = VEC ? max(lo, (k1 - k0) / (U * kStreamStep)) : lo;
    if (!VEC || hi > groups) hi = lo = groups;
    pos = item_pos<T, VEC>(k0, 0, threadIdx.x);
    next_l = row.L + pos;
    next_s = row.S + pos;
    p = row.P + pos;
    in = smem_u32(ring);
    in_stay = smem_u32(stay);
    out = ring;
    out_stay = stay;
  }
  __device__ __forceinline__ FusedRow<T, F, VEC> anew() const { return FusedRow<T, F, VEC>(rows, r); }
  __device__ __forceinline__ bool whole(int at) const { return VEC && at >= row.sh && at + kHalf<T> + 4 <= k1; }
  __device__ __forceinline__ void copy(int u) const {
#pragma unroll
    for (int k = 0; k < Cp::kPieces; ++k) {
      const uint32_t dst =
          k < Cp::kStay ? in_stay + u * Cp::kItemBytes + k * PC : in + (u * Cp::kRing + k - Cp::kStay) * PC;
      if (k < W) {
        if (row.has_l()) copy16(dst, next_l + u * kStreamStep + k * kHalf<T>);
      } else {
        if (row.has_s()) copy16(dst, next_s + u * kStreamStep + (k - W) * kHalf<T>);
      }
    }
  }
  // The next group's copies, one commit (empty past the last).
  __device__ __forceinline__ void fetch() {
    if (next_group < groups) {
      if (next_group >= lo && next_group < hi) {
#pragma unroll
        for (int u = 0; u < U; ++u) copy(u);
      } else {
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (whole(item_pos<T, VEC>(k0, next_group * U + u, threadIdx.x))) copy(u);
      }
      ++next_group;
      next_l += U * kStreamStep;
      next_s += U * kStreamStep;
      if (Cp::kRing > 0) in = in == smem_u32(ring) + (D - 1) * kRingGroup ? smem_u32(ring) : in + kRingGroup;
      in_stay += kStayGroup;
    }
    copies_commit();
  }
  __device__ __forceinline__ void begin() {
    if constexpr (VEC) {
#pragma unroll 1
      for (int d = 0; d < D; ++d) fetch();
    }
  }
  __device__ __forceinline__ void drain() const {
    if constexpr (VEC) copies_wait<0>();
  }
  // Item u of the current group.
  __device__ __forceinline__ void take(int u, Item<T, F, VEC>& v) const {
    v.k = pos + u * kStreamStep;
#pragma unroll
    for (int k = 0; k < W; ++k) {
      const auto at = [&](int q) {
        return q < Cp::kStay ? out_stay + u * Cp::kItemBytes + q * PC : out + (u * Cp::kRing + q - Cp::kStay) * PC;
      };
      if (row.has_l()) v.l.w[k] = *reinterpret_cast<const uint4*>(at(k));
      if constexpr (F != kPlain) {
        if (row.has_s()) v.s.w[k] = *reinterpret_cast<const uint4*>(at(W + k));
      }
    }
    if (!row.has_l()) v.l.fill(0.f);
    if constexpr (F != kPlain) {
      if (!row.has_s()) v.s.fill(0.f);
    }
  }
  // l_P of whole item u of the current group (u may run past it). ALIGNED: the prior's
  // own place against 16 bytes, which is -sh, is 0.
  template <bool ALIGNED>
  __device__ __forceinline__ void prior(int u, float (&x)[8]) const {
    if constexpr (F != kPlain) {
      const float* at = p + u * kStreamStep;
      if (!row.has_p()) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = 0.f;
      } else if (ALIGNED) {
        const float4 y = __ldg(reinterpret_cast<const float4*>(at));
        const float4 z = __ldg(reinterpret_cast<const float4*>(at + kHalf<T>));
        x[0] = y.x; x[1] = y.y; x[2] = y.z; x[3] = y.w; x[4] = z.x; x[5] = z.y; x[6] = z.z; x[7] = z.w;
      } else {
        prior4(at, -row.sh & 3, x);
        prior4(at + kHalf<T>, -row.sh & 3, x + 4);
      }
    }
  }
  __device__ __forceinline__ bool prior_aligned() const { return (row.sh & 3) == 0; }
  template <typename Whole, typename Ragged>
  __device__ __forceinline__ void run(Whole&& f_whole, Ragged&& f_ragged) {
#pragma unroll 1
    for (int g = 0; g < groups; ++g) {
      if constexpr (VEC) copies_wait<D - 1>();
      if (g >= lo && g < hi) {
        f_whole(g);
      } else {
#pragma unroll 1
        for (int u = 0; u < U; ++u) {
          const int at = pos + u * kStreamStep;
          Item<T, F, VEC> v;
          float pr[8];
          if (whole(at)) {
            take(u, v);
            prior<false>(u, pr);
          } else {
            v.load(anew(), at, k1, pr);
          }
          f_ragged(v, pr, g * U + u);
        }
      }
      if constexpr (VEC) fetch();
      pos += U * kStreamStep;
      if (F != kPlain) p += U * kStreamStep;
      if (Cp::kRing > 0) out = out == ring + (D - 1) * kRingGroup ? ring : out + kRingGroup;
      out_stay += kStayGroup;
    }
    drain();
  }
  // As whole(group) of run(): f(item, l_P, it) for each item, the prior out of L2 an
  // item ahead, in two sets of registers by turns (copies between them took 8
  // instructions an item, loads at their use 700 cycles).
  template <bool ALIGNED, typename Fn>
  __device__ __forceinline__ void each_of(int g, float (&pa)[8], float (&pb)[8], Fn&& f) const {
    static_assert(U % 2 == 0 || F == kPlain, "two sets by turns");
    if (g == lo) prior<ALIGNED>(0, pa);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      Item<T, F, VEC> v;
      take(u, v);
      if (u + 1 < U || g + 1 < hi) prior<ALIGNED>(u + 1, u & 1 ? pa : pb);
      f(v, u & 1 ? pb : pa, g * U + u);
    }
  }
  template <typename Fn>
  __device__ __forceinline__ void each(int g, float (&pa)[8], float (&pb)[8], Fn&& f) const {
    if (F == kPlain || prior_aligned()) each_of<true>(g, pa, pb, f);
    else each_of<false>(g, pa, pb, f);
  }
};

// The two halves of a cluster barrier (all threads of all its CTAs).
__device__ __forceinline__ void cluster_arrive_relaxed() {
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_arrive() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// A row kernel's launch over the rows of `a`, of `smem(in)` dynamic bytes a CTA.
//
// `split`: where a CTA has a row, the rows past the last whole round of CTAs would leave most
// of the device idle for a round. They get a launch of their own with more CTAs a row,
// which starts as soon as those of the first have (programmatic launch) and fills
// the places that they leave. It does not wait for the first launch, whose rows are
// others (what is before both has ended: every CTA of the first has waited for it);
// but what comes after must, so one more cluster of it does nothing but that wait.
// Fused bf16 rows of 151936, one launch and two, us: 1024 rows the loss 133, 127, the
// gradient 178, 162, scoring 166, 159; 500 rows 85, 74, 106, 84, 105, 84. Short rows
// lose by it (1024 of 16384: 23.0, 27.0; 32.5, 32.4; 32.4, 39.8): see the callers' bounds.
template <typename Args, typename Smem>
cudaError_t launch_rows(void (*k)(Args), const Args& a, bool clusters, bool split, Smem&& smem, cudaStream_t s) {
  const auto launch = [&](const Args& part) {
    const size_t bytes = smem(part.in);
    const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(k), bytes);
    if (e != cudaSuccess) return e;
    const dim3 grid((unsigned)((long long)(part.in.count + part.in.beside) * part.in.cluster));
    return launch_pdl_cluster(k, grid, dim3(kStreamThreads), bytes, s, clusters ? part.in.cluster : 1, part);
  };
  const int sms = device_sm_count();
  if (split && a.in.cluster == 1 && a.in.count > sms) {
    int per_sm = 0;
    const size_t bytes = smem(a.in);
    cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(k), bytes);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, k, kStreamThreads, bytes);
    if (e != cudaSuccess) return e;
    const int round = per_sm * sms, rest = round > 0 ? a.in.count % round : 0;
    Args tail = a;
    plan_cluster(tail.in, rest, sms);
    if (rest > 0 && rest < a.in.count && tail.in.cluster > 1) {
      Args whole = a;
      whole.in.count = a.in.count - rest;
      e = launch(whole);
      if (e != cudaSuccess) return e;
      tail.in.first = whole.in.count;
      tail.in.count = rest;
      tail.in.beside = 1;
      return launch(tail);
    }
  }
  return launch(a);
}
// Bytes of a row's logits.
template <typename T, int F>
long long row_bytes(const StreamRows& in) {
  return (long long)in.V * (int)sizeof(T) * (F ? 2 : 1);
}
// The row of a CTA, once it may begin; in.rows: the cluster that waits (and has).
__device__ __forceinline__ unsigned begin_row(const StreamRows& in) {
  const unsigned r = (unsigned)in.first + blockIdx.x / (unsigned)in.cluster;
  if (!in.beside || r == (unsigned)in.rows) pdl_wait();
  if (threadIdx.x == 0) pdl_trigger();
  return r;
}

// The kernel of a call: its logits' type, its rows' terms, and whether they lie alike
// against 16-byte boundaries. launch(type, terms, vec) takes them as types.
template <typename T>
struct TypeOf {
  using type = T;
};
template <typename Launch>
cudaError_t dispatch_rows(const StreamRows& in, bool f32, bool fused, bool vec, Launch&& launch) {
  const bool full = in.longp && in.shortp && in.prior;
  const auto with_terms = [&](auto type) {
    using std::integral_constant;
    if (!fused)
      return vec ? launch(type, integral_constant<int, kPlain>{}, std::true_type{})
                 : launch(type, integral_constant<int, kPlain>{}, std::false_type{});
    if (full && vec) return launch(type, integral_constant<int, kFull>{}, std::true_type{});
    return vec ? launch(type, integral_constant<int, kSome>{}, std::true_type{})
               : launch(type, integral_constant<int, kSome>{}, std::false_type{});
  };
  return f32 ? with_terms(TypeOf<float>{}) : with_terms(TypeOf<uint16_t>{});
}

}  // namespace dels
