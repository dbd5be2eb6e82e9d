// Distillation of the local head from a teacher's top entries, through the
// fusion: per row the Kullback-Leibler divergence of the student's
// q = softmax(l / T), l = (l_L + alpha l_S) - beta l_P, from the teacher's p over
// its listed ids i_k, and its gradient.
//
//   renormalised: p_k = softmax_k(t_k / T);        L = sum_k p_k (ln p_k - ln q_ik)
//                 dL/dl_v = (q_v - p_v) / T
//   with a tail:  p_k = exp t_k, p_t = 1 - sum p_k, q_t = sum of q over the others
//                 L = sum_k p_k (ln p_k - ln q_ik) + p_t (ln p_t - ln q_t)
//                 dL/dl_v = (q_v M - p_v) / T listed, q_v (M - p_t / q_t) / T others,
//                 M = sum_k p_k + p_t = 1 (sum_k p_k where it has passed 1 by rounding)
//   dL/dl_S = alpha dL/dl;  dL/dalpha = sum_v dL/dl_v l_S[v];  dL/dbeta = -sum_v dL/dl_v l_P[v]
//
// The listed ids are held out of the stream by a bitmap of the slice and summed
// apart, so that q_t is a sum of its own terms (1 - sum q_ik would lose its digits
// where the listed ids have nearly all mass), and the weights' gradients come from
// sums taken along with the softmax's: no pass over the rows is added for them.
//
// What bounds it, on fused rows of 151936: 1024 bf16 rows' loss takes 128 us (4.9 TB/s:
// instructions, see row_stream.cuh), their gradient 158 us (5.9 TB/s: the bytes), both as
// one step 287 us, 64 rows 31 to 34 us; 256 float32 rows 55, 81 and 142 us (5.7 and 5.8 TB/s).
// A row's bytes in one pass would be 3 s V: the step that reads once (GRAD below) is the
// faster one for few rows only, as distill_step_fits() says.
#include <algorithm>
#include <cfloat>

#include "row_stream.cuh"

namespace dels {

namespace {

enum { kFlagAny = 1, kFlagBadId = 2, kFlagBadLogit = 4, kFlagTwice = 8 };

// Sums of the columns that are not listed, relative to f, the reference of m, an entry
// among them: sum 2^z, sum 2^z (l_S - s_ref) and sum 2^z (l_P - p_ref). (A row's gradient
// sums to zero: what all its l_S, or all of l_P, have in common drops out of the weights'
// gradients, and would take its digits from them.)
struct TailRec {
  float m;
  Ref f;
  float sum, s, p;
};
// Those of the listed: m the largest, rest = sum 2^((l - m) c) without one that
// attains it (the student's whole mass may be there: ln(1 + rest) keeps its digits).
struct ListRec {
  float m, rest;
};
// What a warp has of a row.
struct __align__(16) WarpRec {
  TailRec t;
  ListRec l;
};
static_assert(sizeof(WarpRec) == 32, "two 16-byte words");

// A row's sums in units in which that of the columns that are not listed is from 1 to 2:
// the reference came from some of a row's first columns, 2^100 below others perhaps. What is
// asked of the sums (how far the listed ones are above them, 1 / (sum + listed)) is then
// asked of the sums and not of the reference. Scaled by powers of two: no digit changes.
__device__ __forceinline__ void settle(TailRec& t) {
  if (!(t.sum >= 2.f && t.sum < INFINITY)) return;        // 0: none; NaN: flagged later
  const int k = (int)(__float_as_uint(t.sum) >> 23) - 127;
  const float by = __uint_as_float((unsigned)(127 - k) << 23);
  t.f.r += (float)k;
  t.sum *= by;
  t.s *= by;
  t.p *= by;
}

// `n` records (at most 64) merged by a warp (all lanes converged), the result in
// every lane, in a fixed order.
__device__ __forceinline__ void merge_records(const WarpRec* recs, int n, float c, TailRec& t, ListRec& l) {
  const int lane = threadIdx.x & 31;
  const WarpRec none{TailRec{-INFINITY, Ref{0.f, 0.f}, 0.f, 0.f, 0.f}, ListRec{-INFINITY, 0.f}};
  const WarpRec a = lane < n ? recs[lane] : none;
  WarpRec b = none;
  if (n > 32) b = lane + 32 < n ? recs[lane + 32] : none;
  // not listed: the reference of the largest
  const bool second = b.t.m > a.t.m;
  const float m = second ? b.t.m : a.t.m;
  const Ref f = second ? b.t.f : a.t.f;
  t.m = warp_max(m);
  const int who = __ffs(__ballot_sync(0xFFFFFFFFu, m == t.m)) - 1;
  t.f.off = __shfl_sync(0xFFFFFFFFu, f.off, who);
  t.f.r = __shfl_sync(0xFFFFFFFFu, f.r, who);
  const float ka = a.t.m == -INFINITY ? 1.f : ex2_approx(ref_shift(a.t.f, t.f, c));   // (none: 0, or NaN, stays)
  const float kb = b.t.m == -INFINITY ? 1.f : ex2_approx(ref_shift(b.t.f, t.f, c));
  t.sum = ka * a.t.sum + kb * b.t.sum;
  t.s = ka * a.t.s + kb * b.t.s;
  t.p = ka * a.t.p + kb * b.t.p;
  // listed: one entry of the largest value stays out
  l.m = warp_max(fmaxf(a.l.m, b.l.m));
  const bool has = l.m > -INFINITY;
  const unsigned at_a = __ballot_sync(0xFFFFFFFFu, a.l.m == l.m), at_b = __ballot_sync(0xFFFFFFFFu, b.l.m == l.m);
  const bool out_a = lane == __ffs(at_a) - 1, out_b = at_a == 0u && lane == __ffs(at_b) - 1;
  const float la = a.l.m == -INFINITY ? 0.f : ex2_approx((a.l.m - l.m) * c);
  const float lb = b.l.m == -INFINITY ? 0.f : ex2_approx((b.l.m - l.m) * c);
  l.rest = (a.l.m == -INFINITY ? a.l.rest : la * a.l.rest) + (b.l.m == -INFINITY ? b.l.rest : lb * b.l.rest);
  if (has) l.rest += (out_a ? 0.f : la) + (out_b ? 0.f : lb);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    t.sum += __shfl_xor_sync(0xFFFFFFFFu, t.sum, d);
    t.s += __shfl_xor_sync(0xFFFFFFFFu, t.s, d);
    t.p += __shfl_xor_sync(0xFFFFFFFFu, t.p, d);
    l.rest += __shfl_xor_sync(0xFFFFFFFFu, l.rest, d);
  }
  settle(t);
}

// What three columns have in common: their middle value, 0 if that is masked by infinities or huge values.
__device__ __forceinline__ float middle(float a, float b, float c) {
  const float m = fmaxf(fminf(a, b), fminf(fmaxf(a, b), c));
  return fabsf(m) <= 0x1p96f ? m : 0.f;
}

// One lane's sums over the columns that are not listed, under its warp's reference:
// that of the largest entry of the warp's first items. Nothing else is compared: the
// sums' digits do not depend on the reference, and an entry 2^100 times as likely as
// those (or one that is not a number) shows in sums that are not below 2^100, which are
// then taken again (redo; the sums of a row's 64 warps together stay below 2^107). A
// running maximum took 10 instructions of an item's 100.
template <bool FUSED>
struct WarpTail {
  float m;             // the same in every lane, as f
  Ref f;
  f32x2 sum, s, p;
  __device__ __forceinline__ void init() {
    m = -INFINITY;
    f = Ref{0.f, 0.f};
    sum = s = p = 0ull;
  }
  // Whether there is a reference, and it is a whole number.
  __device__ __forceinline__ bool settled() const { return m > -INFINITY && f.off == 0.f; }
  // One item's values, all lanes converged: x becomes 2^z.
  template <bool SETTLED>
  __device__ __forceinline__ void push(float (&x)[8], const float (&sv)[8], const float (&pr)[8], float c,
                                       float s_ref, float p_ref) {
    if (!SETTLED) {
      if (m == -INFINITY) {
        m = warp_max(max8(x));
        if (m > -INFINITY) f = make_ref(m, c);
      }
      if (f.off != 0.f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] -= f.off;
      }
    }
    const f32x2 c2 = both2(c), nr = both2(-f.r), ns = both2(-s_ref), np = both2(-p_ref);
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      float z0, z1;
      split2(fma2(pair2(x[i], x[i + 1]), c2, nr), z0, z1);
      x[i] = ex2_approx(z0);
      x[i + 1] = ex2_approx(z1);
      const f32x2 e = pair2(x[i], x[i + 1]);
      sum = add2(sum, e);
      if constexpr (FUSED) {
        s = fma2(e, add2(pair2(sv[i], sv[i + 1]), ns), s);
        p = fma2(e, add2(pair2(pr[i], pr[i + 1]), np), p);
      }
    }
  }
  __device__ __forceinline__ TailRec record() const {
    TailRec r{m, f, sum2(sum), sum2(s), sum2(p)};
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      r.sum += __shfl_xor_sync(0xFFFFFFFFu, r.sum, d);
      if constexpr (FUSED) {
        r.s += __shfl_xor_sync(0xFFFFFFFFu, r.s, d);
        r.p += __shfl_xor_sync(0xFFFFFFFFu, r.p, d);
      }
    }
    return r;
  }
};
// Where those are not finite (a later entry far above the first ones, a masked l_S of
// -inf, an entry that is not a number): the warp's items again, element by element, the
// largest entry first. `kept`: the step's place of 2^z, or null.
//
// This is slow, without copies ahead and twice over. Loss of fused rows of 151936, us:
//                                               1024 bf16   64 bf16   256 float32
//   none of it                                     128         17          54
//   256 padded columns of -inf in l_S (a warp)    1090         63         360
//   3 % of l_S at -inf (all warps)                2440        184         612
//   the first 256 columns masked by -1e4           805         72          55
//   the first 2048 so                             2410        178         610
//   a temperature of 0.1                           396         67         300
// (Columns masked by -inf in l_L alone, or by the lowest finite value in l_S, cost nothing.)
template <typename T, int F, bool VEC>
__device__ __noinline__ TailRec redo_tail(const FusedRow<T, F, VEC>& row, int k0, int k1, const unsigned* bitmap,
                                          float* kept, float c, float s_ref, float p_ref) {
  const int items = (k1 - k0 + kStreamStep - 1) / kStreamStep, tid = threadIdx.x;
  auto value = [&](int it, int i, int& q) {
    q = elem_pos<T, VEC>(item_pos<T, VEC>(k0, it, tid), i);
    const bool in = q >= row.sh && q < k1 && !(bitmap[(q - k0) >> 5] >> ((q - k0) & 31) & 1u);
    return in ? row.contracted(row.l_at(q), row.s_at(q), row.p_at(q)) : -INFINITY;
  };
  int q;
  float m = -INFINITY;
  for (int it = 0; it < items; ++it)
    for (int i = 0; i < 8; ++i) m = fmaxf(m, value(it, i, q));
  TailRec r{warp_max(m), Ref{0.f, 0.f}, 0.f, 0.f, 0.f};
  if (r.m > -INFINITY) r.f = make_ref(r.m, c);
  for (int it = 0; it < items; ++it)
    for (int i = 0; i < 8; ++i) {
      const float x = value(it, i, q), e = ex2_approx(ref_z(x, r.f, c));
      r.sum += e;
      if (F && e != 0.f) {                     // (masked: neither l_S nor l_P counts)
        r.s += e * (row.s_at(q) - s_ref);
        r.p += e * (row.p_at(q) - p_ref);
      }
      if (kept) kept[((it * 2 + (i >> 2)) * kStreamThreads + tid) * 4 + (i & 3)] = e;
    }
  for (int d = 16; d > 0; d >>= 1) {
    r.sum += __shfl_xor_sync(0xFFFFFFFFu, r.sum, d);
    r.s += __shfl_xor_sync(0xFFFFFFFFu, r.s, d);
    r.p += __shfl_xor_sync(0xFFFFFFFFu, r.p, d);
  }
  return r;
}

// Copies ahead of the loss and gradient kernels, and of the step's, whose items stay: only
// fused float32 rows have a ring beside them, of 32 KB, which with 8 items (66 KB) leaves
// room for a second CTA on the SM and with 10 does not.
template <typename T, int F>
using LossCopies = std::conditional_t<F == kPlain, Copies<T, F, sizeof(T) == 2 ? 4 : 2, 2>,
                                      Copies<T, F, 2, sizeof(T) == 2 ? 3 : 2>>;
template <typename T, int F>
using StepCopies = Copies<T, F, 2, sizeof(T) == 4 && F ? 2 : 4, true>;
template <typename T, int F, bool GRAD>
using RowCopies = std::conditional_t<GRAD, StepCopies<T, F>, LossCopies<T, F>>;

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  uint32_t w;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  return w;
}
__device__ __forceinline__ void grad_elem(float* g, long long i, float v) { g[i] = v; }
__device__ __forceinline__ void grad_elem(uint16_t* g, long long i, float v) { g[i] = (uint16_t)bf16_pair(v, 0.f); }
__device__ __forceinline__ void grad_vec(float* g, const float (&v)[8]) {
  __stcs(reinterpret_cast<float4*>(g), make_float4(v[0], v[1], v[2], v[3]));
  __stcs(reinterpret_cast<float4*>(g + kHalf<float>), make_float4(v[4], v[5], v[6], v[7]));
}
__device__ __forceinline__ void grad_vec(uint16_t* g, const float (&v)[8]) {
  __stcs(reinterpret_cast<uint4*>(g),
         make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])));
}
// An item's gradient at position k of a row whose position 0 is at g; vec: the
// gradient's rows lie like the logits' against 16-byte boundaries.
template <typename T, bool VEC>
__device__ __forceinline__ void grad_item(T* g, int k, int begin, int stop, bool vec, const float (&v)[8]) {
  if (VEC && vec && k >= begin && k + kHalf<T> + 4 <= stop) {
    grad_vec(g + k, v);
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int q = elem_pos<T, VEC>(k, i);
    if (q >= begin && q < stop) grad_elem(g, q, v[i]);
  }
}
// g = k 2^z of 8 values.
__device__ __forceinline__ void unlisted_grad(float (&x)[8], const Ref& f, float c, float k, float (&g)[8]) {
  if (f.off != 0.f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] -= f.off;
  }
  const f32x2 c2 = both2(c), nr = both2(-f.r), k2 = both2(k);
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    float z0, z1;
    split2(fma2(pair2(x[i], x[i + 1]), c2, nr), z0, z1);
    split2(mul2(k2, pair2(ex2_approx(z0), ex2_approx(z1))), g[i], g[i + 1]);
  }
}

// The teacher's side of a row.
struct Teacher {
  float t_max, t_scale, log_norm;   // ln p_k = (t_k - t_max) t_scale - log_norm
  float sum, rest;                  // sum p_k; 1 - sum p_k where there is a tail
};

struct LossShared {
  WarpRec recs[kMaxCluster * kStreamWarps];        // every warp's of the cluster
  float4 sums[kMaxCluster * kStreamWarps];         // first CTA: their shares of the row's loss and weights' gradients
  float2 red[kStreamWarps];
  float logit[kMaxTopK];            // the teacher's as stored; -inf: left out
  Teacher teacher;
  int flags;
};

// One warp: the teacher's normaliser, or its tail. 1 - sum p_k is taken from what
// the largest entry leaves of 1 (-expm1): its digits outlast a sum next to 1.
__device__ __forceinline__ void teacher_side(LossShared& sh, int K, bool tail, float inv_t) {
  const int lane = threadIdx.x & 31;
  float top = -INFINITY;
  for (int k = lane; k < K; k += 32) top = fmaxf(top, sh.logit[k]);
  top = warp_max(top);
  int first = kMaxTopK;
  for (int k = lane; k < K; k += 32)
    if (sh.logit[k] == top) first = min(first, k);
  first = __reduce_min_sync(0xFFFFFFFFu, first);
  const float shift = tail ? 0.f : top, scale = tail ? 1.f : inv_t;
  float others = 0.f;                              // without the first of the largest
  for (int k = lane; k < K; k += 32) {
    const float t = sh.logit[k];
    if (t > -INFINITY && k != first) others += expf((t - shift) * scale);
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) others += __shfl_xor_sync(0xFFFFFFFFu, others, d);
  if (lane == 0) {
    Teacher& te = sh.teacher;
    te.t_max = shift;
    te.t_scale = scale;
    te.log_norm = tail ? 0.f : log1pf(others);
    te.sum = tail ? expf(top) + others : 1.f;
    te.rest = tail ? fmaxf(-expm1f(top) - others, 0.f) : 0.f;
  }
}

// The student's sums of a row: S = sum over all columns = listed + not listed, in units
// of the reference f of those that are not listed (of the largest listed where there
// are none), and with the teacher's side dL/dl of a column that is not listed:
//   (M - p_t / q_t) q = (M / S - p_t / sum) 2^z = factor 2^z,   q_t = sum / S.
struct RowSums {
  Ref f;
  float z_l;        // of the largest listed; -inf: none
  float list_sum;   // the listed ones' (may be infinite: the others then have nothing)
  float factor, mass;
  bool has_tail, ok;
  __device__ __forceinline__ RowSums(const TailRec& t, const ListRec& l, const Teacher& te, bool tail, float c) {
    f = t.m == -INFINITY ? make_ref(l.m, c) : t.f;
    const bool none = l.m == -INFINITY;
    z_l = none ? -INFINITY : ref_z(l.m, f, c);
    list_sum = none ? l.rest : (1.f + l.rest) * ex2_approx(z_l);
    has_tail = tail && te.rest > 0.f && t.sum > 0.f;
    mass = has_tail ? 1.f : te.sum;
    factor = __fdividef(mass, t.sum + list_sum) - (has_tail ? __fdividef(te.rest, t.sum) : 0.f);
    const float top = fmaxf(t.m, l.m);
    ok = top > -INFINITY && top < INFINITY && t.sum >= 0.f && t.sum < INFINITY && l.rest >= 0.f && l.rest < INFINITY;
  }
};
// And its logarithms: ln q = (l - base) / T - base_ln, from the largest listed entry,
// whose digits that keeps, unless the others are far above it.
struct RowLogs {
  float base, base_ln;
  __device__ __forceinline__ RowLogs(const TailRec& t, const ListRec& l, const RowSums& s) {
    const bool from_list = l.m > -INFINITY && s.z_l >= -20.f;
    base = from_list ? l.m : s.f.off;
    base_ln = from_list ? log1pf(l.rest + t.sum * ex2_approx(-s.z_l)) : s.f.r * kLn2 + logf(t.sum + s.list_sum);
  }
};
// ln q_t = -ln(1 + list_sum / sum)
__device__ __forceinline__ float tail_ln(const TailRec& t, const ListRec& l, const RowSums& s) {
  return s.z_l > 60.f ? -(s.z_l * kLn2 + logf((1.f + l.rest) / t.sum)) : -log1pf(s.list_sum / t.sum);
}

// q M - p of a listed id from its logarithms: where p and q are next to 1 and to
// each other their difference keeps its digits.
__device__ __forceinline__ float listed_grad(float lq, float lp, float mass) {
  const float p = expf(lp), d = lq - lp;
  return d < 1.f ? p * expm1f(d) + expf(lq) * (mass - 1.f) : expf(lq) * mass - p;
}

// Sums over the rows of each weight, in a fixed order, by a whole CTA of NT threads
// (the rows' records past L1: other CTAs of the grid may have written them).
template <int NT>
__device__ void weight_grads(const DistillArgs& a, int j, float2* red) {
  const int n = a.in.n_weights;
  float da = 0.f, db = 0.f;
  for (long long r = j + (long long)threadIdx.x * n; r < a.in.rows; r += (long long)NT * n) {
    const float g = a.grad_loss ? a.grad_loss[r] : 1.f;
    const float2 d = __ldcg(reinterpret_cast<const float2*>(&a.state[r].d_alpha));
    if (__ldcg(&a.state[r].weight) != 0.f) {
      da += g * d.x;
      db += g * d.y;
    }
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    da += __shfl_xor_sync(0xFFFFFFFFu, da, d);
    db += __shfl_xor_sync(0xFFFFFFFFu, db, d);
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) {
    red[threadIdx.x >> 5] = make_float2(da, db);
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    da = db = 0.f;
    for (int k = 0; k < NT / 32; ++k) {
      da += red[k].x;
      db += red[k].y;
    }
    if (a.grad_alpha) a.grad_alpha[j] = da;
    if (a.grad_beta) a.grad_beta[j] = db;
  }
}

// The first CTA of a row's cluster, when the row is done: the last row of the grid
// sums the gradients of up to kTicketWeights weights (its count starts the next call at zero).
__device__ __forceinline__ void finish_rows(const DistillArgs& a, LossShared& sh) {
  if (!a.grad_alpha && !a.grad_beta) return;
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    sh.flags = atomicAdd(a.ticket, 1) == a.in.rows - 1;
  }
  __syncthreads();
  if (!sh.flags) return;
  __threadfence();
  for (int j = 0; j < a.in.n_weights; ++j) weight_grads<kStreamThreads>(a, j, sh.red);
  if (threadIdx.x == 0) *a.ticket = 0;
}

// Gradients of listed ids where some are listed twice (all threads): an id's last
// entry writes the sum of all its entries', in their order. `g`: of the calling
// thread's entry.
template <typename T>
__device__ void twice_grads(const DistillArgs& a, LossShared& sh, long long r, bool mine, int id, float g, T* out) {
  __syncthreads();
  if (threadIdx.x < kMaxTopK) sh.logit[threadIdx.x] = g;     // (the teacher's are not needed any more)
  __syncthreads();
  if (!mine) return;
  float sum = 0.f;
  for (int k = 0; k < a.K; ++k) {
    if (__ldg(a.ids + r * a.K + k) != id || __ldg(a.teacher + r * a.K + k) == -INFINITY) continue;
    if (k > (int)threadIdx.x) return;
    sum += sh.logit[k];
  }
  grad_elem(out, 0, sum);
}

// Loss and statistics of the rows, a cluster per row, a slice per CTA; GRAD: and
// the gradient of l_S. The slice's 2^z then stay in shared memory between the pass that
// sums them and the one that scales them, so that the rows are read once: 3 s V bytes
// a row instead of 5 s V. Each thread reads back what it wrote itself.
template <typename T, int F, bool VEC, bool GRAD>
__global__ void __launch_bounds__(kStreamThreads, (GRAD ? 2 : 3) - kFewer<T, F>) k_distill_loss(DistillArgs a) {
  extern __shared__ __align__(16) unsigned bitmap[];   // one bit per position of the slice: listed
  __shared__ LossShared sh;
  const long long r = begin_row(a.in);
  if (r == a.in.rows) return;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int C = a.in.cluster, K = a.K, V = a.in.V;
  const int rank = (int)(blockIdx.x & (C - 1));
  const float c = a.in.scale, inv_t = a.in.inv_t;
  const float weight = a.row_weight ? __ldg(a.row_weight + r) : 1.f;
  // thread k has entry k (kMaxTopK <= kStreamThreads)
  int id = -1;
  float logit = -INFINITY;
  if (tid < K) {
    id = __ldg(a.ids + r * K + tid);
    logit = __ldg(a.teacher + r * K + tid);
  }
  using Cp = RowCopies<T, F, GRAD>;
  const int words = (a.in.slice_cols + Cp::U * kStreamStep - 1) / (Cp::U * kStreamStep) * (Cp::U * kStreamStep / 128);
  uint8_t* ring = reinterpret_cast<uint8_t*>(bitmap + words * 4);
  uint8_t* kept = ring + (VEC ? Cp::kRingBytes : 0);           // GRAD: the slice's values, 32 bytes an item
  RowStream<Cp, T, F, VEC> stream(a.in, r, rank, ring, kept);
  const FusedRow<T, F, VEC>& row = stream.row;
  const int k0 = stream.k0, k1 = stream.k1;
  // (looked at when the copies are under way: before them their latency came on top, 64 bf16 rows 18.9, 18.5 us)
  float s_some[3] = {0.f, 0.f, 0.f}, p_some[3] = {0.f, 0.f, 0.f};
  if (weight != 0.f) {
    if constexpr (F != kPlain) {
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        const int at = row.sh + (i == 0 ? V / 4 : i == 1 ? V / 2 : V - 1 - V / 4);
        s_some[i] = row.s_at(at);
        p_some[i] = row.p_at(at);
      }
    }
    stream.begin();
  }
  T* out = nullptr;                                // the row's gradient at position 0
  if constexpr (GRAD) out = static_cast<T*>(a.grad) + r * a.ld_grad - row.sh;

  for (int i = tid; i < words; i += kStreamThreads) reinterpret_cast<uint4*>(bitmap)[i] = make_uint4(0u, 0u, 0u, 0u);
  if (tid == 0) sh.flags = 0;
  unsigned flags = 0u;
  if (tid < K) {
    if (id >= V) flags |= kFlagBadId;
    else if (id >= 0 && !(logit < INFINITY)) flags |= kFlagBadLogit;
    if (id < 0 || id >= V || logit == -INFINITY) {
      id = -1;
      logit = -INFINITY;
    } else {
      flags |= kFlagAny;
    }
    sh.logit[tid] = logit;
  }
  const int at = id + row.sh - k0;                 // its place in the slice
  const bool mine = id >= 0 && at >= 0 && at < k1 - k0;
  __syncthreads();
  if (mine) {
    const unsigned bit = 1u << (at & 31);
    if (atomicOr(&bitmap[at >> 5], bit) & bit) flags |= kFlagTwice;
  }
  if (warp * 32 < K) {
    flags = __reduce_or_sync(0xFFFFFFFFu, flags);
    if (lane == 0 && flags) atomicOr(&sh.flags, (int)flags);
  }
  __syncthreads();
  flags = (unsigned)sh.flags;
  if (weight == 0.f || !(flags & (kFlagAny | kFlagBadLogit))) {     // left out
    stream.drain();
    if constexpr (GRAD) {
      const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      for (int it = 0; it < stream.items; ++it)
        grad_item<T, VEC>(out, item_pos<T, VEC>(k0, it, tid), row.sh, k1, a.grad_vec, zero);
    }
    if (rank == 0 && tid == 0) {
      if (weight != 0.f && (flags & kFlagBadId)) raise_status(a.status, DELS_STATUS_BAD_TOKEN);
      if (a.out_loss) a.out_loss[r] = 0.f;
      a.state[r] = DistillState{};
    }
    if constexpr (GRAD) {
      if (rank == 0) finish_rows(a, sh);
    }
    return;
  }
  if (C > 1) cluster_arrive_relaxed();
  float l_k = -INFINITY, s_k = 0.f, p_k = 0.f;     // the listed column's terms
  if (mine) {
    l_k = row.l_at(k0 + at);
    s_k = row.s_at(k0 + at);
    p_k = row.p_at(k0 + at);
  }
  if (warp == kStreamWarps - 1) teacher_side(sh, K, a.tail != 0, inv_t);

  const float s_ref = middle(s_some[0], s_some[1], s_some[2]);
  const float p_ref = middle(p_some[0], p_some[1], p_some[2]);
  // the columns that are not listed
  WarpTail<F != kPlain> st;
  st.init();
  float pa[8], pb[8];
  const unsigned char* bits8 = reinterpret_cast<const unsigned char*>(bitmap);
  const auto item_of = [&](auto& v, auto& pr, int it, auto settled) {
    float x[8], s[8];
    v.template values<true>(row, pr, x, s);
    if constexpr (VEC) {
      // the item's 8 bits (positions past the slice are -inf already, their bits 0)
      unsigned bits;
      if constexpr (sizeof(T) == 2) {
        bits = bits8[it * kStreamThreads + tid];
      } else {
        const unsigned lo = bits8[(it * 2) * (kStreamThreads / 2) + (tid >> 1)];
        const unsigned hi = bits8[(it * 2 + 1) * (kStreamThreads / 2) + (tid >> 1)];
        bits = (lo >> (tid & 1) * 4 & 15u) | (hi >> (tid & 1) * 4 & 15u) << 4;
      }
      if (bits) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (bits >> i & 1u) x[i] = -INFINITY;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int b = elem_pos<T, VEC>(v.k, i) - k0;
        if (bitmap[b >> 5] >> (b & 31) & 1u) x[i] = -INFINITY;
      }
    }
    st.template push<decltype(settled)::value>(x, s, pr, c, s_ref, p_ref);
    if constexpr (GRAD) {
      float4* keep = reinterpret_cast<float4*>(kept) + it * (2 * kStreamThreads) + tid;
      keep[0] = make_float4(x[0], x[1], x[2], x[3]);
      keep[kStreamThreads] = make_float4(x[4], x[5], x[6], x[7]);
    }
  };
  const auto any_of = [&](auto& v, auto& pr, int it) { item_of(v, pr, it, std::false_type{}); };
  const auto settled_of = [&](auto& v, auto& pr, int it) { item_of(v, pr, it, std::true_type{}); };
  stream.run(
      [&](int g) {
        if (st.settled()) stream.each(g, pa, pb, settled_of);
        else stream.each(g, pa, pb, any_of);
      },
      any_of);
  WarpRec rec{st.record(), ListRec{-INFINITY, 0.f}};
  if (!(fabsf(rec.t.sum) + fabsf(rec.t.s) + fabsf(rec.t.p) < 0x1p100f)) {
    const FusedRow<T, F, VEC> its = stream.anew();   // (the call takes its address: the stream's stays in registers)
    rec.t = redo_tail<T, F, VEC>(its, k0, k1, bitmap, GRAD ? reinterpret_cast<float*>(kept) : nullptr, c, s_ref, p_ref);
  }

  // the listed columns of this slice; an id listed twice counts once in the student's sums
  bool once = mine;
  const float x_k = mine ? row.contracted(l_k, s_k, p_k) : -INFINITY;
  if (__any_sync(0xFFFFFFFFu, mine)) {
    if (mine && (flags & kFlagTwice))
      for (int k = 0; k < tid; ++k)
        if (sh.logit[k] > -INFINITY && __ldg(a.ids + r * K + k) == id) once = false;
    rec.l.m = warp_max(once && x_k == x_k ? x_k : -INFINITY);
    const unsigned who = __ballot_sync(0xFFFFFFFFu, once && x_k == rec.l.m && rec.l.m > -INFINITY);
    float e = 0.f;
    if (once && x_k != -INFINITY && lane != __ffs(who) - 1) e = ex2_approx((x_k - rec.l.m) * c);
    if (once && x_k != x_k) e = NAN;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) e += __shfl_xor_sync(0xFFFFFFFFu, e, d);
    rec.l.rest = e;
  }
  // every warp's record to every CTA of the cluster
  if (C > 1) {
    cluster_wait();                // every CTA of the cluster runs before its shared memory is written
    if (lane < C) {
      const uint32_t to = cluster_map(smem_u32(&sh.recs[rank * kStreamWarps + warp]), (uint32_t)lane);
      st_cluster_v4(to, rec.t.m, rec.t.f.off, rec.t.f.r, rec.t.sum);
      st_cluster_v4(to + 16, rec.t.s, rec.t.p, rec.l.m, rec.l.rest);
    }
    __syncwarp();
    cluster_sync_all();
  } else {
    if (lane == 0) sh.recs[warp] = rec;
    __syncthreads();
  }
  TailRec tail;
  ListRec listed;
  merge_records(sh.recs, C * kStreamWarps, c, tail, listed);
  const Teacher te = sh.teacher;
  const RowSums sums(tail, listed, te, a.tail != 0, c);
  const bool ok = sums.ok && !(flags & kFlagBadLogit);
  const float up = weight * inv_t * (F ? row.a : 1.f);   // dL/dl -> what the gradient holds
  // the listed columns' share of the loss and of the weights' gradients, to the first CTA
  float g_k = 0.f;
  if (warp * 32 < K) {
    float v[3] = {0.f, 0.f, 0.f};
    if (__any_sync(0xFFFFFFFFu, mine)) {
      const RowLogs logs(tail, listed, sums);
      if (mine) {
        const float lp = (logit - te.t_max) * te.t_scale - te.log_norm, p = expf(lp);
        const float lq = (x_k - logs.base) * inv_t - logs.base_ln;
        const float g = once ? listed_grad(lq, lp, sums.mass) : -p;
        v[0] = p > 0.f ? p * (lp - lq) : 0.f;
        v[1] = g * (fmaxf(s_k, -FLT_MAX) - s_ref);
        v[2] = g * (p_k - p_ref);
        g_k = ok ? up * g : NAN;
      }
#pragma unroll
      for (int d = 16; d > 0; d >>= 1)
#pragma unroll
        for (int j = 0; j < 3; ++j) v[j] += __shfl_xor_sync(0xFFFFFFFFu, v[j], d);
    }
    if (lane == 0) {
      float4* to = &sh.sums[rank * kStreamWarps + warp];
      if (C > 1) st_cluster_v4(cluster_map(smem_u32(to), 0), v[0], v[1], v[2], 0.f);
      else *to = make_float4(v[0], v[1], v[2], 0.f);
    }
  }
  __syncwarp();
  // (before the gradient is written: the arrival waits for every store before it)
  if (C > 1) cluster_arrive();
  if constexpr (GRAD) {
    // this warp's 2^z are relative to its own reference, perhaps far below the row's: brought to
    // the row's first, where at most 1 is left of them, then multiplied (their factors' product alone
    // may leave the range)
    const float d = rec.t.m > -INFINITY ? ref_shift(rec.t.f, sums.f, c) : 0.f, d1 = fmaxf(d, -100.f);
    const f32x2 unit = both2(ex2_approx(d1)), kk = both2(ok ? up * sums.factor * ex2_approx(d - d1) : NAN);
    const float4* got = reinterpret_cast<const float4*>(kept) + tid;
#pragma unroll 2
    for (int it = 0; it < stream.items; ++it) {
      const float4 y = got[it * 2 * kStreamThreads], w = got[(it * 2 + 1) * kStreamThreads];
      float gr[8];
      split2(mul2(kk, mul2(unit, pair2(y.x, y.y))), gr[0], gr[1]);
      split2(mul2(kk, mul2(unit, pair2(y.z, y.w))), gr[2], gr[3]);
      split2(mul2(kk, mul2(unit, pair2(w.x, w.y))), gr[4], gr[5]);
      split2(mul2(kk, mul2(unit, pair2(w.z, w.w))), gr[6], gr[7]);
      grad_item<T, VEC>(out, item_pos<T, VEC>(k0, it, tid), row.sh, k1, a.grad_vec, gr);
    }
  }

  if (GRAD || C == 1) __syncthreads();             // the unlisted columns' gradients are written
  if constexpr (GRAD) {
    if (flags & kFlagTwice) twice_grads(a, sh, r, mine, id, g_k, out + k0 + at);
    else if (mine) grad_elem(out, k0 + at, g_k);
  }
  if (rank != 0) return;
  if (C > 1) cluster_wait();
  if (warp == 0) {
    float v[3] = {0.f, 0.f, 0.f};
    for (int i = lane; i < C * kStreamWarps; i += 32) {
      if ((i & (kStreamWarps - 1)) * 32 >= K) continue;
      const float4 q = sh.sums[i];
      v[0] += q.x;
      v[1] += q.y;
      v[2] += q.z;
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1)
#pragma unroll
      for (int j = 0; j < 3; ++j) v[j] += __shfl_xor_sync(0xFFFFFFFFu, v[j], d);
    if (lane == 0) {
      if (!ok) raise_status(a.status, DELS_STATUS_NONFINITE);
      if (flags & kFlagBadId) raise_status(a.status, DELS_STATUS_BAD_TOKEN);
      const RowLogs logs(tail, listed, sums);
      float loss = v[0];
      if (sums.has_tail)
        loss += te.rest * ((te.rest > 0.5f ? log1pf(-te.sum) : logf(te.rest)) - tail_ln(tail, listed, sums));
      if (a.out_loss) a.out_loss[r] = ok ? weight * loss : NAN;
      DistillState o{};
      o.f_off = sums.f.off;
      o.f_r = sums.f.r;
      o.factor = ok ? sums.factor : NAN;
      o.base = logs.base;
      o.base_ln = logs.base_ln;
      o.mass = ok ? sums.mass : NAN;
      o.t_max = te.t_max;
      o.t_scale = te.t_scale;
      o.log_norm = te.log_norm;
      o.weight = weight;
      o.d_alpha = ok ? weight * inv_t * (sums.factor * tail.s + v[1]) : NAN;
      o.d_beta = ok ? -weight * inv_t * (sums.factor * tail.p + v[2]) : NAN;
      a.state[r] = o;
    }
  }
  if constexpr (GRAD) finish_rows(a, sh);
}

// The gradient of l_S from the statistics: every column as one that is not listed,
// then the listed ones over it. The rows' own logits may be the output (each column
// is read before it is written).
template <typename T, int F, bool VEC>
__global__ void __launch_bounds__(kStreamThreads, 3 - kFewer<T, F>) k_distill_grad(DistillArgs a) {
  extern __shared__ __align__(16) uint8_t ring[];
  const long long r = begin_row(a.in);
  if (r == a.in.rows) return;
  const int tid = threadIdx.x;
  const int C = a.in.cluster, K = a.K;
  const int rank = (int)(blockIdx.x & (C - 1));
  RowStream<LossCopies<T, F>, T, F, VEC> stream(a.in, r, rank, ring, nullptr);
  const FusedRow<T, F, VEC>& row = stream.row;
  const int k0 = stream.k0, k1 = stream.k1, items = stream.items;
  const DistillState st = a.state[r];
  const float up = a.grad_loss ? __ldg(a.grad_loss + r) : 1.f;
  T* out = static_cast<T*>(a.grad) + r * a.ld_grad - row.sh;
  if (st.weight == 0.f) {                          // left out
    const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int it = 0; it < items; ++it)
      grad_item<T, VEC>(out, item_pos<T, VEC>(k0, it, tid), row.sh, k1, a.grad_vec, zero);
    return;
  }
  const float g0 = up * st.weight * a.in.inv_t * (F ? row.a : 1.f);
  const float c = a.in.scale;
  stream.begin();

  // thread k has entry k: its logit is read before it may be written over
  __shared__ int ids[kMaxTopK];                    // -1: none of this slice
  __shared__ float probs[kMaxTopK];
  int id = -1;
  float lp = 0.f, x_k = 0.f;
  if (tid < K) {
    id = __ldg(a.ids + r * K + tid);
    const float t = __ldg(a.teacher + r * K + tid);
    if (id < 0 || id + row.sh < k0 || id + row.sh >= k1 || t == -INFINITY) id = -1;
    if (id >= 0) {
      lp = (t - st.t_max) * st.t_scale - st.log_norm;
      x_k = row.contracted(row.l_at(id + row.sh), row.s_at(id + row.sh), row.p_at(id + row.sh));
      probs[tid] = expf(lp);
    }
    ids[tid] = id;
  }
  __syncthreads();                                 // the output may be l_S itself
  const float k2 = g0 * st.factor;
  const Ref f{st.f_off, st.f_r};
  float pa[8], pb[8];
  const auto item_of = [&](auto& v, auto& pr, int) {
    float x[8], s[8], g[8];
    v.template values<true>(row, pr, x, s);
    unlisted_grad(x, f, c, k2, g);
    grad_item<T, VEC>(out, v.k, row.sh, k1, a.grad_vec, g);
  };
  stream.run([&](int g) { stream.each(g, pa, pb, item_of); }, item_of);
  __syncthreads();                                 // the columns as ones that are not listed are written
  if (id < 0) return;
  // every entry with this id, in their order; the last of them writes
  float before = 0.f;
  for (int k = 0; k < K; ++k) {
    if (ids[k] != id || k == tid) continue;
    if (k > tid) return;
    before += probs[k];
  }
  const float lq = (x_k - st.base) * a.in.inv_t - st.base_ln;
  grad_elem(out, id + row.sh, g0 * (listed_grad(lq, lp, st.mass) - before));
}

__global__ void __launch_bounds__(256) k_weight_grads(DistillArgs a) {
  __shared__ float2 red[8];
  pdl_wait();
  if (threadIdx.x == 0) pdl_trigger();
  weight_grads<256>(a, blockIdx.x, red);
}

// Shared memory of the loss kernel: the bitmap (of whole groups of items), the ring,
// and with GRAD the slice's values.
template <typename Cp>
size_t loss_items(const StreamRows& in) {
  return ((size_t)in.slice_cols + Cp::U * kStreamStep - 1) / (Cp::U * kStreamStep) * Cp::U;
}
template <typename T, int F, bool VEC, bool GRAD>
size_t loss_smem(const StreamRows& in) {
  using Cp = RowCopies<T, F, GRAD>;
  const size_t items = loss_items<Cp>(in);
  return items * (kStreamStep / 8) + (VEC ? Cp::kRingBytes : 0) + (GRAD ? items * kStreamStep * 4 : 0);
}

// Rows from which a round of CTAs that is not full is split (launch_rows), us without
// and with: 608 rows of 256 KB (65536 fused bf16) 40.6, 37.4 and the gradient 57.6,
// 53.1; of 128 KB (the same alone) 16.9, 17.3. The loss of float32 rows is not: its
// reads fill the time as they are (500 fused of 151936: 109, 119; their gradient 170, 145).
constexpr int kSplitBytes = 1 << 18;

template <typename T, int F, bool VEC, bool GRAD>
cudaError_t launch_loss_t(const DistillArgs& a, cudaStream_t s) {
  const auto k = k_distill_loss<T, F, VEC, GRAD>;
  const bool split = sizeof(T) == 2 && row_bytes<T, F>(a.in) >= kSplitBytes;
  return launch_rows(k, a, true, split, loss_smem<T, F, VEC, GRAD>, s);
}

template <typename T, int F, bool VEC>
cudaError_t launch_grad_t(const DistillArgs& a, cudaStream_t s) {
  const auto k = k_distill_grad<T, F, VEC>;
  const size_t bytes = VEC ? LossCopies<T, F>::kRingBytes : 0;
  return launch_rows(k, a, false, row_bytes<T, F>(a.in) >= kSplitBytes, [&](const StreamRows&) { return bytes; }, s);
}

}  // namespace

cudaError_t launch_distill_loss(const DistillArgs& a, bool f32, bool fused, bool vec, cudaStream_t s) {
  return dispatch_rows(a.in, f32, fused, vec, [&](auto t, auto f, auto v) {
    return launch_loss_t<typename decltype(t)::type, decltype(f)::value, decltype(v)::value, false>(a, s);
  });
}
cudaError_t launch_distill_step(const DistillArgs& a, bool f32, bool fused, bool vec, cudaStream_t s) {
  return dispatch_rows(a.in, f32, fused, vec, [&](auto t, auto f, auto v) {
    return launch_loss_t<typename decltype(t)::type, decltype(f)::value, decltype(v)::value, true>(a, s);
  });
}
// Whether the step reads its rows once (k_distill_loss with GRAD, a launch less) or
// twice (k_distill_loss, then k_distill_grad). Once needs room for the slice's 2^z
// beside the ring, and with it few CTAs share an SM: 1 to 3, which hide less of a CTA's
// start and exchange than the 3 to 6 of the two launches. us, once against twice, the
// gradients of 16 weights among them:
//   one round of CTAs     24 bf16 rows of 151936: 12.6, 19.5 fused; 8.8, 14.8 plain
//   more, fused bf16      40: 22.7, 23.1; 160: 59.8, 58.7; 1024: 327, 279
//   up to two, plain bf16 57: 15.5, 22.5; 100 of 100003: 18.5, 27.9 (but 76 of 151936, 24.4,
//                         19.8); more: 160: 37.3, 34.0; 600: 129, 98
//   float32, two on an SM 160 of 100003: 64, 80 fused; 600: 115, 139 plain
//   float32, one on an SM 256 of 151936 fused: 174, 141
bool distill_step_fits(const DistillArgs& a, bool f32, bool fused, bool vec, int sms) {
  size_t bytes = 0;
  int per_sm = 0;
  dispatch_rows(a.in, f32, fused, vec, [&](auto t, auto f, auto v) {
    using T = typename decltype(t)::type;
    constexpr int F = decltype(f)::value;
    bytes = loss_smem<T, F, decltype(v)::value, true>(a.in);
    per_sm = std::min((F ? 2 : 3) - kFewer<T, F>, (int)((228u << 10) / (bytes + 1024)));
    return cudaSuccess;
  });
  if (bytes > (size_t)kStepSmemBytes) return false;
  if (f32 && per_sm >= 2) return true;
  const long long ctas = (long long)a.in.rows * a.in.cluster, round = (long long)sms * per_sm;
  return fused ? ctas * 5 <= round * 4 : ctas <= round * 2;
}
cudaError_t launch_distill_grad(const DistillArgs& a, bool f32, bool fused, bool vec, cudaStream_t s) {
  return dispatch_rows(a.in, f32, fused, vec, [&](auto t, auto f, auto v) {
    return launch_grad_t<typename decltype(t)::type, decltype(f)::value, decltype(v)::value>(a, s);
  });
}
cudaError_t launch_weight_grads(const DistillArgs& a, cudaStream_t s) {
  return launch_pdl(k_weight_grads, dim3((unsigned)a.in.n_weights), dim3(256), 0, s, a);
}

}  // namespace dels
