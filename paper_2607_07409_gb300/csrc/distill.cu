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
// What bounds it: the rows' bytes (read both, write the gradient).
#include <cfloat>

#include "row_stream.cuh"

namespace dels {

namespace {

enum { kFlagAny = 1, kFlagBadId = 2, kFlagBadLogit = 4, kFlagTwice = 8 };

// Sums of the columns that are not listed, relative to m: `rest` without one entry
// that attains m, s = sum 2^t l_S and p = sum 2^t (l_P - ref) over all of them.
struct TailRec {
  float m, rest, s, p;
};
__device__ __forceinline__ void tail_add(TailRec& r, const TailRec& b, float c, bool stays_out) {
  const float f = b.m == -INFINITY ? (b.rest != b.rest ? NAN : 0.f) : ex2_approx((b.m - r.m) * c);
  r.rest += f * b.rest + (b.m == -INFINITY || stays_out ? 0.f : f);
  r.s += f * b.s;
  r.p += f * b.p;
}
__device__ __forceinline__ TailRec tail_merge(const TailRec& a, const TailRec& b, float c) {
  TailRec r{fmaxf(a.m, b.m), 0.f, 0.f, 0.f};
  tail_add(r, a, c, a.m >= b.m);
  tail_add(r, b, c, a.m < b.m);
  return r;
}

// The teacher's side of a row.
struct Teacher {
  float t_max, t_scale, log_norm;   // ln p_k = (t_k - t_max) t_scale - log_norm
  float sum, rest;                  // sum p_k; 1 - sum p_k where there is a tail
};

struct LossShared {
  TailRec warps[kStreamWarps];
  float members[kStreamWarps][2];   // largest listed entry, sum of the listed without one that attains it
  float ctas[kMaxCluster][8];       // TailRec, then the listed pair
  float sums[kStreamWarps][4];
  float last[kMaxCluster][4];
  float logit[kMaxTopK];            // the teacher's as stored; -inf: left out
  Teacher teacher;
  int flags;
};

// One warp: the teacher's normaliser, or its tail. 1 - sum p_k is taken from what
// the largest entry leaves of 1 (-expm1): its digits outlast a sum next to 1.
__device__ __forceinline__ void teacher_side(LossShared& sh, int K, bool tail, float inv_t) {
  const int lane = threadIdx.x & 31;
  constexpr int N = kMaxTopK / 32;
  float t[N], top = -INFINITY;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int k = i * 32 + lane;
    t[i] = k < K ? sh.logit[k] : -INFINITY;
    top = fmaxf(top, t[i]);
  }
  top = warp_max(top);
  int first = kMaxTopK;
#pragma unroll
  for (int i = N - 1; i >= 0; --i)
    if (t[i] == top) first = i * 32 + lane;
  first = __reduce_min_sync(0xFFFFFFFFu, first);
  const float shift = tail ? 0.f : top, scale = tail ? 1.f : inv_t;
  float others = 0.f;                              // without the first of the largest
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (t[i] > -INFINITY && i * 32 + lane != first) others += expf((t[i] - shift) * scale);
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

// q M - p of a listed id from its logarithms: where p and q are next to 1 and to
// each other their difference keeps its digits.
__device__ __forceinline__ float listed_grad(float lq, float lp, float mass) {
  const float p = expf(lp), d = lq - lp;
  return d < 1.f ? p * expm1f(d) + expf(lq) * (mass - 1.f) : expf(lq) * mass - p;
}

template <typename T, bool FUSED, bool VEC>
__global__ void __launch_bounds__(kStreamThreads, 2) k_distill_loss(DistillArgs a) {
  extern __shared__ unsigned bitmap[];             // one bit per column of the slice: listed
  __shared__ LossShared sh;
  pdl_wait();
  if (threadIdx.x == 0) pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int C = a.in.cluster, K = a.K, V = a.in.V;
  const int rank = (int)(blockIdx.x % C);
  const long long r = blockIdx.x / C;
  const float c = a.in.scale, inv_t = a.in.inv_t;
  const float weight = a.row_weight ? __ldg(a.row_weight + r) : 1.f;
  const long long first = (long long)rank * a.in.slice_cols;
  const int c0 = (int)min(first, (long long)V), c1 = (int)min(first + a.in.slice_cols, (long long)V);

  for (int i = tid; i < (a.in.slice_cols + 31) / 32; i += kStreamThreads) bitmap[i] = 0u;
  if (tid == 0) sh.flags = 0;
  // thread k has entry k (kMaxTopK <= kStreamThreads)
  int id = -1;
  float logit = -INFINITY;
  unsigned flags = 0u;
  if (tid < K) {
    id = __ldg(a.ids + r * K + tid);
    logit = __ldg(a.teacher + r * K + tid);
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
  const bool mine = id >= c0 && id < c1 && id >= 0;
  __syncthreads();
  if (mine) {
    const unsigned bit = 1u << ((id - c0) & 31);
    if (atomicOr(&bitmap[(id - c0) >> 5], bit) & bit) flags |= kFlagTwice;
  }
  if (tid < kMaxTopK) {
    flags = __reduce_or_sync(0xFFFFFFFFu, flags);
    if (lane == 0 && flags) atomicOr(&sh.flags, (int)flags);
  }
  __syncthreads();
  flags = (unsigned)sh.flags;
  if (weight == 0.f || !(flags & (kFlagAny | kFlagBadLogit))) {     // left out: the logits are not read
    if (rank == 0 && tid == 0) {
      if (weight != 0.f && (flags & kFlagBadId)) raise_status(a.status, DELS_STATUS_BAD_TOKEN);
      if (a.out_loss) a.out_loss[r] = 0.f;
      a.state[r] = DistillState{};
    }
    return;
  }
  const FusedRow<T, FUSED> row(a.in, r);
  // a constant in the prior drops out of the gradient's sum with it: taken out first
  const float p_ref = FUSED ? row.p_at(V / 2) : 0.f;
  float x_k = -INFINITY, s_k = 0.f, p_k = 0.f;
  if (mine) {
    x_k = row.at(id);
    s_k = fmaxf(row.s_at(id), -FLT_MAX);
    p_k = row.p_at(id) - p_ref;
  }

  // the columns that are not listed
  TailRec st{-INFINITY, 0.f, 0.f, 0.f};
  float off = 0.f;
  bool holds = false;
  const int items = (c1 - c0 + kStreamStep - 1) / kStreamStep;
  for (int it = 0; it < items; ++it) {
    const int col = item_col<VEC>(c0, it, tid);
    float l[8], s[8], p[8], x[8];
    row.template load<VEC, true>(col, c1, l, s, p);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = row.combine(l[i], s[i], p[i]);
      const int k = elem_col<VEC>(col, i) - c0;
      if (k < c1 - c0 && (bitmap[k >> 5] >> (k & 31) & 1u)) x[i] = -INFINITY;
    }
    const float vm = max8(x);
    if (__any_sync(0xFFFFFFFFu, vm > st.m)) {
      const float nt = warp_max(vm);
      const float f = st.m == -INFINITY ? (st.rest != st.rest ? NAN : 0.f) : ex2_approx((st.m - nt) * c);
      st.rest = st.rest * f + (holds ? f : 0.f);
      st.s *= f;
      st.p *= f;
      st.m = off = nt;
      const unsigned who = __ballot_sync(0xFFFFFFFFu, vm == nt);
      holds = lane == __ffs(who) - 1;
      if (holds) {
        bool kept = false;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (!kept && x[i] == nt) {
            kept = true;
            x[i] = -INFINITY;
            if constexpr (FUSED) {
              st.s += s[i];
              st.p += p[i] - p_ref;
            }
          }
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float e = ex2_approx((x[i] - off) * c);
      st.rest += e;
      if constexpr (FUSED) {
        st.s += e * fmaxf(s[i], -FLT_MAX);         // a masked entry: 0
        st.p += e * (p[i] - p_ref);
      }
    }
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    st.rest += __shfl_xor_sync(0xFFFFFFFFu, st.rest, d);
    st.s += __shfl_xor_sync(0xFFFFFFFFu, st.s, d);
    st.p += __shfl_xor_sync(0xFFFFFFFFu, st.p, d);
  }
  if (lane == 0) sh.warps[warp] = st;

  // the listed columns of this slice; an id listed twice counts once in the student's sums
  bool once = mine;
  if (mine && (flags & kFlagTwice))
    for (int k = 0; k < tid; ++k)
      if (sh.logit[k] > -INFINITY && __ldg(a.ids + r * K + k) == id) once = false;
  const float m_k = warp_max(once && x_k == x_k ? x_k : -INFINITY);
  {
    const unsigned who = __ballot_sync(0xFFFFFFFFu, once && x_k == m_k && m_k > -INFINITY);
    float e = 0.f;
    if (once && x_k != -INFINITY && lane != __ffs(who) - 1) e = ex2_approx((x_k - m_k) * c);
    if (once && x_k != x_k) e = NAN;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) e += __shfl_xor_sync(0xFFFFFFFFu, e, d);
    if (lane == 0) {
      sh.members[warp][0] = m_k;
      sh.members[warp][1] = e;
    }
  }
  if (warp == kStreamWarps - 1) teacher_side(sh, K, a.tail != 0, inv_t);
  __syncthreads();
  TailRec tail = sh.warps[0];
  TailRec listed{sh.members[0][0], sh.members[0][1], 0.f, 0.f};
  for (int k = 1; k < kStreamWarps; ++k) {
    tail = tail_merge(tail, sh.warps[k], c);
    listed = tail_merge(listed, TailRec{sh.members[k][0], sh.members[k][1], 0.f, 0.f}, c);
  }
  if (C > 1) {
    cluster_sync_all();            // every CTA of the cluster runs before its shared memory is written
    if (tid < C) {
      const uint32_t to = cluster_map(smem_u32(&sh.ctas[rank][0]), (uint32_t)tid);
      st_cluster_v4(to, tail.m, tail.rest, tail.s, tail.p);
      st_cluster_v4(to + 16, listed.m, listed.rest, 0.f, 0.f);
    }
    cluster_sync_all();
    tail = TailRec{sh.ctas[0][0], sh.ctas[0][1], sh.ctas[0][2], sh.ctas[0][3]};
    listed = TailRec{sh.ctas[0][4], sh.ctas[0][5], 0.f, 0.f};
    for (int k = 1; k < C; ++k) {
      tail = tail_merge(tail, TailRec{sh.ctas[k][0], sh.ctas[k][1], sh.ctas[k][2], sh.ctas[k][3]}, c);
      listed = tail_merge(listed, TailRec{sh.ctas[k][4], sh.ctas[k][5], 0.f, 0.f}, c);
    }
  }
  const TailRec all = tail_merge(tail, listed, c);        // its s and p: the unlisted columns' alone
  const float m = all.m, S = 1.f + all.rest, inv_s = 1.f / S, ln_s = log1pf(all.rest);
  const bool ok = m > -INFINITY && m < INFINITY && all.rest >= 0.f && all.rest < INFINITY && !(flags & kFlagBadLogit);
  const Teacher te = sh.teacher;
  // q_t = tail_sum / S, from the unlisted columns' own sum; ln q_t = -ln(1 + listed_sum / tail_sum)
  const float f_tail = tail.m == -INFINITY ? 0.f : ex2_approx((tail.m - m) * c);
  const float f_list = listed.m == -INFINITY ? 0.f : ex2_approx((listed.m - m) * c);
  const float tail_sum = f_tail * (1.f + tail.rest), list_sum = f_list * (1.f + listed.rest);
  const bool has_tail = a.tail && te.rest > 0.f && tail_sum > 0.f;
  const float mass = has_tail ? 1.f : te.sum;
  const float coef_n = has_tail ? mass - te.rest * (S / tail_sum) : mass;

  float v[3] = {0.f, 0.f, 0.f};
  if (mine) {
    const float lp = (logit - te.t_max) * te.t_scale - te.log_norm, p = expf(lp);
    const float lq = (x_k - m) * inv_t - ln_s;
    const float g = once ? listed_grad(lq, lp, mass) : -p;
    v[0] = p > 0.f ? p * (lp - lq) : 0.f;
    v[1] = g * s_k;
    v[2] = g * p_k;
  }
#pragma unroll
  for (int j = 0; j < 3; ++j) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v[j] += __shfl_xor_sync(0xFFFFFFFFu, v[j], d);
    if (lane == 0) sh.sums[warp][j] = v[j];
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 3; ++j) {
    v[j] = 0.f;
    for (int k = 0; k < kStreamWarps; ++k) v[j] += sh.sums[k][j];
  }
  if (C > 1) {
    if (tid == 0) st_cluster_v4(cluster_map(smem_u32(&sh.last[rank][0]), 0), v[0], v[1], v[2], 0.f);
    cluster_sync_all();
    if (rank != 0) return;
#pragma unroll
    for (int j = 0; j < 3; ++j) {
      v[j] = 0.f;
      for (int k = 0; k < C; ++k) v[j] += sh.last[k][j];
    }
  }
  if (tid != 0) return;
  if (!ok) raise_status(a.status, DELS_STATUS_NONFINITE);
  if (flags & kFlagBadId) raise_status(a.status, DELS_STATUS_BAD_TOKEN);
  float loss = v[0];
  if (has_tail) {
    const float log_rest = te.rest > 0.5f ? log1pf(-te.sum) : logf(te.rest);
    loss += te.rest * (log_rest + log1pf(list_sum / tail_sum));
  }
  if (a.out_loss) a.out_loss[r] = ok ? weight * loss : NAN;
  DistillState o{};
  o.m = m;
  o.inv_s = inv_s;
  o.ln_s = ln_s;
  o.coef_n = ok ? coef_n : NAN;
  o.mass = ok ? mass : NAN;
  o.t_max = te.t_max;
  o.t_scale = te.t_scale;
  o.log_norm = te.log_norm;
  o.weight = weight;
  o.d_alpha = ok ? weight * inv_t * (coef_n * inv_s * all.s + v[1]) : NAN;
  o.d_beta = ok ? -weight * inv_t * (coef_n * inv_s * all.p + v[2]) : NAN;
  a.state[r] = o;
}

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  uint32_t w;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  return w;
}
__device__ __forceinline__ void grad_elem(float* g, long long i, float v) { g[i] = v; }
__device__ __forceinline__ void grad_elem(uint16_t* g, long long i, float v) { g[i] = (uint16_t)bf16_pair(v, 0.f); }
__device__ __forceinline__ void grad_vec(float* g, const float (&v)[8]) {
  __stcs(reinterpret_cast<float4*>(g), make_float4(v[0], v[1], v[2], v[3]));
  __stcs(reinterpret_cast<float4*>(g) + 1, make_float4(v[4], v[5], v[6], v[7]));
}
__device__ __forceinline__ void grad_vec(uint16_t* g, const float (&v)[8]) {
  __stcs(reinterpret_cast<uint4*>(g),
         make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])));
}

// The gradient of l_S from the statistics: every column as one that is not listed,
// then the listed ones over it. The rows' own logits may be the output (each column
// is read before it is written).
template <typename T, bool FUSED, bool VEC>
__global__ void __launch_bounds__(kStreamThreads, 2) k_distill_grad(DistillArgs a) {
  pdl_wait();
  if (threadIdx.x == 0) pdl_trigger();
  const int tid = threadIdx.x;
  const int C = a.in.cluster, K = a.K, V = a.in.V;
  const int rank = (int)(blockIdx.x % C);
  const long long r = blockIdx.x / C;
  const long long first = (long long)rank * a.in.slice_cols;
  const int c0 = (int)min(first, (long long)V), c1 = (int)min(first + a.in.slice_cols, (long long)V);
  const DistillState st = a.state[r];
  const float up = a.grad_loss ? __ldg(a.grad_loss + r) : 1.f;
  const FusedRow<T, FUSED> row(a.in, r);
  T* out = static_cast<T*>(a.grad) + r * a.ld_grad;
  const bool left_out = st.weight == 0.f;
  const float g0 = up * st.weight * a.in.inv_t * (FUSED ? row.a : 1.f);
  const float c = a.in.scale;

  int id = -1;
  float g_k = 0.f;
  if (tid < K && !left_out) {
    id = __ldg(a.ids + r * K + tid);
    const float t = __ldg(a.teacher + r * K + tid);
    if (id < c0 || id >= c1 || t == -INFINITY) id = -1;
    if (id >= 0) {
      // every entry with this id, in their order; the last of them writes
      const float lp = (t - st.t_max) * st.t_scale - st.log_norm, x = row.at(id);
      float before = 0.f;
      for (int k = 0; k < K; ++k) {
        if (k == tid || __ldg(a.ids + r * K + k) != id) continue;
        const float tk = __ldg(a.teacher + r * K + k);
        if (tk == -INFINITY) continue;
        if (k > tid) {
          id = -1;
          break;
        }
        before += expf((tk - st.t_max) * st.t_scale - st.log_norm);
      }
      const float lq = (x - st.m) * a.in.inv_t - st.ln_s;
      g_k = g0 * (listed_grad(lq, lp, st.mass) - before);
    }
  }
  __syncthreads();
  const float f = g0 * st.coef_n * st.inv_s;
  const int items = (c1 - c0 + kStreamStep - 1) / kStreamStep;
  for (int it = 0; it < items; ++it) {
    const int col = item_col<VEC>(c0, it, tid);
    float g[8];
    if (left_out) {
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] = 0.f;
    } else {
      float l[8], s[8], p[8];
      row.template load<VEC, true>(col, c1, l, s, p);
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] = f * ex2_approx((row.combine(l[i], s[i], p[i]) - st.m) * c);
    }
    if (VEC && col + 8 <= c1) {
      grad_vec(out + col, g);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int k = elem_col<VEC>(col, i);
        if (k < c1) grad_elem(out, k, g[i]);
      }
    }
  }
  __syncthreads();
  if (id >= 0) grad_elem(out, id, g_k);
}

// Sums over the rows of each weight, in a fixed order: one CTA per weight.
__global__ void __launch_bounds__(256) k_weight_grads(DistillArgs a) {
  pdl_wait();
  if (threadIdx.x == 0) pdl_trigger();
  __shared__ float red[8][2];
  const int j = blockIdx.x, n = a.in.n_weights;
  float da = 0.f, db = 0.f;
  for (long long r = j + (long long)threadIdx.x * n; r < a.in.rows; r += 256LL * n) {
    const float g = a.grad_loss ? a.grad_loss[r] : 1.f;
    if (a.state[r].weight != 0.f) {
      da += g * a.state[r].d_alpha;
      db += g * a.state[r].d_beta;
    }
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    da += __shfl_xor_sync(0xFFFFFFFFu, da, d);
    db += __shfl_xor_sync(0xFFFFFFFFu, db, d);
  }
  if ((threadIdx.x & 31) == 0) {
    red[threadIdx.x >> 5][0] = da;
    red[threadIdx.x >> 5][1] = db;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    da = db = 0.f;
    for (int k = 0; k < 8; ++k) {
      da += red[k][0];
      db += red[k][1];
    }
    if (a.grad_alpha) a.grad_alpha[j] = da;
    if (a.grad_beta) a.grad_beta[j] = db;
  }
}

template <typename T>
cudaError_t launch_t(const DistillArgs& a, bool grad, bool fused, bool vec, cudaStream_t s) {
  const dim3 grid((unsigned)((long long)a.in.rows * a.in.cluster)), block(kStreamThreads);
  if (grad) {
    auto k = fused ? (vec ? k_distill_grad<T, true, true> : k_distill_grad<T, true, false>)
                   : (vec ? k_distill_grad<T, false, true> : k_distill_grad<T, false, false>);
    return launch_pdl(k, grid, block, 0, s, a);
  }
  auto k = fused ? (vec ? k_distill_loss<T, true, true> : k_distill_loss<T, true, false>)
                 : (vec ? k_distill_loss<T, false, true> : k_distill_loss<T, false, false>);
  const size_t bytes = (size_t)(a.in.slice_cols + 31) / 32 * 4;
  const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(k), bytes);
  if (e != cudaSuccess) return e;
  return launch_pdl_cluster(k, grid, block, bytes, s, a.in.cluster, a);
}

}  // namespace

cudaError_t launch_distill_loss(const DistillArgs& a, bool f32, bool fused, bool vec, cudaStream_t s) {
  return f32 ? launch_t<float>(a, false, fused, vec, s) : launch_t<uint16_t>(a, false, fused, vec, s);
}
cudaError_t launch_distill_grad(const DistillArgs& a, bool f32, bool fused, bool vec, cudaStream_t s) {
  return f32 ? launch_t<float>(a, true, fused, vec, s) : launch_t<uint16_t>(a, true, fused, vec, s);
}
cudaError_t launch_weight_grads(const DistillArgs& a, cudaStream_t s) {
  return launch_pdl(k_weight_grads, dim3((unsigned)a.in.n_weights), dim3(256), 0, s, a);
}

}  // namespace dels
