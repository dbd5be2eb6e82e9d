// Scoring of vocabulary rows: the log-probability of one given token of each
// row, the row's entropy and its top_k most likely entries, in one pass.
//
//   log q_v = (l_v - m) / T - ln S,   S = sum_v exp((l_v - m) / T)
//   H       = ln S - (1 / S) sum_v exp((l_v - m) / T) (l_v - m) / T
//
// What bounds it: the read of the logits. The alternatives cost no second read of
// the row: every thread keeps the largest of its own entries, the K-th largest of
// those is at most the K-th largest entry of the slice, and only the items of the
// few threads above that threshold are read again (out of L2) for their entries.
#include <climits>

#include "row_stream.cuh"

namespace dels {

namespace {

// Entries of equal order: larger values first, then lower columns. No NaN; 0 is
// below every entry.
__device__ __forceinline__ unsigned order_u32(float x) {
  const int i = __float_as_int(x + 0.f);   // -0 as +0
  return i < 0 ? ~(unsigned)i : (unsigned)i | 0x80000000u;
}
__device__ __forceinline__ float from_order_u32(unsigned u) {
  return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}
__device__ __forceinline__ unsigned long long entry_key(float x, int col) {
  return ((unsigned long long)order_u32(x) << 32) | (0xFFFFFFFFu - (unsigned)col);
}

constexpr int kCandidates = kStreamWarps * 256 + 4 * kMaxTopK;   // one round of rescanned items, and what was kept

struct ScoreShared {
  unsigned long long cand[kCandidates];
  unsigned long long best[kMaxTopK];       // this CTA's entries in order, 0 where there are none
  int groups[kStreamThreads];
  SoftRec warps[kStreamWarps];
  SoftRec ctas[kMaxCluster];
  int ncand, ngroups;
};

// The K largest of cand[0 .. n) to best[] in order (all threads; n <= kCandidates).
__device__ void sort_best(ScoreShared& sh, int n, int K) {
  for (int k = threadIdx.x; k < K; k += kStreamThreads) sh.best[k] = 0ull;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kStreamThreads) {
    const unsigned long long x = sh.cand[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += sh.cand[j] > x;
    if (rank < K && x) sh.best[rank] = x;
  }
  __syncthreads();
}

// This CTA's K largest entries of its slice into sh.best. `top`: the largest
// entry of the calling thread.
template <typename T, bool FUSED, bool VEC>
__device__ void slice_top(ScoreShared& sh, const FusedRow<T, FUSED>& row, int c0, int c1, int K, float top) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // The K-th largest thread maximum, from its highest bit down; -inf where fewer
  // than K threads have an entry.
  const unsigned key = top > -INFINITY ? order_u32(top) : 0u;
  unsigned tau = 0u;
  if (__syncthreads_count(key > 0u) >= K) {
    for (int bit = 31; bit >= 0; --bit) {
      const unsigned t = tau | (1u << bit);
      const int n = __syncthreads_count(key >= t);
      if (n >= K) tau = t;
      if (n == K) break;
    }
  }
  if (tid == 0) sh.ncand = sh.ngroups = 0;
  __syncthreads();
  if (key > 0u && key >= tau) sh.groups[atomicAdd(&sh.ngroups, 1)] = tid;
  __syncthreads();
  const int items = (c1 - c0 + kStreamStep - 1) / kStreamStep;      // per thread
  const int parts = (items + 31) / 32;                              // a warp's rounds for one thread's items
  const int jobs = sh.ngroups * parts;
  unsigned long long floor_key = (unsigned long long)tau << 32;     // what an entry has to exceed or equal
  for (int j0 = 0; j0 < jobs; j0 += kStreamWarps) {
    if (j0 > 0) {
      __syncthreads();
      const int n = sh.ncand;
      __syncthreads();
      if (n > kCandidates - kStreamWarps * 256) {                   // room for one more round
        sort_best(sh, n, K);
        for (int k = tid; k < K; k += kStreamThreads) sh.cand[k] = sh.best[k];
        if (sh.best[K - 1]) floor_key = sh.best[K - 1];
        if (tid == 0) sh.ncand = K;
        __syncthreads();
      }
    }
    const int j = j0 + warp;
    if (j < jobs) {
      const int g = sh.groups[j / parts], it = (j % parts) * 32 + lane;
      const int c = item_col<VEC>(c0, it, g);
      if (it < items && c < c1) {
        float l[8], s[8], p[8];
        row.template load<VEC, true>(c, c1, l, s, p);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int col = elem_col<VEC>(c, i);
          const float x = row.combine(l[i], s[i], p[i]);
          if (col < c1 && x > -INFINITY) {
            const unsigned long long e = entry_key(x, col);
            if (e >= floor_key) sh.cand[atomicAdd(&sh.ncand, 1)] = e;
          }
        }
      }
    }
  }
  __syncthreads();
  sort_best(sh, sh.ncand, K);
}

template <typename T, bool FUSED, bool VEC>
__global__ void __launch_bounds__(kStreamThreads, 2) k_score_rows(ScoreArgs a) {
  __shared__ ScoreShared sh;
  pdl_wait();
  if (threadIdx.x == 0) pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int C = a.in.cluster, K = a.top_k;
  const int rank = (int)(blockIdx.x % C);
  const long long r = blockIdx.x / C;
  const int V = a.in.V;
  const float c = a.in.scale;
  const int tok = a.tokens ? __ldg(a.tokens + r) : 0;
  if (a.tokens && tok == -1) {     // left out: not read
    if (rank == 0) {
      if (tid == 0) {
        if (a.out_lp) a.out_lp[r] = 0.f;
        if (a.out_entropy) a.out_entropy[r] = 0.f;
      }
      for (int k = tid; k < K; k += kStreamThreads) {
        a.out_ids[r * K + k] = -1;
        a.out_top_lp[r * K + k] = -INFINITY;
      }
    }
    return;
  }
  const FusedRow<T, FUSED> row(a.in, r);
  const bool tok_ok = tok >= 0 && tok < V;
  float x_tok = 0.f;
  if (rank == 0 && tid == 0 && a.tokens && tok_ok) x_tok = row.at(tok);
  const long long first = (long long)rank * a.in.slice_cols;
  const int c0 = (int)min(first, (long long)V), c1 = (int)min(first + a.in.slice_cols, (long long)V);

  WarpSoft st;
  st.init();
  float top = -INFINITY;
  const int items = (c1 - c0 + kStreamStep - 1) / kStreamStep;
  for (int it = 0; it < items; ++it) {
    const int col = item_col<VEC>(c0, it, tid);
    float l[8], s[8], p[8], x[8];
    row.template load<VEC, true>(col, c1, l, s, p);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = row.combine(l[i], s[i], p[i]);
    const float vm = max8(x);
    top = fmaxf(top, vm);
    if (__any_sync(0xFFFFFFFFu, vm > st.ref)) {
      const float nt = warp_max(vm);
      st.move(nt, c);
      const unsigned who = __ballot_sync(0xFFFFFFFFu, vm == nt);
      if (lane == __ffs(who) - 1) {
        bool kept = false;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (!kept && x[i] == nt) {
            kept = true;
            x[i] = -INFINITY;
          }
        st.holds = true;
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float t = (x[i] - st.off) * c;
      const float e = ex2_approx(t);
      st.rest += e;
      st.w += e * fmaxf(t, kLowT);
    }
  }
  const SoftRec wr = st.record();
  if (lane == 0) sh.warps[warp] = wr;
  __syncthreads();
  SoftRec cta = sh.warps[0];
  for (int k = 1; k < kStreamWarps; ++k) cta = softrec_merge(cta, sh.warps[k], c);

  if (K > 0) slice_top<T, FUSED, VEC>(sh, row, c0, c1, K, top);
  SoftRec all = cta;
  if (C > 1) {
    cluster_sync_all();            // every CTA of the cluster runs before its shared memory is written
    if (tid < 3) {
      const float v = tid == 0 ? cta.m : tid == 1 ? cta.rest : cta.w;
      st_cluster_f32(cluster_map(smem_u32(&sh.ctas[rank]), 0) + 4 * tid, v);
    }
    // the slices' entries into the first CTA's candidates (its own are free again)
    if (K > 0) {
      const uint32_t to = cluster_map(smem_u32(&sh.cand[(size_t)rank * K]), 0);
      for (int k = tid; k < K; k += kStreamThreads) {
        const unsigned long long e = sh.best[k];
        st_cluster_f32(to + 8 * k, __uint_as_float((unsigned)e));
        st_cluster_f32(to + 8 * k + 4, __uint_as_float((unsigned)(e >> 32)));
      }
    }
    cluster_sync_all();
    if (rank != 0) return;
    all = sh.ctas[0];
    for (int k = 1; k < C; ++k) all = softrec_merge(all, sh.ctas[k], c);
    if (K > 0) sort_best(sh, C * K, K);
  }
  const bool ok = softrec_valid(all);
  const float ln_s = log1pf(all.rest), inv_t = a.in.inv_t;
  if (tid == 0) {
    if (!ok) raise_status(a.status, DELS_STATUS_NONFINITE);
    if (a.tokens && !tok_ok) raise_status(a.status, DELS_STATUS_BAD_TOKEN);
    if (a.out_lp) a.out_lp[r] = ok && tok_ok ? (x_tok - all.m) * inv_t - ln_s : NAN;
    if (a.out_entropy) a.out_entropy[r] = ok ? ln_s - kLn2 * (all.w / (1.f + all.rest)) : NAN;
  }
  for (int k = tid; k < K; k += kStreamThreads) {
    const unsigned long long e = sh.best[k];
    const bool has = ok && e != 0ull;
    a.out_ids[r * K + k] = has ? (int)(0xFFFFFFFFu - (unsigned)e) : -1;
    a.out_top_lp[r * K + k] = !ok ? NAN : has ? (from_order_u32((unsigned)(e >> 32)) - all.m) * inv_t - ln_s : -INFINITY;
  }
}

template <typename T>
cudaError_t launch_score_t(const ScoreArgs& a, bool fused, bool vec, cudaStream_t s) {
  const dim3 grid((unsigned)((long long)a.in.rows * a.in.cluster)), block(kStreamThreads);
  auto k = fused ? (vec ? k_score_rows<T, true, true> : k_score_rows<T, true, false>)
                 : (vec ? k_score_rows<T, false, true> : k_score_rows<T, false, false>);
  return launch_pdl_cluster(k, grid, block, 0, s, a.in.cluster, a);
}

}  // namespace

cudaError_t launch_score_rows(const ScoreArgs& a, bool f32, bool fused, bool vec, cudaStream_t s) {
  return f32 ? launch_score_t<float>(a, fused, vec, s) : launch_score_t<uint16_t>(a, fused, vec, s);
}

}  // namespace dels
