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
  unsigned long long slices[kMaxCluster * kMaxTopK];   // first CTA: all slices' entries
  int groups[kStreamThreads];
  SoftRec warps[kStreamWarps];
  SoftRec ctas[kMaxCluster];
  int ncand, ngroups;
};

// The K largest of cand[0 .. n) to best[] in order (all threads): a warp counts
// what is above one candidate, 32 at a time.
__device__ void sort_best(ScoreShared& sh, const unsigned long long* cand, int n, int K) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int k = threadIdx.x; k < K; k += kStreamThreads) sh.best[k] = 0ull;
  __syncthreads();
  for (int i = warp; i < n; i += kStreamWarps) {
    const unsigned long long x = cand[i];
    int rank = 0;
    for (int j = lane; j < n; j += 32) rank += cand[j] > x;
    rank = __reduce_add_sync(0xFFFFFFFFu, rank);
    if (lane == 0 && rank < K && x) sh.best[rank] = x;
  }
  __syncthreads();
}

// The entries of an item that reach `floor_key`, into cand[] as far as it has room.
template <typename T, bool FUSED, bool VEC>
__device__ __forceinline__ void keep_entries(ScoreShared& sh, const FusedRow<T, FUSED, VEC>& row, int pos, int k1,
                                             unsigned long long floor_key) {
  Item<T, FUSED, VEC> v;
  v.load(row, pos, k1);
  float x[8], s[8], p[8];
  v.template values<true>(row, k1, x, s, p);
  const float least = from_order_u32((unsigned)(floor_key >> 32));
  if (!(max8(x) >= least)) return;                 // most items: nothing
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (!(x[i] >= least && x[i] > -INFINITY)) continue;
    const unsigned long long e = entry_key(x[i], elem_pos<VEC>(pos, i) - row.sh);
    if (e < floor_key) continue;
    const int at = atomicAdd(&sh.ncand, 1);
    if (at < kCandidates) sh.cand[at] = e;
  }
}

// This CTA's K largest entries of its slice into sh.best. `top`: the largest
// entry of the calling thread.
template <typename T, bool FUSED, bool VEC>
__device__ void slice_top(ScoreShared& sh, const FusedRow<T, FUSED, VEC>& row, int k0, int k1, int K, float top) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // About the K-th largest thread maximum, from its highest bit down; 0 where
  // fewer than K threads have an entry.
  const unsigned key = top > -INFINITY ? order_u32(top) : 0u;
  unsigned tau = 0u;
  if (tid == 0) sh.ncand = sh.ngroups = 0;
  if (__syncthreads_count(key > 0u) >= K) {
    for (int bit = 31; bit >= 0; --bit) {
      const unsigned t = tau | (1u << bit);
      const int n = __syncthreads_count(key >= t);
      if (n >= K) tau = t;
      if (n >= K && n <= K + 8) break;
    }
  }
  if (key > 0u && key >= tau) sh.groups[atomicAdd(&sh.ngroups, 1)] = tid;
  __syncthreads();
  const int items = (k1 - k0 + kStreamStep - 1) / kStreamStep;      // per thread
  const int parts = (items + 31) / 32;                              // a warp's rounds for one thread's items
  const int jobs = sh.ngroups * parts;
  if (tau == 0u) tau = order_u32(-INFINITY);
  unsigned long long floor_key = (unsigned long long)tau << 32;     // what an entry has to reach
  for (int j = warp; j < jobs; j += kStreamWarps) {
    const int it = (j % parts) * 32 + lane;
    if (it < items) keep_entries(sh, row, item_pos<VEC>(k0, it, sh.groups[j / parts]), k1, floor_key);
  }
  __syncthreads();
  if (sh.ncand > kCandidates) {
    // more entries than there is room for: a round of items at a time, the best
    // of them kept as soon as the next round might not fit
    __syncthreads();
    if (tid == 0) sh.ncand = 0;
    __syncthreads();
    for (int j0 = 0; j0 < jobs; j0 += kStreamWarps) {
      const int n = sh.ncand;
      __syncthreads();
      if (n > kCandidates - kStreamWarps * 256) {
        sort_best(sh, sh.cand, n, K);
        for (int k = tid; k < K; k += kStreamThreads) sh.cand[k] = sh.best[k];
        floor_key = sh.best[K - 1];                                 // n > K: there are K
        if (tid == 0) sh.ncand = K;
        __syncthreads();
      }
      const int j = j0 + warp, it = (j % parts) * 32 + lane;
      if (j < jobs && it < items) keep_entries(sh, row, item_pos<VEC>(k0, it, sh.groups[j / parts]), k1, floor_key);
      __syncthreads();
    }
  }
  sort_best(sh, sh.cand, sh.ncand, K);
}

template <typename T, bool FUSED, bool VEC>
__global__ void __launch_bounds__(kStreamThreads, 4) k_score_rows(ScoreArgs a) {
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
  if (C > 1) cluster_arrive_relaxed();
  const FusedRow<T, FUSED, VEC> row(a.in, r);
  const bool tok_ok = tok >= 0 && tok < V;
  float x_tok = 0.f;
  if (rank == 0 && tid == 0 && a.tokens && tok_ok) x_tok = row.at(tok + row.sh);
  const long long first = (long long)rank * a.in.slice_cols;
  const int k0 = (int)min(first, (long long)row.end), k1 = (int)min(first + a.in.slice_cols, (long long)row.end);

  // items in flight per thread: 64 bytes of bf16 rows, 64 to 128 of the others
  constexpr int U = sizeof(T) == 2 ? (FUSED ? 2 : 4) : (FUSED ? 1 : 2);
  WarpSoft st;
  st.init();
  float top = -INFINITY;
  stream_items<U>(row, k0, k1, [&](auto& v, auto checked) {
    constexpr int N = sizeof(v) / sizeof(v[0]);
    float x[N][8], s[8], p[8], vm = -INFINITY;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      v[u].template values<decltype(checked)::value>(row, k1, x[u], s, p);
      vm = fmaxf(vm, max8(x[u]));
    }
    top = fmaxf(top, vm);
    st.push(x, vm, c);
  });
  const SoftRec wr = st.record();
  if (lane == 0) sh.warps[warp] = wr;
  __syncthreads();
  const SoftRec cta = softrec_merge8(sh.warps[lane & 7], c);

  if (K > 0) slice_top(sh, row, k0, k1, K, top);
  SoftRec all = cta;
  if (C > 1) {
    cluster_wait();                // every CTA of the cluster runs before its shared memory is written
    if (tid < 3) {
      const float v = tid == 0 ? cta.m : tid == 1 ? cta.rest : cta.w;
      st_cluster_f32(cluster_map(smem_u32(&sh.ctas[rank]), 0) + 4 * tid, v);
    }
    if (K > 0) {
      const uint32_t to = cluster_map(smem_u32(&sh.slices[(size_t)rank * K]), 0);
      for (int k = tid; k < K; k += kStreamThreads) {
        const unsigned long long e = sh.best[k];
        st_cluster_f32(to + 8 * k, __uint_as_float((unsigned)e));
        st_cluster_f32(to + 8 * k + 4, __uint_as_float((unsigned)(e >> 32)));
      }
    }
    cluster_arrive();
    if (rank != 0) return;
    cluster_wait();
    all = softrec_merge8((lane & 7) < C ? sh.ctas[lane & 7] : softrec_init(), c);
    if (K > 0) sort_best(sh, sh.slices, C * K, K);
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
