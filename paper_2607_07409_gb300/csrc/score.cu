// Scoring of vocabulary rows: the log-probability of one given token of each
// row, the row's entropy and its top_k most likely entries, in one pass.
//
//   log q_v = (l_v - m) / T - ln S,   S = sum_v exp((l_v - m) / T)
//   H       = ln S - (1 / S) sum_v exp((l_v - m) / T) (l_v - m) / T
//
// What bounds it: the read of the logits. The alternatives cost no second read of
// the row: every thread keeps the largest entry of each of its blocks of a few
// items; the K-th largest thread maximum is at most the K-th largest entry of the
// slice, and only the blocks that reach it are read again for their entries.
#include <cuda_bf16.h>

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

constexpr int kJobs = 2048;          // blocks read again
constexpr int kCandidates = 2048;    // their entries that are kept
constexpr int kSlots = 20;           // block maxima per thread: 20 KB of float

// What the selection needs once the ring is done with (in its place).
struct SelectShared {
  unsigned long long cand[kCandidates];
  int jobs[kJobs];
};
struct ScoreShared {
  unsigned long long best[kMaxTopK];       // this CTA's entries in order, 0 where there are none
  SoftRec warps[kStreamWarps];
  SoftRec ctas[kMaxCluster];
  int ncand, njobs;
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
template <typename T, int F, bool VEC>
__device__ __forceinline__ void keep_entries(ScoreShared& sh, SelectShared& sel, const FusedRow<T, F, VEC>& row,
                                             int pos, int k1, unsigned long long floor_key) {
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int q = elem_pos<T, VEC>(pos, i);
    x[i] = q >= row.sh && q < k1 ? row.at(q) : -INFINITY;
  }
  const float least = from_order_u32((unsigned)(floor_key >> 32));
  if (!(max8(x) >= least)) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (!(x[i] >= least && x[i] > -INFINITY)) continue;
    const unsigned long long e = entry_key(x[i], elem_pos<T, VEC>(pos, i) - row.sh);
    if (e < floor_key) continue;
    const int at = atomicAdd(&sh.ncand, 1);
    if (at < kCandidates) sel.cand[at] = e;
  }
}

// This CTA's K largest entries of its slice into sh.best. `top`: the largest
// entry of the calling thread; bmax: [slot][thread] the largest of a thread's groups
// slot << shift .. of the stream.
template <int U, typename T, int F, bool VEC>
__device__ void slice_top(ScoreShared& sh, SelectShared& sel, const float* bmax, int shift,
                          const FusedRow<T, F, VEC>& row, int k0, int k1, int K, float top) {
  const int tid = threadIdx.x;
  const int items = (k1 - k0 + kStreamStep - 1) / kStreamStep, groups = (items + U - 1) / U;
  const int slots = (groups + (1 << shift) - 1) >> shift;
  // About the K-th largest thread maximum, from its highest bit down; -inf where
  // fewer than K threads have an entry.
  const unsigned key = top > -INFINITY ? order_u32(top) : 0u;
  unsigned tau = 0u;
  if (tid == 0) sh.ncand = sh.njobs = 0;
  if (__syncthreads_count(key > 0u) >= K) {
    for (int bit = 31; bit >= 0; --bit) {
      const unsigned t = tau | (1u << bit);
      const int n = __syncthreads_count(key >= t);
      if (n >= K) tau = t;
      if (n >= K && n <= K + 8) break;
    }
  } else {
    tau = order_u32(-INFINITY);
  }
  const float least = from_order_u32(tau);
  unsigned long long floor_key = (unsigned long long)tau << 32;     // what an entry has to reach
  if (top >= least && top > -INFINITY) {
    for (int b = 0; b < slots; ++b)
      if (bmax[b * kStreamThreads + tid] >= least) {
        const int at = atomicAdd(&sh.njobs, 1);
        if (at < kJobs) sel.jobs[at] = b * kStreamThreads + tid;
      }
  }
  __syncthreads();
  if (sh.njobs <= kJobs) {
    // a lane per item of a job
    const int per = U << shift, n = sh.njobs * per;
    for (int i = tid; i < n; i += kStreamThreads) {
      const int job = sel.jobs[i / per], o = i % per;
      const int it = (job / kStreamThreads) * per + o;
      if (it >= items) continue;
      keep_entries(sh, sel, row, item_pos<T, VEC>(k0, it, job % kStreamThreads), k1, floor_key);
    }
  }
  __syncthreads();
  if (sh.njobs > kJobs || sh.ncand > kCandidates) {
    // more than there is room for: the slice again, 128 items at a time, the best of
    // them kept as soon as the next might not fit
    __syncthreads();
    if (tid == 0) sh.ncand = 0;
    __syncthreads();
    for (int j = 0; j < 2 * items; ++j) {
      const int n = sh.ncand;
      __syncthreads();
      if (n > kCandidates - 128 * 8) {
        sort_best(sh, sel.cand, n, K);
        for (int k = tid; k < K; k += kStreamThreads) sel.cand[k] = sh.best[k];
        floor_key = sh.best[K - 1];                                 // n > K: there are K
        if (tid == 0) sh.ncand = K;
        __syncthreads();
      }
      if ((tid >> 7) == (j & 1)) keep_entries(sh, sel, row, item_pos<T, VEC>(k0, j >> 1, tid), k1, floor_key);
      __syncthreads();
    }
  }
  sort_best(sh, sel.cand, sh.ncand, K);
}

// Packed maximum of 8 bf16 (NaN ignored), and every one raised to at least `low`
// (NaN stays).
__device__ __forceinline__ float max8_bf16(const uint4& w) {
  const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&w);
  const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
  return fmaxf(__low2float(m), __high2float(m));
}
__device__ __forceinline__ void raise8_bf16(uint4& w, __nv_bfloat162 low) {
  __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&w);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __hmax2_nan(h[i], low);
}

// Copies ahead: 32 KB of plain rows (four CTAs on an SM), 48 KB of two rows (three).
template <typename T, int F>
using ScoreCopies = std::conditional_t<F == kPlain, Copies<T, F, sizeof(T) == 2 ? 4 : 2, 2>,
                                       Copies<T, F, 2, sizeof(T) == 2 ? 3 : 2>>;

// Dynamic shared memory: the ring (later SelectShared), the block maxima, and for a
// cluster the entries of all slices.
template <typename T, int F, bool VEC>
constexpr size_t ring_bytes() {
  const size_t ring = VEC ? ScoreCopies<T, F>::kRingBytes : 0;
  return ring > sizeof(SelectShared) ? ring : sizeof(SelectShared);
}

template <typename T, int F, bool VEC>
__global__ void __launch_bounds__(kStreamThreads, F ? 3 : 4) k_score_rows(ScoreArgs a) {
  extern __shared__ __align__(16) uint8_t dyn[];
  __shared__ ScoreShared sh;
  pdl_wait();
  if (threadIdx.x == 0) pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int C = a.in.cluster, K = a.top_k;
  const int rank = (int)(blockIdx.x & (C - 1));
  const long long r = blockIdx.x / (unsigned)C;
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
  using Cp = ScoreCopies<T, F>;
  RowStream<Cp, T, F, VEC> stream(a.in, r, rank, dyn, nullptr);
  stream.begin();
  const FusedRow<T, F, VEC>& row = stream.row;
  const int k0 = stream.k0, k1 = stream.k1;
  const bool tok_ok = tok >= 0 && tok < V;
  float x_tok = 0.f;
  if (rank == 0 && tid == 0 && a.tokens && tok_ok) x_tok = row.at(tok + row.sh);

  constexpr int U = Cp::U;
  float* bmax = reinterpret_cast<float*>(dyn + ring_bytes<T, F, VEC>());
  unsigned long long* slices = reinterpret_cast<unsigned long long*>(bmax + (K > 0 ? kSlots * kStreamThreads : 0));
  int shift = 0;                   // groups per block maximum: 1 << shift
  while (((stream.groups - 1) >> shift) >= kSlots) ++shift;

  WarpSoft st;
  st.init();
  float top = -INFINITY, block = -INFINITY;
  // the largest of the items' block so far
  const auto note = [&](float vm, int it) {
    if (K > 0) {
      top = fmaxf(top, vm);
      block = (it & ((U << shift) - 1)) == 0 ? vm : fmaxf(block, vm);
      bmax[(it / U >> shift) * kStreamThreads + tid] = block;
    }
  };
  float pa[8], pb[8];
  if constexpr (sizeof(T) == 2 && F == kPlain) {
    // bf16 as stored: the maximum and the clamp of masked entries on pairs
    const __nv_bfloat162 low2 = __float2bfloat162_rn(a.low);
    const auto items_of = [&](auto& v, int it) {
      constexpr int N = sizeof(v) / sizeof(v[0]);
      float vm = max8_bf16(v[0].l.w[0]);
#pragma unroll
      for (int u = 1; u < N; ++u) vm = fmaxf(vm, max8_bf16(v[u].l.w[0]));
      if (__any_sync(0xFFFFFFFFu, vm > st.m)) {
        const float nt = warp_max(vm);
        bool out = st.raise(nt, vm, c);
#pragma unroll
        for (int u = 0; u < N; ++u) {
          float x[8];
          v[u].l.unpack(x);
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (out && x[i] == nt) {
              out = false;
              v[u].l.set(i, -INFINITY);
            }
        }
      }
      if (st.f.off == 0.f) {
#pragma unroll
        for (int u = 0; u < N; ++u) {
          float x[8];
          raise8_bf16(v[u].l.w[0], low2);
          v[u].l.unpack(x);
          st.template add<true>(x, c);
        }
      } else {                     // all so far masked by huge values: their differences
#pragma unroll
        for (int u = 0; u < N; ++u) {
          float x[8];
          v[u].l.unpack(x);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            x[i] -= st.f.off;
            if (x[i] < a.low) x[i] = a.low;
          }
          st.template add<true>(x, c);
        }
      }
      note(vm, it);
    };
    stream.run(
        [&](int g) {
          Item<T, F, VEC> v[U];
#pragma unroll
          for (int u = 0; u < U; ++u) stream.take(u, v[u]);
          items_of(v, g * U);
        },
        [&](auto& v, auto&, int it) {
          Item<T, F, VEC> one[1] = {v};
          items_of(one, it);
        });
  } else {
    const auto item_of = [&](auto& v, auto& pr, int it) {
      float x[8], s[8];
      v.template values<false>(row, pr, x, s);
      const float vm = max8(x);
      if (__any_sync(0xFFFFFFFFu, vm > st.m)) {
        const float nt = warp_max(vm);
        bool out = st.raise(nt, vm, c);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (out && x[i] == nt) {
            out = false;
            x[i] = -INFINITY;
          }
      }
      if (st.f.off != 0.f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] -= st.f.off;
      }
      st.template add<false>(x, c);
      note(vm, it);
    };
    stream.run([&](int g) { stream.each(g, pa, pb, item_of); }, item_of);
  }
  const SoftRec wr = st.record();
  if (lane == 0) sh.warps[warp] = wr;
  __syncthreads();
  const SoftRec cta = softrec_merge8(sh.warps[lane & 7], c);

  if (K > 0) slice_top<U>(sh, *reinterpret_cast<SelectShared*>(dyn), bmax, shift, row, k0, k1, K, top);
  SoftRec all = cta;
  if (C > 1) {
    cluster_wait();                // every CTA of the cluster runs before its shared memory is written
    if (tid < 5) {
      const float v = tid == 0 ? cta.m : tid == 1 ? cta.f.off : tid == 2 ? cta.f.r : tid == 3 ? cta.rest : cta.w;
      st_cluster_f32(cluster_map(smem_u32(&sh.ctas[rank]), 0) + 4 * tid, v);
    }
    if (K > 0) {
      const uint32_t to = cluster_map(smem_u32(slices + (size_t)rank * K), 0);
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
    if (K > 0) sort_best(sh, slices, C * K, K);
  }
  const bool ok = softrec_valid(all);
  const float z_m = ref_z(all.m, all.f, c), e_m = ex2_approx(z_m);
  const float ln_s = log1pf(all.rest / e_m), inv_t = a.in.inv_t;
  if (tid == 0) {
    if (!ok) raise_status(a.status, DELS_STATUS_NONFINITE);
    if (a.tokens && !tok_ok) raise_status(a.status, DELS_STATUS_BAD_TOKEN);
    if (a.out_lp) a.out_lp[r] = ok && tok_ok ? (x_tok - all.m) * inv_t - ln_s : NAN;
    if (a.out_entropy) a.out_entropy[r] = ok ? ln_s - kLn2 * ((all.w - z_m * all.rest) / (e_m + all.rest)) : NAN;
  }
  for (int k = tid; k < K; k += kStreamThreads) {
    const unsigned long long e = sh.best[k];
    const bool has = ok && e != 0ull;
    a.out_ids[r * K + k] = has ? (int)(0xFFFFFFFFu - (unsigned)e) : -1;
    a.out_top_lp[r * K + k] = !ok ? NAN : has ? (from_order_u32((unsigned)(e >> 32)) - all.m) * inv_t - ln_s : -INFINITY;
  }
}

template <typename T, int F, bool VEC>
cudaError_t launch_score_t(const ScoreArgs& a, cudaStream_t s) {
  const auto k = k_score_rows<T, F, VEC>;
  const size_t bytes = ring_bytes<T, F, VEC>() + (a.top_k > 0 ? (size_t)kSlots * kStreamThreads * 4 : 0) +
                       (a.in.cluster > 1 ? (size_t)a.in.cluster * a.top_k * 8 : 0);
  const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(k), bytes);
  if (e != cudaSuccess) return e;
  const dim3 grid((unsigned)((long long)a.in.rows * a.in.cluster));
  return launch_pdl_cluster(k, grid, dim3(kStreamThreads), bytes, s, a.in.cluster, a);
}

}  // namespace

cudaError_t launch_score_rows(const ScoreArgs& a, bool f32, bool fused, bool vec, cudaStream_t s) {
  return dispatch_rows(a.in, f32, fused, vec, [&](auto t, auto f, auto v) {
    return launch_score_t<typename decltype(t)::type, decltype(f)::value, decltype(v)::value>(a, s);
  });
}

}  // namespace dels
