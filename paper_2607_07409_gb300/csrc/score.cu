// Scoring of vocabulary rows: the log-probability of one given token of each
// row, the row's entropy and its top_k most likely entries, in one pass.
//
//   log q_v = (l_v - m) / T - ln S,   S = sum_v exp((l_v - m) / T)
//   H       = ln S - (1 / S) sum_v exp((l_v - m) / T) (l_v - m) / T
//
// The alternatives cost no second read of the row: every thread keeps the largest entry
// of each of its blocks of a few items; a value that K threads' largest reach is at most
// the K-th largest entry of the slice, and only the blocks that reach it are read again
// for their entries.
//
// What bounds it, on rows of 151936: without alternatives 1024 bf16 rows take 58 us
// (5.4 TB/s), the stream's instructions beside the reads. 64 alternatives make them 78 us
// (4.0 TB/s): lists, gathers and sorts are some 13,000 cycles of latency for each CTA
// that other CTAs' streams only partly hide, which is why few CTAs share a row. 128
// fused float32 rows with 8 take 37 us (4.3 TB/s), 1024 fused bf16 rows with 20 157 us
// (4.0 TB/s: 21 instructions a column, as every operation of the fused value is rounded).
// One row is 10 us, the latency of one slice's stream, selection and merge.
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
  float lanes[kStreamWarps][32];           // each warp's thread maxima in order, and how many there are
  int counts[kStreamWarps];
  int ncand, njobs;
};

// The K largest of cand[0 .. n) to best[] in order (all threads). Up to 128: each one's
// place is the number above it, counted by the threads that share it. More: a bitonic
// network, E a thread, exchanges inside a warp by shuffles. (Cycles of 36, 95 and 220:
// 1300, 2700 and 9000 counted, 3500, 5000 and 6500 by the network.)
template <int E>
__device__ __forceinline__ void sort_network(ScoreShared& sh, SelectShared& sel, int n, int K) {
  const int tid = threadIdx.x;
  unsigned long long x[E];
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = e * kStreamThreads + tid < n ? sel.cand[e * kStreamThreads + tid] : 0ull;
  int size = 32;
  while (size < n) size *= 2;
  for (int k = 2; k <= size; k *= 2)
    for (int d = k >> 1; d > 0; d >>= 1) {
      if (d >= kStreamThreads) {                             // between a thread's own
#pragma unroll
        for (int m = 1; m < E; m *= 2) {
          if (d != m * kStreamThreads) continue;
#pragma unroll
          for (int e = 0; e < E; ++e) {
            if (e & m) continue;
            const bool down = ((e * kStreamThreads + tid) & k) == 0;
            const unsigned long long lo = x[e], hi = x[e | m];
            x[e] = down == (lo > hi) ? lo : hi;
            x[e | m] = down == (lo > hi) ? hi : lo;
          }
        }
        continue;
      }
      if (d >= 32) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < E; ++e) sel.cand[e * kStreamThreads + tid] = x[e];
        __syncthreads();
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int i = e * kStreamThreads + tid;
        const unsigned long long o =
            d >= 32 ? sel.cand[i ^ d] : __shfl_xor_sync(0xFFFFFFFFu, x[e], d);
        const bool larger = ((i & k) == 0) == ((i & d) == 0);
        x[e] = larger == (o > x[e]) ? o : x[e];
      }
    }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (e * kStreamThreads + tid < K) sh.best[e * kStreamThreads + tid] = x[e];
  __syncthreads();
}
__device__ void sort_best(ScoreShared& sh, SelectShared& sel, int n, int K) {
  const int tid = threadIdx.x;
  if (n > 128 && n <= kStreamThreads) return sort_network<1>(sh, sel, n, K);
  if (n > 128 && n <= 2 * kStreamThreads) return sort_network<2>(sh, sel, n, K);
  if (n > 128 && n <= 4 * kStreamThreads) return sort_network<4>(sh, sel, n, K);
  if (n > 128) return sort_network<8>(sh, sel, n, K);
  static_assert(kCandidates <= 8 * kStreamThreads, "eight a thread at most");
  for (int k = tid; k < K; k += kStreamThreads) sh.best[k] = 0ull;
  __syncthreads();
  int log_share = 0;               // 2^log_share threads a candidate
  while (log_share < 5 && n << (log_share + 1) <= kStreamThreads) ++log_share;
  const int share = 1 << log_share, part = tid & (share - 1);
  for (int i = tid >> log_share; i - (tid >> log_share) < n; i += kStreamThreads >> log_share) {
    const unsigned long long x = i < n ? sel.cand[i] : 0ull;
    int rank = 0;
#pragma unroll 4
    for (int j = part; j < n; j += share) rank += sel.cand[j] > x;
    for (int d = share >> 1; d > 0; d >>= 1) rank += __shfl_xor_sync(0xFFFFFFFFu, rank, d);
    if (part == 0 && x && rank < K) sh.best[rank] = x;
  }
  __syncthreads();
}

// The values of an item at `pos`, -inf outside the row (not in a stream's turn).
template <typename T, int F, bool VEC>
__device__ __forceinline__ void item_values(const FusedRow<T, F, VEC>& row, int pos, int k1, float (&x)[8]) {
  Item<T, F, VEC> v;
  float pr[8], s[8];
  if (VEC && pos >= row.sh && pos + kHalf<T> + 4 <= k1) {
    v.load_whole(row, pos, pr);
  } else {
    v.load(row, pos, k1, pr);
  }
  v.template values<false>(row, pr, x, s);
}

// Where this lane's `n` things go in a list that `count` counts: one addition a warp
// (all lanes converged).
__device__ __forceinline__ int reserve(int* count, int n) {
  const int lane = threadIdx.x & 31;
  int up = n;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int o = __shfl_up_sync(0xFFFFFFFFu, up, d);
    if (lane >= d) up += o;
  }
  int base = 0;
  if (lane == 31 && up > 0) base = atomicAdd(count, up);
  return __shfl_sync(0xFFFFFFFFu, base, 31) + up - n;
}

// The entries among x[8] of an item at `pos` that reach `floor_key`, into cand[] as far
// as it has room (all lanes converged; of no thread's item: x = -inf).
template <typename T, int F, bool VEC>
__device__ __forceinline__ void keep_entries(ScoreShared& sh, SelectShared& sel, const FusedRow<T, F, VEC>& row,
                                             int pos, const float (&x)[8], unsigned long long floor_key) {
  const float least = from_order_u32((unsigned)(floor_key >> 32));
  unsigned hits = 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i) hits |= x[i] >= least && x[i] > -INFINITY ? 1u << i : 0u;
  if (!__any_sync(0xFFFFFFFFu, hits != 0u)) return;
  for (int at = reserve(&sh.ncand, __popc(hits)); hits; hits &= hits - 1, ++at) {
    const int i = __ffs(hits) - 1;
    float v = x[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) v = i == j ? x[j] : v;
    const unsigned long long e = entry_key(v, elem_pos<T, VEC>(pos, i) - row.sh);
    if (at < kCandidates) sel.cand[at] = e >= floor_key ? e : 0ull;   // (of a tie past the floor: none)
  }
}

// The K largest of C lists of K entries in order (0 past their ends) to best[]: those
// that reach what K of them do, either K divided among the lists (the least of those) or
// all of one list (the largest of those).
__device__ void merge_best(ScoreShared& sh, SelectShared& sel, const unsigned long long* lists, int C, int K) {
  const int tid = threadIdx.x, lane = tid & 31, each = (K + C - 1) / C;
  if (tid == 0) sh.ncand = 0;
  unsigned long long fair = lane < C ? lists[lane * K + each - 1] : ~0ull;
  unsigned long long one = lane < C ? lists[lane * K + K - 1] : 0ull;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    const unsigned long long f = __shfl_xor_sync(0xFFFFFFFFu, fair, d), o = __shfl_xor_sync(0xFFFFFFFFu, one, d);
    fair = f < fair ? f : fair;
    one = o > one ? o : one;
  }
  const unsigned long long least = fair > one ? fair : one;
  __syncthreads();
  for (int i0 = tid - lane; i0 < C * K; i0 += kStreamThreads) {
    const int i = i0 + lane;
    const unsigned long long e = i < C * K ? lists[i] : 0ull;
    const bool in = e && e >= least;
    const int at = reserve(&sh.ncand, in ? 1 : 0);
    if (in) sel.cand[at] = e;
  }
  __syncthreads();
  sort_best(sh, sel, sh.ncand, K);
}

// What at least K entries of the slice reach, as order_u32, for more than 128 entries
// (all threads): four lists a warp of 32 maxima in order, each of every fourth block of
// its threads, and of each list its share of K. From the threads' maxima alone 256 entries
// are the least of all of them, which thousands reach (one row: 200 us, from these 33).
__device__ __noinline__ unsigned reached_by_blocks(SelectShared& sel, const float* bmax, int slots, int K) {
  constexpr int kPer = 4;
  static_assert(kStreamWarps * kPer == 32, "a lane for every list");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  float* lists = reinterpret_cast<float*>(sel.cand);
  int* counts = sel.jobs;
  for (int j = 0; j < kPer; ++j) {
    float t = -INFINITY;
    for (int b = j; b < slots; b += kPer) t = fmaxf(t, bmax[b * kStreamThreads + tid]);
    const int have = __popc(__ballot_sync(0xFFFFFFFFu, t > -INFINITY));
#pragma unroll
    for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
      for (int d = k >> 1; d > 0; d >>= 1) {
        const float o = __shfl_xor_sync(0xFFFFFFFFu, t, d);
        t = ((lane & k) == 0) == ((lane & d) == 0) ? fmaxf(t, o) : fminf(t, o);
      }
    lists[(warp * kPer + j) * 32 + lane] = t;
    if (lane == 0) counts[warp * kPer + j] = have;
  }
  __syncthreads();
  const int cnt = counts[lane];
  const int live = __popc(__ballot_sync(0xFFFFFFFFu, cnt > 0));
  const int each = live ? (K + live - 1) / live : K;
  const bool fair = __all_sync(0xFFFFFFFFu, cnt == 0 || cnt >= each) && live;
  const float least = -warp_max(cnt > 0 && cnt >= each ? -lists[lane * 32 + each - 1] : -INFINITY);
  __syncthreads();                 // (the lists' place is the jobs' and the entries')
  return order_u32(fair ? least : -INFINITY);
}

// This CTA's K largest entries of its slice into sh.best. `top`: the largest
// entry of the calling thread; bmax: [slot][thread] the largest of a thread's groups
// slot << shift .. of the stream.
template <int U, typename T, int F, bool VEC>
__device__ void slice_top(ScoreShared& sh, SelectShared& sel, const float* bmax, int shift,
                          const FusedRow<T, F, VEC>& row, int k0, int k1, int K, float top) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int items = (k1 - k0 + kStreamStep - 1) / kStreamStep, groups = (items + U - 1) / U;
  const int slots = (groups + (1 << shift) - 1) >> shift;
  // What at least K entries reach: the warps' thread maxima in order, and of them either
  // K divided among the warps (the least of those), or all K of one warp (the largest of
  // those); both count entries of K threads or more.
  float t = top;
#pragma unroll
  for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
    for (int d = k >> 1; d > 0; d >>= 1) {
      const float o = __shfl_xor_sync(0xFFFFFFFFu, t, d);
      t = ((lane & k) == 0) == ((lane & d) == 0) ? fmaxf(t, o) : fminf(t, o);
    }
  sh.lanes[warp][lane] = t;
  const int have = __popc(__ballot_sync(0xFFFFFFFFu, top > -INFINITY));
  if (lane == 0) sh.counts[warp] = have;
  if (tid == 0) sh.ncand = sh.njobs = 0;
  __syncthreads();
  unsigned tau;
  {
    const int w = lane & (kStreamWarps - 1), cnt = sh.counts[w];
    const int live = __popc(__ballot_sync(0xFFFFFFFFu, cnt > 0)) / (32 / kStreamWarps);
    const int each = live ? (K + live - 1) / live : K;
    const bool fair = __all_sync(0xFFFFFFFFu, cnt == 0 || cnt >= each) && live;
    float least_of = cnt > 0 && cnt >= each ? sh.lanes[w][each - 1] : INFINITY;
    least_of = -warp_max(-least_of);
    const float one = warp_max(K <= cnt ? sh.lanes[w][K - 1] : -INFINITY);
    tau = order_u32(fmaxf(fair ? least_of : -INFINITY, one));
  }
  if (K > 128) tau = reached_by_blocks(sel, bmax, slots, K);
  const float least = from_order_u32(tau);
  unsigned long long floor_key = (unsigned long long)tau << 32;     // what an entry has to reach
  unsigned hits = 0u;                                               // (kSlots bits)
  if (top >= least && top > -INFINITY) {
    for (int b = 0; b < slots; ++b) hits |= bmax[b * kStreamThreads + tid] >= least ? 1u << b : 0u;
  }
  for (int j = reserve(&sh.njobs, __popc(hits)); hits; hits &= hits - 1, ++j)
    if (j < kJobs) sel.jobs[j] = (__ffs(hits) - 1) * kStreamThreads + tid;
  __syncthreads();
  if (sh.njobs <= kJobs) {
    // a lane per item of a job, two of them at a time
    constexpr int kLogU = U == 4 ? 2 : U == 2 ? 1 : 0;
    static_assert(U == 1 << kLogU, "a power of two");
    const int log_per = kLogU + shift, n = sh.njobs << log_per;
    for (int i0 = warp * 32; i0 < n; i0 += 2 * kStreamThreads) {
      float x[2][8];
      int pos[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int i = i0 + h * kStreamThreads + lane;
        pos[h] = k1;
        if (i < n) {
          const unsigned job = (unsigned)sel.jobs[i >> log_per];
          const int it = ((int)(job / kStreamThreads) << log_per) + (i & ((1 << log_per) - 1));
          if (it < items) pos[h] = item_pos<T, VEC>(k0, it, (int)(job % kStreamThreads));
        }
        if (pos[h] < k1) {
          item_values(row, pos[h], k1, x[h]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[h][e] = -INFINITY;
        }
      }
      keep_entries(sh, sel, row, pos[0], x[0], floor_key);
      if (i0 + kStreamThreads < n) keep_entries(sh, sel, row, pos[1], x[1], floor_key);
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
        sort_best(sh, sel, n, K);
        for (int k = tid; k < K; k += kStreamThreads) sel.cand[k] = sh.best[k];
        floor_key = sh.best[K - 1];                                 // n > K: there are K
        if (tid == 0) sh.ncand = K;
        __syncthreads();
      }
      if ((tid >> 7) == (j & 1)) {
        const int pos = item_pos<T, VEC>(k0, j >> 1, tid);
        float x[8];
        item_values(row, pos, k1, x);
        keep_entries(sh, sel, row, pos, x, floor_key);
      }
      __syncthreads();
    }
  }
  sort_best(sh, sel, sh.ncand, K);
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
__global__ void __launch_bounds__(kStreamThreads, (F ? 3 : 4) - kFewer<T, F>) k_score_rows(ScoreArgs a) {
  extern __shared__ __align__(16) uint8_t dyn[];
  __shared__ ScoreShared sh;
  const long long r = begin_row(a.in);
  if (r == a.in.rows) return;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int C = a.in.cluster, K = a.top_k;
  const int rank = (int)(blockIdx.x & (C - 1));
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

  if (K > 0) slice_top<U>(sh, *reinterpret_cast<SelectShared*>(dyn), bmax, shift, stream.anew(), k0, k1, K, top);
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
    if (K > 0) merge_best(sh, *reinterpret_cast<SelectShared*>(dyn), slices, C, K);
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
    const float lq = (from_order_u32((unsigned)(e >> 32)) - all.m) * inv_t - ln_s;
    a.out_top_lp[r * K + k] = !ok ? NAN : has ? lq : -INFINITY;
  }
}

template <typename T, int F, bool VEC>
cudaError_t launch_score_t(const ScoreArgs& a, cudaStream_t s) {
  const auto k = k_score_rows<T, F, VEC>;
  // the split: 1024, 608 and 500 bf16 rows of 608 KB gain 4 to 20 %, 1024 of 256 KB lose
  // 3; float32 rows, whose reads fill the time as they are, lose too (500: 134, 143 us)
  return launch_rows(
      k, a, true, sizeof(T) == 2 && row_bytes<T, F>(a.in) > 1 << 19,
      [&](const StreamRows& in) {
        return ring_bytes<T, F, VEC>() + (a.top_k > 0 ? (size_t)kSlots * kStreamThreads * 4 : 0) +
               (in.cluster > 1 ? (size_t)in.cluster * a.top_k * 8 : 0);
      },
      s);
}

}  // namespace

cudaError_t launch_score_rows(const ScoreArgs& a, bool f32, bool fused, bool vec, cudaStream_t s) {
  return dispatch_rows(a.in, f32, fused, vec, [&](auto t, auto f, auto v) {
    return launch_score_t<typename decltype(t)::type, decltype(f)::value, decltype(v)::value>(a, s);
  });
}

}  // namespace dels
