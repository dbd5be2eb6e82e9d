// Speculative sampling from given probabilities and uniforms.
//
// A cluster of 1 to 8 CTAs takes a request. The first warp of each finds the tokens kept, a
// lane a position, so that their reads wait for one another no more than once; then the row that the
// bonus token comes from is summed, once: a warp has a run of groups of 256 columns. The
// warps' sums meet in shared memory, the CTAs' in each other's; the CTA that has the border reads
// the run it lies in again, out of L2, a sixteenth a warp, and the warp whose group has it finds the column.
//
// Sums decide which token comes out, so float32's are not enough, and float64 itself issues
// at 1/64 of float32's rate here: a lane keeps a float32 sum and what its additions
// rounded off (Knuth's two-sum), 48 bits, two such in packed pairs, and only totals are float64, in one warp, of
// a row and, where it is long, of each of its parts. A difference p - q is kept the same way.
//
// What bounds it: latency, one part after another. 64 blocks of 16 over 151936 (78 MB, 11.5 us at a
// copy's rate) 18 us, 64 draws 10.6 (5.8): 2 for the tokens, the stream in two CTAs an SM (1.7 of them), 4 for
// the sums, the exchange, the border's run and its column; one block of 8 over 32000 6.9 us. (One warp that walked the
// border's run alone, by sums kept on the way: 24, 13.2, 7.8. The rows through a ring of asynchronous copies
// hid the latency of blocks' reads and not what its instructions cost draws: 23.1 and 15.6 then.)
#include <cfloat>

#include "dels_device.cuh"
#include "row_stream.cuh"

namespace dels {
namespace {

constexpr int kGivenThreads = 512, kGivenWarps = kGivenThreads / 32;
constexpr int kGroup = 256;                // columns of a warp's step, 8 a lane
// Groups after which a warp closes a sum and adds it up in float64: more than a warp has of a row of 262144 columns. What
// additions rounded off is itself rounded: of 256 a sum of the lane, 2^-33 of it at worst. (Closed never, a
// row of 2^28 weights, the first half 1.1, came out some columns off.)
constexpr int kClose = 64;

__device__ __forceinline__ bool is_probability(float x) { return x >= 0.f && x < INFINITY; }

struct Kept {
  int a;               // tokens kept
  int token;           // the one rejected, or -1: all were kept
  int code;            // status bits
};

template <typename P, typename Q, bool DRAFT>
__device__ __forceinline__ Kept count_kept(const VerifyGivenArgs& a, int b) {
  const int lane = threadIdx.x & 31;
  Kept k{0, -1, 0};
  const float* u = a.uniforms + (long long)b * (a.n + 1);
  const int len = a.lengths ? __ldg(a.lengths + b) : a.n;
  const float last = __ldg(u + a.n);
  if (len < 0 || len > a.n || !(last >= 0.f && last < 1.f)) {
    k.code = DELS_STATUS_BAD_VALUE;
    return k;
  }
  for (int j0 = 0; j0 < len; j0 += 32) {
    const int j = j0 + lane;
    int token = -1, code = 0;
    bool stop = false;
    if (j < len) {
      token = __ldg(a.tokens + (long long)b * a.n + j);
      const float uj = __ldg(u + j);
      if (token < 0 || token >= a.V) code |= DELS_STATUS_BAD_TOKEN;
      if (!(uj >= 0.f && uj < 1.f)) code |= DELS_STATUS_BAD_VALUE;
      if (!code) {
        const float p = row_elem(static_cast<const P*>(a.target.p), b * a.target.ld_b + j * a.target.ld + token);
        const float q =
            DRAFT ? row_elem(static_cast<const Q*>(a.draft.p), b * a.draft.ld_b + j * a.draft.ld + token) : 1.f;
        if (!is_probability(p) || !is_probability(q)) code = DELS_STATUS_NONFINITE;
        stop = !((double)uj * (double)q < (double)p);       // (both exact)
      }
      stop |= code != 0;
    }
    const unsigned who = __ballot_sync(0xFFFFFFFFu, stop);
    if (who) {
      const int first = __ffs(who) - 1;
      k.a = j0 + first;
      k.token = __shfl_sync(0xFFFFFFFFu, token, first);
      k.code = __shfl_sync(0xFFFFFFFFu, code, first);
      return k;
    }
  }
  k.a = len;
  return k;
}

// 8 elements of a row for a lane: consecutive ones, or 32 apart where the rows lie anywhere
// (0 past the row's end).
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* p, int v0, int V, float (&x)[8]) {
  const int lane = threadIdx.x & 31;
  if (VEC && v0 + kGroup <= V) {
    const T* at = p + v0 + lane * 8;
    Raw8<T> w;
#pragma unroll
    for (int k = 0; k < Raw8<T>::W; ++k) w.w[k] = __ldg(reinterpret_cast<const uint4*>(at + 4 * k));
    w.unpack(x);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int v = VEC ? v0 + lane * 8 + i : v0 + i * 32 + lane;
      x[i] = v < V ? row_elem(p, v) : 0.f;
    }
  }
}

struct Sum2 {
  float hi, lo;
  // Adds x >= 0, and y, far below it.
  __device__ __forceinline__ void add(float x, float y) {
    const float t = __fadd_rn(hi, x), b = __fsub_rn(t, hi);
    const float e = __fadd_rn(__fsub_rn(hi, __fsub_rn(t, b)), __fsub_rn(x, b));
    hi = t;
    lo = __fadd_rn(lo, __fadd_rn(e, y));
  }
};
__device__ __forceinline__ f32x2 sub2(f32x2 a, f32x2 b) { return fma2(b, both2(-1.f), a); }
// Two of them in pairs of float32, two operations an instruction.
struct Sum2Pair {
  f32x2 hi, lo;
  __device__ __forceinline__ f32x2 left(f32x2 x) {       // what the addition of x rounds off
    const f32x2 t = add2(hi, x), b = sub2(t, hi);
    const f32x2 e = add2(sub2(hi, sub2(t, b)), sub2(x, b));
    hi = t;
    return e;
  }
  __device__ __forceinline__ void add(f32x2 x) { lo = add2(lo, left(x)); }
  __device__ __forceinline__ void add(f32x2 x, f32x2 y) { lo = add2(lo, add2(left(x), y)); }
  __device__ __forceinline__ Sum2 both() const {
    float h0, h1, l0, l1;
    split2(hi, h0, h1);
    split2(lo, l0, l1);
    Sum2 s{h0, l0};
    s.add(h1, l1);
    return s;
  }
};
// max(0, p - q) as float32 and what it rounded off (p > q >= 0: both exact, Dekker's fast two-sum).
__device__ __forceinline__ void rest_of(const float* p, const float* q, float* w, float* e) {
  const f32x2 p2 = pair2(p[0], p[1]), q2 = pair2(q[0], q[1]), d2 = sub2(p2, q2);
  float d[2];
  split2(d2, d[0], d[1]);
  split2(sub2(sub2(p2, d2), q2), e[0], e[1]);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    w[i] = fmaxf(d[i], 0.f);
    e[i] = d[i] > 0.f ? e[i] : 0.f;
  }
}

// A warp's sum, in every lane (fixed order).
__device__ __forceinline__ Sum2 warp_sum2(Sum2 s) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    const float hi = __shfl_xor_sync(0xFFFFFFFFu, s.hi, d), lo = __shfl_xor_sync(0xFFFFFFFFu, s.lo, d);
    s.add(hi, lo);
  }
  return s;
}
__device__ __forceinline__ double total_of(const Sum2& s) { return (double)s.hi + (double)s.lo; }
// Sums up to and including each lane's.
__device__ __forceinline__ double warp_scan(double x, int lanes) {
  const int lane = threadIdx.x & 31;
  for (int d = 1; d < lanes; d <<= 1) {
    const double up = __shfl_up_sync(0xFFFFFFFFu, x, d);
    if (lane >= d) x += up;
  }
  return x;
}

// The first lane whose sum up to and including its own is over the border, of those with weight: sums up to the same
// column differ with the order they were taken in, and an empty lane's may be over where the one before it is not. By
// roundings none may be over: then the last with weight (-1: none has any).
__device__ __forceinline__ int first_over(bool over, bool weight) {
  const unsigned some = __ballot_sync(0xFFFFFFFFu, weight), at = __ballot_sync(0xFFFFFFFFu, over) & some;
  return at ? __ffs(at) - 1 : 31 - __clz(some);
}

struct SlicePart {
  double sum;
  int bad, pad;
};
// What the first warp of a CTA finds from the sums.
struct Border {
  double at;           // u times the whole
  double before;       // the sum up to the run
  int run;             // the warp whose columns have the border, or -1
  int again;           // nothing is left of p - q
  int code;
};

// A warp's sum so far, added to *far in float64.
__device__ __noinline__ void close_sum(double* far, f32x2 hi, f32x2 lo) {
  const Sum2 s = warp_sum2(Sum2Pair{hi, lo}.both());
  if ((threadIdx.x & 31) == 0) *far += total_of(s);
}

// FAR: a warp has more than kClose groups.
template <typename P, typename Q, bool DRAFT, bool VEC, bool FAR>
__global__ void __launch_bounds__(kGivenThreads, 2) k_verify_given(const VerifyGivenArgs a, int cluster) {
  __shared__ Sum2 warp_sum[kGivenWarps];
  __shared__ double warp_far[kGivenWarps];           // what a warp's sum has been closed at, with warp_sum behind it
  __shared__ int warp_bad[kGivenWarps];
  __shared__ SlicePart parts[2][kMaxCluster];
  __shared__ Border border;
  __shared__ Kept kept;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int b = blockIdx.x / cluster, rank = blockIdx.x - b * cluster;
  if (cluster > 1) cluster_arrive_relaxed();
  pdl_wait();
  if (tid == 0) pdl_trigger();
  if (warp == 0) {
    const Kept k = count_kept<P, Q, DRAFT>(a, b);
    if (lane == 0) kept = k;
  }
  __syncthreads();
  const Kept k = kept;
  if (cluster > 1) cluster_wait();
  int bonus = -1, code = k.code;
  bool mine = false;
  if (!code) {                              // (the same in every CTA of the request)
    const P* p = static_cast<const P*>(a.target.p) + b * a.target.ld_b + k.a * a.target.ld;
    const Q* q = DRAFT ? static_cast<const Q*>(a.draft.p) + b * a.draft.ld_b + k.a * a.draft.ld : nullptr;
    const int groups = (a.V + kGroup - 1) / kGroup, runs = cluster * kGivenWarps;
    const auto first_of = [&](int w) { return (int)((long long)groups * (rank * kGivenWarps + w) / runs); };
    // The weights of a group: from max(0, p - q), or from p.
    const auto weights = [&](bool rest, int g, const float (&x)[8], const float (&y)[8], float (&w)[8], float (&e)[8]) {
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        if (DRAFT && rest) {
          rest_of(x + i, y + i, w + i, e + i);
        } else {
          w[i] = x[i], w[i + 1] = x[i + 1];
          e[i] = e[i + 1] = 0.f;
        }
      }
      if (!DRAFT && rest && (unsigned)(k.token - g * kGroup) < (unsigned)kGroup) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (g * kGroup + (VEC ? lane * 8 + i : i * 32 + lane) == k.token) w[i] = 0.f;
      }
    };
    // The sum of warp `lane`, and whether it has any weight, as the first warp reads them.
    const auto warp_total = [&] {
      if (lane >= kGivenWarps) return 0.0;
      return FAR ? warp_far[lane] + total_of(warp_sum[lane]) : total_of(warp_sum[lane]);
    };
    const auto warp_some = [&] {
      return lane < kGivenWarps && (warp_sum[lane].hi > 0.f || (FAR && warp_far[lane] > 0.0));
    };
    bool rest = k.token >= 0;
    for (int pass = 0;; ++pass) {
      Sum2Pair sums{0ull, 0ull};
      unsigned most = 0;                    // of the bits: what is no probability is above infinity's, or it
      const auto add = [&](int g, const float (&x)[8], const float (&y)[8]) {
        // + 0: -0 is a probability
        const auto look = [&](const float (&z)[8]) {
#pragma unroll
          for (int i = 0; i < 8; i += 2) {
            float z0, z1;
            split2(add2(pair2(z[i], z[i + 1]), 0ull), z0, z1);
            most = max(most, max(__float_as_uint(z0), __float_as_uint(z1)));
          }
        };
        float w[8], e[8];
        weights(rest, g, x, y, w, e);
        look(x);
        if (DRAFT && rest) look(y);
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          if (DRAFT) sums.add(pair2(w[i], w[i + 1]), pair2(e[i], e[i + 1]));
          else sums.add(pair2(w[i], w[i + 1]));
        }
      };
      if (FAR && lane == 0) warp_far[warp] = 0.0;
      const int g1 = first_of(warp + 1);
      constexpr int kAhead = 2;              // groups read at a time (four of plain rows spill: 64 draws 12.2 us for 11.0)
      for (int g = first_of(warp);;) {
        const int stop = FAR ? min(g + kClose, g1) : g1;
        for (; g < stop; g += kAhead) {
          float x[kAhead][8], y[kAhead][8];
#pragma unroll
          for (int u = 0; u < kAhead; ++u) {
            if (g + u >= stop) continue;
            load8<P, VEC>(p, (g + u) * kGroup, a.V, x[u]);
            if (DRAFT && rest) load8<Q, VEC>(q, (g + u) * kGroup, a.V, y[u]);
          }
#pragma unroll
          for (int u = 0; u < kAhead; ++u)
            if (g + u < stop) add(g + u, x[u], y[u]);
        }
        if (!FAR || g >= g1) break;
        close_sum(&warp_far[warp], sums.hi, sums.lo);
        sums = Sum2Pair{0ull, 0ull};
      }
      const Sum2 s = warp_sum2(sums.both());
      const int bad = __any_sync(0xFFFFFFFFu, most >= 0x7F800000u);
      if (lane == 0) {
        warp_sum[warp] = s;
        warp_bad[warp] = bad;
      }
      __syncthreads();
      // float64 from here on, by the first warp: every warp's instruction takes 16 cycles of the SM's
      double own = 0.0;
      if (warp == 0) {
        own = warp_scan(warp_total(), kGivenWarps);
        const int own_bad = __any_sync(0xFFFFFFFFu, lane < kGivenWarps && warp_bad[lane]);
        const double sum = __shfl_sync(0xFFFFFFFFu, own, kGivenWarps - 1);
        if (cluster > 1) {
          if (lane < cluster) {
            const uint32_t at = cluster_map(smem_u32(&parts[pass][rank]), (uint32_t)lane);
            const long long bits = __double_as_longlong(sum);
            st_cluster_f32(at, __int_as_float((int)(bits & 0xFFFFFFFFll)));
            st_cluster_f32(at + 4, __int_as_float((int)(bits >> 32)));
            st_cluster_f32(at + 8, __int_as_float(own_bad));
          }
        } else if (lane == 0) {
          parts[pass][0] = SlicePart{sum, own_bad, 0};
        }
        __syncwarp();
      }
      if (cluster > 1) {
        cluster_arrive();
        cluster_wait();
      }
      if (warp == 0) {
        // (every CTA of the request has the same parts, takes the same steps and finds the same one)
        const SlicePart part = lane < cluster ? parts[pass][lane] : SlicePart{0.0, 0, 0};
        const double upto = warp_scan(part.sum, kMaxCluster);
        const double total = __shfl_sync(0xFFFFFFFFu, upto, kMaxCluster - 1);
        // (a run's sum in float32 pairs is beyond them where the whole is: the same in any split)
        const bool any_bad = __any_sync(0xFFFFFFFFu, part.bad != 0) || !(total <= (double)FLT_MAX);
        Border f{(double)__ldg(a.uniforms + (long long)b * (a.n + 1) + a.n) * total, 0.0, -1, 0, 0};
        if (any_bad || (!(total > 0.0) && !rest)) f.code = DELS_STATUS_NONFINITE;
        else if (!(total > 0.0)) f.again = 1;
        else if (first_over(upto > f.at, part.sum > 0.0) == rank) {
          const double before = __shfl_sync(0xFFFFFFFFu, upto, max(rank - 1, 0));
          const double c = (rank ? before : 0.0) + own;            // up to and including the lane's run
          f.run = first_over(c > f.at, warp_some());
          const double prev = __shfl_sync(0xFFFFFFFFu, c, max(f.run - 1, 0));
          f.before = f.run ? prev : (rank ? before : 0.0);
        }
        if (lane == 0) border = f;
      }
      __syncthreads();
      const Border f = border;
      if (f.again) {
        rest = false;
        __syncthreads();                    // (the sums are written again)
        continue;
      }
      code = f.code;
      if (f.run >= 0) {
        // The run in sixteen parts, a warp each, the one with the border in sixteen again, until a part is a group at
        // most, which then lies in its warp's registers. (f.run and f.before become those of the part.)
        float w[8], e[8];
        int at, lo = first_of(f.run), hi = first_of(f.run + 1);
        double base = f.before;
        int part;
        for (;;) {
          const auto edge = [&](int w2) { return lo + (int)((long long)(hi - lo) * w2 / kGivenWarps); };
          Sum2 t{0.f, 0.f};
#pragma unroll
          for (int i = 0; i < 8; ++i) w[i] = e[i] = 0.f;
          at = edge(warp);
          if (FAR && lane == 0) warp_far[warp] = 0.0;
          for (int g = at; g < edge(warp + 1); ++g) {
            if (FAR && g > at && (g - at) % (kClose / 2) == 0) {
              const Sum2 far = warp_sum2(t);
              if (lane == 0) warp_far[warp] += total_of(far);
              t = Sum2{0.f, 0.f};
            }
            float x[8], y[8];
            load8<P, VEC>(p, g * kGroup, a.V, x);
            if (DRAFT && rest) load8<Q, VEC>(q, g * kGroup, a.V, y);
            weights(rest, g, x, y, w, e);
#pragma unroll
            for (int i = 0; i < 8; ++i) t.add(w[i], e[i]);
          }
          t = warp_sum2(t);
          if (lane == 0) warp_sum[warp] = t;
          __syncthreads();
          if (warp == 0) {
            const double c = base + warp_scan(warp_total(), kGivenWarps);
            const int pick = max(first_over(c > f.at, warp_some()), 0);
            const double prev = __shfl_sync(0xFFFFFFFFu, c, max(pick - 1, 0));
            if (lane == 0) {
              border.run = pick;
              border.before = pick ? prev : base;
            }
          }
          __syncthreads();
          part = border.run;
          base = border.before;
          if (hi - lo <= kGivenWarps) break;
          const int next = edge(part);
          hi = edge(part + 1);
          lo = next;
        }
        mine = warp == part;
        if (mine) {
          // The column. VEC: the lanes in order, each its 8; else 8 times the lanes in order.
          constexpr int kParts = VEC ? 1 : 8, kEach = 8 / kParts;
          bool found = false;
#pragma unroll
          for (int h = 0; h < kParts; ++h) {
            if (found) continue;
            Sum2 t{0.f, 0.f};
#pragma unroll
            for (int i = 0; i < kEach; ++i) t.add(w[h * kEach + i], e[h * kEach + i]);
            Sum2 upto = t;                    // up to and including the lane's
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
              const float hi = __shfl_up_sync(0xFFFFFFFFu, upto.hi, d), lo = __shfl_up_sync(0xFFFFFFFFu, upto.lo, d);
              if (lane >= d) upto.add(hi, lo);
            }
            const double incl = total_of(upto);
            const double up = __shfl_up_sync(0xFFFFFFFFu, incl, 1);
            const int who = first_over(base + incl > f.at, t.hi > 0.f);
            const bool over = __any_sync(0xFFFFFFFFu, base + incl > f.at && t.hi > 0.f);
            if (who >= 0) {                   // the border, or for now the last with weight
              const double left = f.at - (base + (lane ? up : 0.0));       // of the lane's own
              const float left_hi = (float)left, left_lo = (float)(left - (double)left_hi);
              int v = -1;
              bool past = false;
              Sum2 c{0.f, 0.f};
#pragma unroll
              for (int i = 0; i < kEach; ++i) {
                const float w2 = w[h * kEach + i];
                c.add(w2, e[h * kEach + i]);
                if (!past && w2 > 0.f) v = at * kGroup + (VEC ? lane * 8 + i : h * 32 + lane);
                past |= v >= 0 && __fadd_rn(__fsub_rn(c.hi, left_hi), __fsub_rn(c.lo, left_lo)) > 0.f;
              }
              bonus = __shfl_sync(0xFFFFFFFFu, v, who);
            }
            found = over;
            base += __shfl_sync(0xFFFFFFFFu, incl, 31);
          }
        }
      }
      break;
    }
  }
  if (mine && lane == 0) a.out_bonus[b] = bonus;
  if (rank == 0 && tid == 0) {
    a.out_accept[b] = k.a;
    if (code) {
      a.out_bonus[b] = -1;
      raise_status(a.status, code);
    }
  }
}

template <typename P, typename Q, bool DRAFT>
cudaError_t launch_types(const VerifyGivenArgs& a, bool vec, int cluster, cudaStream_t s) {
  const bool far = (long long)a.V > (long long)kClose * kGroup * kGivenWarps * cluster;
  const auto k = far ? (vec ? k_verify_given<P, Q, DRAFT, true, true> : k_verify_given<P, Q, DRAFT, false, true>)
                     : (vec ? k_verify_given<P, Q, DRAFT, true, false> : k_verify_given<P, Q, DRAFT, false, false>);
  return launch_pdl_cluster(k, dim3((unsigned)a.B * (unsigned)cluster), dim3(kGivenThreads), 0, s, cluster, a, cluster);
}

// All rows start on 16-byte boundaries.
bool rows_aligned(const GivenRows& g) {
  const int es = g.f32 ? 4 : 2;
  return (reinterpret_cast<uintptr_t>(g.p) & 15u) == 0 && g.ld * es % 16 == 0 && g.ld_b * es % 16 == 0;
}

}  // namespace

cudaError_t launch_verify_given(const VerifyGivenArgs& a, cudaStream_t s) {
  const int sms = device_sm_count();
  if (sms <= 0) return cudaErrorInvalidValue;
  // as many CTAs a request as two an SM hold, at a warp's group each or nearly
  int c = 1;
  while (c < kMaxCluster && (long long)a.B * 2 * c <= 2 * sms && a.V >= 2 * c * 8 * kGroup) c *= 2;
  const bool vec = rows_aligned(a.target) && (!a.draft.p || rows_aligned(a.draft));
  const auto with_draft = [&](auto p) {
    using P = typename decltype(p)::type;
    if (!a.draft.p) return launch_types<P, P, false>(a, vec, c, s);
    return a.draft.f32 ? launch_types<P, float, true>(a, vec, c, s) : launch_types<P, uint16_t, true>(a, vec, c, s);
  };
  return a.target.f32 ? with_draft(TypeOf<float>{}) : with_draft(TypeOf<uint16_t>{});
}

}  // namespace dels
