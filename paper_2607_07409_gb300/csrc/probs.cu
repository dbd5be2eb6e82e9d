// Probabilities of plain or fused rows: p_v = exp(z_v - m) / sum exp(z - m), z = l / T.
//
// A cluster of 1 to 8 CTAs takes a row, each a slice of its columns. A slice is read once: its
// values (as stored where they are plain, else fused, in float32) stay in shared memory,
// so that a row costs its bytes in and its bytes out. A CTA takes its slice's largest value
// and the sum beside it; the CTAs exchange the two, and what is left is a factor for
// each. Rows whose slices do not fit are read three times.
//
// What bounds it: the bytes of plain rows (1088 bf16 rows of 151936 to float32 160 us, 147 at a
// copy's rate); of fused float32 rows three CTAs an SM, in 2.2 rounds, that load, exchange and store one
// after another (128 rows of 151936 59 us, 34.7 at that rate). An exponential is taken twice (for the
// sum, for the output), which costs less than keeping it where the slice is held in bf16.
#include <algorithm>

#include <cuda_bf16.h>

#include "row_stream.cuh"

namespace dels {
namespace {

// 2^(d c), d = x - m <= 0 (or NaN), c + c_lo = log2(e) / T. d c takes one rounding, which differs from
// entry to entry; c's own would be the same in all of them, and the second fma puts it right
// (without it probabilities were off by 6e-7 of the row's norm, a library's softmax by 1.5e-7). c_lo > 0
// keeps d = -inf from being NaN, which stays NaN. In pairs: two roundings an instruction. (d c split
// into a whole number and the rest took three times the instructions, for a tenth of the error left.)
struct Exponent {
  float m, c, c_lo;
  __device__ __forceinline__ f32x2 two(f32x2 x) const {
    const f32x2 d = add2(x, both2(-m));
    float z0, z1;
    split2(fma2(d, both2(c_lo), mul2(d, both2(c))), z0, z1);
    return pair2(ex2_approx(z0), ex2_approx(z1));
  }
  __device__ __forceinline__ float operator()(float x) const {
    float a, b;
    split2(two(both2(x)), a, b);
    return a;
  }
};

struct SliceSum {
  float m, s;
};

__device__ __forceinline__ void held_put(float* h, int i, float x) { h[i] = x; }
__device__ __forceinline__ void held_put(uint16_t* h, int i, float x) { h[i] = (uint16_t)(__float_as_uint(x) >> 16); }
__device__ __forceinline__ float held_get(const float* h, int i) { return h[i]; }
__device__ __forceinline__ float held_get(const uint16_t* h, int i) { return bf16_to_f(h[i]); }

// Four values from element i of a slice; `whole`: they lie on 4 elements' boundary.
template <typename H>
__device__ __forceinline__ void held_get4(const H* h, int i, bool whole, float (&x)[4]) {
  if (whole) {
    if constexpr (sizeof(H) == 4) {
      const float4 u = *reinterpret_cast<const float4*>(h + i);
      x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w;
    } else {
      const uint2 u = *reinterpret_cast<const uint2*>(h + i);
      x[0] = bf16lo(u.x); x[1] = bf16hi(u.x); x[2] = bf16lo(u.y); x[3] = bf16hi(u.y);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = held_get(h, i + j);
  }
}

// Four outputs from `out` on, which lies on their 16 (bf16: 8) bytes.
__device__ __forceinline__ void put4(float* out, const float (&x)[4]) {
  __stcs(reinterpret_cast<float4*>(out), make_float4(x[0], x[1], x[2], x[3]));
}
__device__ __forceinline__ void put4(__nv_bfloat16* out, const float (&x)[4]) {
  const __nv_bfloat162 lo = __floats2bfloat162_rn(x[0], x[1]), hi = __floats2bfloat162_rn(x[2], x[3]);
  __stcs(reinterpret_cast<uint2*>(out),
         make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi)));
}
__device__ __forceinline__ void put1(float* out, float x) { *out = x; }
__device__ __forceinline__ void put1(__nv_bfloat16* out, float x) { *out = __float2bfloat16_rn(x); }

// CTAs an SM (its registers): five of plain rows and of fused bf16 ones that are held, of other fused ones four (774 fused
// bf16 rows of 32000, to float32: at three 67.7 us, at five 57.9; 155 of 32003 to bf16 20.5 and 16.9. Not held, 64 of
// 500000, float32 and bf16: at three 285 and 231 us, at four 258 and 219, where the float32 ones spill some
// registers; bf16 at five 256).
template <typename T, int F, bool HOLD>
constexpr int kProbsCtas = F == kPlain || (HOLD && sizeof(T) == 2) ? 5 : 4;

template <typename T, int F, bool VEC, typename O, bool HOLD>
__global__ void __launch_bounds__(kStreamThreads, kProbsCtas<T, F, HOLD>) k_row_probs(const ProbsArgs a) {
  using H = std::conditional_t<F == kPlain, T, float>;
  extern __shared__ __align__(16) uint8_t smem[];
  H* held = reinterpret_cast<H*>(smem);
  __shared__ float red[kStreamWarps], red_s[kStreamWarps];
  __shared__ SliceSum slices[kMaxCluster];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const unsigned C = a.in.cluster, r = blockIdx.x / C, rank = blockIdx.x - r * C;
  if (C > 1) cluster_arrive_relaxed();      // (the row's other CTAs have begun: waited for before they are written to)
  pdl_wait();
  if (tid == 0) pdl_trigger();
  const FusedRow<T, F, VEC> row(a.in, r);
  const long long first = (long long)rank * a.in.slice_cols;
  const int k0 = (int)min(first, (long long)row.end), k1 = (int)min(first + a.in.slice_cols, (long long)row.end);
  const int items = (k1 - k0 + kStreamStep - 1) / kStreamStep;

  const auto load = [&](int it, Item<T, F, VEC>& v, float (&pr)[8]) {
    const int pos = item_pos<T, VEC>(k0, it, tid);
    if (VEC && pos >= row.sh && pos + kHalf<T> + 4 <= k1) v.load_whole(row, pos, pr);
    else v.load(row, pos, k1, pr);           // -inf outside
  };
  // f(values, first position) of every item of the thread
  const auto each = [&](auto&& f) {
    constexpr int U = F == kPlain ? 4 : 2;
    for (int it = 0; it < items; it += U) {
      Item<T, F, VEC> v[U];
      float pr[U][8], x[8], sv[8];
#pragma unroll
      for (int u = 0; u < U; ++u) load(it + u, v[u], pr[u]);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        v[u].template values<true>(row, pr[u], x, sv);
        f(x, v[u].k);
      }
    }
  };

  float m = -INFINITY;                      // (NaN shows in the sums)
  const auto hold = [&](const float (&x)[8], int k) {
    if (VEC && k + kHalf<T> + 4 <= k1) {
      if constexpr (sizeof(H) == 2) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          w[i] = __byte_perm(__float_as_uint(x[2 * i]), __float_as_uint(x[2 * i + 1]), 0x7632);
        *reinterpret_cast<uint4*>(held + k - k0) = make_uint4(w[0], w[1], w[2], w[3]);
      } else {
        *reinterpret_cast<float4*>(held + k - k0) = make_float4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<float4*>(held + k - k0 + kHalf<T>) = make_float4(x[4], x[5], x[6], x[7]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int q = elem_pos<T, VEC>(k, i);
        if (q < k1) held_put(held, q - k0, x[i]);
      }
    }
  };
  if constexpr (VEC && HOLD && F != kSome) {
    // Whole items straight to their place, all of a thread's at once: l_L, and bf16 rows' l_S behind it, in the
    // 32 bytes that the 8 values then take as float32. (Through registers, four items in flight: 1088
    // plain bf16 rows 189 us.)
    const auto whole = [&](int pos) { return pos >= row.sh && pos + kHalf<T> + 4 <= k1; };
    for (int it = 0; it < items; ++it) {
      const int pos = item_pos<T, VEC>(k0, it, tid);
      if (!whole(pos)) continue;
      const uint32_t dst = smem_u32(held + (pos - k0));
      copy16(dst, row.L + pos);
      if constexpr (sizeof(T) == 4) copy16(dst + 4 * kHalf<T>, row.L + pos + kHalf<T>);
      else if constexpr (F != kPlain) copy16(dst + 16, row.S + pos);
    }
    copies_commit();
    // The whole ones U at a time: what they take beside their copies is read before the copies are waited for. Those
    // at the row's or the slice's ends one by one.
    constexpr int U = F == kPlain ? 1 : 2;
    const int p0 = item_pos<T, VEC>(k0, 0, tid), lead = p0 >= row.sh ? 0 : 1;
    const int past = k1 - kHalf<T> - 4 - p0 < 0 ? 0 : (k1 - kHalf<T> - 4 - p0) / kStreamStep + 1;
    const auto beside = [&](int pos, Item<T, F, VEC>& v, float (&pr)[8]) {
      v.k = pos;
      if constexpr (F != kPlain) {
        if constexpr (sizeof(T) == 4) v.s.load(row.S + pos, kHalf<T>);
        if (row.has_p() && (row.sh & 3) == 0) {        // (on its 16 bytes too: the prior starts there)
          const float4 a4 = __ldg(reinterpret_cast<const float4*>(row.P + pos));
          const float4 b4 = __ldg(reinterpret_cast<const float4*>(row.P + pos + kHalf<T>));
          pr[0] = a4.x; pr[1] = a4.y; pr[2] = a4.z; pr[3] = a4.w;
          pr[4] = b4.x; pr[5] = b4.y; pr[6] = b4.z; pr[7] = b4.w;
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) pr[i] = row.p_at(elem_pos<T, VEC>(pos, i));
        }
      }
    };
    const auto take = [&](Item<T, F, VEC>& v, const float (&pr)[8]) {
      const uint4* at = reinterpret_cast<const uint4*>(held + (v.k - k0));
      v.l.w[0] = at[0];
      if constexpr (sizeof(T) == 4) v.l.w[1] = *reinterpret_cast<const uint4*>(held + (v.k - k0) + kHalf<T>);
      else if constexpr (F != kPlain) v.s.w[0] = at[1];
      float x[8], sv[8];
      v.template values<true>(row, pr, x, sv);
      m = fmaxf(m, max8(x));
      if (F != kPlain) hold(x, v.k);
    };
    bool waited = false;
    int it = lead;
    for (; it + U <= past; it += U) {
      Item<T, F, VEC> v[U];
      float pr[U][8];
#pragma unroll
      for (int u = 0; u < U; ++u) beside(p0 + (it + u) * kStreamStep, v[u], pr[u]);
      if (!waited) copies_wait<0>();
      waited = true;
#pragma unroll
      for (int u = 0; u < U; ++u) take(v[u], pr[u]);
    }
    if (!waited) copies_wait<0>();
    const int left = it;
#pragma unroll 1
    for (it = lead ? 0 : left; it < items; it = it < lead ? left : it + 1) {
      const int pos = p0 + it * kStreamStep;
      if (pos >= k1) break;
      Item<T, F, VEC> v;
      float pr[8], x[8], sv[8];
      if (whole(pos)) {
        beside(pos, v, pr);
        take(v, pr);
      } else {
        v.load(row, pos, k1, pr);
        v.template values<true>(row, pr, x, sv);
        m = fmaxf(m, max8(x));
        hold(x, v.k);
      }
    }
  } else {
    each([&](float (&x)[8], int k) {
      m = fmaxf(m, max8(x));
      if constexpr (HOLD) hold(x, k);
    });
  }
  m = warp_max(m);
  if (lane == 0) red[warp] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kStreamWarps; ++i) m = fmaxf(m, red[i]);
  // A slice of -inf alone has no reference: any finite one gives 0, and shows a NaN in it.
  const bool some = m > -INFINITY;
  const float ref = some ? m : 0.f;
  const Exponent ex{ref, a.in.scale, a.scale_lo};
  f32x2 s2 = 0ull;
  const auto add = [&](const float (&x)[8]) {
    s2 = add2(s2, add2(add2(ex.two(pair2(x[0], x[1])), ex.two(pair2(x[2], x[3]))),
                       add2(ex.two(pair2(x[4], x[5])), ex.two(pair2(x[6], x[7])))));
  };
  if constexpr (HOLD) {
    const int n = k1 - k0;
    constexpr int kApart = sizeof(H) == 4 ? 4 * kStreamThreads : 4;      // an item's fours, as in RowStream
    for (int i = tid * (sizeof(H) == 4 ? 4 : 8); i < n; i += kStreamStep) {
      float x[8], lo[4], hi[4];
      if (i + kApart + 4 <= n) {
        held_get4(held, i, true, lo);
        held_get4(held, i + kApart, true, hi);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          lo[j] = i + j < n ? held_get(held, i + j) : -INFINITY;
          hi[j] = i + kApart + j < n ? held_get(held, i + kApart + j) : -INFINITY;
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = lo[j], x[4 + j] = hi[j];
      add(x);
    }
  } else {
    each([&](float (&x)[8], int) { add(x); });
  }
  float s = sum2(s2);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
  if (lane == 0) red_s[warp] = s;
  __syncthreads();
  s = 0.f;
#pragma unroll
  for (int i = 0; i < kStreamWarps; ++i) s += red_s[i];

  float M = m, S = s;
  if (C > 1) {
    cluster_wait();
    if (tid < C) {                            // this slice's place in every CTA of the row
      const uint32_t at = cluster_map(smem_u32(&slices[rank]), (uint32_t)tid);
      st_cluster_f32(at, m);
      st_cluster_f32(at + 4, s);
    }
    cluster_arrive();
    cluster_wait();
    M = -INFINITY;
    for (unsigned i = 0; i < C; ++i) M = fmaxf(M, slices[i].m);
    const Exponent to{M, a.in.scale, a.scale_lo};
    S = 0.f;
    for (unsigned i = 0; i < C; ++i) S += slices[i].m > -INFINITY ? slices[i].s * to(slices[i].m) : slices[i].s;
  }
  const bool ok = M > -INFINITY && M < INFINITY && S > 0.f && S < INFINITY;
  if (!ok && tid == 0) raise_status(a.status, DELS_STATUS_NONFINITE);
  const Exponent to{M, a.in.scale, a.scale_lo};
  const float factor = !ok ? NAN : some ? to(m) / S : 0.f;
  const f32x2 factor2 = both2(factor);

  O* out = static_cast<O*>(a.out) + (long long)r * a.ld_out - row.sh;     // by position
  const int from = max(k0, row.sh);
  if constexpr (HOLD) {
    // fours that lie on a boundary of the output's
    __syncthreads();
    const int skew = (int)((reinterpret_cast<uintptr_t>(out + from) / sizeof(O)) & 3u), start = from - skew;
    const bool whole = ((start - k0) & 3) == 0;
    for (int k = start + tid * 4; k < k1; k += 4 * kStreamThreads) {
      if (k >= from && k + 4 <= k1) {
        float x[4];
        held_get4(held, k - k0, whole, x);
        split2(mul2(ex.two(pair2(x[0], x[1])), factor2), x[0], x[1]);
        split2(mul2(ex.two(pair2(x[2], x[3])), factor2), x[2], x[3]);
        put4(out + k, x);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (k + i >= from && k + i < k1) put1(out + k + i, ex(held_get(held, k + i - k0)) * factor);
      }
    }
  } else {
    each([&](float (&x)[8], int k) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int q = elem_pos<T, VEC>(k, i);
        if (q >= from && q < k1) put1(out + q, ex(x[i]) * factor);
      }
    });
  }
}

}  // namespace

cudaError_t launch_row_probs(const ProbsArgs& args, bool f32, bool fused, bool vec, cudaStream_t s) {
  const int sms = device_sm_count(), most = device_max_smem_optin() - 1024;
  if (sms <= 0 || most <= 0) return cudaErrorInvalidValue;
  ProbsArgs a = args;
  const int held = fused || f32 ? 4 : 2;
  // CTAs of a row: as few as leave five slices on an SM, so that one's loads run beside another's
  // stores, more where the rows are few
  const auto cols = [&](int c) { return (int)(((long long)a.in.V + 7 + c - 1) / c + 63) / 64 * 64; };
  int c = 1;
  while (c < kMaxCluster && ((long long)cols(c) * held > 40 * 1024 ||
                             ((long long)a.in.rows * c < 2 * sms && cols(2 * c) >= 2 * kStreamStep)))
    c *= 2;
  a.in.cluster = c;
  a.in.slice_cols = c == 1 ? (a.in.V + 7 + 7) / 8 * 8 : cols(c);
  const long long bytes = (long long)a.in.slice_cols * held;
  const bool hold = bytes <= most;
  return dispatch_rows(a.in, f32, fused, vec, [&](auto type, auto terms, auto v) {
    using T = typename decltype(type)::type;
    constexpr int F = decltype(terms)::value;
    constexpr bool VEC = decltype(v)::value;
    const auto k = a.out_f32 ? (hold ? k_row_probs<T, F, VEC, float, true> : k_row_probs<T, F, VEC, float, false>)
                             : (hold ? k_row_probs<T, F, VEC, __nv_bfloat16, true>
                                     : k_row_probs<T, F, VEC, __nv_bfloat16, false>);
    const size_t smem = hold ? (size_t)bytes : 0;
    const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(k), smem, true);
    if (e != cudaSuccess) return e;
    return launch_pdl_cluster(k, dim3((unsigned)a.in.rows * (unsigned)c), dim3(kStreamThreads), smem, s, c, a);
  });
}

}  // namespace dels
