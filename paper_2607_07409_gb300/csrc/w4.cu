// Products with 4-bit weights: the layout of the codes, and y = W x.
#include <algorithm>
#include <type_traits>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "dels_device.cuh"

namespace dels {
namespace {

constexpr int kPackThreads = 128;
constexpr int kW4MaxStages = 16;

// How a product runs: warps of 32 rows and of a block's inputs in a CTA, its ring and features.
struct W4Plan {
  int wr, wk;
  int items;           // of 32 wr rows
  int stages, stage_bytes;
  int resident;        // the features stay in shared memory
  int x_off;           // of a stage's features, where they do not
  int smem;
};

// A CTA lays out blocks of 128 inputs of 32 rows, a warp one unit of 32 inputs.
__global__ void __launch_bounds__(kPackThreads) k_w4_pack(const W4PackArgs a) {
  pdl_wait();
  if (threadIdx.x == 0) pdl_trigger();
  const int lane = threadIdx.x & 31, u = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const long long tile = blockIdx.x;
  const int groups = (a.K + a.group - 1) / a.group;
  bool bad = false;
  for (int kb = blockIdx.y; kb < a.lay.blocks; kb += gridDim.y) {
    const int units = min(4, a.lay.units - 4 * kb), ng = (units * kW4Unit + a.group - 1) / a.group;
    uint8_t* block = a.packed + w4_block_at(a.lay, tile, kb);
    if (u < units) {
      uint32_t w[4];
      for (int j = 0; j < 4; ++j) {              // word 2 (rows' half) + k-step
        uint32_t x = 0;
        for (int q = 0; q < 8; ++q) {
          const long long v = tile * kW4Rows + (j >> 1) * 16 + (q & 1) * 8 + g;
          const int k = kb * kW4Block + u * kW4Unit + 8 * t + 4 * (j & 1) + ((q >> 1) & 1) * 2 + (q >> 2);
          uint32_t c = 0;
          if (v < a.V && k < a.K) c = a.codes[v * a.K + k];
          bad |= c > 15;
          x |= (c & 15u) << (4 * q);
        }
        w[j] = x;
      }
      reinterpret_cast<uint4*>(block)[u * 32 + lane] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    if (u < ng) {
      const int grp = kb * (kW4Block / a.group) + u;
      const long long v = tile * kW4Rows + t * 8 + g;      // rows g + 8 t
      uint16_t* sc = reinterpret_cast<uint16_t*>(block + units * 512 + u * 64);
      sc[g * 4 + t] = v < a.V ? a.scales[v * groups + grp] : 0;
      if (a.zeros) {
        uint32_t z = v < a.V ? a.zeros[v * groups + grp] : 0;
        bad |= z > 15;
        z = (z & 15u) << (4 * t);
        z |= __shfl_xor_sync(0xFFFFFFFFu, z, 1);
        z |= __shfl_xor_sync(0xFFFFFFFFu, z, 2);
        if (t == 0) reinterpret_cast<uint16_t*>(block + units * 512 + ng * 64 + u * 16)[g] = (uint16_t)z;
      }
    }
  }
  if (bad) raise_status(a.status, DELS_STATUS_BAD_VALUE);
}

// ---------------------------------------------------------------------------
// y = W x on the tensor cores' register path (mma.m16n8k16, float32 sums).
//
// A code minus its zero point is a whole number of -15 .. 15, and a bf16 feature has 8
// significant bits: the products are exact, and a group's sum is scaled in float32.
// * HALF, few requests: fp16 operands. Its 10 bits of mantissa hold a code where it lies in
//   a byte, low or high, so that a word of 8 codes takes 4 masks and one shift (a bf16 operand 4
//   and 3, and these are what bounds few requests: the ALU pipe issues every other cycle).
//   (w & 0x000F000F) | 0x6400 is 1024 + c and the high ones' 1024 + 16 c; an fma takes the zero
//   point off. A request's features are scaled by a power of two to at most 2^15: fp16 then
//   holds bf16 features exactly down to 2^-32 of the request's largest, and what is
//   smaller to 2^-40 of that. Float32 features are three fp16 terms, to the same 2^-40.
// * else bf16 operands, the features as they are or in three bf16 terms by truncation, exactly:
//   (w & 0x000F000F) | 0x4300 is 128 + c, minus 128 + z the weight.
//
// The codes stream through a ring in shared memory (bulk copies by one thread, a stage at a
// time), so that a warp's arithmetic never waits for memory itself; the features, a few KB,
// stay there for the whole launch where they fit, else a stage holds its inputs' part. A warp
// takes 32 rows; wk of them share a stage's rows, a block of 128 inputs each, and their sums
// meet in shared memory, where the epilogue reads them along the vocabulary.
// ---------------------------------------------------------------------------
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
               "l"(src), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}
template <bool HALF>
__device__ __forceinline__ void mma16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (HALF)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Zero points of rows g, g + 8, g + 16, g + 24 as weights_of() takes them; z: four nibbles.
template <bool HALF>
struct ZeroPoints {
  uint32_t low[4], high[HALF ? 4 : 1];
  __device__ __forceinline__ void set(uint32_t z) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t d = ((z >> (4 * i)) & 15u) * 0x00010001u;
      if constexpr (HALF) {
        low[i] = 0x64006400u + d;                // 1024 + z
        high[i] = 0xD400D400u + (d << 4);        // -(64 + z)
      } else {
        low[i] = 0x43004300u + d;                // 128 + z
      }
    }
  }
};
// (w & mask) | base in one instruction: given as two constants the compiler made two of it.
__device__ __forceinline__ uint32_t pick(uint32_t w, uint32_t mask, uint32_t base) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(w), "r"(mask), "r"(base));
  return r;
}
// The four registers of a word's weights: codes of nibbles q and q + 4, rows `half` and half + 1 of the lane's.
// base: 1024 (bf16: 128) twice, in a register.
template <bool HALF>
__device__ __forceinline__ void weights_of(uint32_t word, uint32_t base, const ZeroPoints<HALF>& z, int half,
                                           uint32_t (&m)[4]) {
  if constexpr (HALF) {
    const uint32_t next = word >> 8;
    const uint32_t c[4] = {pick(word, 0x000F000Fu, base), pick(word, 0x00F000F0u, base), pick(next, 0x000F000Fu, base),
                           pick(next, 0x00F000F0u, base)};
#pragma unroll
    for (int q = 0; q < 4; q += 2) {
      asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(m[q]) : "r"(c[q]), "r"(z.low[half]));
      asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(m[q + 1]) : "r"(c[q + 1]), "r"(0x2C002C00u), "r"(z.high[half + 1]));
    }
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint32_t c = pick(word >> (4 * q), 0x000F000Fu, base);
      asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(m[q]) : "r"(c), "r"(z.low[half + (q & 1)]));
    }
  }
}

// 8 features of a row from column k on (0 past K, and past the last row).
__device__ __forceinline__ void load_features(const W4Args& a, int b, int k, float (&f)[8]) {
  const int n = b < a.B ? min(8, a.K - k) : 0;
  if (a.x_f32) {
    const float* x = static_cast<const float*>(a.x) + b * a.ld_x + k;
    if (n == 8 && (reinterpret_cast<uintptr_t>(x) & 15u) == 0) {
      const float4 u = __ldg(reinterpret_cast<const float4*>(x)), v = __ldg(reinterpret_cast<const float4*>(x) + 1);
      f[0] = u.x; f[1] = u.y; f[2] = u.z; f[3] = u.w; f[4] = v.x; f[5] = v.y; f[6] = v.z; f[7] = v.w;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = i < n ? __ldg(x + i) : 0.f;
    }
  } else {
    const uint16_t* x = static_cast<const uint16_t*>(a.x) + b * a.ld_x + k;
    if (n == 8 && (reinterpret_cast<uintptr_t>(x) & 15u) == 0) {
      const uint4 u = __ldg(reinterpret_cast<const uint4*>(x));
      f[0] = bf16lo(u.x); f[1] = bf16hi(u.x); f[2] = bf16lo(u.y); f[3] = bf16hi(u.y);
      f[4] = bf16lo(u.z); f[5] = bf16hi(u.z); f[6] = bf16lo(u.w); f[7] = bf16hi(u.w);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = i < n ? bf16_to_f(__ldg(x + i)) : 0.f;
    }
  }
}

constexpr int kW4Pitch = 36;             // floats of a request's 32 rows in the sums' tile: conflict-free both ways
constexpr int kW4Producers = 96;         // threads that stage features where those do not stay

template <int NT>
constexpr int kW4Warps = NT <= 2 ? 16 : 8;      // warps that multiply, at most

// A request's power of two: its features' largest, of these bits, comes to 2^14 .. 2^15.
// Where there is an infinity or NaN its outputs are those of these alone: the others count as 0.
constexpr int kNotFinite = 1 << 20;
__device__ __forceinline__ int feature_shift(uint32_t bits) {
  if (bits >= 0x7F800000u) return kNotFinite;
  return bits ? 14 - ilogbf(__uint_as_float(bits)) : 0;
}
__device__ __forceinline__ float pow2i(int e) { return __int_as_float((e + 127) << 23); }    // -126 .. 127

// Fragments of a unit's features, request 8 j + g and inputs 8 t .. 8 t + 7 of its 32 in lane
// 4 g + t: [TERMS][NT][32 lanes] of 16 bytes. sh: HALF, the request's power.
template <int NT, int TERMS, bool HALF>
__device__ __forceinline__ void put_features(const float (&f)[8], int j, int sh, uint4* dst) {
  uint32_t t[TERMS][8];
  if constexpr (HALF) {
    // (in two factors: the power itself may be past float32's range)
    const float s0 = sh == kNotFinite ? 1.f : pow2i(sh / 2), s1 = sh == kNotFinite ? 1.f : pow2i(sh - sh / 2);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float r = sh != kNotFinite ? f[i] * s0 * s1 : fabsf(f[i]) < INFINITY ? 0.f : f[i];
#pragma unroll
      for (int k = 0; k < TERMS; ++k) {
        const __half h = __float2half_rn(r);
        t[k][i] = __half_as_ushort(h);
        r = sh != kNotFinite ? r - __half2float(h) : 0.f;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float r = f[i];
      const bool finite = fabsf(f[i]) < INFINITY;
#pragma unroll
      for (int k = 0; k < TERMS; ++k) {
        // truncated, 8 significant bits each: no term overflows, and three of them hold 24 bits.
        // Infinities and NaN (whose bits may all be in the lower half) stay in the first.
        const float h = __uint_as_float(__float_as_uint(r) & 0xFFFF0000u);
        t[k][i] = finite ? __float_as_uint(h) >> 16 : k ? 0u : f[i] != f[i] ? 0x7FC0u : __float_as_uint(f[i]) >> 16;
        r = finite ? r - h : 0.f;
      }
    }
  }
#pragma unroll
  for (int k = 0; k < TERMS; ++k)
    dst[(k * NT + j) * 32 + (threadIdx.x & 31)] =
        make_uint4(t[k][0] | t[k][1] << 16, t[k][2] | t[k][3] << 16, t[k][4] | t[k][5] << 16, t[k][6] | t[k][7] << 16);
}
__device__ __forceinline__ void load_unit(const W4Args& a, int b0, int unit, int j, float (&f)[8]) {
  const int lane = threadIdx.x & 31;
  load_features(a, b0 + 8 * j + (lane >> 2), unit * kW4Unit + 8 * (lane & 3), f);
}

// One warp's unit: 32 rows, 32 inputs.
template <int NT, int TERMS, bool HALF>
__device__ __forceinline__ void multiply_unit(const uint4 w4, uint32_t base, const ZeroPoints<HALF>& z, const uint4* x,
                                              float (&acc)[2][NT][4]) {
  uint32_t m[4][4];
  weights_of<HALF>(w4.x, base, z, 0, m[0]);
  weights_of<HALF>(w4.y, base, z, 0, m[1]);
  weights_of<HALF>(w4.z, base, z, 2, m[2]);
  weights_of<HALF>(w4.w, base, z, 2, m[3]);
  // (a sum's two products stand four apart: one waits for the other)
  constexpr int J = NT > 1 ? 2 : 1;
#pragma unroll
  for (int term = 0; term < TERMS; ++term)
#pragma unroll
    for (int j0 = 0; j0 < NT; j0 += J) {
      uint4 f[J];
#pragma unroll
      for (int j = 0; j < J; ++j) f[j] = x[(term * NT + j0 + j) * 32];
#pragma unroll
      for (int j = 0; j < J; ++j) {
        mma16<HALF>(acc[0][j0 + j], m[0], f[j].x, f[j].y);
        mma16<HALF>(acc[1][j0 + j], m[2], f[j].x, f[j].y);
      }
#pragma unroll
      for (int j = 0; j < J; ++j) {
        mma16<HALF>(acc[0][j0 + j], m[1], f[j].z, f[j].w);
        mma16<HALF>(acc[1][j0 + j], m[3], f[j].z, f[j].w);
      }
    }
}
template <int NT>
__device__ __forceinline__ void scale_group(const uint2 s, float (&acc)[2][NT][4], float (&tot)[2][NT][4]) {
  const float sc[4] = {bf16lo(s.x), bf16hi(s.x), bf16lo(s.y), bf16hi(s.y)};
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        tot[h][j][i] = fmaf(sc[2 * h + (i >> 1)], acc[h][j][i], tot[h][j][i]);
        acc[h][j][i] = 0.f;
      }
}

// n <= 4 outputs from element `at` on.
__device__ __forceinline__ void store_outputs(const W4Args& a, long long at, const float4& y, int n) {
  const float f[4] = {y.x, y.y, y.z, y.w};
  if (a.out_f32) {
    float* out = static_cast<float*>(a.out) + at;
    if (n == 4 && (reinterpret_cast<uintptr_t>(out) & 15u) == 0) {
      *reinterpret_cast<float4*>(out) = y;
      return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) out[i] = f[i];
  } else {
    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out) + at;
    const __nv_bfloat162 lo = __floats2bfloat162_rn(f[0], f[1]), hi = __floats2bfloat162_rn(f[2], f[3]);
    if (n == 4 && (reinterpret_cast<uintptr_t>(out) & 7u) == 0) {
      uint2 u;
      u.x = *reinterpret_cast<const uint32_t*>(&lo);
      u.y = *reinterpret_cast<const uint32_t*>(&hi);
      *reinterpret_cast<uint2*>(out) = u;
      return;
    }
    const __nv_bfloat16 h[4] = {lo.x, lo.y, hi.x, hi.y};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) out[i] = h[i];
  }
}

template <int NT, int TERMS, bool HALF>
__global__ void __launch_bounds__(kW4Warps<NT> * 32 + 32 + (HALF ? 0 : kW4Producers), 1)
    k_w4_project(const W4Args a, const W4Plan p) {
  extern __shared__ __align__(128) uint8_t smem[];
  constexpr int N = NT * 8;
  constexpr int kXBlock = 4 * TERMS * NT * 512;
  __shared__ uint64_t full[kW4MaxStages], empty[kW4MaxStages];
  __shared__ int abort_flag;
  __shared__ uint32_t largest[N];          // HALF: bits of the requests' largest features
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = p.wr * p.wk;
  const int b0 = blockIdx.y * N;
  uint8_t* ring = smem;                                                     // stages of p.stage_bytes
  uint8_t* xres = smem + (size_t)p.stages * p.stage_bytes;                  // features that stay
  float* sums = reinterpret_cast<float*>(xres + (p.resident ? (size_t)a.lay.blocks * kXBlock : 0));
  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int i = 0; i < p.stages; ++i) {
      mbar_init(&full[i], p.resident ? 1 : 1 + kW4Producers);
      mbar_init(&empty[i], warps);
    }
    fence_mbarrier_init();
  }
  if (HALF && threadIdx.x < N) largest[threadIdx.x] = 0;
  __syncthreads();
  pdl_wait();
  if (threadIdx.x == 0) pdl_trigger();
  uint64_t deadline;                       // of the waits of an item
  const int steps = (a.lay.blocks + p.wk - 1) / p.wk;
  bool dead = false;                       // a wait ran out: the rest runs through without waiting

  if (warp > warps) {
    // ---- features of every stage
    if constexpr (!HALF) {
      const int t0 = warp - warps - 1;
      int st = 0, ph = 0;
      for (int it = blockIdx.x; it < p.items; it += gridDim.x) {
        deadline = globaltimer_ns() + kWaitBudgetNs;
        for (int step = 0; step < steps; ++step) {
          if (!dead) dead = !mbar_wait(&empty[st], ph ^ 1, deadline, &abort_flag);
          uint4* dst = reinterpret_cast<uint4*>(ring + (size_t)st * p.stage_bytes + p.x_off);
          const int units = min(4 * p.wk, a.lay.units - step * p.wk * 4);
          for (int i = t0; i < units * NT; i += kW4Producers / 32) {
            const int u = i / NT, j = i - u * NT;
            float f[8];
            load_unit(a, b0, step * p.wk * 4 + u, j, f);
            put_features<NT, TERMS, HALF>(f, j, 0, dst + u * (TERMS * NT * 32));
          }
          mbar_arrive(&full[st]);
          if (++st == p.stages) st = 0, ph ^= 1;
        }
      }
    }
  } else if (warp == warps) {
    // ---- codes, scales and zero points
    if (lane == 0) {
      fence_proxy_async_global();
      int st = 0, ph = 0;
      long long issued = 0;
      for (int it = blockIdx.x; it < p.items; it += gridDim.x) {
        deadline = globaltimer_ns() + kWaitBudgetNs;
        const long long tile0 = (long long)it * p.wr;
        const int live = (int)min((long long)p.wr, a.lay.tiles - tile0);
        for (int step = 0; step < steps; ++step) {
          if (!dead) dead = !mbar_wait(&empty[st], ph ^ 1, deadline, &abort_flag);
          if (dead) break;
          // an input block of the live tiles is one piece
          const int kb0 = step * p.wk, kb1 = min(a.lay.blocks, kb0 + p.wk);
          const uint32_t whole = (uint32_t)live * a.lay.block_bytes, last = (uint32_t)live * a.lay.last_bytes;
          mbar_arrive_expect_tx(&full[st], kb1 < a.lay.blocks ? (kb1 - kb0) * whole : (kb1 - kb0 - 1) * whole + last);
          for (int kb = kb0; kb < kb1; ++kb)
            bulk_load(ring + (size_t)st * p.stage_bytes + (kb - kb0) * p.wr * a.lay.block_bytes,
                      a.packed + w4_block_at(a.lay, tile0, kb), kb + 1 < a.lay.blocks ? whole : last, &full[st]);
          ++issued;
          if (++st == p.stages) st = 0, ph ^= 1;
        }
        if (dead) break;
      }
      // a CTA that gives up has its copies in flight land first
      if (dead) {
        const uint64_t limit = globaltimer_ns() + kWaitBudgetNs / 4;
        for (long long i = max(0ll, issued - p.stages); i < issued; ++i)
          while (!mbar_try_wait(&full[i % p.stages], (int)((i / p.stages) & 1)) && globaltimer_ns() < limit) {}
      }
    }
  } else {
    // ---- products
    const int wr = warp / p.wk, wk = warp - wr * p.wk, g = lane >> 2, t = lane & 3;
    if (p.resident) {
      // A warp's units of features, the first ones' kept from the search for the requests' largest.
      constexpr int kKept = 2;
      const int tasks = a.lay.units * NT;
      float f[kKept][8];
#pragma unroll
      for (int i = 0; i < kKept; ++i) {
        const int task = warp + i * warps;
        if (task < tasks) load_unit(a, b0, task / NT, task % NT, f[i]);
      }
      if constexpr (HALF) {
        const auto look = [&](const float (&x)[8], int j) {
          uint32_t m = 0;
#pragma unroll
          for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(fabsf(x[i])));      // NaN above infinity
          m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
          m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
          if (t == 0) atomicMax(&largest[8 * j + g], m);
        };
        for (int task = warp + kKept * warps; task < tasks; task += warps) {
          float x[8];
          load_unit(a, b0, task / NT, task % NT, x);
          look(x, task % NT);
        }
#pragma unroll
        for (int i = 0; i < kKept; ++i)
          if (warp + i * warps < tasks) look(f[i], (warp + i * warps) % NT);
        asm volatile("bar.sync 1, %0;" ::"r"(warps * 32) : "memory");
      }
      const auto place = [&](const float (&x)[8], int task) {
        const int j = task % NT;
        put_features<NT, TERMS, HALF>(x, j, HALF ? feature_shift(largest[8 * j + g]) : 0,
                                      reinterpret_cast<uint4*>(xres) + (task / NT) * (TERMS * NT * 32));
      };
#pragma unroll
      for (int i = 0; i < kKept; ++i)
        if (warp + i * warps < tasks) place(f[i], warp + i * warps);
      for (int task = warp + kKept * warps; task < tasks; task += warps) {
        float x[8];
        load_unit(a, b0, task / NT, task % NT, x);
        place(x, task);
      }
      asm volatile("bar.sync 1, %0;" ::"r"(warps * 32) : "memory");
    }
    const int gunits = a.group / kW4Unit, glog = gunits == 1 ? 0 : gunits == 2 ? 1 : 2;
    const int wr_log = 31 - __clz(p.wr);
    int st = 0, ph = 0;
    ZeroPoints<HALF> z;
    z.set(0x8888u);
    uint32_t base = HALF ? 0x64006400u : 0x43004300u;
    asm("" : "+r"(base));                  // (a register, not a constant)
    for (int it = blockIdx.x; it < p.items; it += gridDim.x) {
      deadline = globaltimer_ns() + kWaitBudgetNs;
      const long long tile0 = (long long)it * p.wr;
      float tot[2][NT][4], acc[2][NT][4];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) tot[h][j][i] = acc[h][j][i] = 0.f;
      for (int step = 0; step < steps; ++step) {
        if (!dead) dead = !mbar_wait(&full[st], ph, deadline, &abort_flag);
        const int kb = step * p.wk + wk;
        if (kb < a.lay.blocks && tile0 + wr < a.lay.tiles) {
          const uint8_t* block = ring + (size_t)st * p.stage_bytes + (size_t)wk * p.wr * a.lay.block_bytes +
                                 (size_t)wr * (kb + 1 < a.lay.blocks ? a.lay.block_bytes : a.lay.last_bytes);
          const uint4* codes = reinterpret_cast<const uint4*>(block) + lane;
          const int units = min(4, a.lay.units - 4 * kb);
          const uint4* x = (p.resident ? reinterpret_cast<const uint4*>(xres) + kb * (kXBlock / 16)
                                       : reinterpret_cast<const uint4*>(ring + (size_t)st * p.stage_bytes + p.x_off) +
                                             wk * (kXBlock / 16)) + lane;
          const uint8_t* scales = block + units * 512 + g * 8;
          const uint8_t* zeros = block + units * 512 + ((units + gunits - 1) >> glog) * 64 + g * 2;
          const auto unit = [&](int u, int grp, bool first, bool last) {
            if (first && a.zeros) z.set(*reinterpret_cast<const uint16_t*>(zeros + grp * 16));
            multiply_unit<NT, TERMS, HALF>(codes[u * 32], base, z, x + u * (TERMS * NT * 32), acc);
            if (last) scale_group<NT>(*reinterpret_cast<const uint2*>(scales + grp * 64), acc, tot);
          };
          // (a whole block straight on for each group size: with tests between its units 85 instructions a unit)
          const auto whole = [&](auto group_units) {
            constexpr int G = decltype(group_units)::value;
#pragma unroll
            for (int u = 0; u < 4; ++u) unit(u, u / G, u % G == 0, u % G == G - 1);
          };
          if (units == 4) {
            if (glog == 0) whole(std::integral_constant<int, 1>{});
            else if (glog == 1) whole(std::integral_constant<int, 2>{});
            else whole(std::integral_constant<int, 4>{});
          } else {
#pragma unroll 1
            for (int u = 0; u < units; ++u)
              unit(u, u >> glog, (u & (gunits - 1)) == 0, u + 1 == units || ((u + 1) & (gunits - 1)) == 0);
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&empty[st]);
        if (++st == p.stages) st = 0, ph ^= 1;
      }
      // ---- the parts' sums, along the vocabulary: 8 lanes have 32 rows of a request
      float* part = sums + (size_t)warp * N * kW4Pitch;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            part[(8 * j + 2 * t + (i & 1)) * kW4Pitch + h * 16 + (i >> 1) * 8 + g] = tot[h][j][i];
      asm volatile("bar.sync 1, %0;" ::"r"(warps * 32) : "memory");
      const int lines = min(N, a.B - b0) << wr_log;
      for (int i = warp * 4 + (lane >> 3); i < lines; i += warps * 4) {
        const int b = i >> wr_log, r = i & (p.wr - 1);
        const float* src = sums + ((size_t)r * p.wk * N + b) * kW4Pitch + (lane & 7) * 4;
        float4 y = *reinterpret_cast<const float4*>(src);
        for (int k = 1; k < p.wk; ++k) {
          const float4 w = *reinterpret_cast<const float4*>(src + (size_t)k * N * kW4Pitch);
          y.x += w.x; y.y += w.y; y.z += w.z; y.w += w.w;
        }
        if constexpr (HALF) {
          const int up = feature_shift(largest[b]), sh = up == kNotFinite ? 0 : -up;
          const float s0 = pow2i(sh / 2), s1 = pow2i(sh - sh / 2);
          y.x = y.x * s0 * s1; y.y = y.y * s0 * s1; y.z = y.z * s0 * s1; y.w = y.w * s0 * s1;
        }
        const long long v = (tile0 + r) * kW4Rows + (lane & 7) * 4;
        store_outputs(a, (long long)(b0 + b) * a.ld_out + v, y, (int)min(4ll, (long long)a.V - v));
      }
      asm volatile("bar.sync 1, %0;" ::"r"(warps * 32) : "memory");
    }
    if (dead && lane == 0) raise_status(a.status, DELS_STATUS_TIMEOUT);
  }
}

// Warps of a CTA, where the features lie, stages of the ring. The cost of an item of wr x 32
// rows, in units of a warp's block of 128 inputs: its steps, what the memory takes for its
// blocks beside the other SMs, and a start.
template <int NT, int TERMS>
bool plan_w4(const W4Args& a, int sms, int smem, bool resident, W4Plan* best) {
  const int xblock = 4 * TERMS * NT * 512, btiles = (a.B + NT * 8 - 1) / (NT * 8);
  const int ctas = std::max(1, sms / btiles);
  double least = 1e30;
  for (int wk = 1; wk <= kW4Warps<NT>; wk *= 2) {
    if (wk > 1 && wk >= 2 * a.lay.blocks) break;
    for (int wr = 1; wr * wk <= kW4Warps<NT>; wr *= 2) {
      W4Plan p{};
      p.wr = wr;
      p.wk = wk;
      const long long items = (a.lay.tiles + wr - 1) / wr;
      if (items > (1 << 30)) continue;
      p.items = (int)items;
      const int sums = wr * wk * NT * 8 * kW4Pitch * 4, codes = wr * wk * a.lay.block_bytes;
      const long long stay = (long long)a.lay.blocks * xblock;
      p.resident = resident;
      if (resident && smem - sums - stay < 3ll * codes) continue;
      p.x_off = codes;
      p.stage_bytes = codes + (p.resident ? 0 : wk * xblock);
      const long long room = smem - sums - (p.resident ? stay : 0);
      p.stages = (int)std::min<long long>(kW4MaxStages, room / p.stage_bytes);
      if (p.stages < 2) continue;
      p.smem = (int)((long long)p.stages * p.stage_bytes + (p.resident ? stay : 0) + sums);
      const long long rounds = (items + ctas - 1) / ctas;
      const double steps = (a.lay.blocks + wk - 1) / wk;
      const double step = std::max(1.0 + 0.3 * NT * TERMS, wr * wk * 0.15 * std::min<double>(1.0, (double)items / ctas));
      const double cost = rounds * (steps * step + 3.0);
      if (cost < least) {
        least = cost;
        *best = p;
      }
    }
  }
  return least < 1e30;
}

template <int NT, int TERMS, bool HALF>
cudaError_t launch_plan(const W4Args& a, const W4Plan& p, int sms, cudaStream_t s) {
  const auto k = k_w4_project<NT, TERMS, HALF>;
  const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(k), p.smem);
  if (e != cudaSuccess) return e;
  const int btiles = (a.B + NT * 8 - 1) / (NT * 8), ctas = std::max(1, sms / btiles);
  const int threads = p.wr * p.wk * 32 + 32 + (p.resident ? 0 : kW4Producers);
  return launch_pdl(k, dim3((unsigned)std::min(p.items, ctas), (unsigned)btiles), dim3(threads), (size_t)p.smem, s, a, p);
}

template <int NT, int TERMS>
cudaError_t launch_nt(const W4Args& a, cudaStream_t s) {
  const int sms = device_sm_count(), smem = device_max_smem_optin() - 1024;
  W4Plan p;
  if (sms <= 0) return cudaErrorInvalidValue;
  const bool stays = plan_w4<NT, TERMS>(a, sms, smem, true, &p);
  if (!stays && !plan_w4<NT, TERMS>(a, sms, smem, false, &p)) return cudaErrorInvalidValue;
  if constexpr (NT <= 2) {
    if (stays) return launch_plan<NT, TERMS, true>(a, p, sms, s);
  }
  return launch_plan<NT, TERMS, false>(a, p, sms, s);
}

}  // namespace

cudaError_t launch_w4_pack(const W4PackArgs& a, cudaStream_t s) {
  const dim3 grid((unsigned)a.lay.tiles, (unsigned)(a.lay.blocks < 64 ? a.lay.blocks : 64));
  return launch_pdl(k_w4_pack, grid, dim3(kPackThreads), 0, s, a);
}

cudaError_t launch_w4_project(const W4Args& a, cudaStream_t s) {
  if (a.x_f32) {
    if (a.B <= 8) return launch_nt<1, 3>(a, s);
    if (a.B <= 16) return launch_nt<2, 3>(a, s);
    return a.B <= 32 ? launch_nt<4, 3>(a, s) : launch_nt<8, 3>(a, s);
  }
  if (a.B <= 8) return launch_nt<1, 1>(a, s);
  if (a.B <= 16) return launch_nt<2, 1>(a, s);
  return a.B <= 32 ? launch_nt<4, 1>(a, s) : launch_nt<8, 1>(a, s);
}

}  // namespace dels
