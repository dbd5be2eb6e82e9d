// Products with 4-bit weights: the layout of the codes, and y = W x.
#include <algorithm>

#include <cuda_bf16.h>

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
    uint8_t* block = a.packed + tile * a.lay.tile_bytes + (long long)kb * a.lay.block_bytes;
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
// y = W x on the tensor cores' register path (mma.m16n8k16, bf16 in, float32 out).
//
// A code minus its zero point is a whole number of -15 .. 15, exact in bf16, so that the
// products with a bf16 feature are exact too; a group's sum is scaled in float32. Float32
// features are three bf16 terms by truncation, again exact. The codes of a word become an
// operand's registers by a mask each: the 4 bits over bf16's 0x4300 are 128 + c, minus
// 128 + z the weight.
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
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Weights of register q of a word: codes of nibbles q and q + 4, minus zero points; base: 128 + z twice.
__device__ __forceinline__ uint32_t weights_of(uint32_t word, int q, uint32_t base) {
  const uint32_t c = ((word >> (4 * q)) & 0x000F000Fu) | 0x43004300u;
  uint32_t r;
  asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(c), "r"(base));
  return r;
}

// 8 features of a row from column k on (0 past K), as TERMS bf16 terms.
template <int TERMS>
__device__ __forceinline__ void load_features(const W4Args& a, int b, int k, uint4 (&out)[TERMS]) {
  const int n = b < a.B ? min(8, a.K - k) : 0;
  if constexpr (TERMS == 1) {
    uint32_t h[8];
    const uint16_t* x = static_cast<const uint16_t*>(a.x) + b * a.ld_x + k;
    if (n == 8 && (reinterpret_cast<uintptr_t>(x) & 15u) == 0) {
      out[0] = __ldg(reinterpret_cast<const uint4*>(x));
      return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = i < n ? __ldg(x + i) : 0u;
    out[0] = make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
  } else {
    const float* x = static_cast<const float*>(a.x) + b * a.ld_x + k;
    float f[8];
    if (n == 8 && (reinterpret_cast<uintptr_t>(x) & 15u) == 0) {
      const float4 u = __ldg(reinterpret_cast<const float4*>(x)), v = __ldg(reinterpret_cast<const float4*>(x) + 1);
      f[0] = u.x; f[1] = u.y; f[2] = u.z; f[3] = u.w; f[4] = v.x; f[5] = v.y; f[6] = v.z; f[7] = v.w;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = i < n ? __ldg(x + i) : 0.f;
    }
    uint32_t t[TERMS][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float r = f[i];
#pragma unroll
      for (int j = 0; j < TERMS; ++j) {
        // truncated, 8 significant bits each: no term overflows, and three of them hold 24 bits.
        // Infinities and NaN (whose bits may all be in the lower half) stay in the first.
        const float h = __uint_as_float(__float_as_uint(r) & 0xFFFF0000u);
        const bool finite = fabsf(f[i]) < INFINITY;
        t[j][i] = finite ? __float_as_uint(h) >> 16 : j ? 0u : f[i] != f[i] ? 0x7FC0u : __float_as_uint(f[i]) >> 16;
        r = finite ? r - h : 0.f;
      }
    }
#pragma unroll
    for (int j = 0; j < TERMS; ++j)
      out[j] = make_uint4(t[j][0] | t[j][1] << 16, t[j][2] | t[j][3] << 16, t[j][4] | t[j][5] << 16,
                          t[j][6] | t[j][7] << 16);
  }
}

constexpr int kW4Pitch = 36;             // floats of a request's 32 rows in the sums' tile: conflict-free both ways
constexpr int kW4Producers = 96;         // threads that stage features where those do not stay

template <int NT>
constexpr int kW4Warps = NT <= 2 ? 16 : 8;      // warps that multiply, at most

// Fragments of a block's features: [4 units][TERMS][NT][32 lanes] of 16 bytes; lane 4 g + t
// has request 8 j + g, inputs 8 t .. 8 t + 7 of the unit's 32.
template <int NT, int TERMS>
__device__ __forceinline__ void stage_features(const W4Args& a, int b0, int unit, int j, uint4* dst) {
  const int lane = threadIdx.x & 31;
  uint4 f[TERMS];
  load_features<TERMS>(a, b0 + 8 * j + (lane >> 2), unit * kW4Unit + 8 * (lane & 3), f);
#pragma unroll
  for (int t = 0; t < TERMS; ++t) dst[(t * NT + j) * 32 + lane] = f[t];
}

template <int NT, int TERMS, bool ZEROS>
__global__ void __launch_bounds__(kW4Warps<NT> * 32 + 32 + kW4Producers, 1) k_w4_project(const W4Args a, const W4Plan p) {
  extern __shared__ __align__(128) uint8_t smem[];
  constexpr int N = NT * 8;
  constexpr int kXBlock = 4 * TERMS * NT * 512;
  __shared__ uint64_t full[kW4MaxStages], empty[kW4MaxStages];
  __shared__ int abort_flag;
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
  __syncthreads();
  pdl_wait();
  if (threadIdx.x == 0) pdl_trigger();
  uint64_t deadline;                       // of the waits of an item
  const int steps = (a.lay.blocks + p.wk - 1) / p.wk;
  bool dead = false;                       // a wait ran out: the rest runs through without waiting

  if (warp > warps) {
    // ---- features of every stage
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
          stage_features<NT, TERMS>(a, b0, step * p.wk * 4 + u, j, dst + u * (TERMS * NT * 32));
        }
        mbar_arrive(&full[st]);
        if (++st == p.stages) st = 0, ph ^= 1;
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
          const long long from = (long long)step * p.wk * a.lay.block_bytes;
          const long long to = min(a.lay.tile_bytes, from + (long long)p.wk * a.lay.block_bytes);
          const uint32_t bytes = (uint32_t)(to - from);
          mbar_arrive_expect_tx(&full[st], bytes * live);
          for (int r = 0; r < live; ++r)
            bulk_load(ring + (size_t)st * p.stage_bytes + r * p.wk * a.lay.block_bytes,
                      a.packed + (tile0 + r) * a.lay.tile_bytes + from, bytes, &full[st]);
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
      for (int i = warp; i < a.lay.units * NT; i += warps) {
        const int u = i / NT, j = i - u * NT;
        stage_features<NT, TERMS>(a, b0, u, j, reinterpret_cast<uint4*>(xres) + u * (TERMS * NT * 32));
      }
      asm volatile("bar.sync 1, %0;" ::"r"(warps * 32) : "memory");
    }
    const int gunits = a.group / kW4Unit;
    int st = 0, ph = 0;
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
          const uint8_t* block = ring + (size_t)st * p.stage_bytes + (size_t)(wr * p.wk + wk) * a.lay.block_bytes;
          const int units = min(4, a.lay.units - 4 * kb);
          const uint4* x = p.resident ? reinterpret_cast<const uint4*>(xres) + kb * (kXBlock / 16)
                                      : reinterpret_cast<const uint4*>(ring + (size_t)st * p.stage_bytes + p.x_off) +
                                            wk * (kXBlock / 16);
          const uint8_t* scales = block + units * 512;
          const uint8_t* zeros = scales + (units + gunits - 1) / gunits * 64;
          uint32_t base[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) base[i] = 0x43084308u;
          for (int u = 0; u < units; ++u) {
            const int grp = u / gunits;
            if (ZEROS && u == grp * gunits) {
              const uint32_t z = reinterpret_cast<const uint16_t*>(zeros + grp * 16)[g];
#pragma unroll
              for (int i = 0; i < 4; ++i) base[i] = 0x43004300u + ((z >> (4 * i)) & 15u) * 0x00010001u;
            }
            const uint4 w4 = reinterpret_cast<const uint4*>(block)[u * 32 + lane];
            const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
            uint32_t m[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int q = 0; q < 4; ++q) m[i][q] = weights_of(w[i], q, base[(i >> 1) * 2 + (q & 1)]);
#pragma unroll
            for (int term = 0; term < TERMS; ++term)
#pragma unroll
              for (int j = 0; j < NT; ++j) {
                const uint4 f = x[((u * TERMS + term) * NT + j) * 32 + lane];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                  mma_bf16(acc[h][j], m[2 * h], f.x, f.y);
                  mma_bf16(acc[h][j], m[2 * h + 1], f.z, f.w);
                }
              }
            if (u + 1 == units || u + 1 == (grp + 1) * gunits) {
              const uint2 s = reinterpret_cast<const uint2*>(scales + grp * 64)[g];
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
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&empty[st]);
        if (++st == p.stages) st = 0, ph ^= 1;
      }
      // ---- the parts' sums, along the vocabulary
      float* part = sums + (size_t)warp * N * kW4Pitch;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            part[(8 * j + 2 * t + (i & 1)) * kW4Pitch + h * 16 + (i >> 1) * 8 + g] = tot[h][j][i];
      asm volatile("bar.sync 1, %0;" ::"r"(warps * 32) : "memory");
      const int nb = min(N, a.B - b0);
      for (int i = warp; i < nb * p.wr; i += warps) {
        const int b = i / p.wr, r = i - b * p.wr;
        const long long v = (tile0 + r) * kW4Rows + lane;
        const float* src = sums + ((size_t)r * p.wk * N + b) * kW4Pitch + lane;
        float y = src[0];
        for (int k = 1; k < p.wk; ++k) y += src[(size_t)k * N * kW4Pitch];
        if (v < a.V) {
          const long long at = (long long)(b0 + b) * a.ld_out + v;
          if (a.out_f32) static_cast<float*>(a.out)[at] = y;
          else static_cast<__nv_bfloat16*>(a.out)[at] = __float2bfloat16_rn(y);
        }
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
bool plan_w4(const W4Args& a, int sms, int smem, W4Plan* best) {
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
      p.resident = stay <= 96 * 1024 && smem - sums - stay >= 3ll * codes;
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

template <int NT, int TERMS>
cudaError_t launch_nt(const W4Args& a, cudaStream_t s) {
  const int sms = device_sm_count(), smem = device_max_smem_optin() - 1024;
  W4Plan p;
  if (sms <= 0 || !plan_w4<NT, TERMS>(a, sms, smem, &p)) return cudaErrorInvalidValue;
  const auto k = a.zeros ? k_w4_project<NT, TERMS, true> : k_w4_project<NT, TERMS, false>;
  const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(k), p.smem);
  if (e != cudaSuccess) return e;
  const int btiles = (a.B + NT * 8 - 1) / (NT * 8), ctas = std::max(1, sms / btiles);
  const int threads = p.wr * p.wk * 32 + 32 + (p.resident ? 0 : kW4Producers);
  return launch_pdl(k, dim3((unsigned)std::min(p.items, ctas), (unsigned)btiles), dim3(threads), (size_t)p.smem, s, a, p);
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
