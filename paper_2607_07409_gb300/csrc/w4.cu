// Products with 4-bit weights: the layout of the codes, and y = W x.
#include <algorithm>
#include <type_traits>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "row_stream.cuh"

namespace dels {
namespace {

constexpr int kPackThreads = 128;

// A thread lays out a row's codes of a block of 128 inputs.
__global__ void __launch_bounds__(kPackThreads) k_w4_pack(const W4PackArgs a) {
  pdl_wait();
  if (threadIdx.x == 0) pdl_trigger();
  const int row = threadIdx.x;
  const long long tile = blockIdx.x, v = tile * kW4Rows + row;
  const int groups = (a.K + a.group - 1) / a.group;
  bool bad = false;
  for (int kb = blockIdx.y; kb < a.lay.blocks; kb += gridDim.y) {
    const int ng = kW4Block / a.group;
    uint8_t* block = a.packed + tile * a.lay.tile_bytes + (long long)kb * a.lay.block_bytes;
    for (int u = 0; u < 4; ++u) {
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k = kb * kW4Block + u * kW4Unit + 8 * j;
        const uint8_t* from = a.codes + v * a.K + k;
        uint32_t c[8];
        if (v < a.V && k + 8 <= a.K && (reinterpret_cast<uintptr_t>(from) & 7u) == 0) {
          const uint2 x = __ldg(reinterpret_cast<const uint2*>(from));
#pragma unroll
          for (int i = 0; i < 8; ++i) c[i] = ((i < 4 ? x.x : x.y) >> (8 * (i & 3))) & 255u;
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) c[i] = v < a.V && k + i < a.K ? __ldg(from + i) : 0u;
        }
        uint32_t x = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          bad |= c[i] > 15;
          x |= (c[i] & 15u) << (4 * (i >> 1) + 16 * (i & 1));
        }
        w[j] = x;
      }
      reinterpret_cast<uint4*>(block + u * kW4UnitBytes)[row] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    for (int h = 0; h < ng; ++h) {
      const int grp = kb * ng + h;
      const long long at = v * groups + grp;
      const bool there = v < a.V && grp < groups;
      uint8_t* scales = block + 4 * kW4UnitBytes + h * 256;
      reinterpret_cast<uint16_t*>(scales)[row] = there ? a.scales[at] : 0;
      if (a.zeros) {
        const uint32_t z = there ? a.zeros[at] : 0;
        bad |= z > 15;
        const uint32_t other = __shfl_down_sync(0xFFFFFFFFu, z, 1);
        if ((row & 1) == 0) block[4 * kW4UnitBytes + ng * 256 + h * 64 + row / 2] = (uint8_t)((z & 15u) | (other & 15u) << 4);
      }
    }
  }
  if (bad) raise_status(a.status, DELS_STATUS_BAD_VALUE);
}

// ---------------------------------------------------------------------------
// y = W x on the tensor cores (tcgen05, the weights from tensor memory).
//
// A code minus its zero point is a whole number of -15 .. 15: fp16 operands hold it, its products with
// a feature's 11 bits are exact, and a group's sum is float32 and scaled there. Codes become fp16 by the
// published way of writing a small whole number into the mantissa of a number whose last place is 1, and taking
// that number off (Kim et al. 2022, "Who Says Elephants Can't Run"): fp16's 10 bits of mantissa hold a code
// where it lies in a byte, low or high: (w & 0x000F000F) | 0x6400 is 1024 + c
// and the high ones' 1024 + 16 c, so that a word of 8 codes takes 4 masks and a shift, and an fma a
// pair takes the zero point off. (Without an exponent, as multiples of 2^-24, the codes need neither, but the
// tensor cores align such numbers' products by the exponent they do not have, ten bits too far
// up: sums were off by 8e-7 of themselves, now by 1e-7.) A request's features are scaled by a power of
// two: bf16 ones to 2^16 at most, so that fp16 holds them exactly down to 2^-32 of the request's
// largest and what is smaller to 2^-40 of that; float32 ones, to 2^15, are three terms, two of 12 bits of a fixed
// point with their signs and one of 11, to 2^-35 of the largest. (A request with infinities or NaN has NaN throughout.)
// mma.sync, with the same operands, issues at most one such product in 32 cycles of a quarter
// SM: 151936 x 2560 for 8 requests 45 us, 151936 x 256 for 64 37 us, at that rate.
//
// Four warps (eight from 17 requests on) take a tile of 128 rows, a thread a row: codes of a block of 128 inputs
// from shared memory (bulk copies into a ring of their own, blocks ahead), operand pairs into
// tensor memory, one thread's MMAs over them with the features as the other operand,
// the groups' sums back and scaled into the thread's registers. Up to four such groups on an SM
// run beside one another and share nothing but the features: one's waits are the others' time. Few tiles of a
// long K are shared by several groups, each a range of it. A group's products and copies are issued by a warp
// of its own, which meets the others at one named barrier a step; these go on without waiting there. (At an
// mbarrier, with a time limit: 2 to 4 % more.)
// (With every part of a step in warps of its own, behind mbarriers with buffers to spare, the
// hand-overs' instructions took more than the overlap gave: 103 us against 80 at 8 requests.)
// The features stay in shared memory; a K whose features do not fit is taken in parts.
//
// What bounds it: the length of a step's chain (four units of 32 inputs, two with 9 to 16 requests and with more than
// 32): it goes from one of its parts to the next, 1300 cycles, most of them the instructions that take the codes apart. With
// 8 requests the warps issue in two thirds of all cycles, with one and with 64 in half of them, the tensor cores
// are busy for 9 to 15 % (ncu, cold). 151936 x 1024 for one request 17.6 us, x 2560 for 8 35.4 us
// (12.3 and 30.7 for the bytes at a copy's rate), 151936 x 256 for 64 16.7 us (6.1), 32003 x 1000 for 5 with
// float32 features 9.4 us (2.7; a start of 4 us, eight steps one after another, some registers spilled).
//
// Records of a drafted position come in the products' turn from the same warps: 64 requests and K 256 take 0.67 ms a
// block of 16 where a bf16 matrix takes 0.45 (temperature 0; 0.77 and 0.58 at 1), one request and K 1024 0.58 for 0.88.
// ---------------------------------------------------------------------------
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
               "l"(src), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}
// D[tmem] (+)= A[tmem] B[smem]^T: fp16 operands, float32 sums.
__device__ __forceinline__ void mma_from_tmem(uint32_t d, uint32_t a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_st_x16(uint32_t at, const uint32_t (&u)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(at),
      "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]),
      "r"(u[10]), "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15])
      : "memory");
}
// 8, 16 or 32 sums of the thread's row, the wait for them in the same statement: nothing that uses
// them can come before it.
__device__ __forceinline__ void tmem_ld_now(uint32_t at, float (&r)[8]) {
  uint32_t* u = reinterpret_cast<uint32_t*>(r);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7])
      : "r"(at)
      : "memory");
}
__device__ __forceinline__ void tmem_ld_now(uint32_t at, float (&r)[16]) {
  uint32_t* u = reinterpret_cast<uint32_t*>(r);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]),
        "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
      : "r"(at)
      : "memory");
}
__device__ __forceinline__ void tmem_ld_now(uint32_t at, float (&r)[32]) {
  uint32_t* u = reinterpret_cast<uint32_t*>(r);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]),
        "=r"(u[8]), "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]),
        "=r"(u[16]), "=r"(u[17]), "=r"(u[18]), "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]),
        "=r"(u[24]), "=r"(u[25]), "=r"(u[26]), "=r"(u[27]), "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
      : "r"(at)
      : "memory");
}
// Shared-memory matrix descriptor, K-major without swizzle: 8 rows x 16 bytes are 128 bytes side by
// side, `lead` bytes from one 8 inputs to the next, `stride` from 8 rows to the next.
__device__ __forceinline__ uint64_t smem_desc_plain(uint32_t addr, uint32_t lead, uint32_t stride) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(stride >> 4) << 32 |
         (uint64_t)1 << 46;
}
// fp16 operands, float32 sums, both K-major.
__host__ __device__ constexpr uint32_t idesc_f16_f32(int M, int N) {
  return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
// (w & mask) | base in one instruction: given as two constants the compiler made two of it.
__device__ __forceinline__ uint32_t pick(uint32_t w, uint32_t mask, uint32_t base) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(w), "r"(mask), "r"(base));
  return r;
}
// Zero points as pairs_of() takes them off.
struct ZeroPoint {
  uint32_t low, high;      // 1024 + z and -(64 + z), twice
  __device__ __forceinline__ explicit ZeroPoint(uint32_t z)
      : low(0x64006400u + z * 0x00010001u), high(0xD400D400u + z * 0x00100010u) {}
};
// Operand pairs of a word of 8 codes. base: 0x64006400, in a register.
__device__ __forceinline__ void pairs_of(uint32_t w, uint32_t base, const ZeroPoint& z, uint32_t* m) {
  const uint32_t next = w >> 8;
  const uint32_t c[4] = {pick(w, 0x000F000Fu, base), pick(w, 0x00F000F0u, base), pick(next, 0x000F000Fu, base),
                         pick(next, 0x00F000F0u, base)};
#pragma unroll
  for (int q = 0; q < 4; q += 2) {
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(m[q]) : "r"(c[q]), "r"(z.low));
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(m[q + 1]) : "r"(c[q + 1]), "r"(0x2C002C00u), "r"(z.high));
  }
}

// 8 features of a row as they are stored.
template <bool F32>
struct Features {
  uint4 w[F32 ? 2 : 1];
  // From column k on (0 past K, and past the last row).
  __device__ __forceinline__ void load(const W4Args& a, int b, int k) {
    using T = std::conditional_t<F32, uint32_t, uint16_t>;
    const T* x = static_cast<const T*>(a.x) + b * a.ld_x + k;
    const int n = b < a.B ? a.K - k : 0;
    if (n >= 8 && (reinterpret_cast<uintptr_t>(x) & 15u) == 0) {
#pragma unroll
      for (int i = 0; i < (F32 ? 2 : 1); ++i) w[i] = __ldg(reinterpret_cast<const uint4*>(x) + i);
      return;
    }
    uint32_t h[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = i < n ? (uint32_t)__ldg(x + i) : 0u;
    if constexpr (F32) {
      w[0] = make_uint4(h[0], h[1], h[2], h[3]);
      w[1] = make_uint4(h[4], h[5], h[6], h[7]);
    } else {
      w[0] = make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
    }
  }
  __device__ __forceinline__ void unpack(float (&f)[8]) const {
    if constexpr (F32) {
      f[0] = __uint_as_float(w[0].x); f[1] = __uint_as_float(w[0].y);
      f[2] = __uint_as_float(w[0].z); f[3] = __uint_as_float(w[0].w);
      f[4] = __uint_as_float(w[1].x); f[5] = __uint_as_float(w[1].y);
      f[6] = __uint_as_float(w[1].z); f[7] = __uint_as_float(w[1].w);
    } else {
      f[0] = bf16lo(w[0].x); f[1] = bf16hi(w[0].x); f[2] = bf16lo(w[0].y); f[3] = bf16hi(w[0].y);
      f[4] = bf16lo(w[0].z); f[5] = bf16hi(w[0].z); f[6] = bf16lo(w[0].w); f[7] = bf16hi(w[0].w);
    }
  }
};

// A request's power of two: its features' largest, of these bits, comes to 2^15 .. 2^16 (a bf16 number there is below fp16's
// largest, 65504), of several terms to 2^14 .. 2^15 (the first one is rounded, up to 2^15).
template <int TERMS>
__device__ __forceinline__ int feature_shift(uint32_t bits) {
  return bits ? (TERMS == 1 ? 15 : 14) - ilogbf(__uint_as_float(bits)) : 0;
}
__device__ __forceinline__ float pow2i(int e) { return __int_as_float((e + 127) << 23); }    // -126 .. 127

// 8 features of a lane, scaled by f.x f.y (two factors: the power may be past float32's range), as TERMS
// fp16 terms, `apart` 16-byte places from one to the next.
template <int TERMS>
__device__ __forceinline__ void put_features(const float (&x)[8], const float2& f, int apart, uint4* dst) {
  const f32x2 f0 = both2(f.x), f1 = both2(f.y);
  uint32_t t[TERMS][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f32x2 r = mul2(mul2(pair2(x[2 * i], x[2 * i + 1]), f0), f1);
#pragma unroll
    for (int k = 0; k < TERMS; ++k) {
      // of several terms each but the last is a whole multiple of its place, 2^11 of them at most: 2^4, and 2^-8 of what
      // is left; the last one is rounded, by 2^-21 at most
      f32x2 d = r;
      float d0, d1;
      if (k + 1 < TERMS) {
        const float place = k ? 49152.f : 201326592.f;                    // 1.5 2^(23 - 8), 1.5 2^(23 + 4)
        d = add2(add2(r, both2(place)), both2(-place));
        split2(d, d0, d1);
        r = add2(r, pair2(-d0, -d1));
      }
      split2(d, d0, d1);
      const __half2 h = __floats2half2_rn(d0, d1);
      t[k][i] = *reinterpret_cast<const uint32_t*>(&h);
    }
  }
#pragma unroll
  for (int k = 0; k < TERMS; ++k) dst[k * apart] = make_uint4(t[k][0], t[k][1], t[k][2], t[k][3]);
}

constexpr int kW4Stages = 8;               // of a ring, at most

// How a product runs: groups of four warps in a CTA, their rings, parts of K, units of an operand.
struct W4Plan {
  int groups;
  int stages, stage_bytes;
  int split;           // groups that share a tile, each a range of its blocks (features resident)
  int part_units;      // a multiple of 4: the features of so many units stay (all of them, or a part at a time)
  int parts;
  int a_cols, d_cols;  // tensor memory of a group: its operand, its sums
  uint32_t tmem_cols;
  int smem;
  int stall;           // of the self test: 1 no block is copied, 2 no product's end is reported
  unsigned budget_ns;  // of a wait
};

template <int NB>
constexpr int kW4Groups = NB >= 32 ? 2 : 4;
// Units of an operand: as many as leave registers for the sums (32 requests, 151936 x 1024: 2 33.0 us, 4 30.6).
template <int NB>
constexpr int kW4Step = NB == 8 || NB == 32 ? 4 : 2;
// Halves of a group: with 64 requests eight warps take a tile, every four half of its operand and half of the
// requests' sums. (Three groups of four warps, a thread with all 64 sums in 168 registers: 24.6 us, and 1.04 ms a
// block of 16 where this takes 0.72; three of eight warps spill: 23.2, 0.87.)
template <int NB>
constexpr int kW4Halves = NB >= 32 ? 2 : 1;
// Threads of a group: the warps that take codes apart and add sums up and, of outputs, one that issues products and
// copies. (Issued by one of the others: 18.8 us for one request, 38.5 for 8, 22.6 for 64, in place of 17.9, 36.0, 19.1.
// Records need more registers than the 96 that this leaves a thread: 0.69 ms a block of 16 for 64 requests, with it 0.87.)
template <int NB, bool APART>
constexpr int kW4Group = 128 * kW4Halves<NB> + 32 * APART;

__device__ __forceinline__ bool elect_one() {
  uint32_t yes;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
  return yes != 0;
}
// The products of UNITS units: operand columns from `acol`, sums from `dcol`, features from
// the descriptor's low word `x`; GUNITS units a group; ADD: to what the sums hold. (All of it known but for
// three words: what the compiler has to fetch from a thread's register for each product takes 60
// cycles a product.) The smallest terms first: the tensor cores cut what they add off at the last place of
// the largest, and of the largest terms, whole multiples of one number, there is then nothing to cut.
template <int NB, int TERMS, int UNITS, int GUNITS, bool ADD>
__device__ __forceinline__ void issue_products(uint32_t dcol, uint32_t acol, uint32_t x, uint32_t part_units) {
  constexpr int N = NB < 16 ? 16 : NB;
  constexpr uint32_t kHigh = (NB < 16 ? 0u : 128u >> 4) | 1u << 14;      // of the descriptor
#pragma unroll
  for (int g = 0; g < UNITS / GUNITS; ++g)
#pragma unroll
    for (int term = TERMS - 1; term >= 0; --term)
#pragma unroll
      for (int v = 0; v < GUNITS; ++v)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int u = g * GUNITS + v;
          mma_from_tmem(dcol + g * N, acol + u * 16 + k * 8,
                        (uint64_t)kHigh << 32 | (x + (term ? term * part_units * 4 * NB : 0u) + u * 4 * NB + k * 2 * NB),
                        idesc_f16_f32(128, N), ADD || term + 1 < TERMS || v || k);
        }
}

// Where a group waits.
struct W4Waits {
  uint64_t full[kW4Stages];          // a block of codes has come
  uint64_t done;                     // a step's products are done
  uint64_t last;                     // and all of them, where a wait has run out
  volatile int passed;               // steps for which every warp has arrived, mod 2, as the issuing one has seen
};

// What a launch does with its products: outputs, or records of the fused rows at temperature 0 or 1.
enum { kOutputs = 0, kRecords = 1, kKeys = 2 };

// The fused rows' records: a group of warps lays a tile's products out by requests, 32 at a time, and
// every thread goes along as many columns of one: 8 of its products, logits and priors a step. (Each
// warp's 32 rows of every request by shuffles, with no layout between, took 64 requests' block
// of 16 2.4 ms.)
template <int NB>
constexpr int kW4Side = NB < 32 ? NB : 32 / kW4Halves<NB>;      // requests laid out at a time, and a thread's columns
constexpr int kW4Pitch = kW4Rows + 4;
struct RowTop {
  float best, second, m, s;                            // m: the sum's reference
  int idx;
};

// One product of the thread's own row: what one and two requests take, with no layout (0.59 ms a block of 16
// where it took 0.67).
template <bool KEYS>
__device__ __forceinline__ void combine_one(const W4Args& a, float y, int b, long long v, RowTop& r) {
  const long long at = b * a.ld_long + v;
  const float l = a.long_f32 ? __ldcs(static_cast<const float*>(a.longp) + at)
                             : bf16_to_f(__ldcs(static_cast<const uint16_t*>(a.longp) + at));
  const float f[1] = {fmaf(-a.beta, __ldg(a.prior + v), fmaf(a.alpha, y, l))};
  top2_push(KEYS ? f[0] + gumbel_at(a.seed, a.step, b, a.j, kStreamDraft, v) : f[0], (int)v, r.best, r.second, r.idx);
  lse_chunk_ex2<1>(f, r.best, r.m, r.s);
}

template <int S, bool KEYS>
__device__ __forceinline__ void combine_columns(const W4Args& a, const float* y, int b, long long v0, RowTop& r) {
#pragma unroll
  for (int c = 0; c < S; c += 8) {
    const long long v = v0 + c;
    if (v >= a.V) return;                              // (V is a multiple of 8)
    const float4 y0 = *reinterpret_cast<const float4*>(y + c), y1 = *reinterpret_cast<const float4*>(y + c + 4);
    const float4 p0 = __ldg(reinterpret_cast<const float4*>(a.prior + v));
    const float4 p1 = __ldg(reinterpret_cast<const float4*>(a.prior + v + 4));
    float f[8];
    if (a.long_f32) {
      const float4* l = reinterpret_cast<const float4*>(static_cast<const float*>(a.longp) + b * a.ld_long + v);
      const float4 l0 = __ldcs(l), l1 = __ldcs(l + 1);
      f[0] = l0.x; f[1] = l0.y; f[2] = l0.z; f[3] = l0.w; f[4] = l1.x; f[5] = l1.y; f[6] = l1.z; f[7] = l1.w;
    } else {
      const uint4 l = __ldcs(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.longp) + b * a.ld_long + v));
      f[0] = bf16lo(l.x); f[1] = bf16hi(l.x); f[2] = bf16lo(l.y); f[3] = bf16hi(l.y);
      f[4] = bf16lo(l.z); f[5] = bf16hi(l.z); f[6] = bf16lo(l.w); f[7] = bf16hi(l.w);
    }
    const float yy[8] = {y0.x, y0.y, y0.z, y0.w, y1.x, y1.y, y1.z, y1.w};
    const float pp[8] = {p0.x, p0.y, p0.z, p0.w, p1.x, p1.y, p1.z, p1.w};
    float k[8], top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) k[i] = f[i] = fmaf(-a.beta, pp[i], fmaf(a.alpha, yy[i], f[i]));
    if constexpr (KEYS) {
      float g[8];
      gumbel8(a.seed, a.step, b, a.j, kStreamDraft, v >> 3, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) k[i] += g[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, k[i]);
    if (top > r.second) {                              // (others change neither the largest nor the runner-up)
#pragma unroll
      for (int i = 0; i < 8; ++i) top2_push(k[i], (int)v + i, r.best, r.second, r.idx);
    }
    lse_chunk_ex2<8>(f, r.best, r.m, r.s);
  }
}

// SPLIT: tiles are shared by p.split groups (else its registers cost 2 to 4 %).
template <int NB, int TERMS, int EPI, bool SPLIT>
__global__ void __launch_bounds__(kW4Groups<NB> * kW4Group<NB, EPI == kOutputs>, 1)
    k_w4_project(const W4Args a, const W4Plan p) {
  extern __shared__ __align__(128) uint8_t smem[];
  constexpr int N = NB < 16 ? 16 : NB;                  // requests of an MMA: rows past NB are its first ones again
  constexpr int H = kW4Halves<NB>, kMine = NB / H;      // requests of a thread
  // Named barriers, behind that of __syncthreads(): each group's, of all its warps; each half's of a group, of its
  // workers; each tile's that groups share. An id has one number of threads at a time: with a half's the same as its group's, at
  // which the issuing warp was already waiting for the next step, a kernel faulted.
  constexpr int kGroupBarrier = 1, kHalfBarrier = kGroupBarrier + kW4Groups<NB>;
  constexpr int kTileBarrier = kHalfBarrier + kW4Groups<NB> * H;
  static_assert(kTileBarrier + kW4Groups<NB> <= 16, "a CTA's named barriers");
  __shared__ W4Waits waits[kW4Groups<NB>];
  __shared__ uint32_t tmem_base;
  __shared__ volatile int abort_flag;
  __shared__ uint32_t largest[NB];          // bits of the requests' largest features
  __shared__ float2 scaled[NB];             // their powers of two, in two factors
  __shared__ __align__(16) float back[2][NB];      // what takes them back, the same way
  // (through a reduction, which leaves it in a uniform register: the products' operands are then worked
  // out there, and not fetched from a thread's registers one by one)
  const int tid = threadIdx.x, lane = tid & 31, warp = (int)__reduce_max_sync(0xFFFFFFFFu, (unsigned)tid >> 5);
  constexpr bool kApart = EPI == kOutputs;              // the issuing warps are others than the workers, the last ones
  const int workers = p.groups * 4 * H, warps = workers + (kApart ? p.groups : 0);
  const bool issues = kApart && warp >= workers;
  const int grp = issues ? warp - workers : warp / (4 * H), half = H > 1 ? warp / 4 % H : 0, row = tid & 127;
  // else of a group's warps one issues products and the next one copies: not in the same quarter of the SM in all groups
  const int place = warp % (4 * H), issuer = grp & 3, copier = issuer ^ 1;
  const int b0 = blockIdx.y * NB;
  W4Waits& bar = waits[grp];
  uint8_t* ring = smem + (size_t)grp * p.stages * p.stage_bytes;
  uint4* operand = reinterpret_cast<uint4*>(smem + (size_t)p.groups * p.stages * p.stage_bytes);
  if (warp == 0) {
    tmem_alloc(&tmem_base, p.tmem_cols);
    tmem_relinquish();
  }
  if (tid == 0) {
    abort_flag = 0;
    for (int g = 0; g < p.groups; ++g) {
      for (int i = 0; i < p.stages; ++i) mbar_init(&waits[g].full[i], 1);
      mbar_init(&waits[g].done, 1);
      mbar_init(&waits[g].last, 1);
      waits[g].passed = 0;
    }
    fence_mbarrier_init();
  }
  if (tid < NB) largest[tid] = 0;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_wait();
  if (tid == 0) pdl_trigger();

  // ---- a group's tiles: every (CTAs x groups)th, and its copies, a block each
  const int split = SPLIT ? p.split : 1, slot = grp / split, share = grp - slot * split;
  const int kb0 = a.lay.blocks * share / split, own_blocks = a.lay.blocks * (share + 1) / split - kb0;
  const long long tile0 = (long long)slot * gridDim.x + blockIdx.x, apart = (long long)gridDim.x * (p.groups / split);
  const long long rounds = (a.lay.tiles + apart - 1) / apart;
  const int copies = p.stall != 1 && tile0 < a.lay.tiles ? (int)((a.lay.tiles - tile0 + apart - 1) / apart) * own_blocks : 0;
  int to_copy = copies - p.stages, next_kb = p.stages % own_blocks, next_st = 0;            // of the thread that copies
  const uint8_t* next_block = a.packed + (tile0 + p.stages / own_blocks * apart) * a.lay.tile_bytes +
                              (long long)(kb0 + next_kb) * a.lay.block_bytes;
  const auto issue_copy = [&] {
    if (to_copy <= 0) return;
    --to_copy;
    mbar_arrive_expect_tx(&bar.full[next_st], a.lay.block_bytes);
    bulk_load(ring + next_st * p.stage_bytes, next_block, a.lay.block_bytes, &bar.full[next_st]);
    next_block += a.lay.block_bytes;
    if (++next_st == p.stages) next_st = 0;
    if (++next_kb == own_blocks) {
      next_kb = 0;
      next_block += apart * a.lay.tile_bytes - (long long)own_blocks * a.lay.block_bytes;
    }
  };
  // ---- the requests' features, read before the first copies take the memory; those of a warp's first
  // units stay in registers from the search for their largest
  using X = Features<TERMS == 3>;
  constexpr int kKept = TERMS == 3 ? 3 : 6;
  const int all_units = 4 * a.lay.blocks, all = all_units * (NB / 8);
  const auto load_task = [&](int task, X& x) {
    x.load(a, b0 + 8 * (task % (NB / 8)) + (lane >> 2), task / (NB / 8) * kW4Unit + 8 * (lane & 3));
  };
  X kept[kKept];
#pragma unroll
  for (int i = 0; i < kKept; ++i)
    if (warp + i * warps < all) load_task(warp + i * warps, kept[i]);
  fence_proxy_async_global();
  if ((kApart ? issues : place == copier) && lane < p.stages) {             // the first ones, a lane each
    const long long tile = tile0 + lane / own_blocks * apart;
    const int kb = kb0 + lane % own_blocks;
    if (lane < copies) {
      mbar_arrive_expect_tx(&bar.full[lane], a.lay.block_bytes);
      bulk_load(ring + (size_t)lane * p.stage_bytes,
                a.packed + tile * a.lay.tile_bytes + (long long)kb * a.lay.block_bytes, a.lay.block_bytes,
                &bar.full[lane]);
    }
  }

  const auto look = [&](const X& x, int task) {
    float f[8];
    x.unpack(f);
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(f[i]) & 0x7FFFFFFFu);      // NaN above infinity
    m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
    m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
    if ((lane & 3) == 0) atomicMax(&largest[8 * (task % (NB / 8)) + (lane >> 2)], m);
  };
  for (int task = warp + kKept * warps; task < all; task += warps) {
    X x;
    load_task(task, x);
    look(x, task);
  }
#pragma unroll
  for (int i = 0; i < kKept; ++i)
    if (warp + i * warps < all) look(kept[i], warp + i * warps);
  __syncthreads();
  if (tid < NB) {
    const bool finite = largest[tid] < 0x7F800000u;
    const int up = finite ? feature_shift<TERMS>(largest[tid]) : 0, sh = -up;
    scaled[tid] = make_float2(pow2i(up / 2), pow2i(up - up / 2));
    back[0][tid] = finite ? pow2i(sh / 2) : NAN;
    back[1][tid] = finite ? pow2i(sh - sh / 2) : NAN;
  }
  __syncthreads();
  // The features of units u0 .. u1 - 1.
  const int gunits = a.group / kW4Unit, glog = 31 - __clz(gunits);
  const auto stage = [&](int u0, int u1, bool from_kept) {
    const auto place = [&](const X& raw, int task) {
      float x[8];
      raw.unpack(x);
      const int n = 8 * (task % (NB / 8)) + (lane >> 2), u = task / (NB / 8);
      uint4* dst = operand + ((u - u0) * 4 + (lane & 3)) * NB + n;
      put_features<TERMS>(x, scaled[n], p.part_units * 4 * NB, dst);
    };
    const int t0 = u0 * (NB / 8), t1 = u1 * (NB / 8);
    int task = t0 + warp;
    if (from_kept) {
#pragma unroll
      for (int i = 0; i < kKept; ++i, task += warps)
        if (task < t1) place(kept[i], task);
    }
    for (; task < t1; task += warps) {
      X x;
      load_task(task, x);
      place(x, task);
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
  };
  const bool resident = p.parts == 1;
  if (resident) stage(0, all_units, true);

  const uint32_t acol = __reduce_max_sync(0xFFFFFFFFu, tmem_base) + (uint32_t)grp * (p.a_cols + p.d_cols);
  const uint32_t dcol = acol + p.a_cols;
  const uint32_t quadrant = (uint32_t)(warp & 3) << 21;                // the warp's 32 lanes of tensor memory
  const uint32_t x0 = (uint32_t)smem_desc_plain(smem_u32(operand), NB * 16, 0) + (uint32_t)(kb0 * 4) * (4 * NB);
  bool dead = false;                        // a wait ran out: the rest runs through without waiting
  const auto ran_out = [&](uint32_t polls, uint64_t& deadline) {
    // (the clock is read in long waits alone: a reading takes about 1000 cycles)
    if (polls & 255u) return;
    if (!deadline) deadline = globaltimer_ns() + p.budget_ns;
    else if (abort_flag || globaltimer_ns() > deadline) abort_flag = dead = true;
  };
  const auto wait = [&](uint64_t* at, int parity) {
    uint64_t deadline = 0;
    for (uint32_t polls = 1; !mbar_try_wait(at, (uint32_t)parity) && !dead; ++polls) ran_out(polls, deadline);
    __syncwarp();
  };
  // A step's products, `step` its number mod 2. They are done: every warp of the group has arrived for the step, and this
  // one may for the next. A thread that waits for them no more waits for that itself: two arrivals of a warp in one step would
  // stand for another's, the issuing warp's among them, which would be left without partners at its last. (It comes: each
  // warp arrives once for each step, and waits for nothing else without a limit.)
  const auto wait_done = [&](int step) {
    uint64_t deadline = 0;
    for (uint32_t polls = 1; dead || !mbar_try_wait(&bar.done, (uint32_t)step); ++polls) {
      if (dead) {
        const uint64_t limit = globaltimer_ns() + p.budget_ns;
        while (bar.passed == step && globaltimer_ns() < limit) {}
        break;
      }
      ran_out(polls, deadline);
    }
    __syncwarp();
  };
  int st = 0, ph = 0, dph = 0;
  uint32_t base = 0x64006400u;
  asm("" : "+r"(base));                   // (a register, not a constant)
  f32x2 tot[kMine / 2];
  constexpr int S = kW4Side<NB>;
  // shares of tiles [slots][split - 1][NB][128]
  float* joins = reinterpret_cast<float*>(operand + (size_t)TERMS * p.part_units * 4 * NB);
  float* sides = joins + (SPLIT ? (size_t)(p.groups - p.groups / split) * NB * kW4Rows : 0);                 // of the records
  const bool own_rows = EPI != kOutputs && NB == 8 && a.B <= 2;
  constexpr int kTops = NB == 8 ? 2 : kMine / S;
  RowTop tops[kTops];                       // of the half's requests row % S, row % S + S; of 0 and 1 where these have their own rows
#pragma unroll
  for (int h = 0; h < kTops; ++h) tops[h] = RowTop{-INFINITY, -INFINITY, -INFINITY, 0.f, 0x7FFFFFFF};

  // Sums of an operand's group i, scaled.
  const auto add_sums = [&](int i, float scale) {
    const f32x2 s2 = both2(scale);
    float acc[kMine];
    tmem_ld_now(dcol + quadrant + i * N + half * kMine, acc);
#pragma unroll
    for (int n = 0; n < kMine; n += 2) tot[n / 2] = fma2(s2, pair2(acc[n], acc[n + 1]), tot[n / 2]);
  };

  // Blocks of a part, U units an operand, G a group: while a step's products run the next one's codes are
  // taken apart.
  const auto run = [&](int blocks, auto step_units, auto group_units) {
    constexpr int U = decltype(step_units)::value, G = decltype(group_units)::value, NG = U > G ? U / G : 1;
    constexpr int kSteps = 4 / U, UH = U / H;            // units that a half takes apart
    uint32_t m[UH * 16];
    float scale[NG];
    const auto load = [&](int i) {
      const int s0 = i % kSteps * U;
      if (s0 == 0) wait(&bar.full[st], ph);
      const uint8_t* block = ring + (size_t)st * p.stage_bytes;
      const uint8_t* scales = block + 4 * kW4UnitBytes + s0 / G * 256 + row * 2;
      const uint8_t* zeros = block + 4 * kW4UnitBytes + 4 / G * 256 + s0 / G * 64 + (row >> 1);
      uint4 w[UH];
#pragma unroll
      for (int u = 0; u < UH; ++u)
        w[u] = (reinterpret_cast<const uint4*>(block + (s0 + half * UH) * kW4UnitBytes) + row)[u * kW4Rows];
#pragma unroll
      for (int g = 0; g < NG; ++g) scale[g] = bf16_to_f(*reinterpret_cast<const uint16_t*>(scales + g * 256));
      constexpr int NZ = (NG + H - 1) / H;               // groups of the half's units
#pragma unroll
      for (int g = 0; g < NZ; ++g) {
        const ZeroPoint z(a.zeros ? zeros[(NG > 1 ? half * NZ + g : 0) * 64] >> (4 * (row & 1)) & 15u : 8u);
#pragma unroll
        for (int u = g * (UH / NZ); u < (g + 1) * (UH / NZ); ++u) {
          pairs_of(w[u].x, base, z, m + u * 16);
          pairs_of(w[u].y, base, z, m + u * 16 + 4);
          pairs_of(w[u].z, base, z, m + u * 16 + 8);
          pairs_of(w[u].w, base, z, m + u * 16 + 12);
        }
      }
      if (s0 + U == 4 && ++st == p.stages) st = 0, ph ^= 1;
    };
    const auto issue = [&](int i) {         // (every worker has left a step's operand in its place)
      asm volatile("bar.sync %0, %1;" ::"r"(kGroupBarrier + grp), "n"(kW4Group<NB, kApart>) : "memory");
      tc_fence_after();
      if (elect_one()) {
        const uint32_t x = x0 + (uint32_t)(i * U) * (4 * NB);
        if (G > U && i % kSteps > 0) issue_products<NB, TERMS, U, U, true>(dcol, acol, x, p.part_units);
        else issue_products<NB, TERMS, U, (G > U ? U : G), false>(dcol, acol, x, p.part_units);
        if (p.stall != 2) tc_commit(&bar.done);
        bar.passed = dph ^ 1;
      }
      __syncwarp();
    };
    // (and read its block. Not once a wait has run out: its last copy may be on its way, and the next would count into
    // that one's phase. A worker has waited for that itself.)
    const auto copy_next = [&](int i) {
      if (i % kSteps == kSteps - 1 && lane == 0 && !(kApart ? abort_flag != 0 : dead)) issue_copy();
      __syncwarp();
    };
    if (issues) {
      for (int i = 0; i < blocks * kSteps; ++i) {
        issue(i);
        copy_next(i);
        dph ^= 1;
      }
      return;
    }
    load(0);
    for (int i = 0; i < blocks * kSteps; ++i) {
      const int at = i % kSteps * U;
#pragma unroll
      for (int u = 0; u < UH; ++u)
        tmem_st_x16(acol + quadrant + (half * UH + u) * 16, *reinterpret_cast<uint32_t(*)[16]>(m + u * 16));
      float s_now[NG];
#pragma unroll
      for (int g = 0; g < NG; ++g) s_now[g] = scale[g];
      tmem_st_wait();
      tc_fence_before();
      if (!kApart && place == issuer) issue(i);
      else asm volatile("bar.arrive %0, %1;" ::"r"(kGroupBarrier + grp), "n"(kW4Group<NB, kApart>) : "memory");
      if (i + 1 < blocks * kSteps) load(i + 1);
      wait_done(dph);
      dph ^= 1;
      tc_fence_after();
      if (!kApart && place == copier) copy_next(i);
      if (G <= U || at + U == 4) {
#pragma unroll
        for (int g = 0; g < NG; ++g) add_sums(g, s_now[g]);
      }
    }
  };

  for (long long r = 0; r < rounds; ++r) {
    const long long tile = tile0 + r * apart;
    const bool live = tile < a.lay.tiles;   // (a group without a tile keeps to the barriers)
#pragma unroll
    for (int n = 0; n < kMine / 2; ++n) tot[n] = 0ull;
    for (int part = 0; part < p.parts; ++part) {
      const int pu0 = part * p.part_units, pu1 = min(all_units, pu0 + p.part_units);
      if (!resident) {
        __syncthreads();                    // (the products of the part before have been waited for)
        stage(pu0, pu1, false);
      }
      if (!live) continue;
      using std::integral_constant;
      const int blocks = resident ? own_blocks : (pu1 - pu0) / 4;
      const integral_constant<int, 1> one;
      const integral_constant<int, 2> two;
      const integral_constant<int, 4> four;
      constexpr integral_constant<int, kW4Step<NB>> step_units;
      if (glog == 0) run(blocks, step_units, one);
      else if (glog == 1) run(blocks, step_units, two);
      else run(blocks, step_units, four);
    }
    if (issues) continue;
    if (SPLIT && live) {
      // ---- the shares of a tile, added up by its first group in their order
      const auto all_shares = [&] {
        asm volatile("bar.sync %0, %1;" ::"r"(kTileBarrier + slot), "r"(split * 128 * H) : "memory");
      };
      float* at = joins + ((size_t)slot * (split - 1) * NB + half * kMine) * kW4Rows + row;
      if (share) {
        at += (size_t)(share - 1) * NB * kW4Rows;
#pragma unroll
        for (int n = 0; n < kMine; n += 2) split2(tot[n / 2], at[n * kW4Rows], at[(n + 1) * kW4Rows]);
      }
      all_shares();
      if (!share)
        for (int i = 1; i < split; ++i, at += (size_t)NB * kW4Rows)
#pragma unroll
          for (int n = 0; n < kMine; n += 2)
            tot[n / 2] = add2(tot[n / 2], pair2(at[n * kW4Rows], at[(n + 1) * kW4Rows]));
      all_shares();                         // (read: the next tile's may come)
      if (share) continue;
    }
    const long long v = tile * kW4Rows + row;
    const int n0 = half * kMine, nb = min(kMine, a.B - b0 - n0);        // the thread's requests
    float* side = sides + (size_t)(grp * H + half) * S * kW4Pitch;
    const auto together = [&] { asm volatile("bar.sync %0, 128;" ::"r"(kHalfBarrier + grp * H + half) : "memory"); };
    // Products of 8 requests, n on. (All of them before any is stored: the compiler keeps each reading of back[]
    // behind the stores before it, and one after another they took half of 64 requests' time.)
    const auto products = [&](int n, float (&y)[8]) {
      float4 f[2][2];
#pragma unroll
      for (int k = 0; k < 4; ++k) f[k >> 1][k & 1] = *reinterpret_cast<const float4*>(&back[k >> 1][n0 + n + 4 * (k & 1)]);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const f32x2* t = tot + n / 2 + 2 * k;
        split2(mul2(mul2(t[0], pair2(f[0][k].x, f[0][k].y)), pair2(f[1][k].x, f[1][k].y)), y[4 * k], y[4 * k + 1]);
        split2(mul2(mul2(t[1], pair2(f[0][k].z, f[0][k].w)), pair2(f[1][k].z, f[1][k].w)), y[4 * k + 2], y[4 * k + 3]);
      }
    };
    const auto lay_out = [&](int h) {       // S requests' products of the tile, h S on, by requests
#pragma unroll
      for (int n = 0; n < S; n += 8) {
        float y[8];
        products(h * S + n, y);
#pragma unroll
        for (int i = 0; i < 8; ++i) side[(n + i) * kW4Pitch + row] = y[i];
      }
      together();
    };
    if constexpr (EPI == kOutputs) {
      // ---- outputs: a warp's 32 rows side by side
      if (live && v < a.V) {
#pragma unroll
        for (int n = 0; n < kMine; n += 8) {
          float y[8];
          products(n, y);
          const long long at = (long long)(b0 + n0 + n) * a.ld_out + v;
          const auto put = [&](auto* out, auto value) {
            if (n + 8 <= nb) {
#pragma unroll
              for (int i = 0; i < 8; ++i) out[i * a.ld_out] = value(y[i]);
            } else {
#pragma unroll
              for (int i = 0; i < 8; ++i)
                if (n + i < nb) out[i * a.ld_out] = value(y[i]);
            }
          };
          if (a.out_f32) put(static_cast<float*>(a.out) + at, [](float x) { return x; });
          else put(static_cast<__nv_bfloat16*>(a.out) + at, [](float x) { return __float2bfloat16_rn(x); });
        }
      }
    } else if (live && own_rows) {
      if (v < a.V) {
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          if (n >= nb) break;
          float y[2];
          split2(tot[0], y[0], y[1]);
          combine_one<EPI == kKeys>(a, y[n] * back[0][n] * back[1][n], b0 + n, v, tops[n]);
        }
      }
    } else if (live) {
      // ---- records of the fused rows
#pragma unroll
      for (int h = 0; h < kMine / S; ++h) {
        if (h * S >= nb) break;
        lay_out(h);
        const int n = row % S, c0 = row / S * S;
        if (h * S + n < nb)
          combine_columns<S, EPI == kKeys>(a, side + n * kW4Pitch + c0, b0 + n0 + h * S + n, tile * kW4Rows + c0, tops[h]);
        together();
      }
    }
  }
  if constexpr (EPI != kOutputs) {
    // ---- the CTA's records, one a thread, through the rings' memory
    __syncthreads();
    float4* all_recs = reinterpret_cast<float4*>(smem);                  // [groups][128 / S][NB], or [warps][NB]
    if (issues) {
    } else if (own_rows) {
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        RowAcc r;
        r.m = tops[n].best; r.s = tops[n].s; r.second = tops[n].second; r.idx = tops[n].idx;
        r = rowacc_warp_reduce(r);
        if (lane == 0) all_recs[warp * NB + n] = make_float4(r.m, r.s, r.second, __int_as_float(r.idx));
      }
    } else {
#pragma unroll
      for (int h = 0; h < kMine / S; ++h)
        all_recs[(grp * (128 / S) + row / S) * NB + half * kMine + h * S + row % S] =
            make_float4(tops[h].best, tops[h].s, tops[h].second, __int_as_float(tops[h].idx));
    }
    __syncthreads();
    if (tid < min(NB, a.B - b0)) {
      RowAcc r = rowacc_init();
      for (int i = 0; i < (own_rows ? workers : p.groups * (128 / S)); ++i) {
        const float4 x = all_recs[i * NB + tid];
        RowAcc o;
        o.m = x.x; o.s = x.y; o.second = x.z; o.idx = __float_as_int(x.w);
        r = rowacc_merge(r, o);
      }
      reinterpret_cast<float4*>(a.partials)[(long long)(b0 + tid) * a.partial_ld + blockIdx.x] =
          make_float4(r.m, r.s, r.second, __int_as_float(r.idx));
    }
  }
  if (dead && lane == 0) raise_status(a.status, DELS_STATUS_TIMEOUT);
  tc_fence_before();
  __syncthreads();
  if (abort_flag) {                         // a CTA that gives up has its copies and products in flight end first
    if ((kApart ? issues : place == copier) && lane == 0) {
      const uint64_t limit = globaltimer_ns() + p.budget_ns / 4;
      const int issued = min(copies, copies - to_copy);
      for (int i = max(0, issued - p.stages); i < issued; ++i)
        while (!mbar_try_wait(&bar.full[i % p.stages], (i / p.stages) & 1) && globaltimer_ns() < limit) {}
    }
    __syncwarp();
    if ((kApart ? issues : place == issuer) && elect_one()) {      // (the thread that issued them)
      const uint64_t limit = globaltimer_ns() + p.budget_ns / 4;
      tc_commit(&bar.last);
      while (!mbar_try_wait(&bar.last, 0) && globaltimer_ns() < limit) {}
    }
    __syncthreads();
  }
  if (warp == 0) tmem_dealloc(tmem_base, p.tmem_cols);
}

int w4_ctas(const W4Args& a, int NB, int sms) {
  const int btiles = (a.B + NB - 1) / NB;
  return (int)std::min<long long>(std::max(1, sms / btiles), a.lay.tiles);
}
int w4_requests(int B) { return B <= 8 ? 8 : B <= 16 ? 16 : B <= 32 ? 32 : 64; }    // of a CTA

template <int NB, int TERMS, int EPI>
cudaError_t launch_nb(const W4Args& a, cudaStream_t s) {
  const int sms = device_sm_count();
  const int side = EPI == kOutputs ? 0 : kW4Groups<NB> * kW4Halves<NB> * kW4Side<NB> * kW4Pitch * 4;
  int room = device_max_smem_optin() - 4096 - side;
  if (sms <= 0 || room <= 0) return cudaErrorInvalidValue;
  const int btiles = (a.B + NB - 1) / NB, ctas = w4_ctas(a, NB, sms);
  W4Plan p{};
  constexpr int N = NB < 16 ? 16 : NB;
  const int gunits = a.group / kW4Unit;
  p.stage_bytes = (a.lay.block_bytes + 127) / 128 * 128;
  const long long unit = (long long)TERMS * 4 * NB * 16, whole = 4 * a.lay.blocks * unit;
  // Groups that share a tile: as many as get through the CTA's tiles soonest, what comes with sharing (a join, and all
  // groups' first copies at once) taken as four steps' time, a block being one step or two. 8 requests of 17789 x
  // 4096: one group a tile 22.4 us, four 13.8; one of 10000 x 1024: 8.1, 6.9; 32003 x 1000 for 5: 9.8, two 10.1.
  constexpr int kStep = kW4Step<NB>;
  const auto join_bytes = [](int slots, int split) { return (long long)slots * (split - 1) * NB * kW4Rows * 4; };
  long long best = 0;
  for (int split = 1; split <= kW4Groups<NB> && split <= a.lay.blocks; split *= 2) {
    const int slots = (int)std::min<long long>(kW4Groups<NB> / split, (a.lay.tiles + ctas - 1) / ctas);
    const long long rounds = (a.lay.tiles + (long long)ctas * slots - 1) / ((long long)ctas * slots);
    const long long time = rounds * ((a.lay.blocks + split - 1) / split) + (split > 1 ? kStep : 0);
    const long long left = room - join_bytes(slots, split) - 2ll * slots * split * p.stage_bytes;
    if (split > 1 && (time >= best || left < whole)) continue;
    best = time;
    p.split = split;
    p.groups = slots * split;
  }
  const int join = (int)join_bytes(p.groups / p.split, p.split);
  room -= join;
  p.a_cols = 16 * kStep;
  p.d_cols = (kStep + gunits - 1) / gunits * N;
  static_assert(kW4Groups<NB> * kStep * (16 + N) <= 512, "a group's operand and sums, of one unit a group of inputs");
  p.tmem_cols = 32;
  while ((int)p.tmem_cols < p.groups * (p.a_cols + p.d_cols)) p.tmem_cols *= 2;
  // the features, or of those that do not fit as many as leave two stages; what they leave is the rings'
  const long long beside = room - 2ll * p.groups * p.stage_bytes;
  p.part_units = (int)(std::min(whole, beside) / unit / 4 * 4);
  p.parts = (4 * a.lay.blocks + p.part_units - 1) / p.part_units;
  p.stages = (int)std::min<long long>(kW4Stages, (room - p.part_units * unit) / ((long long)p.groups * p.stage_bytes));
  p.stall = a.stall;
  p.budget_ns = (unsigned)(a.stall ? kWaitBudgetNs / 20 : kWaitBudgetNs);
  p.smem = (int)(p.groups * p.stages * p.stage_bytes + p.part_units * unit) + join + side;
  const auto k = p.split > 1 ? k_w4_project<NB, TERMS, EPI, true> : k_w4_project<NB, TERMS, EPI, false>;
  const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(k), p.smem);
  if (e != cudaSuccess) return e;
  return launch_pdl(k, dim3((unsigned)ctas, (unsigned)btiles), dim3(p.groups * kW4Group<NB, EPI == kOutputs>),
                    (size_t)p.smem, s, a, p);
}

}  // namespace

cudaError_t launch_w4_pack(const W4PackArgs& a, cudaStream_t s) {
  const dim3 grid((unsigned)a.lay.tiles, (unsigned)(a.lay.blocks < 64 ? a.lay.blocks : 64));
  return launch_pdl(k_w4_pack, grid, dim3(kPackThreads), 0, s, a);
}

int w4_records(const W4Args& a, int sms) { return w4_ctas(a, w4_requests(a.B), sms); }

cudaError_t launch_w4_project(const W4Args& a, cudaStream_t s) {
  const auto launch = [&](auto terms, auto epi) {
    constexpr int T = decltype(terms)::value, E = decltype(epi)::value;
    switch (w4_requests(a.B)) {
      case 8: return launch_nb<8, T, E>(a, s);
      case 16: return launch_nb<16, T, E>(a, s);
      case 32: return launch_nb<32, T, E>(a, s);
      default: return launch_nb<64, T, E>(a, s);
    }
  };
  using std::integral_constant;
  if (a.partials)
    return a.sample ? launch(integral_constant<int, 1>{}, integral_constant<int, kKeys>{})
                    : launch(integral_constant<int, 1>{}, integral_constant<int, kRecords>{});
  return a.x_f32 ? launch(integral_constant<int, 3>{}, integral_constant<int, kOutputs>{})
                 : launch(integral_constant<int, 1>{}, integral_constant<int, kOutputs>{});
}

}  // namespace dels
