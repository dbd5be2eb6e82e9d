// Products with 4-bit weights: the layout of the codes, and y = W x.
#include <cuda_bf16.h>

#include "dels_device.cuh"

namespace dels {
namespace {

constexpr int kPackThreads = 128;

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

__device__ __forceinline__ void put(void* out, int f32, long long i, float x) {
  if (f32) static_cast<float*>(out)[i] = x;
  else static_cast<__nv_bfloat16*>(out)[i] = __float2bfloat16_rn(x);
}

// A thread takes an output.
__global__ void __launch_bounds__(128) k_w4_project(const W4Args a) {
  pdl_wait();
  if (threadIdx.x == 0) pdl_trigger();
  const long long v = (long long)blockIdx.x * 128 + threadIdx.x;
  const int b = blockIdx.y;
  if (v >= a.V) return;
  const long long tile = v / kW4Rows;
  const int row = (int)(v % kW4Rows), g = row & 7, i = row >> 3;
  float y = 0.f;
  for (int kb = 0; kb < a.lay.blocks; ++kb) {
    const int units = min(4, a.lay.units - 4 * kb), ng = (units * kW4Unit + a.group - 1) / a.group;
    const uint8_t* block = a.packed + tile * a.lay.tile_bytes + (long long)kb * a.lay.block_bytes;
    for (int h = 0; h < ng; ++h) {
      const float s = bf16_to_f(reinterpret_cast<const uint16_t*>(block + units * 512 + h * 64)[g * 4 + i]);
      int z = 8;
      if (a.zeros) z = (reinterpret_cast<const uint16_t*>(block + units * 512 + ng * 64 + h * 16)[g] >> (4 * i)) & 15;
      float sum = 0.f;
      const int end = min(kW4Block, min((h + 1) * a.group, a.K - kb * kW4Block));
      for (int k = h * a.group; k < end; ++k) {
        const int t = (k & 31) >> 3, e = k & 7;
        const uint32_t w =
            reinterpret_cast<const uint32_t*>(block)[((k >> 5) * 32 + g * 4 + t) * 4 + (i >> 1) * 2 + (e >> 2)];
        const int c = (w >> (4 * (((e >> 1) & 1) * 2 + (i & 1) + 4 * (e & 1)))) & 15;
        const long long at = b * a.ld_x + kb * kW4Block + k;
        const float x = a.x_f32 ? static_cast<const float*>(a.x)[at] : bf16_to_f(static_cast<const uint16_t*>(a.x)[at]);
        sum = fmaf((float)(c - z), x, sum);
      }
      y = fmaf(s, sum, y);
    }
  }
  put(a.out, a.out_f32, b * a.ld_out + v, y);
}

}  // namespace

cudaError_t launch_w4_pack(const W4PackArgs& a, cudaStream_t s) {
  const dim3 grid((unsigned)a.lay.tiles, (unsigned)(a.lay.blocks < 64 ? a.lay.blocks : 64));
  return launch_pdl(k_w4_pack, grid, dim3(kPackThreads), 0, s, a);
}

cudaError_t launch_w4_project(const W4Args& a, cudaStream_t s) {
  return launch_pdl(k_w4_project, dim3((unsigned)((a.V + 127) / 128), (unsigned)a.B), dim3(128), 0, s, a);
}

}  // namespace dels
