// 8-bit projection with block scales,
//   D[m, n] = sum_b sa[m, b] sw[n / 128, b] sum_{k in block b} a[m, k] w[n, k]   (+ bias[n]) (+ what D holds),
// a and w e4m3, blocks of 128 along K, fp32 accumulation.
#pragma once

#include <cuda_fp8.h>

#include "common.cuh"

namespace srm {
namespace g8 {

struct Args {
  int64_t M, N, K;             // K a multiple of 16
  const uint8_t* A; int64_t a_stride;
  const float* sa; int64_t sa_row, sa_blk;
  const uint8_t* W; int64_t w_stride;
  const float* sw; int64_t sw_row, sw_blk;
  const float* bias;           // [N] or nullptr
  int accumulate;              // D += (fp32 output only)
  void* out; int64_t out_stride;
  uint32_t* status;
};

__device__ __forceinline__ void unpack16(uint4 u, float (&f)[16]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[i >> 1] >> (16 * (i & 1))), __NV_E4M3);
    const float2 v = __half22float2(__half2(h));
    f[2 * i] = v.x; f[2 * i + 1] = v.y;
  }
}

// One output per thread: every product in fp32, a sum per block of 128.
template <typename OT>
__global__ void __launch_bounds__(256) gemm8_simple_kernel(const Args g) {
  pdl_trigger();
  pdl_wait();
  const int64_t n = (int64_t)blockIdx.x * 16 + (threadIdx.x & 15), m = (int64_t)blockIdx.y * 16 + (threadIdx.x >> 4);
  if (m >= g.M || n >= g.N) return;
  const uint8_t *a = g.A + m * g.a_stride, *w = g.W + n * g.w_stride;
  float acc = 0.f;
  for (int64_t b = 0; b * 128 < g.K; ++b) {
    const int64_t k1 = b * 128 + 128 < g.K ? b * 128 + 128 : g.K;
    float s = 0.f;
    for (int64_t k = b * 128; k < k1; k += 16) {
      float fa[16], fw[16];
      unpack16(__ldg(reinterpret_cast<const uint4*>(a + k)), fa);
      unpack16(__ldg(reinterpret_cast<const uint4*>(w + k)), fw);
#pragma unroll
      for (int i = 0; i < 16; ++i) s = fmaf(fa[i], fw[i], s);
    }
    acc = fmaf(g.sa[m * g.sa_row + b * g.sa_blk] * g.sw[n / 128 * g.sw_row + b * g.sw_blk], s, acc);
  }
  if (g.bias != nullptr) acc += g.bias[n];
  OT* out = static_cast<OT*>(g.out) + m * g.out_stride + n;
  if (g.accumulate) acc += to_float(*out);
  *out = from_float<OT>(acc);
}

}  // namespace g8
}  // namespace srm
