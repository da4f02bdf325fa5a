// Matrices in 8 bits (e4m3) with an fp32 scale per block of 128 columns: quantisation, and the RMS norm that writes its
// result that way. A block's scale is s = max(amax / 448, 2^-100) (448: the largest e4m3 value; the floor gives blocks of
// zeros a scale) and its values are q = e4m3(x / s), to nearest even, saturating. A NaN or infinity gives its block a
// scale that is none either, so that it reaches whatever reads the block.
#pragma once

#include <cuda_fp8.h>

#include "common.cuh"

namespace srm {
namespace q8 {

constexpr float kE4m3Max = 448.0f;
constexpr float kLeastScale = 7.888609052210118e-31f;      // 2^-100

// block scale of the largest magnitude among a block's values, given as the bits of its absolute value (as integers these are
// ordered like the values, with NaN above infinity)
__device__ __forceinline__ float block_scale(uint32_t amax_bits) {
  const float s = __uint_as_float(amax_bits) / kE4m3Max;
  return s < kLeastScale ? kLeastScale : s;                 // (a NaN stays)
}

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t abs_max4(float4 v) {
  return max(max(abs_bits(v.x), abs_bits(v.y)), max(abs_bits(v.z), abs_bits(v.w)));
}

// A block's divisor: x / s as x * (1 / s) and one correction by the remainder, which gives the quotient's own rounding. (The
// product alone is off by up to two roundings, and bf16 values over the scale of a bf16 maximum lie halfway between two codes
// often enough for that to show.) An infinite scale has no remainder.
struct Divisor {
  float inv, s;
  __device__ explicit Divisor(float scale) : inv(1.0f / scale), s(scale < INFINITY ? scale : 0.0f) {}
  __device__ __forceinline__ float operator()(float x) const {
    const float q = x * inv;
    return fmaf(-fmaf(q, s, -x), inv, q);            // (in this order a zero keeps its sign)
  }
};

// four values over their block's scale, as e4m3 bytes (the conversion of a NaN is the NaN code)
__device__ __forceinline__ uint32_t pack4(float4 v, const Divisor& d) {
  const __nv_fp8x2_storage_t lo = __nv_cvt_float2_to_fp8x2(make_float2(d(v.x), d(v.y)), __NV_SATFINITE, __NV_E4M3);
  const __nv_fp8x2_storage_t hi = __nv_cvt_float2_to_fp8x2(make_float2(d(v.z), d(v.w)), __NV_SATFINITE, __NV_E4M3);
  return (uint32_t)lo | ((uint32_t)hi << 16);
}

// Rounding of a sum to the stored type, and its store. (The conversions in common.cuh clamp to fp16's finite range, which is
// right for the cache and would hide an infinity or a NaN here.)
template <typename T> __device__ __forceinline__ float4 round4(float4 v);
template <> __device__ __forceinline__ float4 round4<float>(float4 v) { return v; }
template <> __device__ __forceinline__ float4 round4<bf16>(float4 v) {
  return make_float4(__bfloat162float(__float2bfloat16_rn(v.x)), __bfloat162float(__float2bfloat16_rn(v.y)),
                     __bfloat162float(__float2bfloat16_rn(v.z)), __bfloat162float(__float2bfloat16_rn(v.w)));
}
template <> __device__ __forceinline__ float4 round4<fp16>(float4 v) {
  return make_float4(__half2float(__float2half_rn(v.x)), __half2float(__float2half_rn(v.y)), __half2float(__float2half_rn(v.z)),
                     __half2float(__float2half_rn(v.w)));
}
__device__ __forceinline__ void store4(float* p, float4 v) { st4(p, v); }
__device__ __forceinline__ void store4(bf16* p, float4 v) { st4(p, v); }
__device__ __forceinline__ void store4(fp16* p, float4 v) {
  const __half2 a = __floats2half2_rn(v.x, v.y), b = __floats2half2_rn(v.z, v.w);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

// ---- RMS norm with the residual's addition --------------------------------------------------------------
struct NormArgs {
  int64_t R;
  int d;                       // multiple of 16
  const void* x; int64_t x_stride;
  const void* delta; int64_t delta_stride;      // nullptr: none
  const float* g;
  float eps;
  void* sum; int64_t sum_stride;                // nullptr: the sum is not stored
  uint8_t* q; int64_t q_stride;
  float* scale; int64_t scale_row, scale_blk;
};

// h = x + delta, rounded to x's type (what a later reader of the stored sum sees is what is normed); y = h / rms(h) * g.
// One block per row; the row stays in registers (NV groups of four channels per thread, a warp's 32 groups are one scale
// block), so memory is passed over once.
template <int NV, typename XT, typename DT>
__global__ void rms_norm_fp8_kernel(const NormArgs p) {
  pdl_trigger();
  pdl_wait();
  __shared__ float part[32];
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, warps = blockDim.x >> 5;
  const XT* x = static_cast<const XT*>(p.x) + row * p.x_stride;
  const int n4 = p.d >> 2;
  float4 v[NV];
  float ss = 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int i = j * blockDim.x + tid;
    v[j] = i < n4 ? ld4(x + 4 * i) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  if (p.delta != nullptr) {
    const DT* dl = static_cast<const DT*>(p.delta) + row * p.delta_stride;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int i = j * blockDim.x + tid;
      if (i < n4) {
        const float4 e = ld4(dl + 4 * i);
        v[j] = round4<XT>(make_float4(v[j].x + e.x, v[j].y + e.y, v[j].z + e.z, v[j].w + e.w));
        if (p.sum != nullptr) store4(static_cast<XT*>(p.sum) + row * p.sum_stride + 4 * i, v[j]);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < NV; ++j)
    ss += (v[j].x * v[j].x + v[j].y * v[j].y) + (v[j].z * v[j].z + v[j].w * v[j].w);
  ss = warp_sum(ss);
  if (warps > 1) {
    if (lane == 0) part[warp] = ss;
    __syncthreads();
    ss = warp_sum(lane < warps ? part[lane] : 0.f);
  }
  // (an infinite sum would leave zeros in every block but the infinity's own, and in all of them where only squares were too large)
  const float rstd = ss < INFINITY ? rsqrtf(ss / (float)p.d + p.eps) : __int_as_float(0x7fffffff);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int i = j * blockDim.x + tid;
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
    if (i < n4) {
      const float4 g = ldg4(p.g + 4 * i);
      y = make_float4(v[j].x * rstd * g.x, v[j].y * rstd * g.y, v[j].z * rstd * g.z, v[j].w * rstd * g.w);
    }
    const float s = block_scale(__reduce_max_sync(0xffffffffu, abs_max4(y)));
    if (i < n4) {
      *reinterpret_cast<uint32_t*>(p.q + row * p.q_stride + 4 * i) = pack4(y, Divisor(s));
      if (lane == 0) p.scale[row * p.scale_row + (i >> 5) * p.scale_blk] = s;
    }
  }
}

// ---- quantisation -----------------------------------------------------------------------------------------
struct QuantArgs {
  int64_t R;
  int64_t K;                   // multiple of 16
  const void* x; int64_t x_stride;
  uint8_t* q; int64_t q_stride;
  float* scale; int64_t scale_row, scale_blk;
};

constexpr int kQuantThreads = 256;

// Eight values of a row as they are stored (16 bytes, or 32 for fp32): they wait for their block's maximum in that form, in half the
// registers that floats would take.
template <typename T> struct Eight;
template <> struct Eight<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = ld4(p); b = ld4(p + 4); }
  __device__ __forceinline__ void clear() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ uint32_t largest() const { return max(abs_max4(a), abs_max4(b)); }
  __device__ __forceinline__ float4 low() const { return a; }
  __device__ __forceinline__ float4 high() const { return b; }
};
// (of two 16-bit floats in a word, magnitudes as integers: both at once)
template <typename T> struct EightHalves {
  uint4 u;
  __device__ __forceinline__ void load(const T* p) { u = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void clear() { u = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ uint32_t largest() const {
    const uint32_t m = __vmaxu2(__vmaxu2(u.x & 0x7fff7fffu, u.y & 0x7fff7fffu), __vmaxu2(u.z & 0x7fff7fffu, u.w & 0x7fff7fffu));
    const unsigned short h = (unsigned short)max(m & 0xffffu, m >> 16);
    return __float_as_uint(to_float(*reinterpret_cast<const T*>(&h)));
  }
  __device__ __forceinline__ float4 low() const { return ld4(reinterpret_cast<const T*>(&u)); }
  __device__ __forceinline__ float4 high() const { return ld4(reinterpret_cast<const T*>(&u) + 4); }
};
template <> struct Eight<bf16> : EightHalves<bf16> {};
template <> struct Eight<fp16> : EightHalves<fp16> {};

template <typename T>
__device__ __forceinline__ void put8(uint8_t* q, const Eight<T>& v, const Divisor& by) {
  *reinterpret_cast<uint2*>(q) = make_uint2(pack4(v.low(), by), pack4(v.high(), by));
}

// 1 x 128 blocks: half a warp per block, its maximum by shuffles. Bound by the bytes it moves; every value is read once.
template <typename XT>
__global__ void __launch_bounds__(kQuantThreads) quant_rows_kernel(const QuantArgs p) {
  pdl_trigger();
  pdl_wait();
  const int half = threadIdx.x & 15;
  const int64_t kb = (p.K + 127) / 128, n = p.R * kb;
  const int64_t w = (int64_t)blockIdx.x * (kQuantThreads / 16) + (threadIdx.x >> 4);
  const int64_t row = w < n ? w / kb : 0, b = w < n ? w - row * kb : 0, c = b * 128 + 8 * half;
  const bool in = w < n && c < p.K;
  Eight<XT> v;
  if (in) v.load(static_cast<const XT*>(p.x) + row * p.x_stride + c);
  else v.clear();
  uint32_t m = v.largest();
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
  const float s = block_scale(m);
  if (in) put8(p.q + row * p.q_stride + c, v, Divisor(s));
  if (w < n && half == 0) p.scale[row * p.scale_row + b * p.scale_blk] = s;
}

// 128 x 128 blocks: a thread block per block, 16 rows at a time, all in registers until the maximum is known. (Four values per thread
// and load, as floats: 3 blocks per SM and 44 us for 32000 x 1536 from bf16, 147 MB.)
template <typename XT>
__global__ void __launch_bounds__(kQuantThreads) quant_tiles_kernel(const QuantArgs p) {
  pdl_trigger();
  pdl_wait();
  constexpr int kRows = kQuantThreads / 16, kSteps = 128 / kRows;
  __shared__ uint32_t part[kQuantThreads / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t kb = (p.K + 127) / 128;
  const int64_t rb = blockIdx.x / kb, b = blockIdx.x - rb * kb, c = b * 128 + 8 * (threadIdx.x & 15), r0 = rb * 128 + (threadIdx.x >> 4);
  const bool in = c < p.K;
  Eight<XT> v[kSteps];
#pragma unroll
  for (int j = 0; j < kSteps; ++j) {
    const int64_t r = r0 + j * kRows;
    if (in && r < p.R) v[j].load(static_cast<const XT*>(p.x) + r * p.x_stride + c);
    else v[j].clear();
  }
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < kSteps; ++j) m = max(m, v[j].largest());
  m = __reduce_max_sync(0xffffffffu, m);
  if (lane == 0) part[warp] = m;
  __syncthreads();
  m = __reduce_max_sync(0xffffffffu, part[lane & (kQuantThreads / 32 - 1)]);
  const float s = block_scale(m);
  const Divisor by(s);
#pragma unroll
  for (int j = 0; j < kSteps; ++j) {
    const int64_t r = r0 + j * kRows;
    if (in && r < p.R) put8(p.q + r * p.q_stride + c, v[j], by);
  }
  if (threadIdx.x == 0) p.scale[rb * p.scale_row + b * p.scale_blk] = s;
}

}  // namespace q8
}  // namespace srm
