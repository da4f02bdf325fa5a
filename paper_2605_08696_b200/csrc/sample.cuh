// Token selection with each row's own temperature, top-k, top-p and min-p, from given random numbers.
//
// Per row, with w_i = exp((l_i - l_max) / T) and the order (logit descending, id ascending):
//   the first top_k of the order; of these the shortest prefix whose mass reaches top_p times their mass; of these the
//   tokens with w_i >= min_p; then the lowest id whose cumulative mass, ids ascending, exceeds u times the mass kept.
// What is kept is always a prefix of the order: every key above a border key, and at the border the lowest ids.
#pragma once

#include "common.cuh"

namespace srm {
namespace smp {

struct Args {
  int64_t R;
  int V;
  const void* logits; int64_t stride;
  const float* u;
  const float* temperature;    // each [R] or nullptr: 1, no limit, no limit, no limit
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  int32_t* tok;
  uint32_t* status;
};

constexpr float kLeastTemperature = 7.888609052210118e-31f;      // 2^-100; anything below counts as greedy

// Keys are ordered like the logits; 0 stands for a token that cannot be picked (minus infinity, NaN). (The zeros of both signs
// are one value.)
__device__ __forceinline__ uint32_t logit_key(float l) {
  const uint32_t u = __float_as_uint(l + 0.0f);
  return !(l > -INFINITY) ? 0u : (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float key_logit(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k); }

template <typename T> __device__ __forceinline__ float load_logit(const Args& p, int64_t row, int i) {
  return to_float(static_cast<const T*>(p.logits)[row * p.stride + i]);
}

// Weight of a token in 64 bits; l_max itself (infinite or not) has 1.
__device__ __forceinline__ double weight64(float l, float l_max, double inv_temp) {
  return l == l_max ? 1.0 : exp(((double)l - (double)l_max) * inv_temp);
}

struct BlockScratch { double d[32]; unsigned long long n[32]; };

// Sums over the block, the same order every time; all threads get them.
__device__ inline void block_sum(double& d, unsigned long long& n, BlockScratch& s) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    d += __shfl_xor_sync(0xffffffffu, d, o);
    n += __shfl_xor_sync(0xffffffffu, n, o);
  }
  __syncthreads();
  if (lane == 0) { s.d[warp] = d; s.n[warp] = n; }
  __syncthreads();
  d = 0.0; n = 0;
  for (int w = 0; w < warps; ++w) { d += s.d[w]; n += s.n[w]; }
}

// Count and mass of the keys >= t.
template <typename T>
__device__ inline void above(const Args& p, int64_t row, uint32_t t, float l_max, double inv_temp, double& mass, unsigned long long& count,
                             BlockScratch& s) {
  mass = 0.0; count = 0;
  for (int i = threadIdx.x; i < p.V; i += blockDim.x) {
    const float l = load_logit<T>(p, row, i);
    const uint32_t k = logit_key(l);
    if (k != 0u && k >= t) { mass += weight64(l, l_max, inv_temp); ++count; }
  }
  block_sum(mass, count, s);
}

constexpr int kSimpleThreads = 512;

template <typename T>
__global__ void __launch_bounds__(kSimpleThreads) sample_simple_kernel(const Args p) {
  pdl_trigger();
  pdl_wait();
  __shared__ BlockScratch sc;
  __shared__ uint32_t sh_key[kSimpleThreads / 32];
  __shared__ int sh_tok, sh_last;
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  // ---- largest key ----
  uint32_t kmax = 0;
  bool odd = false;
  for (int i = tid; i < p.V; i += blockDim.x) {
    const float l = load_logit<T>(p, row, i);
    odd |= !(l < INFINITY);
    kmax = max(kmax, logit_key(l));
  }
  if (odd) raise_status(p.status, kStatusNonFinite);
  kmax = __reduce_max_sync(0xffffffffu, kmax);
  if (lane == 0) sh_key[warp] = kmax;
  if (tid == 0) { sh_tok = 0x7fffffff; sh_last = -1; }
  __syncthreads();
  for (int w = 0; w < kSimpleThreads / 32; ++w) kmax = max(kmax, sh_key[w]);
  if (kmax == 0u) {                                  // nothing can be picked
    if (tid == 0) { raise_status(p.status, kStatusNonFinite); p.tok[row] = 0; }
    return;
  }
  const float l_max = key_logit(kmax);
  const float T0 = p.temperature != nullptr ? p.temperature[row] : 1.0f;
  const bool greedy = !(T0 >= kLeastTemperature);
  const double inv_temp = greedy ? 1.0 : 1.0 / (double)T0;
  int top_k = greedy ? 1 : p.top_k != nullptr ? p.top_k[row] : 0;
  if (top_k <= 0 || top_k > p.V) top_k = p.V;
  const float top_p = p.top_p != nullptr ? p.top_p[row] : 1.0f;
  const float mp = p.min_p != nullptr ? p.min_p[row] : 0.0f;
  const double min_p = mp > 0.0f ? (double)fminf(mp, 1.0f) : 0.0;
  double u = (double)p.u[row];
  u = u > 0.0 ? u : 0.0;

  // border: keys above `t` are kept, and at `t` the `m` lowest ids
  uint32_t t = 1u;
  unsigned long long m = ~0ull;
  double Z1, mass;
  unsigned long long count;
  above<T>(p, row, 1u, l_max, inv_temp, Z1, count, sc);
  if (count > (unsigned long long)top_k) {           // the top_k-th largest key, bit by bit
    uint32_t key = 0;
    for (int b = 31; b >= 0; --b) {
      above<T>(p, row, key | (1u << b), l_max, inv_temp, mass, count, sc);
      if (count >= (unsigned long long)top_k) key |= 1u << b;
    }
    t = key;
    above<T>(p, row, t + 1u, l_max, inv_temp, mass, count, sc);
    m = (unsigned long long)top_k - count;
    Z1 = mass + (double)m * weight64(key_logit(t), l_max, inv_temp);
  }
  if (top_p < 1.0f) {
    const double want = (double)top_p * Z1;
    uint32_t key = 0;                                // the largest key whose mass reaches `want`
    for (int b = 31; b >= 0; --b) {
      above<T>(p, row, key | (1u << b), l_max, inv_temp, mass, count, sc);
      if (count != 0 && (want <= 0.0 || mass >= want)) key |= 1u << b;
    }
    if (key > t || (key == t && key != 0u)) {
      above<T>(p, row, key + 1u, l_max, inv_temp, mass, count, sc);
      unsigned long long c = 1;
      const double w = weight64(key_logit(key), l_max, inv_temp);
      while (c < (key == t ? m : (unsigned long long)p.V) && mass + (double)c * w < want) ++c;
      t = key;
      m = c;
    }
  }
  // ---- draw: two ordered passes over the ids, the mass kept and then the place of u times it ----
  double Z = 0.0;
  for (int pass = 0; pass < 2; ++pass) {
    const double target = u * Z;
    double run = 0.0;
    unsigned long long ties = 0;
    for (int base = 0; base < p.V; base += kSimpleThreads) {
      const int i = base + tid;
      uint32_t k = 0;
      double w = 0.0;
      if (i < p.V) {
        const float l = load_logit<T>(p, row, i);
        k = logit_key(l);
        if (k >= t && k != 0u) w = weight64(l, l_max, inv_temp);
        if (!(w >= min_p)) { w = 0.0; k = 0; }
      }
      const bool tie = k != 0u && k == t;
      const uint32_t bal = __ballot_sync(0xffffffffu, tie);
      __syncthreads();
      if (lane == 0) sc.n[warp] = __popc(bal);
      __syncthreads();
      unsigned long long before = ties, all = ties;
      for (int q = 0; q < kSimpleThreads / 32; ++q) { if (q < warp) before += sc.n[q]; all += sc.n[q]; }
      before += __popc(bal & ((1u << lane) - 1u));
      ties = all;
      const bool kept = k > t || (tie && before < m);
      if (!kept) w = 0.0;
      double incl = w;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const double x = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += x;
      }
      __syncthreads();
      if (lane == 31) sc.d[warp] = incl;
      __syncthreads();
      double off = run;
      for (int q = 0; q < kSimpleThreads / 32; ++q) { if (q < warp) off += sc.d[q]; run += sc.d[q]; }
      if (pass == 1 && kept) {
        atomicMax(&sh_last, i);
        if (off + incl > target) atomicMin(&sh_tok, i);
      }
    }
    Z = run;
  }
  __syncthreads();
  if (tid == 0) p.tok[row] = sh_tok != 0x7fffffff ? sh_tok : sh_last;
}

}  // namespace smp
}  // namespace srm
