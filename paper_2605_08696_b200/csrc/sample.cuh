// Token selection with each row's own temperature, top-k, top-p and min-p, from given random numbers.
//
// Per row, with w_i = exp((l_i - l_max) / T) and the order (logit descending, id ascending):
//   the first top_k of the order; of these the shortest prefix whose mass reaches top_p times their mass; of these the
//   tokens with w_i >= min_p; then the lowest id whose cumulative mass, ids ascending, exceeds u times the mass kept.
// What is kept is always a prefix of the order.
//
// A row is read once: its weights stay in the registers of one block (32 per thread; a cluster of blocks where the vocabulary is
// longer than 32768) as fp32 values whose error is bounded (kSlack). Borders are searched on those: a threshold probe costs
// three instructions per element and a reduction. The few tokens that the bounds leave undecided (at most kCap of them, or all
// that can be kept when these are so few) go to shared memory, where they are sorted and weighed in 64 bits; sums that a decision
// depends on more closely than the bounds allow are formed again in 64 bits from the logits, in a second read that finds them in
// L2. So the token is the one that 64-bit arithmetic gives, and nearly all of the arithmetic is not 64-bit.
#pragma once

#include <cooperative_groups.h>

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

constexpr int kWarpIds = 1024;                   // consecutive ids of a warp: 8 groups of 128, four per lane
constexpr int kMaxWarps = 32;
constexpr int kCap = 1024;                       // tokens that are sorted
constexpr int kMaxRanks = 8;
// Bound on the relative error of an fp32 weight above kLeast and of sums of them: the difference to the maximum, the factor
// 1 / (T ln 2) and their product are rounded once each, which moves a weight 2^x by 3 |x| 2^-24 ln 2 (|x| <= 80: 1.0e-5), ex2 by
// 2^-22, a thread's sum of 32 and two levels of five by 42 roundings (2.5e-6).
constexpr float kSlack = 2e-5f;
constexpr float kLeast = 8.271806125530277e-25f; // 2^-80: all weights below it together are under 64-bit rounding (2^18 ids)
constexpr int kProbes = 40;

// 2^y for y <= 0 in 64 bits: the power of two by the exponent field, the rest by the series of exp to the 12th power of an
// argument of at most ln 2 / 2 (the remainder is under 2e-16).
__device__ __forceinline__ double pow2_64(double y) {
  if (!(y > -1000.0)) return 0.0;
  const double n = rint(y), t = (y - n) * 0.693147180559945309417;
  double s = 1.0 / 479001600;
  s = fma(s, t, 1.0 / 39916800); s = fma(s, t, 1.0 / 3628800); s = fma(s, t, 1.0 / 362880); s = fma(s, t, 1.0 / 40320);
  s = fma(s, t, 1.0 / 5040); s = fma(s, t, 1.0 / 720); s = fma(s, t, 1.0 / 120); s = fma(s, t, 1.0 / 24); s = fma(s, t, 1.0 / 6);
  s = fma(s, t, 0.5); s = fma(s, t, 1.0); s = fma(s, t, 1.0);
  return __hiloint2double(__double2hiint(s) + ((int)n << 20), __double2loint(s));
}

// Weight of a token in 64 bits; l_max itself (infinite or not) has 1. `rate`: 1 / (T ln 2).
__device__ __forceinline__ double weight64(float l, float l_max, double rate) {
  return l == l_max ? 1.0 : pow2_64(((double)l - (double)l_max) * rate);
}

__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ double warp_sum64(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Sortable word of a token: ascending order is (logit descending, id ascending).
__device__ __forceinline__ unsigned long long word_of(float l, int id) {
  return ((unsigned long long)(~logit_key(l)) << 32) | (uint32_t)id;
}
__device__ __forceinline__ float word_logit(unsigned long long w) { return key_logit(~(uint32_t)(w >> 32)); }

// Parameters of a row, the same in every thread.
struct RowArgs {
  int64_t row;
  float l_max;
  double rate;                 // 1 / (T ln 2)
  int top_k;                   // 1 .. V
  double top_p, min_p;         // top_p >= 1, min_p = 0: no effect
  double u;
};

struct Scratch {
  unsigned long long cand[kCap];
  double weight[kCap], run[kCap];      // of the sorted candidates: weights, and running sums of them
  double warp_sum[kMaxRanks * kMaxWarps];
  double d[2][kMaxWarps], rank_d[2][kMaxRanks];
  float f[2][kMaxWarps], rank_f[2][kMaxRanks];
  uint32_t n[2][kMaxWarps], rank_n[2][kMaxRanks];
  uint32_t count;
  int keep, unsure, tok, last;
};

// What a block (or, with CL, a cluster) knows and does together. Reductions use two sets of places in turn, so one barrier each is
// enough; their order is fixed, so results are the same every time, in every thread.
template <bool CL>
struct Group {
  Scratch& s;
  int tid, lane, warp, warps, rank, ranks;
  int turn = 0;

  __device__ void sync_all() {
    if (CL) cooperative_groups::this_cluster().sync();
    else __syncthreads();
  }
  template <typename V> __device__ void to_ranks(V* place, V v) {        // thread 0: v to place[rank] of every rank
    if (CL)
      for (int r = 0; r < ranks; ++r) cooperative_groups::this_cluster().map_shared_rank(place, r)[rank] = v;
  }
  __device__ float max_of(float v) {
    const int b = turn;
    turn ^= 1;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    if (lane == 0) s.f[b][warp] = v;
    __syncthreads();
    v = lane < warps ? s.f[b][lane] : -INFINITY;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    if (CL) {
      if (tid == 0) to_ranks(s.rank_f[b], v);
      sync_all();
      for (int r = 0; r < ranks; ++r) v = fmaxf(v, s.rank_f[b][r]);
    }
    return v;
  }
  __device__ uint32_t min_of(uint32_t v) {
    const int b = turn;
    turn ^= 1;
    v = __reduce_min_sync(0xffffffffu, v);
    if (lane == 0) s.n[b][warp] = v;
    __syncthreads();
    v = __reduce_min_sync(0xffffffffu, lane < warps ? s.n[b][lane] : 0xffffffffu);
    if (CL) {
      if (tid == 0) to_ranks(s.rank_n[b], v);
      sync_all();
      for (int r = 0; r < ranks; ++r) v = min(v, s.rank_n[b][r]);
    }
    return v;
  }
  // a sum of masses and one of counts
  __device__ void add(float& m, uint32_t& n) {
    const int b = turn;
    turn ^= 1;
    m = srm::warp_sum(m);
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) { s.f[b][warp] = m; s.n[b][warp] = n; }
    __syncthreads();
    m = srm::warp_sum(lane < warps ? s.f[b][lane] : 0.f);
    n = __reduce_add_sync(0xffffffffu, lane < warps ? s.n[b][lane] : 0u);
    if (CL) {
      if (tid == 0) { to_ranks(s.rank_f[b], m); to_ranks(s.rank_n[b], n); }
      sync_all();
      m = 0.f;
      n = 0u;
      for (int r = 0; r < ranks; ++r) { m += s.rank_f[b][r]; n += s.rank_n[b][r]; }
    }
  }
  __device__ double add64(double m) {
    const int b = turn;
    turn ^= 1;
    m = warp_sum64(m);
    if (lane == 0) s.d[b][warp] = m;
    __syncthreads();
    m = warp_sum64(lane < warps ? s.d[b][lane] : 0.0);
    if (CL) {
      if (tid == 0) to_ranks(s.rank_d[b], m);
      sync_all();
      m = 0.0;
      for (int r = 0; r < ranks; ++r) m += s.rank_d[b][r];
    }
    return m;
  }
};

__device__ inline void sort_words(unsigned long long* w, int n, int tid, int threads) {
  int P = 2;
  while (P < n) P <<= 1;
  for (int i = n + tid; i < P; i += threads) w[i] = ~0ull;
  __syncthreads();
  for (int size = 2; size <= P; size <<= 1)
    for (int stride = size >> 1; stride > 0; stride >>= 1) {
      for (int i = tid; i < P / 2; i += threads) {
        const int a = 2 * i - (i & (stride - 1)), b = a + stride;
        const unsigned long long x = w[a], y = w[b];
        if ((x > y) == ((a & size) == 0)) { w[a] = y; w[b] = x; }
      }
      __syncthreads();
    }
}

// run[i] = d[0] + .. + d[i] for i < n: each thread a run of consecutive places, in a fixed order.
__device__ inline void running_sums(const double* d, double* run, int n, int tid, int threads, double* part) {
  const int per = (n + threads - 1) / threads, i0 = min(n, tid * per), i1 = min(n, i0 + per);
  const int lane = tid & 31, warp = tid >> 5;
  double incl = 0.0;
  for (int i = i0; i < i1; ++i) incl += d[i];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const double x = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += x;
  }
  double at = __shfl_up_sync(0xffffffffu, incl, 1);
  if (lane == 0) at = 0.0;
  __syncthreads();
  if (lane == 31) part[warp] = incl;
  __syncthreads();
  for (int w = 0; w < warp; ++w) at += part[w];
  for (int i = i0; i < i1; ++i) {
    at += d[i];
    run[i] = at;
  }
  __syncthreads();
}

// ---- rows whose border the search cannot close in on --------------------------------------------------------------
// (Thousands of tokens with one and the same weight.) One block, all in 64 bits: the border key bit by bit, a pass over the row
// each, then the ids in order.
template <typename T>
__device__ __noinline__ int slow_row(const Args& p, const RowArgs& a, Scratch& s) {
  Group<false> g{s, (int)threadIdx.x, (int)threadIdx.x & 31, (int)threadIdx.x >> 5, (int)blockDim.x >> 5, 0, 1};
  const int threads = blockDim.x;
  double mass;
  uint32_t count;
  auto above = [&](uint32_t t) {
    mass = 0.0;
    count = 0;
    for (int i = g.tid; i < p.V; i += threads) {
      const float l = load_logit<T>(p, a.row, i);
      const uint32_t k = logit_key(l);
      if (k != 0u && k >= t) { mass += weight64(l, a.l_max, a.rate); ++count; }
    }
    float none = 0.f;
    mass = g.add64(mass);
    g.add(none, count);
  };
  uint32_t t = 1u, m = 0xffffffffu;                  // keys above t are kept, and at t the m lowest ids
  above(1u);
  double Z1 = mass;
  if (count > (uint32_t)a.top_k) {
    uint32_t key = 0;
    for (int b = 31; b >= 0; --b) {
      above(key | (1u << b));
      if (count >= (uint32_t)a.top_k) key |= 1u << b;
    }
    t = key;
    above(t + 1u);
    m = (uint32_t)a.top_k - count;
    Z1 = mass + (double)m * weight64(key_logit(t), a.l_max, a.rate);
  }
  if (a.top_p < 1.0) {
    const double want = a.top_p * Z1;
    uint32_t key = 0;                                // the largest key whose mass reaches `want`
    for (int b = 31; b >= 0; --b) {
      above(key | (1u << b));
      if (count != 0 && (want <= 0.0 || mass >= want)) key |= 1u << b;
    }
    if (key >= t) {
      above(key + 1u);
      const double w = weight64(key_logit(key), a.l_max, a.rate);
      const uint32_t most = key == t ? m : (uint32_t)p.V;
      // the first c >= 1 with mass + c w >= want
      double c = w > 0.0 ? ceil((want - mass) / w) : 1.0;
      c = c < 1.0 ? 1.0 : c;
      while (c > 1.0 && mass + (c - 1.0) * w >= want) c -= 1.0;
      while (c < (double)most && mass + c * w < want) c += 1.0;
      t = key;
      m = c < (double)most ? (uint32_t)c : most;
    }
  }
  double Z = 0.0;
  __syncthreads();
  if (g.tid == 0) { s.tok = 0x7fffffff; s.last = -1; }
  for (int pass = 0; pass < 2; ++pass) {
    const double target = a.u * Z;
    double run = 0.0;
    uint32_t ties = 0;
    for (int base = 0; base < p.V; base += threads) {
      const int i = base + g.tid;
      uint32_t k = 0;
      double w = 0.0;
      if (i < p.V) {
        const float l = load_logit<T>(p, a.row, i);
        k = logit_key(l);
        if (k >= t && k != 0u) w = weight64(l, a.l_max, a.rate);
        if (!(w >= a.min_p)) { w = 0.0; k = 0; }
      }
      const bool tie = k != 0u && k == t;
      const uint32_t bal = __ballot_sync(0xffffffffu, tie);
      __syncthreads();
      if (g.lane == 0) s.n[0][g.warp] = __popc(bal);
      __syncthreads();
      uint32_t before = ties;
      for (int q = 0; q < g.warps; ++q) { if (q < g.warp) before += s.n[0][q]; ties += s.n[0][q]; }
      before += __popc(bal & ((1u << g.lane) - 1u));
      const bool kept = k > t || (tie && before < m);
      double incl = kept ? w : 0.0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const double x = __shfl_up_sync(0xffffffffu, incl, o);
        if (g.lane >= o) incl += x;
      }
      if (g.lane == 31) s.d[0][g.warp] = incl;
      __syncthreads();
      double off = run;
      for (int q = 0; q < g.warps; ++q) { if (q < g.warp) off += s.d[0][q]; run += s.d[0][q]; }
      if (pass == 1 && kept) {
        atomicMax(&s.last, i);
        if (off + incl > target) atomicMin(&s.tok, i);
      }
    }
    Z = run;
  }
  __syncthreads();
  return s.tok != 0x7fffffff ? s.tok : s.last;
}

// ---- the kernel -----------------------------------------------------------------------------------------------------
template <typename T, bool CL>
__global__ void __launch_bounds__(kMaxWarps * 32) sample_kernel(const Args p, const int per_rank) {
  pdl_trigger();
  __shared__ Scratch s;
  Group<CL> g{s, (int)threadIdx.x, (int)threadIdx.x & 31, (int)threadIdx.x >> 5, (int)blockDim.x >> 5, CL ? (int)blockIdx.x : 0, CL ? (int)gridDim.x : 1};
  const int threads = blockDim.x;
  const int64_t row = CL ? blockIdx.y : blockIdx.x;
  Scratch& lead = *(CL ? cooperative_groups::this_cluster().map_shared_rank(&s, 0) : &s);      // the rank that keeps the candidates
  const int id0 = g.rank * per_rank + g.warp * kWarpIds, end = min(p.V, (g.rank + 1) * per_rank);
  const T* lr = static_cast<const T*>(p.logits) + row * p.stride;
  pdl_wait();

  // ---- the row into registers: element (j, e) of a lane is id id0 + 128 j + 4 lane + e ----
  float w[32];
  bool odd = false;
  if (reinterpret_cast<uintptr_t>(lr) % (4 * sizeof(T)) == 0) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int i = id0 + 128 * j + 4 * g.lane;
      float4 v = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
      if (i + 3 < end) v = ld4(lr + i);
      else if (i < end) {
        v.x = to_float(lr[i]);
        if (i + 1 < end) v.y = to_float(lr[i + 1]);
        if (i + 2 < end) v.z = to_float(lr[i + 2]);
      }
      w[4 * j] = v.x; w[4 * j + 1] = v.y; w[4 * j + 2] = v.z; w[4 * j + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      const int i = id0 + 128 * (j >> 2) + 4 * g.lane + (j & 3);
      w[j] = i < end ? to_float(lr[i]) : -INFINITY;
    }
  }
  RowArgs a;
  a.row = row;
  const float T0 = p.temperature != nullptr ? p.temperature[row] : 1.0f;
  const int k0 = p.top_k != nullptr ? p.top_k[row] : 0;
  const float p0 = p.top_p != nullptr ? p.top_p[row] : 1.0f, q0 = p.min_p != nullptr ? p.min_p[row] : 0.0f, u0 = p.u[row];
  a.top_k = k0 <= 0 || k0 > p.V ? p.V : k0;
  a.top_p = p0 < 1.0f ? (double)fmaxf(p0, 0.0f) : 1.0;
  a.min_p = q0 > 0.0f ? (double)fminf(q0, 1.0f) : 0.0;
  a.u = u0 > 0.0f ? (double)u0 : 0.0;
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    odd |= !(w[i] < INFINITY);
    w[i] = w[i] > -INFINITY ? w[i] : -INFINITY;      // (a NaN masks its token)
    top = fmaxf(top, w[i]);
  }
  if (odd) raise_status(p.status, kStatusNonFinite);
  a.l_max = g.max_of(top);
  if (a.l_max == -INFINITY) {                        // nothing can be picked
    if (g.tid == 0 && g.rank == 0) { raise_status(p.status, kStatusNonFinite); p.tok[row] = 0; }
    if (CL) g.sync_all();
    return;
  }
  auto id_of = [&](int i) { return id0 + 128 * (i >> 2) + 4 * g.lane + (i & 3); };
  if (!(T0 >= kLeastTemperature) || a.top_k == 1 || a.top_p <= 0.0) {      // the first of the order
    uint32_t best = 0xffffffffu;
#pragma unroll
    for (int i = 31; i >= 0; --i) best = w[i] == a.l_max ? (uint32_t)id_of(i) : best;
    best = g.min_of(best);
    if (g.tid == 0 && g.rank == 0) p.tok[row] = (int)best;
    if (CL) g.sync_all();
    return;
  }
  a.rate = 1.4426950408889634074 / (double)T0;
  bool slow = !(T0 <= 1e30f);
  const float rate = (float)fmin(a.rate, 3e38);
  // ---- weights ----
  float mass = 0.f;
  uint32_t count = 0;
  const bool need_p = a.top_p < 1.0;
  bool need_k = a.top_k < p.V;
  const float least = need_k && need_p ? kLeast : fmaxf(kLeast, (float)a.min_p * (1.0f - kSlack));
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    w[i] = w[i] == a.l_max ? 1.0f : ex2((w[i] - a.l_max) * rate);
    w[i] = w[i] >= kLeast ? w[i] : 0.0f;             // (and an infinite maximum leaves zeros)
    mass += w[i];
    count += w[i] >= least ? 1u : 0u;
  }
  g.add(mass, count);
  const float Z = mass;                              // of the whole row
  const uint32_t in_all = count;

  auto probe = [&](float t) {
    mass = 0.f;
    count = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      mass += w[i] >= t ? w[i] : 0.f;
      count += w[i] >= t ? 1u : 0u;
    }
    g.add(mass, count);
  };

  // ---- thresholds lo < hi: {w >= lo} holds all that is kept, all of {w >= hi} is kept; n_*, m_* their counts and masses ----
  float lo = least, hi = 2.0f, m_lo = Z, m_hi = 0.f;
  uint32_t n_lo = in_all, n_hi = 0;
  // Narrows [lo, hi) to at most kCap tokens, or down to the first kCap of the order (hi = 2). by_count: the border is the want_n-th
  // token; else where the mass reaches want_m.
  auto search = [&](bool by_count, uint32_t want_n, float want_m) {
    const float sure = want_m * (1.0f + kSlack) + Z * kSlack, unsure = want_m * (1.0f - kSlack) - Z * kSlack;
    uint32_t between_lo = 0, between_hi = 0;         // bits of thresholds that are neither
    for (int it = 0; it < kProbes; ++it) {
      if (n_lo <= (uint32_t)kCap) { hi = 2.0f; n_hi = 0; m_hi = 0.f; return true; }
      if (n_lo - n_hi <= (uint32_t)kCap && (n_hi > (uint32_t)kCap / 2 || it > 12)) return true;
      const uint32_t b_lo = __float_as_uint(lo), b_hi = __float_as_uint(hi);
      uint32_t b;
      if (between_lo != 0u) {
        b = (it & 1) ? b_lo + (between_lo - b_lo) / 2 : between_hi + (b_hi - between_hi) / 2;
      } else if (hi > 1.5f) {                        // nothing known above: down from 2^-6 in steps that double
        b = it == 0 && lo < 0.0078125f ? __float_as_uint(0.015625f) : b_lo + (b_hi - b_lo) / 2;
      } else if (lo <= least && lo < 1e-12f) {       // nothing known below
        const uint32_t d = __float_as_uint(1.0f) - b_hi;
        b = max(b_hi - max(d, 1u << 24), b_lo + (b_hi - b_lo) / 8);
      } else {                                       // by interpolation between the two, or halfway, in turn
        float f = by_count ? ((float)want_n - (float)n_hi) / ((float)n_lo - (float)n_hi) : (want_m - m_hi) / (m_lo - m_hi);
        f = (it & 1) ? 0.5f : fminf(fmaxf(f, 0.1f), 0.9f);
        b = b_hi - (uint32_t)((float)(b_hi - b_lo) * f);
      }
      if (b <= b_lo || b >= b_hi) break;
      const float t = __uint_as_float(b);
      probe(t);
      const bool enough = by_count ? count >= want_n : mass >= sure, few = by_count ? count < want_n : mass < unsure;
      if (enough) { lo = t; n_lo = count; m_lo = mass; if (between_lo != 0u && between_lo <= b) between_lo = between_hi = 0u; }
      else if (few) { hi = t; n_hi = count; m_hi = mass; if (between_hi != 0u && between_hi >= b) between_lo = between_hi = 0u; }
      else {
        between_lo = between_lo == 0u ? b : min(between_lo, b);
        between_hi = max(between_hi, b);
      }
    }
    return n_lo - n_hi <= (uint32_t)kCap;
  };
  // The tokens of [lo, hi) as sorted words with weights and running sums, in the leading rank.
  int n = 0;
  auto gather = [&]() {
    if (g.tid == 0) s.count = 0;
    g.sync_all();
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (w[i] >= lo && w[i] < hi) {
        const uint32_t at = atomicAdd(&lead.count, 1u);
        if (at < (uint32_t)kCap) lead.cand[at] = (unsigned long long)id_of(i);
      }
    g.sync_all();
    if (g.rank != 0) return;
    n = (int)min(s.count, (uint32_t)kCap);
    for (int i = g.tid; i < n; i += threads) s.cand[i] = word_of(to_float(lr[s.cand[i]]), (int)s.cand[i]);
    __syncthreads();
    sort_words(s.cand, n, g.tid, threads);
    for (int i = g.tid; i < n; i += threads) s.weight[i] = weight64(word_logit(s.cand[i]), a.l_max, a.rate);
    __syncthreads();
    running_sums(s.weight, s.run, n, g.tid, threads, s.d[0]);
  };
  // Sums in 64 bits over the row's own logits: of all weights, and of those at or above hi (also per warp, in the leading rank).
  double all64 = 0.0, above64 = 0.0;
  auto weigh = [&](bool whole) {
    double x = 0.0, y = 0.0;
#pragma unroll 4
    for (int i = 0; i < 32; ++i) {
      const int id = id_of(i);
      if (id >= end) continue;
      const float l = to_float(lr[id]);
      if (!(l > -INFINITY)) continue;
      const float wf = l == a.l_max ? 1.0f : ex2((l - a.l_max) * rate);
      const bool over = wf >= hi && wf >= kLeast;
      if (!over && !whole) continue;
      const double v = weight64(l, a.l_max, a.rate);
      x += v;
      y += over ? v : 0.0;
    }
    y = warp_sum64(y);
    if (g.lane == 0) lead.warp_sum[id0 / kWarpIds] = y;
    above64 = g.add64(g.lane == 0 ? y : 0.0);
    if (whole) all64 = g.add64(x);
  };
  // How many of the gathered tokens are kept (leading rank). k_left: places that top_k leaves them; want: the mass that ends the
  // nucleus, counted from `before` on; limit: only words up to it. unsure: how far `want` may be off.
  auto decide = [&](int k_left, bool by_mass, double want, double before, unsigned long long limit, double off, bool floor_p, int* unsure) {
    if (g.tid == 0) { s.keep = 0; s.unsure = 0; }
    __syncthreads();
    int mine = 0, doubt = 0;
    for (int i = g.tid; i < n; i += threads) {
      const double b = before + (i > 0 ? s.run[i - 1] : 0.0);
      const bool in = i < k_left && s.cand[i] <= limit && (!floor_p || s.weight[i] >= a.min_p);
      const bool first = i == 0 && before == 0.0;
      mine += in && (!by_mass || first || b < want) ? 1 : 0;
      doubt |= by_mass && in && !first && fabs(b - want) <= off ? 1 : 0;
    }
    if (mine) atomicAdd(&s.keep, mine);
    if (doubt) atomicOr(&s.unsure, 1);
    __syncthreads();
    const int keep = s.keep;
    if (unsure != nullptr) *unsure = s.unsure;
    __syncthreads();
    return keep;
  };

  int keep = 0;
  unsigned long long border = ~0ull;                 // words up to it are kept
  double mass_k = -1.0;                              // mass of the first top_k, where a list gave it
  if (!slow && need_k && in_all > (uint32_t)a.top_k && in_all > (uint32_t)kCap) {
    bool found = false;
    if (!CL && a.top_k <= 256 && 2 * a.top_k <= threads) {
      // The top_k-th largest of the threads' maxima, 16 bits of it: at least top_k weights are as large, and few more.
      float mx = 0.f;
#pragma unroll
      for (int i = 0; i < 32; ++i) mx = fmaxf(mx, w[i]);
      const uint32_t bits = __float_as_uint(mx);
      uint32_t t = 0;
      for (int b = 29; b >= 14; --b)
        if (__syncthreads_count(bits >= (t | (1u << b))) >= a.top_k) t |= 1u << b;
      const float tf = __uint_as_float(t);
      if (tf > lo) {
        probe(tf);
        if (count <= (uint32_t)kCap && count >= (uint32_t)a.top_k) { lo = tf; n_lo = count; m_lo = mass; found = true; }
      }
    }
    if (!found) found = search(true, (uint32_t)a.top_k, 0.f);
    slow = !found;
    if (found && hi < 1.5f && need_p) {
      // Too many for one list: the border of top_k first, and the mass inside it
      gather();
      weigh(false);
      double info[2] = {0.0, 0.0};
      if (g.rank == 0) {
        keep = decide(a.top_k - (int)n_hi, false, 0.0, above64, ~0ull, 0.0, false, nullptr);
        info[0] = above64 + s.run[keep - 1];
        if (CL && g.tid == 0) s.d[0][0] = info[0], s.run[0] = __longlong_as_double((long long)s.cand[keep - 1]);
        border = s.cand[keep - 1];
      }
      if (CL) {
        g.sync_all();
        info[0] = lead.d[0][0];
        border = (unsigned long long)__double_as_longlong(lead.run[0]);
        g.sync_all();
      }
      mass_k = info[0];
      hi = 2.0f; n_hi = 0; m_hi = 0.f;
      slow = !search(false, 0, (float)(a.top_p * mass_k));
      need_k = false;
    }
  } else if (need_k && in_all <= (uint32_t)a.top_k) {
    need_k = false;                                  // top_k ends behind all weights that count
  }
  bool k_by_list = need_k && !slow, by_mass = need_p;      // the list holds the border of top_k, of the nucleus
  if (!slow && !k_by_list && mass_k < 0.0 && in_all > (uint32_t)kCap) {
    if (need_p) {
      const float want = (float)a.top_p * Z;
      // (min_p may end the kept tokens above the nucleus' border: then it alone decides)
      probe(least);
      if (mass < want * (1.0f - kSlack) - Z * kSlack) {
        hi = fmaxf(least, (float)a.min_p * (1.0f + 2.0f * kSlack));
        probe(hi);
        n_hi = count;
        slow = n_lo - n_hi > (uint32_t)kCap;
      } else {
        m_lo = mass;
        slow = !search(false, 0, want);
      }
    } else {
      hi = a.min_p > 0.0 ? (float)a.min_p * (1.0f + 2.0f * kSlack) : kLeast;
      if (a.min_p > 0.0) {
        probe(hi);
        n_hi = count;
        slow = n_lo - n_hi > (uint32_t)kCap;
      } else {
        lo = hi;                                     // everything is kept: no list
        n_hi = n_lo;
      }
    }
  }
  if (!slow && a.min_p > 0.0 && hi < (float)a.min_p * (1.0f + 2.0f * kSlack)) {
    // not all above the border has min_p: it ends the kept tokens by itself, unless both lie within the bounds
    const float t = (float)a.min_p * (1.0f - 2.0f * kSlack);
    slow = hi > t;
    if (!slow) {
      k_by_list = by_mass = false;
      border = ~0ull;
      lo = t;
      probe(lo);
      n_lo = count;
      hi = 2.0f;
      n_hi = 0;
      if (n_lo > (uint32_t)kCap) {
        hi = (float)a.min_p * (1.0f + 2.0f * kSlack);
        probe(hi);
        n_hi = count;
        slow = n_lo - n_hi > (uint32_t)kCap;
      }
    }
  }
  if (slow) {
    if (CL) g.sync_all();
    if (g.rank == 0) {
      const int tok = slow_row<T>(p, a, s);
      if (g.tid == 0) p.tok[row] = tok;
    }
    return;
  }
  const bool whole_list = hi > 1.5f;
  gather();
  if (!whole_list) weigh(by_mass && mass_k < 0.0);
  // ---- the border, and which of the gathered tokens are kept ----
  if (g.rank == 0) {
    const int k_left = k_by_list ? a.top_k - (int)n_hi : n;
    if (k_by_list && by_mass && whole_list) mass_k = s.run[min(k_left, n) - 1];
    const double total = mass_k >= 0.0 ? mass_k : !whole_list ? all64 : (double)Z;
    const bool rough = by_mass && mass_k < 0.0 && whole_list;
    int doubt = 0;
    keep = decide(k_left, by_mass, a.top_p * total, whole_list ? 0.0 : above64, border, rough ? 2.0 * kSlack * Z : 0.0, a.min_p > 0.0, &doubt);
    if (CL && g.tid == 0) s.keep = doubt;
    if (CL) __syncthreads();
    if (!CL && doubt) {                              // the fp32 total is not enough
      weigh(true);
      keep = decide(k_left, by_mass, a.top_p * all64, 0.0, border, 0.0, a.min_p > 0.0, nullptr);
    }
  }
  if (CL) {
    g.sync_all();
    const int doubt = lead.keep;
    g.sync_all();
    if (doubt) {
      weigh(true);
      if (g.rank == 0) keep = decide(k_by_list ? a.top_k - (int)n_hi : n, by_mass, a.top_p * all64, 0.0, border, 0.0, a.min_p > 0.0, nullptr);
    } else if (!whole_list) {
      g.sync_all();                                  // (the warps' sums are in the leading rank)
    }
    if (g.rank != 0) { g.sync_all(); return; }
  }

  // ---- the draw (leading rank) ----
  if (whole_list && keep <= 128) {
    if (g.tid == 0) { s.tok = 0x7fffffff; s.last = -1; }
    __syncthreads();
    for (int i = g.tid; i < keep; i += threads) {
      const uint32_t id = (uint32_t)s.cand[i];
      double c = 0.0, z = 0.0;
      for (int j = 0; j < keep; ++j) {
        const double x = s.weight[j];
        z += x;
        c += (uint32_t)s.cand[j] <= id ? x : 0.0;
      }
      atomicMax(&s.last, (int)id);
      if (c > a.u * z) atomicMin(&s.tok, (int)id);
    }
    __syncthreads();
    if (g.tid == 0) p.tok[row] = s.tok != 0x7fffffff ? s.tok : s.last;
  } else {
    // masses per stretch of 1024 ids, the stretch that u falls in, and its ids one after the other
    const int stretches = (p.V + kWarpIds - 1) / kWarpIds;
    for (int q = g.warp; q < stretches; q += g.warps) {
      double x = 0.0;
      for (int i = g.lane; i < keep; i += 32) x += ((uint32_t)s.cand[i] >> 10) == (uint32_t)q ? s.weight[i] : 0.0;
      x = warp_sum64(x);
      if (g.lane == 0) s.warp_sum[q] = (whole_list ? 0.0 : s.warp_sum[q]) + x;
    }
    __syncthreads();
    if (g.warp == 0) {
      double z = 0.0;
      for (int q = 0; q < stretches; ++q) z += s.warp_sum[q];
      const double target = a.u * z;
      double run = 0.0;
      int at = -1, last = 0;
      for (int q = 0; q < stretches && at < 0; ++q) {
        const double x = s.warp_sum[q];
        if (x > 0.0) last = q;
        if (run + x > target) at = q;
        else run += x;
      }
      // (rounding may put u behind the last stretch: the last token kept then)
      const bool past = at < 0;
      if (past) at = last;
      const unsigned long long upto = keep > 0 ? s.cand[keep - 1] : 0ull;      // last word kept of the list
      int tok = -1, end_tok = -1;
      for (int i0 = at * kWarpIds; i0 < min(p.V, (at + 1) * kWarpIds) && tok < 0; i0 += 32) {
        const int id = i0 + g.lane;
        double x = 0.0;
        if (id < p.V) {
          const float l = to_float(lr[id]);
          if (l > -INFINITY) {
            const float wf = l == a.l_max ? 1.0f : ex2((l - a.l_max) * rate);
            const bool kept = wf >= kLeast && (wf >= hi || (keep > 0 && wf >= lo && word_of(l, id) <= upto));
            if (kept) x = weight64(l, a.l_max, a.rate);
          }
        }
        double incl = x;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const double y = __shfl_up_sync(0xffffffffu, incl, o);
          if (g.lane >= o) incl += y;
        }
        const uint32_t any = __ballot_sync(0xffffffffu, x > 0.0), hit = __ballot_sync(0xffffffffu, x > 0.0 && !past && run + incl > target);
        if (any != 0u) end_tok = i0 + 31 - __clz(any);
        if (hit != 0u) tok = i0 + __ffs(hit) - 1;
        run += __shfl_sync(0xffffffffu, incl, 31);
      }
      if (g.lane == 0) p.tok[row] = tok >= 0 ? tok : end_tok;
    }
  }
  if (CL) g.sync_all();
}

}  // namespace smp
}  // namespace srm
