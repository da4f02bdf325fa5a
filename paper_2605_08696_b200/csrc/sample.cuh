// Token selection with each row's own temperature, top-k, top-p and min-p, from given random numbers.
//
// Per row, with w_i = exp((l_i - l_max) / T) and the order (logit descending, id ascending):
//   the first top_k of the order; of these the shortest prefix whose mass reaches top_p times their mass; of these the
//   tokens with w_i >= min_p; then the lowest id whose cumulative mass, ids ascending, exceeds u times the mass kept.
// What is kept is always a prefix of the order.
//
// A block takes a row (a cluster of blocks, where there are few rows and many ids) and passes over it as often as the row needs,
// from HBM the first time, from L2 after that; several blocks per SM overlap their passes. First pass: the maximum, and each
// thread's own one; the k-th largest of those is a threshold that at least k tokens reach, and few more. Second pass: the tokens
// that reach it go to shared memory, where they are sorted and weighed in 64 bits; that is all for top-k, and for a nucleus that
// lies inside them. Otherwise the border is closed in on by thresholds, three per pass, with fp32 masses whose error is bounded
// (kSlack), until at most kCap tokens are left undecided; those are decided in 64 bits, with 64-bit sums over the rest where the
// bounds do not suffice. So the token is the one that 64-bit arithmetic gives, and nearly all of the arithmetic is not 64-bit.
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

// A warp reads `E` logits per lane at a time, a stretch of 32 E consecutive ids: 16, or 4 where the ids are few (more threads then share
// a row, and their maxima tell more of it). us (events around a launch, L2 flushed before it) with 16 / 4: 2000 rows of 1352 119 / 67, of
// 4096 80 / 96 (the border lies between the two), 4096 rows of 8000 184 / 207.
constexpr int kFewIds = 4096;
constexpr int kMaxStretches = 512;               // 262144 ids
constexpr int kMaxWarps = 32;
constexpr int kCap = 1024;                       // tokens that are sorted
constexpr int kMaxRanks = 8;
// Bound on the relative error of a sum of fp32 weights above 2^-80: the difference to the maximum, the factor 1 / (T ln 2) and
// their product are rounded once each, which moves a weight 2^x by 3 |x| 2^-24 ln 2 (|x| <= 80: 1.0e-5), ex2 by 2^-22, and the sums
// of at most 512 weights in a thread's run and two levels of five add 522 roundings (3.2e-5).
constexpr float kSlack = 5e-5f;
// The same for weights and sums in 64 bits: the difference, 1 / (T ln 2) and their product are off by 2^-51 together, which moves a weight
// 2^x by |x| 2^-51 ln 2 (|x| <= 80: 2.5e-14), the series and its evaluation by 2e-15, and 530 sums by 5.9e-14.
constexpr double kSlack64 = 1e-13;
constexpr double kLeastLog2 = -80.0;             // all weights below 2^-80 together are under 64-bit rounding (2^18 ids), and outside every nucleus
constexpr double kNoLog2 = -1076.0;              // below it a weight is 0 in 64 bits. Without a nucleus all others count: u may be 0 (or tiny),
                                                 // and then falls on the first of them
constexpr int kRounds = 40;                      // of a search: every other one takes two bits off the distance of lo and hi as keys

// 2^y for y <= 0 in 64 bits: the power of two by the exponent field, the rest by the series of exp to the 12th power of an
// argument of at most ln 2 / 2 (the remainder is under 2e-16). Rounding to the whole number by adding 1.5 2^52, whose low word then
// holds it (the conversion instructions have an eighth of the rate). Below 2^-1000 results come near the denormal numbers; those
// are rare and out of line (inline they cost every pass in 64 bits: 344 instead of 340 us for 4096 rows of 32000).
__device__ __noinline__ double pow2_tiny(double y) { return exp2(y); }
__device__ __forceinline__ double pow2_64(double y) {
  if (!(y > -1000.0)) return y > kNoLog2 ? pow2_tiny(y) : 0.0;
  const double shifted = y + 6755399441055744.0, n = shifted - 6755399441055744.0, t = (y - n) * 0.693147180559945309417;
  double s = 1.0 / 479001600;
  s = fma(s, t, 1.0 / 39916800); s = fma(s, t, 1.0 / 3628800); s = fma(s, t, 1.0 / 362880); s = fma(s, t, 1.0 / 40320);
  s = fma(s, t, 1.0 / 5040); s = fma(s, t, 1.0 / 720); s = fma(s, t, 1.0 / 120); s = fma(s, t, 1.0 / 24); s = fma(s, t, 1.0 / 6);
  s = fma(s, t, 0.5); s = fma(s, t, 1.0); s = fma(s, t, 1.0);
  return __hiloint2double(__double2hiint(s) + (__double2loint(shifted) << 20), __double2loint(s));
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

struct Scratch {
  unsigned long long cand[kCap];
  double weight[kCap], run[kCap];      // of the sorted candidates: weights, and running sums of them
  double part[kMaxStretches];          // mass kept of each stretch
  uint32_t ties[kMaxStretches];
  double d[2][kMaxWarps], rank_d[2][kMaxRanks];
  float f[2][kMaxWarps], rank_f[2][kMaxRanks];
  uint32_t n[2][kMaxWarps], rank_n[2][kMaxRanks];
  uint32_t block_n[kMaxWarps];
  float f4[2][4][kMaxWarps], rank_f4[2][kMaxRanks][4];
  uint32_t n3[2][3][kMaxWarps], rank_n3[2][kMaxRanks][3];
  uint32_t count;
  int keep, unsure, tok, last;
  double box[2];                       // from the leading rank to the others
};

// Cluster barrier in two halves, for all threads of all blocks.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

// What a block (or, with CL, a cluster) knows and does together. Reductions use two sets of places in turn, so one barrier each is
// enough: who writes a set again has passed the barrier of the reduction between, and so has every reader (of all ranks: only
// reductions in which they all wait take the sets). Their order is fixed, so results are the same every time, in every thread.
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
  __device__ uint32_t block_max(uint32_t v) {                          // of this block alone; used once, in places of its own
    v = __reduce_max_sync(0xffffffffu, v);
    if (lane == 0) s.block_n[warp] = v;
    __syncthreads();
    return __reduce_max_sync(0xffffffffu, lane < warps ? s.block_n[lane] : 0u);
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
  // four masses and three counts at once
  __device__ void add7(float (&m)[4], uint32_t (&n)[3]) {
    const int b = turn;
    turn ^= 1;
#pragma unroll
    for (int i = 0; i < 4; ++i) m[i] = srm::warp_sum(m[i]);
#pragma unroll
    for (int i = 0; i < 3; ++i) n[i] = __reduce_add_sync(0xffffffffu, n[i]);
    if (lane == 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s.f4[b][i][warp] = m[i];
#pragma unroll
      for (int i = 0; i < 3; ++i) s.n3[b][i][warp] = n[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) m[i] = srm::warp_sum(lane < warps ? s.f4[b][i][lane] : 0.f);
#pragma unroll
    for (int i = 0; i < 3; ++i) n[i] = __reduce_add_sync(0xffffffffu, lane < warps ? s.n3[b][i][lane] : 0u);
    if (CL) {
      if (tid < ranks) {                             // a thread per rank
        Scratch& to = *cooperative_groups::this_cluster().map_shared_rank(&s, tid);
#pragma unroll
        for (int i = 0; i < 4; ++i) to.rank_f4[b][rank][i] = m[i];
#pragma unroll
        for (int i = 0; i < 3; ++i) to.rank_n3[b][rank][i] = n[i];
      }
      sync_all();
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        m[i] = 0.f;
        for (int r = 0; r < ranks; ++r) m[i] += s.rank_f4[b][r][i];
      }
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        n[i] = 0u;
        for (int r = 0; r < ranks; ++r) n[i] += s.rank_n3[b][r][i];
      }
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

// The same for short lists, by counting: eight lanes per word find how many are smaller. `from` and `to` are different.
__device__ inline void sort_short(const unsigned long long* from, unsigned long long* to, int n, int tid, int threads) {
  for (int c0 = 0; c0 < n; c0 += threads >> 3) {
    const int c = c0 + (tid >> 3);
    const unsigned long long mine = c < n ? from[c] : 0ull;
    int rank = 0;
    for (int j = tid & 7; j < n; j += 8) rank += from[j] < mine ? 1 : 0;
    rank += __shfl_xor_sync(0xffffffffu, rank, 1);
    rank += __shfl_xor_sync(0xffffffffu, rank, 2);
    rank += __shfl_xor_sync(0xffffffffu, rank, 4);
    if (c < n && (tid & 7) == 0) to[rank] = mine;
  }
  __syncthreads();
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

// largest of three, NaN if one of them is
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// A list of at most 32 R tokens that holds all that is kept, from order to token, by one warp: place e of the order is register
// e / 32 of lane e % 32. (As steps of the block, a barrier and more between each two, the same took four times as long and fifteen
// warps' issue slots with it.) total: the mass that top_p counts, negative: that of the first k_left. Returns -1 when a border lies
// closer to the nucleus' mass than `off`.
template <int R, typename W>
__device__ __noinline__ int short_list(const unsigned long long* list, int n, int k_left, bool by_mass, double top_p, double total, double off,
                                       unsigned long long limit, double min_p, double u, int lane, W weight_of) {
  unsigned long long w[R];
#pragma unroll
  for (int r = 0; r < R; ++r) w[r] = 32 * r + lane < n ? list[32 * r + lane] : ~0ull;
#pragma unroll 1
  for (int size = 2; size <= 32 * R; size <<= 1) {
#pragma unroll
    for (int d = R / 2; d > 0; d >>= 1)              // places 32 d apart: other registers of the lane
      if (size > 32 * d) {
#pragma unroll
        for (int r = 0; r < R; ++r)
          if ((r & d) == 0) {
            const bool up = ((32 * r) & size) == 0;
            const unsigned long long x = w[r], y = w[r + d];
            if ((x > y) == up) { w[r] = y; w[r + d] = x; }
          }
      }
#pragma unroll 1
    for (int d = min(size >> 1, 16); d > 0; d >>= 1) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const unsigned long long y = __shfl_xor_sync(0xffffffffu, w[r], d);
        const bool up = ((32 * r + lane) & size) == 0, low = (lane & d) == 0;
        w[r] = (w[r] > y) == (up == low) ? y : w[r];
      }
    }
  }
  double x[R], before[R];
  double run = 0.0;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    x[r] = 32 * r + lane < n ? weight_of(word_logit(w[r])) : 0.0;
    double incl = x[r];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const double y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    const double prev = __shfl_up_sync(0xffffffffu, incl, 1);
    before[r] = run + (lane == 0 ? 0.0 : prev);
    if (total < 0.0 && by_mass) {                    // up to place k_left - 1
      const int last = min(k_left, n) - 1;
      const double t = __shfl_sync(0xffffffffu, run + incl, last & 31);
      if (last >> 5 == r) total = t;
    }
    run += __shfl_sync(0xffffffffu, incl, 31);
  }
  const double want = top_p * total;
  int keep = 0;
  bool doubt = false;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int e = 32 * r + lane;
    const bool in = e < k_left && e < n && w[r] <= limit && (!(min_p > 0.0) || x[r] >= min_p);
    keep += __popc(__ballot_sync(0xffffffffu, in && (!by_mass || e == 0 || before[r] < want)));
    doubt |= by_mass && in && e > 0 && fabs(before[r] - want) < off;
  }
  if (__any_sync(0xffffffffu, doubt)) return -1;
  double z = 0.0, c[R];
#pragma unroll
  for (int r = 0; r < R; ++r) c[r] = 0.0;
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll 4
    for (int j = 0; j < min(32, keep - 32 * r); ++j) {
      const uint32_t id = __shfl_sync(0xffffffffu, (uint32_t)w[r], j);
      const double y = __shfl_sync(0xffffffffu, x[r], j);
      z += y;
#pragma unroll
      for (int q = 0; q < R; ++q) c[q] += id <= (uint32_t)w[q] ? y : 0.0;
    }
  uint32_t tok = 0xffffffffu, last = 0;
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (32 * r + lane < keep) {
      last = max(last, (uint32_t)w[r]);
      if (c[r] > u * z) tok = min(tok, (uint32_t)w[r]);
    }
  tok = __reduce_min_sync(0xffffffffu, tok);
  last = __reduce_max_sync(0xffffffffu, last);
  return (int)(tok != 0xffffffffu ? tok : last);
}

// ---- the kernel -----------------------------------------------------------------------------------------------------
// Row r is block r; with CL, ranks [0, gridDim.x) of cluster r, each with `per_rank` stretches.
template <typename T, bool CL, int E>
__global__ void __launch_bounds__(512, 2) sample_kernel(const Args p, const int per_rank) {
  constexpr int kStretch = 32 * E;
  pdl_trigger();
  // A block's shared memory may be reached from others once all blocks of the cluster run: waited for in front of the first reduction,
  // behind the first pass.
  if (CL) cluster_arrive();
  __shared__ Scratch s;
  Group<CL> g{s, (int)threadIdx.x, (int)threadIdx.x & 31, (int)threadIdx.x >> 5, (int)blockDim.x >> 5, CL ? (int)blockIdx.x : 0, CL ? (int)gridDim.x : 1};
  const int threads = blockDim.x;
  const int64_t row = CL ? blockIdx.y : blockIdx.x;
  Scratch& lead = *(CL ? cooperative_groups::this_cluster().map_shared_rank(&s, 0) : &s);      // the rank that keeps the list
  const int stretches = (p.V + kStretch - 1) / kStretch;
  const int q0 = CL ? g.rank * per_rank : 0, q1 = CL ? min(stretches, q0 + per_rank) : stretches;
  const T* lr = static_cast<const T*>(p.logits) + row * p.stride;
  const bool wide = reinterpret_cast<uintptr_t>(lr) % (4 * sizeof(T)) == 0;
  pdl_wait();

  // f(E logits, stretch): this thread's of the block's stretches. Loops and bodies are kept short: most of this kernel's code runs
  // once or twice per row, so that its instructions are fetched anew.
  auto id_at = [&](int q, int j) { return q * kStretch + (wide ? 128 * (j >> 2) + 4 * g.lane + (j & 3) : 32 * j + g.lane); };
  auto each_lane = [&](auto&& f) {
#pragma unroll 1
    for (int q = q0 + g.warp; q < q1; q += g.warps) {
      float v[E];
      if (wide && (q + 1) * kStretch <= p.V) {
#pragma unroll
        for (int j = 0; j < E / 4; ++j) {
          const float4 x = ld4(lr + q * kStretch + 128 * j + 4 * g.lane);
          v[4 * j] = x.x; v[4 * j + 1] = x.y; v[4 * j + 2] = x.z; v[4 * j + 3] = x.w;
        }
      } else {
#pragma unroll
        for (int j = 0; j < E; ++j) {
          const int i = id_at(q, j);
          v[j] = i < p.V ? to_float(lr[i]) : -INFINITY;
        }
      }
      f(v, q);
    }
  };
  auto largest = [](const float (&v)[E]) {          // NaN if one of them is
    float m = max3_nan(v[0], v[1], v[2]);
#pragma unroll
    for (int j = 3; j + 1 < E; j += 2) m = max3_nan(m, v[j], v[j + 1]);
    return max3_nan(m, v[E - 1], v[E - 1]);
  };
  // f(logit, id), one by one
  auto each = [&](auto&& f) {
#pragma unroll 1
    for (int q = q0 + g.warp; q < q1; q += g.warps)
#pragma unroll 4
      for (int i = q * kStretch + g.lane; i < min(p.V, (q + 1) * kStretch); i += 32) f(to_float(lr[i]), i);
  };

  // ---- parameters and the maximum ----
  const float T0 = p.temperature != nullptr ? p.temperature[row] : 1.0f;
  const int k0 = p.top_k != nullptr ? p.top_k[row] : 0;
  const float p0 = p.top_p != nullptr ? p.top_p[row] : 1.0f, f0 = p.min_p != nullptr ? p.min_p[row] : 0.0f, u0 = p.u[row];
  const int top_k = k0 <= 0 || k0 > p.V ? p.V : k0;
  const double top_p = p0 < 1.0f ? (double)fmaxf(p0, 0.0f) : 1.0, min_p = f0 > 0.0f ? (double)fminf(f0, 1.0f) : 0.0, u = u0 > 0.0f ? (double)u0 : 0.0;
  float top = -INFINITY;                             // this thread's largest logit
  each_lane([&](const float (&v)[E], int) { top = max3_nan(top, largest(v), top); });
  if (!(top < INFINITY)) {
    raise_status(p.status, kStatusNonFinite);
    if (top != top) {                                // a NaN masks its token: it fails every comparison
      top = -INFINITY;                               // (over the same ids again: this thread's alone)
      each_lane([&](const float (&v)[E], int) {
#pragma unroll
        for (int j = 0; j < E; ++j) top = fmaxf(top, v[j]);
      });
    }
  }
  if (CL) cluster_wait();
  const float l_max = g.max_of(top);
  if (l_max == -INFINITY) {                          // nothing can be picked
    if (g.tid == 0 && g.rank == 0) { raise_status(p.status, kStatusNonFinite); p.tok[row] = 0; }
    if (CL) g.sync_all();
    return;
  }
  if (!(T0 >= kLeastTemperature) || top_k == 1 || top_p <= 0.0) {      // the first of the order
    uint32_t best = 0xffffffffu;
    each([&](float l, int id) { best = l == l_max ? min(best, (uint32_t)id) : best; });
    best = g.min_of(best);
    if (g.tid == 0 && g.rank == 0) p.tok[row] = (int)best;
    if (CL) g.sync_all();
    return;
  }
  // T ln 2, and its reciprocal: the fp32 one and two Newton steps (a division would be forty instructions in every warp). For an infinite
  // T an octave beyond all differences, and a rate that stays 0: every weight is 1, but those of masked tokens (0 times infinity).
  const double octave = T0 < INFINITY ? (double)T0 * 0.693147180559945309417 : 1e300;
  double rate64 = (double)(1.0f / (float)octave);
  rate64 = fma(rate64, fma(-octave, rate64, 1.0), rate64);
  rate64 = fma(rate64, fma(-octave, rate64, 1.0), rate64);
  const float rate = (float)fmin(rate64, 3e38);
  auto weight_of = [&](float l) { return weight64(l, l_max, rate64); };
  // the logit with weight 2^x, as a finite float
  auto logit_at = [&](double x) {
    const double v = fma(x, octave, (double)l_max);
    return v > -3.4e38 ? (float)v : -3.402823466e38f;
  };
  const bool limit_k = top_k < p.V, limit_p = top_p < 1.0;
  const float least = l_max == INFINITY ? INFINITY : logit_at(limit_p ? kLeastLog2 : kNoLog2);
  // min_p as logits: surely below, surely above
  float floor_lo = least, floor_hi = least;
  if (min_p > 0.0 && l_max < INFINITY) {
    const bool tiny = min_p < 0x1p-100;              // (2^64 times as much is a normal number)
    const double x = (double)__log2f((float)(tiny ? min_p * 0x1p64 : min_p)) - (tiny ? 64.0 : 0.0), v = fma(x, octave, (double)l_max);       // (off by 3.6e-7 (1 + |x|) at most)
    const double off = 1e-6 * (fabs(v) + fabs((double)l_max) + octave * (1.0 - x));
    floor_lo = fmaxf(least, v - off > -3.4e38 ? (float)(v - off) : least);
    floor_hi = fmaxf(least, v + off > -3.4e38 ? (float)(v + off) : least);
  }

  // ---- thresholds lo < hi: {l >= lo} holds all that is kept, {l >= hi} is kept (above min_p); counts and masses ----
  const float no_top = __int_as_float(0x7fffffff);                     // (nothing compares as at or above a NaN)
  const float beyond = INFINITY;                     // hi: nothing lies above it (l_max of infinity is told apart by `whole`)
  float lo = least, hi = beyond, m_lo = 0.f, m_hi = 0.f, Z = 0.f;
  uint32_t n_lo = 0xffffffffu, n_hi = 0;
  double all64 = 0.0, above64 = 0.0;
  bool whole = true;                                 // the list holds every token from l_max down to lo
  float m3[3];
  uint32_t n3[3];
  double x3[3];
  // The list: collect_begin, the tokens of a range from all threads, collect_end (all ranks get their number).
  int n = 0;
  auto collect_begin = [&]() {
    if (g.tid == 0) s.count = 0;
    __syncthreads();
  };
  auto collect = [&](float l, int id) {
    const uint32_t at = atomicAdd(&s.count, 1u);
    if (at < (uint32_t)kCap) s.cand[at] = word_of(l, id);
  };
  auto collect_end = [&]() {
    g.sync_all();
    if (CL) {                                        // the other ranks' behind the leading rank's own
      if (g.rank != 0) {
        const uint32_t mine = s.count;
        if (g.tid == 0) s.n[0][0] = atomicAdd(&lead.count, mine);
        __syncthreads();
        const uint32_t base = s.n[0][0];
        for (uint32_t i = g.tid; i < min(mine, (uint32_t)kCap) && base + i < (uint32_t)kCap; i += threads) lead.cand[base + i] = s.cand[i];
      }
      g.sync_all();
    }
    n = (int)min(lead.count, (uint32_t)kCap + 1u);
    g.sync_all();
    return (uint32_t)n;
  };
  // This thread's tokens of a stretch in [from, to) to the list: as a mask first, so that all lanes add their first one at once (a
  // branch per logit cost 5000 clocks a pass); the logit is read again.
  auto pick = [&](const float (&v)[E], int q, float from, float to) {
    uint32_t mask = 0;
#pragma unroll
    for (int j = 0; j < E; ++j) mask |= v[j] >= from && !(v[j] >= to) ? 1u << j : 0u;
#pragma unroll 1
    while (mask != 0u) {
      const int i = id_at(q, __ffs(mask) - 1);
      mask &= mask - 1u;
      collect(to_float(lr[i]), i);
    }
  };
  // Counts and masses at or above three thresholds t3[0] >= t3[1] >= t3[2], and the mass of everything.
  float t3[3];
  auto sum3 = [&](bool exact, bool list) {
    if (!exact) {
      const bool inf = l_max == INFINITY;
      const float half_max = 0.5f * l_max, rate2 = 2.0f * rate;
      const float a = t3[0], b = t3[1], c = t3[2];
      float m[4] = {0.f, 0.f, 0.f, 0.f};
      uint32_t k[3] = {0u, 0u, 0u};
      each_lane([&](const float (&v)[E], int q) {
#pragma unroll
        for (int i = 0; i < E; ++i) {
          // (halves, whose difference is always finite. A NaN or minus infinity ends as 0, whatever the rate, the maximum as 1; weights
          // under 2^-80 do no harm)
          float w = ex2(fmaxf(fmaf(0.5f, v[i], -half_max) * rate2, -INFINITY));
          if (inf) w = v[i] == l_max ? 1.0f : 0.0f;
          m[3] += w;
          if (v[i] >= c) { m[2] += w; ++k[2]; }
          if (v[i] >= b) { m[1] += w; ++k[1]; }
          if (v[i] >= a) { m[0] += w; ++k[0]; }
        }
        if (list && !(largest(v) < a)) pick(v, q, a, no_top);
      });
      g.add7(m, k);
      Z = m[3];
#pragma unroll
      for (int i = 0; i < 3; ++i) { m3[i] = m[i]; n3[i] = k[i]; x3[i] = (double)m[i]; }
    } else {
      double all = 0.0;
      uint32_t k[3] = {0u, 0u, 0u};
#pragma unroll
      for (int i = 0; i < 3; ++i) x3[i] = 0.0;
      each([&](float l, int) {
        if (l >= least) {
          const double w = weight_of(l);
          all += w;
#pragma unroll
          for (int i = 0; i < 3; ++i)
            if (l >= t3[i]) { x3[i] += w; ++k[i]; }
        }
      });
      all64 = g.add64(all);
#pragma unroll
      for (int i = 0; i < 3; ++i) x3[i] = g.add64(x3[i]);
      float unused[4] = {0.f, 0.f, 0.f, 0.f};
      g.add7(unused, k);
#pragma unroll
      for (int i = 0; i < 3; ++i) n3[i] = k[i];
    }
  };
  // Takes over what a threshold says. by_count: the border is token want_n of the order; else where the mass reaches want.
  bool even = false;                                 // a threshold, at `even_at`, with just the mass that is wanted (to the bounds)
  float even_at = 0.f;
  auto place = [&](bool by_count, uint32_t want_n, double want, double slack, double total) {
#pragma unroll
    for (int i = 2; i >= 0; --i) {
      const bool enough = by_count ? n3[i] >= want_n : x3[i] >= want + (want + total) * slack;
      const bool few = by_count ? n3[i] < want_n : x3[i] < want - (want + total) * slack;
      if (enough && t3[i] >= lo) { lo = t3[i]; n_lo = n3[i]; m_lo = (float)x3[i]; }
      if (few && t3[i] < hi) { hi = t3[i]; n_hi = n3[i]; m_hi = (float)x3[i]; }
      if (!enough && !few) { even = true; even_at = t3[i]; }
    }
  };
  // Closes in until the first kCap of the order reach the border (whole), or at most kCap tokens lie between lo and hi. False: the
  // border lies in a group of equal logits, all that is left between lo and hi; or (not exact) among too many tokens for the bounds.
  auto search = [&](bool by_count, uint32_t want_n, double want, bool exact) {
    const double slack = exact ? kSlack64 : (double)kSlack;
    double down = 4.0;                               // octaves below the maximum, while nothing is known below
    even = false;
    for (int it = 0; it < kRounds; ++it) {
      if (n_lo <= (uint32_t)kCap) { whole = true; return true; }
      if (n_lo != 0xffffffffu && n_lo - n_hi <= (uint32_t)kCap && (n_hi > (uint32_t)kCap / 2 || it > 4)) { whole = false; return true; }
      const bool unbounded = n_lo == 0xffffffffu;
      const uint32_t k_lo = logit_key(lo), k_hi = hi < beyond ? logit_key(hi) : logit_key(l_max) + 1u;
      if (!unbounded && k_hi - k_lo <= 1u) break;
      if (unbounded) {                               // down from the top in growing steps
        t3[0] = it == 0 ? l_max : fmaxf(least, logit_at(-down));
        t3[1] = fmaxf(least, logit_at(-1.5 * down));
        t3[2] = it >= 8 ? least : fmaxf(least, logit_at(-2.25 * down));
        down *= it == 0 ? 2.25 : 3.375;
      } else if ((it & 1) && hi < beyond) {          // around an estimate
        float c = by_count ? ((float)want_n - (float)n_hi) / ((float)n_lo - (float)n_hi) : ((float)want - m_hi) / (m_lo - m_hi);
        c = fminf(fmaxf(c, 0.08f), 0.92f);
#pragma unroll
        for (int i = 0; i < 3; ++i) t3[i] = (float)((double)hi - ((double)hi - (double)lo) * (double)(c + 0.06f * (float)(i - 1)));
      } else {                                       // at quarters of the keys
        const uint32_t d = k_hi - k_lo;
        t3[0] = key_logit(k_hi - max(d / 4, 1u));
        t3[1] = key_logit(k_lo + d / 2);
        t3[2] = key_logit(k_lo + max(d / 4, 1u));
      }
      const bool quarters = !unbounded && !((it & 1) && hi < beyond);
      const float lo_was = lo, hi_was = hi;
      sum3(exact, false);
      place(by_count, want_n, want, slack, exact ? all64 : (double)Z);
      if (exact && even) break;                      // the nucleus ends with the tokens that reach this threshold
      if (unbounded && n_lo == 0xffffffffu && t3[2] <= least) { lo = least; n_lo = n3[2]; m_lo = (float)x3[2]; }
      if (!exact && !by_count && quarters && lo == lo_was && hi == hi_was) break;
    }
    whole = false;
    return !(exact && even) && n_lo != 0xffffffffu && n_lo - n_hi <= (uint32_t)kCap;
  };
  // The list sorted, with weights and running sums (leading rank).
  auto order = [&]() {
    if (g.rank != 0) return;
    unsigned long long* other = reinterpret_cast<unsigned long long*>(s.run);
    if (n <= 192) {
      sort_short(s.cand, other, n, g.tid, threads);
      for (int i = g.tid; i < n; i += threads) {
        const unsigned long long w = other[i];
        s.cand[i] = w;
        s.weight[i] = weight_of(word_logit(w));
      }
    } else {
      sort_words(s.cand, n, g.tid, threads);
      for (int i = g.tid; i < n; i += threads) s.weight[i] = weight_of(word_logit(s.cand[i]));
    }
    __syncthreads();
    running_sums(s.weight, s.run, n, g.tid, threads, s.d[0]);
  };
  auto gather = [&]() {
    collect_begin();
    const float from = lo, to = whole ? no_top : hi;
    each_lane([&](const float (&v)[E], int q) {
      if (!(largest(v) < from)) pick(v, q, from, to);
    });
    return collect_end();
  };
  // Sums in 64 bits: of the tokens that `kept` takes, also per stretch (in the leading rank), and, with all, of everything.
  auto weigh = [&](bool all, auto&& kept) {
    double x = 0.0, y = 0.0;
#pragma unroll 1
    for (int q = q0 + g.warp; q < q1; q += g.warps) {
      double in = 0.0;
#pragma unroll 4
      for (int i = q * kStretch + g.lane; i < min(p.V, (q + 1) * kStretch); i += 32) {
        const float l = to_float(lr[i]);
        const bool k = l >= least && kept(l, i);
        if (k || (all && l >= least)) {
          const double w = weight_of(l);
          x += w;
          in += k ? w : 0.0;
        }
      }
      in = warp_sum64(in);
      y += in;
      if (g.lane == 0) lead.part[q] = in;
    }
    above64 = g.add64(g.lane == 0 ? y : 0.0);
    if (all) all64 = g.add64(x);
  };
  // How many of the list are kept (leading rank): the first k_left, words up to `limit`, what begins below the mass `want`
  // (counted from `before` on), and what has min_p. *unsure: a border closer to `want` than `off`.
  auto decide = [&](int k_left, bool by_mass, double want, double before, unsigned long long limit, double off, bool by_floor, int* unsure) {
    if (g.tid == 0) { s.keep = 0; s.unsure = 0; }
    __syncthreads();
    int mine = 0, doubt = 0;
    for (int i = g.tid; i < n; i += threads) {
      const double b = before + (i > 0 ? s.run[i - 1] : 0.0);
      const bool in = i < k_left && s.cand[i] <= limit && (!by_floor || s.weight[i] >= min_p), first = i == 0 && before == 0.0;
      mine += in && (!by_mass || first || b < want) ? 1 : 0;
      doubt |= by_mass && in && !first && fabs(b - want) < off ? 1 : 0;
    }
    if (mine) atomicAdd(&s.keep, mine);
    if (doubt) atomicOr(&s.unsure, 1);
    __syncthreads();
    const int keep = s.keep;
    if (unsure != nullptr) *unsure = s.unsure;
    __syncthreads();
    return keep;
  };
  // From the leading rank to all.
  auto tell = [&](double a, double b, double& x, double& y) {
    __syncthreads();
    if (g.tid == 0 && g.rank == 0) { s.box[0] = a; s.box[1] = b; }
    g.sync_all();
    x = lead.box[0];
    y = lead.box[1];
    g.sync_all();
  };

  // ---- which tokens the border lies among ----
  bool by_k = limit_k, by_mass = limit_p, listed = false, tie = false, all_kept = false;
  unsigned long long border = ~0ull;                 // words up to it are kept
  double mass_k = -1.0;                              // mass of the first top_k, once known
  const int guess = limit_k ? top_k : 64;            // a threshold that about so many tokens reach
  float first = -INFINITY;
  const int goal = CL ? (guess + g.ranks - 1) / g.ranks : guess;        // of this block
  if ((limit_k || limit_p) && 2 * goal <= threads) {
    // the guess-th largest of the threads' maxima, halving keys until few more threads reach it
    const uint32_t key = logit_key(top);
    uint32_t a = ~g.block_max(key != 0u ? ~key : 0u), b = logit_key(l_max) + 1u;      // a: all that have one, b: too few
    if (__syncthreads_count(key != 0u) >= goal) {
#pragma unroll 1
      for (int i = 0; i < 16 && b - a > 1u; ++i) {
        const uint32_t t = a + (b - a) / 2;
        const int c = __syncthreads_count(key >= t);
        if (c >= goal) {
          a = t;
          if (c <= goal + goal / 8 + 2) break;
        } else {
          b = t;
        }
      }
      first = key_logit(a);
    }
    if (CL) first = -g.max_of(-first);               // (every rank has its share of them above the least)
  }
  const float floor_list = limit_k && limit_p ? least : floor_lo;      // (top_p counts the mass of top_k without regard to min_p)
  if (limit_k) {
    if (first > -INFINITY) {
      lo = fmaxf(first, floor_list);
      n_lo = gather();
      listed = n_lo <= (uint32_t)kCap;
      if (!listed) {                                 // (more than the list counted)
        if (lo > floor_list) {
          t3[0] = t3[1] = t3[2] = lo;
          sum3(false, false);
          n_lo = n3[0];
          m_lo = m3[0];
        } else {
          n_lo = 0xffffffffu;
        }
      }
    }
    if (!listed && n_lo == 0xffffffffu) {            // few tokens in all?
      lo = floor_list;
      n_lo = gather();
      listed = n_lo <= (uint32_t)kCap;
      if (!listed) {
        t3[0] = t3[1] = t3[2] = lo;
        sum3(false, false);
        n_lo = n3[0];
        by_k = n_lo >= (uint32_t)top_k;
        if (by_k) n_lo = 0xffffffffu;                // (the search begins at the top)
      }
    }
    if (!listed && by_k) {
      tie = !search(true, (uint32_t)top_k, 0.0, false);
      if (tie && limit_p) {                          // the mass of top_k; its nucleus may end above the equal logits
        const float v = lo;
        weigh(false, [&](float l, int) { return l > v; });
        mass_k = above64 + (double)((uint32_t)top_k - n_hi) * weight_of(v);
        if (top_p * mass_k <= above64) {
          tie = by_k = false;
          hi = beyond; n_hi = 0; m_hi = 0.f;
        }
      }
    }
    if (!listed && by_k && !tie && !whole && limit_p) {
      // too many for one list: the border of top_k first, and the mass inside it
      gather();
      order();
      const float above = hi;
      weigh(false, [&](float l, int) { return l >= above; });
      double b = 0.0;
      if (g.rank == 0) {
        const int keep = decide(top_k - (int)n_hi, false, 0.0, above64, ~0ull, 0.0, false, nullptr);
        tell(above64 + s.run[keep - 1], __longlong_as_double((long long)s.cand[keep - 1]), mass_k, b);
      } else {
        tell(0.0, 0.0, mass_k, b);
      }
      border = (unsigned long long)__double_as_longlong(b);
      by_k = false;
      hi = beyond; n_hi = 0; m_hi = 0.f;
      whole = true;
    }
  }
  if (!listed && !tie && by_mass && !by_k) {
    double want = top_p * mass_k;
    bool ok = false;
    if (mass_k < 0.0) {
      // the mass of all, and a first list in the same pass
      t3[0] = fmaxf(first, floor_lo);
      t3[1] = fmaxf(least, logit_at(-6.0));
      t3[2] = fmaxf(least, logit_at(-12.0));
      if (t3[1] > t3[0]) t3[1] = t3[0];
      if (t3[2] > t3[1]) t3[2] = t3[1];
      const bool try_list = first > -INFINITY;
      if (try_list) collect_begin();
      sum3(false, try_list);
      want = top_p * (double)Z;
      place(false, 0, want, (double)kSlack, (double)Z);
      // the first list serves if the nucleus, or min_p, ends inside it
      if (try_list && n3[0] <= (uint32_t)kCap && (lo >= t3[0] || t3[0] <= floor_lo)) {
        lo = t3[0];
        n_lo = n3[0];
        listed = true;
        collect_end();
      } else if (try_list) {
        collect_end();
      }
    }
    if (!listed) {
      ok = search(false, 0, want, false);
      if (!ok) {                                     // too many tokens within the bounds: the same in 64 bits
        lo = least; hi = beyond; n_lo = 0xffffffffu; n_hi = 0; m_hi = 0.f;
        if (mass_k < 0.0) {
          weigh(true, [&](float, int) { return true; });
          mass_k = all64;
          want = top_p * all64;
        }
        ok = search(false, 0, want, true);
        if (!ok && even) {                           // (a whole sum of equal weights, say: the border lies between two values)
          all_kept = true;
          border = min(border, word_of(even_at, 0) | 0xffffffffull);
        } else {
          tie = !ok;
        }
      }
    }
  }
  bool floor_later = false;
  if (!listed && !tie && !by_k && !by_mass) {
    if (min_p > 0.0) {
      lo = floor_lo;
      listed = gather() <= (uint32_t)kCap;
    }
    all_kept = !listed;                              // down to min_p
  } else if (!listed && !tie && !all_kept && !whole && min_p > 0.0 && hi < floor_hi) {
    // not everything above the border has min_p
    if (hi <= floor_lo) {
      all_kept = true;                               // min_p ends the kept tokens above it
      border = ~0ull;
    } else {
      floor_later = true;                            // both lie within the bounds of each other
    }
  }

  // ---- the border, and how many of the list are kept ----
  int keep = 0;
  unsigned long long upto = ~0ull;                   // without a list: words up to it are kept, down to min_p
  if (!tie && !all_kept) {
    whole = whole || listed;
    if (whole) n_hi = 0;
    if (!listed) gather();
    if (whole && n <= 128) {
      const bool of_list = by_k && mass_k < 0.0, rough = by_mass && mass_k < 0.0 && !by_k;
      int tok = 0;
      if (g.rank == 0 && g.warp == 0) {
        const double total = mass_k >= 0.0 ? mass_k : of_list ? -1.0 : (double)Z, off = rough ? 2.0 * (double)kSlack * (double)Z : 0.0;
        const int k_left = by_k ? top_k : n;
        if (n <= 64) tok = short_list<2>(s.cand, n, k_left, by_mass, top_p, total, off, border, min_p, u, g.lane, weight_of);
        else tok = short_list<4>(s.cand, n, k_left, by_mass, top_p, total, off, border, min_p, u, g.lane, weight_of);
        if (g.lane == 0 && tok >= 0) p.tok[row] = tok;
      }
      if (rough) {                                   // the fp32 total may not be enough
        double t = (double)tok, none = 0.0;
        tell(t, none, t, none);
        tok = (int)t;
      }
      if (!rough || tok >= 0) {
        if (CL) g.sync_all();
        return;
      }
    }
    order();
    const float above = hi;
    const bool sums = !whole;
    if (sums) weigh(by_mass && mass_k < 0.0, [&](float l, int) { return l >= above; });
    const int k_left = by_k ? top_k - (int)n_hi : n;
    const bool by_floor = min_p > 0.0 && !floor_later;
    double doubt = 0.0, word = 0.0;
    if (g.rank == 0) {
      if (by_k && by_mass && whole) mass_k = s.run[min(k_left, n) - 1];
      const bool rough = by_mass && mass_k < 0.0 && whole;
      const double total = mass_k >= 0.0 ? mass_k : whole ? (double)Z : all64;
      int d = 0;
      keep = decide(k_left, by_mass, top_p * total, sums ? above64 : 0.0, border, rough ? 2.0 * (double)kSlack * (double)Z : 0.0, by_floor, &d);
      doubt = (double)d;
      word = __longlong_as_double((long long)(keep > 0 ? s.cand[keep - 1] : word_of(hi, 0) | 0xffffffffull));
    }
    if (CL) tell(doubt, word, doubt, word);
    if (doubt != 0.0) {                              // the fp32 total is not enough
      weigh(true, [&](float, int) { return false; });
      if (g.rank == 0) keep = decide(k_left, by_mass, top_p * all64, 0.0, border, 0.0, by_floor, nullptr);
    }
    upto = (unsigned long long)__double_as_longlong(word);
  } else if (tie) {
    // More equal logits than the list holds: all between lo and hi are one value v, and the border is the m-th of them by id.
    const float v = lo;
    weigh(by_mass && mass_k < 0.0, [&](float l, int) { return l > v; });
    const double above_v = above64, w = weight_of(v), total = mass_k >= 0.0 ? mass_k : all64;
    uint32_t left = 0xffffffffu;
    if (by_k) left = (uint32_t)top_k - n_hi;
    if (by_mass) {                                   // the first c >= 1 with above_v + c w >= want
      const double want = top_p * total;
      double c = w > 0.0 ? ceil((want - above_v) / w) : 1.0;
      if (c > 1.0 && above_v + (c - 1.0) * w >= want) c -= 1.0;
      if (above_v + c * w < want) c += 1.0;
      c = fmax(c, 1.0);
      left = c < (double)left ? (uint32_t)c : left;
    }
    // the id of that one: ties per stretch, the stretch, the place in it
#pragma unroll 1
    for (int q = q0 + g.warp; q < q1; q += g.warps) {
      uint32_t c = 0;
      for (int i = q * kStretch + g.lane; i < min(p.V, (q + 1) * kStretch); i += 32) c += to_float(lr[i]) == v ? 1u : 0u;
      c = __reduce_add_sync(0xffffffffu, c);
      if (g.lane == 0) lead.ties[q] = c;
    }
    g.sync_all();
    double id = -1.0, unused = 0.0;                  // (none: they are fewer, and all kept)
    if (g.rank == 0 && g.warp == 0) {
      int at = -1;
      for (int q = 0; q < stretches && at < 0; ++q) {
        if (s.ties[q] >= left) at = q;
        else left -= s.ties[q];
      }
      if (at >= 0)
        for (int i0 = at * kStretch; i0 < (at + 1) * kStretch && id < 0.0; i0 += 32) {
          const uint32_t bal = __ballot_sync(0xffffffffu, i0 + g.lane < p.V && to_float(lr[min(i0 + g.lane, p.V - 1)]) == v);
          if ((uint32_t)__popc(bal) >= left) id = (double)(i0 + (int)__fns(bal, 0, (int)left));
          else left -= __popc(bal);
        }
    }
    tell(id, 0.0, id, unused);
    upto = word_of(v, id >= 0.0 ? (int)id : -1);
  }
  const bool from_list = !tie && !all_kept && !floor_later;
  if (!from_list) {
    // masses kept per stretch
    upto = upto < border ? upto : border;
    const bool by_floor = min_p > 0.0;
    weigh(false, [&](float l, int i) { return word_of(l, i) <= upto && (!by_floor || l >= floor_hi || (l >= floor_lo && weight_of(l) >= min_p)); });
  }
  if (CL && g.rank != 0) { g.sync_all(); return; }

  // ---- the draw (leading rank) ----
  if (from_list && whole && keep <= 192) {
    // cumulative masses by id, eight lanes per token
    if (g.tid == 0) { s.tok = 0x7fffffff; s.last = -1; }
    __syncthreads();
    for (int c0 = 0; c0 < keep; c0 += threads >> 3) {
      const int c = c0 + (g.tid >> 3);
      const uint32_t id = c < keep ? (uint32_t)s.cand[c] : 0u;
      double in = 0.0, z = 0.0;
      for (int j = g.tid & 7; j < keep; j += 8) {
        const double w = s.weight[j];
        z += w;
        in += (uint32_t)s.cand[j] <= id ? w : 0.0;
      }
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) {
        z += __shfl_xor_sync(0xffffffffu, z, o);
        in += __shfl_xor_sync(0xffffffffu, in, o);
      }
      if (c < keep && (g.tid & 7) == 0) {
        atomicMax(&s.last, (int)id);
        if (in > u * z) atomicMin(&s.tok, (int)id);
      }
    }
    __syncthreads();
    if (g.tid == 0) p.tok[row] = s.tok != 0x7fffffff ? s.tok : s.last;
  } else {
    // masses per stretch, the stretch that u falls in, and its ids one after the other
    if (from_list) {
      upto = keep > 0 ? s.cand[keep - 1] : 0ull;
      for (int q = g.warp; q < stretches; q += g.warps) {
        double x = 0.0;
        for (int i = g.lane; i < keep; i += 32) x += (uint32_t)s.cand[i] / kStretch == (uint32_t)q ? s.weight[i] : 0.0;
        x = warp_sum64(x);
        if (g.lane == 0) s.part[q] = (whole ? 0.0 : s.part[q]) + x;
      }
    }
    __syncthreads();
    if (g.warp == 0) {
      double z = 0.0;
      for (int q = 0; q < stretches; ++q) z += s.part[q];
      const double target = u * z;
      double run = 0.0;
      int at = -1, last = 0;
      for (int q = 0; q < stretches && at < 0; ++q) {
        const double x = s.part[q];
        if (x > 0.0) last = q;
        if (run + x > target) at = q;
        else run += x;
      }
      const bool past = at < 0;                      // (rounding put u behind the last stretch: the last token kept then)
      if (past) at = last;
      int tok = -1, end_tok = -1;
      for (int i0 = at * kStretch; i0 < min(p.V, (at + 1) * kStretch) && tok < 0; i0 += 32) {
        const int id = i0 + g.lane;
        double x = 0.0;
        if (id < p.V) {
          const float l = to_float(lr[id]);
          const bool over = from_list && !whole && l >= hi;
          if (l >= least && (over || word_of(l, id) <= upto)) {
            x = weight_of(l);
            if (!from_list && !(x >= min_p)) x = 0.0;
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
