// 8-bit projection with block scales,
//   D[m, n] = sum_b sa[m, b] sw[n / 128, b] sum_{k in block b} a[m, k] w[n, k]   (+ bias[n]) (+ what D holds),
// a and w e4m3, blocks of 128 along K, on the 5th-generation tensor cores (tcgen05.mma.kind::f8f6f4, fp32 accumulators).
//
// The scales change from block to block of K, so a block's product (four instructions of K = 32) goes to tensor memory by
// itself and is added, times its scales, to a sum in the registers of the adding warps; tensor memory holds the products of
// two blocks, so that the warps add one while the tensor pipe computes the next.
#pragma once

#include "gemm8_ptx.cuh"

namespace srm {
namespace g8 {

constexpr int kBK = 128;                         // one block of scales = 128 bytes of a row (the swizzle span)

struct Args {
  int64_t M, N, K;             // K a multiple of 16
  const float* sa; int64_t sa_row, sa_blk;
  const float* sw; int64_t sw_row, sw_blk;
  const float* bias;           // [N] or nullptr
  int accumulate;              // D += (fp32 output only)
  void* out; int64_t out_stride;
  uint32_t* status;
};

// ---- few rows ------------------------------------------------------------------------------------------------
// The weights take the side of the 128 accumulator lanes and NT rows of A the columns, so a pass over the weights costs
// 128 x NT products per 128 x 128 weights however few rows there are. A tile (128 weight rows x NT rows of A) is one cluster:
// its S CTAs share out the blocks of K, and join their sums through distributed shared memory, each for its part of the
// columns, in the order of the ranks (so the result is the same every time). What bounds it: the weights' bytes, of
// which the two CTAs of an SM keep 96 to 160 KB on their way.
// Warps: 0 loads (TMA), 1 issues the MMAs and owns tensor memory, the others add: warp w reads the lanes 32 (w % 4) .. + 31,
// with NT = 128 eight of them split the columns.
template <int NT>
struct Few {
  static constexpr int kAddWarps = NT == 128 ? 8 : 4;
  static constexpr int kCols = NT == 128 ? 64 : NT;                    // columns per adding warp
  static constexpr int kThreads = 64 + 32 * kAddWarps;
  static constexpr int kWBytes = 128 * kBK, kABytes = NT * kBK;
  static constexpr int kStage = kWBytes + kABytes;
  static constexpr int kStages = NT == 128 ? 3 : NT == 64 ? 4 : 5;     // two CTAs per SM
  static constexpr int kRing = kStages * kStage;
  static constexpr int kJoin = 128 * NT * 4;                           // a CTA's sums on their way to the cluster (in the ring)
  static_assert(kJoin <= kRing, "the sums take the place of the operands");
  static constexpr int kScale = kAddWarps * 2 * kCols * 4;
  static constexpr int kBytes = kRing + kScale + 256 + 1024;
  static constexpr int kTmCols = 2 * NT < 32 ? 32 : 2 * NT;
};

template <int NT, typename OT>
__global__ void __launch_bounds__(Few<NT>::kThreads) gemm8_few_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmW,
                                                                      const Args g) {
  using F = Few<NT>;
  pdl_trigger();
  extern __shared__ uint8_t raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  float* scale = reinterpret_cast<float*>(smem + F::kRing);            // [warp][2][kCols]
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + F::kRing + F::kScale);
  uint64_t* empty = full + F::kStages;
  uint64_t* tfull = empty + F::kStages;
  uint64_t* tempty = tfull + 2;
  uint32_t* slot = reinterpret_cast<uint32_t*>(tempty + 2);

  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int ranks = gridDim.x, rank = blockIdx.x;                      // the cluster is the grid's x dimension
  const int n0 = blockIdx.y * 128, m0 = blockIdx.z * NT;
  const int kb_all = (int)((g.K + kBK - 1) / kBK), per = (kb_all + ranks - 1) / ranks;
  const int kb0 = rank * per, kbn = max(0, min(per, kb_all - kb0));

  if (threadIdx.x == 0) {
    for (int s = 0; s < F::kStages; ++s) { bar_init(&full[s], 1); bar_init(&empty[s], 1); }
    for (int a = 0; a < 2; ++a) { bar_init(&tfull[a], 1); bar_init(&tempty[a], F::kAddWarps); }
    bar_init_fence();
  }
  if (warp == 1) tm_alloc<1>(slot, F::kTmCols);
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tm = *slot;
  pdl_wait();

  float acc[F::kCols];
#pragma unroll
  for (int c = 0; c < F::kCols; ++c) acc[c] = 0.f;
  const int quad = warp & 3, cg = (warp - 2) >> 2;                      // (adding warps)
  if (warp == 0) {
    if (one_lane()) {
      map_prefetch(&tmA);
      map_prefetch(&tmW);
      uint32_t phase = 0;
      int stage = 0;
      for (int i = 0; i < kbn; ++i) {
        if (!bar_wait(&empty[stage], phase ^ 1u, g.status)) { drain_copies(); break; }
        const uint32_t bar = smem_addr(&full[stage]);
        bar_expect(bar, F::kStage);
        tile_load<1>(smem_addr(smem + stage * F::kStage), &tmW, bar, (kb0 + i) * kBK, n0);
        tile_load<1>(smem_addr(smem + stage * F::kStage + F::kWBytes), &tmA, bar, (kb0 + i) * kBK, m0);
        if (++stage == F::kStages) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp == 1) {
    if (one_lane()) {
      uint32_t phase = 0;
      int stage = 0;
      for (int i = 0; i < kbn; ++i) {
        const int buf = i & 1;
        if (!bar_wait(&tempty[buf], ((i >> 1) & 1) ^ 1u, g.status)) break;
        if (!bar_wait(&full[stage], phase, g.status)) break;
        fence_after();
        const uint64_t dw = tile_desc(smem_addr(smem + stage * F::kStage)), da = tile_desc(smem_addr(smem + stage * F::kStage + F::kWBytes));
#pragma unroll
        for (int k = 0; k < 4; ++k) mma8<1>(tm + buf * NT, dw + 2 * k, da + 2 * k, mma_desc(128, NT), k != 0);
        mma_commit<1>(&empty[stage]);
        mma_commit<1>(&tfull[buf]);
        if (++stage == F::kStages) { stage = 0; phase ^= 1u; }
      }
    }
  } else {
    float* sc = scale + (warp - 2) * 2 * F::kCols;
    const float* sw = g.sw + (int64_t)(n0 >> 7) * g.sw_row + (int64_t)kb0 * g.sw_blk;
    const float* sa = g.sa + (int64_t)kb0 * g.sa_blk;
    constexpr int kPer = (F::kCols + 31) / 32;
    const int64_t last = g.M - 1;
    int64_t off[kPer];                                                  // this lane's rows of A (beyond the last one: the last)
    float next[kPer], wnext = 0.f;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int64_t m = m0 + cg * F::kCols + j * 32 + lane;
      off[j] = (m < last ? m : last) * g.sa_row;
      next[j] = kbn > 0 ? sa[off[j]] : 0.f;
    }
    if (kbn > 0) wnext = *sw;
    bool ok = true;
    for (int i = 0; i < kbn; ++i) {
      const int buf = i & 1;
      float* mine = sc + buf * F::kCols;
#pragma unroll
      for (int j = 0; j < kPer; ++j)
        if (j * 32 + lane < F::kCols) mine[j * 32 + lane] = next[j] * wnext;
      if (i + 1 < kbn) {
#pragma unroll
        for (int j = 0; j < kPer; ++j) next[j] = sa[off[j] + (i + 1) * g.sa_blk];
        wnext = sw[(i + 1) * g.sw_blk];
      }
      __syncwarp();
      if (!bar_wait(&tfull[buf], (i >> 1) & 1, g.status)) { ok = false; break; }
      fence_after();
      const uint32_t t = tm + ((uint32_t)(quad * 32) << 16) + buf * NT + cg * F::kCols;
#pragma unroll
      for (int c = 0; c < F::kCols; c += 16) {
        uint32_t r[16];
        tm_load16(t + c, r);
        tm_load_wait();
        keep_order(r);
        if (c + 16 == F::kCols) {
          fence_before();
          __syncwarp();
          if (lane == 0) bar_arrive(smem_addr(&tempty[buf]));
        }
#pragma unroll
        for (int q = 0; q < 16; q += 4) {
          const float4 s = *reinterpret_cast<const float4*>(mine + c + q);
          acc[c + q] = fmaf(s.x, __uint_as_float(r[q]), acc[c + q]);
          acc[c + q + 1] = fmaf(s.y, __uint_as_float(r[q + 1]), acc[c + q + 1]);
          acc[c + q + 2] = fmaf(s.z, __uint_as_float(r[q + 2]), acc[c + q + 2]);
          acc[c + q + 3] = fmaf(s.w, __uint_as_float(r[q + 3]), acc[c + q + 3]);
        }
      }
    }
    (void)ok;
  }
  // Every block of this CTA has been multiplied: the ring's bytes are free for the sums.
  const int64_t n = n0 + quad * 32 + lane;
  OT* out = static_cast<OT*>(g.out);
  if (ranks == 1) {
    if (warp >= 2 && n < g.N) {
      const float b = g.bias != nullptr ? g.bias[n] : 0.f;
#pragma unroll
      for (int c = 0; c < F::kCols; ++c) {
        const int64_t m = m0 + cg * F::kCols + c;
        if (m < g.M) {
          OT* o = out + m * g.out_stride + n;
          float v = acc[c] + b;
          if (g.accumulate) v += to_float(*o);
          *o = from_float<OT>(v);
        }
      }
    }
  } else {
    float* join = reinterpret_cast<float*>(smem);                       // [column][128 lanes]
    if (warp >= 2) {
#pragma unroll
      for (int c = 0; c < F::kCols; ++c) join[(cg * F::kCols + c) * 128 + quad * 32 + lane] = acc[c];
    }
    sync_cluster();
    const int cols = (int)min((int64_t)NT, g.M - m0);
    const uint32_t base = smem_addr(join);
    for (int e = threadIdx.x + rank * F::kThreads; e < cols * 128; e += ranks * F::kThreads) {
      float v = 0.f;
      for (int r = 0; r < ranks; ++r) v += peer_load(peer_addr(base + e * 4, r));
      const int64_t col = n0 + (e & 127), m = m0 + (e >> 7);
      if (col < g.N) {
        OT* o = out + m * g.out_stride + col;
        if (g.bias != nullptr) v += g.bias[col];
        if (g.accumulate) v += to_float(*o);
        *o = from_float<OT>(v);
      }
    }
    sync_cluster();                                                     // no CTA leaves while its sums are read
  }
  fence_before();
  __syncthreads();
  if (warp == 1) {
    fence_after();
    tm_free<1>(tm, F::kTmCols);
  }
}

// ---- many rows -----------------------------------------------------------------------------------------------
// A CTA pair owns a 256 x 256 tile (256 rows of A over both CTAs' accumulator lanes, 256 weight rows); persistent, tiles taken
// round-robin, rows fastest. A block of K is four MMAs (256 x 256 x 32) into one of two accumulators, which the eight adding
// warps of each CTA (32 lanes x 128 columns each, one weight scale) fetch while the next block is multiplied. (Halves of 128
// columns would give them the time of three halves, but an instruction of 128 columns asks shared memory for 128 bytes a clock,
// its limit, and took 1.27 of its share of the time.) The adding warps hold 128 sums a thread and fetch 32 columns ahead of the
// ones they add: they take the registers that the warpgroup of the loads and the MMAs gives up. A warp of its own keeps the
// scales of the next blocks coming into shared memory (fetched by the adding warps one block ahead they cost 330 of 1220 clocks a
// block). What bounds it now is the adding: 870 clocks a block, of which the MMAs need 512. It is a chain of waits rather than a count of
// instructions: 128 scalar multiply-adds of two warps per scheduler are 256 issue slots, and half of all slots stay empty.
// M = 16384, N = 6144, K = 1536, bf16 output: 175 to 177 us a pass among others, 1.75 PFLOP/s at the power cap (1.52 GHz).
// A tile's output is staged whole (64 KB per CTA in bf16, 128 KB in fp32, which leaves three stages for the operands), and stored while
// the next tile is computed: all CTAs finish their tiles at about the same time, so that the stores come in bursts that memory takes
// as long for as the tile's products (with half of an fp32 tile staged, the adding warps waited for the other half: M = 4096,
// N = 32000, K = 1024: 212 us).
template <typename OT>
struct Many {
  static constexpr int kCols = 128;
  static constexpr int kBoxes = kCols * (int)sizeof(OT) / 128;          // of a warp
  static constexpr int kStages = sizeof(OT) == 4 ? 3 : 4;
  static constexpr int kSlots = kStages + 2;                            // blocks whose scales are there: the stages, two accumulators
  static constexpr int kABytes = 128 * kBK, kWBytes = 128 * kBK;       // per CTA and block
  static constexpr int kStage = kABytes + kWBytes;
  static constexpr int kAddWarps = 8;
  static constexpr int kThreads = 128 + 32 * kAddWarps;                 // 168 registers a thread at launch
  static constexpr int kRegsFew = 40, kRegsAdd = 232;                   // 4 x 40 + 8 x 232 = 12 x 168 (warps)
  static constexpr int kBox = 32 * 128;                                 // staged output: 32 rows x 128 bytes
  static constexpr int kScales = kSlots * 130 * 4;                      // per slot: 128 rows, 2 groups of 128 columns
  static constexpr int kBarriers = (2 * kStages + 4 + kSlots + 1) * 8;
  static constexpr int kBytes = kStages * kStage + kAddWarps * kBoxes * kBox + kScales + kBarriers;
  static_assert(kBytes <= 232448, "shared memory of a block");
};

// A warp's staging box: 32 rows x 128 bytes of finished output (v: the lane's row), the 16-byte pieces of a row swizzled as the
// output's tensor map has them (which also spreads eight lanes over all banks).
__device__ __forceinline__ void fill_box(uint8_t* box, int lane, const uint32_t (&v)[32]) {
#pragma unroll
  for (int q = 0; q < 8; ++q)
    *reinterpret_cast<uint4*>(box + lane * 128 + ((q ^ (lane & 7)) << 4)) = make_uint4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
}

// A filled box to rows row0 .., columns col0 .. with plain stores, row by row: outputs whose rows' pitch is no multiple of 16 bytes
// (they have no tensor map).
template <typename OT>
__device__ __forceinline__ void write_box(const Args& g, const uint8_t* box, int lane, int64_t row0, int64_t col0) {
  constexpr int kPer = 128 / (int)sizeof(OT);
  const int rows = (int)min((int64_t)32, g.M - row0);
  for (int r = 0; r < rows; ++r) {
    OT* o = static_cast<OT*>(g.out) + (row0 + r) * g.out_stride + col0;
#pragma unroll
    for (int e = 0; e < kPer; e += 32) {
      const int c = e + lane, byte = c * (int)sizeof(OT);
      const OT x = *reinterpret_cast<const OT*>(box + r * 128 + ((((byte >> 4) ^ (r & 7)) << 4) | (byte & 15)));
      if (col0 + c < g.N) o[c] = g.accumulate ? from_float<OT>(to_float(x) + to_float(o[c])) : x;
    }
  }
}

// MAPPED: the output has a tensor map; BIAS: there is one. (Each its own kernel: with both in one, the code of a tile's output,
// unrolled over 128 columns, missed the instruction cache every time and cost as much as six blocks of K.)
template <typename OT, bool MAPPED, bool BIAS>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(Many<OT>::kThreads, 1)
gemm8_many_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmD,
                  const Args g) {
  using F = Many<OT>;
  pdl_trigger();
  // (no room for rounding up: a block's dynamic shared memory starts on a boundary of 1024 bytes where it has no static one)
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t* boxes = smem + F::kStages * F::kStage;
  float* scales = reinterpret_cast<float*>(boxes + F::kAddWarps * F::kBoxes * F::kBox);
  uint64_t* full = reinterpret_cast<uint64_t*>(reinterpret_cast<uint8_t*>(scales) + F::kScales);      // leader's: both CTAs' copies of a stage, their scale warps' word
  uint64_t* empty = full + F::kStages;                                  // per CTA: the stage may be filled again
  uint64_t* tfull = empty + F::kStages;                                 // per CTA [2]: a block's product is there
  uint64_t* tempty = tfull + 2;                                         // leader's [2]: both CTAs' warps have fetched it
  uint64_t* sfull = tempty + 2;                                         // per CTA [kSlots]: a block's scales are there
  uint32_t* slot = reinterpret_cast<uint32_t*>(sfull + F::kSlots);
  if ((smem_addr(smem) & 1023u) != 0u) {                                // (never seen; every CTA alike)
    raise_status(g.status, kStatusWaitTimeout);
    return;
  }

  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const uint32_t rank = cta_rank();
  const uint32_t first = blockIdx.x >> 1, step = gridDim.x >> 1;
  if (threadIdx.x == 0) {
    for (int s = 0; s < F::kStages; ++s) { bar_init(&full[s], 4); bar_init(&empty[s], 1); }
    for (int a = 0; a < 2; ++a) { bar_init(&tfull[a], 1); bar_init(&tempty[a], 2 * F::kAddWarps); }
    for (int a = 0; a < F::kSlots; ++a) bar_init(&sfull[a], 32);
    bar_init_fence();
  }
  if (warp == 1) tm_alloc<2>(slot, 512);
  fence_before();
  sync_cluster();
  fence_after();
  const uint32_t tm = *slot;
  pdl_wait();

  const uint32_t m_tiles = (uint32_t)((g.M + 255) / 256), tiles = m_tiles * (uint32_t)((g.N + 255) / 256);      // (fits: checked)
  const int kbs = (int)((g.K + kBK - 1) / kBK);
  if (warp < 4) give_registers<F::kRegsFew>();
  if (warp == 0) {
    if (one_lane()) {
      map_prefetch(&tmA);
      map_prefetch(&tmW);
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (uint32_t q = first; ok && q < tiles; q += step) {
        const int m0 = (int)(q % m_tiles * 256 + rank * 128), n0 = (int)(q / m_tiles * 256 + rank * 128);
        for (int kb = 0; kb < kbs; ++kb) {
          if (!bar_wait(&empty[stage], phase ^ 1u, g.status)) { ok = false; break; }
          const uint32_t bar = peer_addr(smem_addr(&full[stage]), 0), dst = smem_addr(smem + stage * F::kStage);
          bar_expect(bar, F::kStage);
          tile_load<2>(dst, &tmA, bar, kb * kBK, m0);
          tile_load<2>(dst + F::kABytes, &tmW, bar, kb * kBK, n0);
          if (++stage == F::kStages) { stage = 0; phase ^= 1u; }
        }
      }
      if (!ok) drain_copies();
    }
  } else if (warp == 1) {
    if (rank == 0 && one_lane()) {
      int stage = 0;
      uint32_t phase = 0, it = 0;
      bool ok = true;
      for (uint32_t q = first; ok && q < tiles; q += step) {
        for (int kb = 0; kb < kbs; ++kb, ++it) {
          const int buf = (int)(it & 1u);
          if (!bar_wait(&full[stage], phase, g.status) || !bar_wait(&tempty[buf], ((it >> 1) & 1u) ^ 1u, g.status)) { ok = false; break; }
          fence_after();
          const uint32_t src = smem_addr(smem + stage * F::kStage);
          const uint64_t da = tile_desc(src), dw = tile_desc(src + F::kABytes);
#pragma unroll
          for (int k = 0; k < 4; ++k) mma8<2>(tm + buf * 256, da + 2 * k, dw + 2 * k, mma_desc(256, 256), k != 0);
          mma_commit<2>(&tfull[buf]);
          mma_commit<2>(&empty[stage]);
          if (++stage == F::kStages) { stage = 0; phase ^= 1u; }
        }
      }
    }
  } else if (warp == 2) {
    // A block's scales take the slot of the block kStages + 2 before it, whose sums are done: this block's stage is free, so the MMAs
    // are past the block kStages before it, and they are never more than two blocks ahead of the sums. The block's MMAs wait for this
    // warp's arrival, which comes when all its lanes have seen the stage free: they could complete the barrier's next phase under it
    // otherwise (they need no scales, and run ahead of the sums), and the wait by parity would miss its own.
    int stage = 0, at = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (uint32_t q = first; ok && q < tiles; q += step) {
      const float* sa[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) sa[j] = g.sa + min((int64_t)(q % m_tiles * 256 + rank * 128 + j * 32 + lane), g.M - 1) * g.sa_row;
      const float* sw = g.sw + (min((int64_t)(q / m_tiles) * 256 + (lane & 1) * 128, g.N - 1) >> 7) * g.sw_row;
      for (int kb = 0; kb < kbs; ++kb) {
        if (!__all_sync(0xffffffffu, bar_wait(&empty[stage], phase ^ 1u, g.status))) { ok = false; break; }
        if (lane == 0) bar_arrive(peer_addr(smem_addr(&full[stage]), 0));
        float* to = scales + at * 130;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          copy4(smem_addr(to + j * 32 + lane), sa[j]);
          sa[j] += g.sa_blk;
        }
        if (lane < 2) copy4(smem_addr(to + 128 + lane), sw);
        sw += g.sw_blk;
        copies_arrive(&sfull[at]);
        if (++at == F::kSlots) at = 0;
        if (++stage == F::kStages) { stage = 0; phase ^= 1u; }
      }
    }
    copies_wait();
  } else if (warp >= 4) {
    take_registers<F::kRegsAdd>();
    const int quad = warp & 3, cg = (warp - 4) >> 2;
    uint8_t* box = boxes + (warp - 4) * F::kBoxes * F::kBox;
    const uint32_t drained = peer_addr(smem_addr(&tempty[0]), 0);
    const uint32_t lanes = tm + ((uint32_t)(quad * 32) << 16) + cg * F::kCols;
    uint32_t it = 0, at = 0, at_phase = 0;
    bool ok = true;
    if (MAPPED && lane == 0) map_prefetch(&tmD);
    constexpr int kPer = 128 / (int)sizeof(OT);                         // columns of a box
    // The boxes of the last tile go out one by one, a block of K apart: the TMA unit takes its work in order, and the operands of the
    // next blocks would wait behind a whole tile's stores (128 KB of fp32 took 3200 clocks of a tile's 12 400).
    int64_t out_row = 0, out_col = 0;
    int out_box = F::kBoxes;                                            // the next one to store
    auto store_box = [&]() {
      if (!MAPPED || out_box >= F::kBoxes) return;
      const int64_t col = out_col + out_box * kPer;
      if (col < g.N && one_lane()) {
        const uint32_t src = smem_addr(box + out_box * F::kBox);
        if (sizeof(OT) == 4 && g.accumulate) tile_add(&tmD, src, (int)col, (int)out_row);
        else if (sizeof(OT) == 4) tile_store_streaming(&tmD, src, (int)col, (int)out_row);
        else tile_store(&tmD, src, (int)col, (int)out_row);
        stores_commit();
      }
      __syncwarp();
      ++out_box;
    };
    for (uint32_t q = first; ok && q < tiles; q += step) {
      const int64_t row0 = q % m_tiles * 256 + rank * 128 + quad * 32, col0 = (int64_t)(q / m_tiles) * 256 + cg * F::kCols;
      float acc[F::kCols], s_next = 0.f;
      uint32_t ra[32], rb[32];
      // the next block: its scales, and the first columns of its product on their way
      auto begin = [&]() {
        if (!bar_wait(&sfull[at], at_phase, g.status)) return false;
        s_next = scales[at * 130 + quad * 32 + lane] * scales[at * 130 + 128 + cg];
        if (++at == (uint32_t)F::kSlots) { at = 0; at_phase ^= 1u; }
        if (!bar_wait(&tfull[it & 1u], (it >> 1) & 1u, g.status)) return false;
        fence_after();
        tm_load32(lanes + (it & 1u) * 256, ra);
        return true;
      };
      // a block added (the first one sets the sums); the next one is begun before the last columns are
      auto block = [&](auto set, bool more) {
        const float s = s_next;
        const uint32_t buf = it & 1u, t = lanes + buf * 256;
        bool fine = true;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t (&cur)[32] = (c & 1) ? rb : ra;
          uint32_t (&nxt)[32] = (c & 1) ? ra : rb;
          tm_load_wait();
          keep_order(cur);
          if (c < 3) {
            tm_load32(t + 32 * (c + 1), nxt);
          } else {                                                      // everything has left tensor memory
            fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(drained + buf * 8u);
            ++it;
            if (more) fine = begin();
          }
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            if (set) acc[32 * c + j] = s * __uint_as_float(cur[j]);
            else acc[32 * c + j] = fmaf(s, __uint_as_float(cur[j]), acc[32 * c + j]);
          }
        }
        return fine;
      };
      ok = begin();
      if (ok) ok = block(Yes(), kbs > 1);
      store_box();
      for (int kb = 1; ok && kb < kbs; ++kb) {
        ok = block(No(), kb + 1 < kbs);
        store_box();
      }
      if (!ok) break;
      while (MAPPED && out_box < F::kBoxes) store_box();
      if (row0 < g.M && col0 < g.N) {
        if (MAPPED && one_lane()) stores_wait_read();                   // the last tile's boxes have been read
        __syncwarp();
#pragma unroll
        for (int c = 0; c < F::kCols; c += kPer) {
          uint32_t v[32];
#pragma unroll
          for (int j = 0; j < kPer; j += 2) {
            float x = acc[c + j], y = acc[c + j + 1];
            if (BIAS) {
              x += col0 + c + j < g.N ? __ldg(g.bias + col0 + c + j) : 0.f;
              y += col0 + c + j + 1 < g.N ? __ldg(g.bias + col0 + c + j + 1) : 0.f;
            }
            if (sizeof(OT) == 4) {
              v[j % 32] = __float_as_uint(x);
              v[j % 32 + 1] = __float_as_uint(y);
            } else {
              const __nv_bfloat162 b = __floats2bfloat162_rn(x, y);
              v[j / 2 % 32] = *reinterpret_cast<const uint32_t*>(&b);
            }
          }
          fill_box(box + c / kPer * F::kBox, lane, v);
        }
        if (MAPPED) fence_async();
        __syncwarp();
        if (MAPPED) {
          out_row = row0;
          out_col = col0;
          out_box = 0;
        } else {
#pragma unroll 1
          for (int b = 0; b < F::kBoxes; ++b) write_box<OT>(g, box + b * F::kBox, lane, row0, col0 + b * kPer);
          __syncwarp();
        }
      }
    }
    while (MAPPED && out_box < F::kBoxes) store_box();
    if (MAPPED && one_lane()) stores_wait();                            // the boxes are out before shared memory goes away
  }
  fence_before();
  sync_cluster();                                                       // the leader's MMAs use the peer's memory until here
  if (warp == 1) {
    fence_after();
    tm_free<2>(tm, 512);
  }
}

}  // namespace g8
}  // namespace srm
