// C ABI of the 8-bit operators and of the sampler with parameters per row (see include/srm.h for the contract): argument
// checking and launches.
#include <numeric>

#include "host.cuh"

#include "gemm8.cuh"
#include "quant8.cuh"
#include "sample.cuh"

using namespace srm;

namespace {

bool dtype_ok(int t) { return t == SRM_DTYPE_FP32 || t == SRM_DTYPE_BF16 || t == SRM_DTYPE_FP16; }
int64_t dtype_bytes(int t) { return t == SRM_DTYPE_FP32 ? 4 : 2; }

// f(T{}) with the element type of an SRM_DTYPE_* code
template <typename F>
int with_type(int t, F&& f) {
  return t == SRM_DTYPE_BF16 ? f(bf16{}) : t == SRM_DTYPE_FP16 ? f(fp16{}) : f(float{});
}

// Rows of `cols` elements that are read or written 16 bytes at a time: base and pitch on 16-byte boundaries, rows not overlapping.
int rows_ok(const void* p, int64_t rows, int64_t cols, int64_t stride, int64_t elem) {
  if (p == nullptr || (rows > 1 && stride < cols)) return SRM_ERR_INVALID_ARG;
  if (!aligned(p, 16) || (rows > 1 && stride * elem % 16)) return SRM_ERR_ALIGNMENT;
  return SRM_OK;
}
int floats_ok(const void* p) { return p == nullptr ? SRM_ERR_INVALID_ARG : !aligned(p, 4) ? SRM_ERR_ALIGNMENT : SRM_OK; }
// Scales of a matrix, rows x blks of them. Written ones each in a place of its own: places i row + b blk of two scales are the same where
// their rows are a multiple of blk / gcd apart and their blocks the same multiple of row / gcd.
int written_scales_ok(const float* p, int64_t rows, int64_t blks, int64_t row, int64_t blk) {
  if ((rows > 1 && row < 1) || (blks > 1 && blk < 1)) return SRM_ERR_INVALID_ARG;
  if (rows > 1 && blks > 1) {
    const int64_t g = std::gcd(row, blk);
    if (blk / g < rows && row / g < blks) return SRM_ERR_INVALID_ARG;
  }
  return floats_ok(p);
}
// Read ones with any stride from 0.
int read_scales_ok(const float* p, int64_t rows, int64_t blks, int64_t row, int64_t blk) {
  return (rows > 1 && row < 0) || (blks > 1 && blk < 0) ? SRM_ERR_INVALID_ARG : floats_ok(p);
}

constexpr int64_t kMaxGrid = 0x7fffffff;

template <typename XT, typename DT>
int launch_norm(const q8::NormArgs& p, cudaStream_t st) {
  const int n4 = p.d / 4;
  const dim3 grid((unsigned)p.R);
  auto threads = [&](int nv) { return dim3((unsigned)((n4 + nv * 32 - 1) / (nv * 32) * 32)); };
  ++g_kernel_launches;
  if (n4 <= 256) SRM_CUDA(launch_kernel(q8::rms_norm_fp8_kernel<1, XT, DT>, grid, threads(1), 0, st, p));
  else if (n4 <= 1024) SRM_CUDA(launch_kernel(q8::rms_norm_fp8_kernel<2, XT, DT>, grid, threads(2), 0, st, p));
  else SRM_CUDA(launch_kernel(q8::rms_norm_fp8_kernel<4, XT, DT>, grid, threads(4), 0, st, p));
  return SRM_OK;
}

// Tensor map of a row-major matrix, box_rows rows x 128 bytes, 128-byte swizzle. (Boxes may reach beyond the matrix: zeros are
// read there, nothing is written.)
int byte_map(CUtensorMap* map, CUtensorMapDataType type, int elem, const void* base, int64_t rows, int64_t cols, int64_t stride, int box_rows) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (fn == nullptr) { g_last_cuda_error = (int)cudaErrorNotSupported; return SRM_ERR_CUDA; }
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, pitch[1] = {(cuuint64_t)(stride * elem)};
  const cuuint32_t box[2] = {(cuuint32_t)(128 / elem), (cuuint32_t)box_rows}, one[2] = {1, 1};
  const CUresult r = fn(map, type, 2, const_cast<void*>(base), dims, pitch, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                        CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) { g_last_cuda_error = 10000 + (int)r; return SRM_ERR_CUDA; }
  return SRM_OK;
}

// Rows that stand alone may be given any stride; a tensor map wants a pitch that covers the row and is a multiple of 16 bytes.
int64_t map_stride(int64_t rows, int64_t cols, int64_t stride, int64_t elem) {
  return rows > 1 ? stride : (cols * elem + 15) / 16 * 16 / elem;
}

template <int NT, typename OT>
int launch_few(const g8::Args& g, const uint8_t* A, int64_t a_stride, const uint8_t* W, int64_t w_stride, int ranks, cudaStream_t st) {
  using F = g8::Few<NT>;
  const auto kernel = g8::gemm8_few_kernel<NT, OT>;
  int rc = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), F::kBytes);
  if (rc != SRM_OK) return rc;
  CUtensorMap ta, tw;
  if ((rc = byte_map(&ta, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, A, g.M, g.K, map_stride(g.M, g.K, a_stride, 1), NT)) != SRM_OK) return rc;
  if ((rc = byte_map(&tw, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, W, g.N, g.K, map_stride(g.N, g.K, w_stride, 1), 128)) != SRM_OK) return rc;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ranks, (unsigned)((g.N + 127) / 128), (unsigned)((g.M + NT - 1) / NT));
  cfg.blockDim = dim3(F::kThreads);
  cfg.dynamicSmemBytes = F::kBytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)ranks; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  ++g_kernel_launches;
  SRM_CUDA(cudaLaunchKernelEx(&cfg, kernel, ta, tw, g));
  return SRM_OK;
}

template <typename OT>
int launch_many(const g8::Args& g, const uint8_t* A, int64_t a_stride, const uint8_t* W, int64_t w_stride, int sms, cudaStream_t st) {
  const int elem = (int)sizeof(OT);
  const int64_t pitch = map_stride(g.M, g.N, g.out_stride, elem);
  const bool mapped = aligned(g.out, 16) && pitch * elem % 16 == 0;
  const auto kernel = mapped ? (g.bias != nullptr ? g8::gemm8_many_kernel<OT, true, true> : g8::gemm8_many_kernel<OT, true, false>)
                             : (g.bias != nullptr ? g8::gemm8_many_kernel<OT, false, true> : g8::gemm8_many_kernel<OT, false, false>);
  int rc = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), g8::Many<OT>::kBytes);
  if (rc != SRM_OK) return rc;
  CUtensorMap ta, tw, td;
  if ((rc = byte_map(&ta, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, A, g.M, g.K, map_stride(g.M, g.K, a_stride, 1), 128)) != SRM_OK) return rc;
  if ((rc = byte_map(&tw, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, W, g.N, g.K, map_stride(g.N, g.K, w_stride, 1), 128)) != SRM_OK) return rc;
  td = ta;
  if (mapped && (rc = byte_map(&td, elem == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, elem, g.out, g.M, g.N, pitch, 32)) != SRM_OK)
    return rc;
  const int64_t tiles = (g.M + 255) / 256 * ((g.N + 255) / 256), pairs = sms / 2;
  ++g_kernel_launches;
  SRM_CUDA(launch_kernel(kernel, dim3(2u * (unsigned)(tiles < pairs ? tiles : pairs)), dim3(g8::Many<OT>::kThreads), g8::Many<OT>::kBytes, st, ta, tw, td, g));
  return SRM_OK;
}

template <typename OT>
int launch_gemm8(const g8::Args& g, const uint8_t* A, int64_t a_stride, const uint8_t* W, int64_t w_stride, cudaStream_t st) {
  int sms = 0;
  const int rc = device_sm_count(&sms);
  if (rc != SRM_OK) return rc;
  const int64_t n_tiles = (g.N + 127) / 128, kb = (g.K + 127) / 128;
  // The 256 x 256 tiles of the pairs from 65 rows on where they are sixteen or more, from 385 rows on else. us (events around a launch, L2
  // flushed before it), few / many kernel: N = 6144, K = 1536, bf16 out (24 tiles to 256 rows): 100 rows 25 / 16, 256: 35 / 16, 768: 33 / 16;
  // N = 32000, K = 1024, fp32 out: 100 rows 29 / 23, 512: 82 / 37; N = 1024, K = 4096, bf16 out (4 tiles): 100 rows 14 / 22, 256: 23 / 23,
  // 384 (8): 25 / 24, 512: 33 / 23.
  const int64_t pair_tiles = (g.M + 255) / 256 * ((g.N + 255) / 256);
  if (g.N > 128 && g.M > 64 && (pair_tiles >= 16 || g.M > 384)) return launch_many<OT>(g, A, a_stride, W, w_stride, sms, st);
  const int nt = g.M <= 16 ? 16 : g.M <= 32 ? 32 : g.M <= 64 ? 64 : 128;
  const int64_t m_tiles = (g.M + nt - 1) / nt;
  // More tiles than a grid's y or z counts: the pairs walk over theirs in a loop.
  if (n_tiles > 65535 || m_tiles > 65535) return launch_many<OT>(g, A, a_stride, W, w_stride, sms, st);
  // Ranks for two CTAs per SM. us (as above) with / without: N = 1024, K = 4096, 27 rows 10 / 21, 200 rows 21 / 31; N = 6144, K = 1536,
  // 1 row 9.6 / 11.5.
  int ranks = 1;
  while (ranks < 8 && 2 * ranks <= kb && n_tiles * m_tiles * ranks * 2 <= 2 * sms) ranks *= 2;
  if (nt == 16) return launch_few<16, OT>(g, A, a_stride, W, w_stride, ranks, st);
  if (nt == 32) return launch_few<32, OT>(g, A, a_stride, W, w_stride, ranks, st);
  if (nt == 64) return launch_few<64, OT>(g, A, a_stride, W, w_stride, ranks, st);
  return launch_few<128, OT>(g, A, a_stride, W, w_stride, ranks, st);
}

// A block of up to 512 threads per row, two per SM; few rows of many ids: a cluster of blocks each, as long as all find room at once.
// us (events around a launch, L2 flushed before it) with / without: 1 row of 131072 29 / 36, 8 rows 48 / 139, 32 rows of 60000 94 / 135.
template <typename T>
int launch_sample(const smp::Args& p, cudaStream_t st) {
  int sms = 0;
  const int rc = device_sm_count(&sms);
  if (rc != SRM_OK) return rc;
  const int ids = p.V <= smp::kFewIds ? 128 : 512, stretches = (p.V + ids - 1) / ids;
  ++g_kernel_launches;
  int ranks = 1;
  while (ids == 512 && ranks < smp::kMaxRanks && stretches > 32 * ranks && 2 * ranks * p.R <= 2 * sms) ranks *= 2;
  if (ranks == 1) {
    const int warps = stretches < 16 ? stretches : 16;
    SRM_CUDA(launch_kernel(ids == 128 ? smp::sample_kernel<T, false, 4> : smp::sample_kernel<T, false, 16>, dim3((unsigned)p.R), dim3(32 * warps), 0, st,
                           p, stretches));
    return SRM_OK;
  }
  const int per_rank = (stretches + ranks - 1) / ranks, warps = per_rank < 16 ? per_rank : 16;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ranks, (unsigned)p.R);                  // (few rows)
  cfg.blockDim = dim3(32 * warps);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)ranks; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  SRM_CUDA(cudaLaunchKernelEx(&cfg, smp::sample_kernel<T, true, 16>, p, per_rank));
  return SRM_OK;
}

}  // namespace

extern "C" {

int srm_k_rms_norm_fp8(int64_t R, int32_t d, const void* d_x, int32_t x_dtype, int64_t x_stride, const void* d_delta,
                       int32_t delta_dtype, int64_t delta_stride, const float* d_g, float eps, void* d_sum, int64_t sum_stride,
                       uint8_t* d_q, int64_t q_stride, float* d_scale, int64_t scale_row, int64_t scale_blk, void* stream) {
  if (R < 0 || d < 1 || !dtype_ok(x_dtype) || !(eps >= 0.f)) return SRM_ERR_INVALID_ARG;
  if (d_delta != nullptr && !dtype_ok(delta_dtype)) return SRM_ERR_INVALID_ARG;
  if (d_delta == nullptr && d_sum != nullptr) return SRM_ERR_INVALID_ARG;
  if (d % 16 || d > 16384 || R > kMaxGrid) return SRM_ERR_UNSUPPORTED;
  if (R == 0) return SRM_OK;
  int rc;
  if ((rc = rows_ok(d_x, R, d, x_stride, dtype_bytes(x_dtype))) != SRM_OK) return rc;
  if (d_delta != nullptr && (rc = rows_ok(d_delta, R, d, delta_stride, dtype_bytes(delta_dtype))) != SRM_OK) return rc;
  if (d_sum == d_x && R > 1 && sum_stride != x_stride) return SRM_ERR_INVALID_ARG;      // (a row's sums over another row's x)
  if (d_sum != nullptr && (rc = rows_ok(d_sum, R, d, sum_stride, dtype_bytes(x_dtype))) != SRM_OK) return rc;
  if ((rc = rows_ok(d_q, R, d, q_stride, 1)) != SRM_OK) return rc;
  if ((rc = rows_ok(d_g, 1, d, d, 4)) != SRM_OK) return rc;
  if ((rc = written_scales_ok(d_scale, R, (d + 127) / 128, scale_row, scale_blk)) != SRM_OK) return rc;
  const q8::NormArgs p{R, d, d_x, x_stride, d_delta, delta_stride, d_g, eps, d_sum, sum_stride, d_q, q_stride, d_scale, scale_row, scale_blk};
  return with_type(x_dtype, [&](auto x) {
    return with_type(d_delta != nullptr ? delta_dtype : SRM_DTYPE_FP32,
                     [&](auto dl) { return launch_norm<decltype(x), decltype(dl)>(p, static_cast<cudaStream_t>(stream)); });
  });
}

int srm_k_quant_fp8(int64_t R, int64_t K, const void* d_x, int32_t x_dtype, int64_t x_stride, int32_t block_rows, uint8_t* d_q,
                    int64_t q_stride, float* d_scale, int64_t scale_row, int64_t scale_blk, void* stream) {
  if (R < 0 || K < 1 || !dtype_ok(x_dtype) || (block_rows != 1 && block_rows != 128)) return SRM_ERR_INVALID_ARG;
  const int64_t kb = (K + 127) / 128;
  if (K % 16 || kb > kMaxGrid || R > kMaxGrid) return SRM_ERR_UNSUPPORTED;
  const int64_t grid = block_rows == 1 ? (R * kb + q8::kQuantThreads / 16 - 1) / (q8::kQuantThreads / 16) : (R + 127) / 128 * kb;
  if (grid > kMaxGrid) return SRM_ERR_UNSUPPORTED;
  if (R == 0) return SRM_OK;
  int rc;
  if ((rc = rows_ok(d_x, R, K, x_stride, dtype_bytes(x_dtype))) != SRM_OK) return rc;
  if ((rc = rows_ok(d_q, R, K, q_stride, 1)) != SRM_OK) return rc;
  if ((rc = written_scales_ok(d_scale, (R + block_rows - 1) / block_rows, kb, scale_row, scale_blk)) != SRM_OK) return rc;
  const q8::QuantArgs p{R, K, d_x, x_stride, d_q, q_stride, d_scale, scale_row, scale_blk};
  return with_type(x_dtype, [&](auto x) -> int {
    using XT = decltype(x);
    ++g_kernel_launches;
    SRM_CUDA(launch_kernel(block_rows == 1 ? q8::quant_rows_kernel<XT> : q8::quant_tiles_kernel<XT>, dim3((unsigned)grid),
                           dim3(q8::kQuantThreads), 0, static_cast<cudaStream_t>(stream), p));
    return SRM_OK;
  });
}

int srm_k_gemm_fp8(int64_t M, int64_t N, int64_t K, const uint8_t* d_A, int64_t a_stride, const float* d_sa, int64_t sa_row,
                   int64_t sa_blk, const uint8_t* d_W, int64_t w_stride, const float* d_sw, int64_t sw_row, int64_t sw_blk,
                   const float* d_bias, int32_t accumulate, void* d_out, int32_t out_dtype, int64_t out_stride, uint32_t* d_status,
                   void* stream) {
  if (M < 0 || N < 1 || K < 1 || (accumulate != 0 && accumulate != 1)) return SRM_ERR_INVALID_ARG;
  if (out_dtype != SRM_DTYPE_FP32 && out_dtype != SRM_DTYPE_BF16) return SRM_ERR_INVALID_ARG;
  if (K % 16 || K > (1 << 20) || M > (1 << 30) || N > (1 << 30) || (accumulate && out_dtype != SRM_DTYPE_FP32)) return SRM_ERR_UNSUPPORTED;
  if ((M + 255) / 256 * ((N + 255) / 256) > 0x3fffffff) return SRM_ERR_UNSUPPORTED;      // (tiles are counted in 32 bits)
  if (M == 0) return SRM_OK;
  int rc;
  if ((rc = rows_ok(d_A, M, K, a_stride, 1)) != SRM_OK) return rc;
  if ((rc = rows_ok(d_W, N, K, w_stride, 1)) != SRM_OK) return rc;
  const int64_t kb = (K + 127) / 128;
  if ((rc = read_scales_ok(d_sa, M, kb, sa_row, sa_blk)) != SRM_OK || (rc = read_scales_ok(d_sw, (N + 127) / 128, kb, sw_row, sw_blk)) != SRM_OK) return rc;
  if (d_bias != nullptr && (rc = floats_ok(d_bias)) != SRM_OK) return rc;
  if (d_out == nullptr || (M > 1 && out_stride < N)) return SRM_ERR_INVALID_ARG;
  if (!aligned(d_out, (size_t)dtype_bytes(out_dtype)) || !aligned(d_status, 4)) return SRM_ERR_ALIGNMENT;
  const g8::Args g{M, N, K, d_sa, sa_row, sa_blk, d_sw, sw_row, sw_blk, d_bias, accumulate, d_out, out_stride, d_status};
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (out_dtype == SRM_DTYPE_FP32) return launch_gemm8<float>(g, d_A, a_stride, d_W, w_stride, st);
  return launch_gemm8<bf16>(g, d_A, a_stride, d_W, w_stride, st);
}

int srm_k_sample(int64_t R, int32_t V, const void* d_logits, int32_t logits_dtype, int64_t logits_stride, const float* d_u,
                 const float* d_temperature, const int32_t* d_top_k, const float* d_top_p, const float* d_min_p, int32_t* d_tok,
                 uint32_t* d_status, void* stream) {
  if (R < 0 || V < 1 || !dtype_ok(logits_dtype)) return SRM_ERR_INVALID_ARG;
  if (V > 262144 || R > kMaxGrid) return SRM_ERR_UNSUPPORTED;
  if (R == 0) return SRM_OK;
  if (d_logits == nullptr || d_u == nullptr || d_tok == nullptr || (R > 1 && logits_stride < V)) return SRM_ERR_INVALID_ARG;
  if (!aligned(d_logits, (size_t)dtype_bytes(logits_dtype)) || !aligned(d_u, 4) || !aligned(d_temperature, 4) || !aligned(d_top_k, 4) ||
      !aligned(d_top_p, 4) || !aligned(d_min_p, 4) || !aligned(d_tok, 4) || !aligned(d_status, 4))
    return SRM_ERR_ALIGNMENT;
  const smp::Args p{R, V, d_logits, logits_stride, d_u, d_temperature, d_top_k, d_top_p, d_min_p, d_tok, d_status};
  return with_type(logits_dtype, [&](auto t) { return launch_sample<decltype(t)>(p, static_cast<cudaStream_t>(stream)); });
}

}  // extern "C"
