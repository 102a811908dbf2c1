// 4-bit operators of include/dit_ops.h: argument checks, tensor maps, launch rules.
#include <algorithm>
#include <mutex>

#include "common.cuh"
#include "fp4_gemm.cuh"
#include "fp4_quant.cuh"
#include "ops_launch.h"

using namespace dit;

namespace {

constexpr int64_t kMaxSize = INT32_MAX - 1024;
constexpr int64_t kMaxCols = 1 << 30;            // of a row: places in it, a CTA's stride further on, are counted in 32 bits

int type_bytes(dit_type t) { return t == DIT_TYPE_F32 ? 4 : 2; }
bool type_ok(dit_type t) { return t == DIT_TYPE_F16 || t == DIT_TYPE_BF16 || t == DIT_TYPE_F32; }
bool aligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

std::mutex g_mutex;
struct Prepared { bool ready; int pairs; } g_prepared[kOpsMaxDevices];

template <class Kernel>
cudaError_t allow_smem(Kernel kernel, int bytes) {
  return cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
}
template <int EPI, int G>
cudaError_t allow_gemm() {
  cudaError_t e = allow_smem(&gemm_fp4_pair_kernel<EPI, G>, fgemm::Cfg<G>::SMEM_BYTES);
  if (e == cudaSuccess) e = allow_smem(&gemm_fp4_split_kernel<EPI, G, 16>, Fp4SplitCfg<16, G>::SMEM_BYTES);
  if (e == cudaSuccess) e = allow_smem(&gemm_fp4_split_kernel<EPI, G, 32>, Fp4SplitCfg<32, G>::SMEM_BYTES);
  if (e == cudaSuccess) e = allow_smem(&gemm_fp4_split_kernel<EPI, G, 64>, Fp4SplitCfg<64, G>::SMEM_BYTES);
  return e;
}

// The device's state for products; *pairs: CTA pairs of the pair kernel that are resident at once.
cudaError_t prepare(const OpsDevice& d, int* pairs) {
  std::lock_guard<std::mutex> lock(g_mutex);
  Prepared& s = g_prepared[d.index];
  if (!s.ready) {
    cudaError_t e;
    if ((e = allow_gemm<kBlkF16, 16>()) != cudaSuccess || (e = allow_gemm<kBlkBF16, 16>()) != cudaSuccess || (e = allow_gemm<kBlkF32, 16>()) != cudaSuccess ||
        (e = allow_gemm<kBlkF16, 32>()) != cudaSuccess || (e = allow_gemm<kBlkBF16, 32>()) != cudaSuccess || (e = allow_gemm<kBlkF32, 32>()) != cudaSuccess)
      return e;
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3(d.num_sms & ~1); lc.blockDim = dim3(fgemm::THREADS); lc.dynamicSmemBytes = fgemm::Cfg<16>::SMEM_BYTES;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = 2; at.val.clusterDim.y = 1; at.val.clusterDim.z = 1;
    lc.attrs = &at; lc.numAttrs = 1;
    int clusters = 0;
    if ((e = cudaOccupancyMaxActiveClusters(&clusters, reinterpret_cast<const void*>(&gemm_fp4_pair_kernel<kBlkF16, 16>), &lc)) != cudaSuccess) return e;
    s.pairs = std::max(1, std::min(clusters, d.num_sms / 2));
    s.ready = true;
  }
  *pairs = s.pairs;
  return cudaSuccess;
}

// Codes [rows, bytes]: boxes of 128 bytes x box_rows, 128-byte swizzle, zeros outside.
bool code_map(const OpsDevice& d, CUtensorMap* m, const void* ptr, uint64_t bytes, uint64_t rows, uint64_t pitch, uint32_t box_rows) {
  const cuuint64_t dims[2] = {bytes, rows};
  const cuuint64_t strides[1] = {pitch};
  const cuuint32_t box[2] = {128, box_rows};
  const cuuint32_t estr[2] = {1, 1};
  return d.encode(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Scale tiles [row tiles][chunks] of 512 bytes (128 words): boxes of box_chunks x box_tiles.
bool scale_map(const OpsDevice& d, CUtensorMap* m, const void* ptr, uint64_t tiles, uint64_t chunks, uint32_t box_chunks, uint32_t box_tiles) {
  const cuuint64_t dims[3] = {128, chunks, tiles};
  const cuuint64_t strides[2] = {512, 512 * chunks};
  const cuuint32_t box[3] = {128, box_chunks, box_tiles};
  const cuuint32_t estr[3] = {1, 1, 1};
  return d.encode(m, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Output matrix: boxes of 128 bytes x 32 rows, 128-byte swizzle.
bool out_map(const OpsDevice& d, CUtensorMap* m, void* ptr, dit_type type, uint64_t n, uint64_t rows, uint64_t ld) {
  const bool wide = type == DIT_TYPE_F32;
  const cuuint64_t dims[2] = {n, rows};
  const cuuint64_t strides[1] = {ld * (wide ? 4 : 2)};
  const cuuint32_t box[2] = {wide ? 32u : 64u, 32u};
  const cuuint32_t estr[2] = {1, 1};
  const CUtensorMapDataType t = wide ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : (type == DIT_TYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16);
  return d.encode(m, t, 2, ptr, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int EPI, int G, int BT>
cudaError_t launch_split(const CUtensorMap& tmA, const CUtensorMap& tmB, const dit_gemm_fp4_args& a, const Fp4GemmParams& p, int splits, cudaStream_t st) {
  using C = Fp4SplitCfg<BT, G>;
  const long long tiles = static_cast<long long>((p.N + 127) / 128) * ((p.M + BT - 1) / BT);
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3(static_cast<unsigned>(tiles * splits)); lc.blockDim = dim3(C::THREADS);
  lc.dynamicSmemBytes = C::SMEM_BYTES; lc.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = splits; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
  lc.attrs = at; lc.numAttrs = splits > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&lc, &gemm_fp4_split_kernel<EPI, G, BT>, tmA, tmB, static_cast<const uint8_t*>(a.a_scales), static_cast<const uint8_t*>(a.b_scales), p, splits);
}

template <int EPI, int G, int BT>
cudaError_t launch_split(const OpsDevice& d, const CUtensorMap& tmA, const CUtensorMap& tmB, const dit_gemm_fp4_args& a, const Fp4GemmParams& p, cudaStream_t st) {
  const long long tiles = static_cast<long long>((p.N + 127) / 128) * ((p.M + BT - 1) / BT);
  const int stages = (p.K + 255) / 256;
  // CTAs per tile: doubled up to two CTAs per SM as long as each keeps a stage of four or more; with 32 rows or fewer, beyond one per SM only
  // where each has more than eight stages to share (us for 1, 2, 4, 8: 144 tiles of 16 stages 12.6, 9.5, 17.2, 22.9; 72 of 16 13.0, 9.5, 12.5, 15.1;
  // 32 of 16 12.3, 8.4, 6.4, 6.8; with 64 rows 32 of 16 15.3, 12.9, 9.2, 9.5; 12 of 2 7.0, 8.7).
  int splits = 1;
  while (splits < 8 && tiles * 2 * splits <= 2ll * d.num_sms && stages >= std::max(4, 2 * splits) &&
         (BT == 64 || tiles * 2 * splits <= d.num_sms || stages > 8 * splits))
    splits *= 2;
  return launch_split<EPI, G, BT>(tmA, tmB, a, p, splits, st);
}

template <int EPI, int G>
cudaError_t launch_product(const OpsDevice& d, int pairs, const dit_gemm_fp4_args& a, Fp4GemmParams p, cudaStream_t st) {
  using S = Fp4Scales<G>;
  CUtensorMap tmA, tmB, tmSA, tmSB;
  const uint64_t bytes = (static_cast<uint64_t>(p.K) + 1) / 2;
  const long long tiles_n = (p.N + 127) / 128;
  const long long pair_tiles = static_cast<long long>((p.M + 255) / 256) * ((p.N + 255) / 256);
  // Few rows, or so few tiles of 128 x 64 that most of the pair kernel's would be missing: the split kernel.
  if (p.M <= 32 || 3 * tiles_n * ((p.M + 63) / 64) <= 2ll * d.num_sms) {
    const int bt = p.M <= 16 ? 16 : (p.M <= 32 ? 32 : 64);
    if (!code_map(d, &tmA, a.a, bytes, p.M, a.lda, bt) || !code_map(d, &tmB, a.b, bytes, p.N, a.ldb, 128)) return cudaErrorInvalidValue;
    if (bt == 16) return launch_split<EPI, G, 16>(d, tmA, tmB, a, p, st);
    if (bt == 32) return launch_split<EPI, G, 32>(d, tmA, tmB, a, p, st);
    return launch_split<EPI, G, 64>(d, tmA, tmB, a, p, st);
  }
  const uint64_t chunks = (static_cast<uint64_t>(p.K) + 4 * G - 1) / (4 * G);
  if (!code_map(d, &tmA, a.a, bytes, p.M, a.lda, 128) || !code_map(d, &tmB, a.b, bytes, p.N, a.ldb, 128) ||
      !scale_map(d, &tmSA, a.a_scales, (p.M + 127) / 128, chunks, S::TILES, 1) || !scale_map(d, &tmSB, a.b_scales, (p.N + 127) / 128, chunks, S::TILES, 2))
    return cudaErrorInvalidValue;
  {  // tile order: hold the panels of whichever operand costs fewer DRAM reads in L2 (as launch_gemm of the step does)
    const long long panel = 128ll * p.K, num_m = (p.M + 255) / 256, num_n = (p.N + 255) / 256;
    const long long fit = std::max(1ll, (38ll << 20) / panel);
    const long long rb = std::min(fit, num_m), cb = std::min(fit, num_n);
    const long long cost_rows = num_m * panel + num_n * panel * ((num_m + rb - 1) / rb);
    const long long cost_cols = num_n * panel + num_m * panel * ((num_n + cb - 1) / cb);
    p.band = cost_cols < cost_rows ? -static_cast<int>(cb) : static_cast<int>(rb);
  }
  CUtensorMap tmOut = tmA;                       // unused where the output is written directly
  if (p.vec_out && !out_map(d, &tmOut, a.out, a.out_type, p.N, p.M, a.ld_out)) return cudaErrorInvalidValue;
  const int grid = 2 * static_cast<int>(std::min<long long>(pair_tiles, pairs));
  return launch_overlapping(&gemm_fp4_pair_kernel<EPI, G>, dim3(grid), fgemm::THREADS, fgemm::Cfg<G>::SMEM_BYTES, st, tmA, tmB, tmSA, tmSB, tmOut, p);
}

template <int G>
cudaError_t dispatch_product(const OpsDevice& d, int pairs, const dit_gemm_fp4_args& a, const Fp4GemmParams& p, cudaStream_t st) {
  if (a.out_type == DIT_TYPE_F16) return launch_product<kBlkF16, G>(d, pairs, a, p, st);
  if (a.out_type == DIT_TYPE_BF16) return launch_product<kBlkBF16, G>(d, pairs, a, p, st);
  return launch_product<kBlkF32, G>(d, pairs, a, p, st);
}

template <int kType, int G, int kBytes, int THREADS>
cudaError_t launch_rows(const Fp4QuantParams& p, long long loads, cudaStream_t st) {
  constexpr int CTA = THREADS == 32 ? 256 : THREADS, PER = CTA / THREADS;
  const unsigned grid = (static_cast<unsigned>((static_cast<long long>(p.rows) + 127) / 128 * 128) + PER - 1) / PER;
  const long long each = (loads + THREADS - 1) / THREADS;
  if constexpr (kBytes == 32) {
    if (each <= 1) return launch_overlapping(&quantize_fp4_kernel<kType, G, kBytes, THREADS, 1>, dim3(grid), CTA, 0, st, p);
    if (each <= 2) return launch_overlapping(&quantize_fp4_kernel<kType, G, kBytes, THREADS, 2>, dim3(grid), CTA, 0, st, p);
    return launch_overlapping(&quantize_fp4_kernel<kType, G, kBytes, THREADS, 3>, dim3(grid), CTA, 0, st, p);
  } else {
    if (each <= 1) return launch_overlapping(&quantize_fp4_kernel<kType, G, kBytes, THREADS, 1>, dim3(grid), CTA, 0, st, p);
    if (each <= 2) return launch_overlapping(&quantize_fp4_kernel<kType, G, kBytes, THREADS, 2>, dim3(grid), CTA, 0, st, p);
    if (each <= 4) return launch_overlapping(&quantize_fp4_kernel<kType, G, kBytes, THREADS, 4>, dim3(grid), CTA, 0, st, p);
    return launch_overlapping(&quantize_fp4_kernel<kType, G, kBytes, THREADS, 6>, dim3(grid), CTA, 0, st, p);
  }
}
template <int kType, int G, int kBytes>
cudaError_t launch_quant(const Fp4QuantParams& p, cudaStream_t st) {
  // As few lanes per row as hold it in 96 bytes each: what a row's maximum costs grows with them.  (Loads of 32 bytes: 9216 x 12288 fp16 62 -> 49 us)
  constexpr int EPL = QuantIn<kType>::EPL * (kBytes == 32 ? 2 : 1), MOST = kBytes == 32 ? 3 : 6;
  const long long loads = (static_cast<long long>(p.cols) + EPL - 1) / EPL;
  if (loads <= 32 * MOST) return launch_rows<kType, G, kBytes, 32>(p, loads, st);
  if (loads <= 64 * MOST) return launch_rows<kType, G, kBytes, 64>(p, loads, st);
  if (loads <= 128 * MOST) return launch_rows<kType, G, kBytes, 128>(p, loads, st);
  if (loads <= 256 * MOST) return launch_rows<kType, G, kBytes, 256>(p, loads, st);
  return launch_rows<kType, G, kBytes, 512>(p, loads, st);
}
template <int kType, int G>
cudaError_t launch_quant(const Fp4QuantParams& p, int bytes, cudaStream_t st) {
  if (bytes == 32) return launch_quant<kType, G, 32>(p, st);
  return bytes == 16 ? launch_quant<kType, G, 16>(p, st) : launch_quant<kType, G, 0>(p, st);
}
template <int kType>
cudaError_t launch_quant(const Fp4QuantParams& p, int group, int bytes, cudaStream_t st) {
  return group == 16 ? launch_quant<kType, 16>(p, bytes, st) : launch_quant<kType, 32>(p, bytes, st);
}

template <int kType, bool kVec>
cudaError_t launch_weight(const Fp4QuantWeightParams& p, int group, cudaStream_t st) {
  const unsigned k_tiles = static_cast<unsigned>((static_cast<long long>(p.in_dim) + 127) / 128);
  const unsigned grid = static_cast<unsigned>((static_cast<long long>(p.out_dim) + 127) / 128 * 2) * k_tiles;
  if (group == 16) {
    cudaError_t e = cudaMemsetAsync(p.row_scales, 0, static_cast<size_t>(p.out_dim) * sizeof(float), st);
    if (e != cudaSuccess) return e;
    const unsigned columns = static_cast<unsigned>((static_cast<long long>(p.out_dim) + 63) / 64) * static_cast<unsigned>((static_cast<long long>(p.in_dim) + kColumnRows - 1) / kColumnRows);
    fp4_column_scales_kernel<kType, kVec><<<columns, 256, 0, st>>>(p);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    return launch_overlapping(&quantize_weight_fp4_kernel<kType, 16, kVec>, dim3(grid), 256, 0, st, p);
  }
  return launch_overlapping(&quantize_weight_fp4_kernel<kType, 32, kVec>, dim3(grid), 256, 0, st, p);
}

template <int kType, int G, int kBytes>
cudaError_t launch_values(const OpsDevice& d, const Fp4ValuesParams& p, cudaStream_t st) {
  constexpr int COLS = kBytes == 32 ? 512 : 256;
  auto ctas = [&](int rows) { return ((static_cast<long long>(p.rows) + rows - 1) / rows) * ((static_cast<long long>(p.cols) + COLS - 1) / COLS); };
  // Four rows per warp (9216 x 12288 fp16: 45 us; eight 46, 82 against 78 in fp32), two where those would not fill the device (77 x 2056: 1.6 us against 2.9
  // with eight).
  if (ctas(kValueWarps * 4) >= 4ll * d.num_sms)
    return launch_overlapping(&dequantize_fp4_kernel<kType, G, kBytes, 4>, dim3(static_cast<unsigned>(ctas(kValueWarps * 4))), kValueWarps * 32, 0, st, p);
  return launch_overlapping(&dequantize_fp4_kernel<kType, G, kBytes, 2>, dim3(static_cast<unsigned>(ctas(kValueWarps * 2))), kValueWarps * 32, 0, st, p);
}
template <int kType>
cudaError_t launch_values(const OpsDevice& d, const Fp4ValuesParams& p, int group, int bytes, cudaStream_t st) {
  if (bytes == 32) return group == 16 ? launch_values<kType, 16, 32>(d, p, st) : launch_values<kType, 32, 32>(d, p, st);
  if (bytes == 16) return group == 16 ? launch_values<kType, 16, 16>(d, p, st) : launch_values<kType, 32, 16>(d, p, st);
  return group == 16 ? launch_values<kType, 16, 0>(d, p, st) : launch_values<kType, 32, 0>(d, p, st);
}

// What a matrix's rows start on multiples of.
int row_alignment(const void* x, int64_t ld, dit_type type) {
  auto starts_at = [&](int n) { return aligned(x, n) && ld * type_bytes(type) % n == 0; };
  return starts_at(32) ? 32 : starts_at(16) ? 16 : 0;
}

dit_status status_of(cudaError_t e) { return e == cudaSuccess ? DIT_OK : DIT_ERR_CUDA; }

// Sizes of a quantised matrix.
dit_status check_matrix(int64_t rows, int64_t cols, int32_t group) {
  if (group != 16 && group != 32) return DIT_ERR_INVALID_ARG;
  if (rows < 0) return DIT_ERR_INVALID_ARG;
  if (cols < 1 || cols > kMaxCols || rows > kMaxSize) return DIT_ERR_SHAPE;
  // tiles of 128 x 128 (64 x 128 of a weight) are counted in 32 bits
  if (((rows + 127) / 128) * ((cols + 127) / 128) > INT32_MAX / 16) return DIT_ERR_SHAPE;
  return DIT_OK;
}
bool codes_ok(const void* codes, int64_t ld, int64_t cols) { return codes && aligned(codes, 16) && ld % 16 == 0 && ld >= (cols + 1) / 2; }
int chunks_of(int64_t cols, int32_t group) { return static_cast<int>((cols + 4 * group - 1) / (4 * group)); }

}  // namespace

// =============================================================================================== C ABI
extern "C" {

size_t dit_fp4_scale_bytes(int64_t rows, int64_t cols, int32_t group) {
  if (check_matrix(rows, cols, group) != DIT_OK) return 0;
  return static_cast<size_t>((rows + 127) / 128) * chunks_of(cols, group) * 512;
}

dit_status dit_quantize_fp4(const void* x, dit_type type, int64_t ld, int64_t rows, int64_t cols, int32_t group, void* codes, int64_t ld_codes,
                            void* scales, float* row_scales, void* stream) {
  if (!type_ok(type)) return DIT_ERR_INVALID_ARG;
  const dit_status bad = check_matrix(rows, cols, group);
  if (bad != DIT_OK) return bad;
  if (rows == 0) return DIT_OK;
  if (!x || !codes_ok(codes, ld_codes, cols) || !scales || !aligned(scales, 16) || (group == 16) != (row_scales != nullptr) || !aligned(row_scales, 4) ||
      ld < cols || !aligned(x, type_bytes(type)))
    return DIT_ERR_INVALID_ARG;
  OpsDevice d;
  const dit_status s = ops_device(&d);
  if (s != DIT_OK) return s;
  Fp4QuantParams p{};
  p.x = x; p.codes = static_cast<uint8_t*>(codes); p.scales = static_cast<uint8_t*>(scales); p.row_scales = row_scales;
  p.ld = ld; p.ld_codes = ld_codes; p.rows = static_cast<int>(rows); p.cols = static_cast<int>(cols); p.chunks = chunks_of(cols, group);
  const int bytes = row_alignment(x, ld, type);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (type == DIT_TYPE_F16) return status_of(launch_quant<0>(p, group, bytes, st));
  if (type == DIT_TYPE_BF16) return status_of(launch_quant<1>(p, group, bytes, st));
  return status_of(launch_quant<2>(p, group, bytes, st));
}

dit_status dit_quantize_weight_fp4(const void* w, dit_type type, int64_t ld, int64_t in_dim, int64_t out_dim, int32_t group, void* codes,
                                   int64_t ld_codes, void* scales, float* row_scales, void* stream) {
  if (!type_ok(type)) return DIT_ERR_INVALID_ARG;
  if (out_dim < 1) return DIT_ERR_SHAPE;
  const dit_status bad = check_matrix(out_dim, in_dim, group);
  if (bad != DIT_OK) return bad;
  if (!w || !codes_ok(codes, ld_codes, in_dim) || !scales || !aligned(scales, 16) || (group == 16) != (row_scales != nullptr) || !aligned(row_scales, 4) ||
      ld < out_dim || !aligned(w, type_bytes(type)))
    return DIT_ERR_INVALID_ARG;
  OpsDevice d;
  const dit_status s = ops_device(&d);
  if (s != DIT_OK) return s;
  Fp4QuantWeightParams p{};
  p.w = w; p.codes = static_cast<uint8_t*>(codes); p.scales = static_cast<uint8_t*>(scales); p.row_scales = row_scales;
  p.ld = ld; p.ld_codes = ld_codes; p.in_dim = static_cast<int>(in_dim); p.out_dim = static_cast<int>(out_dim); p.chunks = chunks_of(in_dim, group);
  const bool vec = aligned(w, 16) && ld * type_bytes(type) % 16 == 0;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (type == DIT_TYPE_F16) return status_of(vec ? launch_weight<0, true>(p, group, st) : launch_weight<0, false>(p, group, st));
  if (type == DIT_TYPE_BF16) return status_of(vec ? launch_weight<1, true>(p, group, st) : launch_weight<1, false>(p, group, st));
  return status_of(vec ? launch_weight<2, true>(p, group, st) : launch_weight<2, false>(p, group, st));
}

dit_status dit_dequantize_fp4(const void* codes, int64_t ld_codes, const void* scales, const float* row_scales, int64_t rows, int64_t cols,
                              int32_t group, void* out, dit_type out_type, int64_t ld_out, void* stream) {
  if (!type_ok(out_type)) return DIT_ERR_INVALID_ARG;
  const dit_status bad = check_matrix(rows, cols, group);
  if (bad != DIT_OK) return bad;
  if (rows == 0) return DIT_OK;
  if (!codes_ok(codes, ld_codes, cols) || !scales || !aligned(scales, 16) || !aligned(row_scales, 4) || !out || ld_out < cols || !aligned(out, type_bytes(out_type)))
    return DIT_ERR_INVALID_ARG;
  OpsDevice d;
  const dit_status s = ops_device(&d);
  if (s != DIT_OK) return s;
  Fp4ValuesParams p{};
  p.codes = static_cast<const uint8_t*>(codes); p.scales = static_cast<const uint8_t*>(scales); p.row_scales = row_scales; p.out = out;
  p.ld_codes = ld_codes; p.ld_out = ld_out; p.rows = static_cast<int>(rows); p.cols = static_cast<int>(cols); p.chunks = chunks_of(cols, group);
  const int bytes = row_alignment(out, ld_out, out_type);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (out_type == DIT_TYPE_F16) return status_of(launch_values<0>(d, p, group, bytes, st));
  if (out_type == DIT_TYPE_BF16) return status_of(launch_values<1>(d, p, group, bytes, st));
  return status_of(launch_values<2>(d, p, group, bytes, st));
}

dit_status dit_gemm_fp4(const dit_gemm_fp4_args* a, void* stream) {
  if (!a || !type_ok(a->out_type)) return DIT_ERR_INVALID_ARG;
  dit_status s = check_matrix(a->m, a->k, a->group);
  if (s != DIT_OK) return s;
  if (a->n < 1) return DIT_ERR_SHAPE;
  if ((s = check_matrix(a->n, a->k, a->group)) != DIT_OK || (s = check_matrix(a->m, a->n, a->group)) != DIT_OK) return s;
  if (a->m == 0) return DIT_OK;
  if (!codes_ok(a->a, a->lda, a->k) || !codes_ok(a->b, a->ldb, a->k) || !a->a_scales || !aligned(a->a_scales, 16) || !a->b_scales || !aligned(a->b_scales, 16) ||
      !aligned(a->a_rows, 4) || !aligned(a->b_rows, 4) || !aligned(a->bias, 4) || !a->out || a->ld_out < a->n || !aligned(a->out, type_bytes(a->out_type)))
    return DIT_ERR_INVALID_ARG;
  OpsDevice d;
  s = ops_device(&d);
  if (s != DIT_OK) return s;
  int pairs = 0;
  if (prepare(d, &pairs) != cudaSuccess) return DIT_ERR_CUDA;
  Fp4GemmParams p{};
  p.M = static_cast<int>(a->m); p.N = static_cast<int>(a->n); p.K = static_cast<int>(a->k);
  p.ra = a->a_rows; p.rb = a->b_rows; p.bias = a->bias; p.out = a->out; p.ld_out = a->ld_out;
  p.vec_out = aligned(a->out, 16) && a->ld_out * type_bytes(a->out_type) % 16 == 0;
  p.status = d.status;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  return status_of(a->group == 16 ? dispatch_product<16>(d, pairs, *a, p, st) : dispatch_product<32>(d, pairs, *a, p, st));
}

}  // extern "C"
