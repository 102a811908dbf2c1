// The context-free operators of include/dit_ops.h: argument checks, tensor maps, launch rules.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <mutex>
#include <type_traits>

#include "block_attention.cuh"
#include "block_gemm.cuh"
#include "block_quant.cuh"
#include "common.cuh"
#include "ops_launch.h"

using namespace dit;

namespace {

constexpr int kMaxDevices = kOpsMaxDevices;
constexpr int64_t kMaxSize = INT32_MAX - 1024;
// selecting kernel: means of eight query blocks, then the scores of one to eight rows
constexpr int kSelectFixedSmem = kSelectRows * kSelectPitch * 8;
constexpr int kSelectSmemMax = kSelectFixedSmem + kMaxKeyBlocks * 8;

// One status word per device, for waits that ran out.  In host code its name is a handle; the device
// address is looked up once per device, with that device current.
static __device__ int g_ops_status;

struct DeviceState {
  bool ready;
  int index, num_sms, pairs;                  // pairs: CTA pairs of the pair kernel that are resident at once
  int* status;
};
std::mutex g_mutex;
DeviceState g_device[kMaxDevices];
EncodeTiledFn g_encode = nullptr;

template <class Kernel>
cudaError_t allow_smem(Kernel kernel, int bytes) {
  return cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
}
template <int EPI>
cudaError_t allow_gemm() {
  cudaError_t e = allow_smem(&gemm_block128_pair_kernel<EPI>, bgemm::Cfg<EPI>::SMEM_BYTES);
  if (e == cudaSuccess) e = allow_smem(&gemm_block128_split_kernel<EPI, 16>, SplitCfg<16>::SMEM_BYTES);
  if (e == cudaSuccess) e = allow_smem(&gemm_block128_split_kernel<EPI, 32>, SplitCfg<32>::SMEM_BYTES);
  if (e == cudaSuccess) e = allow_smem(&gemm_block128_split_kernel<EPI, 64>, SplitCfg<64>::SMEM_BYTES);
  return e;
}

template <int D, bool BF16>
cudaError_t allow_attention() {
  cudaError_t e = allow_smem(&block_attention_kernel<D, BF16>, BlockAttnCfg<D>::SMEM_BYTES);
  if (e == cudaSuccess) e = allow_smem(&block_rows_kernel<D, BF16>, BlockRowsCfg<D>::SMEM_BYTES);
  return e;
}

// The current device's state, prepared on its first use.  *unsupported is set on anything but compute capability 10.x.
cudaError_t device_state(const DeviceState** out, bool* unsupported) {
  *unsupported = false;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(g_mutex);
  DeviceState& s = g_device[dev];
  if (!s.ready) {
    int major = 0;
    if ((e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev)) != cudaSuccess) return e;
    if (major != 10) { *unsupported = true; return cudaErrorNotSupported; }
    if ((e = cudaDeviceGetAttribute(&s.num_sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
    if (!g_encode) {
      void* fn = nullptr;
      cudaDriverEntryPointQueryResult found;
      if ((e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found)) != cudaSuccess) return e;
      if (!fn || found != cudaDriverEntryPointSuccess) return cudaErrorNotSupported;
      g_encode = reinterpret_cast<EncodeTiledFn>(fn);
    }
    void* p = nullptr;
    if ((e = cudaGetSymbolAddress(&p, g_ops_status)) != cudaSuccess) return e;
    s.status = static_cast<int*>(p);
    if ((e = allow_gemm<kBlkF16>()) != cudaSuccess || (e = allow_gemm<kBlkBF16>()) != cudaSuccess || (e = allow_gemm<kBlkF32>()) != cudaSuccess ||
        (e = allow_gemm<kBlkGeluF16>()) != cudaSuccess || (e = allow_gemm<kBlkGateResidF32>()) != cudaSuccess)
      return e;
    if ((e = allow_attention<64, false>()) != cudaSuccess || (e = allow_attention<64, true>()) != cudaSuccess ||
        (e = allow_attention<128, false>()) != cudaSuccess || (e = allow_attention<128, true>()) != cudaSuccess ||
        (e = allow_smem(&block_select_kernel, kSelectSmemMax)) != cudaSuccess)
      return e;
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3(s.num_sms & ~1); lc.blockDim = dim3(bgemm::THREADS); lc.dynamicSmemBytes = bgemm::Cfg<kBlkF16>::SMEM_BYTES;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = 2; at.val.clusterDim.y = 1; at.val.clusterDim.z = 1;
    lc.attrs = &at; lc.numAttrs = 1;
    int clusters = 0;
    if ((e = cudaOccupancyMaxActiveClusters(&clusters, reinterpret_cast<const void*>(&gemm_block128_pair_kernel<kBlkF16>), &lc)) != cudaSuccess) return e;
    s.pairs = std::max(1, std::min(clusters, s.num_sms / 2));
    s.index = dev;
    s.ready = true;
  }
  *out = &s;
  return cudaSuccess;
}

dit_status ready(const DeviceState** s) {
  bool unsupported = false;
  const cudaError_t e = device_state(s, &unsupported);
  if (unsupported) return DIT_ERR_UNSUPPORTED_ARCH;
  return e == cudaSuccess ? DIT_OK : DIT_ERR_CUDA;
}

int type_bytes(dit_type t) { return t == DIT_TYPE_F32 ? 4 : 2; }
bool type_ok(dit_type t) { return t == DIT_TYPE_F16 || t == DIT_TYPE_BF16 || t == DIT_TYPE_F32; }
bool aligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// Byte matrix [rows, inner] with `pitch` bytes between rows: boxes of 128 bytes x box_rows, 128-byte swizzle, zeros outside.
bool byte_map(CUtensorMap* m, const void* ptr, uint64_t inner, uint64_t rows, uint64_t pitch, uint32_t box_rows) {
  const cuuint64_t dims[2] = {inner, rows};
  const cuuint64_t strides[1] = {pitch};
  const cuuint32_t box[2] = {128, box_rows};
  const cuuint32_t estr[2] = {1, 1};
  return g_encode(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Output matrix: boxes of 128 bytes x 32 rows, 128-byte swizzle.
bool out_map(CUtensorMap* m, const BlockProduct& b, const void* matrix) {
  const bool wide = b.epilogue == kBlkF32 || b.epilogue == kBlkGateResidF32;
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(b.n), static_cast<cuuint64_t>(b.m)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(b.ld_out) * (wide ? 4 : 2)};
  const cuuint32_t box[2] = {wide ? 32u : 64u, 32u};
  const cuuint32_t estr[2] = {1, 1};
  const CUtensorMapDataType type = wide ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : (b.epilogue == kBlkBF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16);
  return g_encode(m, type, 2, const_cast<void*>(matrix), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// 16-bit matrix [rows, cols] with row stride ld: boxes of 64 columns x box_rows rows, 128-byte swizzle, zeros outside.
bool half_map(CUtensorMap* m, const void* ptr, uint64_t cols, uint64_t rows, uint64_t ld, uint32_t box_rows = 128) {
  const cuuint64_t dims[2] = {cols, rows};
  const cuuint64_t strides[1] = {ld * 2};
  const cuuint32_t box[2] = {64, box_rows};
  const cuuint32_t estr[2] = {1, 1};
  return g_encode(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Checks what the selector and the attention share and lays the batch out.  `values`: v is needed as well.
dit_status plan_batch(const dit_attention_batch* a, bool values, BlockBatch* b) {
  if (!a || a->n_requests < 0 || a->n_heads < 1 || (a->type != DIT_TYPE_F16 && a->type != DIT_TYPE_BF16)) return DIT_ERR_INVALID_ARG;
  if (a->head_dim != 64 && a->head_dim != 128) return DIT_ERR_SHAPE;
  if (a->n_requests > DIT_MAX_REQUESTS) return DIT_ERR_CAPACITY;
  if (a->n_requests > 0 && (!a->q_lens || !a->kv_lens)) return DIT_ERR_INVALID_ARG;
  if (static_cast<int64_t>(a->n_heads) * a->head_dim > (1 << 20)) return DIT_ERR_SHAPE;
  int64_t q = 0, kv = 0, qb = 0, kb = 0;
  b->n = a->n_requests;
  for (int r = 0; r <= a->n_requests; ++r) {
    b->cu_q[r] = static_cast<int>(q); b->cu_kv[r] = static_cast<int>(kv);
    b->first_qblock[r] = static_cast<int>(qb); b->first_kblock[r] = static_cast<int>(kb);
    if (r == a->n_requests) break;
    if (a->q_lens[r] < 0 || a->kv_lens[r] < 0) return DIT_ERR_INVALID_ARG;
    const int64_t kblocks = (static_cast<int64_t>(a->kv_lens[r]) + 127) / 128;
    if (kblocks > kMaxKeyBlocks) return DIT_ERR_SHAPE;
    q += a->q_lens[r]; kv += a->kv_lens[r];
    qb += (static_cast<int64_t>(a->q_lens[r]) + 127) / 128; kb += kblocks;
    if (q > kMaxSize || kv > kMaxSize) return DIT_ERR_SHAPE;
    b->order[r] = r;
  }
  for (int i = 1; i < b->n; ++i)                 // requests with the most query rows first (insertion sort: stable, at most 64)
    for (int j = i; j > 0 && a->q_lens[b->order[j]] > a->q_lens[b->order[j - 1]]; --j) std::swap(b->order[j], b->order[j - 1]);
  const int64_t width = static_cast<int64_t>(a->n_heads) * a->head_dim;
  auto matrix = [&](const void* p, int64_t ld, int64_t rows) { return rows == 0 || (p && aligned(p, 16) && ld >= width && ld % 8 == 0); };
  if (!matrix(a->q, a->ld_q, q) || !matrix(a->k, a->ld_k, kv) || (values && !matrix(a->v, a->ld_v, kv))) return DIT_ERR_INVALID_ARG;
  // grids are counted in 32 bits
  if ((qb + kb) * a->n_heads > INT32_MAX / 16) return DIT_ERR_SHAPE;
  return DIT_OK;
}

template <int D, bool BF16>
cudaError_t launch_rows(const CUtensorMap& tmK, const CUtensorMap& tmV, const BlockAttnParams& p, const dit_attention_batch& a, const BlockBatch& b,
                        int splits, cudaStream_t st) {
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3(static_cast<unsigned>(b.n) * a.n_heads * splits); lc.blockDim = dim3(BlockRowsCfg<D>::THREADS);
  lc.dynamicSmemBytes = BlockRowsCfg<D>::SMEM_BYTES; lc.stream = st;
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = splits; at.val.clusterDim.y = 1; at.val.clusterDim.z = 1;
  lc.attrs = &at; lc.numAttrs = splits > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&lc, &block_rows_kernel<D, BF16>, tmK, tmV, p, static_cast<const uint16_t*>(a.q), static_cast<long long>(a.ld_q), b, splits);
}

template <int D, bool BF16>
cudaError_t launch_attend(const DeviceState& d, const dit_attention_batch& a, const BlockBatch& b, const BlockAttnParams& p, cudaStream_t st) {
  const uint64_t width = static_cast<uint64_t>(a.n_heads) * D;
  const int q_rows = b.cu_q[b.n], kv_rows = b.cu_kv[b.n];
  int most = 0, qblocks = 0, longest = 0;
  for (int r = 0; r < b.n; ++r) {
    const int rows = b.cu_q[r + 1] - b.cu_q[r];
    most = std::max(most, rows);
    longest = std::max(longest, b.first_kblock[r + 1] - b.first_kblock[r]);
    qblocks += (rows + BlockAttnCfg<D>::Q_ROWS - 1) / BlockAttnCfg<D>::Q_ROWS;
  }
  CUtensorMap tmQ, tmK, tmV;
  // without keys nothing is loaded; the maps still have to describe some memory
  const void* k = kv_rows > 0 ? a.k : a.q;
  const void* v = kv_rows > 0 ? a.v : a.q;
  const uint32_t box = most <= kRowsMax ? kRowsTile : 128;
  if (!half_map(&tmK, k, width, std::max(kv_rows, 1), kv_rows > 0 ? a.ld_k : a.ld_q, box) ||
      !half_map(&tmV, v, width, std::max(kv_rows, 1), kv_rows > 0 ? a.ld_v : a.ld_q, box))
    return cudaErrorInvalidValue;
  if (most <= kRowsMax) {
    // A cluster of CTAs per (request, head): the largest power of two with which all are resident at once, two CTAs per
    // SM, and no more than there are blocks to share (96 items, 16 blocks each: 1, 2, 3, 4 CTAs 27, 20, 27, 27 us; clusters
    // of three do not pack into the SMs' clusters, four of 96 need a second wave).
    const int items = b.n * a.n_heads;
    const long long listed = std::min<long long>(longest, p.ld_index);
    int splits = 1;
    while (splits < 8 && 2 * splits <= listed && 2ll * splits * items <= 2ll * d.num_sms) splits *= 2;
    return launch_rows<D, BF16>(tmK, tmV, p, a, b, splits, st);
  }
  if (!half_map(&tmQ, a.q, width, q_rows, a.ld_q)) return cudaErrorInvalidValue;
  BlockAttnParams q = p;
  q.items = qblocks * a.n_heads;
  q.wide_out = aligned(p.out, 32) && p.ld_out % 16 == 0;
  block_attention_kernel<D, BF16><<<std::min(q.items, d.num_sms), BlockAttnCfg<D>::THREADS, BlockAttnCfg<D>::SMEM_BYTES, st>>>(tmQ, tmK, tmV, q, b);
  return cudaGetLastError();
}

const SeqInfo kNoSeq{};

template <int EPI, int BT>
cudaError_t launch_split(const CUtensorMap& tmA, const CUtensorMap& tmB, const BlockGemmParams& p, const SeqInfo& seq, int splits, cudaStream_t st) {
  const long long tiles = static_cast<long long>((p.N + 127) / 128) * ((p.M + BT - 1) / BT);
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3(static_cast<unsigned>(tiles * splits)); lc.blockDim = dim3(SplitCfg<BT>::THREADS);
  lc.dynamicSmemBytes = SplitCfg<BT>::SMEM_BYTES; lc.stream = st;
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = splits; at.val.clusterDim.y = 1; at.val.clusterDim.z = 1;
  lc.attrs = &at; lc.numAttrs = splits > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&lc, &gemm_block128_split_kernel<EPI, BT>, tmA, tmB, p, seq, splits);
}

template <int EPI>
cudaError_t launch_product(const DeviceState& d, const BlockProduct& b, BlockGemmParams p, const SeqInfo& seq, cudaStream_t st) {
  CUtensorMap tmA, tmB;
  const long long tiles_n = (p.N + 127) / 128;
  const int groups = (p.K + 127) / 128;
  const int rows = b.plan_m;
  const long long pair_tiles = static_cast<long long>((p.M + 255) / 256) * ((p.N + 255) / 256);
  // The pair kernel moves residual rows in boxes of 32 columns and reads bias and gates in fours.
  const bool resid_ok = EPI != kBlkGateResidF32 || (p.vec_out && aligned(p.resid, 16) && aligned(p.bias, 16) && aligned(p.gate, 16) && p.gate_stride % 4 == 0 && p.N % 32 == 0);
  // Few rows, or a product with so few tiles of 128 x 64 that most of the pair kernel's 256 x 256 ones would be missing: the split
  // kernel.  Measured, us, split against pair: n 3072, k 3072: m 64 9 / 15, m 128 11 / 16, m 256 17 / 16; n 3072, k 12288:
  // m 64 14 / 45, m 256 37 / 45, m 512 51 / 46; n 9216, k 3072: m 64 14 / 16, m 128 17 / 17, m 256 21 / 17.
  if (rows <= 32 || 3 * tiles_n * ((rows + 63) / 64) <= 2ll * d.num_sms || !resid_ok) {
    const int bt = rows <= 16 ? 16 : (rows <= 32 ? 32 : 64);
    const long long tiles = tiles_n * ((rows + bt - 1) / bt);
    // CTAs per tile: doubled up to about four CTAs per three SMs as long as each keeps two groups, and up to two per SM as long as
    // each keeps twelve (us for 1, 2, 4, 8: 24 tiles of 24 groups 11, 8, 6, 7; 72 tiles of 24 groups 11, 9, 11, 15;
    // 24 tiles of 96 groups 35, 21, 12, 10; 144 tiles of 24 groups 11.6, 10.9, 17, 25)
    int splits = 1;
    while (splits < 8) {
      const long long ctas = tiles * 2 * splits, each = groups / (2 * splits);
      if (!(3 * ctas <= 4ll * d.num_sms ? each >= 2 : (ctas <= 2ll * d.num_sms && each >= 12))) break;
      splits *= 2;
    }
    if (!byte_map(&tmA, b.a, p.K, p.M, b.lda, bt) || !byte_map(&tmB, b.b, p.K, p.N, b.ldb, 128)) return cudaErrorInvalidValue;
    if (bt == 16) return launch_split<EPI, 16>(tmA, tmB, p, seq, splits, st);
    if (bt == 32) return launch_split<EPI, 32>(tmA, tmB, p, seq, splits, st);
    return launch_split<EPI, 64>(tmA, tmB, p, seq, splits, st);
  }
  if (!byte_map(&tmA, b.a, p.K, p.M, b.lda, 128) || !byte_map(&tmB, b.b, p.K, p.N, b.ldb, 128)) return cudaErrorInvalidValue;
  {  // tile order: hold the panels of whichever operand costs fewer DRAM reads in L2 (as launch_gemm of the step does)
    const long long panel = 256ll * p.K, num_m = (p.M + 255) / 256, num_n = (p.N + 255) / 256;
    const long long fit = std::max(1ll, (38ll << 20) / panel);
    const long long rb = std::min(fit, num_m), cb = std::min(fit, num_n);
    const long long cost_rows = num_m * panel + num_n * panel * ((num_m + rb - 1) / rb);
    const long long cost_cols = num_n * panel + num_m * panel * ((num_n + cb - 1) / cb);
    p.band = cost_cols < cost_rows ? -static_cast<int>(cb) : static_cast<int>(rb);
  }
  const int grid = 2 * static_cast<int>(std::min<long long>(pair_tiles, d.pairs));
  CUtensorMap tmOut = tmA, tmResid = tmA;        // unused where the output is written directly, without a residual
  if (p.vec_out && !out_map(&tmOut, b, b.out)) return cudaErrorInvalidValue;
  if (EPI == kBlkGateResidF32 && !out_map(&tmResid, b, b.resid)) return cudaErrorInvalidValue;
  gemm_block128_pair_kernel<EPI><<<grid, bgemm::THREADS, bgemm::Cfg<EPI>::SMEM_BYTES, st>>>(tmA, tmB, tmOut, tmResid, p, seq);
  return cudaGetLastError();
}

template <int kType>
cudaError_t launch_quant(const QuantParams& p, long long tasks, bool vec, cudaStream_t st) {
  const unsigned grid = static_cast<unsigned>((tasks + kQuantBlockWarps - 1) / kQuantBlockWarps);
  if (vec) quantize_block128_kernel<kType, true><<<grid, kQuantBlockWarps * 32, 0, st>>>(p);
  else quantize_block128_kernel<kType, false><<<grid, kQuantBlockWarps * 32, 0, st>>>(p);
  return cudaGetLastError();
}
template <int kType>
cudaError_t launch_quant_weight(const QuantWeightParams& p, bool vec, cudaStream_t st) {
  const unsigned grid = static_cast<unsigned>(static_cast<long long>(p.in_groups) * ((p.out_dim + 127) / 128));
  if (vec) quantize_weight_block128_kernel<kType, true><<<grid, 256, 0, st>>>(p);
  else quantize_weight_block128_kernel<kType, false><<<grid, 256, 0, st>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_select(const dit_attention_batch& a, const BlockBatch& b, BlockSelectParams p, int32_t* index, int32_t* count, int64_t ld_index,
                          void* workspace, cudaStream_t st) {
  p.q = static_cast<const uint16_t*>(a.q); p.k = static_cast<const uint16_t*>(a.k);
  p.ld_q = a.ld_q; p.ld_k = a.ld_k;
  p.n_heads = a.n_heads; p.head_dim = a.head_dim; p.width = a.n_heads * a.head_dim;
  const int q_blocks = b.first_qblock[b.n], k_blocks = b.first_kblock[b.n];
  p.q_mean = static_cast<double*>(workspace);
  p.k_mean = p.q_mean + static_cast<size_t>(q_blocks) * p.width;
  p.index = index; p.count = count; p.ld_index = ld_index;
  int longest = 1;
  for (int r = 0; r < b.n; ++r) longest = std::max(longest, b.first_kblock[r + 1] - b.first_kblock[r]);
  p.rows = std::max(1, std::min(kSelectRows, (kSelectSmemMax - kSelectFixedSmem) / (longest * 8)));
  const unsigned grid = static_cast<unsigned>(q_blocks + k_blocks) * ((p.width + 255) / 256);
  if (a.type == DIT_TYPE_BF16) block_means_kernel<true><<<grid, 256, 0, st>>>(p, b);
  else block_means_kernel<false><<<grid, 256, 0, st>>>(p, b);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  unsigned groups = 0;
  for (int r = 0; r < b.n; ++r) groups += (b.first_qblock[r + 1] - b.first_qblock[r] + p.rows - 1) / p.rows;
  block_select_kernel<<<groups * a.n_heads, kSelectThreads, kSelectFixedSmem + static_cast<size_t>(p.rows) * longest * 8, st>>>(p, b);
  return cudaGetLastError();
}

cudaError_t launch_block_attention(const dit_attention_batch& a, const BlockBatch& b, const int32_t* index, const int32_t* count, int64_t ld_index,
                                   float scale, void* out, int64_t ld_out, int* status, bool clamp, const DeviceState& d, cudaStream_t st) {
  BlockAttnParams p{};
  p.out = out; p.ld_out = ld_out; p.index = index; p.count = count; p.ld_index = ld_index; p.n_heads = a.n_heads;
  p.scale_log2 = 1.4426950408889634f * (scale > 0.f ? scale : 1.0f / sqrtf(static_cast<float>(a.head_dim)));
  p.status = status ? status : d.status;
  p.clamp = clamp;
  if (a.head_dim == 128) return a.type == DIT_TYPE_BF16 ? launch_attend<128, true>(d, a, b, p, st) : launch_attend<128, false>(d, a, b, p, st);
  return a.type == DIT_TYPE_BF16 ? launch_attend<64, true>(d, a, b, p, st) : launch_attend<64, false>(d, a, b, p, st);
}

}  // namespace

namespace dit {

cudaError_t ops_prepare_device() {
  const DeviceState* d;
  bool unsupported;
  return device_state(&d, &unsupported);
}

dit_status ops_device(OpsDevice* d) {
  const DeviceState* state;
  const dit_status s = ready(&state);
  if (s != DIT_OK) return s;
  *d = OpsDevice{state->index, state->num_sms, state->status, g_encode};
  return DIT_OK;
}

cudaError_t launch_block_product(const BlockProduct& b, const SeqInfo& seq, cudaStream_t st) {
  const int elem = (b.epilogue == kBlkF32 || b.epilogue == kBlkGateResidF32) ? 4 : 2;
  const bool vec_out = aligned(b.out, 16) && b.ld_out * elem % 16 == 0;
  if (b.epilogue == kBlkGeluF16 && !vec_out) return cudaErrorInvalidValue;     // (the step's widths are multiples of 64)
  const DeviceState* d;
  bool unsupported;
  const cudaError_t e = device_state(&d, &unsupported);
  if (e != cudaSuccess) return e;
  BlockGemmParams p{};
  p.M = b.m; p.N = b.n; p.K = b.k;
  p.sa = b.a_scales; p.sb = b.b_scales; p.bias = b.bias; p.out = b.out;
  p.ld_sa = b.ld_a_scales; p.ld_out = b.ld_out;
  p.vec_out = vec_out;
  p.status = b.status ? b.status : d->status;
  p.row0 = b.row0; p.resid = b.resid; p.gate = b.gate; p.gate_stride = b.gate_stride;
  switch (b.epilogue) {
    case kBlkF16: return launch_product<kBlkF16>(*d, b, p, seq, st);
    case kBlkBF16: return launch_product<kBlkBF16>(*d, b, p, seq, st);
    case kBlkF32: return launch_product<kBlkF32>(*d, b, p, seq, st);
    case kBlkGeluF16: return launch_product<kBlkGeluF16>(*d, b, p, seq, st);
    case kBlkGateResidF32: return launch_product<kBlkGateResidF32>(*d, b, p, seq, st);
  }
  return cudaErrorInvalidValue;
}

cudaError_t launch_quantize_rows(const void* x, dit_type type, long long ld, long long rows, long long cols, void* codes,
                                 long long ld_codes, float* scales, long long ld_scales, cudaStream_t st) {
  const DeviceState* d;
  bool unsupported;
  const cudaError_t e = device_state(&d, &unsupported);
  if (e != cudaSuccess) return e;
  QuantParams p{};
  p.x = x; p.codes = static_cast<uint8_t*>(codes); p.scales = scales;
  p.ld = ld; p.ld_codes = ld_codes; p.ld_scales = ld_scales;
  p.rows = static_cast<int>(rows); p.cols = static_cast<int>(cols); p.groups = static_cast<int>((cols + 127) / 128);
  // runs of 32 rows per warp once that fills the device, of 8 below
  p.rows_per_task = (rows + 31) / 32 * p.groups >= 16ll * d->num_sms ? 32 : 8;
  const long long tasks = (rows + p.rows_per_task - 1) / p.rows_per_task * p.groups;
  if (tasks > 8ll * INT32_MAX - 8) return cudaErrorInvalidValue;
  const bool vec = aligned(x, 16) && ld * type_bytes(type) % 16 == 0;
  if (type == DIT_TYPE_F16) return launch_quant<0>(p, tasks, vec, st);
  if (type == DIT_TYPE_BF16) return launch_quant<1>(p, tasks, vec, st);
  return launch_quant<2>(p, tasks, vec, st);
}

cudaError_t launch_quantize_weight(const void* w, dit_type type, long long ld, int in_dim, int out_dim, void* codes, long long ld_codes,
                                   float* scales, cudaStream_t st) {
  QuantWeightParams p{};
  p.w = w; p.codes = static_cast<uint8_t*>(codes); p.scales = scales; p.ld = ld; p.ld_codes = ld_codes;
  p.in_dim = in_dim; p.out_dim = out_dim; p.in_groups = (in_dim + 127) / 128;
  const bool vec = aligned(w, 16) && ld * type_bytes(type) % 16 == 0;
  if (type == DIT_TYPE_F16) return launch_quant_weight<0>(p, vec, st);
  if (type == DIT_TYPE_BF16) return launch_quant_weight<1>(p, vec, st);
  return launch_quant_weight<2>(p, vec, st);
}

dit_status run_block_attention(const dit_attention_batch* a, const int32_t* block_index, const int32_t* block_count, int64_t ld_index,
                               float scale, void* out, int64_t ld_out, int* status, bool clamp, cudaStream_t st) {
  BlockBatch b;
  dit_status s = plan_batch(a, true, &b);
  if (s != DIT_OK) return s;
  if (b.cu_q[b.n] == 0) return DIT_OK;
  if (!block_index || !block_count || !out || ld_index < 1) return DIT_ERR_INVALID_ARG;
  if (!aligned(block_index, 4) || !aligned(block_count, 4) || !aligned(out, 16) || ld_out % 8 || ld_out < static_cast<int64_t>(a->n_heads) * a->head_dim)
    return DIT_ERR_INVALID_ARG;
  if (!(scale >= 0.f) || !(scale <= 2.0e38f)) return DIT_ERR_INVALID_ARG;      // scale * log2(e) has to be finite
  const DeviceState* d;
  s = ready(&d);
  if (s != DIT_OK) return s;
  return launch_block_attention(*a, b, block_index, block_count, ld_index, scale, out, ld_out, status, clamp, *d, st) == cudaSuccess ? DIT_OK : DIT_ERR_CUDA;
}

}  // namespace dit

// =============================================================================================== C ABI
extern "C" {

dit_status dit_quantize_block128(const void* x, dit_type type, int64_t ld, int64_t rows, int64_t cols, void* codes,
                                 int64_t ld_codes, float* scales, int64_t ld_scales, void* stream) {
  if (rows < 0 || !type_ok(type)) return DIT_ERR_INVALID_ARG;
  if (cols < 1 || cols > kMaxSize || rows > kMaxSize) return DIT_ERR_SHAPE;
  if (rows == 0) return DIT_OK;
  if (!x || !codes || !scales) return DIT_ERR_INVALID_ARG;
  if (ld < cols || ld_codes < cols || ld_codes % 16 || ld_scales < rows) return DIT_ERR_INVALID_ARG;
  if (!aligned(x, type_bytes(type)) || !aligned(codes, 16) || !aligned(scales, 4)) return DIT_ERR_INVALID_ARG;
  const DeviceState* d;
  const dit_status s = ready(&d);
  if (s != DIT_OK) return s;
  return launch_quantize_rows(x, type, ld, rows, cols, codes, ld_codes, scales, ld_scales, static_cast<cudaStream_t>(stream)) == cudaSuccess
             ? DIT_OK : DIT_ERR_CUDA;
}

dit_status dit_quantize_weight_block128(const void* w, dit_type type, int64_t ld, int64_t in_dim, int64_t out_dim, void* codes,
                                        int64_t ld_codes, float* scales, void* stream) {
  if (!type_ok(type)) return DIT_ERR_INVALID_ARG;
  if (in_dim < 1 || out_dim < 1 || in_dim > kMaxSize || out_dim > kMaxSize) return DIT_ERR_SHAPE;
  if (((in_dim + 127) / 128) * ((out_dim + 127) / 128) > INT32_MAX) return DIT_ERR_SHAPE;
  if (!w || !codes || !scales) return DIT_ERR_INVALID_ARG;
  if (ld < out_dim || ld_codes < in_dim || ld_codes % 16) return DIT_ERR_INVALID_ARG;
  if (!aligned(w, type_bytes(type)) || !aligned(codes, 16) || !aligned(scales, 4)) return DIT_ERR_INVALID_ARG;
  const DeviceState* d;
  const dit_status s = ready(&d);
  if (s != DIT_OK) return s;
  return launch_quantize_weight(w, type, ld, static_cast<int>(in_dim), static_cast<int>(out_dim), codes, ld_codes, scales,
                                static_cast<cudaStream_t>(stream)) == cudaSuccess ? DIT_OK : DIT_ERR_CUDA;
}

dit_status dit_gemm_block128(const dit_gemm_block128_args* a, void* stream) {
  if (!a || a->m < 0 || !type_ok(a->out_type)) return DIT_ERR_INVALID_ARG;
  if (a->n < 1 || a->k < 1 || a->m > kMaxSize || a->n > kMaxSize || a->k > kMaxSize) return DIT_ERR_SHAPE;
  if (a->m == 0) return DIT_OK;
  if (!a->a || !a->a_scales || !a->b || !a->b_scales || !a->out) return DIT_ERR_INVALID_ARG;
  if (a->lda < a->k || a->ldb < a->k || a->lda % 16 || a->ldb % 16 || a->ld_a_scales < a->m || a->ld_out < a->n) return DIT_ERR_INVALID_ARG;
  if (!aligned(a->a, 16) || !aligned(a->b, 16) || !aligned(a->a_scales, 4) || !aligned(a->b_scales, 4) || !aligned(a->bias, 4) ||
      !aligned(a->out, type_bytes(a->out_type)))
    return DIT_ERR_INVALID_ARG;
  // tiles of 128 x 128 are counted in 32 bits, with room for CTAs per tile; the split kernel's smaller ones (128 columns x 16, 32 or 64
  // rows) are few by the rule that chooses it
  if (((a->m + 127) / 128) * ((a->n + 127) / 128) > INT32_MAX / 16) return DIT_ERR_SHAPE;
  const DeviceState* d;
  const dit_status s = ready(&d);
  if (s != DIT_OK) return s;
  BlockProduct b{};
  b.a = a->a; b.a_scales = a->a_scales; b.b = a->b; b.b_scales = a->b_scales; b.bias = a->bias; b.out = a->out;
  b.lda = a->lda; b.ld_a_scales = a->ld_a_scales; b.ldb = a->ldb; b.ld_out = a->ld_out;
  b.m = static_cast<int>(a->m); b.n = static_cast<int>(a->n); b.k = static_cast<int>(a->k);
  b.plan_m = b.m;
  b.epilogue = a->out_type == DIT_TYPE_F16 ? kBlkF16 : (a->out_type == DIT_TYPE_BF16 ? kBlkBF16 : kBlkF32);
  return launch_block_product(b, kNoSeq, static_cast<cudaStream_t>(stream)) == cudaSuccess ? DIT_OK : DIT_ERR_CUDA;
}

size_t dit_select_blocks_workspace(const dit_attention_batch* a) {
  BlockBatch b;
  dit_attention_batch shape;
  if (!a) return 0;
  shape = *a;                                    // sizes only: the matrices need not exist yet
  shape.q = shape.k = shape.v = reinterpret_cast<const void*>(static_cast<uintptr_t>(16));
  shape.ld_q = shape.ld_k = shape.ld_v = INT64_MAX / 16 * 8;
  if (plan_batch(&shape, false, &b) != DIT_OK) return 0;
  const size_t blocks = static_cast<size_t>(b.first_qblock[b.n]) + b.first_kblock[b.n];
  return std::max<size_t>(16, blocks * a->n_heads * a->head_dim * sizeof(double));
}

dit_status dit_select_blocks(const dit_attention_batch* a, const int32_t* keep, const int32_t* tail_rows, int32_t* block_index,
                             int32_t* block_count, int64_t ld_index, void* workspace, size_t workspace_bytes, void* stream) {
  BlockBatch b;
  dit_status s = plan_batch(a, false, &b);
  if (s != DIT_OK) return s;
  if (b.first_qblock[b.n] == 0) return DIT_OK;
  if (!keep || !block_index || !block_count || !workspace || !aligned(workspace, 16) || !aligned(block_index, 4) || !aligned(block_count, 4))
    return DIT_ERR_INVALID_ARG;
  BlockSelectParams p{};
  for (int r = 0; r < b.n; ++r) {
    if (keep[r] < 1 || (tail_rows && tail_rows[r] < 0)) return DIT_ERR_INVALID_ARG;
    p.keep[r] = keep[r];
    p.tail[r] = tail_rows ? tail_rows[r] : 0;
    p.widest = std::max(p.widest, keep[r]);
  }
  if (ld_index < p.widest) return DIT_ERR_INVALID_ARG;
  if (workspace_bytes < dit_select_blocks_workspace(a)) return DIT_ERR_CAPACITY;
  const DeviceState* d;
  s = ready(&d);
  if (s != DIT_OK) return s;
  return launch_select(*a, b, p, block_index, block_count, ld_index, workspace, static_cast<cudaStream_t>(stream)) == cudaSuccess ? DIT_OK : DIT_ERR_CUDA;
}

dit_status dit_block_attention(const dit_attention_batch* a, const int32_t* block_index, const int32_t* block_count, int64_t ld_index,
                               float scale, void* out, int64_t ld_out, void* stream) {
  return run_block_attention(a, block_index, block_count, ld_index, scale, out, ld_out, nullptr, false, static_cast<cudaStream_t>(stream));
}

dit_status dit_ops_poll_status(void) {
  const DeviceState* d;
  const dit_status s = ready(&d);
  if (s != DIT_OK) return s;
  int value = 0;
  if (cudaDeviceSynchronize() != cudaSuccess) return DIT_ERR_CUDA;
  if (cudaMemcpy(&value, d->status, sizeof(value), cudaMemcpyDeviceToHost) != cudaSuccess) return DIT_ERR_CUDA;
  if (value == kStatusOk) return DIT_OK;
  if (cudaMemset(d->status, 0, sizeof(int)) != cudaSuccess) return DIT_ERR_CUDA;
  return DIT_ERR_TIMEOUT;
}

}  // extern "C"
