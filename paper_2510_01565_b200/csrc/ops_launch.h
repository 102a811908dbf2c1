// Launchers of the context-free operators for the step (dit_api.cu).  The kernels and their per-device
// preparation live in ops_api.cu.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include "common.cuh"

namespace dit {

// Epilogues of the block-scaled product that the step uses beside the plain ones.
struct BlockProduct {
  const void* a;             // e4m3 [m, lda]
  const float* a_scales;     // [groups, ld_a_scales]
  const void* b;             // e4m3 [n, ldb]
  const float* b_scales;     // [ceil(n / 128), groups]
  const float* bias;
  void* out;
  long long lda, ld_a_scales, ldb, ld_out;
  int m, n, k;
  int plan_m;                // rows by which the kernel is chosen: the whole batch's where a launch covers a slice of its rows, so
                             // that every element is summed in the same order as in one launch
  int epilogue;              // BlockGemmEpilogue; kBlkGeluF16 wants rows of out on 16-byte boundaries
  int row0;                  // gated residual only: packed row of row 0, residual, gate vectors
  const float* resid;
  const float* gate;
  long long gate_stride;
  int* status;               // device word for waits that ran out; NULL: the device's own (dit_ops_poll_status)
};

cudaError_t ops_prepare_device();                      // sets kernel attributes once per device
cudaError_t launch_block_product(const BlockProduct& b, const SeqInfo& seq, cudaStream_t st);
// dit_block_attention with a status word of the caller's.  clamp: infinite results become the largest finite value, as in every
// activation of a step, where an infinity would meet zeros further on.
dit_status run_block_attention(const dit_attention_batch* batch, const int32_t* block_index, const int32_t* block_count, int64_t ld_index, float scale,
                               void* out, int64_t ld_out, int* status, bool clamp, cudaStream_t st);
cudaError_t launch_quantize_rows(const void* x, dit_type type, long long ld, long long rows, long long cols, void* codes,
                                 long long ld_codes, float* scales, long long ld_scales, cudaStream_t st);
cudaError_t launch_quantize_weight(const void* w, dit_type type, long long ld, int in_dim, int out_dim, void* codes, long long ld_codes,
                                   float* scales, cudaStream_t st);

}  // namespace dit
