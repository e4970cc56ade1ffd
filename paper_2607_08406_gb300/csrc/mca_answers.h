// Layers in 8-bit integers and log probabilities of given symbols: the kernels' arguments and launchers, between the
// entry points (mca_answers.cu) and the kernels.
#pragma once

#include <cstdint>

#include <cuda_runtime.h>

#include "../../include/mca.h"

namespace mca {

inline size_t dtype_bytes(int dtype) { return dtype == MCA_DTYPE_FP32 ? 4 : 2; }

// mca_quant.cu
cudaError_t launch_quantize_rows(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx,
                                 int8_t* codes, int64_t ldc, float* scale, cudaStream_t s);
cudaError_t launch_fill(float* p, int64_t n, float v, cudaStream_t s);

// mca_code_linear.cu: operands, sizes and pointers as checked by the entry point.
size_t code_linear_workspace(const mca_code_linear_args& a);
cudaError_t launch_code_linear(const mca_code_linear_args& a, cudaStream_t s);

// mca_logprobs.cu. The target of row r is targets[(r / period) * pitch + r % period].
struct LogprobArgs {
  mca_token_logprobs_args a;
  int64_t period, pitch;
};
cudaError_t launch_logprobs(const LogprobArgs& a, cudaStream_t s);
cudaError_t launch_logprobs_backward(const mca_token_logprobs_backward_args& a, cudaStream_t s);

constexpr int kMaxTop = 32;                  // alternatives of a row

}  // namespace mca
