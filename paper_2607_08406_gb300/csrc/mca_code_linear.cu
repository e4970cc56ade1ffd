// A layer on 8-bit codes (mca_code_linear): y = act((x w^T) * x_scale * w_scale + bias).
#include "mca_answers.h"
#include "mca_code_linear.cuh"

namespace mca {

namespace {

constexpr int kTile = 64;      // rows and outputs per CTA, and the depth of a step

// Four consecutive codes of a row from column k (zeros behind the last column).
__device__ __forceinline__ int codes4(const int8_t* row, int k, int n) {
  unsigned int v = 0u;
#pragma unroll
  for (int q = 0; q < 4; ++q)
    if (k + q < n) v |= (unsigned int)(uint8_t)row[k + q] << (8 * q);
  return (int)v;
}

template <int DT>
__global__ void __launch_bounds__(256) code_linear_kernel(mca_code_linear_args a) {
  __shared__ int s_x[kTile / 4][kTile + 1], s_w[kTile / 4][kTile + 1];
  const int64_t r0 = (int64_t)blockIdx.x * kTile;
  const int n0 = blockIdx.y * kTile, tid = threadIdx.x, tr = tid >> 4, tn = tid & 15;
  int acc[4][4] = {};
  for (int k0 = 0; k0 < a.n_in; k0 += kTile) {
    for (int e = tid; e < kTile * kTile / 4; e += 256) {
      const int i = e / (kTile / 4), q = e % (kTile / 4);
      s_x[q][i] = r0 + i < a.rows ? codes4(a.x + (r0 + i) * a.ldx, k0 + 4 * q, a.n_in) : 0;
      s_w[q][i] = n0 + i < a.n_out ? codes4(a.w + (int64_t)(n0 + i) * a.ldw, k0 + 4 * q, a.n_in) : 0;
    }
    __syncthreads();
#pragma unroll 4
    for (int q = 0; q < kTile / 4; ++q)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[i][j] = __dp4a(s_x[q][tr + 16 * i], s_w[q][tn + 16 * j], acc[i][j]);
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t r = r0 + tr + 16 * i;
      const int n = n0 + tn + 16 * j;
      if (r < a.rows && n < a.n_out)
        static_cast<elem_t<DT>*>(a.y)[r * a.ldy + n] = elem_of<DT>(
            code_output(acc[i][j], a.x_scale[r], a.w_scale[n], a.bias ? a.bias[n] : 0.0f,
                        a.bias != nullptr, a.act, a.act_param));
    }
}

}  // namespace

size_t code_linear_workspace(const mca_code_linear_args&) { return 0; }

cudaError_t launch_code_linear(const mca_code_linear_args& a, cudaStream_t s) {
  const dim3 grid((unsigned int)((a.rows + kTile - 1) / kTile), (a.n_out + kTile - 1) / kTile);
  switch (a.dtype) {
    case MCA_DTYPE_FP32: code_linear_kernel<MCA_DTYPE_FP32><<<grid, 256, 0, s>>>(a); break;
    case MCA_DTYPE_FP16: code_linear_kernel<MCA_DTYPE_FP16><<<grid, 256, 0, s>>>(a); break;
    default: code_linear_kernel<MCA_DTYPE_BF16><<<grid, 256, 0, s>>>(a);
  }
  return cudaGetLastError();
}

}  // namespace mca
