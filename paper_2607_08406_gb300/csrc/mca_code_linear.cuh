// What the kernels of mca_code_linear share: the output of an integer sum, codes as fp16, tensor maps.
//
// An 8-bit code is an fp16 number exactly, products of two are integers below 2^14, and a sum of 1024 of them
// stays within 2^24 = 128 * 128 * 1024, so that kind::f16 MMAs accumulate it exactly in fp32: sm_103a has no
// tcgen05 form for 8-bit integers, and mma.sync's is slow. Longer sums are taken out of tensor memory after every
// 1024 columns (kExactK) and added up as integers.
#pragma once

#include <cuda.h>

#include "mca_answers.h"
#include "mca_elem.cuh"

namespace mca {

constexpr int kExactK = 1024;

// The transfer functions as they are defined, for outputs that a caller sees: relative accuracy near 0 and
// for small tails, which the trial loop's forms (mca_device.cuh) leave out. NaN stays NaN.
__device__ __forceinline__ float act_accurate(int act, float z, float g) {
  switch (act) {
    case MCA_ACT_TANH: return tanhf(z);
    case MCA_ACT_SIGMOID: return 1.0f / (1.0f + expf(-z));
    case MCA_ACT_RELU: return z < 0.0f ? 0.0f : z;
    case MCA_ACT_GAUSSIAN: return expf(-g * z * z);
    case MCA_ACT_GELU: return 0.5f * z * erfcf(-0.7071067811865476f * z);
    default: return z;
  }
}

// act(float(s) * xs * ws + b), products and sum rounded one after the other.
__device__ __forceinline__ float code_output(int s, float xs, float ws, float b, bool bias, int act,
                                             float g) {
  float z = __fmul_rn(__fmul_rn(__int2float_rn(s), xs), ws);
  if (bias) z = __fadd_rn(z, b);
  return act == MCA_ACT_IDENTITY ? z : act_accurate(act, z, g);
}

// Four codes as two pairs of fp16, of the bytes 0 and 2, and 1 and 3: a permutation of the columns, the same for both
// operands. A byte b xor 0x80 is b + 128; under the exponent of 1024 it is 1024 + 128 + b.
__device__ __forceinline__ void codes_f16(unsigned int v, unsigned int& lo, unsigned int& hi) {
  const unsigned int a = (v & 0x00ff00ffu) ^ 0x64806480u;
  const unsigned int b = ((v >> 8) & 0x00ff00ffu) ^ 0x64806480u;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(a), "r"(0x64806480u));
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(b), "r"(0x64806480u));
}

// One thread: a box of a 2-D tensor map (x: byte column, a multiple of 16; y: row) into shared memory;
// elements outside the matrix arrive as zeros. Completes bytes on bar.
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
      "[%0], [%1, {%2, %3}], [%4];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar)
      : "memory");
}

// Map of a code matrix [rows x cols], row distance ld (a multiple of 16, base too), in boxes of box_rows
// x 128 bytes whose 16-byte units are stored exchanged (128-byte swizzle: unit j of row r at j ^ (r % 8)).
cudaError_t code_map(CUtensorMap* map, const int8_t* p, int64_t rows, int64_t cols, int64_t ld,
                     int box_rows);

// mca_code_linear_tc.cu: operands on 16-byte boundaries.
cudaError_t launch_code_linear_split(const mca_code_linear_args& a, cudaStream_t s);

}  // namespace mca
