// What the kernels of mca_code_linear share: the output of an integer sum.
#pragma once

#include "mca_elem.cuh"

namespace mca {

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

}  // namespace mca
