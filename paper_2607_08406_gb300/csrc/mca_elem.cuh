// Element types of callers' matrices (mca_dtype).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "../../include/mca.h"

namespace mca {

template <int DT>
struct Elem;
template <>
struct Elem<MCA_DTYPE_FP32> {
  using type = float;
};
template <>
struct Elem<MCA_DTYPE_FP16> {
  using type = __half;
};
template <>
struct Elem<MCA_DTYPE_BF16> {
  using type = __nv_bfloat16;
};
template <int DT>
using elem_t = typename Elem<DT>::type;

__device__ __forceinline__ float elem_f32(float v) { return v; }
__device__ __forceinline__ float elem_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float elem_f32(__nv_bfloat16 v) { return __bfloat162float(v); }

template <int DT>
__host__ __device__ __forceinline__ elem_t<DT> elem_of(float v) {
  if constexpr (DT == MCA_DTYPE_FP32)
    return v;
  else if constexpr (DT == MCA_DTYPE_FP16)
    return __float2half_rn(v);
  else
    return __float2bfloat16_rn(v);
}

constexpr float kRound = 12582912.0f;         // 1.5 * 2^23: x + kRound rounds |x| <= 2^22 to an integer,
constexpr int kRoundBits = 0x4B400000;        // whose bits follow those of kRound

// The integer next to x (halves to the even one), |x| <= 2^22, as an integer and as fp32.
__device__ __forceinline__ int near_int(float x) { return __float_as_int(__fadd_rn(x, kRound)) - kRoundBits; }
__device__ __forceinline__ float near_f32(float x) { return __fsub_rn(__fadd_rn(x, kRound), kRound); }

}  // namespace mca
