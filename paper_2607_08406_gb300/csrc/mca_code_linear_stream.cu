// A layer on 8-bit codes for few samples: the weights stream once from memory through registers.
//
// A warp takes 32 outputs by up to 64 samples and a slice of the columns. A thread loads 16 codes of a row at a time,
// turns them into fp16 and has in each word's four codes its part of an m16n8k16 MMA: which four of the MMA's 16
// columns they are does not matter as long as weights and samples agree. So nothing goes through shared memory, no
// barrier is in the loop, and a warp keeps 4 KB of weights in flight. The warps of a CTA take the slices in turn; a
// slice has at most 1024 columns, so that its sums are exact in fp32, and adds them as integers in shared
// memory (in any order: integers).
//
// What bounds it are the loads in flight: 4096 -> 16384 takes 14 us for up to 8 samples, 4.9 of the 6.8 TB/s that a
// copy reaches, with a fifth of the warps active, and 56 of its 512 CTAs run in a second wave; 22 us for 16 and 24
// for 32, where the MMAs count, which take a warp scheduler 30 cycles each. (The tcgen05 form of this, with weights
// by TMA into a ring, converted by warps into tensor memory, spent most of its time in hand-overs: a wait for an
// mbarrier takes 200 cycles even if nothing is left to wait for, and a warp's share of a stage was worth 600.)
#include <algorithm>

#include "mca_code_linear.cuh"

namespace mca {

namespace {

constexpr int kThreads = 256;
constexpr int kOut = 32;                       // outputs per CTA
constexpr int kStep = 64;                      // columns per iteration: four threads' 16 codes

__device__ __forceinline__ void mma_codes(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                          uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t word(const uint4& v, int i) {
  return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
}

// NT: groups of 8 samples.
template <int NT, int DT>
__global__ void __launch_bounds__(kThreads, NT <= 2 ? 3 : NT <= 4 ? 2 : 1)
    code_linear_stream_kernel(mca_code_linear_args a, int slice) {
  __shared__ int s_sum[NT * 8][kOut];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int n0 = blockIdx.x * kOut;
  const int64_t r0 = (int64_t)blockIdx.y * (NT * 8);
  const int nt = (int)min((int64_t)(NT * 8), a.rows - r0);
  for (int e = tid; e < NT * 8 * kOut; e += kThreads) (&s_sum[0][0])[e] = 0;
  __syncthreads();
  // rows behind the last are read as the last; their sums are not used
  const int8_t* w[4];
  const int8_t* x[NT];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = a.w + (int64_t)min(n0 + g + 8 * i, a.n_out - 1) * a.ldw;
#pragma unroll
  for (int j = 0; j < NT; ++j) x[j] = a.x + (r0 + min(g + 8 * j, nt - 1)) * a.ldx;
  for (int k0 = warp * slice; k0 < a.n_in; k0 += (kThreads / 32) * slice) {
    const int k1 = min(k0 + slice, a.n_in);
    float c[2][NT][4];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) c[m][j][q] = 0.0f;
#pragma unroll 2
    for (int k = k0 + 16 * t; k - 16 * t < k1; k += kStep) {
      uint4 wv[4], xv[NT];
#pragma unroll
      for (int i = 0; i < 4; ++i) wv[i] = load_codes16(w[i], k, k1);
#pragma unroll
      for (int j = 0; j < NT; ++j) xv[j] = load_codes16(x[j], k, k1);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t lo[4], hi[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) codes_f16(word(wv[i], q), lo[i], hi[i]);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          uint32_t b0, b1;
          codes_f16(word(xv[j], q), b0, b1);
          mma_codes(c[0][j], lo[0], lo[1], hi[0], hi[1], b0, b1);
          mma_codes(c[1][j], lo[2], lo[3], hi[2], hi[3], b0, b1);
        }
      }
    }
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          atomicAdd(&s_sum[8 * j + 2 * t + (q & 1)][16 * m + g + 8 * (q >> 1)], __float2int_rn(c[m][j][q]));
  }
  __syncthreads();
  const int n = n0 + lane;
  if (n >= a.n_out) return;
  const float ws = __ldg(a.w_scale + n), b = a.bias ? __ldg(a.bias + n) : 0.0f;
  constexpr int kWarps = kThreads / 32;
  for (int s0 = warp; s0 < nt; s0 += 4 * kWarps) {
    float z[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int s = min(s0 + i * kWarps, nt - 1);
      z[i] = code_field(__int2float_rn(s_sum[s][lane]), __ldg(a.x_scale + r0 + s), ws, b, a.bias != nullptr);
    }
    act_block(z, a.act, a.act_param);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (s0 + i * kWarps < nt)
        static_cast<elem_t<DT>*>(a.y)[(r0 + s0 + i * kWarps) * a.ldy + n] = elem_of<DT>(z[i]);
  }
}

template <int NT>
cudaError_t launch_stream(const mca_code_linear_args& a, cudaStream_t s) {
  const dim3 grid((a.n_out + kOut - 1) / kOut, (unsigned int)((a.rows + NT * 8 - 1) / (NT * 8)));
  // a slice per warp, of whole steps and at most kExactK columns
  const int per = (a.n_in + kThreads / 32 - 1) / (kThreads / 32);
  const int slice = std::min(kExactK, (per + kStep - 1) / kStep * kStep);
  switch (a.dtype) {
    case MCA_DTYPE_FP32: code_linear_stream_kernel<NT, MCA_DTYPE_FP32><<<grid, kThreads, 0, s>>>(a, slice); break;
    case MCA_DTYPE_FP16: code_linear_stream_kernel<NT, MCA_DTYPE_FP16><<<grid, kThreads, 0, s>>>(a, slice); break;
    default: code_linear_stream_kernel<NT, MCA_DTYPE_BF16><<<grid, kThreads, 0, s>>>(a, slice);
  }
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_code_linear_stream(const mca_code_linear_args& a, cudaStream_t s) {
  if (a.rows <= 8) return launch_stream<1>(a, s);
  if (a.rows <= 16) return launch_stream<2>(a, s);
  if (a.rows <= 32) return launch_stream<4>(a, s);
  return launch_stream<8>(a, s);
}

}  // namespace mca
