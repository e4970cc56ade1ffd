// What the kernels of mca_code_linear share: the output of an integer sum, codes as fp16.
//
// An 8-bit code is an fp16 number exactly, products of two are integers below 2^14, and a sum of 1024 of them
// stays within 2^24 = 128 * 128 * 1024, so that kind::f16 MMAs accumulate it exactly in fp32: sm_103a has no
// tcgen05 form for 8-bit integers, and mma.sync's is slow. Longer sums are taken out of tensor memory after every
// 1024 columns (kExactK) and added up as integers.
#pragma once

#include "mca_answers.h"
#include "mca_device.cuh"
#include "mca_elem.cuh"
#include "mca_tc.cuh"

namespace mca {

constexpr int kExactK = 1024;
constexpr int kM = 128;                       // outputs per CTA (a CTA's rows of the MMA's M)

// The transfer functions as they are defined, for outputs that a caller sees: relative accuracy near 0 and
// for small tails, which the trial loop's forms (mca_device.cuh) leave out. NaN stays NaN.
__device__ __forceinline__ float act_accurate(int act, float z, float g) {
  switch (act) {
    case MCA_ACT_TANH: return tanhf(z);
    case MCA_ACT_SIGMOID: return 1.0f / (1.0f + expf(-z));
    case MCA_ACT_RELU: return z < 0.0f ? 0.0f : z;
    case MCA_ACT_GAUSSIAN: return expf(-g * z * z);
    default: return z;
  }
}

// z Phi(z) = max(z, 0) - a Q(a), a = |z|, with the normal distribution's tail Q(a) = exp(-a^2/2) t P(t), t = 1 / (1 +
// p a), in the form that Hastings gave (Approximations for Digital Computers, 1955); P fitted here to the tail in 64
// bits, off by 0.9 * 2^-24 at most. In half steps of fp32 relative to the value an output is off by at most 18 + 1.5
// z^2: exponent 1.5 z^2 and 4 for ex2, 3 roundings of t that count 2.3 times, 3 for P's sum, 1 for its fit, 3 for the
// products. Tails below 2^-126 are 0; the limit -0 of -infinity is taken. Pairs of fields: 13 instructions each, 245
// us for 14346 x 64 -> 15616 fp16, where erfcf's 60 took 474.
template <int N>
__device__ __forceinline__ void gelu_block(float (&v)[N]) {
  static_assert(N % 2 == 0, "pairs");
  constexpr float kP = 0.35f, kFar = 20.0f;
  constexpr float kC[9] = {0x1.1df1eap-3f,  0x1.1e6e70p-3f, 0x1.eaea60p-4f, 0x1.afda7ep-4f, -0x1.77cdbep-6f,
                           0x1.457ccep-3f, -0x1.05a306p-2f, 0x1.26a684p-3f, -0x1.dd32c8p-6f};
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    float2 a, t, e;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(a.x) : "f"(fabsf(v[i])), "f"(kFar));
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(a.y) : "f"(fabsf(v[i + 1])), "f"(kFar));
    const float2 den = fma2(a, make_float2(kP, kP), make_float2(1.0f, 1.0f));
    t = make_float2(rcp_ftz(den.x), rcp_ftz(den.y));
    float2 q = make_float2(-kC[8], -kC[8]);
#pragma unroll
    for (int k = 7; k >= 0; --k) q = fma2(q, t, make_float2(-kC[k], -kC[k]));
    const float2 x = mul2(mul2(a, a), make_float2(-0.5f * kLog2e, -0.5f * kLog2e));
    e = make_float2(ex2_ftz(x.x), ex2_ftz(x.y));
    q = mul2(mul2(q, t), e);
    q = fma2(a, q, make_float2(fmaxf(v[i], 0.0f), fmaxf(v[i + 1], 0.0f)));
    v[i] = q.x;
    v[i + 1] = q.y;
  }
}

template <int ACT, int N>
__device__ __forceinline__ void act_block(float (&v)[N], float g) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = act_accurate(ACT, v[i], g);
}
// The same for a block of fields: one branch for all (left to each field, the compiler evaluates every function and
// selects: 400 cycles an output).
template <int N>
__device__ __forceinline__ void act_block(float (&v)[N], int act, float g) {
  if (act == MCA_ACT_IDENTITY) return;
  switch (act) {
    case MCA_ACT_TANH: act_block<MCA_ACT_TANH>(v, g); break;
    case MCA_ACT_SIGMOID: act_block<MCA_ACT_SIGMOID>(v, g); break;
    case MCA_ACT_RELU: act_block<MCA_ACT_RELU>(v, g); break;
    case MCA_ACT_GAUSSIAN: act_block<MCA_ACT_GAUSSIAN>(v, g); break;
    default: gelu_block(v);
  }
}

// A field from the sum as fp32: s * xs * ws + b, products and sum rounded one after the other.
__device__ __forceinline__ float code_field(float s, float xs, float ws, float b, bool bias) {
  const float z = __fmul_rn(__fmul_rn(s, xs), ws);
  return bias ? __fadd_rn(z, b) : z;
}

// The same for 16 samples of an output, in pairs.
__device__ __forceinline__ void code_fields(float (&v)[16], const float4* xs, float ws, float b, bool bias) {
  const float2 w = make_float2(ws, ws), bb = make_float2(b, b);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 x = xs[i];
    float2 lo = mul2(mul2(make_float2(v[4 * i], v[4 * i + 1]), make_float2(x.x, x.y)), w);
    float2 hi = mul2(mul2(make_float2(v[4 * i + 2], v[4 * i + 3]), make_float2(x.z, x.w)), w);
    if (bias) {
      lo = add2(lo, bb);
      hi = add2(hi, bb);
    }
    v[4 * i] = lo.x;
    v[4 * i + 1] = lo.y;
    v[4 * i + 2] = hi.x;
    v[4 * i + 3] = hi.y;
  }
}

// Four codes as two pairs of fp16, of the bytes 0 and 2, and 1 and 3: a permutation of the columns, the same for both
// operands. A byte b xor 0x80 is b + 128; under the exponent of 1024 it is 1024 + 128 + b.
__device__ __forceinline__ void codes_f16(unsigned int v, unsigned int& lo, unsigned int& hi) {
  const unsigned int a = (v & 0x00ff00ffu) ^ 0x64806480u;
  const unsigned int b = ((v >> 8) & 0x00ff00ffu) ^ 0x64806480u;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(a), "r"(0x64806480u));
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(b), "r"(0x64806480u));
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync_all() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;"
               ::: "memory");
}
__device__ __forceinline__ int ld_cluster(uint32_t addr, uint32_t rank) {
  uint32_t a;
  int v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ int ld_shared(uint32_t a) {
  int v;
  asm volatile("ld.shared.s32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void sts128(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w)
               : "memory");
}

// 16 codes of a row (on a 16-byte boundary) from column k; zeros behind column n, which is not read beyond.
__device__ __forceinline__ uint4 load_codes16(const int8_t* p, int k, int n) {
  if (k + 16 <= n) {
    uint4 v;
    asm volatile("ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p + k));
    return v;
  }
  uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (k + i < n) w[i >> 2] |= (uint32_t)(uint8_t)p[k + i] << (8 * (i & 3));
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// One lane of a converged warp arrives; the warp stays converged for the tensor-memory instructions.
__device__ __forceinline__ void warp_arrive(uint64_t* bar) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
  __syncwarp();
}
// The warp's agreement on a wait.
__device__ __forceinline__ bool warp_all(bool ok) {
  ok = __all_sync(0xffffffffu, ok);
  __syncwarp();
  return ok;
}

// Rows that start on 16-byte boundaries.
inline bool code_rows_aligned(const int8_t* p, int64_t rows, int64_t ld) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (rows == 1 || ld % 16 == 0);
}

// mca_code_linear_stream.cu: few samples; operands' rows on 16-byte boundaries.
cudaError_t launch_code_linear_stream(const mca_code_linear_args& a, cudaStream_t s);
// mca_code_linear_tc.cu: some dozens of samples; operands' rows on 16-byte boundaries. Its time for more than 64.
double code_linear_split_us(const mca_code_linear_args& a);
cudaError_t launch_code_linear_split(const mca_code_linear_args& a, cudaStream_t s);
// mca_code_linear_pair.cu: many samples; in a.workspace the operands as fp16.
size_t code_linear_pair_workspace(const mca_code_linear_args& a);
cudaError_t launch_code_linear_pair(const mca_code_linear_args& a, cudaStream_t s);

}  // namespace mca
