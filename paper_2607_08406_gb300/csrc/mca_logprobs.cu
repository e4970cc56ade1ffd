// Log probabilities of given symbols, entropy and alternatives (mca_token_logprobs) and their gradient.
#include <climits>

#include "mca_answers.h"
#include "mca_elem.cuh"

namespace mca {

namespace {

constexpr int kThreads = 256;

struct MaxOp {
  __device__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct SumOp {
  __device__ float operator()(float a, float b) const { return a + b; }
};
template <class Op>
__device__ float block_all(float v, Op op) {
  __shared__ float red[kThreads / 32];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  v = red[0];
  for (int q = 1; q < kThreads / 32; ++q) v = op(v, red[q]);
  return v;
}

// Values in the order of their size, equal ones with the lower index first, as unsigned numbers.
__device__ __forceinline__ unsigned long long order_key(float v, int i) {
  const unsigned int b = __float_as_uint(v);
  const unsigned int u = b & 0x80000000u ? ~b : b | 0x80000000u;
  return (unsigned long long)u << 32 | (unsigned int)~i;
}

template <int DT>
__global__ void __launch_bounds__(kThreads) logprobs_kernel(LogprobArgs p) {
  __shared__ unsigned long long s_best;
  const mca_token_logprobs_args& a = p.a;
  const int64_t r = blockIdx.x;
  const elem_t<DT>* x = static_cast<const elem_t<DT>*>(a.logits) + r * a.ld;
  float m = -INFINITY;
  bool bad = false;
  for (int v = threadIdx.x; v < a.vocab; v += kThreads) {
    const float z = elem_f32(x[v]);
    bad |= !(z < INFINITY);
    m = fmaxf(m, z);
  }
  bad = __syncthreads_or(bad);
  m = block_all(m, MaxOp());
  const bool none = m == -INFINITY;
  float se = 0.0f, sd = 0.0f;
  for (int v = threadIdx.x; v < a.vocab; v += kThreads) {
    const float d = elem_f32(x[v]) - m;
    if (!none && d > -INFINITY) {
      const float e = expf(d);
      se += e;
      sd += e * d;
    }
  }
  se = block_all(se, SumOp());
  sd = block_all(sd, SumOp());
  const float ls = logf(se);
  if (threadIdx.x == 0) {
    if (a.lse) a.lse[r] = bad ? NAN : none ? -INFINITY : m + ls;
    if (a.entropy) a.entropy[r] = bad ? NAN : none ? 0.0f : ls - sd / se;
    if (a.logprob) {
      const int t = a.targets[r / p.period * p.pitch + r % p.period];
      float lp = 0.0f;
      if (t != -1)
        lp = t < 0 || t >= a.vocab || bad ? NAN : none ? -INFINITY : (elem_f32(x[t]) - m) - ls;
      a.logprob[r] = lp;
    }
  }
  unsigned long long last = ~0ull;
  for (int k = 0; k < a.top; ++k) {
    __syncthreads();
    if (threadIdx.x == 0) s_best = 0ull;
    __syncthreads();
    unsigned long long best = 0ull;
    if (!bad)
      for (int v = threadIdx.x; v < a.vocab; v += kThreads) {
        const float z = elem_f32(x[v]);
        const unsigned long long key = z > -INFINITY ? order_key(z + 0.0f, v) : 0ull;
        if (key < last && key > best) best = key;
      }
    atomicMax(&s_best, best);
    __syncthreads();
    last = s_best;
    if (threadIdx.x == 0) {
      const int i = last ? (int)~(unsigned int)last : -1;
      a.top_index[r * a.top + k] = i;
      a.top_logprob[r * a.top + k] = bad ? NAN : i < 0 ? -INFINITY : (elem_f32(x[i]) - m) - ls;
    }
    if (last == 0ull) last = 1ull;       // no symbols left
  }
}

template <int DT>
__global__ void __launch_bounds__(kThreads) logprobs_backward_kernel(mca_token_logprobs_backward_args a) {
  const int64_t r = blockIdx.x;
  const elem_t<DT>* x = static_cast<const elem_t<DT>*>(a.logits) + r * a.ld;
  elem_t<DT>* out = static_cast<elem_t<DT>*>(a.grad) + r * a.ldg;
  const float lse = a.lse[r];
  int t = -1;
  float gl = 0.0f;
  if (a.g_logprob) {
    t = a.targets[r];
    if (t != -1) gl = t < 0 || t >= a.vocab ? NAN : a.g_logprob[r];
  }
  const float ge = a.g_entropy ? a.g_entropy[r] : 0.0f, h = a.g_entropy ? a.entropy[r] : 0.0f;
  const bool none = lse == -INFINITY;
  for (int v = threadIdx.x; v < a.vocab; v += kThreads) {
    const float lp = elem_f32(x[v]) - lse;
    float g = (v == t ? gl : 0.0f);
    if (lp > -INFINITY || lp != lp) {
      const float e = expf(lp);
      g -= e * (gl + ge * (lp + h));
    }
    out[v] = elem_of<DT>(none ? 0.0f : g);
  }
}

}  // namespace

cudaError_t launch_logprobs(const LogprobArgs& p, cudaStream_t s) {
  const unsigned int grid = (unsigned int)p.a.rows;
  switch (p.a.dtype) {
    case MCA_DTYPE_FP32: logprobs_kernel<MCA_DTYPE_FP32><<<grid, kThreads, 0, s>>>(p); break;
    case MCA_DTYPE_FP16: logprobs_kernel<MCA_DTYPE_FP16><<<grid, kThreads, 0, s>>>(p); break;
    default: logprobs_kernel<MCA_DTYPE_BF16><<<grid, kThreads, 0, s>>>(p);
  }
  return cudaGetLastError();
}

cudaError_t launch_logprobs_backward(const mca_token_logprobs_backward_args& a, cudaStream_t s) {
  const unsigned int grid = (unsigned int)a.rows;
  switch (a.dtype) {
    case MCA_DTYPE_FP32: logprobs_backward_kernel<MCA_DTYPE_FP32><<<grid, kThreads, 0, s>>>(a); break;
    case MCA_DTYPE_FP16: logprobs_backward_kernel<MCA_DTYPE_FP16><<<grid, kThreads, 0, s>>>(a); break;
    default: logprobs_backward_kernel<MCA_DTYPE_BF16><<<grid, kThreads, 0, s>>>(a);
  }
  return cudaGetLastError();
}

}  // namespace mca
