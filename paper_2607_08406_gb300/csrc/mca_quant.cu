// Rows in 8-bit codes with a scale each (mca_quantize_rows): scale = max |x| / 127, code = x / scale to the nearest
// integer. One read of x and one write of the codes bound it (2 + 1 bytes per bf16 element); a row's elements
// wait in registers between the two steps: 8 lanes have a row up to 256 columns, a warp up to 1024, a CTA up to 32768.
// Longer rows are read a second time, mostly from L2. An element's quotient is a product with 1 / scale, rounded by an
// addition, seven instructions with its place in the output; the pieces with one next to a half (one of 600) are
// looked at again. 8192 x 8192 bf16 takes 42 us, 30 of them the memory's; rows off 16-byte boundaries go an element at a
// time (8192 x 8193: 122 us).
#include "mca_answers.h"
#include "mca_device.cuh"
#include "mca_elem.cuh"

namespace mca {

namespace {

constexpr int kRowThreads = 256;   // a CTA's threads, of short rows
constexpr int kLongThreads = 1024; // threads of a CTA whose row does not fit in registers

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

struct RowScale {
  float s, inv, up;                // scale and its inverse for elements multiplied by up
};

__device__ __forceinline__ RowScale row_scale(float s) {
  // scales near the subnormal numbers: 2^64 times everything
  const float up = s < 0x1p-100f ? 0x1p64f : 1.0f;
  return {s * up, 1.0f / (s * up), up};
}

// x / s for |x| / s <= 127.5 to the nearest integer, halves to the even one. The product with 1 / s is off
// by less than 127 * 3 * 2^-24 = 2.3e-5; where that might cross a half, the sign of |x| - (f + 1/2) s decides,
// whose product is exact in an fma (8 + 24 bits) and whose difference rounds once, which keeps its sign (s is no
// subnormal number: see row_scale).
__device__ __forceinline__ int exact_code(float x, const RowScale& r) {
  const float a = fabsf(x) * r.up;
  const float t = a * r.inv;
  float c = near_f32(t);
  if (fabsf(t - c) > 0.4999f) {
    const float f = c <= t ? c : c - 1.0f;                      // the half is f + 1/2
    const float d = fmaf(-(f + 0.5f), r.s, a);
    c = d > 0.0f || (d == 0.0f && (near_int(f) & 1)) ? f + 1.0f : f;
  }
  c = fminf(c, 127.0f);            // a scale that was rounded down to a subnormal number
  return near_int(copysignf(c, x));
}

// Sixteen bytes of elements, or one element where rows lie off 16-byte boundaries.
template <int DT, bool WIDE>
struct Pack {
  static constexpr int N = WIDE ? 16 / (int)sizeof(elem_t<DT>) : 1;
  union {
    uint4 u;
    elem_t<DT> e[16 / sizeof(elem_t<DT>)];
  };
  __device__ __forceinline__ void load(const elem_t<DT>* x, int64_t c, int64_t cols) {
    if constexpr (WIDE) {
      if (c + N <= cols) {
        u = __ldg(reinterpret_cast<const uint4*>(x + c));
        return;
      }
      u = make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int q = 0; q < N; ++q) e[q] = c + q < cols ? x[c + q] : elem_of<DT>(0.0f);
  }
  // The largest magnitude, of those here and t; NaN if one is.
  __device__ __forceinline__ float top(float t) const {
    if constexpr (WIDE && DT != MCA_DTYPE_FP32) {
      unsigned int m[4] = {u.x & 0x7fff7fffu, u.y & 0x7fff7fffu, u.z & 0x7fff7fffu, u.w & 0x7fff7fffu};
#pragma unroll
      for (int k = 2; k > 0; k >>= 1)
#pragma unroll
        for (int q = 0; q < k; ++q) {
          if constexpr (DT == MCA_DTYPE_BF16)
            asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(m[q]) : "r"(m[q]), "r"(m[q + k]));
          else
            asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(m[q]) : "r"(m[q]), "r"(m[q + k]));
        }
      const elem_t<DT>* h = reinterpret_cast<const elem_t<DT>*>(&m[0]);
      return max_nan(t, max_nan(elem_f32(h[0]), elem_f32(h[1])));
    } else {
#pragma unroll
      for (int q = 0; q < N; ++q) t = max_nan(t, fabsf(elem_f32(e[q])));
      return t;
    }
  }
  __device__ __forceinline__ void store(int8_t* codes, int64_t c, int64_t cols, const RowScale& r,
                                        bool live) const {
    // a code's bits are the lowest byte of its sum with kRound
    unsigned int v[N];
    float off = 0.0f;
    if constexpr (WIDE) {
      const float2 inv = make_float2(r.inv, r.inv), up = make_float2(kRound, kRound),
                   down = make_float2(-kRound, -kRound), neg = make_float2(-1.0f, -1.0f);
#pragma unroll
      for (int q = 0; q < N; q += 2) {
        const float2 t = mul2(make_float2(elem_f32(e[q]), elem_f32(e[q + 1])), inv), c = add2(t, up);
        const float2 d = fma2(add2(c, down), neg, t);
        off = fmaxf(off, fmaxf(fabsf(d.x), fabsf(d.y)));
        v[q] = __float_as_uint(c.x);
        v[q + 1] = __float_as_uint(c.y);
      }
    } else {
      const float t = elem_f32(e[0]) * r.inv, c = __fadd_rn(t, kRound);
      off = fabsf(t - __fsub_rn(c, kRound));
      v[0] = __float_as_uint(c);
    }
    if (off > 0.4999f || r.up != 1.0f) {
#pragma unroll
      for (int q = 0; q < N; ++q) v[q] = (unsigned int)exact_code(elem_f32(e[q]), r);
    }
    if (!live) {
#pragma unroll
      for (int q = 0; q < N; ++q) v[q] = 0u;
    }
    if constexpr (WIDE) {
      if (c + N <= cols) {
        unsigned int w[N / 4];
#pragma unroll
        for (int q = 0; q < N / 4; ++q)
          w[q] = __byte_perm(__byte_perm(v[4 * q], v[4 * q + 1], 0x0040),
                             __byte_perm(v[4 * q + 2], v[4 * q + 3], 0x0040), 0x5410);
        if constexpr (N == 8)
          *reinterpret_cast<uint2*>(codes + c) = make_uint2(w[0], w[1]);
        else
          *reinterpret_cast<unsigned int*>(codes + c) = w[0];
        return;
      }
    }
#pragma unroll
    for (int q = 0; q < N; ++q)
      if (c + q < cols) codes[c + q] = (int8_t)(v[q] & 0xffu);
  }
};

// The largest of a row's values over its threads.
template <int TPR>
__device__ __forceinline__ float row_top(float t) {
#pragma unroll
  for (int o = (TPR < 32 ? TPR : 32) / 2; o > 0; o >>= 1) t = max_nan(t, __shfl_xor_sync(0xffffffffu, t, o));
  if constexpr (TPR > 32) {
    __shared__ float s_red[TPR / 32];
    if ((threadIdx.x & 31) == 0) s_red[threadIdx.x >> 5] = t;
    __syncthreads();
    t = s_red[threadIdx.x & (TPR / 32 - 1)];
#pragma unroll
    for (int o = TPR / 64; o > 0; o >>= 1) t = max_nan(t, __shfl_xor_sync(0xffffffffu, t, o));
  }
  return t;
}

// TPR threads per row, which hold its elements, E each: at most TPR * E columns.
template <int DT, bool WIDE, int TPR, int E>
__global__ void __launch_bounds__(TPR > kRowThreads ? TPR : kRowThreads) quantize_rows_kernel(
    const void* __restrict__ xv, int64_t rows, int cols, int64_t ldx, int8_t* __restrict__ codes, int64_t ldc,
    float* __restrict__ scale) {
  using P = Pack<DT, WIDE>;
  constexpr int NP = E / P::N, kPer = TPR > kRowThreads ? 1 : kRowThreads / TPR;
  const int64_t row = (int64_t)blockIdx.x * kPer + threadIdx.x / TPR;
  const bool there = row < rows;               // threads behind the last row take part in shuffles
  const int64_t r = there ? row : rows - 1;
  const int t = threadIdx.x % TPR;
  const elem_t<DT>* x = static_cast<const elem_t<DT>*>(xv) + r * ldx;
  P p[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i)
    if (i * TPR * P::N < cols) p[i].load(x, (i * TPR + t) * P::N, cols);
  float top = 0.0f;
#pragma unroll
  for (int i = 0; i < NP; ++i)
    if (i * TPR * P::N < cols) top = p[i].top(top);
  top = row_top<TPR>(top);
  if (!there) return;
  const float s = top < INFINITY ? top / 127.0f : NAN;
  if (t == 0) scale[r] = s;
  const RowScale rs = row_scale(s);
#pragma unroll
  for (int i = 0; i < NP; ++i)
    if (i * TPR * P::N < cols) p[i].store(codes + r * ldc, (i * TPR + t) * P::N, cols, rs, s > 0.0f);
}

template <int DT, bool WIDE>
__global__ void __launch_bounds__(kLongThreads) quantize_long_rows_kernel(
    const void* __restrict__ xv, int64_t cols, int64_t ldx, int8_t* __restrict__ codes, int64_t ldc,
    float* __restrict__ scale) {
  using P = Pack<DT, WIDE>;
  const int64_t r = blockIdx.x;
  const elem_t<DT>* x = static_cast<const elem_t<DT>*>(xv) + r * ldx;
  float top = 0.0f;
#pragma unroll 4
  for (int64_t c = (int64_t)threadIdx.x * P::N; c < cols; c += kLongThreads * P::N) {
    P p;
    p.load(x, c, cols);
    top = p.top(top);
  }
  top = row_top<kLongThreads>(top);
  const float s = top < INFINITY ? top / 127.0f : NAN;
  if (threadIdx.x == 0) scale[r] = s;
  const RowScale rs = row_scale(s);
#pragma unroll 2
  for (int64_t c = (int64_t)threadIdx.x * P::N; c < cols; c += kLongThreads * P::N) {
    P p;
    p.load(x, c, cols);
    p.store(codes + r * ldc, c, cols, rs, s > 0.0f);
  }
}

__global__ void fill_kernel(float* p, int64_t n, float v) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i < n) p[i] = v;
}

template <int DT, bool WIDE, int TPR, int E>
void launch_rows_t(const void* x, int64_t rows, int64_t cols, int64_t ldx, int8_t* codes, int64_t ldc,
                   float* scale, cudaStream_t s) {
  constexpr int kThreads = TPR > kRowThreads ? TPR : kRowThreads, kPer = kThreads / TPR;
  quantize_rows_kernel<DT, WIDE, TPR, E><<<(unsigned int)((rows + kPer - 1) / kPer), kThreads, 0, s>>>(
      x, rows, (int)cols, ldx, codes, ldc, scale);
}

template <int DT, bool WIDE>
void launch_rows(const void* x, int64_t rows, int64_t cols, int64_t ldx, int8_t* codes, int64_t ldc,
                 float* scale, cudaStream_t s) {
  if (cols <= 8 * 32)
    launch_rows_t<DT, WIDE, 8, 32>(x, rows, cols, ldx, codes, ldc, scale, s);
  else if (cols <= 32 * 32)
    launch_rows_t<DT, WIDE, 32, 32>(x, rows, cols, ldx, codes, ldc, scale, s);
  else if (cols <= 256 * 32)
    launch_rows_t<DT, WIDE, 256, 32>(x, rows, cols, ldx, codes, ldc, scale, s);
  else if (cols <= 512 * 32)
    launch_rows_t<DT, WIDE, 512, 32>(x, rows, cols, ldx, codes, ldc, scale, s);
  else if (cols <= 1024 * 32)
    launch_rows_t<DT, WIDE, 1024, 32>(x, rows, cols, ldx, codes, ldc, scale, s);
  else
    quantize_long_rows_kernel<DT, WIDE><<<(unsigned int)rows, kLongThreads, 0, s>>>(
        x, cols, ldx, codes, ldc, scale);
}

template <int DT>
void launch_type(const void* x, int64_t rows, int64_t cols, int64_t ldx, int8_t* codes, int64_t ldc,
                 float* scale, cudaStream_t s) {
  constexpr int es = (int)sizeof(elem_t<DT>), out = 16 / es;     // a pack's bytes of codes
  const bool wide = reinterpret_cast<uintptr_t>(x) % 16 == 0 &&
                    reinterpret_cast<uintptr_t>(codes) % out == 0 &&
                    (rows == 1 || (ldx % out == 0 && ldc % out == 0));
  if (wide)
    launch_rows<DT, true>(x, rows, cols, ldx, codes, ldc, scale, s);
  else
    launch_rows<DT, false>(x, rows, cols, ldx, codes, ldc, scale, s);
}

}  // namespace

cudaError_t launch_fill(float* p, int64_t n, float v, cudaStream_t s) {
  if (n > 0) fill_kernel<<<(unsigned int)((n + 255) / 256), 256, 0, s>>>(p, n, v);
  return cudaGetLastError();
}

cudaError_t launch_quantize_rows(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx,
                                 int8_t* codes, int64_t ldc, float* scale, cudaStream_t s) {
  if (dtype == MCA_DTYPE_FP32)
    launch_type<MCA_DTYPE_FP32>(x, rows, cols, ldx, codes, ldc, scale, s);
  else if (dtype == MCA_DTYPE_FP16)
    launch_type<MCA_DTYPE_FP16>(x, rows, cols, ldx, codes, ldc, scale, s);
  else
    launch_type<MCA_DTYPE_BF16>(x, rows, cols, ldx, codes, ldc, scale, s);
  return cudaGetLastError();
}

}  // namespace mca
