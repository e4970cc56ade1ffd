// A layer on 8-bit codes (mca_code_linear): y = act((x w^T) * x_scale * w_scale + bias). Choice of the kernel, and
// aligned copies of operands whose rows lie off 16-byte boundaries.
#include "mca_code_linear.cuh"

namespace mca {

namespace {

constexpr int64_t kPairRows = 128;

bool use_pair(const mca_code_linear_args& a) { return a.rows > kPairRows; }

int64_t round16(int64_t n) { return (n + 15) / 16 * 16; }
size_t align256(size_t n) { return (n + 255) & ~size_t(255); }

// Sixteen codes per thread, behind the last column zeros.
__global__ void __launch_bounds__(256) align_rows_kernel(const int8_t* __restrict__ src, int64_t rows,
                                                         int cols, int64_t ld, int8_t* __restrict__ dst,
                                                         int units) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t r = i / units;
  const int c = (int)(i - r * units) * 16;
  if (r >= rows) return;
  const int8_t* p = src + r * ld + c;
  union {
    int8_t b[16];
    uint4 u;
  } v;
#pragma unroll
  for (int q = 0; q < 16; ++q) v.b[q] = c + q < cols ? p[q] : (int8_t)0;
  *reinterpret_cast<uint4*>(dst + r * (int64_t)units * 16 + c) = v.u;
}

cudaError_t align_rows(const int8_t** p, int64_t rows, int cols, int64_t* ld, char** ws, cudaStream_t s) {
  if (code_rows_aligned(*p, rows, *ld)) return cudaSuccess;
  int8_t* dst = reinterpret_cast<int8_t*>(*ws);
  const int units = (cols + 15) / 16;
  align_rows_kernel<<<(unsigned int)((rows * units + 255) / 256), 256, 0, s>>>(*p, rows, cols, *ld, dst,
                                                                             units);
  *p = dst;
  *ld = round16(cols);
  *ws += align256((size_t)rows * (size_t)*ld);
  return cudaGetLastError();
}

}  // namespace

size_t code_linear_workspace(const mca_code_linear_args& a) {
  if (use_pair(a)) return code_linear_pair_workspace(a);
  size_t n = 0;
  if (!code_rows_aligned(a.x, a.rows, a.ldx)) n += align256((size_t)a.rows * (size_t)round16(a.n_in));
  if (!code_rows_aligned(a.w, a.n_out, a.ldw)) n += align256((size_t)a.n_out * (size_t)round16(a.n_in));
  return n;
}

cudaError_t launch_code_linear(const mca_code_linear_args& args, cudaStream_t s) {
  if (use_pair(args)) return launch_code_linear_pair(args, s);
  mca_code_linear_args a = args;
  char* ws = static_cast<char*>(a.workspace);
  cudaError_t e = align_rows(&a.x, a.rows, a.n_in, &a.ldx, &ws, s);
  if (e == cudaSuccess) e = align_rows(&a.w, a.n_out, a.n_in, &a.ldw, &ws, s);
  if (e != cudaSuccess) return e;
  return launch_code_linear_split(a, s);
}

cudaError_t code_map(CUtensorMap* map, const int8_t* p, int64_t rows, int64_t cols, int64_t ld,
                     int box_rows) {
  using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                              const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                              CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                              CUtensorMapFloatOOBfill);
  static const Encode encode = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult r;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &r) !=
            cudaSuccess ||
        r != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      f = nullptr;
    }
    return reinterpret_cast<Encode>(f);
  }();
  if (!encode) return cudaErrorNotSupported;
  const cuuint64_t dim[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t stride[1] = {(cuuint64_t)(rows == 1 ? round16(cols) : ld)};
  const cuuint32_t box[2] = {128, (cuuint32_t)box_rows}, step[2] = {1, 1};
  const CUresult e = encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<int8_t*>(p), dim, stride, box,
                            step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return e == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

}  // namespace mca
