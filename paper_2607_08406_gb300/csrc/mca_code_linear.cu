// A layer on 8-bit codes (mca_code_linear): y = act((x w^T) * x_scale * w_scale + bias). Choice of the kernel, and
// aligned copies of operands whose rows lie off 16-byte boundaries.
#include "mca_code_linear.cuh"

namespace mca {

namespace {

enum class Kernel { kStream, kSplit, kPair };

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The kernel by sizes, from times measured on GB300 (us; stream / cluster / pair):
//   rows   n_in n_out              rows    n_in n_out
//     16   4096  4096   9.5 / 12     16   16384  1024  27 / 17
//     64   1024  1024   6.7 / 9      64    8192  8192  52 / 33
//    256   1024  1024   7.0 / 10 / 13    64   4096 16384  57 / 34 / 61
//    128   8192  8192  102 / 39 / 74    512    8192  8192  - / 146 / 77
//    256   4096  4096   57 / 23 / 33    512    4096  4096  - / 38 / 34
//    512  16384  1024  100 / 40 / 86    128     784  4096  14 / 13 / 12
// Few samples stream the weights, as long as a CTA's 32 outputs by 64 samples all run at once and their columns
// are not too many; other products of up to 64 samples take the cluster kernel. Beyond, the cluster kernel (in tiles
// of 128 samples) takes about 3 us and, for each round of its CTAs, 4 us and 1.03 us for every stage of 128 columns,
// the pair kernel 9 us, the operands' way to fp16 and back (3 bytes a code) and 4.1 ns for each column of its rounds
// of tiles. Not in the rule: the copy of operands whose rows lie off 16-byte boundaries (a launch, in either of the
// first two kernels), and few outputs, which leave most of a tile of 128 or 256 idle in both (60000 x 4096 -> 10
// takes 167 us, 37 of them the samples' way from memory).
Kernel choose(const mca_code_linear_args& a) {
  const int64_t rows = a.rows, n_in = a.n_in, n_out = a.n_out, sms = 152;
  if (rows <= 8) return Kernel::kStream;
  if (rows <= 32) return n_in <= 8192 ? Kernel::kStream : Kernel::kSplit;
  if (n_in <= 2560 && ceil_div(n_out, 32) * ceil_div(rows, 64) <= sms) return Kernel::kStream;
  if (rows <= 64) return Kernel::kSplit;
  const double split = code_linear_split_us(a);
  const double pair = 9.0 + 3.0 * (double)n_in * (double)(n_out + rows) / 5.5e6 +
                      0.0041 * (double)(ceil_div(ceil_div(n_out, 256) * ceil_div(rows, 256), sms / 2) * n_in);
  return split < pair ? Kernel::kSplit : Kernel::kPair;
}

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
  if (choose(a) == Kernel::kPair) return code_linear_pair_workspace(a);
  size_t n = 0;
  if (!code_rows_aligned(a.x, a.rows, a.ldx)) n += align256((size_t)a.rows * (size_t)round16(a.n_in));
  if (!code_rows_aligned(a.w, a.n_out, a.ldw)) n += align256((size_t)a.n_out * (size_t)round16(a.n_in));
  return n;
}

cudaError_t launch_code_linear(const mca_code_linear_args& args, cudaStream_t s) {
  if (choose(args) == Kernel::kPair) return launch_code_linear_pair(args, s);
  mca_code_linear_args a = args;
  char* ws = static_cast<char*>(a.workspace);
  cudaError_t e = align_rows(&a.x, a.rows, a.n_in, &a.ldx, &ws, s);
  if (e == cudaSuccess) e = align_rows(&a.w, a.n_out, a.n_in, &a.ldw, &ws, s);
  if (e != cudaSuccess) return e;
  return choose(a) == Kernel::kStream ? launch_code_linear_stream(a, s) : launch_code_linear_split(a, s);
}

}  // namespace mca
