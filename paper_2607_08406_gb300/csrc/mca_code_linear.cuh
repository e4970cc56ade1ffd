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
#include "mca_tc.cuh"

namespace mca {

constexpr int kExactK = 1024;
constexpr int kM = 128;                       // outputs per CTA (a CTA's rows of the MMA's M)
constexpr int kRawK = 128;                    // columns per stage of raw codes
constexpr int kSubK = 64;                     // columns per converted operand
constexpr uint32_t kRawW = kM * kRawK;        // bytes
constexpr uint32_t kColsA = kSubK / 2;        // tensor-memory columns of a converted W (two fp16 each)

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

// A field from the sum as fp32: s * xs * ws + b, products and sum rounded one after the other.
__device__ __forceinline__ float code_field(float s, float xs, float ws, float b, bool bias) {
  const float z = __fmul_rn(__fmul_rn(s, xs), ws);
  return bias ? __fadd_rn(z, b) : z;
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
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ void sts128(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w)
               : "memory");
}

// 32 codes of a row (row r of a swizzled box at base, columns 32 part ..) as 16 pairs of fp16.
__device__ __forceinline__ void load_codes(uint32_t base, int r, int part, uint32_t (&v)[16]) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const uint4 q = lds128(base + (uint32_t)r * kRawK + (uint32_t)(((part * 2 + j) ^ (r & 7)) << 4));
    codes_f16(q.x, v[8 * j], v[8 * j + 1]);
    codes_f16(q.y, v[8 * j + 2], v[8 * j + 3]);
    codes_f16(q.z, v[8 * j + 4], v[8 * j + 5]);
    codes_f16(q.w, v[8 * j + 6], v[8 * j + 7]);
  }
}

// The same into the core-matrix layout of an operand of `rows` rows at `to`: units of 8 columns rows * 16 bytes
// apart (part: of the operand's columns).
__device__ __forceinline__ void store_codes(uint32_t to, int r, int rows, int part, const uint32_t (&v)[16]) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
    sts128(to + (uint32_t)((part * 4 + j) * rows + r) * 16u, v[4 * j], v[4 * j + 1], v[4 * j + 2],
           v[4 * j + 3]);
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

__device__ __forceinline__ void tmem_st16u(uint32_t taddr, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16};"
      ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]),
        "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]),
        "r"(v[15])
      : "memory");
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

// Rows that start on 16-byte boundaries.
inline bool code_rows_aligned(const int8_t* p, int64_t rows, int64_t ld) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (rows == 1 || ld % 16 == 0);
}

// mca_code_linear_tc.cu: few samples; operands' rows on 16-byte boundaries.
cudaError_t launch_code_linear_split(const mca_code_linear_args& a, cudaStream_t s);
// mca_code_linear_pair.cu: many samples; in a.workspace the operands as fp16.
size_t code_linear_pair_workspace(const mca_code_linear_args& a);
cudaError_t launch_code_linear_pair(const mca_code_linear_args& a, cudaStream_t s);

}  // namespace mca
