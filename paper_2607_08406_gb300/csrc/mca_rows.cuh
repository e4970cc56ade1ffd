// Rows of a caller's logits as 16-byte pieces, for the kernels that read every logit once: a team of W warps has a row, or
// a CTA of a cluster a part of one.
#pragma once

#include <cstdint>
#include <type_traits>

#include <cuda_runtime.h>

#include "mca_elem.cuh"

namespace mca {

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// A team of W warps: a warp by itself, or a CTA.
template <int W>
__device__ __forceinline__ void team_sync() {
  __syncwarp();
  if constexpr (W > 1) __syncthreads();
}

// A row's 16-byte pieces: piece j holds the logits j N - head .. of the row (the first and the last in part).
template <int DT>
struct Pieces {
  static constexpr int N = 16 / (int)sizeof(elem_t<DT>);
  const elem_t<DT>* x;
  int V, head, count;
  __host__ __device__ __forceinline__ Pieces(const elem_t<DT>* x_, int V_) : x(x_), V(V_) {
    head = (int)(reinterpret_cast<uintptr_t>(x) % 16 / sizeof(elem_t<DT>));
    count = (int)(((int64_t)V + head + N - 1) / N);
  }
  __host__ __device__ __forceinline__ int index(int j, int i) const { return j * N - head + i; }
  __host__ __device__ __forceinline__ bool whole(int j) const {
    return j * N >= head && (int64_t)(j + 1) * N <= (int64_t)V + head;
  }
  __host__ __device__ __forceinline__ const uint4* pieces() const { return reinterpret_cast<const uint4*>(x - head); }
  __host__ __device__ __forceinline__ uint4 raw(int j) const { return pieces()[j]; }
  __device__ __forceinline__ static void values(const uint4& q, float (&v)[N]) {
    const unsigned int w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (DT == MCA_DTYPE_FP32)
        v[i] = __uint_as_float(w[i]);
      else if constexpr (DT == MCA_DTYPE_BF16)
        v[i] = __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
      else
        v[i] = __half2float(__ushort_as_half((unsigned short)(i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xffffu)));
    }
  }
  // Any piece of the row, -inf in the place of what is outside.
  __host__ __device__ __forceinline__ uint4 bits(int j) const {
    return whole(j) ? raw(j) : part(x, V, index(j, 0));
  }
  __host__ __device__ __noinline__ static uint4 part(const elem_t<DT>* x, int V, int at) {
    union {
      elem_t<DT> e[N];
      uint4 u;
    } o;
#pragma unroll
    for (int i = 0; i < N; ++i) o.e[i] = at + i >= 0 && at + i < V ? x[at + i] : elem_of<DT>(-INFINITY);
    return o.u;
  }
  __device__ __forceinline__ void load(int j, float (&v)[N]) const { values(bits(j), v); }
};

// The largest logit of a piece (NaN if one is).
template <int DT>
__device__ __forceinline__ float largest(const uint4& q) {
  if constexpr (DT == MCA_DTYPE_FP32) {
    return max_nan(max_nan(__uint_as_float(q.x), __uint_as_float(q.y)),
                   max_nan(__uint_as_float(q.z), __uint_as_float(q.w)));
  } else if constexpr (DT == MCA_DTYPE_BF16) {
    unsigned int m;
    asm("{\n\t.reg .b32 a, b;\n\tmax.NaN.bf16x2 a, %1, %2;\n\tmax.NaN.bf16x2 b, %3, %4;\n\t"
        "max.NaN.bf16x2 %0, a, b;\n\t}" : "=r"(m) : "r"(q.x), "r"(q.y), "r"(q.z), "r"(q.w));
    return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
  } else {
    unsigned int m;
    asm("{\n\t.reg .b32 a, b;\n\tmax.NaN.f16x2 a, %1, %2;\n\tmax.NaN.f16x2 b, %3, %4;\n\t"
        "max.NaN.f16x2 %0, a, b;\n\t}" : "=r"(m) : "r"(q.x), "r"(q.y), "r"(q.z), "r"(q.w));
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&m));
    return max_nan(f.x, f.y);
  }
}

// Rows whose pieces are cut from two 16-byte blocks, because they lie `by` bytes behind the pieces of another row of V
// elements (`head` of them less in its first piece): the first of the pieces whose blocks hold the row's own elements
// alone, and the one behind the last. What else a block at an end of the row holds is not the caller's to read from.
__host__ __device__ inline int first_of_own_blocks(int head, int by, int bytes) { return (head * bytes + by + 15) / 16; }
__host__ __device__ inline int end_of_own_blocks(int V, int head, int by, int bytes) {
  const int64_t to = (int64_t)(V + head) * bytes + by;         // from the first block's start to the row's end
  return (int)(to / 16) - (by ? 1 : 0);
}

// The 16 bytes that start `by` bytes (a multiple of 2) behind the start of lo.
__device__ __forceinline__ uint4 shifted(const uint4& lo, const uint4& hi, unsigned int by) {
  unsigned int w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
  if (by & 8u) {
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
  }
  if (by & 4u) {
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
  }
  const unsigned int bits = (by & 3u) * 8u;
  return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits),
                    __funnelshift_r(w[2], w[3], bits), __funnelshift_r(w[3], w[4], bits));
}

struct NoRounds {};

// Pieces j0 + tid, j0 + tid + 32 W, .. below j1 of a row, in this order: take(piece, j), after begin(). `AHEAD` of them are
// on their way to shared memory, each to its thread's own places: no registers, no barriers. A piece at an end of the row
// that is not whole is put there by its thread. Or rounds(one) has a warp's rounds, whose pieces start at base, in turn by
// one(base, what), all lanes: take(piece, what).
template <int DT, int W, int AHEAD, class Begin, class Rounds, class Take>
__device__ __forceinline__ void stream_pieces(const Pieces<DT>& row, int j0, int j1, uint4 (&s_ring)[AHEAD][32 * W],
                                              Begin begin, Rounds rounds, Take take) {
  constexpr int kTeam = 32 * W;
  const int tid = threadIdx.x;
  const unsigned int ring = (unsigned int)__cvta_generic_to_shared(&s_ring[0][tid]);
  constexpr unsigned int kSlot = kTeam * 16;
  const int w0 = row.whole(0) ? 0 : 1, whole = row.count - w0 - (row.whole(row.count - 1) ? 0 : 1);
  unsigned int slot = ring;
  int next = j0 + tid;
  const uint4* x = row.pieces() + next;                         // of piece `next`
  auto ask = [&] {
    if (next < j1) {
      if ((unsigned int)(next - w0) < (unsigned int)whole) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(slot), "l"(x) : "memory");
      } else {
        const uint4 q = Pieces<DT>::part(row.x, row.V, row.index(next, 0));
        asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};"
                     ::"r"(slot), "r"(q.x), "r"(q.y), "r"(q.z), "r"(q.w) : "memory");
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    next += kTeam;
    x += kTeam;
    slot = slot == ring + (AHEAD - 1) * kSlot ? ring : slot + kSlot;
  };
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) ask();
  begin();
  auto next_piece = [&](auto what) {
    uint4 q;
    asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD - 1) : "memory");
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "r"(slot) : "memory");
    take(q, what);
    ask();
  };
  if constexpr (std::is_same_v<Rounds, NoRounds>) {
    for (int j = j0 + tid; j < j1; j += kTeam) next_piece(j);
  } else {
    rounds([&](int base, auto what) {
      if (base + (tid & 31) < j1) next_piece(what);
    });
  }
}

__device__ __forceinline__ unsigned int cluster_rank() {
  unsigned int r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_arrive() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
  __syncwarp();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ unsigned int first_cta(const void* p) {      // the address in the cluster's first CTA
  unsigned int a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;"
               : "=r"(a) : "r"((unsigned int)__cvta_generic_to_shared(p)));
  return a;
}

// One launch of `grid` CTAs, `split` of which are a cluster.
template <class... Params, class... Args>
inline cudaError_t launch_clusters(void (*kernel)(Params...), int64_t grid, int threads, int split, cudaStream_t s,
                                   Args... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned int)grid);
  cfg.blockDim = dim3((unsigned int)threads);
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned int)split;
  at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace mca
