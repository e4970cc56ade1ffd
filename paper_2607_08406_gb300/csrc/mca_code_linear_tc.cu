// A layer on 8-bit codes for few samples, on the tensor cores: 128 outputs by up to 64 samples per CTA, the columns split
// over the CTAs of a cluster where tiles are few.
//
// The transposed tile D[128 outputs x T samples] = W X^T is what a CTA computes, so that the weights, which are
// most of what is read, are the A operand. TMA brings stages of 128 columns of both code matrices into a ring
// in shared memory; eight warps turn the weights' codes into fp16 in registers and store them to tensor memory (a
// thread per row, 64 columns at a time), four others the samples' codes into the core-matrix layout of the B
// operand in shared memory; one thread issues the MMAs. Weights thus pass through shared memory once as bytes and
// are read back once, which is what limits the rate at which a CTA may take them.
//
// Each CTA of a cluster takes a part of the columns; the sums meet as integers in shared memory, where every CTA of
// the cluster adds up and writes its share of the samples (their order cannot change a result).
//
// Every wait is bounded (2 s). After one that ran out the CTA waits for its own copies, frees its tensor memory and writes
// NaN in its place of y.
#include <algorithm>

#include "mca_code_linear.cuh"

namespace mca {

namespace {

constexpr int kThreads = 448;                 // warps 0-7 convert W, 8-11 X, 12 copies, 13 MMAs
constexpr int kCopyWarp = 12, kMmaWarp = 13;

// T: most samples per tile. NR stages of raw codes, NC of converted ones. (256 tensor-memory columns and
// less than half of the shared memory, so that two CTAs share an SM.)
template <int T>
struct Shape {
  static constexpr int NR = T > 32 ? 3 : 4;
  static constexpr int NC = T > 32 ? 3 : 4;
  static constexpr uint32_t kRaw = kRawW + T * kRawK;
  static constexpr uint32_t kConv = T * kSubK * 2;
  static constexpr uint32_t kSmem = NR * kRaw + NC * kConv + 1024;
};

struct SplitArgs {
  mca_code_linear_args a;
  int splits, stages;                         // CTAs per cluster; stages of all columns
  int box;                                    // samples per box of x's map, a multiple of 16
};

template <int T, int DT>
__global__ void __launch_bounds__(kThreads, 2) code_linear_split_kernel(
    const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap xmap, SplitArgs p) {
  using S = Shape<T>;
  extern __shared__ unsigned char dyn[];
  __shared__ __align__(8) uint64_t s_rawfull[S::NR], s_rawfree[S::NR], s_full[S::NC], s_free[S::NC],
      s_sum, s_taken;
  __shared__ uint32_t s_tmem;
  __shared__ int s_fail;
  const mca_code_linear_args& a = p.a;
  const int tid = threadIdx.x, warp = tid >> 5;
  const int rank = p.splits > 1 ? (int)cluster_rank() : 0;
  const int tile = (int)(blockIdx.x / p.splits), ntiles = (a.n_out + kM - 1) / kM;
  const int n0 = tile % ntiles * kM;
  const int64_t r0 = (int64_t)(tile / ntiles) * T;
  const int nt = (int)min((int64_t)T, a.rows - r0);
  const int n16 = (nt + 15) / 16 * 16;                     // MMA N
  const int c0 = (int)((int64_t)p.stages * rank / p.splits);
  const int nst = (int)((int64_t)p.stages * (rank + 1) / p.splits) - c0;
  constexpr int kPer = kExactK / kRawK;                    // stages whose sum is exact
  const uint32_t raw = (smem_u32(dyn) + 1023u) & ~1023u;
  const uint32_t conv = raw + S::NR * S::kRaw;

  if (warp == kCopyWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 256;"
                 ::"r"(smem_u32(&s_tmem)));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  if (tid == 0) {
    for (int q = 0; q < S::NR; ++q) {
      mbar_init(&s_rawfull[q], 1);
      mbar_init(&s_rawfree[q], kCopyWarp);     // the converting warps
    }
    for (int q = 0; q < S::NC; ++q) {
      mbar_init(&s_full[q], kCopyWarp / 2);
      mbar_init(&s_free[q], 1);
    }
    mbar_init(&s_sum, 1);
    mbar_init(&s_taken, 8);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    s_fail = 0;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  const uint32_t tmem_a = tmem + T;                        // D in columns 0 .. T - 1

  constexpr int kAcc = T / 2;                              // a thread's sums: an output, half of the samples
  int acc[kAcc];
#pragma unroll
  for (int q = 0; q < kAcc; ++q) acc[q] = 0;
  const int half = warp >> 2;                              // of the samples, in the warps 0-7

  if (warp == kCopyWarp) {
    if (elect_one()) {
      int issued = 0;
      for (int c = 0; c < nst; ++c) {
        const int st = c % S::NR;
        if (c >= S::NR && !mbar_wait(&s_rawfree[st], (uint32_t)(c / S::NR - 1) & 1u)) {
          s_fail = 1;
          break;
        }
        const uint32_t bar = smem_u32(&s_rawfull[st]), at = raw + (uint32_t)st * S::kRaw;
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;"
                     ::"r"(bar), "r"(kRawW + (uint32_t)p.box * kRawK) : "memory");
        tma_load(at, &wmap, (c0 + c) * kRawK, n0, bar);
        tma_load(at + kRawW, &xmap, (c0 + c) * kRawK, (int)r0, bar);
        issued = c + 1;
      }
      // copies in flight land before the CTA leaves
      for (int c = issued > S::NR ? issued - S::NR : 0; c < issued; ++c)
        if (!mbar_wait(&s_rawfull[c % S::NR], (uint32_t)(c / S::NR) & 1u)) s_fail = 1;
    }
  } else if (warp == kMmaWarp) {
    if (elect_one()) {
      const uint32_t idesc = tc_idesc_f16(kM, 16) + ((uint32_t)((n16 >> 3) - 2) << 17);
      for (int u = 0; u < 2 * nst; ++u) {
        const int st = u % S::NC, in = u % (2 * kPer);
        if (in == 0 && u > 0 && !mbar_wait(&s_taken, (uint32_t)(u / (2 * kPer) - 1) & 1u)) {
          s_fail = 1;
          break;
        }
        if (!mbar_wait(&s_full[st], (uint32_t)(u / S::NC) & 1u)) {
          s_fail = 1;
          break;
        }
        tc_fence_after();
#pragma unroll
        for (int k = 0; k < kSubK / 16; ++k)
          mma_ts_f16(tmem, tmem_a + (uint32_t)st * kColsA + (uint32_t)k * 8,
                     umma_desc(conv + (uint32_t)st * S::kConv + (uint32_t)k * 2u * (T / 8) * 128,
                               (T / 8) * 128, 128),
                     idesc, in == 0 && k == 0 ? 0u : 1u);
        umma_commit(&s_free[st]);
        if (in == 2 * kPer - 1 || u == 2 * nst - 1) umma_commit(&s_sum);
      }
    }
  } else {
    // stage c holds two operands' columns; half of the warps convert the first, half the second
    const bool isx = warp >= 8;
    const int h = isx ? (warp - 8) >> 1 : warp >> 2;
    const int row = isx ? tid & 63 : tid & 127;
    bool ok = true;
    for (int c = 0; c < nst && ok; ++c) {
      const int st = c % S::NR, u = 2 * c + h, cs = u % S::NC;
      const uint32_t at = raw + (uint32_t)st * S::kRaw + (isx ? kRawW : 0u);
      ok = warp_all(mbar_wait(&s_rawfull[st], (uint32_t)(c / S::NR) & 1u));
      if (ok && u >= S::NC) ok = warp_all(mbar_wait(&s_free[cs], (uint32_t)(u / S::NC - 1) & 1u));
      if (!ok) break;
      tc_fence_after();
#pragma unroll
      for (int part = 0; part < 2; ++part) {
        uint32_t v[16];
        if (!isx) {
          load_codes(at, row, 2 * h + part, v);
          tmem_st16u(tmem_a + (uint32_t)cs * kColsA + (uint32_t)part * 16u +
                         ((uint32_t)((warp & 3) * 32) << 16), v);
        } else if (row < n16) {
          load_codes(at, row, 2 * h + part, v);
          store_codes(conv + (uint32_t)cs * S::kConv, row, T, part, v);
        }
      }
      warp_arrive(&s_rawfree[st]);
      if (!isx) {
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        tc_fence_before();
      } else {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      }
      warp_arrive(&s_full[cs]);
      if (!isx && (c % kPer == kPer - 1 || c == nst - 1)) {   // an exact sum is complete
        ok = warp_all(mbar_wait(&s_sum, (uint32_t)(c / kPer) & 1u));
        if (!ok) break;
        tc_fence_after();
        const uint32_t from = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(half * kAcc);
#pragma unroll
        for (int q = 0; q < kAcc; q += 16) {
          if (half * kAcc + q < n16) {
            float d[16];
            tmem_ld16(from + (uint32_t)q, d);
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[q + i] += __float2int_rn(d[i]);
          }
        }
        tc_fence_before();
        warp_arrive(&s_taken);
      }
    }
    // every MMA's arrival comes before the CTA leaves
    for (int u = max(0, 2 * nst - S::NC); u < 2 * nst && ok; ++u)
      ok = warp_all(mbar_wait(&s_free[u % S::NC], (uint32_t)(u / S::NC) & 1u));
    if (!ok) s_fail = 1;
  }
  __syncwarp();
  __syncthreads();
  const bool fail = s_fail != 0;
  const int ch = tid & 127, n = n0 + ch;
  // the parts of the cluster's CTAs, [sample][output], in the place of the rings
  if (tid < 256) {
#pragma unroll
    for (int q = 0; q < kAcc; ++q)
      if (half * kAcc + q < nt)
        asm volatile("st.shared.s32 [%0], %1;"
                     ::"r"(raw + (uint32_t)((half * kAcc + q) * kM + ch) * 4u), "r"(acc[q])
                     : "memory");
  }
  if (p.splits > 1)
    cluster_sync_all();
  else
    __syncthreads();
  if (tid < 256 && n < a.n_out) {
    const float ws = __ldg(a.w_scale + n), b = a.bias ? __ldg(a.bias + n) : 0.0f;
    elem_t<DT>* y = static_cast<elem_t<DT>*>(a.y) + r0 * a.ldy + n;
    // any CTA of a cluster that failed: its part is missing in every sample
    for (int t = fail ? half : rank * 2 + half; t < nt; t += fail ? 2 : 2 * p.splits) {
      int s = 0;
      if (p.splits > 1)
        for (int q = 0; q < p.splits; ++q) s += ld_cluster(raw + (uint32_t)(t * kM + ch) * 4u, q);
      else
        s = ld_shared(raw + (uint32_t)(t * kM + ch) * 4u);
      const float z = code_field(__int2float_rn(s), __ldg(a.x_scale + r0 + t), ws, b, a.bias != nullptr);
      y[t * a.ldy] = elem_of<DT>(fail ? NAN : act_accurate(a.act, z, a.act_param));
    }
  }
  tc_fence_before();
  if (p.splits > 1)
    cluster_sync_all();
  else
    __syncthreads();
  if (warp == kCopyWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 256;" ::"r"(tmem));
}

template <int T, int DT>
cudaError_t launch_split(const SplitArgs& p, const CUtensorMap& wmap, const CUtensorMap& xmap,
                         cudaStream_t s) {
  constexpr int smem = (int)Shape<T>::kSmem;
  static_assert(Shape<T>::NR * Shape<T>::kRaw + Shape<T>::NC * Shape<T>::kConv >= T * kM * 4,
                "the parts of a split sum take the place of the rings");
  cudaError_t e = cudaFuncSetAttribute(code_linear_split_kernel<T, DT>,
                                       cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned int)(((p.a.n_out + kM - 1) / kM) * ((p.a.rows + T - 1) / T) * p.splits));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned int)p.splits;
  at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, code_linear_split_kernel<T, DT>, wmap, xmap, p);
}

template <int T>
cudaError_t launch_split_t(const SplitArgs& p, const CUtensorMap& wmap, const CUtensorMap& xmap,
                           cudaStream_t s) {
  switch (p.a.dtype) {
    case MCA_DTYPE_FP32: return launch_split<T, MCA_DTYPE_FP32>(p, wmap, xmap, s);
    case MCA_DTYPE_FP16: return launch_split<T, MCA_DTYPE_FP16>(p, wmap, xmap, s);
    default: return launch_split<T, MCA_DTYPE_BF16>(p, wmap, xmap, s);
  }
}

}  // namespace

cudaError_t launch_code_linear_split(const mca_code_linear_args& a, cudaStream_t s) {
  const int T = a.rows <= 32 ? 32 : 64;
  SplitArgs p{};
  p.a = a;
  p.stages = (a.n_in + kRawK - 1) / kRawK;
  p.box = (int)std::min<int64_t>(T, (a.rows + 15) / 16 * 16);
  // clusters of up to 8 CTAs while two CTAs per SM have no tile of their own, two stages each at least
  const int64_t tiles = (int64_t)((a.n_out + kM - 1) / kM) * ((a.rows + T - 1) / T);
  p.splits = 1;
  while (p.splits < 8 && tiles * p.splits * 2 <= 2 * 152 && p.stages >= 4 * p.splits) p.splits *= 2;
  CUtensorMap wmap, xmap;
  cudaError_t e = code_map(&wmap, a.w, a.n_out, a.n_in, a.ldw, kM);
  if (e == cudaSuccess) e = code_map(&xmap, a.x, a.rows, a.n_in, a.ldx, p.box);
  if (e != cudaSuccess) return e;
  return T == 32 ? launch_split_t<32>(p, wmap, xmap, s) : launch_split_t<64>(p, wmap, xmap, s);
}

}  // namespace mca
