// A layer on 8-bit codes for some dozens of samples, on the tensor cores: 128 outputs by up to 128 samples per CTA, the
// columns split over the CTAs of a cluster where tiles are few.
//
// The transposed tile D[128 outputs x T samples] = W X^T is what a CTA computes, so that the weights, which are
// most of what is read, fill the M of the MMAs. Twelve warps load codes, eight the weights' and four the samples',
// 16 rows and 128 columns each at a time, two stages ahead of the one that they turn into fp16 and store in core-matrix
// order for the MMAs (SS form) of one thread. Per stage a warp waits for one barrier, the stage's place: a wait
// takes 200 cycles even if nothing is left to wait for. (With the codes brought by TMA into a ring, converted to
// tensor memory, a warp waited twice for half as many codes: 4096 -> 16384 for 16 samples took 24 us.)
//
// A row's 16 codes lie in two units of 8 columns; four threads of a row and eight rows share a store's quarter. The
// units' distance is a multiple of 128 bytes plus 16, so that a quarter (two rows by four units) meets every bank once.
//
// 8192 -> 8192 takes 39 us for 128 samples, 32 for 64: about 1 us for a CTA's stage of 16 KB of weights, which the
// conversions (130 instructions for 16 rows of 128 columns), the hand-overs and the loads' latency share; an M = 128
// MMA takes 80 cycles even for 16 samples, so that the tensor cores would allow 25 bytes of weights per cycle and SM.
//
// Each CTA of a cluster takes a part of the columns; the sums meet as integers in shared memory, where every CTA of
// the cluster adds up and writes its share of the samples (their order cannot change a result).
//
// Every wait is bounded (2 s). After one that ran out the CTA frees its tensor memory and writes NaN in its place of y.
#include <algorithm>

#include "mca_code_linear.cuh"

namespace mca {

namespace {

constexpr int kStageK = 128;                  // columns per stage
constexpr int kRowsWarp = 16;                 // rows that a warp converts
constexpr int kWWarps = kM / kRowsWarp;

template <int T>
struct Shape {
  static constexpr int kNC = T > 64 ? 3 : 2;                   // stages
  static constexpr int kXWarps = T / kRowsWarp;
  static constexpr int kConvWarps = kWWarps + kXWarps;
  static constexpr int kThreads = 32 * (kConvWarps + 1);       // and one warp that issues MMAs
  static constexpr uint32_t kLboW = kM * 16 + 16, kLboX = T * 16 + 16;     // units of 8 columns
  static constexpr uint32_t kW = (kStageK / 8) * kLboW;
  static constexpr uint32_t kStage = kW + (kStageK / 8) * kLboX;
  static constexpr uint32_t kSmem = kNC * kStage + 128;
  static constexpr uint32_t kTmem = 2 * T;      // the sums of the MMAs, and whole sums as integers
  static constexpr int kParts = T > 64 ? 4 : 2;                // of the samples, of which a warp takes one's sums
  static constexpr int kGroups = kConvWarps / 4;               // of 128 threads that write outputs
  static_assert(kNC * kStage >= T * kM * 4, "the parts of a split sum take the place of the stages");
};

struct SplitArgs {
  mca_code_linear_args a;
  int splits, stages;                         // CTAs per cluster; stages of all columns
};

// A thread's codes of a stage: rows g and g + 8 of its warp's, 16 columns from 16 t and from 64 + 16 t.
struct Codes {
  uint4 v[4];
  __device__ __forceinline__ void load(const int8_t* r0, const int8_t* r1, int k, int n) {
    v[0] = load_codes16(r0, k, n);
    v[1] = load_codes16(r0, k + 64, n);
    v[2] = load_codes16(r1, k, n);
    v[3] = load_codes16(r1, k + 64, n);
  }
  __device__ __forceinline__ void store(uint32_t to, int row, int t, uint32_t lbo) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t h[8];
      codes_f16(v[i].x, h[0], h[1]);
      codes_f16(v[i].y, h[2], h[3]);
      codes_f16(v[i].z, h[4], h[5]);
      codes_f16(v[i].w, h[6], h[7]);
      const uint32_t at = to + (uint32_t)(2 * t + 8 * (i & 1)) * lbo + (uint32_t)(row + 8 * (i >> 1)) * 16u;
      sts128(at, h[0], h[1], h[2], h[3]);
      sts128(at + lbo, h[4], h[5], h[6], h[7]);
    }
  }
};

template <int T, int DT>
__global__ void __launch_bounds__(Shape<T>::kThreads, T > 64 ? 1 : 2) code_linear_split_kernel(SplitArgs p) {
  using S = Shape<T>;
  constexpr int kNC = S::kNC;
  extern __shared__ unsigned char dyn[];
  __shared__ __align__(8) uint64_t s_full[kNC], s_free[kNC], s_sum, s_taken;
  __shared__ uint32_t s_tmem;
  __shared__ int s_fail;
  __shared__ float s_scale[T];
  const mca_code_linear_args& a = p.a;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = p.splits > 1 ? (int)cluster_rank() : 0;
  const int tile = (int)(blockIdx.x / p.splits), ntiles = (a.n_out + kM - 1) / kM;
  const int n0 = tile % ntiles * kM;
  const int64_t r0 = (int64_t)(tile / ntiles) * T;
  const int nt = (int)min((int64_t)T, a.rows - r0);
  const int n16 = (nt + 15) / 16 * 16;                     // MMA N
  const int c0 = (int)((int64_t)p.stages * rank / p.splits);
  const int nst = (int)((int64_t)p.stages * (rank + 1) / p.splits) - c0;
  constexpr int kPer = kExactK / kStageK;                  // stages whose sum is exact
  const uint32_t buf = (smem_u32(dyn) + 127u) & ~127u;

  if (warp == S::kConvWarps) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32(&s_tmem)), "n"(S::kTmem));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  if (tid == 0) {
    for (int q = 0; q < kNC; ++q) {
      mbar_init(&s_full[q], kWWarps + n16 / kRowsWarp);
      mbar_init(&s_free[q], 1);
    }
    mbar_init(&s_sum, 1);
    mbar_init(&s_taken, 4 * S::kParts);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    s_fail = 0;
  }
  if (tid < nt) s_scale[tid] = __ldg(a.x_scale + r0 + tid);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;

  constexpr int kPart = T / S::kParts;

  if (warp == S::kConvWarps) {
    if (elect_one()) {
      const uint32_t idesc = tc_idesc_f16(kM, 16) + ((uint32_t)((n16 >> 3) - 2) << 17);
      bool ok = true;
      for (int c = 0; c < nst; ++c) {
        const int st = c % kNC, in = c % kPer;
        if (in == 0 && c > 0) ok = mbar_wait(&s_taken, (uint32_t)(c / kPer - 1) & 1u);
        ok = ok && mbar_wait(&s_full[st], (uint32_t)(c / kNC) & 1u);
        if (!ok) {
          s_fail = 1;
          break;
        }
        tc_fence_after();
        const uint32_t w = buf + (uint32_t)st * S::kStage, x = w + S::kW;
#pragma unroll
        for (uint32_t k = 0; k < kStageK / 16; ++k)
          mma_ss_f16(tmem, umma_desc(w + 2u * k * S::kLboW, S::kLboW, 128),
                     umma_desc(x + 2u * k * S::kLboX, S::kLboX, 128), idesc, in == 0 && k == 0 ? 0u : 1u);
        umma_commit(&s_free[st]);
        if (in == kPer - 1 || c == nst - 1) umma_commit(&s_sum);
      }
    }
  } else {
    const bool isx = warp >= kWWarps;
    const int t = lane & 3, row = (isx ? warp - kWWarps : warp) * kRowsWarp + (lane >> 2);
    // rows behind the last are read as the last; their sums are not used
    const int8_t* const p0 = isx ? a.x + (r0 + min(row, nt - 1)) * a.ldx
                                 : a.w + (int64_t)min(n0 + row, a.n_out - 1) * a.ldw;
    const int8_t* const p1 = isx ? a.x + (r0 + min(row + 8, nt - 1)) * a.ldx
                                 : a.w + (int64_t)min(n0 + row + 8, a.n_out - 1) * a.ldw;
    const uint32_t lbo = isx ? S::kLboX : S::kLboW;
    const bool has = !isx || row < n16, sums = warp < 4 * S::kParts;
    bool ok = true;
    // two stages of codes on their way: each is asked for when the one before the last has been stored
    Codes even, odd;
    auto load = [&](Codes& v, int c) {
      if (has && c < nst) v.load(p0, p1, (c0 + c) * kStageK + 16 * t, a.n_in);
    };
    auto convert = [&](Codes& v, int c) {
      if (!has) return;
      const int st = c % kNC;
      if (c >= kNC) ok = warp_all(mbar_wait(&s_free[st], (uint32_t)(c / kNC - 1) & 1u));
      if (!ok) return;
      v.store(buf + (uint32_t)st * S::kStage + (isx ? S::kW : 0u), row, t, lbo);
      load(v, c + 2);
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      warp_arrive(&s_full[st]);
    };
    load(even, 0);
    load(odd, 1);
    for (int c = 0; c < nst && ok; c += 2) {
      convert(even, c);
      if (ok && c + 1 < nst) convert(odd, c + 1);
      const int last = min(c + 1, nst - 1);
      if (sums && ok && (last % kPer == kPer - 1 || last == nst - 1)) {   // an exact sum is complete
        ok = warp_all(mbar_wait(&s_sum, (uint32_t)(last / kPer) & 1u));
        if (!ok) break;
        tc_fence_after();
        // added to what is there already; the last one leaves for shared memory, [sample][output], in the place
        // of the stages, which the MMAs have read
        const int t0 = (warp >> 2) * kPart;
        const uint32_t from = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)t0;
        const uint32_t to = buf + (uint32_t)(t0 * kM + (warp & 3) * 32 + lane) * 4u;
#pragma unroll 1
        for (int q = 0; q < kPart && t0 + q < n16; q += 16) {
          float d[16], e[16];
          tmem_ld16(from + (uint32_t)q, d);
          if (last >= kPer) tmem_ld16(from + (uint32_t)(T + q), e);
          int v[16];
#pragma unroll
          for (int i = 0; i < 16; ++i)
            v[i] = __float2int_rn(d[i]) + (last >= kPer ? __float_as_int(e[i]) : 0);
          if (last == nst - 1) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
              asm volatile("st.shared.s32 [%0], %1;" ::"r"(to + (uint32_t)((q + i) * kM) * 4u), "r"(v[i])
                           : "memory");
          } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) e[i] = __int_as_float(v[i]);
            tmem_st16(from + (uint32_t)(T + q), e);
          }
        }
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        tc_fence_before();
        warp_arrive(&s_taken);
      }
    }
    // every MMA's arrival comes before the CTA leaves
    for (int c = max(0, nst - kNC); c < nst && ok && has; ++c)
      ok = warp_all(mbar_wait(&s_free[c % kNC], (uint32_t)(c / kNC) & 1u));
    if (!ok) s_fail = 1;
  }
  tc_fence_before();
  __syncwarp();
  __syncthreads();
  // The sums are in shared memory. Tensor memory goes back before the CTA waits for others: a kernel that wants it on
  // this SM may hold up one that the cluster's other CTAs wait for.
  if (warp == S::kConvWarps) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::kTmem));
  }
  bool fail = s_fail != 0;
  if (p.splits > 1) {
    cluster_sync_all();
    for (int q = 0; q < p.splits; ++q) fail |= ld_cluster(smem_u32(&s_fail), q) != 0;
  }
  const int ch = tid & 127, grp = tid >> 7, n = n0 + ch;
  if (grp < S::kGroups && n < a.n_out) {
    const float ws = __ldg(a.w_scale + n), b = a.bias ? __ldg(a.bias + n) : 0.0f;
    const int step = S::kGroups * p.splits;
    int t = rank * S::kGroups + grp;
    elem_t<DT>* y = static_cast<elem_t<DT>*>(a.y) + (r0 + t) * a.ldy + n;
    const int64_t ystep = (int64_t)step * a.ldy;
    uint32_t at = buf + (uint32_t)(t * kM + ch) * 4u;
    for (; t < nt; t += 8 * step, at += (uint32_t)(8 * step * kM) * 4u) {
      int v[8];
      float z[8];
      if (p.splits == 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = t + i * step < nt ? ld_shared(at + (uint32_t)(i * step * kM) * 4u) : 0;
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0;
        for (int q = 0; q < p.splits; ++q)
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (t + i * step < nt) v[i] += ld_cluster(at + (uint32_t)(i * step * kM) * 4u, q);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        z[i] = code_field(__int2float_rn(v[i]), s_scale[min(t + i * step, T - 1)], ws, b, a.bias != nullptr);
      act_block(z, a.act, a.act_param);
#pragma unroll
      for (int i = 0; i < 8; ++i, y += ystep)
        if (t + i * step < nt) *y = elem_of<DT>(fail ? NAN : z[i]);
    }
  }
  if (p.splits > 1) cluster_sync_all();          // the others have read this CTA's sums
}

template <int T, int DT>
cudaError_t launch_split(const SplitArgs& p, cudaStream_t s) {
  constexpr int smem = (int)Shape<T>::kSmem;
  cudaError_t e = cudaFuncSetAttribute(code_linear_split_kernel<T, DT>,
                                       cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned int)(((p.a.n_out + kM - 1) / kM) * ((p.a.rows + T - 1) / T) * p.splits));
  cfg.blockDim = dim3(Shape<T>::kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned int)p.splits;
  at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, code_linear_split_kernel<T, DT>, p);
}

template <int T>
cudaError_t launch_split_t(const SplitArgs& p, cudaStream_t s) {
  switch (p.a.dtype) {
    case MCA_DTYPE_FP32: return launch_split<T, MCA_DTYPE_FP32>(p, s);
    case MCA_DTYPE_FP16: return launch_split<T, MCA_DTYPE_FP16>(p, s);
    default: return launch_split<T, MCA_DTYPE_BF16>(p, s);
  }
}

constexpr int kSms = 152;

// Samples per tile, and CTAs per cluster: up to 8 while places for CTAs have no tile of their own, two stages
// each at least.
struct Plan {
  int T, per_sm, splits, stages;
  int64_t tiles;
  explicit Plan(const mca_code_linear_args& a) {
    T = a.rows <= 32 ? 32 : a.rows <= 64 ? 64 : 128;
    per_sm = T > 64 ? 1 : 2;
    stages = (a.n_in + kStageK - 1) / kStageK;
    tiles = (int64_t)((a.n_out + kM - 1) / kM) * ((a.rows + T - 1) / T);
    splits = 1;
    while (splits < 8 && tiles * splits * 2 <= per_sm * kSms && stages >= 4 * splits) splits *= 2;
  }
};

}  // namespace

double code_linear_split_us(const mca_code_linear_args& a) {
  const Plan p(a);
  const int64_t places = p.per_sm * kSms, rounds = (p.tiles * p.splits + places - 1) / places;
  return 3.0 + (double)rounds * (4.0 + 1.03 * (double)((p.stages + p.splits - 1) / p.splits));
}

cudaError_t launch_code_linear_split(const mca_code_linear_args& a, cudaStream_t s) {
  const Plan plan(a);
  SplitArgs p{};
  p.a = a;
  p.stages = plan.stages;
  p.splits = plan.splits;
  return plan.T == 32   ? launch_split_t<32>(p, s)
         : plan.T == 64 ? launch_split_t<64>(p, s)
                        : launch_split_t<128>(p, s);
}

}  // namespace mca
