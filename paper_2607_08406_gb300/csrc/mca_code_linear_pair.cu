// A layer on 8-bit codes for many samples, on the tensor cores: pairs of CTAs (tcgen05 cta_group::2) on tiles of 256
// outputs by 256 samples, one persistent pair per two SMs.
//
// The codes of both operands are first written out as fp16 (code_image_kernel), in the order in which the MMAs read
// them: blocks of 128 rows, cut into chunks of 64 columns, a chunk's units of 8 columns one after another. That
// is 3 bytes of traffic per code, once, while a tile's products would convert every code again for each 256 rows
// of the other operand: with converting warps between a ring of codes and the MMAs (1740 cycles per 128 columns, 560
// of them issuing the conversions, against 896 cycles of MMAs) 8192 x 8192 -> 8192 took 965 us.
//
// Each CTA of a pair takes 128 of the outputs and half of the samples; the MMA reads both halves of the samples.
// Tensor copies bring chunks (16 KB of each operand) into a ring of six stages. The sums have two places in tensor
// memory (2 x 256 columns): while one is read, scaled and written, the next tile's MMAs run.
//
// The first CTA's MMAs read what both CTAs' copies brought: the copies of both (cta_group::2) count their bytes on the
// first CTA's barrier, which orders them for the cluster. That the second CTA's sums have been read is passed on by one
// of its threads, with the cluster's scope: an arrival of that scope takes 1200 cycles, which nothing waits for there
// (from each warp that takes sums 14346 x 64 -> 15616 fp16 took 171 us, so 157 on the same GPU; with a thread that
// handed over each chunk 8192 x 8192 -> 8192 took 1600 us, so 600).
//
// 8192 x 8192 -> 8192: 594 us, 1.85 PFLOP/s with the conversion, the tensor cores 87 % busy. With few columns the
// operands' way from L2 bounds it: 784 -> 4096 on 60000 samples takes 255 us (outputs fp16), 206 of them MMAs at the
// measured peak, while 13 TB/s leave L2 and 0.5 GB of outputs are written; transfer functions add to that (Gaussian:
// 293 us). With fewer still it is the outputs' instructions, 11 a field and the function's: 14346 x 64 -> 15616 fp16
// takes 147 us, Gaussian 214, GELU 245 (66 are the outputs' way to memory).
//
// Warps: 0 copies, 1 issues MMAs (in the pair's first CTA) or passes on that sums are read (in the second), 4-19 take
// the sums (each 32 outputs and a quarter of the samples). Sums of more than 1024 columns are added up as integers in
// registers and returned to tensor memory as fp32, from where the outputs are written in one loop.
//
// Every wait is bounded (2 s). After one that ran out the later ones do too, and the outputs not yet written
// become NaN.
#include <algorithm>

#include <cuda.h>

#include "mca_code_linear.cuh"

namespace mca {

namespace {

constexpr int kTB = 128;                        // samples per CTA
constexpr int kT = 2 * kTB;                     // samples per tile (MMA N)
constexpr int kFirstSum = 4, kSumWarps = 16;    // warps that take the sums
constexpr int kPart = kT / (kSumWarps / 4);     // samples of one
constexpr int kPairThreads = 32 * (kFirstSum + kSumWarps);
constexpr int kSubK = 64;                       // columns per chunk
constexpr int kStages = 6;
constexpr uint32_t kChunk = kM * kSubK * 2;     // bytes of a block's chunk of 64 columns
constexpr uint32_t kStage = 2 * kChunk;
// The images as a matrix of 32-bit words for the tensor copies: a chunk is a box of kBoxRows rows.
constexpr uint32_t kBoxWords = 256, kBoxRows = kChunk / (4 * kBoxWords);
constexpr uint32_t kPairSmem = kStages * kStage + 1024;
constexpr int kGroup = 8;                       // tiles of outputs that are taken together: so many at least,
constexpr size_t kGroupBytes = 32 << 20;        //   and all whose weights are in so many bytes of L2
constexpr uint32_t kIdesc = tc_idesc_f16(2 * kM, kT);

struct PairArgs {
  mca_code_linear_args a;
  CUtensorMap images;                           // of the weights, and behind them of the samples
  int ximg;                                     // the samples' first chunk
  int chunks;                                   // of 64 columns
  int nt_out, nt_rows;                          // tiles
  int group;                                    // tiles of outputs that are taken together
};

// Rows' codes as fp16 in chunks of kM rows by 64 columns. A thread: a row's 64 columns (behind the last column
// zeros; rows behind the last row are left as they are, and reach only sums that nobody reads).
struct ImageArgs {
  const int8_t* p;
  int64_t rows, ld;
  unsigned char* img;
  int wide;                                     // rows start on 16-byte boundaries
};

__global__ void __launch_bounds__(kM) code_image_kernel(ImageArgs w, ImageArgs x, int64_t wblocks, int cols,
                                                        int chunks) {
  const int64_t blk = (int64_t)blockIdx.x / chunks;
  const int c = (int)(blockIdx.x - blk * chunks);
  const ImageArgs& o = blk < wblocks ? w : x;
  const int64_t b = blk < wblocks ? blk : blk - wblocks;
  const int64_t r = b * kM + threadIdx.x;
  if (r >= o.rows) return;
  const int8_t* p = o.p + r * o.ld + (int64_t)c * kSubK;
  const int n = cols - c * kSubK;               // columns left
  uint4 q[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (o.wide && 16 * j + 16 <= n) {
      q[j] = __ldg(reinterpret_cast<const uint4*>(p) + j);
    } else {
      uint32_t v[4] = {0u, 0u, 0u, 0u};
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (16 * j + i < n) v[i >> 2] |= (uint32_t)(uint8_t)p[16 * j + i] << (8 * (i & 3));
      q[j] = make_uint4(v[0], v[1], v[2], v[3]);
    }
  }
  unsigned char* to = o.img + ((size_t)b * chunks + c) * kChunk + threadIdx.x * 16u;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    uint4 u;
    const uint32_t a0 = j & 1 ? q[j >> 1].z : q[j >> 1].x, a1 = j & 1 ? q[j >> 1].w : q[j >> 1].y;
    codes_f16(a0, u.x, u.y);
    codes_f16(a1, u.z, u.w);
    *reinterpret_cast<uint4*>(to + (size_t)j * kM * 16u) = u;
  }
}

__device__ __forceinline__ void mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t acc) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
               "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}\n"
               ::"r"(d), "l"(a), "l"(b), "r"(kIdesc), "r"(acc));
}
// Arrive on both CTAs' barrier once every MMA issued before has completed.
__device__ __forceinline__ void commit_pair(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 "
               "[%0], %1;"
               ::"r"(smem_u32(bar)), "h"((uint16_t)3) : "memory");
}
// The first CTA's barrier.
__device__ __forceinline__ uint32_t first_bar(uint64_t* bar) {
  uint32_t at;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(at) : "r"(smem_u32(bar)));
  return at;
}
// Arrive there, with what this thread has seen.
__device__ __forceinline__ void arrive_first(uint64_t* bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(first_bar(bar)) : "memory");
}
// One thread: a chunk of the images into shared memory, completing its bytes on the first CTA's bar.
__device__ __forceinline__ void copy_chunk(uint32_t dst, const CUtensorMap* images, int chunk, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes "
               "[%0], [%1, {%2, %3}], [%4];"
               ::"r"(dst), "l"(images), "r"(0), "r"(chunk * (int)kBoxRows), "r"(bar) : "memory");
}
// mbar_wait for arrivals of the other CTA.
__device__ __forceinline__ bool wait_pair(uint64_t* bar, uint32_t parity) {
  const uint32_t at = smem_u32(bar);
  unsigned long long t0 = 0ull;
  for (unsigned int it = 0;; ++it) {
    uint32_t done;
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}\n" : "=r"(done) : "r"(at), "r"(parity) : "memory");
    if (done) return true;
    if ((it & 1023u) == 1023u) {
      const unsigned long long now = globaltimer_ns();
      if (t0 == 0ull)
        t0 = now;
      else if (now - t0 > kBarrierTimeoutNs)
        return false;
    }
  }
}

// Tile of place i in the order of work: some tiles of outputs at a time, for all samples, so that the pairs at
// work share their operands in L2.
__device__ __forceinline__ void tile_at(const PairArgs& p, int i, int* n0, int64_t* r0) {
  const int per = p.group * p.nt_rows, g = i / per, k = i - g * per;
  const int gn = min(p.group, p.nt_out - g * p.group);
  *n0 = (g * p.group + k % gn) * 2 * kM;
  *r0 = (int64_t)(k / gn) * kT;
}

template <int DT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
    code_linear_pair_kernel(const __grid_constant__ PairArgs p) {
  extern __shared__ unsigned char dyn[];
  __shared__ __align__(8) uint64_t s_full[kStages], s_free[kStages], s_sum[2], s_taken[2];
  __shared__ uint32_t s_tmem;
  __shared__ __align__(16) float s_scale[kSumWarps][kPart];   // of a tile's samples, for each warp that takes sums
  const mca_code_linear_args& a = p.a;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = (int)cluster_rank();
  const int first = (int)(blockIdx.x >> 1), step = (int)(gridDim.x >> 1), tiles = p.nt_out * p.nt_rows;
  const int nch = p.chunks;
  constexpr int kPer = kExactK / kSubK;                                      // chunks of an exact sum
  const int nsum = (nch + kPer - 1) / kPer;                                  // exact sums per tile
  const uint32_t ring = (smem_u32(dyn) + 1023u) & ~1023u;

  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;"
                 ::"r"(smem_u32(&s_tmem)));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  }
  if (tid == 32) {
    for (int q = 0; q < kStages; ++q) {
      mbar_init(&s_full[q], 1);                   // the first CTA's: the bytes of both
      mbar_init(&s_free[q], 1);
    }
    for (int q = 0; q < 2; ++q) {
      mbar_init(&s_sum[q], 1);
      mbar_init(&s_taken[q], kSumWarps + (rank == 0 ? 1 : 0));   // and the second CTA's thread that passes it on
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem = s_tmem;

  if (warp == 0) {
    if (elect_one()) {
      bool ok = true;
      int at = 0;                               // chunks issued
      for (int i = first; i < tiles && ok; i += step) {
        int n0;
        int64_t r0;
        tile_at(p, i, &n0, &r0);
        const int w = (n0 / kM + rank) * nch, x = p.ximg + (int)(r0 / kTB + rank) * nch;
        for (int c = 0; c < nch; ++c, ++at) {
          const int st = at % kStages;
          if (at >= kStages && !wait_pair(&s_free[st], (uint32_t)(at / kStages - 1) & 1u)) {
            ok = false;
            break;
          }
          const uint32_t bar = first_bar(&s_full[st]), to = ring + (uint32_t)st * kStage;
          if (rank == 0)
            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;"
                         ::"r"(smem_u32(&s_full[st])), "r"(2 * kStage) : "memory");
          copy_chunk(to, &p.images, w + c, bar);
          copy_chunk(to + kChunk, &p.images, x + c, bar);
        }
      }
      // The arrivals of the MMAs that read the last copies come before the CTA leaves: they are issued by the first
      // CTA, whose own have come when the second's may still be on their way. (A wait that ran out has given the
      // copies in flight its 2 s.)
      for (int q = max(0, at - kStages); q < at && ok; ++q)
        ok = wait_pair(&s_free[q % kStages], (uint32_t)(q / kStages) & 1u);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (elect_one()) {
      bool ok = true;
      int u = 0, d = 0;                         // chunks consumed, sums begun (or passed on)
      for (int i = first; i < tiles && ok; i += step) {
        if (rank != 0) {
          for (int m = 0; m < nsum && ok; ++m, ++d) {
            ok = mbar_wait(&s_taken[d & 1], (uint32_t)(d >> 1) & 1u);
            tc_fence_after();
            tc_fence_before();
            if (ok) arrive_first(&s_taken[d & 1]);
          }
          continue;
        }
        for (int c = 0; c < nch && ok; ++c, ++u) {
          const int st = u % kStages, in = c % kPer;
          if (in == 0 && d >= 2) ok = wait_pair(&s_taken[d & 1], (uint32_t)(d / 2 - 1) & 1u);
          ok = ok && wait_pair(&s_full[st], (uint32_t)(u / kStages) & 1u);
          if (!ok) break;
          tc_fence_after();
          const uint32_t w = ring + (uint32_t)st * kStage, x = w + kChunk;
#pragma unroll
          for (uint32_t k = 0; k < kSubK / 16; ++k)
            mma_pair(tmem + (uint32_t)(d & 1) * kT, umma_desc(w + k * 2u * kM * 16u, kM * 16, 128),
                     umma_desc(x + k * 2u * kTB * 16u, kTB * 16, 128), in == 0 && k == 0 ? 0u : 1u);
          commit_pair(&s_free[st]);
          if (in == kPer - 1 || c == nch - 1) {
            commit_pair(&s_sum[d & 1]);
            ++d;
          }
        }
      }
      // every MMA's arrival comes before the CTA leaves
      for (int q = max(0, u - kStages); q < u && ok; ++q)
        ok = wait_pair(&s_free[q % kStages], (uint32_t)(q / kStages) & 1u);
    }
    __syncwarp();
  } else if (warp >= kFirstSum) {
    const int part = (warp - kFirstSum) >> 2;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    bool ok = true;
    int d = 0;
    for (int i = first; i < tiles; i += step) {
      int n0;
      int64_t r0;
      tile_at(p, i, &n0, &r0);
      const int n = n0 + rank * kM + (warp & 3) * 32 + lane;
      r0 += part * kPart;
      const int nt = (int)max((int64_t)0, min((int64_t)kPart, a.rows - r0));
      float* const xs = s_scale[warp - kFirstSum];
      __syncwarp();
#pragma unroll
      for (int q = 0; q < kPart; q += 32)
        if (q + lane < nt) xs[q + lane] = __ldg(a.x_scale + r0 + q + lane);
      __syncwarp();
      uint32_t from = 0u;
      if (nsum == 1) {
        ok = ok && warp_all(wait_pair(&s_sum[d & 1], (uint32_t)(d >> 1) & 1u));
        tc_fence_after();
        from = tmem + lanes + (uint32_t)(d & 1) * kT + (uint32_t)(part * kPart);
        ++d;
      } else {
        int acc[kPart];
#pragma unroll
        for (int q = 0; q < kPart; ++q) acc[q] = 0;
        for (int m = 0; m < nsum; ++m, ++d) {
          ok = ok && warp_all(wait_pair(&s_sum[d & 1], (uint32_t)(d >> 1) & 1u));
          if (!ok) break;
          tc_fence_after();
          from = tmem + lanes + (uint32_t)(d & 1) * kT + (uint32_t)(part * kPart);
#pragma unroll
          for (int q = 0; q < kPart; q += 16) {
            float v[16];
            tmem_ld16(from + (uint32_t)q, v);
#pragma unroll
            for (int k = 0; k < 16; ++k) acc[q + k] += __float2int_rn(v[k]);
          }
          if (m + 1 < nsum) {
            tc_fence_before();
            warp_arrive(&s_taken[d & 1]);
          }
        }
        if (ok) {
#pragma unroll
          for (int q = 0; q < kPart; q += 16) {
            float v[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) v[k] = __int2float_rn(acc[q + k]);
            tmem_st16(from + (uint32_t)q, v);
          }
          asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        }
      }
      const bool live = n < a.n_out;
      const float ws = live ? __ldg(a.w_scale + n) : 0.0f, b = live && a.bias ? __ldg(a.bias + n) : 0.0f;
      elem_t<DT>* y = static_cast<elem_t<DT>*>(a.y) + r0 * a.ldy + n;
#pragma unroll 1
      for (int q = 0; q < nt; q += 16) {
        float v[16];
        if (ok) {
          tmem_ld16(from + (uint32_t)q, v);
          code_fields(v, reinterpret_cast<const float4*>(xs + q), ws, b, a.bias != nullptr);
          act_block(v, a.act, a.act_param);
        } else {
#pragma unroll
          for (int k = 0; k < 16; ++k) v[k] = NAN;
        }
        if (live) {
          if (q + 16 <= nt) {
#pragma unroll
            for (int k = 0; k < 16; ++k, y += a.ldy) *y = elem_of<DT>(v[k]);
          } else {
#pragma unroll
            for (int k = 0; k < 16; ++k, y += a.ldy)
              if (q + k < nt) *y = elem_of<DT>(v[k]);
          }
        }
        __syncwarp();
      }
      if (ok) {
        tc_fence_before();
        warp_arrive(&s_taken[(d - 1) & 1]);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  if (warp == 0)
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

template <int DT>
cudaError_t launch_pair(const PairArgs& p, int pairs, cudaStream_t s) {
  const cudaError_t e = cudaFuncSetAttribute(
      code_linear_pair_kernel<DT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kPairSmem);
  if (e != cudaSuccess) return e;
  code_linear_pair_kernel<DT><<<2 * pairs, kPairThreads, kPairSmem, s>>>(p);
  return cudaGetLastError();
}

int64_t tiles_of(int64_t rows) { return (rows + kT - 1) / kT; }

size_t image_bytes(int64_t rows, int n_in) {
  return (size_t)tiles_of(rows) * 2 * (size_t)((n_in + kSubK - 1) / kSubK) * kChunk;
}

// The images' n chunks as the tensor copies see them; the driver's function by its name, which needs no library to
// link.
cudaError_t images_map(CUtensorMap* map, void* img, size_t n) {
  using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                              const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                              CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  void* f = nullptr;
  cudaDriverEntryPointQueryResult found;
  const cudaError_t e =
      cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found);
  if (e != cudaSuccess) return e;
  if (found != cudaDriverEntryPointSuccess) return cudaErrorNotSupported;
  const cuuint64_t dim[2] = {kBoxWords, n * kBoxRows}, stride[1] = {4 * kBoxWords};
  const cuuint32_t box[2] = {kBoxWords, kBoxRows}, every[2] = {1, 1};
  const CUresult r = reinterpret_cast<Encode>(f)(
      map, CU_TENSOR_MAP_DATA_TYPE_INT32, 2, img, dim, stride, box, every, CU_TENSOR_MAP_INTERLEAVE_NONE,
      CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

}  // namespace

size_t code_linear_pair_workspace(const mca_code_linear_args& a) {
  return image_bytes(a.n_out, a.n_in) + image_bytes(a.rows, a.n_in);
}

cudaError_t launch_code_linear_pair(const mca_code_linear_args& a, cudaStream_t s) {
  PairArgs p{};
  p.a = a;
  p.chunks = (a.n_in + kSubK - 1) / kSubK;
  p.nt_out = (int)tiles_of(a.n_out);
  p.nt_rows = (int)tiles_of(a.rows);
  p.group = (int)std::min<size_t>(p.nt_out, std::max<size_t>(kGroup, kGroupBytes / (2 * (size_t)p.chunks * kChunk)));
  unsigned char* ws = static_cast<unsigned char*>(a.workspace);
  unsigned char* xs = ws + image_bytes(a.n_out, a.n_in);
  p.ximg = (int)(image_bytes(a.n_out, a.n_in) / kChunk);
  cudaError_t e = images_map(&p.images, ws, code_linear_pair_workspace(a) / kChunk);
  if (e != cudaSuccess) return e;
  const ImageArgs w{a.w, a.n_out, a.ldw, ws, code_rows_aligned(a.w, a.n_out, a.ldw)};
  const ImageArgs x{a.x, a.rows, a.ldx, xs, code_rows_aligned(a.x, a.rows, a.ldx)};
  const int64_t wb = (a.n_out + kM - 1) / kM, xb = (a.rows + kM - 1) / kM;
  code_image_kernel<<<(unsigned int)((wb + xb) * p.chunks), kM, 0, s>>>(w, x, wb, a.n_in, p.chunks);
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  const int pairs = (int)std::min<int64_t>(76, (int64_t)p.nt_out * p.nt_rows);
  switch (a.dtype) {
    case MCA_DTYPE_FP32: return launch_pair<MCA_DTYPE_FP32>(p, pairs, s);
    case MCA_DTYPE_FP16: return launch_pair<MCA_DTYPE_FP16>(p, pairs, s);
    default: return launch_pair<MCA_DTYPE_BF16>(p, pairs, s);
  }
}

}  // namespace mca
