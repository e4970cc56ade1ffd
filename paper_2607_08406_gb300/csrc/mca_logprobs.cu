// Log probabilities of given symbols, entropy and alternatives (mca_token_logprobs) and their gradient.
//
// With m the largest logit of a row, d = x - m and e = exp(d), one pass gives s = sum e and u = sum e d; then lse = m
// + ln s and the entropy ln s - u / s (both sums have one sign, nothing cancels). When a larger m comes along,
// with c the change of m, s becomes f s and u becomes f (u + s c), f = exp(c). Differences are taken before anything
// is scaled, so that a common shift of a row loses nothing. Both kernels read every logit once; the gradient is a
// product per logit. What bounds them is the memory: 2048 x 50001 bf16, 0.2 GB, takes 30 us at 6.8 TB/s.
//
// Alternatives without a second pass: a thread remembers in which of its 16-byte pieces its largest logit was (one
// comparison a piece). The k-th largest of the threads' largest is a bound that the k-th alternative cannot be below,
// and just k threads reach it, so that only their pieces are read again (from L2).
#include <algorithm>

#include "mca_answers.h"
#include "mca_device.cuh"
#include "mca_elem.cuh"

namespace mca {

namespace {

using Key = unsigned long long;
constexpr float kLowest = -3.4028235e38f;
constexpr float kNoTerm = -200.0f;        // exp is 0 below -104

// Values in the order of their size, equal ones with the lower index first, as unsigned numbers; 0: none (-inf).
__device__ __forceinline__ Key order_key(float v, int i) {
  const unsigned int b = __float_as_uint(v + 0.0f);             // -0 is 0
  const unsigned int u = b & 0x80000000u ? ~b : b | 0x80000000u;
  return v > -INFINITY ? (Key)u << 32 | (unsigned int)~i : 0ull;
}
__device__ __forceinline__ float key_value(Key k) {
  const unsigned int u = (unsigned int)(k >> 32);
  return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ int key_index(Key k) { return (int)~(unsigned int)k; }

// The largest logit (finite) and the two sums of a part of a row.
struct Sums {
  float m, s, u;
  __device__ __forceinline__ void raise(float to) {              // to >= m, finite
    const float c = m - to, f = ex2_ftz(c * kLog2e);
    u = f > 0.0f ? f * fmaf(s, c, u) : 0.0f;                     // c may overflow where f is 0
    s *= f;
    m = to;
  }
  __device__ __forceinline__ void add(float x) {
    const float d = x - m, e = ex2_ftz(d * kLog2e);              // NaN of a NaN or +inf stays in s
    s += e;
    u = fmaf(e, fmaxf(d, kNoTerm), u);
  }
  __device__ __forceinline__ void join(float om, float os, float ou) {
    const float to = fmaxf(m, om);
    Sums o{om, os, ou};
    o.raise(to);
    raise(to);
    s += o.s;
    u += o.u;
  }
};

// What a row's sums say; one thread.
struct Row {
  float m, ls;
  bool bad, none;
  __device__ __forceinline__ explicit Row(const Sums& t)
      : m(t.m), ls(logf(t.s)), bad(!(t.s >= 0.0f)), none(t.s == 0.0f) {}
  __device__ __forceinline__ float logprob(float x) const { return (x - m) - ls; }
};

template <int DT>
__device__ __forceinline__ void write_row(const LogprobArgs& p, int64_t r, const elem_t<DT>* x, const Sums& t) {
  const mca_token_logprobs_args& a = p.a;
  const Row w(t);
  if (a.lse) a.lse[r] = w.bad ? NAN : w.none ? -INFINITY : w.m + w.ls;
  if (a.entropy) a.entropy[r] = w.bad ? NAN : w.none ? 0.0f : w.ls - t.u / t.s;
  if (a.logprob) {
    const int y = a.targets[r / p.period * p.pitch + r % p.period];
    float lp = 0.0f;
    if (y != -1)
      lp = y < 0 || y >= a.vocab || w.bad ? NAN : w.none ? -INFINITY : w.logprob(elem_f32(x[y]));
    a.logprob[r] = lp;
  }
}

__device__ __forceinline__ void write_top(const mca_token_logprobs_args& a, int64_t r, int k, Key key,
                                          const Row& w) {
  const bool has = key != 0ull && !w.bad;
  a.top_index[r * a.top + k] = has ? key_index(key) : -1;
  a.top_logprob[r * a.top + k] = w.bad ? NAN : has ? w.logprob(key_value(key)) : -INFINITY;
}

// ------------------------------------------------------------------------------------------------
// Small vocabularies: L lanes per row, N logits per lane (lane + L i), all in registers.
// ------------------------------------------------------------------------------------------------
constexpr int kSmallThreads = 128;
constexpr int kSmallVocab = 1024;

template <int L>
__device__ __forceinline__ Key group_max(Key k) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) {
    const Key q = __shfl_xor_sync(0xffffffffu, k, o);
    k = q > k ? q : k;
  }
  return k;
}
template <>
__device__ __forceinline__ Key group_max<32>(Key k) {
  const unsigned int hi = __reduce_max_sync(0xffffffffu, (unsigned int)(k >> 32));
  const unsigned int lo = __reduce_max_sync(0xffffffffu, (unsigned int)(k >> 32) == hi ? (unsigned int)k : 0u);
  return (Key)hi << 32 | lo;
}

template <int DT, int L, int N>
__global__ void __launch_bounds__(kSmallThreads) logprobs_small_kernel(LogprobArgs p) {
  const mca_token_logprobs_args& a = p.a;
  const int64_t row = (int64_t)blockIdx.x * (kSmallThreads / L) + threadIdx.x / L;
  const bool live = row < a.rows;                       // groups behind the last row take part in shuffles
  const int64_t r = live ? row : a.rows - 1;
  const int t = threadIdx.x % L, V = a.vocab;
  const elem_t<DT>* x = static_cast<const elem_t<DT>*>(a.logits) + r * a.ld;
  float z[N];
  float m = kLowest;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    z[i] = t + L * i < V ? elem_f32(x[t + L * i]) : -INFINITY;
    m = fmaxf(m, z[i]);
  }
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  Sums sum{m, 0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < N; ++i) sum.add(z[i]);
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) {
    sum.s += __shfl_xor_sync(0xffffffffu, sum.s, o);
    sum.u += __shfl_xor_sync(0xffffffffu, sum.u, o);
  }
  if (live && t == 0) write_row<DT>(p, r, x, sum);
  if (a.top == 0) return;
  const Row w(sum);
  Key last = ~0ull;
  for (int k = 0; k < a.top; ++k) {                     // the next in order, one round each
    Key best = 0ull;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const Key q = order_key(z[i], t + L * i);
      if (q < last && q > best) best = q;
    }
    best = group_max<L>(best);
    if (live && t == 0) write_top(a, r, k, best, w);
    last = best ? best : 1ull;
  }
}

// ------------------------------------------------------------------------------------------------
// Large vocabularies: a CTA per row, or the CTAs of a cluster.
// ------------------------------------------------------------------------------------------------
constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;

// A row's 16-byte pieces: piece j holds the logits j N - head .. of the row (the first and the last in part).
template <int DT>
struct Pieces {
  static constexpr int N = 16 / (int)sizeof(elem_t<DT>);
  const elem_t<DT>* x;
  int V, head, count;
  __device__ __forceinline__ Pieces(const elem_t<DT>* x_, int V_) : x(x_), V(V_) {
    head = (int)(reinterpret_cast<uintptr_t>(x) % 16 / sizeof(elem_t<DT>));
    count = (int)(((int64_t)V + head + N - 1) / N);
  }
  __device__ __forceinline__ int index(int j, int i) const { return j * N - head + i; }
  __device__ __forceinline__ bool whole(int j) const { return j * N >= head && (int64_t)(j + 1) * N <= (int64_t)V + head; }
  __device__ __forceinline__ uint4 raw(int j) const {
    return *reinterpret_cast<const uint4*>(x + (int64_t)j * N - head);
  }
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
  __device__ __forceinline__ void load(int j, float (&v)[N]) const {
    if (whole(j)) {
      values(raw(j), v);
      return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int64_t q = (int64_t)j * N - head + i;
      v[i] = q >= 0 && q < V ? elem_f32(x[q]) : -INFINITY;
    }
  }
};

__device__ __forceinline__ Key exchange(Key k, int j, bool larger) {
  const Key q = __shfl_xor_sync(0xffffffffu, k, j);
  return (q > k) == larger ? q : k;
}
// A warp's keys in falling order.
__device__ __forceinline__ Key warp_sort(Key k) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int n = 2; n <= 32; n <<= 1)
#pragma unroll
    for (int j = n >> 1; j > 0; j >>= 1) k = exchange(k, j, ((lane & j) == 0) == ((lane & n) == 0));
  return k;
}
// The 32 largest of two lists in falling order.
__device__ __forceinline__ Key warp_merge(Key k, Key reversed) {
  const int lane = threadIdx.x & 31;
  k = reversed > k ? reversed : k;
#pragma unroll
  for (int j = 16; j > 0; j >>= 1) k = exchange(k, j, (lane & j) == 0);
  return k;
}
// The 32 largest of n lists (a power of two, at most kWarps), into the first. The whole CTA.
__device__ __forceinline__ void merge_lists(Key (*list)[32], int n) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __syncthreads();
  for (n >>= 1; n > 0; n >>= 1) {
    if (warp < n) list[warp][lane] = warp_merge(list[warp][lane], list[warp + n][31 - lane]);
    __syncthreads();
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

template <int DT>
__global__ void __launch_bounds__(kThreads, 6) logprobs_kernel(LogprobArgs p, int split) {
  using P = Pieces<DT>;
  __shared__ Sums s_sum[kWarps];
  __shared__ Key s_list[kWarps][32];
  __shared__ Sums s_part[kMaxCluster];
  __shared__ Key s_best[kMaxCluster][32];
  const mca_token_logprobs_args& a = p.a;
  const int64_t r = blockIdx.x / split;
  const int rank = split > 1 ? (int)cluster_rank() : 0;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const P row(static_cast<const elem_t<DT>*>(a.logits) + r * a.ld, a.vocab);
  const int j0 = (int)((int64_t)row.count * rank / split), j1 = (int)((int64_t)row.count * (rank + 1) / split);

  if (split > 1) cluster_arrive();                              // every CTA runs before one writes to another

  // the pass: largest logit, where it was, sums
  Sums sum{kLowest, 0.0f, 0.0f};
  float top = -INFINITY;
  int at = -1;
  auto take = [&](const float (&v)[P::N], int j) {
    float b = v[0];
#pragma unroll
    for (int i = 1; i < P::N; ++i) b = fmaxf(b, v[i]);
    if (b > top) {
      top = b;
      at = j;
    }
    sum.raise(fmaxf(sum.m, b));
#pragma unroll
    for (int i = 0; i < P::N; ++i) sum.add(v[i]);
  };
  int j = j0 + tid;
  constexpr int kAhead = 4;
  for (; j + (kAhead - 1) * kThreads < j1; j += kAhead * kThreads) {
    float v[P::N];
    if (row.whole(j) && row.whole(j + (kAhead - 1) * kThreads)) {
      uint4 q[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) q[i] = row.raw(j + i * kThreads);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        P::values(q[i], v);
        take(v, j + i * kThreads);
      }
    } else {
#pragma unroll 1
      for (int i = 0; i < kAhead; ++i) {
        row.load(j + i * kThreads, v);
        take(v, j + i * kThreads);
      }
    }
  }
#pragma unroll 1
  for (; j < j1; j += kThreads) {
    float v[P::N];
    row.load(j, v);
    take(v, j);
  }

  // the CTA's sums
  Sums all = sum;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    all.join(__shfl_xor_sync(0xffffffffu, all.m, o), __shfl_xor_sync(0xffffffffu, all.s, o),
             __shfl_xor_sync(0xffffffffu, all.u, o));
  if (lane == 0) s_sum[warp] = all;

  // the CTA's alternatives
  if (a.top > 0) {
    Key key = 0ull;
    if (at >= 0) {
      float v[P::N];
      row.load(at, v);
#pragma unroll
      for (int i = P::N - 1; i >= 0; --i)
        if (v[i] == top) key = order_key(top, row.index(at, i));
    }
    if (a.top == 1) {
      const Key b = group_max<32>(key);
      s_list[warp][lane] = lane == 0 ? b : 0ull;
    } else {
      s_list[warp][lane] = warp_sort(key);
    }
    merge_lists(s_list, kWarps);
    if (a.top > 1) {
      const Key bound = s_list[0][a.top - 1];
      __syncthreads();
      Key mine = 0ull;                                          // the warp's list, in falling order
      unsigned int todo = __ballot_sync(0xffffffffu, key >= bound && key != 0ull);
      while (todo) {
        const int owner = __ffs(todo) - 1;
        todo &= todo - 1;
        for (int b = j0 + warp * 32 + owner; b < j1; b += 32 * kThreads) {
          const int jj = b + lane * kThreads;
          float v[P::N];
#pragma unroll
          for (int i = 0; i < P::N; ++i) v[i] = -INFINITY;
          if (jj < j1) row.load(jj, v);
#pragma unroll
          for (int i = 0; i < P::N; ++i) {
            const Key q = order_key(v[i], row.index(jj, i));
            unsigned int found = __ballot_sync(0xffffffffu, q != 0ull && q >= bound);
            while (found) {
              const Key f = __shfl_sync(0xffffffffu, q, __ffs(found) - 1);
              found &= found - 1;
              const Key above = __shfl_up_sync(0xffffffffu, mine, 1);
              if (mine < f) mine = lane == 0 || above > f ? f : above;
            }
          }
        }
      }
      s_list[warp][lane] = mine;
      merge_lists(s_list, kWarps);
    }
  }
  __syncthreads();

  if (split > 1) {                                              // to the cluster's first CTA
    cluster_wait();
    if (warp == 0) {
      if (a.top > 0)
        asm volatile("st.shared::cluster.u64 [%0], %1;"
                     ::"r"(first_cta(&s_best[rank][lane])), "l"(s_list[0][lane]) : "memory");
      if (lane == 0) {
        Sums t = s_sum[0];
        for (int q = 1; q < kWarps; ++q) t.join(s_sum[q].m, s_sum[q].s, s_sum[q].u);
        asm volatile("st.shared::cluster.f32 [%0], %1;\n\tst.shared::cluster.f32 [%0 + 4], %2;\n\t"
                     "st.shared::cluster.f32 [%0 + 8], %3;"
                     ::"r"(first_cta(&s_part[rank])), "f"(t.m), "f"(t.s), "f"(t.u) : "memory");
      }
    }
    cluster_arrive();
    cluster_wait();
    if (rank != 0) return;
    if (a.top > 0) {
      if (warp < split) s_list[warp][lane] = s_best[warp][lane];
      merge_lists(s_list, split);
    }
  }
  if (warp == 0) {
    const Sums* const part = split > 1 ? s_part : s_sum;
    Sums t = part[0];
    for (int q = 1; q < (split > 1 ? split : kWarps); ++q) t.join(part[q].m, part[q].s, part[q].u);
    if (lane == 0) write_row<DT>(p, r, row.x, t);
    if (lane < a.top) write_top(a, r, lane, s_list[0][lane], Row(t));
  }
}

// ------------------------------------------------------------------------------------------------
// Gradient: dx = [v = t] g - p (g + h (ln p + H)), p = exp(x - lse).
// ------------------------------------------------------------------------------------------------
struct Grad {
  float lse, gl, ge, h;
  int t;
  bool none;
  __device__ __forceinline__ Grad(const mca_token_logprobs_backward_args& a, int64_t r)
      : lse(a.lse[r]), gl(0.0f), ge(0.0f), h(0.0f), t(-1) {
    if (a.g_logprob) {
      t = a.targets[r];
      if (t != -1) gl = t < 0 || t >= a.vocab ? NAN : a.g_logprob[r];
    }
    if (a.g_entropy) {
      ge = a.g_entropy[r];
      h = a.entropy[r];
    }
    none = lse == -INFINITY;
  }
  __device__ __forceinline__ float of(float x) const {
    const float lp = x - lse, e = ex2_ftz(lp * kLog2e);
    return none ? 0.0f : -e * fmaf(ge, fmaxf(lp, kNoTerm) + h, gl);
  }
};

// L lanes per row.
template <int DT, int L>
__global__ void __launch_bounds__(kThreads) logprobs_backward_small_kernel(mca_token_logprobs_backward_args a) {
  const int64_t r = (int64_t)blockIdx.x * (kThreads / L) + threadIdx.x / L;
  if (r >= a.rows) return;
  const elem_t<DT>* x = static_cast<const elem_t<DT>*>(a.logits) + r * a.ld;
  elem_t<DT>* out = static_cast<elem_t<DT>*>(a.grad) + r * a.ldg;
  const Grad g(a, r);
#pragma unroll 4
  for (int v = threadIdx.x % L; v < a.vocab; v += L) {
    float d = g.of(elem_f32(x[v]));
    if (v == g.t && !g.none) d += g.gl;
    out[v] = elem_of<DT>(d);
  }
}

// kAhead pieces per thread of a row; logits and gradient lie at the same distance from 16-byte boundaries.
constexpr int kGradAhead = 4;

template <int DT>
__global__ void __launch_bounds__(kThreads) logprobs_backward_kernel(mca_token_logprobs_backward_args a,
                                                                     int parts) {
  using P = Pieces<DT>;
  const int64_t r = blockIdx.x / parts;
  const int j0 = (int)(blockIdx.x - r * parts) * kThreads * kGradAhead + threadIdx.x;
  const P row(static_cast<const elem_t<DT>*>(a.logits) + r * a.ld, a.vocab);
  elem_t<DT>* out = static_cast<elem_t<DT>*>(a.grad) + r * a.ldg;
  const Grad g(a, r);
  uint4 q[kGradAhead];
#pragma unroll
  for (int i = 0; i < kGradAhead; ++i)
    if (j0 + i * kThreads < row.count && row.whole(j0 + i * kThreads)) q[i] = row.raw(j0 + i * kThreads);
#pragma unroll
  for (int i = 0; i < kGradAhead; ++i) {
    const int j = j0 + i * kThreads;
    if (j >= row.count) break;
    const bool whole = row.whole(j);
    float v[P::N];
    if (whole)
      P::values(q[i], v);
    else
      row.load(j, v);
#pragma unroll
    for (int k = 0; k < P::N; ++k) v[k] = g.of(v[k]);
    const int at = g.t - row.index(j, 0);
    if (at >= 0 && at < P::N && !g.none) {
#pragma unroll
      for (int k = 0; k < P::N; ++k)
        if (k == at) v[k] += g.gl;
    }
    if (whole) {
      union {
        elem_t<DT> e[P::N];
        uint4 u;
      } o;
#pragma unroll
      for (int k = 0; k < P::N; ++k) o.e[k] = elem_of<DT>(v[k]);
      *reinterpret_cast<uint4*>(out + (int64_t)j * P::N - row.head) = o.u;
    } else {
#pragma unroll
      for (int k = 0; k < P::N; ++k) {
        const int64_t i2 = (int64_t)j * P::N - row.head + k;
        if (i2 >= 0 && i2 < a.vocab) out[i2] = elem_of<DT>(v[k]);
      }
    }
  }
}

template <int DT, int L, int N>
void launch_small(const LogprobArgs& p, cudaStream_t s) {
  constexpr int kPer = kSmallThreads / L;
  logprobs_small_kernel<DT, L, N><<<(unsigned int)((p.a.rows + kPer - 1) / kPer), kSmallThreads, 0, s>>>(p);
}

template <int DT>
cudaError_t launch_logprobs_t(const LogprobArgs& p, cudaStream_t s) {
  const int V = p.a.vocab;
  if (V <= kSmallVocab) {
    if (V <= 16) launch_small<DT, 4, 4>(p, s);
    else if (V <= 32) launch_small<DT, 8, 4>(p, s);
    else if (V <= 64) launch_small<DT, 16, 4>(p, s);
    else if (V <= 128) launch_small<DT, 32, 4>(p, s);
    else if (V <= 256) launch_small<DT, 32, 8>(p, s);
    else if (V <= 512) launch_small<DT, 32, 16>(p, s);
    else launch_small<DT, 32, 32>(p, s);
    return cudaGetLastError();
  }
  // CTAs per row: while four CTAs per SM have no row of their own, 2048 logits each at least
  int split = 1;
  while (split < kMaxCluster && p.a.rows * split * 2 <= 4 * 152 && V / (split * 2) >= 2048) split *= 2;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned int)(p.a.rows * split));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned int)split;
  at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, logprobs_kernel<DT>, p, split);
}

template <int DT, int L>
void launch_backward_small(const mca_token_logprobs_backward_args& a, cudaStream_t s) {
  constexpr int kPer = kThreads / L;
  logprobs_backward_small_kernel<DT, L><<<(unsigned int)((a.rows + kPer - 1) / kPer), kThreads, 0, s>>>(a);
}

template <int DT>
cudaError_t launch_backward_t(const mca_token_logprobs_backward_args& a, cudaStream_t s) {
  constexpr int es = (int)sizeof(elem_t<DT>), N = 16 / es;
  const int V = a.vocab;
  const bool together = (reinterpret_cast<uintptr_t>(a.logits) - reinterpret_cast<uintptr_t>(a.grad)) % 16 == 0 &&
                        (a.rows == 1 || (a.ld - a.ldg) % N == 0);
  if (V > kSmallVocab && together) {
    const int parts = (int)(((int64_t)V + 2 * N - 2) / N + kThreads * kGradAhead - 1) / (kThreads * kGradAhead);
    if (a.rows * parts <= 0x7fffffff) {
      logprobs_backward_kernel<DT><<<(unsigned int)(a.rows * parts), kThreads, 0, s>>>(a, parts);
      return cudaGetLastError();
    }
  }
  if (V <= 16) launch_backward_small<DT, 4>(a, s);
  else if (V <= 32) launch_backward_small<DT, 8>(a, s);
  else if (V <= 64) launch_backward_small<DT, 16>(a, s);
  else if (V <= kSmallVocab) launch_backward_small<DT, 32>(a, s);
  else launch_backward_small<DT, kThreads>(a, s);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_logprobs(const LogprobArgs& p, cudaStream_t s) {
  if (p.a.dtype == MCA_DTYPE_FP32) return launch_logprobs_t<MCA_DTYPE_FP32>(p, s);
  if (p.a.dtype == MCA_DTYPE_FP16) return launch_logprobs_t<MCA_DTYPE_FP16>(p, s);
  return launch_logprobs_t<MCA_DTYPE_BF16>(p, s);
}

cudaError_t launch_logprobs_backward(const mca_token_logprobs_backward_args& a, cudaStream_t s) {
  if (a.dtype == MCA_DTYPE_FP32) return launch_backward_t<MCA_DTYPE_FP32>(a, s);
  if (a.dtype == MCA_DTYPE_FP16) return launch_backward_t<MCA_DTYPE_FP16>(a, s);
  return launch_backward_t<MCA_DTYPE_BF16>(a, s);
}

}  // namespace mca
