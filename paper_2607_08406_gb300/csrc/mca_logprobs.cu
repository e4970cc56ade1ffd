// Log probabilities of given symbols, entropy and alternatives (mca_token_logprobs) and their gradient.
//
// With m the largest logit of a row, d = x - m and e = exp(d), one pass gives s = sum e and u = sum e d; then lse = m
// + ln s and the entropy ln s - u / s. When a larger m comes along, with c the change of m, s becomes f s and u becomes
// f (u + s c), f = exp(c). (m may lag behind by up to kLead, which see.) Differences are taken before anything
// is scaled, so that a common shift of a row loses nothing. Both kernels read every logit once; the gradient is a
// product per logit. The least they take is the memory's time, 30 us for 2048 x 50001 bf16 (0.2 GB at 6.8 TB/s).
// Measured there: 45 us without alternatives, 53 with 8, and the gradient 67 of 60: some 115 instructions for 8 logits
// (160 of the gradient) keep the schedulers 65 to 80 % busy, and rows end unevenly.
//
// Alternatives without a second pass: a thread keeps the largest logit of each of up to 8 groups of its 16-byte pieces.
// The k-th largest of a row's groups is a bound that the k-th alternative cannot be below; few more than k groups reach
// it (no more, with one warp and no equal logits), and only these are read again (from L2). What is found there is few
// enough to be put in order by counting. (Sorting the threads' largest and merging lists over the CTA took 9 us of a
// row's 25.)
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
    const int y = a.targets[p.pitch == 0 ? r : r / p.period * p.pitch + r % p.period];
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
// Up to which the rounds of the small kernel find several alternatives faster, and rows below which its latency counts:
// 20000 x 1000 bf16 with 8 takes 74 us in rounds and 38 otherwise, 20000 x 200 with 5 17 and 25, 100 x 500 4 and 6.
constexpr int kRoundVocab = 256;
constexpr int kRoundRows = 2048;

// The largest of a value over the L lanes of a row.
template <int L>
__device__ __forceinline__ unsigned int lanes_max(unsigned int v) {
  if constexpr (L == 32) {
    return __reduce_max_sync(0xffffffffu, v);
  } else {
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
  }
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
  unsigned int u[N];                                    // the keys' upper halves; 0: none, or taken
#pragma unroll
  for (int i = 0; i < N; ++i) u[i] = (unsigned int)(order_key(z[i], 0) >> 32);
  for (int k = 0; k < a.top; ++k) {                     // the next in order, one round each
    unsigned int best = 0u, at = 0u;                    // and the complement of its index
#pragma unroll
    for (int i = 0; i < N; ++i) best = max(best, u[i]);
    best = lanes_max<L>(best);
#pragma unroll
    for (int i = N - 1; i >= 0; --i)
      if (u[i] == best) at = ~(unsigned int)(t + L * i);
    at = lanes_max<L>(at);
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (~at == (unsigned int)(t + L * i)) u[i] = 0u;
    if (live && t == 0) write_top(a, r, k, best ? (Key)best << 32 | at : 0ull, w);
  }
}

// ------------------------------------------------------------------------------------------------
// Large vocabularies: a CTA per row, or the CTAs of a cluster.
// ------------------------------------------------------------------------------------------------
constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kAhead = 4;                 // pieces that a thread has on their way (took 51 us; 6: 53, 8: 54)
constexpr int kGroups = 8;                // groups of a thread's pieces
constexpr int kTeamVocab = 2048;          // a warp per row up to this vocabulary

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
  __device__ __forceinline__ bool whole(int j) const {
    return j * N >= head && (int64_t)(j + 1) * N <= (int64_t)V + head;
  }
  __device__ __forceinline__ const uint4* pieces() const { return reinterpret_cast<const uint4*>(x - head); }
  __device__ __forceinline__ uint4 raw(int j) const { return pieces()[j]; }
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
  __device__ __forceinline__ uint4 bits(int j) const {
    return whole(j) ? raw(j) : part(x, V, index(j, 0));
  }
  __device__ __noinline__ static uint4 part(const elem_t<DT>* x, int V, int at) {
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

// A row's pass without special cases: what lies below `low` counts as low (-inf too), whose terms vanish beside a
// largest logit above `high`. Rows without one go through exact_row instead; alternatives that are not above low
// come from rest_of_top.
template <int DT>
struct Range {
  static constexpr float low = DT == MCA_DTYPE_FP16 ? -65504.0f : -0x1p100f;
  static constexpr float high = DT == MCA_DTYPE_FP16 ? -65000.0f : -0x1p99f;
};

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// A piece's logits, at least low (NaN stays), in pairs, and the largest (NaN left out).
template <int DT>
__device__ __forceinline__ float clamp_piece(const uint4& q, float2 (&v)[Pieces<DT>::N / 2]) {
  unsigned int w[4] = {q.x, q.y, q.z, q.w};
  if constexpr (DT == MCA_DTYPE_FP32) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      v[i] = make_float2(max_nan(__uint_as_float(w[2 * i]), Range<DT>::low),
                         max_nan(__uint_as_float(w[2 * i + 1]), Range<DT>::low));
    return fmaxf(fmaxf(v[0].x, v[0].y), fmaxf(v[1].x, v[1].y));
  } else if constexpr (DT == MCA_DTYPE_BF16) {
    unsigned int m;
#pragma unroll
    for (int i = 0; i < 4; ++i) {                               // bf16 -2^100 is 0xf180
      asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(w[i]) : "r"(w[i]), "r"(0xf180f180u));
      v[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    }
    asm("{\n\t.reg .b32 a, b;\n\tmax.bf16x2 a, %1, %2;\n\tmax.bf16x2 b, %3, %4;\n\tmax.bf16x2 %0, a, b;\n\t}"
        : "=r"(m) : "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]));
    return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
  } else {
    unsigned int m;
#pragma unroll
    for (int i = 0; i < 4; ++i) {                               // fp16 -65504 is 0xfbff
      asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(w[i]) : "r"(w[i]), "r"(0xfbfffbffu));
      v[i] = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    }
    asm("{\n\t.reg .b32 a, b;\n\tmax.f16x2 a, %1, %2;\n\tmax.f16x2 b, %3, %4;\n\tmax.f16x2 %0, a, b;\n\t}"
        : "=r"(m) : "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]));
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&m));
    return fmaxf(f.x, f.y);
  }
}

// What a thread has seen. The sums refer to m, which follows the largest logit only when that is more than kLead above
// it: most pieces take no rescaling, and a row that rises slowly takes one for each kLead, not for each piece (every
// one is off by some half steps, 2^-24: by steps of 0.01, the entropy by 76 without a lead and 4 with one). The price
// is that u holds terms of either sign, up to kLead e^kLead, before the last shift, which takes their roundings
// along: with 1 those are some half steps of s more, with 8 the entropy of 80011 logits of which all but some were
// equal was off by 1900. 2048 x 50001 bf16 without alternatives takes 45.0, 44.4 and 43.5 us with 0, 1 and 8.
constexpr float kLead = 1.0f;

//
// The terms of a group of pieces have sums of their own, which go to those of the groups before at its end: a thread's
// chain of additions is a group's, an eighth, and with it what their roundings add up to in rows of few values.
template <int DT>
struct Seen {
  float m = Range<DT>::low, top = Range<DT>::low;
  float2 s = {0.0f, 0.0f}, u = {0.0f, 0.0f};
  Sums all = {Range<DT>::low, 0.0f, 0.0f};  // of the groups before
  __device__ __forceinline__ void raise(float to) {
    const float c = m - to, f = ex2_ftz(c * kLog2e);
    u.x = f > 0.0f ? f * fmaf(s.x, c, u.x) : 0.0f;
    u.y = f > 0.0f ? f * fmaf(s.y, c, u.y) : 0.0f;
    s.x *= f;
    s.y *= f;
    m = to;
  }
  __device__ __forceinline__ float take(const uint4& q) {
    float2 v[Pieces<DT>::N / 2];
    const float b = clamp_piece<DT>(q, v);
    if (b > top) {
      top = b;
      if (b > m + kLead) raise(b);
    }
    const float2 mm = make_float2(-m, -m), l2 = make_float2(kLog2e, kLog2e);
#pragma unroll
    for (int i = 0; i < Pieces<DT>::N / 2; ++i) {
      const float2 d = add2(v[i], mm), p = mul2(d, l2), e = make_float2(ex2_ftz(p.x), ex2_ftz(p.y));
      s = add2(s, e);
      u = fma2(e, d, u);
    }
    return b;
  }
  // The end of a group.
  __device__ __forceinline__ void close() {
    all.raise(m);
    all.s += s.x + s.y;
    all.u += u.x + u.y;
    s = u = make_float2(0.0f, 0.0f);
  }
  // The sums relative to the largest logit.
  __device__ __forceinline__ Sums sums() {
    all.raise(fmaxf(top, all.m));
    return all;
  }
};

// A CTA of W warps has a row (or, of kWarps, a part of one).
template <int W>
__device__ __forceinline__ void team_sync() {
  __syncwarp();
  if constexpr (W > 1) __syncthreads();
}

template <int W>
struct Team {
  static constexpr int kCand = 64 * W;
  static_assert(kCand >= W * 32, "the lists of ordered_top");
  Sums sum[W];
  unsigned int bound[W];
  int n, flagged;                           // candidates; groups whose largest logit reaches the bound
  unsigned short flag[kGroups * 32 * W];    // their threads and numbers
  float top[kGroups][32 * W];               // largest logits of the threads' groups
  Key cand[kCand];
};

template <int W>
__device__ __forceinline__ Sums team_sums(Sums t, Team<W>& s) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    t.join(__shfl_xor_sync(0xffffffffu, t.m, o), __shfl_xor_sync(0xffffffffu, t.s, o),
           __shfl_xor_sync(0xffffffffu, t.u, o));
  if constexpr (W > 1) {
    const int lane = threadIdx.x & 31;
    if (lane == 0) s.sum[threadIdx.x >> 5] = t;
    team_sync<W>();
    t = s.sum[lane % W];
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1)
      t.join(__shfl_xor_sync(0xffffffffu, t.m, o), __shfl_xor_sync(0xffffffffu, t.s, o),
             __shfl_xor_sync(0xffffffffu, t.u, o));
  }
  // the same number in every thread: join rounds by the side that it is called from
  t.m = __shfl_sync(0xffffffffu, t.m, 0);
  t.s = __shfl_sync(0xffffffffu, t.s, 0);
  t.u = __shfl_sync(0xffffffffu, t.u, 0);
  return t;
}

// The candidates: the logits that reach the bound, which lie in the groups whose largest does. Their pieces are read
// again by the whole CTA, all at once. A thread's group g holds its pieces g size .. of the order that it took them
// in.
template <int DT, int W>
__device__ __forceinline__ void find_candidates(const Pieces<DT>& row, int j0, int j1, int size, float top, Key bound,
                                                Team<W>& s) {
  constexpr int N = Pieces<DT>::N, kTeam = 32 * W;
  const int tid = threadIdx.x;
  // (logits at or below the range's low: exact_row, if the row has no others)
  const float low = fmaxf(Range<DT>::low, bound ? key_value(bound) : -INFINITY);
  if (top >= low && top > Range<DT>::low) {
    for (int g = 0; j0 + g * size * kTeam + tid < j1; ++g)
      if (s.top[g][tid] >= low) s.flag[atomicAdd(&s.flagged, 1)] = (unsigned short)(g * kTeam + tid);
  }
  __syncwarp();
  team_sync<W>();
  const int items = s.flagged * size;
  for (int i = tid; i < items; i += kTeam) {
    const int f = s.flag[i / size];
    const int j = j0 + (f / kTeam * size + i % size) * kTeam + f % kTeam;
    if (j >= j1) continue;
    float v[N];
    row.load(j, v);
    float m = v[0];
#pragma unroll
    for (int k = 1; k < N; ++k) m = fmaxf(m, v[k]);
    if (!(m >= low && m > Range<DT>::low)) continue;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      if (v[k] < low || !(v[k] > Range<DT>::low)) continue;
      const Key c = order_key(v[k], row.index(j, k));
      if (c < bound) continue;
      const int slot = atomicAdd(&s.n, 1);
      if (slot < Team<W>::kCand) s.cand[slot] = c;
    }
  }
}

__device__ __forceinline__ Key exchange(Key k, int j, bool larger) {
  const Key q = __shfl_xor_sync(0xffffffffu, k, j);
  return (q > k) == larger ? q : k;
}

// Lists of the n <= 32 largest keys, a key per lane in falling order: q of every lane into it. What lies behind the
// n-th is one of the keys, and not looked at.
__device__ __forceinline__ void keep_largest(Key& mine, Key q, int n) {
  const int lane = threadIdx.x & 31;
  unsigned int found = __ballot_sync(0xffffffffu, q > __shfl_sync(0xffffffffu, mine, n - 1));
  while (found) {
    const int from = __ffs(found) - 1;
    const Key f = __shfl_sync(0xffffffffu, q, from);
    const Key above = __shfl_up_sync(0xffffffffu, mine, 1);
    if (mine < f) mine = lane == 0 || above > f ? f : above;
    found &= ~(1u << from);
    found &= __ballot_sync(0xffffffffu, q > __shfl_sync(0xffffffffu, mine, n - 1));
  }
}

// The warps' lists into one at s.cand, of s.n keys.
template <int W>
__device__ __forceinline__ void merge_lists(Key mine, Team<W>& s) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __syncwarp();
  team_sync<W>();                            // the candidates' places are free
  s.cand[warp * 32 + lane] = mine;
  for (int n = W / 2; n > 0; n >>= 1) {
    team_sync<W>();
    if (warp < n) {
      const Key q = s.cand[(warp + n) * 32 + 31 - lane];
      mine = q > mine ? q : mine;
#pragma unroll
      for (int j = 16; j > 0; j >>= 1) mine = exchange(mine, j, (lane & j) == 0);
    }
    if (warp < n) s.cand[warp * 32 + lane] = mine;
  }
  const int have = __popc(__ballot_sync(0xffffffffu, mine != 0ull));
  if (warp == 0 && lane == 0) s.n = have;
  __syncwarp();
  team_sync<W>();
}

// The alternatives where the candidates are too many (logits in falling order, or many equal ones): each warp keeps the
// n largest in order, a list per warp at s.cand, which are then merged in pairs.
template <int DT, int W>
__device__ __noinline__ void ordered_top(const elem_t<DT>* x, int V, int j0, int j1, int n, float top, Key bound,
                                         Team<W>& s) {
  const Pieces<DT> row(x, V);
  constexpr int N = Pieces<DT>::N;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Key mine = 0ull;
  // the warp takes its threads' pieces one thread after the other, a piece per lane
  unsigned int todo = __ballot_sync(0xffffffffu, top > Range<DT>::low && order_key(top, 0) >= bound);
  while (todo) {
    const int owner = __ffs(todo) - 1;
    todo &= todo - 1;
    for (int b = j0 + warp * 32 + owner; b < j1; b += 32 * 32 * W) {
      const int j = b + lane * 32 * W;
      float v[N];
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = -INFINITY;
      if (j < j1) row.load(j, v);
      __syncwarp();
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const Key q = v[i] > Range<DT>::low ? order_key(v[i], row.index(j, i)) : 0ull;
        keep_largest(mine, q >= bound ? q : 0ull, n);
      }
    }
  }
  merge_lists<W>(mine, s);
}

// The largest n of a row's logits up to `limit`, in order, and how many they are at s.cand and s.n. A warp's pieces
// lie in the order of their index: of equal logits, as a mask leaves them, the first are kept and the others end at
// the vote. (2048 x 50001 bf16, 5 symbols left of 8 asked for: 104 us, where a pass for each alternative took 600.)
template <int DT, int W>
__device__ __noinline__ void rest_of_top(const elem_t<DT>* x, int V, float limit, int n, Team<W>& s) {
  const Pieces<DT> row(x, V);
  constexpr int N = Pieces<DT>::N, kStep = 32 * W, kBatch = 4;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Key mine = 0ull;
  for (int b = warp * 32; b < row.count; b += kBatch * kStep) {
    uint4 q[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      if (b + i * kStep + lane < row.count) q[i] = row.bits(b + i * kStep + lane);
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int j = b + i * kStep + lane;
      float v[N], m = -INFINITY;
      Pieces<DT>::values(q[i], v);
#pragma unroll
      for (int k = 0; k < N; ++k) {
        v[k] = j < row.count && v[k] <= limit ? v[k] : -INFINITY;
        m = fmaxf(m, v[k]);
      }
      __syncwarp();
      const Key last = __shfl_sync(0xffffffffu, mine, n - 1);
      if (!__any_sync(0xffffffffu, order_key(m, max(row.index(j, 0), 0)) > last)) continue;
#pragma unroll
      for (int k = 0; k < N; ++k) keep_largest(mine, order_key(v[k], row.index(j, k)), n);
    }
  }
  merge_lists<W>(mine, s);
}

// Any row, by the definition: passes for the largest logit, and, unless that says it all, for the sums and the
// alternatives.
template <int DT, int W>
__device__ __noinline__ void exact_row(const LogprobArgs& p, int64_t r, Team<W>& s) {
  const mca_token_logprobs_args& a = p.a;
  const Pieces<DT> row(static_cast<const elem_t<DT>*>(a.logits) + r * a.ld, a.vocab);
  constexpr int N = Pieces<DT>::N, kStep = 32 * W, kBatch = 4;
  float top = -INFINITY;                    // NaN if one is
  for (int b = threadIdx.x; b < row.count; b += kBatch * kStep) {
    uint4 q[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      if (b + i * kStep < row.count) q[i] = row.bits(b + i * kStep);
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      float v[N];
      Pieces<DT>::values(q[i], v);
      if (b + i * kStep < row.count) {
#pragma unroll
        for (int k = 0; k < N; ++k) top = max_nan(top, v[k]);
      }
    }
  }
  __syncwarp();
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
  team_sync<W>();
  // the row's largest, with a sum of 0 where all are -inf and NaN where one is NaN or +inf
  Sums t = team_sums<W>({fmaxf(top, kLowest), top < INFINITY ? (top > -INFINITY ? 1.0f : 0.0f) : NAN, 0.0f}, s);
  const bool any = t.s > 0.0f;
  if (any) {
    t.s = t.u = 0.0f;
#pragma unroll 2
    for (int j = threadIdx.x; j < row.count; j += kStep) {
      float v[N];
      row.load(j, v);
#pragma unroll
      for (int k = 0; k < N; ++k) t.add(v[k]);
    }
    __syncwarp();
    team_sync<W>();
    t = team_sums<W>(t, s);
  }
  if (threadIdx.x == 0) write_row<DT>(p, r, row.x, t);
  const Row w(t);
  if (a.top > 0 && any) rest_of_top<DT, W>(row.x, row.V, INFINITY, a.top, s);
  for (int k = threadIdx.x; k < a.top; k += kStep) write_top(a, r, k, any && k < s.n ? s.cand[k] : 0ull, w);
}

// Of n candidates the a.top largest, each at its place: put(place, key).
template <int W, class Put>
__device__ __forceinline__ void place_top(const Key* cand, int n, int top, Put put) {
  for (int i = threadIdx.x; i < n; i += 32 * W) {
    const Key k = cand[i];
    int above = 0;
#pragma unroll 4
    for (int q = 0; q < n; ++q) above += cand[q] > k;
    if (above < top) put(above, k);
  }
}

template <int DT, int W>
__global__ void __launch_bounds__(32 * W, 32 / W) logprobs_kernel(LogprobArgs p, int split) {
  using P = Pieces<DT>;
  constexpr int kTeam = 32 * W;
  __shared__ Team<W> s;
  __shared__ uint4 s_ring[kAhead][kTeam];
  constexpr bool kWhole = W == kWarps;                          // a row may have a cluster's CTAs
  __shared__ Sums s_part[kWhole ? kMaxCluster : 1];
  __shared__ Key s_best[kWhole ? kMaxCluster * 32 : 1];
  const mca_token_logprobs_args& a = p.a;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t r = kWhole ? (int64_t)blockIdx.x / split : (int64_t)blockIdx.x;
  const int rank = kWhole && split > 1 ? (int)cluster_rank() : 0;
  const P row(static_cast<const elem_t<DT>*>(a.logits) + r * a.ld, a.vocab);
  const int j0 = kWhole ? (int)((int64_t)row.count * rank / split) : 0;
  const int j1 = kWhole ? (int)((int64_t)row.count * (rank + 1) / split) : row.count;
  if (kWhole && split > 1) cluster_arrive();                     // every CTA runs before one writes to another
  if (tid == 0) s.n = s.flagged = 0;

  // the pass
  Seen<DT> seen;
  const int size = ((j1 - j0 + kTeam - 1) / kTeam + kGroups - 1) / kGroups;     // of a group
  {
    // kAhead pieces on their way to shared memory, each to its thread's own places: no registers, no barriers. A
    // piece at an end of the row that is not whole is put there by its thread.
    const unsigned int ring = (unsigned int)__cvta_generic_to_shared(&s_ring[0][tid]);
    constexpr unsigned int kSlot = kTeam * 16;
    const int w0 = row.whole(0) ? 0 : 1, whole = row.count - w0 - (row.whole(row.count - 1) ? 0 : 1);
    unsigned int slot = ring;
    int j = j0 + tid, next = j;
    const uint4* x = row.pieces() + j;                          // of piece `next`
    auto ask = [&] {
      if (next < j1) {
        if ((unsigned int)(next - w0) < (unsigned int)whole) {
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(slot), "l"(x) : "memory");
        } else {
          const uint4 q = P::part(row.x, row.V, row.index(next, 0));
          asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};"
                       ::"r"(slot), "r"(q.x), "r"(q.y), "r"(q.z), "r"(q.w) : "memory");
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
      next += kTeam;
      x += kTeam;
      slot = slot == ring + (kAhead - 1) * kSlot ? ring : slot + kSlot;
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) ask();
    float b = -INFINITY;                                        // the group's largest
    int left = size;
    float* group = &s.top[0][tid];
    for (; j < j1; j += kTeam) {
      uint4 q;
      asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
      asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "r"(slot) : "memory");
      b = fmaxf(b, seen.take(q));
      if (--left == 0) {
        *group = b;
        seen.close();
        group += kTeam;
        b = -INFINITY;
        left = size;
      }
      ask();
    }
    if (left < size) {
      *group = b;
      seen.close();
    }
  }
  __syncwarp();
  Sums t = team_sums<W>(seen.sums(), s);

  // the candidates: logits that reach the bound
  if (a.top > 0) {
    // a warp's k / W-th largest group, of equal ones all at once; k groups reach the smallest of the warps' (one
    // thread's largest in place of each group's let through 130 logits for 32 alternatives and one warp, and half the
    // row: 4096 x 32000 bf16 315 us, so 87; with 20 alternatives 86 and 76)
    unsigned int v[kGroups], reach = 0u;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const float b = j0 + g * size * kTeam + tid < j1 ? s.top[g][tid] : -INFINITY;
      v[g] = b > Range<DT>::low ? (unsigned int)(order_key(b, 0) >> 32) : 0u;
    }
    for (int have = 0; have < (a.top + W - 1) / W;) {
      unsigned int best = 0u, n = 0u;
#pragma unroll
      for (int g = 0; g < kGroups; ++g) best = max(best, v[g]);
      reach = best = lanes_max<32>(best);
      if (best == 0u) break;                                    // no more groups: every candidate reaches 0
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        n += v[g] == best;
        v[g] = v[g] == best ? 0u : v[g];
      }
      have += (int)__reduce_add_sync(0xffffffffu, n);
    }
    if constexpr (W > 1) {
      if (lane == 0) s.bound[warp] = reach;
      team_sync<W>();
      for (int q = 0; q < W; ++q) reach = min(reach, s.bound[q]);
    }
    const Key bound = (Key)reach << 32;
    __syncwarp();
    find_candidates<DT, W>(row, j0, j1, size, seen.top, bound, s);
    __syncwarp();
    team_sync<W>();
    if (s.n > Team<W>::kCand) ordered_top<DT, W>(row.x, row.V, j0, j1, a.top, seen.top, bound, s);
  }

  const Key* cand = s.cand;
  int n = a.top > 0 ? s.n : 0;
  if (kWhole && split > 1) {                                    // to the cluster's first CTA
    cluster_wait();
    if (tid < a.top && tid >= n)                                // no candidate for this place
      asm volatile("st.shared::cluster.u64 [%0], %1;"
                   ::"r"(first_cta(&s_best[rank * a.top + tid])), "l"(0ull) : "memory");
    place_top<W>(cand, n, a.top, [&](int at, Key k) {
      asm volatile("st.shared::cluster.u64 [%0], %1;"
                   ::"r"(first_cta(&s_best[rank * a.top + at])), "l"(k) : "memory");
    });
    if (tid == 0)
      asm volatile("st.shared::cluster.f32 [%0], %1;\n\tst.shared::cluster.f32 [%0 + 4], %2;\n\t"
                   "st.shared::cluster.f32 [%0 + 8], %3;"
                   ::"r"(first_cta(&s_part[rank])), "f"(t.m), "f"(t.s), "f"(t.u) : "memory");
    cluster_arrive();
    cluster_wait();
    if (rank != 0) return;
    t = s_part[0];
    for (int q = 1; q < split; ++q) t.join(s_part[q].m, s_part[q].s, s_part[q].u);
    cand = s_best;
    n = split * a.top;
  }
  const Row w(t);
  int found = n;
  if (kWhole && split > 1 && a.top > 0) {                        // empty places of the lists
    found = 0;
    for (int q = 0; q < n; q += 32)
      found += __popc(__ballot_sync(0xffffffffu, q + lane < n && s_best[q + lane] != 0ull));
  }
  if (t.m <= Range<DT>::high) {
    __syncwarp();
    team_sync<W>();
    exact_row<DT, W>(p, r, s);
    return;
  }
  if (tid == 0) write_row<DT>(p, r, row.x, t);
  if (w.bad) {
    if (tid < a.top) write_top(a, r, tid, 0ull, w);
    return;
  }
  place_top<W>(cand, n, a.top, [&](int at, Key k) {
    if (k != 0ull) write_top(a, r, at, k, w);
  });
  if (found < a.top) {                                            // all above low are placed: those below
    __syncwarp();
    team_sync<W>();
    rest_of_top<DT, W>(row.x, row.V, Range<DT>::low, a.top - found, s);
    for (int k = found + tid; k < a.top; k += kTeam) write_top(a, r, k, k - found < s.n ? s.cand[k - found] : 0ull, w);
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
  // The same for two logits, rows that are not none.
  __device__ __forceinline__ float2 of(float2 x) const {
    float2 lp = add2(x, make_float2(-lse, -lse));
    const float2 p = mul2(lp, make_float2(kLog2e, kLog2e));
    const float2 e = make_float2(-ex2_ftz(p.x), -ex2_ftz(p.y));
    lp = add2(make_float2(fmaxf(lp.x, kNoTerm), fmaxf(lp.y, kNoTerm)), make_float2(h, h));
    return mul2(e, fma2(make_float2(ge, ge), lp, make_float2(gl, gl)));
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

// kGradAhead pieces per thread of a row; logits and gradient lie at the same distance from 16-byte boundaries. (2048 x
// 50001 bf16: 66 us with two, 71 with four; the 32 bytes of one thread side by side took 83 when two took 69. Matrices
// that lie differently there go element by element: 208 us for bf16 logits padded to 50008 and a contiguous gradient.)
constexpr int kGradAhead = 2;

template <int DT>
__global__ void __launch_bounds__(kThreads) logprobs_backward_kernel(mca_token_logprobs_backward_args a,
                                                                     int parts) {
  using P = Pieces<DT>;
  const int64_t r = blockIdx.x / parts;
  const int j0 = (int)(blockIdx.x - r * parts) * kThreads * kGradAhead + threadIdx.x;
  const P row(static_cast<const elem_t<DT>*>(a.logits) + r * a.ld, a.vocab);
  elem_t<DT>* out = static_cast<elem_t<DT>*>(a.grad) + r * a.ldg;
  uint4 q[kGradAhead];
#pragma unroll
  for (int i = 0; i < kGradAhead; ++i)
    if (j0 + i * kThreads < row.count && row.whole(j0 + i * kThreads)) q[i] = row.raw(j0 + i * kThreads);
  const Grad g(a, r);
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
    for (int k = 0; k < P::N; k += 2) {
      const float2 d = g.of(make_float2(v[k], v[k + 1]));
      v[k] = g.none ? 0.0f : d.x;
      v[k + 1] = g.none ? 0.0f : d.y;
    }
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

template <int DT, int W>
cudaError_t launch_team(const LogprobArgs& p, cudaStream_t s) {
  logprobs_kernel<DT, W><<<(unsigned int)p.a.rows, 32 * W, 0, s>>>(p, 1);
  return cudaGetLastError();
}

template <int DT>
cudaError_t launch_logprobs_t(const LogprobArgs& p, cudaStream_t s) {
  const int V = p.a.vocab;
  if (V <= kRoundVocab || (V <= kSmallVocab && (p.a.top <= 1 || p.a.rows < kRoundRows))) {
    if (V <= 16) launch_small<DT, 4, 4>(p, s);
    else if (V <= 32) launch_small<DT, 8, 4>(p, s);
    else if (V <= 64) launch_small<DT, 16, 4>(p, s);
    else if (V <= 128) launch_small<DT, 32, 4>(p, s);
    else if (V <= 256) launch_small<DT, 32, 8>(p, s);
    else if (V <= 512) launch_small<DT, 32, 16>(p, s);
    else launch_small<DT, 32, 32>(p, s);
    return cudaGetLastError();
  }
  // Warps per row: as many as run at once, so that all rows do; one for short rows (a CTA's threads would have no piece
  // each). 2048 x 50001 bf16 with 8 alternatives took 51 us with two, 64 with eight in more than two waves.
  const int64_t warps = 32 * 152 / p.a.rows;
  if (V <= kTeamVocab || warps < 2) return launch_team<DT, 1>(p, s);
  if (warps < 4) return launch_team<DT, 2>(p, s);
  if (warps < 8) return launch_team<DT, 4>(p, s);
  // or CTAs of a cluster, while SMs have no row of their own and 2048 logits each at least
  int split = 1;
  while (split < kMaxCluster && p.a.rows * split * 2 <= 152 && V / (split * 2) >= 2048) split *= 2;
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
  return cudaLaunchKernelEx(&cfg, logprobs_kernel<DT, kWarps>, p, split);
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
