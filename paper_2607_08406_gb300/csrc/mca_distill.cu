// The loss of rows of logits against a teacher's listed symbols (mca_distill) and its gradient.
//
// With c = log2(e) / temperature a term of a row's sum is 2^(x c - m), m a reference near the row's largest x c: one fused
// product and one exponential a logit. All that is added up at the end goes by the same m, so that neither its rounding
// nor that of c tells between the symbols. The list is read while the first pieces are on their way. Both kernels read
// every logit once and are bound by the memory.
#include <algorithm>
#include <climits>
#include <type_traits>

#include "mca_answers.h"
#include "mca_device.cuh"
#include "mca_elem.cuh"
#include "mca_row_shapes.h"
#include "mca_rows.cuh"

namespace mca {

namespace {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLeastRest = 0x1p-20f;    // of a teacher's probability: less is what rounded log probabilities leave
constexpr float kLeastLog = -1000.0f;     // a rest below has lost its digits: what is not listed is masked
constexpr float kFar = 0x1p100f;          // rows whose largest x c is as far go by the definition (any_row)
constexpr int kPerLane = kMaxList / 32;   // entries of a list that a lane has: lane, lane + 32, ..

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ float warp_max_nan(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = max_nan(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

__device__ __forceinline__ float list_value(const void* p, int dtype, int64_t i) {
  if (dtype == MCA_DTYPE_FP32) return static_cast<const float*>(p)[i];
  if (dtype == MCA_DTYPE_FP16) return __half2float(static_cast<const __half*>(p)[i]);
  return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
}

// A teacher's list in the registers of a warp: symbols (-1: none, or out of range), probabilities, their logarithms.
struct List {
  // f(q) for the places q of a lane that a list of `top` symbols has.
  template <class F>
  static __device__ __forceinline__ void each(int top, F f) {
    f(0);
    if (top <= 32) return;                // (most lists: one look at `top`)
#pragma unroll
    for (int q = 1; q < kPerLane; ++q)
      if (32 * q < top) f(q);
  }

  int symbol[kPerLane];
  float p[kPerLane], lp[kPerLane];
  float rest, total;                      // P, and the sum of all probabilities
  bool bad;

  // The list as it is, and what it says.
  template <class Args>
  __device__ __forceinline__ void load(const Args& a, int64_t r) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int q = 0; q < kPerLane; ++q) {
      symbol[q] = -1;
      lp[q] = -INFINITY;
    }
    each(a.top, [&](int q) {
      const int j = lane + 32 * q;
      if (j >= a.top) return;
      symbol[q] = a.index[r * a.ldi + j];
      lp[q] = list_value(a.teacher, a.teacher_dtype, r * a.ldt + j);
    });
  }
  template <class Args>
  __device__ __forceinline__ void resolve(const Args& a) {
    bool wrong = false;
    float m = -INFINITY, z = 0.0f;
    each(a.top, [&](int q) {
      if (symbol[q] == -1) lp[q] = -INFINITY;
      if (symbol[q] < -1 || symbol[q] >= a.vocab) {
        wrong = true;
        symbol[q] = -1;
      }
      wrong |= !(lp[q] < INFINITY);
      m = fmaxf(m, lp[q]);
    });
    bad = __any_sync(0xffffffffu, wrong);
    if (!a.tail) {
      m = warp_max(m);
      const float inv = 1.0f / a.temperature;
      each(a.top, [&](int q) { lp[q] = m > -INFINITY ? (lp[q] - m) * inv : -INFINITY; });
    }
#pragma unroll
    for (int q = 0; q < kPerLane; ++q) p[q] = 0.0f;
    each(a.top, [&](int q) {
      p[q] = expf(lp[q]);
      z += p[q];
    });
    z = warp_sum(z);
    rest = 0.0f;
    total = z;
    if (a.tail) {
      rest = 1.0f - z < kLeastRest ? 0.0f : 1.0f - z;
      total = z + rest;
    } else if (z > 0.0f) {
      const float lz = logf(z), rz = 1.0f / z;
      each(a.top, [&](int q) {
        p[q] *= rz;
        lp[q] -= lz;
      });
      total = 1.0f;
    }
  }
  template <class Args>
  __device__ __forceinline__ void read(const Args& a, int64_t r) {
    load(a, r);
    resolve(a);
  }

  // Entries of one symbol to its first one, in the list's order; the others become none. seen: kSeenWords for the warp, a
  // bitmap of the symbols, or of hashed ones, which says where lists of more than 32 need a look at the others (60000 x 300
  // bf16 against 128 symbols 53 us, 84 with every 32 compared; against 32 symbols 35, and 33 compared).
  static constexpr int kSeenWords = 256;
  __device__ __forceinline__ void merge(int top, int vocab, unsigned int* seen) {
    if (top <= 32) {
      merge_step(0, 0u);
      return;
    }
    const int lane = threadIdx.x & 31;
    const bool few = vocab <= 32 * kSeenWords;
    for (int i = lane; i < (few ? (vocab + 31) / 32 : kSeenWords); i += 32) seen[i] = 0u;
    __syncwarp();
    each(top, [&](int q) {
      const unsigned int at = few ? (unsigned int)symbol[q] : (unsigned int)symbol[q] * 2654435761u >> 19;
      const bool may = symbol[q] >= 0 && (atomicOr(&seen[at / 32], 1u << (at % 32)) >> (at % 32) & 1u);
      const unsigned int some = __ballot_sync(0xffffffffu, may);
      if (some) merge_step(q, some);
      __syncwarp();
    });
  }
  // Entries q of all lanes, with one another and with those before; some: lanes that may have met their symbol.
  __device__ __forceinline__ void merge_step(int q, unsigned int some) {
    const int lane = threadIdx.x & 31;
    const unsigned int same = __match_any_sync(0xffffffffu, symbol[q]);
    if (__any_sync(0xffffffffu, symbol[q] >= 0 && same != 1u << lane)) {
      float sum = 0.0f;
      for (int i = 0; i < 32; ++i) {
        const float other = __shfl_sync(0xffffffffu, p[q], i);
        if (same >> i & 1u) sum += other;
      }
      if (symbol[q] >= 0) {
        p[q] = sum;
        if ((same & ((1u << lane) - 1u)) != 0u) symbol[q] = -1;
      }
    }
    unsigned int may = __ballot_sync(0xffffffffu, q > 0 && symbol[q] >= 0 && (same & some) != 0u);
    while (may) {
      const int i = __ffs(may) - 1, other = __shfl_sync(0xffffffffu, symbol[q], i);
      const float po = __shfl_sync(0xffffffffu, p[q], i);
      may &= may - 1;
      bool met = false;
#pragma unroll
      for (int k = 0; k < kPerLane; ++k)
        if (k < q && symbol[k] == other) {
          p[k] += po;
          met = true;
        }
      if (__any_sync(0xffffffffu, met) && lane == i) symbol[q] = -1;
    }
  }

  // Whether a lane's entry q is the first one of its symbol among those of all lanes.
  __device__ __forceinline__ bool leads(int q) const {
    return __ffs(__match_any_sync(0xffffffffu, symbol[q])) - 1 == (int)(threadIdx.x & 31) && symbol[q] >= 0;
  }

  // Whether the teacher gives anything a probability.
  __device__ __forceinline__ bool any() const {
    bool some = rest > 0.0f;
#pragma unroll
    for (int q = 0; q < kPerLane; ++q) some |= p[q] > 0.0f;
    return __any_sync(0xffffffffu, some);
  }
};

// A part of a row's sum: s 2^m.
struct Part {
  float m, s;
  __device__ __forceinline__ void join(float om, float os) {
    const float to = fmaxf(m, om);
    s = s * ex2_ftz(m - to) + os * ex2_ftz(om - to);
    m = to;
  }
  __device__ __forceinline__ void join(const Part& o) { join(o.m, o.s); }
  __device__ __forceinline__ void join_lanes() {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
      join(__shfl_xor_sync(0xffffffffu, m, o), __shfl_xor_sync(0xffffffffu, s, o));
  }
};

// A row's results, by a warp. in, out: the sums of the listed symbols and of the others (all in `out` without tail); z[q]:
// x / T of the lane's listed symbols less what the larger of the sums' m stands for; gap: the same for out.m; base: the
// log-sum-exp of a sum of 1 with m = 0.
__device__ __forceinline__ void finish(const mca_distill_args& a, int64_t r, const List& t, const Part& out,
                                       const Part& in, const float (&z)[kPerLane], float gap, float base) {
  const float to = fmaxf(out.m, in.m);
  const float so = out.s * ex2_ftz(out.m - to), si = in.s * ex2_ftz(in.m - to), s = so + si, ls = logf(s);
  float loss = 0.0f;
  List::each(a.top, [&](int q) {
    if (t.symbol[q] >= 0 && t.p[q] > 0.0f) loss += t.p[q] * (t.lp[q] - (z[q] - ls));
  });
  loss = warp_sum(loss);
  if ((threadIdx.x & 31) != 0) return;
  if (a.rest || t.rest > 0.0f) {
    // of a sum that is nearly all, ln (1 - the other's share) keeps its digits
    const float rest = so >= 0.5f * s ? log1pf(-si / s)
                       : out.s > 0.0f ? (logf(out.s) - ls) + gap
                                      : -INFINITY;
    if (t.rest > 0.0f) loss += t.rest * (logf(t.rest) - rest);
    if (a.rest) a.rest[r] = rest;
  }
  a.loss[r] = t.bad ? NAN : loss;
  if (a.lse) a.lse[r] = base + (to * kLn2 + ls);
}

// The same of a row whose largest logit m (NaN if one is) is no finite number.
__device__ __forceinline__ void finish_without(const mca_distill_args& a, int64_t r, const List& t, float m) {
  const bool any = t.any();
  if ((threadIdx.x & 31) != 0) return;
  const float v = m == -INFINITY ? -INFINITY : NAN;
  a.loss[r] = v != v || t.bad ? NAN : any ? INFINITY : 0.0f;
  if (a.lse) a.lse[r] = v;
  if (a.rest) a.rest[r] = v;
}

// A piece with -inf in the places whose bits are set.
template <int DT>
__device__ __forceinline__ uint4 without(const uint4& q, unsigned int bits) {
  unsigned int w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (DT == MCA_DTYPE_FP32) {
      if (bits >> i & 1u) w[i] = 0xff800000u;
    } else {
      constexpr unsigned int kNone = DT == MCA_DTYPE_FP16 ? 0xfc00u : 0xff80u;
      if (bits >> (2 * i) & 1u) w[i] = (w[i] & 0xffff0000u) | kNone;
      if (bits >> (2 * i + 1) & 1u) w[i] = (w[i] & 0xffffu) | kNone << 16;
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// ------------------------------------------------------------------------------------------------
// Short rows: a warp for each, P pieces to a lane, all in registers. A row is bound by the instructions around its list
// (60000 x 300 bf16 against 32 symbols: 130 us with a warp and a ring of pieces for each, here 37, and 44 with tail).
// ------------------------------------------------------------------------------------------------
constexpr int kSmallThreads = 128;

template <int DT, int P>
__global__ void __launch_bounds__(kSmallThreads) distill_small_kernel(mca_distill_args a, float c) {
  constexpr int N = Pieces<DT>::N;
  __shared__ unsigned int s_listed[kSmallThreads / 32][P * N];         // bits, by places in the row's pieces
  const int64_t r = (int64_t)blockIdx.x * (kSmallThreads / 32) + threadIdx.x / 32;
  if (r >= a.rows) return;
  const int lane = threadIdx.x & 31;
  const Pieces<DT> row(static_cast<const elem_t<DT>*>(a.logits) + r * a.ld, a.vocab);
  unsigned int* listed = s_listed[threadIdx.x / 32];
  List t;
  t.load(a, r);
  uint4 q[P];
#pragma unroll
  for (int i = 0; i < P; ++i)
    if (lane + 32 * i < row.count) q[i] = row.bits(lane + 32 * i);
  t.resolve(a);
  float x[kPerLane];
  List::each(a.top, [&](int k) { x[k] = t.symbol[k] >= 0 ? elem_f32(row.x[t.symbol[k]]) : 0.0f; });
  if (a.tail) {                                         // -inf in the places of the listed symbols
    for (int i = lane; i < P * N; i += 32) listed[i] = 0u;
    __syncwarp();
  }
  float xs[kPerLane];                                   // of the first entry of each symbol
  if (a.tail) {
    List::each(a.top, [&](int k) {
      const int at = t.symbol[k] + row.head;
      bool first = t.symbol[k] >= 0 && !(atomicOr(&listed[at / 32], 1u << (at % 32)) >> (at % 32) & 1u);
      // (of entries that are the same it does not say which is first)
      if (__any_sync(0xffffffffu, first != (t.symbol[k] >= 0))) {
        const unsigned int same = __match_any_sync(0xffffffffu, t.symbol[k]);
        first = (__ballot_sync(0xffffffffu, first) & same) != 0u && __ffs(same) - 1 == lane;
      }
      xs[k] = first ? x[k] : -INFINITY;
      __syncwarp();
    });
#pragma unroll
    for (int i = 0; i < P; ++i) {
      if (lane + 32 * i >= row.count) break;
      const int at = (lane + 32 * i) * N;
      q[i] = without<DT>(q[i], listed[at / 32] >> (at % 32));
    }
  }
  float mo = -INFINITY, mi = -INFINITY;                 // the largest of the others, or of all without tail, and of these
#pragma unroll
  for (int i = 0; i < P; ++i)
    if (lane + 32 * i < row.count) mo = max_nan(mo, largest<DT>(q[i]));
  mo = warp_max_nan(mo);
  float m = mo;                                         // of all (NaN if one is)
  if (a.tail) {
    List::each(a.top, [&](int k) { mi = max_nan(mi, xs[k]); });
    m = max_nan(mo, warp_max_nan(mi));
  }
  if (!(m > -INFINITY && m < INFINITY)) {
    finish_without(a, r, t, m);
    return;
  }
  if (mo == -INFINITY) mo = m;
  float so = 0.0f, si = 0.0f;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    if (lane + 32 * i >= row.count) break;
    float v[N];
    Pieces<DT>::values(q[i], v);
#pragma unroll
    for (int e = 0; e < N; ++e) so += ex2_ftz((v[e] - mo) * c);
  }
  if (a.tail) {
    List::each(a.top, [&](int k) { si += ex2_ftz((xs[k] - m) * c); });
    si = warp_sum(si);
  }
  so = warp_sum(so);
  float z[kPerLane];
  List::each(a.top, [&](int k) { z[k] = (x[k] - m) / a.temperature; });
  finish(a, r, t, {so > 0.0f ? (mo - m) * c : 0.0f, so}, {0.0f, si}, z, (mo - m) / a.temperature, m / a.temperature);
}

// ------------------------------------------------------------------------------------------------
// Large vocabularies: four or eight warps per row, or the CTAs of a cluster.
// ------------------------------------------------------------------------------------------------
constexpr int kWarps = kTeamWarps;
constexpr int kAhead = 4;                 // pieces that a thread has on their way
constexpr float kLead = 10.0f;            // how far (in units of 2) a logit may be above the reference of the sum

// A piece's logits in pairs, and the largest (NaN left out).
template <int DT>
__device__ __forceinline__ float unpack_max(const uint4& q, float2 (&v)[Pieces<DT>::N / 2]) {
  const unsigned int w[4] = {q.x, q.y, q.z, q.w};
  if constexpr (DT == MCA_DTYPE_FP32) {
    v[0] = make_float2(__uint_as_float(w[0]), __uint_as_float(w[1]));
    v[1] = make_float2(__uint_as_float(w[2]), __uint_as_float(w[3]));
    return fmaxf(fmaxf(v[0].x, v[0].y), fmaxf(v[1].x, v[1].y));
  } else if constexpr (DT == MCA_DTYPE_BF16) {
    unsigned int m;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    asm("{\n\t.reg .b32 a, b;\n\tmax.bf16x2 a, %1, %2;\n\tmax.bf16x2 b, %3, %4;\n\tmax.bf16x2 %0, a, b;\n\t}"
        : "=r"(m) : "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]));
    return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
  } else {
    unsigned int m;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    asm("{\n\t.reg .b32 a, b;\n\tmax.f16x2 a, %1, %2;\n\tmax.f16x2 b, %3, %4;\n\tmax.f16x2 %0, a, b;\n\t}"
        : "=r"(m) : "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]));
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&m));
    return fmaxf(f.x, f.y);
  }
}

// The sum of a thread's pieces. The reference m follows the largest x c when that is more than kLead above it; a sum
// holds terms of up to 2^kLead, which costs no digits. Terms go to the sum of their group first, so that a chain of
// additions is short.
template <int DT>
struct Sum {
  float c, m, top;                        // top: the logit that m + kLead stands for; -inf until one is above that
  float2 s, all;
  __device__ __forceinline__ explicit Sum(float c_)
      : c(c_), m(-kFar), top(-INFINITY), s(make_float2(0.0f, 0.0f)), all(s) {}
  __device__ __forceinline__ bool any() const { return top > -INFINITY; }
  __device__ __forceinline__ void raise(float to) {
    const float up = fmaxf(to * c, -kFar), f = ex2_ftz(m - up);
    s.x *= f;
    s.y *= f;
    all.x *= f;
    all.y *= f;
    m = up;
    top = to + kLead / c;
  }
  template <int P>
  __device__ __forceinline__ void take(const float2 (&v)[P], float largest) {
    if (largest > top) raise(largest);
    const float2 cc = make_float2(c, c), mm = make_float2(-m, -m);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const float2 z = fma2(v[i], cc, mm);
      s = add2(s, make_float2(ex2_ftz(z.x), ex2_ftz(z.y)));
    }
  }
  __device__ __forceinline__ void close() {
    all = add2(all, s);
    s = make_float2(0.0f, 0.0f);
  }
  __device__ __forceinline__ Part part() {
    close();
    return {m, all.x + all.y};
  }
};

// The listed symbols of a team's part of a row, which take no part in the sum of the others: mask[w] says in which of (at
// most 32) groups of rounds warp w meets one.
template <int W>
struct Listed {
  alignas(16) int at[kMaxList];           // place in the row's pieces, -1: none
  bool met[kMaxList];                     // the first of its symbol's entries, met by the team
  unsigned int mask[W];
};

__device__ __forceinline__ int group_of(int pieces, int team) {
  return max(1, ((pieces + team - 1) / team + 31) / 32);
}

template <int DT, int W>
__device__ __forceinline__ void mark(const Pieces<DT>& row, int j0, int j1, const List& t, int top, Listed<W>& s) {
  constexpr int N = Pieces<DT>::N;
  const int lane = threadIdx.x & 31, group = group_of(j1 - j0, 32 * W);
  if (lane < W) s.mask[lane] = 0u;
  __syncwarp();
  List::each(top, [&](int q) {
    const int at = t.symbol[q] >= 0 ? t.symbol[q] + row.head : -1, j = at / N;
    s.at[lane + 32 * q] = at;
    s.met[lane + 32 * q] = false;
    if (at >= 0 && j >= j0 && j < j1)
      atomicOr(&s.mask[(j - j0) / 32 % W], 1u << ((j - j0) / (32 * W) / group));
  });
}

// A round in which a warp meets listed symbols, its lanes' pieces being base + lane, below `end`: which places of a lane's
// piece they have, as bits. Every lane of the warp.
template <int DT, int W>
__device__ __forceinline__ unsigned int met_in(int base, int end, int top, Listed<W>& s) {
  constexpr int N = Pieces<DT>::N;
  const int lane = threadIdx.x & 31;
  const unsigned int places = (unsigned int)(min(32, end - base) * N);
  unsigned int gone = 0u;
  for (int k = 0; k < top; k += 32) {
    const int mine = s.at[k + lane] - base * N;
    unsigned int here = __ballot_sync(0xffffffffu, (unsigned int)mine < places);
    while (here) {
      const int e = __ffs(here) - 1, at = __shfl_sync(0xffffffffu, mine, e);
      here &= here - 1;
      if (at / N == lane) {
        s.met[k + e] = !(gone >> at % N & 1u);
        gone |= 1u << at % N;
      }
    }
  }
  return gone;
}
// A warp's rounds, the first at `base`, one every TEAM pieces below `end`: one(base, places that listed symbols have), those
// of a group in which the warp meets some with a look at the list, all others without a question (4096 x 32000 fp16 against
// 20 symbols 60 us with one for each round, 54 so); close() every so often, where CLOSE.
template <int TEAM, bool CLOSE, class Met, class One, class Close>
__device__ __forceinline__ void in_groups(int base, int end, unsigned int mask, int group, Met met, One one,
                                          Close close) {
  const int start = base, step = max(group, 16) * TEAM;
  auto plain = [&](int to) {
    if (!CLOSE) {
      for (; base < to; base += TEAM) one(base, 0u);
      return;
    }
    while (base < to) {
      const int stop = min(to, base + step);
      for (; base < stop; base += TEAM) one(base, 0u);
      close();
    }
  };
  for (; mask; mask &= mask - 1) {
    const int from = start + (__ffs(mask) - 1) * group * TEAM, to = min(end, from + group * TEAM);
    plain(from);
    for (; base < to; base += TEAM) one(base, met(base));
    close();
  }
  plain(end);
}

// Any row by the definition, by the first warp of its team.
template <int DT>
__device__ __noinline__ void any_row(mca_distill_args a, int64_t r, float c) {
  const int lane = threadIdx.x & 31, V = a.vocab;
  List t;
  t.read(a, r);
  const elem_t<DT>* x = static_cast<const elem_t<DT>*>(a.logits) + r * a.ld;
  float m = -INFINITY, z[kPerLane];
  for (int64_t v = lane; v < V; v += 32) m = max_nan(m, elem_f32(x[v]));
  m = warp_max_nan(m);
  if (!(m > -INFINITY && m < INFINITY)) {
    finish_without(a, r, t, m);
    return;
  }
#pragma unroll
  for (int q = 0; q < kPerLane; ++q) z[q] = t.symbol[q] >= 0 ? (elem_f32(x[t.symbol[q]]) - m) / a.temperature : 0.0f;
  // f(logit, whether it is listed), 32 symbols at a time, four times as many on their way
  auto every = [&](auto f) {
    for (int64_t v = 0; v < V; v += 128) {
      float now[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) now[k] = v + 32 * k + lane < V ? elem_f32(x[v + 32 * k + lane]) : -INFINITY;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        unsigned int in = 0u;
        if (a.tail) {
          List::each(a.top, [&](int q) {
            unsigned int here = __ballot_sync(0xffffffffu, t.symbol[q] >= 0 && t.symbol[q] / 32 == (int)(v / 32) + k);
            for (; here; here &= here - 1) in |= 1u << __shfl_sync(0xffffffffu, t.symbol[q], __ffs(here) - 1) % 32;
          });
        }
        f(now[k], (in >> lane & 1u) != 0u);
      }
    }
  };
  float mo = -INFINITY;
  every([&](float l, bool in) { mo = fmaxf(mo, in ? -INFINITY : l); });
  mo = warp_max(mo);
  if (mo == -INFINITY) mo = m;
  float so = 0.0f, si = 0.0f;
  every([&](float l, bool in) {
    const float e = ex2_ftz((l - (in ? m : mo)) * c);
    so += in ? 0.0f : e;
    si += in ? e : 0.0f;
  });
  so = warp_sum(so);
  si = warp_sum(si);
  finish(a, r, t, {so > 0.0f ? (mo - m) * c : 0.0f, so}, {0.0f, si}, z, (mo - m) / a.temperature, m / a.temperature);
}

// The sum of the listed symbols that a team has met, by a warp; x: their logits.
template <int W>
__device__ __forceinline__ Part sum_met(const Listed<W>& s, int top, const float (&x)[kPerLane], float c) {
  const int lane = threadIdx.x & 31;
  Part in{-kFar, 0.0f};
  bool met[kPerLane];
  List::each(top, [&](int q) {
    met[q] = lane + 32 * q < top && s.met[lane + 32 * q];
    if (met[q]) in.m = fmaxf(in.m, x[q] * c);
  });
  in.m = warp_max(in.m);
  List::each(top, [&](int q) {
    if (met[q]) in.s += ex2_ftz(fmaf(x[q], c, -in.m));
  });
  in.s = warp_sum(in.s);
  return in;
}

// A row's results from the sums of its logits (of those not listed and of those listed, with TAIL), by a warp; any: of
// those not listed there are some above -inf, be it lowest values, whose terms are 0.
template <int DT, bool TAIL>
__device__ __forceinline__ void end_row(const mca_distill_args& a, int64_t r, float c, const List& t, const Part& out,
                                        const Part& in, bool any, const float (&x)[kPerLane]) {
  const float to = fmaxf(out.m, in.m), all = out.s + in.s, inv = 1.0f / a.temperature;
  if (!(all > 0.0f && all < INFINITY && to > -kFar && to < kFar) || (TAIL && out.s == 0.0f && any)) {
    any_row<DT>(a, r, c);
    return;
  }
  float z[kPerLane];
  List::each(a.top, [&](int q) {
    z[q] = fmaf(x[q], c, -to) * kLn2;
    if (z[q] == -INFINITY) z[q] = x[q] * inv;                    // (x c has no number, x / T may have one)
  });
  finish(a, r, t, out, in, z, (out.m - to) * kLn2, 0.0f);
}

template <int DT, int W, bool TAIL>
__global__ void __launch_bounds__(32 * W, 32 / W) distill_kernel(mca_distill_args a, float c, int split) {
  using P = Pieces<DT>;
  constexpr int kTeam = 32 * W, N = P::N;
  constexpr bool kWhole = W == kWarps;                          // a row may have a cluster's CTAs
  __shared__ uint4 s_ring[kAhead][kTeam];
  alignas(16) __shared__ Part s_part[kWhole ? kMaxCluster : 1][2];      // written 16 bytes at a time
  __shared__ Part s_warp[W];
  __shared__ int s_any[W], s_any_part[kWhole ? kMaxCluster : 1];
  __shared__ std::conditional_t<TAIL, Listed<W>, int> s_listed;
  const int tid = threadIdx.x, warp = tid >> 5;
  const int64_t r = kWhole ? (int64_t)blockIdx.x / split : (int64_t)blockIdx.x;
  const int rank = kWhole && split > 1 ? (int)cluster_rank() : 0;
  const P row(static_cast<const elem_t<DT>*>(a.logits) + r * a.ld, a.vocab);
  const int j0 = kWhole ? (int)((int64_t)row.count * rank / split) : 0;
  const int j1 = kWhole ? (int)((int64_t)row.count * (rank + 1) / split) : row.count;
  if (kWhole && split > 1) cluster_arrive();                     // every CTA runs before one writes to another

  List t;
  float x[kPerLane];
  Sum<DT> sum(c);
  unsigned int mask = 0u;                                        // groups of rounds with listed symbols
  stream_pieces<DT, W, kAhead>(row, j0, j1, s_ring, [&] {
    if (warp == 0) {
      t.read(a, r);
      List::each(a.top, [&](int q) { x[q] = t.symbol[q] >= 0 ? elem_f32(row.x[t.symbol[q]]) : 0.0f; });
      if constexpr (TAIL) mark<DT, W>(row, j0, j1, t, a.top, s_listed);
    }
    if constexpr (TAIL) {
      team_sync<W>();
      mask = s_listed.mask[warp];
    }
  }, [&](auto one) {
    in_groups<kTeam, true>(j0 + (tid & ~31), j1, mask, group_of(j1 - j0, kTeam), [&](int base) {
      if constexpr (TAIL) return met_in<DT, W>(base, j1, a.top, s_listed);
      return 0u;
    }, one, [&] { sum.close(); });
  }, [&](uint4 q, unsigned int gone) {
    if (TAIL && gone) q = without<DT>(q, gone);
    float2 v[N / 2];
    const float largest = unpack_max<DT>(q, v);
    sum.take(v, largest);
  });
  __syncwarp();
  Part out = sum.part(), in{-kFar, 0.0f};
  int any = TAIL && __any_sync(0xffffffffu, sum.any());
  out.join_lanes();
  if ((tid & 31) == 0) {
    s_warp[warp] = out;
    s_any[warp] = any;
  }
  team_sync<W>();
  if (warp == 0) {
    out = s_warp[0];
    for (int q = 1; q < W; ++q) {
      out.join(s_warp[q]);
      any |= s_any[q];
    }
  }
  if constexpr (TAIL) {
    if (warp == 0) in = sum_met(s_listed, a.top, x, c);
  }
  if (kWhole && split > 1) {                                     // to the cluster's first CTA
    cluster_wait();
    if (tid == 0) {
      asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};"
                   ::"r"(first_cta(&s_part[rank])), "f"(out.m), "f"(out.s), "f"(in.m), "f"(in.s) : "memory");
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(first_cta(&s_any_part[rank])), "r"(any) : "memory");
    }
    cluster_arrive();
    cluster_wait();
    if (rank != 0) return;
    out = s_part[0][0];
    in = s_part[0][1];
    any = s_any_part[0];
    for (int q = 1; q < split; ++q) {
      out.join(s_part[q][0]);
      in.join(s_part[q][1]);
      any |= s_any_part[q];
    }
  }
  if (warp == 0) end_row<DT, TAIL>(a, r, c, t, out, in, any != 0, x);
}

// Rows in between, and many: a CTA of W warps has a row in shared memory, all of it on its way at once, and goes over it
// twice, for the largest logit and for the sums (a reference that follows the logits took 20000 x 4000 bf16 against 32
// symbols 92 us, here 44). With tail the first warp puts -inf in the places of the listed symbols before that and adds them
// up itself: 47 us (174 and 71 with listed symbols told apart round by round, and by bits). Few warps, so that what a row
// takes beside its logits is not their all: twice as many take 10000 x 10000 bf16 66 us for 47, half as many 20000 x 4000
// fp32 69 for 55. Rows of more than 2048 pieces pay with tail (6000 x 20000 bf16 66 for 72 us, 10000 x 10000 fp32 77 for
// 101 at the time), where whole CTAs tell listed symbols apart; without they do not (61 for 46, 73 for 64).
template <int DT, int W>
__global__ void __launch_bounds__(32 * W) distill_row_kernel(mca_distill_args a, float c) {
  using P = Pieces<DT>;
  constexpr int N = P::N, kTeam = 32 * W;
  extern __shared__ uint4 s_row[];
  __shared__ float s_part[2][W];
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const Pieces<DT> row(static_cast<const elem_t<DT>*>(a.logits) + r * a.ld, a.vocab);
  for (int j = tid; j < row.count; j += kTeam) {                // a thread's pieces are read by itself alone
    const unsigned int at = (unsigned int)__cvta_generic_to_shared(&s_row[j]);
    if (row.whole(j))
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(row.pieces() + j) : "memory");
    else
      s_row[j] = P::part(row.x, row.V, row.index(j, 0));
  }
  asm volatile("cp.async.commit_group;" ::: "memory");
  List t;
  float x[kPerLane];
  if (warp == 0) {
    t.read(a, r);
    List::each(a.top, [&](int k) { x[k] = t.symbol[k] >= 0 ? elem_f32(row.x[t.symbol[k]]) : 0.0f; });
  }
  auto team_max = [&](float v, float* part) {                   // NaN if one is
    v = warp_max_nan(v);
    if constexpr (W > 1) {
      if (lane == 0) part[warp] = v;
      team_sync<W>();
      for (int k = 0; k < W; ++k) v = max_nan(v, part[k]);
    }
    return v;
  };
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  float xs[kPerLane];                                           // of the first entry of each symbol
  if (a.tail) {                                                 // -inf in the places of the listed symbols
    team_sync<W>();
    if (warp == 0) {
      elem_t<DT>* places = reinterpret_cast<elem_t<DT>*>(s_row) + row.head;
      List::each(a.top, [&](int k) {
        const bool is = t.symbol[k] >= 0;
        elem_t<DT>& place = places[is ? t.symbol[k] : 0];
        xs[k] = is ? elem_f32(place) : -INFINITY;                         // (-inf if an earlier 32 had it)
        __syncwarp();
        if (is) place = elem_of<DT>((float)lane);
        __syncwarp();
        // two lanes of one symbol: of it the first has the logit
        if (__any_sync(0xffffffffu, is && elem_f32(place) != (float)lane) && !t.leads(k)) xs[k] = -INFINITY;
        __syncwarp();
        if (is) place = elem_of<DT>(-INFINITY);
        __syncwarp();
      });
    }
    team_sync<W>();
  }

  float mo = -INFINITY;                                         // the largest of the others, or of all without tail
#pragma unroll 4
  for (int j = tid; j < row.count; j += kTeam) mo = max_nan(mo, largest<DT>(s_row[j]));
  mo = team_max(mo, s_part[0]);
  float m = mo, mi = -INFINITY;                                 // and of all (NaN if one is)
  if (a.tail) {
    if (warp == 0) {
      List::each(a.top, [&](int k) { mi = max_nan(mi, xs[k]); });
      mi = warp_max_nan(mi);
    }
    m = max_nan(mo, mi);                                        // (other warps: of the others)
  }
  if (warp == 0 && !(m > -INFINITY && m < INFINITY)) finish_without(a, r, t, m);
  if (!(mo > -INFINITY && mo < INFINITY)) mo = 0.0f;
  float2 s2 = make_float2(0.0f, 0.0f);
  const float2 cc = make_float2(c, c), mm = make_float2(-mo, -mo);
#pragma unroll 4
  for (int j = tid; j < row.count; j += kTeam) {
    float v[N];
    Pieces<DT>::values(s_row[j], v);
#pragma unroll
    for (int e = 0; e < N; e += 2) {
      const float2 z = mul2(add2(make_float2(v[e], v[e + 1]), mm), cc);
      s2 = add2(s2, make_float2(ex2_ftz(z.x), ex2_ftz(z.y)));
    }
  }
  float so = warp_sum(s2.x + s2.y);
  if constexpr (W > 1) {
    if (lane == 0) s_part[1][warp] = so;
    team_sync<W>();
    so = 0.0f;
    for (int k = 0; k < W; ++k) so += s_part[1][k];
  }
  if (warp != 0 || !(m > -INFINITY && m < INFINITY)) return;
  float si = 0.0f;
  if (a.tail) {
    List::each(a.top, [&](int k) { si += ex2_ftz((xs[k] - m) * c); });
    si = warp_sum(si);
  }
  float z[kPerLane];
  List::each(a.top, [&](int k) { z[k] = (x[k] - m) / a.temperature; });
  finish(a, r, t, {so > 0.0f ? (mo - m) * c : 0.0f, so}, {0.0f, si}, z, (mo - m) / a.temperature, m / a.temperature);
}

// Long rows, and many: CTAs that stay, each with a row after the other, eight warps that add up pieces, one that reads lists
// and one that writes results. Pieces of the next row are on their way before the row ends, its list is there when it
// begins, and what ends a row holds no other warp up. Lists and sums have two places, which take turns, and three
// barriers for each: `ready` says that a row's list is there, `full` that its sums are, `done` that its results are written
// (one warp for both lists and results took 5.5 us a row, more than a row of 64 kB does; with 16 warps and two CTAs to an
// SM a warp has too few pieces of a row for what each row takes beside them). 4096 x 128000 bf16: 162 us, 96 % of the
// memory's rate; 2048 x 50001 39, with five rows to a CTA of 4.5; 4096 x 32000 fp16 with tail 54, instructions.
constexpr int kStreamWarps = 8;
constexpr int kStreamThreads = 32 * kStreamWarps + 64;

struct Prepared {
  int symbol[kMaxList];
  float p[kMaxList], lp[kMaxList], x[kMaxList];
  float rest, total;
  bool bad;
  Listed<kStreamWarps> listed;
};

// Barriers of the streaming warps and one of the others, and of two others.
constexpr int kReady = 1, kFull = 3, kDone = 5;
constexpr int kStreamTeam = 32 * kStreamWarps;
template <int THREADS = kStreamTeam + 32>
__device__ __forceinline__ void wait_at(int barrier) {
  __syncwarp();
  asm volatile("bar.sync %0, %1;" ::"r"(barrier), "n"(THREADS) : "memory");
}
template <int THREADS = kStreamTeam + 32>
__device__ __forceinline__ void arrive_at(int barrier) {
  __syncwarp();
  asm volatile("bar.arrive %0, %1;" ::"r"(barrier), "n"(THREADS) : "memory");
}

// Rows cut into `parts` of `per` pieces; a CTA has the units blockIdx.x, blockIdx.x + gridDim.x, ..
struct Units {
  int count, per, parts;
  __device__ __forceinline__ int row(int u) const { return parts == 1 ? u : u / parts; }
  __device__ __forceinline__ int first_piece(int u) const { return parts == 1 ? 0 : (u - row(u) * parts) * per; }
};

// The pieces of a CTA's units for the threads of the streaming warps, each thread's in its own order, kAhead of them on
// their way to shared memory, across the units' borders. What is not whole is put there by its thread.
template <int DT>
struct PieceRing {
  using P = Pieces<DT>;
  static constexpr unsigned int kSlot = kStreamTeam * 16;
  const elem_t<DT>* x;
  int64_t ld;
  int V;
  Units units;
  unsigned int ring, slot, whole;
  int unit, next, end, first;               // whole pieces from `first` on without a look at the rest
  const uint4* from;

  __device__ __forceinline__ PieceRing(const void* logits, int64_t ld_, int V_, const Units& units_,
                                       uint4 (&s_ring)[kAhead][kStreamTeam])
      : x(static_cast<const elem_t<DT>*>(logits)), ld(ld_), V(V_), units(units_) {
    ring = slot = (unsigned int)__cvta_generic_to_shared(&s_ring[0][threadIdx.x]);
    unit = blockIdx.x;
    begin();
#pragma unroll
    for (int i = 0; i < kAhead; ++i) ask();
  }
  __device__ __forceinline__ P row_of(int u) const { return P(x + units.row(u) * ld, V); }
  __device__ __forceinline__ void begin() {
    const P row = row_of(unit);
    const int j0 = units.first_piece(unit);
    end = min(row.count, j0 + units.per);
    first = max(j0, row.whole(0) ? 0 : 1);
    whole = (unsigned int)max(0, min(end, row.count - (row.whole(row.count - 1) ? 0 : 1)) - first);
    next = j0 + (int)threadIdx.x;
    from = row.pieces() + next;
  }
  __device__ __forceinline__ void copy() const {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(slot), "l"(from) : "memory");
  }
  __device__ __forceinline__ void at_an_end() {
    while (next >= end) {
      if (units.count - unit <= (int)gridDim.x) {
        unit = units.count;
        return;
      }
      unit += gridDim.x;
      begin();
    }
    if ((unsigned int)(next - first) < whole) {
      copy();
    } else {
      const P row = row_of(unit);
      const uint4 q = P::part(row.x, V, row.index(next, 0));
      asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};"
                   ::"r"(slot), "r"(q.x), "r"(q.y), "r"(q.z), "r"(q.w) : "memory");
    }
  }
  __device__ __forceinline__ void ask() {
    if ((unsigned int)(next - first) < whole)
      copy();
    else if (unit < units.count)
      at_an_end();
    asm volatile("cp.async.commit_group;" ::: "memory");
    next += kStreamTeam;
    from += kStreamTeam;
    slot = slot == ring + (kAhead - 1) * kSlot ? ring : slot + kSlot;
  }
  // The thread's next piece; its place is free after ask().
  __device__ __forceinline__ uint4 take() const {
    uint4 q;
    asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "r"(slot) : "memory");
    return q;
  }
};

template <int DT, bool TAIL>
__global__ void __launch_bounds__(kStreamThreads, kStreamCtas) distill_stream_kernel(mca_distill_args a, float c) {
  using P = Pieces<DT>;
  constexpr int kTeam = kStreamTeam, N = P::N;
  __shared__ uint4 s_ring[kAhead][kTeam];
  __shared__ Part s_sum[2][kStreamWarps];
  __shared__ int s_any[2][kStreamWarps];
  __shared__ Prepared s_list[2];
  const int tid = threadIdx.x, lane = tid & 31, step = gridDim.x;
  auto row_of = [&](int64_t r) { return P(static_cast<const elem_t<DT>*>(a.logits) + r * a.ld, a.vocab); };

  if (tid >= kTeam + 32) {                                       // the warp of results
    int b = 0;
    for (int64_t r = blockIdx.x; r < a.rows; r += step, b ^= 1) {
      wait_at(kFull + b);
      Part out = s_sum[b][lane % kStreamWarps];
      const Prepared& s = s_list[b];
      List u;
      float x[kPerLane];
      List::each(a.top, [&](int q) {
        const int j = lane + 32 * q;
        u.symbol[q] = s.symbol[j];
        u.p[q] = s.p[j];
        u.lp[q] = s.lp[j];
        x[q] = s.x[j];
      });
      u.rest = s.rest;
      u.total = s.total;
      u.bad = s.bad;
      // (lanes behind the first ones have the warps once more)
      const float to = warp_max(out.m);
      out.s = warp_sum(lane < kStreamWarps ? out.s * ex2_ftz(out.m - to) : 0.0f);
      out.m = to;
      const Part in = TAIL ? sum_met(s.listed, a.top, x, c) : Part{-kFar, 0.0f};
      const bool any = TAIL && __any_sync(0xffffffffu, s_any[b][lane % kStreamWarps]);
      end_row<DT, TAIL>(a, r, c, u, out, in, any, x);
      arrive_at<64>(kDone + b);
    }
    return;
  }
  if (tid >= kTeam) {                                            // the warp of lists
    List t;
    t.load(a, blockIdx.x);
    int b = 0, i = 0;
    for (int64_t r = blockIdx.x; r < a.rows; r += step, b ^= 1, ++i) {
      Prepared& s = s_list[b];
      const P row = row_of(r);
      float x[kPerLane];
      List::each(a.top, [&](int q) {
        x[q] = t.symbol[q] >= 0 && t.symbol[q] < a.vocab ? elem_f32(row.x[t.symbol[q]]) : 0.0f;
      });
      t.resolve(a);
      if (i >= 2) wait_at<64>(kDone + b);
      if (TAIL) mark<DT, kStreamWarps>(row, 0, row.count, t, a.top, s.listed);
      List::each(a.top, [&](int q) {
        const int j = lane + 32 * q;
        s.symbol[j] = t.symbol[q];
        s.p[j] = t.p[q];
        s.lp[j] = t.lp[q];
        s.x[j] = x[q];
      });
      s.rest = t.rest;
      s.total = t.total;
      s.bad = t.bad;
      if (r + step < a.rows) t.load(a, r + step);                // on its way until the next row's turn
      arrive_at(kReady + b);
    }
    return;
  }

  PieceRing<DT> ring(a.logits, a.ld, a.vocab, Units{(int)a.rows, INT_MAX / 2, 1}, s_ring);
  int b = 0;
  for (int64_t r = blockIdx.x; r < a.rows; r += step, b ^= 1) {
    const int count = row_of(r).count, group = group_of(count, kTeam);
    wait_at(kReady + b);
    Sum<DT> sum(c);
    in_groups<kTeam, false>(tid - lane, count, TAIL ? s_list[b].listed.mask[tid >> 5] : 0u, group, [&](int base) {
      return TAIL ? met_in<DT, kStreamWarps>(base, count, a.top, s_list[b].listed) : 0u;
    }, [&](int base, unsigned int gone) {
      if (base + lane >= count) return;
      uint4 q = ring.take();
      if (TAIL && gone) q = without<DT>(q, gone);
      float2 v[N / 2];
      const float largest = unpack_max<DT>(q, v);
      sum.take(v, largest);
      ring.ask();
    }, [] {});
    __syncwarp();
    Part out = sum.part();
    const float to = warp_max(out.m);
    out.s = warp_sum(out.s * ex2_ftz(out.m - to));
    const int any = __any_sync(0xffffffffu, sum.any());
    if (lane == 0) {
      s_sum[b][tid >> 5] = {to, out.s};
      s_any[b][tid >> 5] = any;
    }
    arrive_at(kFull + b);
  }
}

// ------------------------------------------------------------------------------------------------
// Gradient: g / T times total q - p for a listed symbol, and for another one total q - P q / exp(rest), a multiple of q
// that is the same for the whole row: sign exp(x / T - lse + k).
// ------------------------------------------------------------------------------------------------
constexpr int kBackThreads = 256;

// What a row's gradient is made of.
struct Coefficients {
  float inv, lse, total, g, k, gs;        // g: of the loss, over the temperature; gs: with the others' sign
  __device__ __forceinline__ void set(const mca_distill_backward_args& a, int64_t r, const List& t) {
    inv = 1.0f / a.temperature;
    lse = a.lse[r];
    total = t.total;
    g = a.g_loss[r] * inv;
    k = total > 0.0f ? logf(total) : -INFINITY;
    float sign = 1.0f;
    if (t.rest > 0.0f && !(a.rest[r] < kLeastLog)) {
      // (of a rest so small that its inverse has no number, nothing else counts)
      const float l = logf(t.rest) - a.rest[r], d = total - expf(l);
      sign = d < 0.0f ? -1.0f : 1.0f;
      k = l > 80.0f ? l : logf(fabsf(d));
    }
    if (t.bad || !(lse < INFINITY)) {
      g = NAN;
    } else if (lse == -INFINITY) {        // no symbol is left: q = 0, and no gradient
      lse = INFINITY;
      g = k = 0.0f;
    }
    gs = sign * g;
  }
  __device__ __forceinline__ float listed(float x, float p) const {
    return g * (total * ex2_ftz(fmaf(x, inv, -lse) * kLog2e) - p);
  }
  // Of two logits that are not listed. Where the result has 16 bits k is taken into lse first (whose rounding, 2^-24 of
  // it, is a thousandth of the result's).
  template <int DT>
  __device__ __forceinline__ float2 others(float2 x) const {
    float2 z;
    if constexpr (DT == MCA_DTYPE_FP32)
      z = add2(fma2(x, make_float2(inv, inv), make_float2(-lse, -lse)), make_float2(k, k));
    else
      z = fma2(x, make_float2(inv, inv), make_float2(k - lse, k - lse));
    z = mul2(z, make_float2(kLog2e, kLog2e));
    return mul2(make_float2(ex2_ftz(z.x), ex2_ftz(z.y)), make_float2(gs, gs));
  }
};

template <int DT>
__device__ __forceinline__ uint4 pack(const float2 (&v)[Pieces<DT>::N / 2]) {
  if constexpr (DT == MCA_DTYPE_FP32) {
    return make_uint4(__float_as_uint(v[0].x), __float_as_uint(v[0].y), __float_as_uint(v[1].x),
                      __float_as_uint(v[1].y));
  } else {
    unsigned int w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (DT == MCA_DTYPE_BF16) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[i].x, v[i].y);
        w[i] = *reinterpret_cast<const unsigned int*>(&h);
      } else {
        const __half2 h = __floats2half2_rn(v[i].x, v[i].y);
        w[i] = *reinterpret_cast<const unsigned int*>(&h);
      }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// The rows of logits and gradient, by 16-byte pieces of the gradient. SAME: both lie at the same distance from 16-byte
// boundaries; otherwise a piece's logits are cut from the two 16-byte blocks that hold them, or read one by one where
// these hold more than the row's own.
template <int DT, bool SAME>
struct GradRow {
  using P = Pieces<DT>;
  static constexpr int N = P::N;
  const elem_t<DT>* x;
  elem_t<DT>* out;
  P row;                                  // of the gradient
  const uint4* blocks;
  unsigned int by, whole, own;
  int first, own_first;                   // whole pieces, and those that are cut from the row's own blocks, from here on

  __device__ __forceinline__ GradRow(const mca_distill_backward_args& a, int64_t r)
      : x(static_cast<const elem_t<DT>*>(a.logits) + r * a.ld), out(static_cast<elem_t<DT>*>(a.grad) + r * a.ldg),
        row(out, a.vocab) {
    const uintptr_t from = reinterpret_cast<uintptr_t>(x - row.head);
    by = SAME ? 0u : (unsigned int)(from & 15u);
    blocks = reinterpret_cast<const uint4*>(from - by);
    first = row.whole(0) ? 0 : 1;
    whole = (unsigned int)max(0, row.count - (row.whole(row.count - 1) ? 0 : 1) - first);
    own_first = SAME ? first : first_of_own_blocks(row.head, (int)by, (int)sizeof(elem_t<DT>));
    own = SAME ? whole
               : (unsigned int)max(0, end_of_own_blocks(row.V, row.head, (int)by, (int)sizeof(elem_t<DT>)) - own_first);
  }
  __device__ __forceinline__ bool is_whole(int j) const { return (unsigned int)(j - first) < whole; }
  __device__ __forceinline__ bool is_own(int j) const { return (unsigned int)(j - own_first) < own; }
  // The logits of piece j as they are, or the two blocks that they are cut from.
  struct Raw {
    uint4 lo, hi;
  };
  __device__ __forceinline__ void ask(int j, Raw& q) const {
    if (is_own(j)) {
      q.lo = blocks[j];
      if (!SAME && by) q.hi = blocks[j + 1];           // (behind a row that lies alike may be nothing)
    } else {
      q.lo = P::part(x, row.V, row.index(j, 0));
    }
  }
  __device__ __forceinline__ void write(int j, const Raw& raw, const Coefficients& w) const {
    const bool all = is_whole(j);
    float v[N];
    float2 d[N / 2];
    P::values(SAME || !is_own(j) ? raw.lo : shifted(raw.lo, raw.hi, by), v);
#pragma unroll
    for (int e = 0; e < N; e += 2) d[e / 2] = w.others<DT>(make_float2(v[e], v[e + 1]));
    const uint4 o = pack<DT>(d);
    if (all) {
      reinterpret_cast<uint4*>(out - row.head)[j] = o;
    } else {
      P::values(o, v);
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (row.index(j, e) >= 0 && row.index(j, e) < row.V) out[row.index(j, e)] = elem_of<DT>(v[e]);
    }
  }
};

// What is listed of symbols v0 .. v1, over what has been written there as if it were not. A warp; x: their logits.
template <int DT>
__device__ __forceinline__ void write_listed(elem_t<DT>* out, const List& t, int top, const Coefficients& w,
                                             const float (&x)[kPerLane], int v0, int v1) {
  List::each(top, [&](int q) {
    const int v = t.symbol[q];
    if (v >= 0 && v >= v0 && v < v1) out[v] = elem_of<DT>(w.listed(x[q], t.p[q]));
  });
}

// Short rows: a warp for each, P pieces to a lane (0: as many as there are, one after the other).
template <int DT, int P, bool SAME>
__global__ void __launch_bounds__(kSmallThreads) distill_backward_small_kernel(mca_distill_backward_args a) {
  __shared__ unsigned int s_seen[kSmallThreads / 32][List::kSeenWords];
  const int64_t r = (int64_t)blockIdx.x * (kSmallThreads / 32) + threadIdx.x / 32;
  if (r >= a.rows) return;
  const int lane = threadIdx.x & 31;
  const GradRow<DT, SAME> g(a, r);
  constexpr int kHold = P > 0 ? P : 4;
  List t;
  t.load(a, r);
  typename GradRow<DT, SAME>::Raw q[kHold];
#pragma unroll
  for (int i = 0; i < kHold; ++i)
    if (lane + 32 * i < g.row.count) g.ask(lane + 32 * i, q[i]);
  float x[kPerLane];
  List::each(a.top, [&](int k) { x[k] = t.symbol[k] >= 0 && t.symbol[k] < a.vocab ? elem_f32(g.x[t.symbol[k]]) : 0.0f; });
  t.resolve(a);
  Coefficients w;
  w.set(a, r, t);
  t.merge(a.top, a.vocab, s_seen[threadIdx.x / 32]);
  __syncwarp();                                         // (the listed symbols' logits are read before another lane writes)
  if constexpr (P > 0) {
#pragma unroll
    for (int i = 0; i < P; ++i)
      if (lane + 32 * i < g.row.count) g.write(lane + 32 * i, q[i], w);
  } else {
    for (int j = lane; j < g.row.count; j += 32 * kHold) {
#pragma unroll
      for (int i = 0; i < kHold; ++i) {
        const int at = j + 32 * i;
        if (at >= g.row.count) break;
        const auto now = q[i];
        if (at + 32 * kHold < g.row.count) g.ask(at + 32 * kHold, q[i]);
        g.write(at, now, w);
      }
    }
  }
  __syncwarp();                                         // (the other symbols are written)
  write_listed<DT>(g.out, t, a.top, w, x, 0, a.vocab);
}

// Long rows that lie differently: `per` pieces to a CTA.
constexpr int kBackAhead = 2;             // pieces whose loads a thread issues together
template <int DT>
__global__ void __launch_bounds__(kBackThreads) distill_backward_kernel(mca_distill_backward_args a, int per,
                                                                        int parts) {
  __shared__ Coefficients s_w;
  __shared__ unsigned int s_seen[List::kSeenWords];
  const int64_t r = blockIdx.x / parts;
  const GradRow<DT, false> g(a, r);
  const int tid = threadIdx.x, j0 = (int)(blockIdx.x - r * parts) * per, j1 = min(g.row.count, j0 + per);
  typename GradRow<DT, false>::Raw q[kBackAhead];
#pragma unroll
  for (int i = 0; i < kBackAhead; ++i)
    if (j0 + tid + kBackThreads * i < j1) g.ask(j0 + tid + kBackThreads * i, q[i]);
  List t;
  float x[kPerLane];
  if (tid < 32) {
    t.load(a, r);
    List::each(a.top, [&](int k) {
      x[k] = t.symbol[k] >= 0 && t.symbol[k] < a.vocab ? elem_f32(g.x[t.symbol[k]]) : 0.0f;
    });
    t.resolve(a);
    if (tid == 0) s_w.set(a, r, t);
    t.merge(a.top, a.vocab, s_seen);
  }
  __syncthreads();
  const Coefficients w = s_w;
  for (int j = j0 + tid; j < j1; j += kBackThreads * kBackAhead) {
#pragma unroll
    for (int i = 0; i < kBackAhead; ++i) {
      const int at = j + kBackThreads * i;
      if (at >= j1) break;
      const auto now = q[i];
      if (at + kBackThreads * kBackAhead < j1) g.ask(at + kBackThreads * kBackAhead, q[i]);
      g.write(at, now, w);
    }
  }
  __syncthreads();
  if (tid < 32) write_listed<DT>(g.out, t, a.top, w, x, g.row.index(j0, 0), g.row.index(j1, 0));
}

// Long rows that lie alike in both matrices: CTAs that stay, as for the loss, with a part of a row after the other. Eight
// warps write every symbol's gradient as if it were not listed; the ninth reads lists, a part ahead, and writes the listed
// symbols' gradients when the others are done with the part. (With a CTA and a list for each part, and a look into the
// bitmap for each piece, 2048 x 50001 bf16 took 86 us.)
constexpr int kBackCtas = 3;              // per SM

struct PartList {
  Coefficients w;
  int symbol[kMaxList];                   // -1: not in the part, or none
  float p[kMaxList], x[kMaxList];         // of all of its entries; its logit
};

template <int DT>
__global__ void __launch_bounds__(kStreamTeam + 32, kBackCtas)
    distill_backward_stream_kernel(mca_distill_backward_args a, Units units) {
  using P = Pieces<DT>;
  constexpr int N = P::N;
  __shared__ uint4 s_ring[kAhead][kStreamTeam];
  __shared__ PartList s_list[2];
  __shared__ unsigned int s_seen[List::kSeenWords];
  const int tid = threadIdx.x, lane = tid & 31, step = gridDim.x;
  const elem_t<DT>* logits = static_cast<const elem_t<DT>*>(a.logits);
  elem_t<DT>* grad = static_cast<elem_t<DT>*>(a.grad);

  if (tid >= kStreamTeam) {                                      // the warp of lists
    List t;
    t.load(a, units.row(blockIdx.x));
    // the listed symbols' gradients of a part that the other warps have written
    auto write_part = [&](int u, int b) {
      wait_at(kDone + b);
      const PartList& s = s_list[b];
      elem_t<DT>* out = grad + units.row(u) * a.ldg;
      List::each(a.top, [&](int q) {
        const int j = lane + 32 * q;
        if (s.symbol[j] >= 0) out[s.symbol[j]] = elem_of<DT>(s.w.listed(s.x[j], s.p[j]));
      });
      __syncwarp();
    };
    int b = 0, u = blockIdx.x;
    for (; u < units.count; u += step, b ^= 1) {
      const int r = units.row(u);
      const P row(logits + r * a.ld, a.vocab);
      const int j0 = units.first_piece(u), j1 = min(row.count, j0 + units.per);
      float x[kPerLane];
      List::each(a.top, [&](int q) {
        x[q] = t.symbol[q] >= 0 && t.symbol[q] < a.vocab ? elem_f32(row.x[t.symbol[q]]) : 0.0f;
      });
      t.resolve(a);
      Coefficients w;
      w.set(a, r, t);
      t.merge(a.top, a.vocab, s_seen);
      if (u - 2 * step >= 0) write_part(u - 2 * step, b);
      PartList& s = s_list[b];
      if (lane == 0) s.w = w;
      List::each(a.top, [&](int q) {
        const int i = t.symbol[q], j = i >= 0 ? (i + row.head) / N : -1;
        s.symbol[lane + 32 * q] = j >= j0 && j < j1 ? i : -1;
        s.p[lane + 32 * q] = t.p[q];
        s.x[lane + 32 * q] = x[q];
      });
      if (u + step < units.count) t.load(a, units.row(u + step));            // on its way until the next part's turn
      arrive_at(kReady + b);
    }
    if (u - 2 * step >= 0) write_part(u - 2 * step, b);
    if (u - step >= 0) write_part(u - step, b ^ 1);
    return;
  }

  PieceRing<DT> ring(a.logits, a.ld, a.vocab, units, s_ring);
  int b = 0;
  for (int u = blockIdx.x; u < units.count; u += step, b ^= 1) {
    const P row = ring.row_of(u);
    elem_t<DT>* out = grad + units.row(u) * a.ldg;
    uint4* pieces = reinterpret_cast<uint4*>(out - row.head);
    const int j0 = units.first_piece(u), j1 = min(row.count, j0 + units.per);
    const int first = row.whole(0) ? 0 : 1;
    const unsigned int whole = (unsigned int)(row.count - (row.whole(row.count - 1) ? 0 : 1) - first);
    wait_at(kReady + b);
    const Coefficients w = s_list[b].w;
    for (int j = j0 + tid; j < j1; j += kStreamTeam) {
      const uint4 q = ring.take();
      float v[N];
      float2 d[N / 2];
      P::values(q, v);
#pragma unroll
      for (int e = 0; e < N; e += 2) d[e / 2] = w.others<DT>(make_float2(v[e], v[e + 1]));
      ring.ask();
      const uint4 o = pack<DT>(d);
      if ((unsigned int)(j - first) < whole) {
        pieces[j] = o;
      } else {
        float e[N];
        P::values(o, e);
#pragma unroll
        for (int k = 0; k < N; ++k)
          if (row.index(j, k) >= 0 && row.index(j, k) < a.vocab) out[row.index(j, k)] = elem_of<DT>(e[k]);
      }
    }
    arrive_at(kDone + b);
  }
}

// ------------------------------------------------------------------------------------------------

float scale_of(float temperature) { return (float)(1.4426950408889634 / (double)temperature); }

template <int DT, int P>
cudaError_t launch_small(const mca_distill_args& a, float c, cudaStream_t s) {
  constexpr int kRows = kSmallThreads / 32;
  distill_small_kernel<DT, P><<<(unsigned int)((a.rows + kRows - 1) / kRows), kSmallThreads, 0, s>>>(a, c);
  return cudaGetLastError();
}

template <int DT, int W>
cudaError_t launch_row(const mca_distill_args& a, float c, int64_t count, cudaStream_t s) {
  const size_t bytes = (size_t)count * 16, beside = 2 * W * sizeof(float);         // (s_part)
  if (bytes + beside > 48 << 10) {
    const cudaError_t e = cudaFuncSetAttribute(distill_row_kernel<DT, W>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               kRowPieces * 16);
    if (e != cudaSuccess) return e;
  }
  distill_row_kernel<DT, W><<<(unsigned int)a.rows, 32 * W, bytes, s>>>(a, c);
  return cudaGetLastError();
}

template <int DT, int W>
cudaError_t launch_team(const mca_distill_args& a, float c, int split, cudaStream_t s) {
  return a.tail ? launch_clusters(distill_kernel<DT, W, true>, a.rows * split, 32 * W, split, s, a, c, split)
                : launch_clusters(distill_kernel<DT, W, false>, a.rows * split, 32 * W, split, s, a, c, split);
}

template <int DT>
cudaError_t launch_distill_t(const mca_distill_args& a, cudaStream_t s) {
  const float c = scale_of(a.temperature);
  const DistillShape h = distill_shape(a.rows, a.vocab, Pieces<DT>::N, a.tail != 0);
  switch (h.by) {
    case DistillBy::kRegisters:
      if (h.n == 1) return launch_small<DT, 1>(a, c, s);
      if (h.n == 2) return launch_small<DT, 2>(a, c, s);
      if (h.n == 4) return launch_small<DT, 4>(a, c, s);
      return launch_small<DT, 8>(a, c, s);
    case DistillBy::kSharedRow: {
      const int64_t count = most_pieces(a.vocab, Pieces<DT>::N);
      if (h.n == 1) return launch_row<DT, 1>(a, c, count, s);
      if (h.n == 2) return launch_row<DT, 2>(a, c, count, s);
      return launch_row<DT, 4>(a, c, count, s);
    }
    case DistillBy::kStaying:
      if (a.tail)
        distill_stream_kernel<DT, true><<<kSms * kStreamCtas, kStreamThreads, 0, s>>>(a, c);
      else
        distill_stream_kernel<DT, false><<<kSms * kStreamCtas, kStreamThreads, 0, s>>>(a, c);
      return cudaGetLastError();
    default:
      return h.n == 4 ? launch_team<DT, 4>(a, c, 1, s) : launch_team<DT, kWarps>(a, c, h.split, s);
  }
}

template <int DT, int P>
cudaError_t launch_backward_small(const mca_distill_backward_args& a, bool same, cudaStream_t s) {
  constexpr int kRows = kSmallThreads / 32;
  const unsigned int grid = (unsigned int)((a.rows + kRows - 1) / kRows);
  if (same)
    distill_backward_small_kernel<DT, P, true><<<grid, kSmallThreads, 0, s>>>(a);
  else
    distill_backward_small_kernel<DT, P, false><<<grid, kSmallThreads, 0, s>>>(a);
  return cudaGetLastError();
}

template <int DT>
cudaError_t launch_backward_t(const mca_distill_backward_args& a, cudaStream_t s) {
  const bool same = (reinterpret_cast<uintptr_t>(a.logits) - reinterpret_cast<uintptr_t>(a.grad)) % 16 == 0 &&
                    (a.rows == 1 || (a.ld - a.ldg) % Pieces<DT>::N == 0);
  const int64_t count = most_pieces(a.vocab, Pieces<DT>::N);
  if (count <= 32) return launch_backward_small<DT, 1>(a, same, s);
  if (count <= 64) return launch_backward_small<DT, 2>(a, same, s);
  if (count <= 128) return launch_backward_small<DT, 4>(a, same, s);
  if (count <= kSmallPieces) return launch_backward_small<DT, 8>(a, same, s);
  if (count <= 1024 && a.rows >= 4 * 152) return launch_backward_small<DT, 0>(a, same, s);
  if (same) {
    constexpr int64_t kCtas = 152 * kBackCtas;
    // Parts of a row: as many as give every CTA one, of a piece a thread at least; where rows are many, halves and
    // quarters if they come out more even.
    auto left = [&](int64_t parts) {                                      // the share of the last round that has no unit
      const int64_t units = a.rows * parts, rounds = (units + kCtas - 1) / kCtas;
      return (double)(rounds * kCtas - units) / (double)(rounds * kCtas);
    };
    int64_t parts = 1;
    while (a.rows * parts < kCtas ? count / (2 * parts) >= kStreamTeam
                                  : count / (2 * parts) >= 4 * kStreamTeam && left(2 * parts) + 0.03 < left(parts))
      parts *= 2;
    const int per = (int)((count + parts - 1) / parts);
    parts = (count + per - 1) / per;
    if (a.rows * parts <= INT_MAX / 2) {
      const Units units{(int)(a.rows * parts), per, (int)parts};
      distill_backward_stream_kernel<DT>
          <<<(unsigned int)std::min<int64_t>(kCtas, units.count), kStreamTeam + 32, 0, s>>>(a, units);
      return cudaGetLastError();
    }
  }
  // eight pieces a thread, fewer where rows are few
  const int64_t per = kBackThreads * std::min<int64_t>(8, std::max<int64_t>(1, a.rows * count / (kBackThreads * 152 * 4)));
  const int parts = (int)((count + per - 1) / per);
  distill_backward_kernel<DT><<<(unsigned int)(a.rows * parts), kBackThreads, 0, s>>>(a, (int)per, parts);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_distill(const mca_distill_args& a, cudaStream_t s) {
  if (a.dtype == MCA_DTYPE_FP32) return launch_distill_t<MCA_DTYPE_FP32>(a, s);
  if (a.dtype == MCA_DTYPE_FP16) return launch_distill_t<MCA_DTYPE_FP16>(a, s);
  return launch_distill_t<MCA_DTYPE_BF16>(a, s);
}

cudaError_t launch_distill_backward(const mca_distill_backward_args& a, cudaStream_t s) {
  if (a.dtype == MCA_DTYPE_FP32) return launch_backward_t<MCA_DTYPE_FP32>(a, s);
  if (a.dtype == MCA_DTYPE_FP16) return launch_backward_t<MCA_DTYPE_FP16>(a, s);
  return launch_backward_t<MCA_DTYPE_BF16>(a, s);
}

}  // namespace mca
