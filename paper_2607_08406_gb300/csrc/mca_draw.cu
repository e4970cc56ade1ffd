// Symbols drawn from rows of logits with given random numbers (mca_sample_tokens), and drafted symbols kept or replaced
// (mca_verify_drafts).
//
// A drawn symbol is where the cumulative sum of weights passes u times their sum, and every weight before it moves its
// border: with sums in fp32 one row in twenty of 128000 symbols would give a neighbour. So weights have an error of 2^-33 of
// themselves at most (2^-32 where a log-sum-exp is taken off), and are summed as integers, in steps of 2^-43 of a power of
// two that is at most 2^1.5 times the largest weight: a weight is the same number of steps in every sum, whatever the order.
// Each symbol may be off by half a step, with one sign for many that are equal, and a lane by two where a larger logit
// makes the steps coarser, which its four symbols and more share: by a step a symbol in all.
//
// x = n ln2 / 128 + d + e: an integer n, ln2 / 128 in two parts, so that d is exact, and e is what the second part gives.
// 2^(n / 128) is a power of two times one of 128 numbers T in a table, each with the logarithm of what its rounding left
// off, which goes to e. With r = d + e the weight is T + T g, g = r + r^2 / 2 + r^3 / 6, |g| < 2^-8, whose rounding is the
// error. 2 + T + T g rounds it to a step of 2^-22; what that leaves off, T g less a difference that is exact, is one fused
// product, and rounded to 2^-43 in the same way; the steps are differences of the results' bits. In all 15 operations of
// the FMA pipe a logit and about as many others: they bound the kernels, not the memory (5000 x 50001 bf16: 322 us, of
// which the memory takes 74; 256 x 50001 fp32: 30 of 8, with a CTA or two to an SM).
#include <algorithm>
#include <type_traits>

#include "mca_answers.h"
#include "mca_device.cuh"
#include "mca_elem.cuh"
#include "mca_row_shapes.h"
#include "mca_rows.cuh"

namespace mca {

namespace {

constexpr float kLn2 = 0.6931471805599453f;
constexpr int kWarps = kTeamWarps, kThreads = 32 * kWarps;
constexpr int kCtas = kDrawCtas;           // per SM: 80 registers a thread, with which constants stay there (with 64 and
                                           // 32 warps 5000 x 50001 bf16 took 390 us, now 322)
constexpr int kGroups = 8;                 // parts of a warp's pieces whose sums are kept
constexpr int kFetch = 256;                // pieces (4 kB) that a warp asks for at once, to L2
constexpr int kCopies = 8;                 // of the table, a quarter of the banks each (16 are no faster)

constexpr int kPowerBits = 7, kPowerCount = 1 << kPowerBits;
constexpr float kSteps = 0x1.715476p+7f;   // 128 / ln2
constexpr float kStep = 0x1.62e43p-8f;      // ln2 / 128 in two parts
constexpr float kStepLow = -0x1.05c61p-36f;
constexpr double kStepAll = 0x1.62e42fefa39efp-8;
constexpr float kHigh = 2.0f;              // and a weight below 2: steps of 2^-22
constexpr float kLow = 0x1.8p-20f;         // and what they leave off: steps of 2^-43
constexpr unsigned int kHighBits = 0x40000000u, kLowBits = 0x35c00000u;
constexpr int kHighShift = 21;             // between the two
constexpr int kUnitBits = 43;
constexpr float kFloor = 80.0f;            // weights below exp(-kFloor) of the largest are 0
constexpr float kMaxRef = 1024.0f;         // logits beyond go by the definition: n and the parts of ln2 have fewer digits
constexpr int kMaxVocab = 1 << 19;         // and so do larger vocabularies (sums below 2^63)
constexpr float kLeastU = 0x1p-24f;        // and numbers below, which draw from what the steps of sums cannot tell

// 2^(j / 128) in fp32 and the logarithm of what the rounding left off (their quotient).
__device__ const float2 kPowers[kPowerCount] = {
    {0x1p+0f, 0x0p+0f}, {0x1.0163dap+0f, 0x1.3dacd2p-25f}, {0x1.02c9a4p+0f, -0x1.844542p-28f},
    {0x1.04315ep+0f, 0x1.0976e4p-25f}, {0x1.059b0ep+0f, -0x1.947416p-25f}, {0x1.0706b2p+0f, 0x1.334fa4p-25f},
    {0x1.087452p+0f, -0x1.d32b6ep-26f}, {0x1.09e3ecp+0f, 0x1.4c0a72p-25f}, {0x1.0b5586p+0f, 0x1.8d96d4p-25f},
    {0x1.0cc922p+0f, 0x1.5cdc9p-25f}, {0x1.0e3ec4p+0f, -0x1.8f4da6p-25f}, {0x1.0fb66ap+0f, 0x1.e240f2p-25f},
    {0x1.11301ep+0f, -0x1.dda2fep-25f}, {0x1.12abdcp+0f, 0x1.935bfp-30f}, {0x1.1429aap+0f, 0x1.b2e50ep-25f},
    {0x1.15a98cp+0f, 0x1.fe3724p-26f}, {0x1.172b84p+0f, -0x1.9c0c22p-27f}, {0x1.18af94p+0f, -0x1.b2ec18p-26f},
    {0x1.1a35bep+0f, 0x1.4bfc22p-25f}, {0x1.1bbe08p+0f, 0x1.cfe886p-27f}, {0x1.1d4874p+0f, -0x1.a2fbb4p-25f},
    {0x1.1ed502p+0f, 0x1.55511p-27f}, {0x1.2063b8p+0f, 0x1.dc5deap-26f}, {0x1.21f49ap+0f, -0x1.99e61ep-25f},
    {0x1.2387a6p+0f, 0x1.964902p-25f}, {0x1.251ce4p+0f, 0x1.b6ba56p-25f}, {0x1.26b456p+0f, 0x1.4728b6p-26f},
    {0x1.284dfep+0f, 0x1.b13006p-28f}, {0x1.29e9ep+0f, -0x1.2b0dbcp-25f}, {0x1.2b87fep+0f, -0x1.9e35bep-25f},
    {0x1.2d285ap+0f, 0x1.76e04p-26f}, {0x1.2ecafap+0f, 0x1.f4214ep-26f}, {0x1.306fep+0f, 0x1.125002p-25f},
    {0x1.32171p+0f, -0x1.8c1444p-27f}, {0x1.33c08cp+0f, -0x1.6a4198p-25f}, {0x1.356c56p+0f, -0x1.69f6fp-30f},
    {0x1.371a74p+0f, -0x1.cde8cep-26f}, {0x1.38cae6p+0f, 0x1.551102p-25f}, {0x1.3a7db4p+0f, -0x1.21376ep-25f},
    {0x1.3c32dcp+0f, 0x1.3eda02p-27f}, {0x1.3dea64p+0f, 0x1.370be4p-25f}, {0x1.3fa45p+0f, 0x1.df22eep-27f},
    {0x1.4160a2p+0f, 0x1.90d1a4p-28f}, {0x1.431f5ep+0f, -0x1.52f5f4p-26f}, {0x1.44e086p+0f, 0x1.336de2p-30f},
    {0x1.46a41ep+0f, 0x1.48dff6p-25f}, {0x1.486a2cp+0f, -0x1.ff1cbep-26f}, {0x1.4a32bp+0f, -0x1.780896p-25f},
    {0x1.4bfdaep+0f, -0x1.0a3552p-25f}, {0x1.4dcb2ap+0f, -0x1.26ea3cp-26f}, {0x1.4f9b28p+0f, -0x1.ca37ep-26f},
    {0x1.516daap+0f, 0x1.10e596p-27f}, {0x1.5342b6p+0f, -0x1.c541b6p-26f}, {0x1.551a4cp+0f, 0x1.f1e18p-26f},
    {0x1.56f474p+0f, -0x1.bbeca4p-26f}, {0x1.58d12ep+0f, -0x1.0f012ap-25f}, {0x1.5ab07ep+0f, -0x1.00d8acp-27f},
    {0x1.5c9268p+0f, 0x1.e66c8p-26f}, {0x1.5e76f2p+0f, -0x1.e2a08p-26f}, {0x1.605e1cp+0f, -0x1.2fe3d6p-26f},
    {0x1.6247ecp+0f, -0x1.6cb284p-25f}, {0x1.643464p+0f, -0x1.0194c8p-25f}, {0x1.662388p+0f, 0x1.aad5bep-28f},
    {0x1.68155ep+0f, -0x1.0a30c8p-25f}, {0x1.6a09e6p+0f, 0x1.26055cp-26f}, {0x1.6c0128p+0f, -0x1.ed07ccp-26f},
    {0x1.6dfb24p+0f, -0x1.42c75ep-27f}, {0x1.6ff7ep+0f, -0x1.297d7p-26f}, {0x1.71f75ep+0f, 0x1.8b2bb8p-26f},
    {0x1.73f9a4p+0f, 0x1.7cd7f6p-26f}, {0x1.75feb6p+0f, -0x1.aab796p-26f}, {0x1.780694p+0f, 0x1.59b5a2p-25f},
    {0x1.7a1148p+0f, -0x1.05cb44p-25f}, {0x1.7c1edp+0f, 0x1.9a7cap-29f}, {0x1.7e2f34p+0f, -0x1.89fa7ap-26f},
    {0x1.804276p+0f, -0x1.f54f9p-26f}, {0x1.82589ap+0f, -0x1.1c2142p-26f}, {0x1.8471a4p+0f, 0x1.02f766p-26f},
    {0x1.868d9ap+0f, -0x1.8d087cp-27f}, {0x1.88ac7ep+0f, -0x1.0d831ap-26f}, {0x1.8ace54p+0f, 0x1.67a1cap-28f},
    {0x1.8cf322p+0f, -0x1.7f8592p-26f}, {0x1.8f1aeap+0f, -0x1.1bebb2p-26f}, {0x1.9145bp+0f, 0x1.d86ad4p-26f},
    {0x1.93737cp+0f, -0x1.348e56p-25f}, {0x1.95a44cp+0f, 0x1.dbe624p-26f}, {0x1.97d82ap+0f, -0x1.526432p-32f},
    {0x1.9a0f18p+0f, -0x1.2fe03cp-25f}, {0x1.9c4918p+0f, 0x1.a3b5e4p-28f}, {0x1.9e8632p+0f, -0x1.e335e2p-27f},
    {0x1.a0c668p+0f, -0x1.6c46c2p-27f}, {0x1.a309bep+0f, 0x1.e08496p-26f}, {0x1.a5503cp+0f, -0x1.0b7ec8p-25f},
    {0x1.a799e2p+0f, -0x1.ef7468p-26f}, {0x1.a9e6b6p+0f, -0x1.94d3dep-26f}, {0x1.ac36bcp+0f, -0x1.a55782p-32f},
    {0x1.ae89fap+0f, -0x1.f9c306p-27f}, {0x1.b0e072p+0f, 0x1.69980cp-26f}, {0x1.b33a2cp+0f, -0x1.21873p-26f},
    {0x1.b59728p+0f, 0x1.04240ep-25f}, {0x1.b7f77p+0f, -0x1.e4c886p-26f}, {0x1.ba5b04p+0f, -0x1.1ca7f8p-25f},
    {0x1.bcc1eap+0f, -0x1.2140f6p-25f}, {0x1.bf2c26p+0f, -0x1.30d0b4p-27f}, {0x1.c199bep+0f, -0x1.6961b4p-28f},
    {0x1.c40ab6p+0f, -0x1.ae9994p-40f}, {0x1.c67f12p+0f, 0x1.02861cp-25f}, {0x1.c8f6dap+0f, -0x1.ad47fp-26f},
    {0x1.cb720ep+0f, -0x1.b5151ep-28f}, {0x1.cdf0b6p+0f, -0x1.7927a4p-26f}, {0x1.d072d4p+0f, 0x1.61cd1p-26f},
    {0x1.d2f87p+0f, 0x1.1a8a98p-26f}, {0x1.d5818ep+0f, -0x1.a5217cp-28f}, {0x1.d80e32p+0f, -0x1.3fc1d4p-26f},
    {0x1.da9e6p+0f, 0x1.0a3ccap-27f}, {0x1.dd322p+0f, -0x1.be1cbep-26f}, {0x1.dfc974p+0f, -0x1.ab7132p-26f},
    {0x1.e26462p+0f, -0x1.76fb0cp-26f}, {0x1.e502eep+0f, 0x1.fdadbcp-27f}, {0x1.e7a52p+0f, -0x1.1bab4p-27f},
    {0x1.ea4afap+0f, 0x1.61428ep-28f}, {0x1.ecf482p+0f, 0x1.c28f6ep-26f}, {0x1.efa1bep+0f, 0x1.db5db6p-26f},
    {0x1.f252b4p+0f, -0x1.1a1198p-26f}, {0x1.f50766p+0f, -0x1.2ad5f8p-27f}, {0x1.f7bfdap+0f, 0x1.baba22p-26f},
    {0x1.fa7c18p+0f, 0x1.a31484p-29f}, {0x1.fd3c22p+0f, 0x1.73f078p-26f}};

using Table = float2[kPowerCount][kCopies];

__device__ __forceinline__ void fill_table(Table& t) {
  for (int i = threadIdx.x; i < kPowerCount * kCopies; i += kThreads) t[i / kCopies][i % kCopies] = kPowers[i / kCopies];
}

// exp(ref) = 2^(l / kPowerCount) exp(high + low), |high| < ln2 / 256, of 30 digits after the point.
struct Ref {
  int l;
  float high, low;
  __device__ __forceinline__ void set(double ref) {
    const double n = rint(ref * (1.0 / kStepAll)), r = ref - n * kStepAll, h = rint(r * 0x1p30) * 0x1p-30;
    l = (int)n;
    high = (float)h;
    low = (float)(r - h);
  }
};

// A weight exp(v - ref) below 2, of two logits: the bits of its two parts, whose differences to kHighBits and kLowBits are
// steps, and the weight itself to fp32's digits. SHIFT: ref.high and ref.low are not 0. (Constants are operands of single
// instructions; pairs of them would be copied into registers each time.)
struct Steps {
  float2 high, low, weight;
};

template <bool SHIFT>
__device__ __forceinline__ Steps steps_of_exp(float2 v, const Ref& ref, const Table& table) {
  const float shift = 12582912.0f - (float)ref.l;               // 1.5 2^23: the sum's bits are those of the integer
  const float2 t = make_float2(fmaf(v.x, kSteps, shift), fmaf(v.y, kSteps, shift));
  const float2 n = make_float2(t.x - shift, t.y - shift);
  float2 d = make_float2(fmaf(n.x, -kStep, v.x), fmaf(n.y, -kStep, v.y));
  const unsigned int bx = __float_as_uint(t.x), by = __float_as_uint(t.y), lane = threadIdx.x % kCopies;
  const float2 px = table[bx % kPowerCount][lane], py = table[by % kPowerCount][lane];
  // (the bits of 1.5 2^23 leave by the shift)
  const float2 T = make_float2(__uint_as_float(((bx >> kPowerBits) << 23) + __float_as_uint(px.x)),
                               __uint_as_float(((by >> kPowerBits) << 23) + __float_as_uint(py.x)));
  float2 e = make_float2(fmaf(n.x, -kStepLow, px.y), fmaf(n.y, -kStepLow, py.y));
  if (SHIFT) {
    d = make_float2(d.x - ref.high, d.y - ref.high);
    e = make_float2(e.x - ref.low, e.y - ref.low);
  }
  const float2 r = add2(d, e);
  const float2 c = make_float2(fmaf(r.x, 1.0f / 6.0f, 0.5f), fmaf(r.y, 1.0f / 6.0f, 0.5f));
  const float2 g = add2(d, fma2(mul2(r, r), c, e));            // exp(d + e) - 1
  Steps s;
  s.weight = fma2(T, g, T);
  s.high = make_float2(s.weight.x + kHigh, s.weight.y + kHigh);
  const float2 left = make_float2(T.x - (s.high.x - kHigh), T.y - (s.high.y - kHigh));      // exact
  const float2 low = fma2(T, g, left);
  s.low = make_float2(low.x + kLow, low.y + kLow);
  return s;
}

// A floor in the logits' type, for both halves of a word of 16-bit ones (to 2^-8 of it, where a hundredth would do).
template <int DT>
__device__ __forceinline__ unsigned int floor_word(float f) {
  if constexpr (DT == MCA_DTYPE_FP32) {
    return __float_as_uint(f);
  } else if constexpr (DT == MCA_DTYPE_BF16) {
    const __nv_bfloat162 h = __float2bfloat162_rn(f);
    return *reinterpret_cast<const unsigned int*>(&h);
  } else {
    const __half2 h = __float2half2_rn(f);
    return *reinterpret_cast<const unsigned int*>(&h);
  }
}
// A piece whose logits below `floor` (or NaN) count as that.
template <int DT>
__device__ __forceinline__ uint4 raised(uint4 q, unsigned int floor) {
  auto one = [&](unsigned int& w) {
    if constexpr (DT == MCA_DTYPE_FP32)
      w = __float_as_uint(fmaxf(__uint_as_float(w), __uint_as_float(floor)));
    else if constexpr (DT == MCA_DTYPE_BF16)
      asm("max.bf16x2 %0, %0, %1;" : "+r"(w) : "r"(floor));
    else
      asm("max.f16x2 %0, %0, %1;" : "+r"(w) : "r"(floor));
  };
  one(q.x);
  one(q.y);
  one(q.z);
  one(q.w);
  return q;
}

// Where a warp's weights come from: pieces of a row x, less those of y where RES.
template <int DT, bool RES>
struct Source {
  using P = Pieces<DT>;
  static constexpr int N = P::N;
  P row;
  const elem_t<DT>* y;
  const uint4* blocks;                      // y's 16-byte blocks: a piece's logits start `by` bytes behind one's start
  unsigned int by;
  Ref rx, ry;
  unsigned int fx, fy;                      // logits below count as these

  struct Raw {
    uint4 x, y, y1;
    bool whole;
  };

  __device__ __forceinline__ Source(const elem_t<DT>* x_, const elem_t<DT>* y_, int V) : row(x_, V), y(y_) {
    if (RES) {
      const uintptr_t from = reinterpret_cast<uintptr_t>(y - row.head);
      by = (unsigned int)(from & 15u);
      blocks = reinterpret_cast<const uint4*>(from - by);
    }
  }
  // Piece j on its way, and where it has come; -inf in the place of what is outside the row, or behind `end`.
  __device__ __forceinline__ Raw ask(int j, bool whole) const {
    Raw q;
    q.whole = whole;
    if (whole) {
      q.x = row.raw(j);
      if (RES) {
        q.y = blocks[j];
        if (by) q.y1 = blocks[j + 1];
      }
    }
    return q;
  }
  __device__ __forceinline__ void take(Raw& q, int j, int end) const {
    if (q.whole) {
      if (RES && by) q.y = shifted(q.y, q.y1, by);
    } else {
      const int at = j < end ? row.index(j, 0) : row.V;
      q.x = P::part(row.x, row.V, at);
      if (RES) q.y = P::part(y, row.V, at);
    }
  }
  // What is in the row of the 4 kB (kFetch pieces) from piece j on, to L2.
  __device__ __forceinline__ void fetch(int j, int end) const {
    const int k = j + (int)(threadIdx.x & 31) * 8;
    if (k < end && row.whole(k)) {
      asm volatile("prefetch.global.L2 [%0];" ::"l"(row.pieces() + k));
      if (RES) asm volatile("prefetch.global.L2 [%0];" ::"l"(blocks + k));
    }
  }
  template <class Span>
  __device__ __forceinline__ void fetch_first(const Span& s) const {
    fetch(s.from, s.to);
    fetch(s.from + kFetch, s.to);
  }
  // A piece's weights in steps: each(place, the bits of two).
  template <class Each>
  __device__ __forceinline__ void weights(const Raw& q, const Table& t, Each each) const {
    float v[N], w[N];
    P::values(raised<DT>(q.x, fx), v);
    if (RES) P::values(raised<DT>(q.y, fy), w);
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const Steps a = steps_of_exp<false>(make_float2(v[i], v[i + 1]), rx, t);
      unsigned int hx = __float_as_uint(a.high.x), hy = __float_as_uint(a.high.y);
      unsigned int lx = __float_as_uint(a.low.x), ly = __float_as_uint(a.low.y);
      if (RES) {
        // the larger weight of two that have the same digits in fp32 has the larger low part
        const Steps b = steps_of_exp<true>(make_float2(w[i], w[i + 1]), ry, t);
        const bool mx = a.weight.x > b.weight.x || (a.weight.x == b.weight.x && a.low.x > b.low.x);
        const bool my = a.weight.y > b.weight.y || (a.weight.y == b.weight.y && a.low.y > b.low.y);
        hx = mx ? hx - __float_as_uint(b.high.x) : 0u;
        lx = mx ? lx - __float_as_uint(b.low.x) : 0u;
        hy = my ? hy - __float_as_uint(b.high.y) : 0u;
        ly = my ? ly - __float_as_uint(b.low.y) : 0u;
      }
      each(i, hx, lx, hy, ly);
    }
  }
  static __device__ __forceinline__ long long steps(unsigned int high, unsigned int low, int n) {
    if (!RES) {
      high -= n * kHighBits;
      low -= n * kLowBits;
    }
    return ((long long)(int)high << kHighShift) + (int)low;
  }
  __device__ __forceinline__ long long sum(const Raw& q, const Table& t) const {
    unsigned int high = 0u, low = 0u;
    weights(q, t, [&](int, unsigned int hx, unsigned int lx, unsigned int hy, unsigned int ly) {
      high += hx + hy;
      low += lx + ly;
    });
    return steps(high, low, N);
  }
};

// ln(n 2^(l / kPowerCount - kUnitBits)), n > 0, as a pair to 2^-40, without the divisions and long polynomials of 64 bits,
// whose units are few (20000 x 10 took 57 us with log() of 64 bits, 35 so): n = 2^k m, m near the T of the table's place j,
// and ln m = j ln2 / 128 - (T's own logarithm) + ln(1 + d), d = (m - T) / T below 2^-7.
__device__ __forceinline__ float2 ln_pair(long long n, int l, const Table& table) {
  const int k = 63 - __clzll(n);
  const unsigned long long m = (unsigned long long)n << (63 - k);                    // 1.63 bits
  const float high = (float)(unsigned int)(m >> 40) * 0x1p-23f;                      // [1, 2) by 24 bits, and the rest
  const float low = (float)(unsigned int)(m >> 8 & 0xffffffffu) * 0x1p-55f;
  int j = (int)(log2f(high) * kPowerCount);
  j = min(max(j, 0), kPowerCount - 1);
  const float2 t = table[j][0];
  const float num = (high - t.x) + low, inv = 1.0f / t.x;                            // high - t.x is exact
  float d = num * inv;
  float rest = fmaf(-d, t.x, high - t.x) + low;                                      // what the quotient leaves
  rest = fmaf(rest, inv, -t.y);
  const float d2 = d * d;
  rest += d2 * fmaf(d, fmaf(d, fmaf(d, 0.2f, -0.25f), 1.0f / 3.0f), -0.5f);
  const float steps = (float)(l + (k - kUnitBits) * kPowerCount + j);                 // below 2^24
  const float a = steps * kStep, ae = fmaf(steps, kStep, -a) + steps * kStepLow;
  const float s = a + d, back = s - a;                                               // a + d, whichever is larger
  return make_float2(s, (a - (s - back)) + (d - back) + ae + rest);
}

template <class T>
__device__ __forceinline__ T warp_add(T v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float warp_max_nan(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = max_nan(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
template <class T>
__device__ __forceinline__ T warp_scan(T v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T below = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += below;
  }
  return v;
}

__device__ __forceinline__ int log2_of(int power) { return 31 - __clz(power); }

// A warp's part of a row: pieces from .. to, lane by lane; its sums after each of kGroups groups of rounds stay in `kept`.
struct Span {
  int from, to, rounds, group, first, whole;           // of which `whole` pieces from `first` on are, of both rows
  // Part `part` of 2^shift.
  template <int DT, bool RES>
  __device__ __forceinline__ Span(const Source<DT, RES>& src, int part, int shift)
      : from((int)((int64_t)src.row.count * part >> shift)), to((int)((int64_t)src.row.count * (part + 1) >> shift)),
        rounds((to - from + 31) / 32), group(max(1, (rounds + kGroups - 1) / kGroups)) {
    const Pieces<DT>& row = src.row;
    int lo = row.whole(0) ? 0 : 1, hi = row.count - (row.whole(row.count - 1) ? 0 : 1);
    if (RES) {
      lo = max(lo, first_of_own_blocks(row.head, (int)src.by, (int)sizeof(elem_t<DT>)));
      hi = min(hi, end_of_own_blocks(row.V, row.head, (int)src.by, (int)sizeof(elem_t<DT>)));
    }
    first = max(from, lo);
    whole = max(0, min(to, hi) - first);
  }
  __device__ __forceinline__ bool is_whole(int j) const { return (unsigned int)(j - first) < (unsigned int)whole; }
};
using Kept = long long[kGroups][32];

// The sum of a span's weights; all: a lane's own so far. before(piece, groups that are complete) at each round.
template <int DT, bool RES, class Before>
__device__ __forceinline__ long long sum_span(const Source<DT, RES>& src, const Span& s, const Table& table, Kept& kept,
                                              long long& all, Before before) {
  const int lane = threadIdx.x & 31;
  int left = s.group, g = 0;
  all = 0;
  auto next = src.ask(s.from + lane, s.is_whole(s.from + lane));
  for (int i = 0; i < s.rounds; ++i) {
    const int j = s.from + 32 * i + lane;
    auto q = next;
    next = src.ask(j + 32, s.is_whole(j + 32));
    if (i % (kFetch / 32) == 0) src.fetch(s.from + 32 * i + 2 * kFetch, s.to);
    src.take(q, j, s.to);
    before(q, g);
    all += src.sum(q, table);
    if (--left == 0) {
      kept[g++][lane] = all;
      left = s.group;
    }
  }
  for (; g < kGroups; ++g) kept[g][lane] = all;
  __syncwarp();
  return warp_add(all);
}

// The steps of a lane's piece, one by one, and their sum.
template <int DT, bool RES>
__device__ __forceinline__ long long steps_of(const Source<DT, RES>& src, const typename Source<DT, RES>::Raw& q,
                                              const Table& table, long long (&each)[Source<DT, RES>::N]) {
  long long sum = 0;
  src.weights(q, table, [&](int k, unsigned int hx, unsigned int lx, unsigned int hy, unsigned int ly) {
    each[k] = src.steps(hx, lx, 1);
    each[k + 1] = src.steps(hy, ly, 1);
    sum += each[k] + each[k + 1];
  });
  return sum;
}
// The symbol where a cumulative sum passes t, of pieces j of all lanes whose steps are `each` and whose sums end at `end`;
// the last one with a weight where none passes. here, some: lanes whose piece passes, or has a weight (one at least).
template <int DT, bool RES, int N>
__device__ __forceinline__ int symbol_at(const Source<DT, RES>& src, int j, const long long (&each)[N], long long sum,
                                         long long end, long long t, unsigned int here, unsigned int some) {
  long long at = end - sum;
  int k = -1, last = 0;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    at += each[e];
    if (each[e] > 0) last = e;
    if (k < 0 && each[e] > 0 && at > t) k = e;
  }
  return __shfl_sync(0xffffffffu, src.row.index(j, k < 0 ? last : k), here ? __ffs(here) - 1 : 31 - __clz(some));
}

// The symbol where a span's cumulative sum passes t, by its warp; the last one with a weight where shifts keep it below; -1
// if the group that t lies in was added up in steps so much finer than the last ones that in these it has no weight.
template <int DT, bool RES>
__device__ __noinline__ int find_in_span(Source<DT, RES> src, Span s, const Table& table, const Kept& kept, long long t) {
  constexpr int N = Source<DT, RES>::N, kEach = 32 / kGroups;
  const int lane = threadIdx.x & 31;
  long long c = 0;                           // kEach lanes add up a group's 32 sums
#pragma unroll
  for (int i = 0; i < kGroups; ++i) c += kept[lane / kEach][lane % kEach + kEach * i];
#pragma unroll
  for (int o = kEach / 2; o > 0; o >>= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
  const long long all = __shfl_sync(0xffffffffu, c, 31);
  const unsigned int over = __ballot_sync(0xffffffffu, all > t ? c > t : c == all);
  const int g = (__ffs(over) - 1) / kEach;
  long long before = __shfl_sync(0xffffffffu, c, max(kEach * g - 1, 0));
  if (g == 0) before = 0;
  int token = -1;
  const int i0 = g * s.group, i1 = min(i0 + s.group, s.rounds);
  auto next = src.ask(s.from + 32 * i0 + lane, s.is_whole(s.from + 32 * i0 + lane));
  for (int i = i0; i < i1; ++i) {
    const int j = s.from + 32 * i + lane;
    auto q = next;
    next = src.ask(j + 32, s.is_whole(j + 32));
    src.take(q, j, s.to);
    long long each[N];
    const long long mine = steps_of(src, q, table, each), end = before + warp_scan(mine);
    const unsigned int some = __ballot_sync(0xffffffffu, mine > 0);
    const unsigned int here = __ballot_sync(0xffffffffu, mine > 0 && end > t);
    before = __shfl_sync(0xffffffffu, end, 31);
    if (!some) continue;
    token = symbol_at(src, j, each, mine, end, t, here, some);
    if (here) break;
  }
  return token;
}

// ------------------------------------------------------------------------------------------------
// By the definition, in 64 bits, by a team of W warps: rows out of the pairs' range.
// ------------------------------------------------------------------------------------------------
template <int W>
__device__ __forceinline__ void sync_warps() {
  __syncwarp();
  if constexpr (W == kWarps)
    __syncthreads();
  else if constexpr (W > 1)
    asm volatile("bar.sync %0, %1;" ::"r"((int)threadIdx.x / (32 * W) + 1), "n"(32 * W) : "memory");
}

// Weights of a row: exp(x - lx), less exp(y - ly) where y is a row too.
template <int DT>
struct Weights {
  const elem_t<DT>* x;
  const elem_t<DT>* y;
  double lx, ly;
  static __device__ __forceinline__ double one(elem_t<DT> v, double l) {
    const float f = elem_f32(v);
    return f == -INFINITY ? 0.0 : exp((double)f - l);
  }
  __device__ __forceinline__ double of(int64_t v) const {
    const double p = one(x[v], lx);
    if (!y) return p;
    const double d = p - one(y[v], ly);
    return d <= 0.0 ? 0.0 : d;              // NaN stays
  }
};

struct ExactShared {
  double part[kWarps];
  int token[kWarps];
};

// (the symbol that u draws or -1, the sum of the weights); of weights that are all 0 the first net's alone.
template <int DT, int W>
__device__ __noinline__ int exact_draw(Weights<DT> w, int V, float u, double& total, ExactShared& s) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, first = warp / W * W;
  const int each = ((V + W - 1) / W + 31) / 32 * 32;
  const int64_t lo = (int64_t)(warp - first) * each, hi = min(lo + each, (int64_t)V);
  for (;;) {
    double sum = 0.0;
    for (int64_t v = lo + lane; v < hi; v += 32) sum += w.of(v);
    sum = warp_add(sum);
    sync_warps<W>();                         // (the sums of a round before are read)
    if (lane == 0) s.part[warp] = sum;
    sync_warps<W>();
    total = 0.0;
    for (int q = 0; q < W; ++q) total += s.part[first + q];
    if (total != 0.0 || !w.y) break;
    w.y = nullptr;
  }
  if (!(total > 0.0) || !(total < INFINITY) || u != u) return -1;
  const double t = fmax((double)u, 0.0) * total;
  double before = 0.0, sum = 0.0;
  int at = -1;
  for (int q = 0; q < W; ++q) {              // the first whose end is above t, or the last with weights
    if (!(s.part[first + q] > 0.0)) continue;
    at = q;
    before = sum;
    sum += s.part[first + q];
    if (sum > t) break;
  }
  if (warp - first == at) {
    int token = -1;
    for (int64_t b = lo; b < hi; b += 32) {
      const double mine = b + lane < hi ? w.of(b + lane) : 0.0, c = before + warp_scan(mine);
      const unsigned int some = __ballot_sync(0xffffffffu, mine > 0.0);
      const unsigned int over = __ballot_sync(0xffffffffu, mine > 0.0 && c > t);
      if (some) token = (int)b + 31 - __clz(some);
      if (over) {
        token = (int)b + __ffs(over) - 1;
        break;
      }
      before = __shfl_sync(0xffffffffu, c, 31);
    }
    if (lane == 0) s.token[first] = token;
  }
  sync_warps<W>();
  return s.token[first];
}

// ------------------------------------------------------------------------------------------------
// W warps have a row, kWarps / W rows a CTA; or the CTAs of a cluster have one.
// ------------------------------------------------------------------------------------------------

// What a warp, or a CTA, has seen of a row: a sum in steps of 2^(l / kPowerCount - kUnitBits), and whether it holds what goes
// by the definition.
struct Seen {
  long long total;
  int l;                                     // a multiple of kPowerCount; kNothing: none
  int bad;
};
constexpr int kNothing = -0x7fffffff - 1;

__device__ __forceinline__ long long steps_at(const Seen& s, int l) {
  if (s.l == kNothing) return 0;
  const int by = (l - s.l) >> kPowerBits;
  return by > 62 ? 0 : s.total >> by;
}

// The sum of what the lanes with `some` have seen; before: of those below this lane's.
__device__ __forceinline__ Seen join_lanes(const Seen& mine, bool some, long long& before) {
  Seen o;
  o.l = __reduce_max_sync(0xffffffffu, some ? mine.l : kNothing);
  o.bad = __any_sync(0xffffffffu, some && mine.bad);
  const long long v = some ? steps_at(mine, o.l) : 0, end = warp_scan(v);
  before = end - v;
  o.total = __shfl_sync(0xffffffffu, end, 31);
  return o;
}

struct Shared {
  Table table;
  Kept kept[kWarps];
  Seen warp[kWarps], cta[kMaxCluster];
  ExactShared exact;
};

// The integer below u total, u in [kLeastU, 1): exactly, so that borders are met where sums are even.
__device__ __forceinline__ long long part_of(long long total, float u) {
  if (!(u >= kLeastU && u < 1.0f)) return 0;
  const unsigned int b = __float_as_uint(u), shift = 150u - (b >> 23);              // 24..47
  const unsigned long long m = (b & 0x7fffffu) | 0x800000u, n = (unsigned long long)total;
  return (long long)(__umul64hi(n, m) << (64u - shift) | n * m >> shift);
}

// A row of one piece to a lane, by a warp: its steps are known when its sum is. Returns the sum; token where it is not 0.
template <int DT, bool RES>
__device__ __forceinline__ long long draw_round(const Source<DT, RES>& src, const typename Source<DT, RES>::Raw& q,
                                                const Table& table, float u, int& token) {
  long long each[Source<DT, RES>::N];
  const long long sum = steps_of(src, q, table, each), end = warp_scan(sum), total = __shfl_sync(0xffffffffu, end, 31);
  const long long t = part_of(total, u);
  const unsigned int here = __ballot_sync(0xffffffffu, sum > 0 && end > t);
  if (here) token = symbol_at(src, threadIdx.x & 31, each, sum, end, t, here, here);
  return total;
}

// The whole row's sum from its warps'; for the warp that u draws from: t, in its own steps, else -1.
template <int W>
__device__ __forceinline__ Seen join_row(const Seen& mine, Shared& s, int split, int rank, float u, long long& t) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, first = warp / W * W;
  if (W == 1) {
    t = mine.total > 0 ? part_of(mine.total, u) : -1;
    return mine;
  }
  if (lane == 0) s.warp[warp] = mine;
  sync_warps<W>();
  long long before, base = 0;
  const Seen w = s.warp[first + lane % W];
  const Seen cta = join_lanes(w, lane < W, before);
  Seen row = cta;
  int mine_of = rank;                        // the CTA that t lies in
  t = -1;
  if (W == kWarps && split > 1) {
    if (threadIdx.x < split) {
      unsigned int to;
      asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                   : "=r"(to) : "r"((unsigned int)__cvta_generic_to_shared(&s.cta[rank])), "r"(threadIdx.x));
      asm volatile("st.shared::cluster.u64 [%0], %1;\n\tst.shared::cluster.v2.u32 [%0 + 8], {%2, %3};"
                   ::"r"(to), "l"(cta.total), "r"(cta.l), "r"(cta.bad) : "memory");
    }
    cluster_arrive();
    cluster_wait();
    row = join_lanes(s.cta[lane % kMaxCluster], lane < split, base);
  }
  if (row.total <= 0) return row;
  long long at = part_of(row.total, u);
  if (W == kWarps && split > 1) {
    // the first CTA whose end is above; there is one, u being below 1
    const long long end = base + (lane < split ? steps_at(s.cta[lane % kMaxCluster], row.l) : 0);
    const unsigned int over = __ballot_sync(0xffffffffu, lane < split && end > at);
    mine_of = __ffs(over) - 1;
    at -= __shfl_sync(0xffffffffu, base, mine_of < 0 ? 0 : mine_of);
  }
  if (mine_of != rank) return row;
  // and its warp: where roundings leave none, the last with weights
  const long long v = lane < W ? steps_at(w, row.l) : 0, end = warp_scan(v);
  const unsigned int over = __ballot_sync(0xffffffffu, v > 0 && end > at), some = __ballot_sync(0xffffffffu, v > 0);
  if (!some) return row;
  const int owner = over ? __ffs(over) - 1 : 31 - __clz(some);
  if (owner != warp - first) return row;
  t = max(0ll, at - __shfl_sync(0xffffffffu, end - v, owner)) << ((row.l - mine.l) >> kPowerBits);
  return row;
}

// ROUND: every row is one of 32 pieces at most, and W = 1.
template <int DT, int W, bool ROUND>
__global__ void __launch_bounds__(kThreads, kCtas) sample_kernel(mca_sample_tokens_args a, int split) {
  using P = Pieces<DT>;
  __shared__ Shared s;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t r = W == kWarps ? (int64_t)blockIdx.x / split : (int64_t)blockIdx.x * (kWarps / W) + warp / W;
  const int rank = W == kWarps && split > 1 ? (int)cluster_rank() : 0;
  if (W == kWarps && split > 1) cluster_arrive();                // every CTA runs before one writes to another
  // (rows behind the last one: none is read)
  Source<DT, false> src(static_cast<const elem_t<DT>*>(a.logits) + min(r, a.rows - 1) * a.ld, nullptr, a.vocab);
  const P& row = src.row;
  const Span span(src, rank * W + warp % W, log2_of(W * split));
  typename Source<DT, false>::Raw only;
  if (ROUND)
    only = src.ask(lane, r < a.rows && span.is_whole(lane));
  else if (r < a.rows)
    src.fetch_first(span);
  fill_table(s.table);
  __syncthreads();
  if (W == kWarps && split > 1) cluster_wait();
  if (r >= a.rows) return;                                       // (whole teams)

  // The warp's sum relative to a power of two above its largest logit so far: a larger one shifts what there is.
  constexpr int kLowest = (int)(-kMaxRef * kLog2e);
  src.rx = {kLowest * kPowerCount, 0.0f, 0.0f};
  src.fx = floor_word<DT>(-kMaxRef - kFloor);
  float top = ((float)kLowest + 0.5f) * kLn2;
  Kept& kept = s.kept[warp];
  Seen mine{0, 0, 0};
  long long sum = 0;
  const float u = a.u[r];
  auto scale = [&](const auto& q, int g) {
    float m = largest<DT>(q.x);
    if (!__any_sync(0xffffffffu, !(m <= top))) return;
    m = warp_max_nan(m);
    if (!(m <= kMaxRef)) {
      mine.bad = 1;
      return;
    }
    const float power = rintf(m * kLog2e) + 1.0f;               // one more than now needed: most rows are raised once
    const int l = (int)power * kPowerCount, by = min((l - src.rx.l) >> kPowerBits, 63);
    sum >>= by;
    for (int i = 0; i < g; ++i) kept[i][lane] >>= by;
    src.rx.l = l;
    src.fx = floor_word<DT>(m - kFloor);
    top = (power + 0.5f) * kLn2;
  };
  int token = -1;
  long long t = -1;
  Seen all;
  if (ROUND) {
    src.take(only, lane, span.to);
    scale(only, 0);
    mine.total = draw_round(src, only, s.table, u, token);
    mine.l = src.rx.l;
    all = mine;
  } else {
    mine.total = sum_span(src, span, s.table, kept, sum, scale);
    mine.l = mine.total > 0 ? src.rx.l : kNothing;
    all = join_row<W>(mine, s, split, rank, u, t);
  }
  float2 lse = make_float2(NAN, 0.0f);
  if (all.bad || all.total <= 0 || a.vocab > kMaxVocab || !(u >= kLeastU && u < 1.0f)) {
    if (rank != 0) return;
    token = -1;
    float m = -INFINITY;
    for (int64_t v = threadIdx.x % (32 * W); v < a.vocab; v += 32 * W) m = max_nan(m, elem_f32(row.x[v]));
    m = warp_max_nan(m);
    if (lane == 0) s.exact.part[warp] = m;
    sync_warps<W>();
    m = -INFINITY;
    for (int q = 0; q < W; ++q) m = max_nan(m, (float)s.exact.part[warp / W * W + q]);
    if (m == -INFINITY) {
      lse.x = -INFINITY;
    } else if (m < INFINITY) {
      double total;
      token = exact_draw<DT, W>({row.x, nullptr, (double)m, 0.0}, a.vocab, u, total, s.exact);
      const double l = (double)m + log(total);
      lse = make_float2((float)l, (float)(l - (double)(float)l));
    }
    if (warp % W != 0) return;
  } else {
    if (!ROUND) {
      if (t < 0) return;
      token = find_in_span(src, span, s.table, kept, t);
      double total;                                              // (the whole row by the warp alone)
      if (token < 0)
        token = exact_draw<DT, 1>({row.x, nullptr, (double)all.l * kStepAll, 0.0}, a.vocab, u, total, s.exact);
    }
    lse = ln_pair(all.total, all.l, s.table);
  }
  if (lane != 0) return;
  a.token[r] = token;
  if (a.lse) a.lse[r] = lse.x + lse.y;
  if (a.logprob) {
    float lp = u != u ? NAN : lse.x;
    if (token >= 0) {
      const float x = elem_f32(row.x[token]), d = x - lse.x, back = d - x;
      lp = d + (((x - (d - back)) + (-lse.x - back)) - lse.y);                       // the difference, rounded once
    }
    a.logprob[r] = lp;
  }
}

// What the drafted symbols of a sequence decide, and the draw that follows.
struct Decision {
  int kept;                                  // symbols kept; -1: a length out of range
  bool all, broken;                          // the draw is from the last row; a number that decides is none
  float lx, ly;                              // log-sum-exps of the rows that the draw is from
  Ref rx, ry;
};

// One warp; lane i: symbol i. lp: its log probability.
template <int DT>
__device__ __forceinline__ Decision decide(const mca_verify_drafts_args& a, int64_t q, float& lp) {
  const int lane = threadIdx.x & 31;
  Decision d{};
  lp = NAN;
  // what does not depend on each other is asked for together
  const bool may = lane < a.drafts;
  const int n = a.lengths ? a.lengths[q] : a.drafts, t = may ? a.tokens[q * a.drafts + lane] : -1;
  const float u = may ? a.u[q * (a.drafts + 1) + lane] : 0.0f;
  const float target_lse = lane <= a.drafts ? a.target_lse[q * (a.drafts + 1) + lane] : 0.0f;
  const float draft_lse = may ? a.draft_lse[q * a.drafts + lane] : 0.0f;
  bool keep = false, broken = false, near = false;
  float xt = 0.0f, yt = 0.0f, lx = 0.0f, ly = 0.0f;
  if (n < 0 || n > a.drafts) {
    d.kept = -1;
    d.broken = true;
    return d;
  }
  if (lane < n) {
    if (t < 0 || t >= a.vocab) {
      broken = true;
    } else {
      const elem_t<DT>* x = static_cast<const elem_t<DT>*>(a.target) + q * a.target_seq + lane * a.target_pos;
      const elem_t<DT>* y = static_cast<const elem_t<DT>*>(a.draft) + q * a.draft_seq + lane * a.draft_pos;
      xt = elem_f32(x[t]);
      yt = elem_f32(y[t]);
      lx = xt == -INFINITY ? -INFINITY : xt - target_lse;
      ly = yt == -INFINITY ? -INFINITY : yt - draft_lse;
      broken = lx != lx || ly != ly || u != u;
      if (lx > -INFINITY) {
        // (expf and its argument are off by less than 2^-16 together for logits up to 2^6; next to u, where f has few
        // digits and for larger logits 64 bits)
        const float f = expf(lx - ly);
        keep = ly == -INFINITY || u < f;
        near = ly > -INFINITY && !(fabsf(u - f) > 0x1p-14f * f && f >= 0x1p-100f && fabsf(lx) < 64.0f && fabsf(ly) < 64.0f);
      }
    }
  }
  if (__any_sync(0xffffffffu, near) && near)
    keep = (double)u < exp(((double)xt - (double)target_lse) - ((double)yt - (double)draft_lse));
  const unsigned int stop = ~__ballot_sync(0xffffffffu, keep && !broken);
  d.kept = min(n, stop ? __ffs(stop) - 1 : 32);
  d.all = d.kept == n;
  const unsigned int wrong = __ballot_sync(0xffffffffu, broken);
  d.broken = !d.all && (wrong >> d.kept & 1u);
  lp = lx;
  if (d.broken) return d;
  d.lx = d.kept < 32 ? __shfl_sync(0xffffffffu, target_lse, d.kept) : a.target_lse[q * (a.drafts + 1) + 32];
  d.ly = d.all ? 0.0f : __shfl_sync(0xffffffffu, draft_lse, d.kept);
  if (fabsf(d.lx) <= kMaxRef && fabsf(d.ly) <= kMaxRef) {
    // all weights times exp(high + low) of the target's, so that its own exponentials need no shift
    d.rx.set((double)d.lx);
    const double shift = (double)d.lx - (double)d.rx.l * kStepAll;
    d.ry.set((double)d.ly - shift);
  }
  return d;
}

// The symbol after those that are kept: from the weights of both rows where RES, else from the target's.
template <int DT, int W, bool ROUND, bool RES>
__device__ __forceinline__ void draw_last(const mca_verify_drafts_args& a, int64_t q, const Decision& d, Shared& s,
                                          int split, int rank) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, k1 = a.drafts + 1;
  const elem_t<DT>* x = static_cast<const elem_t<DT>*>(a.target) + q * a.target_seq + d.kept * a.target_pos;
  const elem_t<DT>* y =
      RES ? static_cast<const elem_t<DT>*>(a.draft) + q * a.draft_seq + d.kept * a.draft_pos : nullptr;
  const float u = a.u[q * k1 + a.drafts], lx = d.lx, ly = d.ly;
  int token = -1;
  bool exact = !(fabsf(lx) <= kMaxRef && fabsf(ly) <= kMaxRef && u >= kLeastU && u < 1.0f && a.vocab <= kMaxVocab);
  if (!exact) {
    Source<DT, RES> src(x, y, a.vocab);
    src.rx = {d.rx.l, 0.0f, 0.0f};
    src.ry = d.ry;
    src.fx = floor_word<DT>(lx - kFloor);
    src.fy = floor_word<DT>(ly - kFloor);
    const Span span(src, rank * W + warp % W, log2_of(W * split));
    float mx = -INFINITY, my = -INFINITY;
    auto look = [&](const auto& p, int) {
      mx = max_nan(mx, largest<DT>(p.x));
      if (RES) my = max_nan(my, largest<DT>(p.y));
    };
    // Log-sum-exps that are not the rows', NaN, and rows that have nearly the same probabilities go by the definition.
    auto bad = [&] { return __any_sync(0xffffffffu, !(mx <= lx + 0.2f) || (RES && !(my <= ly + kFloor))); };
    constexpr long long kLeast = 1ll << (kUnitBits - 10);
    if (ROUND) {
      auto q = src.ask(lane, span.is_whole(lane));
      src.take(q, lane, span.to);
      look(q, 0);
      exact = draw_round(src, q, s.table, u, token) < kLeast || bad();
    } else {
      src.fetch_first(span);
      long long sum = 0, t;
      Seen mine{0, 0, 0};
      mine.total = sum_span(src, span, s.table, s.kept[warp], sum, look);
      mine.bad = bad();
      const Seen all = join_row<W>(mine, s, split, rank, u, t);
      exact = all.bad || all.total < kLeast;
      if (!exact) {
        if (t < 0) return;
        token = find_in_span(src, span, s.table, s.kept[warp], t);
      }
    }
  }
  if (exact) {
    if (rank != 0) return;
    double total;
    token = exact_draw<DT, W>({x, y, (double)lx, (double)ly}, a.vocab, u, total, s.exact);
    if (warp % W != 0) return;
  }
  if (lane != 0) return;
  a.out[q * k1 + d.kept] = token;
  if (a.logprob) a.logprob[q * k1 + d.kept] = token >= 0 ? elem_f32(x[token]) - lx : NAN;
}

template <int DT, int W, bool ROUND>
__global__ void __launch_bounds__(kThreads, kCtas) verify_kernel(mca_verify_drafts_args a, int split) {
  __shared__ Shared s;
  __shared__ Decision s_decision[kWarps / W];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, k1 = a.drafts + 1;
  const int64_t q = W == kWarps ? (int64_t)blockIdx.x / split : (int64_t)blockIdx.x * (kWarps / W) + warp / W;
  const int rank = W == kWarps && split > 1 ? (int)cluster_rank() : 0;
  if (W == kWarps && split > 1) cluster_arrive();                // every CTA runs before one writes to another
  if (warp % W == 0 && q < a.seqs) {
    float lp;
    const Decision d = decide<DT>(a, q, lp);
    if (lane == 0) s_decision[warp / W] = d;
    if (rank == 0) {                                             // all but the symbol that is drawn
      for (int i = lane; i < k1; i += 32) {
        if (i == d.kept && !d.broken) continue;
        a.out[q * k1 + i] = i < d.kept ? a.tokens[q * a.drafts + i] : -1;
        if (a.logprob) a.logprob[q * k1 + i] = d.kept < 0 || i == d.kept ? NAN : i < d.kept ? lp : 0.0f;
      }
      if (lane == 0) a.accepted[q] = d.kept;
    }
  }
  fill_table(s.table);
  __syncthreads();
  if (W == kWarps && split > 1) cluster_wait();
  if (q >= a.seqs) return;                                       // (whole teams)
  const Decision d = s_decision[warp / W];
  if (d.broken) return;
  if (d.all)
    draw_last<DT, W, ROUND, false>(a, q, d, s, split, rank);
  else
    draw_last<DT, W, ROUND, true>(a, q, d, s, split, rank);
}

// f(the shape's warps, and whether a row is a round, as types) with the launch that it says.
template <class F>
cudaError_t with_warps(const DrawShape& h, F f) {
  if (h.round) return f(std::integral_constant<int, 1>(), std::true_type());
  switch (h.warps) {
    case 1: return f(std::integral_constant<int, 1>(), std::false_type());
    case 2: return f(std::integral_constant<int, 2>(), std::false_type());
    case 4: return f(std::integral_constant<int, 4>(), std::false_type());
    default: return f(std::integral_constant<int, kWarps>(), std::false_type());
  }
}

template <int DT>
cudaError_t launch_sample(const mca_sample_tokens_args& a, cudaStream_t s) {
  const DrawShape h(a.rows, a.vocab, Pieces<DT>::N);
  return with_warps(h, [&](auto w, auto round) {
    return launch_clusters(sample_kernel<DT, decltype(w)::value, decltype(round)::value>, h.grid(a.rows), kThreads,
                           h.split, s, a, h.split);
  });
}

template <int DT>
cudaError_t launch_verify(const mca_verify_drafts_args& a, cudaStream_t s) {
  const DrawShape h(a.seqs, a.vocab, Pieces<DT>::N);
  return with_warps(h, [&](auto w, auto round) {
    return launch_clusters(verify_kernel<DT, decltype(w)::value, decltype(round)::value>, h.grid(a.seqs), kThreads,
                           h.split, s, a, h.split);
  });
}

}  // namespace

cudaError_t launch_sample_tokens(const mca_sample_tokens_args& a, cudaStream_t s) {
  if (a.dtype == MCA_DTYPE_FP32) return launch_sample<MCA_DTYPE_FP32>(a, s);
  if (a.dtype == MCA_DTYPE_FP16) return launch_sample<MCA_DTYPE_FP16>(a, s);
  return launch_sample<MCA_DTYPE_BF16>(a, s);
}

cudaError_t launch_verify_drafts(const mca_verify_drafts_args& a, cudaStream_t s) {
  if (a.dtype == MCA_DTYPE_FP32) return launch_verify<MCA_DTYPE_FP32>(a, s);
  if (a.dtype == MCA_DTYPE_FP16) return launch_verify<MCA_DTYPE_FP16>(a, s);
  return launch_verify<MCA_DTYPE_BF16>(a, s);
}

}  // namespace mca
