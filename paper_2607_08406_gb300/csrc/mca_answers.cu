// Entry points of a trained net's answers (include/mca.h): layers on 8-bit codes, log probabilities and their
// gradient, and the same from a handle's net (mca_predict) and samples (mca_score).
#include <algorithm>
#include <cstdarg>
#include <cstdio>
#include <cstdlib>

#include <nvtx3/nvToolsExt.h>

#include "mca_answers.h"
#include "mca_device.cuh"
#include "mca_internal.h"

namespace {

using mca::dtype_bytes;

mca_status fail(mca_handle* h, mca_status st, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  return mca::fail_message(h, st, buf);
}

mca_status launched(mca_handle* h, cudaError_t e, const char* what) {
  if (e == cudaSuccess) return MCA_OK;
  if (h && e != cudaErrorMemoryAllocation) h->broken = true;
  return fail(h, e == cudaErrorMemoryAllocation ? MCA_ERR_OOM : MCA_ERR_CUDA, "%s: %s", what,
              cudaGetErrorString(e));
}

// What a caller's array has to be: device memory of device dev, on its element's alignment.
struct Arg {
  const char* name;
  const void* p;
  size_t align;
  bool nullable;
};

mca_status check_pointers(mca_handle* h, const Arg* args, int n) {
  for (int q = 0; q < n; ++q) {
    if (!args[q].p && !args[q].nullable) return fail(h, MCA_ERR_INVALID, "%s is NULL", args[q].name);
    if (reinterpret_cast<uintptr_t>(args[q].p) % args[q].align)
      return fail(h, MCA_ERR_INVALID, "%s is not aligned to %zu bytes", args[q].name, args[q].align);
  }
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) {
    cudaGetLastError();
    return fail(h, MCA_ERR_INVALID, "no usable current device");
  }
  if (h && dev != h->device)
    return fail(h, MCA_ERR_INVALID, "current device %d is not the handle's device %d", dev, h->device);
  for (int q = 0; q < n; ++q) {
    if (!args[q].p) continue;
    cudaPointerAttributes at;
    if (cudaPointerGetAttributes(&at, args[q].p) != cudaSuccess) {
      cudaGetLastError();
      return fail(h, MCA_ERR_INVALID, "%s is no device pointer", args[q].name);
    }
    if (at.type == cudaMemoryTypeManaged) continue;
    if (at.type != cudaMemoryTypeDevice)
      return fail(h, MCA_ERR_INVALID, "%s is no device pointer", args[q].name);
    if (at.device != dev)
      return fail(h, MCA_ERR_INVALID, "%s is on device %d, current is %d", args[q].name, at.device,
                  dev);
  }
  return MCA_OK;
}

template <int N>
mca_status check_pointers(mca_handle* h, const Arg (&args)[N]) {
  return check_pointers(h, args, N);
}

constexpr int64_t kMaxRows = 0x7fffffff;     // rows of a call: a CTA each at least
constexpr int kMaxIn = 131071;               // codes of a sum: 128 * 128 * kMaxIn < 2^31

mca_status check_rows(mca_handle* h, int64_t rows) {
  if (rows < 0 || rows > kMaxRows)
    return fail(h, MCA_ERR_INVALID, "rows = %lld outside 0..2^31-1", (long long)rows);
  return MCA_OK;
}

mca_status check_matrix(mca_handle* h, const char* name, int64_t rows, int64_t cols, int64_t ld) {
  if (rows > 1 && ld < cols)
    return fail(h, MCA_ERR_INVALID, "%s: row distance %lld < %lld columns", name, (long long)ld,
                (long long)cols);
  if (rows > 1 && ld > (INT64_MAX / 8) / rows)
    return fail(h, MCA_ERR_INVALID, "%s: row distance %lld", name, (long long)ld);
  return MCA_OK;
}

mca_status check_dtype(int dtype) {
  if (dtype < MCA_DTYPE_FP32 || dtype > MCA_DTYPE_BF16)
    return fail(nullptr, MCA_ERR_INVALID, "unknown dtype %d", dtype);
  return MCA_OK;
}

#define MCA_CHECK(expr)                     \
  do {                                      \
    const mca_status rc_ = (expr);          \
    if (rc_ != MCA_OK) return rc_;          \
  } while (0)

// Bytes from the first to behind the last element.
size_t span_bytes(int64_t rows, int64_t cols, int64_t ld, size_t es) {
  return ((size_t)(rows - 1) * (size_t)(rows > 1 ? ld : 0) + (size_t)cols) * es;
}

bool overlap(const void* p, size_t np, const void* q, size_t nq) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return a < b + nq && b < a + np;
}

// The same for two matrices of one row distance: their rows may lie between each other's. Row i of the second starts
// delta + (i - j) ld bytes behind row j of the first, and only the two multiples of ld next to -delta can bring it
// near.
bool rows_overlap(const void* p, const void* q, int64_t rows, int64_t cols, int64_t ld, size_t es) {
  const int64_t delta = (int64_t)(reinterpret_cast<uintptr_t>(q) - reinterpret_cast<uintptr_t>(p));
  const int64_t width = cols * (int64_t)es, step = ld * (int64_t)es;
  for (int64_t k = delta / step - 1; k <= delta / step + 1; ++k)
    if (k > -rows && k < rows && std::llabs(delta - k * step) < width) return true;
  return false;
}

mca_status check_linear(const mca_code_linear_args* a) {
  if (!a) return fail(nullptr, MCA_ERR_INVALID, "NULL argument");
  MCA_CHECK(check_rows(nullptr, a->rows));
  if (a->n_in < 1 || a->n_in > kMaxIn)
    return fail(nullptr, MCA_ERR_INVALID, "n_in = %d outside 1..%d", a->n_in, kMaxIn);
  if (a->n_out < 1 || a->n_out > 1 << 30)
    return fail(nullptr, MCA_ERR_INVALID, "n_out = %d outside 1..2^30", a->n_out);
  MCA_CHECK(check_dtype(a->dtype));
  if (a->act < MCA_ACT_IDENTITY || a->act > MCA_ACT_GELU)
    return fail(nullptr, MCA_ERR_INVALID, "unknown transfer function %d", a->act);
  MCA_CHECK(check_matrix(nullptr, "x", a->rows, a->n_in, a->ldx));
  MCA_CHECK(check_matrix(nullptr, "w", a->n_out, a->n_in, a->ldw));
  return check_matrix(nullptr, "y", a->rows, a->n_out, a->ldy);
}

mca_status check_logprobs(const mca_token_logprobs_args& a, mca_handle* h) {
  if (a.top < 0 || a.top > mca::kMaxTop)
    return fail(h, MCA_ERR_INVALID, "top = %d outside 0..%d", a.top, mca::kMaxTop);
  if (a.top == 0 && (a.top_logprob || a.top_index))
    return fail(h, MCA_ERR_INVALID, "top = 0 with arrays for alternatives");
  if (a.logprob && !a.targets) return fail(h, MCA_ERR_INVALID, "logprob without targets");
  return check_pointers(h, {{"logits", a.logits, dtype_bytes(a.dtype), false},
                            {"targets", a.targets, 4, true},
                            {"logprob", a.logprob, 4, true},
                            {"entropy", a.entropy, 4, true},
                            {"lse", a.lse, 4, true},
                            {"top_logprob", a.top_logprob, 4, a.top == 0},
                            {"top_index", a.top_index, 4, a.top == 0}});
}

// ------------------------------------------------------------------------------------------------
// Logits of a handle's own samples.
// ------------------------------------------------------------------------------------------------

// MLP: output fields, [C x Np] field by field, to activations sample by sample.
__global__ void fields_logits_kernel(const float* __restrict__ z, int N, int Np, int C, int act,
                                     float g, float* __restrict__ logits) {
  const int n = blockIdx.x * blockDim.x + threadIdx.x;
  if (n >= N) return;
  for (int c = 0; c < C; ++c)
    logits[(size_t)n * C + c] = mca::act_call(act, z[(size_t)c * Np + n], g);
}

// Transformer: final layer norm and head of 32 positions per CTA (a lane each). The head's weights are read by all
// lanes at once, a word at a time, and come from L1: 0.27 GFLOP at the config shape, where a whole mca_score with five
// alternatives takes 79 us.
constexpr int kLogitRows = 32;
constexpr int kLogitThreads = 256;

__global__ void __launch_bounds__(kLogitThreads) tfm_logits_kernel(mca::TfmArgs a, int64_t rows,
                                                                   float* __restrict__ logits) {
  __shared__ float s_h[mca::kTfmMaxD][kLogitRows + 1];
  __shared__ float s_out[kLogitRows][mca::kTfmMaxV + 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, d = a.d, V = a.V;
  const int64_t r0 = (int64_t)blockIdx.x * kLogitRows;
  const int nr = (int)min((int64_t)kLogitRows, rows - r0);
  const float* x = a.X + ((size_t)a.nL * (size_t)rows + (size_t)r0) * d;
  for (int t = warp; t < kLogitRows; t += kLogitThreads / 32) {
    float v[mca::kTfmMaxD / 32], s = 0.0f, q = 0.0f;
#pragma unroll
    for (int i = 0; i < mca::kTfmMaxD / 32; ++i) {
      const int c = lane + 32 * i;
      v[i] = t < nr && c < d ? x[t * d + c] : 0.0f;
      s += v[i];
    }
    const float mean = mca::warp_sum(s) / (float)d;
#pragma unroll
    for (int i = 0; i < mca::kTfmMaxD / 32; ++i) {
      const float e = lane + 32 * i < d ? v[i] - mean : 0.0f;
      q = fmaf(e, e, q);
    }
    const float rstd = rsqrtf(mca::warp_sum(q) / (float)d + a.eps);
#pragma unroll
    for (int i = 0; i < mca::kTfmMaxD / 32; ++i) {
      const int c = lane + 32 * i;
      if (c < d) s_h[c][t] = (v[i] - mean) * rstd * a.params[a.o_lnf_g + c] + a.params[a.o_lnf_b + c];
    }
  }
  __syncthreads();
  for (int v0 = 4 * warp; v0 < V; v0 += 4 * (kLogitThreads / 32)) {
    const float* w[4];
    float acc[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int v = min(v0 + j, V - 1);
      w[j] = a.params + a.o_wh + (size_t)v * d;
      acc[j] = 0.0f;
    }
    for (int c = 0; c < d; ++c) {
      const float hv = s_h[c][lane];
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] = fmaf(hv, __ldg(w[j] + c), acc[j]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (v0 + j < V) s_out[lane][v0 + j] = acc[j] + a.params[a.o_bh + v0 + j];
  }
  __syncthreads();
  for (int e = threadIdx.x; e < nr * V; e += kLogitThreads)
    logits[(size_t)r0 * V + e] = s_out[e / V][e % V];
}

// ------------------------------------------------------------------------------------------------
// mca_predict's workspace.
// ------------------------------------------------------------------------------------------------
size_t align256(size_t x) { return (x + 255) & ~size_t(255); }
int64_t round16(int64_t x) { return (x + 15) / 16 * 16; }

// Samples that go through the layers together: their codes and activations (at most 32M of each) stay in L2 from
// one layer to the next, and give the wide layers' products some thousand tiles.
constexpr int64_t kPredictElems = 32 << 20;

struct PredictPlan {
  int64_t chunk, width;           // samples per pass; the widest layer input or output
  size_t codes, scale, hidden, w, w_scale, product, total;   // offsets
};

PredictPlan predict_plan(const mca_handle* h, int64_t n) {
  PredictPlan p{};
  size_t wb = 0, outs = 0;
  for (const mca_layer& L : h->layers) {
    p.width = std::max({p.width, round16(L.n_in), round16(L.n_out)});
    wb += align256((size_t)round16(L.n_in) * (size_t)L.n_out);
    outs += (size_t)L.n_out;
  }
  p.chunk = std::max<int64_t>(1, std::min(n, std::max<int64_t>(256, kPredictElems / p.width / 256 * 256)));
  const size_t e = (size_t)p.chunk * (size_t)p.width;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += align256(bytes);
    return o;
  };
  p.codes = take(e);
  p.scale = take(4 * (size_t)p.chunk);
  p.hidden = take(4 * e);
  p.w = take(wb);
  p.w_scale = take(4 * outs);
  size_t product = 0;
  for (const mca_layer& L : h->layers) {
    for (const int64_t rows : {p.chunk, n % p.chunk}) {        // every pass, and the last one
      if (rows == 0) continue;
      mca_code_linear_args a{};
      a.rows = rows;
      a.n_in = L.n_in;
      a.n_out = L.n_out;
      a.ldx = a.ldw = round16(L.n_in);
      product = std::max(product, mca::code_linear_workspace(a));
    }
  }
  p.product = take(product);
  p.total = at;
  return p;
}

bool bounded_by_one(const mca_layer& L) {
  return L.act == MCA_ACT_TANH || L.act == MCA_ACT_SIGMOID ||
         (L.act == MCA_ACT_GAUSSIAN && L.act_param >= 0.0f);
}

mca_status check_predict(mca_handle* h, int64_t n) {
  if (!h) return fail(nullptr, MCA_ERR_INVALID, "NULL handle");
  if (h->tfm) return fail(h, MCA_ERR_UNSUPPORTED, "answers in 8-bit layers are for MLP handles");
  for (const mca_layer& L : h->layers)
    if (L.n_in > kMaxIn || L.n_out > 1 << 30)
      return fail(h, MCA_ERR_UNSUPPORTED, "a layer of %d inputs and %d outputs: more than %d and 2^30 in 8 bits",
                  L.n_in, L.n_out, kMaxIn);
  return check_rows(h, n);
}

}  // namespace

extern "C" {

mca_status mca_quantize_rows(const void* x, int32_t dtype, int64_t rows, int64_t cols, int64_t ldx,
                             int8_t* codes, int64_t ldc, float* scale, void* stream) {
  MCA_CHECK(check_dtype(dtype));
  MCA_CHECK(check_rows(nullptr, rows));
  if (cols < 1 || cols > 0x7fffffff)
    return fail(nullptr, MCA_ERR_INVALID, "cols = %lld outside 1..2^31-1", (long long)cols);
  MCA_CHECK(check_matrix(nullptr, "x", rows, cols, ldx));
  MCA_CHECK(check_matrix(nullptr, "codes", rows, cols, ldc));
  if (rows == 0) return MCA_OK;
  MCA_CHECK(check_pointers(nullptr, {{"x", x, dtype_bytes(dtype), false},
                                     {"codes", codes, 1, false},
                                     {"scale", scale, 4, false}}));
  return launched(nullptr,
                  mca::launch_quantize_rows(x, dtype, rows, cols, ldx, codes, ldc, scale,
                                            (cudaStream_t)stream),
                  "mca_quantize_rows");
}

mca_status mca_code_linear_workspace_size(const mca_code_linear_args* a, size_t* bytes) {
  MCA_CHECK(check_linear(a));
  if (!bytes) return fail(nullptr, MCA_ERR_INVALID, "bytes is NULL");
  *bytes = a->rows ? mca::code_linear_workspace(*a) : 0;
  return MCA_OK;
}

mca_status mca_code_linear(const mca_code_linear_args* a) {
  MCA_CHECK(check_linear(a));
  if (a->rows == 0) return MCA_OK;
  const size_t need = mca::code_linear_workspace(*a);
  if (need && (!a->workspace || a->workspace_bytes < need))
    return fail(nullptr, MCA_ERR_OOM, "workspace of %zu bytes, needs %zu",
                a->workspace ? a->workspace_bytes : (size_t)0, need);
  MCA_CHECK(check_pointers(nullptr, {{"x", a->x, 1, false},
                                     {"x_scale", a->x_scale, 4, false},
                                     {"w", a->w, 1, false},
                                     {"w_scale", a->w_scale, 4, false},
                                     {"bias", a->bias, 4, true},
                                     {"y", a->y, dtype_bytes(a->dtype), false},
                                     {"workspace", need ? a->workspace : nullptr, 256, true}}));
  return launched(nullptr, mca::launch_code_linear(*a, (cudaStream_t)a->stream), "mca_code_linear");
}

mca_status mca_token_logprobs(const mca_token_logprobs_args* a) {
  if (!a) return fail(nullptr, MCA_ERR_INVALID, "NULL argument");
  MCA_CHECK(check_dtype(a->dtype));
  MCA_CHECK(check_rows(nullptr, a->rows));
  if (a->vocab < 1 || a->vocab > 1 << 30)
    return fail(nullptr, MCA_ERR_INVALID, "vocab = %d outside 1..2^30", a->vocab);
  MCA_CHECK(check_matrix(nullptr, "logits", a->rows, a->vocab, a->ld));
  if (a->rows == 0) return MCA_OK;
  MCA_CHECK(check_logprobs(*a, nullptr));
  mca::LogprobArgs p{*a, a->rows, 0};
  return launched(nullptr, mca::launch_logprobs(p, (cudaStream_t)a->stream), "mca_token_logprobs");
}

mca_status mca_token_logprobs_backward(const mca_token_logprobs_backward_args* a) {
  if (!a) return fail(nullptr, MCA_ERR_INVALID, "NULL argument");
  MCA_CHECK(check_dtype(a->dtype));
  MCA_CHECK(check_rows(nullptr, a->rows));
  if (a->vocab < 1 || a->vocab > 1 << 30)
    return fail(nullptr, MCA_ERR_INVALID, "vocab = %d outside 1..2^30", a->vocab);
  MCA_CHECK(check_matrix(nullptr, "logits", a->rows, a->vocab, a->ld));
  MCA_CHECK(check_matrix(nullptr, "grad", a->rows, a->vocab, a->ldg));
  if (a->rows == 0) return MCA_OK;
  if (!a->g_logprob && !a->g_entropy)
    return fail(nullptr, MCA_ERR_INVALID, "neither g_logprob nor g_entropy");
  if (a->g_logprob && !a->targets)
    return fail(nullptr, MCA_ERR_INVALID, "g_logprob without targets");
  if (a->g_entropy && !a->entropy)
    return fail(nullptr, MCA_ERR_INVALID, "g_entropy without entropy");
  const size_t es = dtype_bytes(a->dtype);
  MCA_CHECK(check_pointers(nullptr, {{"logits", a->logits, es, false},
                                     {"targets", a->targets, 4, true},
                                     {"lse", a->lse, 4, false},
                                     {"entropy", a->entropy, 4, true},
                                     {"g_logprob", a->g_logprob, 4, true},
                                     {"g_entropy", a->g_entropy, 4, true},
                                     {"grad", a->grad, es, false}}));
  const int64_t ld = a->rows > 1 ? a->ld : a->vocab, ldg = a->rows > 1 ? a->ldg : a->vocab;
  if (!(a->grad == a->logits && ld == ldg) &&
      overlap(a->logits, span_bytes(a->rows, a->vocab, ld, es), a->grad,
              span_bytes(a->rows, a->vocab, ldg, es)) &&
      (ld != ldg || rows_overlap(a->logits, a->grad, a->rows, a->vocab, ld, es)))
    return fail(nullptr, MCA_ERR_INVALID, "grad overlaps the logits but is not the same matrix");
  return launched(nullptr, mca::launch_logprobs_backward(*a, (cudaStream_t)a->stream),
                  "mca_token_logprobs_backward");
}

mca_status mca_score(mca_handle* h, float* logits, int32_t top, float* logprob, float* entropy,
                     float* lse, float* top_logprob, int32_t* top_index) {
  if (!h) return fail(nullptr, MCA_ERR_INVALID, "NULL handle");
  if (h->broken) return fail(h, MCA_ERR_CUDA, "handle unusable after an earlier device error");
  if (!h->tfm && h->loss != MCA_LOSS_SOFTMAX_CE)
    return fail(h, MCA_ERR_UNSUPPORTED, "the handle's loss is not softmax_ce: no log probabilities");
  mca::LogprobArgs p{};
  p.a.logits = logits;
  p.a.dtype = MCA_DTYPE_FP32;
  p.a.rows = h->N;
  p.a.vocab = h->tfm ? h->tspec.vocab : h->C;
  p.a.ld = p.a.vocab;
  p.a.targets = h->tfm ? h->tokens + 1 : h->y;
  p.a.logprob = logprob;
  p.a.entropy = entropy;
  p.a.lse = lse;
  p.a.top = top;
  p.a.top_logprob = top_logprob;
  p.a.top_index = top_index;
  p.period = h->tfm ? h->tspec.ctx : h->N;
  p.pitch = h->tfm ? h->tspec.ctx + 1 : 0;
  MCA_CHECK(check_logprobs(p.a, h));
  nvtxRangePushA("mca_score");
  if (h->tfm) {
    tfm_logits_kernel<<<(unsigned int)((h->N + kLogitRows - 1) / kLogitRows), kLogitThreads, 0,
                        h->stream>>>(mca::handle_tfm_args(h), h->N, logits);
  } else {
    const mca_layer& L = h->layers.back();
    fields_logits_kernel<<<(unsigned int)((h->N + 255) / 256), 256, 0, h->stream>>>(
        h->deep ? h->Z.back() : h->srec, (int)h->N, h->Np, h->C, L.act, L.act_param, logits);
  }
  cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess) e = mca::launch_logprobs(p, h->stream);
  nvtxRangePop();
  h->launches += 2;
  return launched(h, e, "mca_score");
}

mca_status mca_predict_workspace_size(mca_handle* h, int64_t n, size_t* bytes) {
  MCA_CHECK(check_predict(h, n));
  if (!bytes) return fail(h, MCA_ERR_INVALID, "bytes is NULL");
  *bytes = n ? predict_plan(h, n).total : 0;
  return MCA_OK;
}

mca_status mca_predict(mca_handle* h, const float* x, int64_t n, int64_t ldx, float* out,
                       void* workspace, size_t workspace_bytes) {
  MCA_CHECK(check_predict(h, n));
  if (h->broken) return fail(h, MCA_ERR_CUDA, "handle unusable after an earlier device error");
  MCA_CHECK(check_matrix(h, "x", n, h->D, ldx));
  if (n == 0) return MCA_OK;
  const PredictPlan p = predict_plan(h, n);
  if (!workspace || workspace_bytes < p.total)
    return fail(h, MCA_ERR_OOM, "workspace of %zu bytes, needs %zu", workspace ? workspace_bytes : 0,
                p.total);
  MCA_CHECK(check_pointers(h, {{"x", x, 4, false}, {"out", out, 4, false},
                               {"workspace", workspace, 256, false}}));
  nvtxRangePushA("mca_predict");
  char* ws = static_cast<char*>(workspace);
  int8_t* codes = reinterpret_cast<int8_t*>(ws + p.codes);
  float* scale = reinterpret_cast<float*>(ws + p.scale);
  int8_t* w = reinterpret_cast<int8_t*>(ws + p.w);
  float* w_scale = reinterpret_cast<float*>(ws + p.w_scale);
  const size_t nl = h->layers.size();
  cudaError_t e = cudaSuccess;
  // the weights in 8 bits
  for (size_t l = 0; l < nl && e == cudaSuccess; ++l) {
    const mca_layer& L = h->layers[l];
    const int64_t ld = round16(L.n_in);
    if (L.wkind == MCA_W_TERNARY_I8) {
      e = cudaMemcpy2DAsync(w, (size_t)ld, h->code[l], (size_t)L.n_in, (size_t)L.n_in,
                            (size_t)L.n_out, cudaMemcpyDeviceToDevice, h->stream);
      if (e == cudaSuccess) e = mca::launch_fill(w_scale, L.n_out, L.scale, h->stream);
    } else {
      e = mca::launch_quantize_rows(h->w_eff[l], MCA_DTYPE_FP32, L.n_out, L.n_in, L.n_in, w, ld,
                                    w_scale, h->stream);
    }
    h->launches += 1;
    w += align256((size_t)ld * (size_t)L.n_out);
    w_scale += L.n_out;
  }
  for (int64_t n0 = 0; n0 < n && e == cudaSuccess; n0 += p.chunk) {
    const int64_t m = std::min(p.chunk, n - n0);
    const void* in = x + n0 * ldx;
    int in_dtype = MCA_DTYPE_FP32;
    int64_t in_ld = ldx;
    w = reinterpret_cast<int8_t*>(ws + p.w);
    w_scale = reinterpret_cast<float*>(ws + p.w_scale);
    for (size_t l = 0; l < nl && e == cudaSuccess; ++l) {
      const mca_layer& L = h->layers[l];
      const bool last = l + 1 == nl;
      mca_code_linear_args a{};
      a.rows = m;
      a.n_in = L.n_in;
      a.n_out = L.n_out;
      a.x = codes;
      a.ldx = round16(L.n_in);
      a.x_scale = scale;
      a.w = w;
      a.ldw = a.ldx;
      a.w_scale = w_scale;
      a.y = last ? static_cast<void*>(out + n0 * L.n_out) : ws + p.hidden;
      a.ldy = last ? L.n_out : round16(L.n_out);
      a.dtype = !last && bounded_by_one(L) ? MCA_DTYPE_FP16 : MCA_DTYPE_FP32;
      a.act = L.act;
      a.act_param = L.act_param;
      a.workspace = ws + p.product;
      e = mca::launch_quantize_rows(in, in_dtype, m, L.n_in, in_ld, codes, a.ldx, scale, h->stream);
      if (e == cudaSuccess) e = mca::launch_code_linear(a, h->stream);
      h->launches += 2;
      in = a.y;
      in_dtype = a.dtype;
      in_ld = a.ldy;
      w += align256((size_t)a.ldw * (size_t)L.n_out);
      w_scale += L.n_out;
    }
  }
  nvtxRangePop();
  return launched(h, e, "mca_predict");
}

}  // extern "C"
