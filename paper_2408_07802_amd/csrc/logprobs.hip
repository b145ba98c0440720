// Log probabilities of given tokens, the entropy and the most likely tokens of rows of logits.
//
// With m the largest logit, s = sum e^(x - m) and u = sum e^(x - m) (x - m):
//   log p(x) = (x - m) - log s,   entropy = log s - u / s.
// Both are formed from differences to m, so an offset of the row costs no precision.
#include <hip/hip_runtime.h>
#include <math.h>

#include "kraken_internal.hpp"
#include "../../include/kraken.h"

namespace kraken {
namespace {

struct LogprobParams {
  const void* logits;
  int64_t ld;
  int rows, vocab, top;
  const int32_t* tokens;
  float *logprob, *entropy;
  int32_t* ids;
  float* top_logprobs;
};

// Order of logits as unsigned integers: larger first means larger, a NaN above +inf, -0 = +0.
__device__ __forceinline__ uint32_t order_of(float x) {
  if (x != x) return 0xffffffffu;
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Block: one row.
template <typename S>
__global__ __launch_bounds__(256) void logprob_kernel(LogprobParams p) {
  __shared__ float red[256], red2[256];
  __shared__ uint64_t key[256];
  const int r = blockIdx.x, tid = threadIdx.x;
  const S* x = static_cast<const S*>(p.logits) + r * p.ld;
  auto join = [&](auto* a, auto v, auto op) {
    a[tid] = v;
    __syncthreads();
    for (int k = 128; k > 0; k >>= 1) {
      if (tid < k) a[tid] = op(a[tid], a[tid + k]);
      __syncthreads();
    }
    const auto res = a[0];
    __syncthreads();
    return res;
  };
  float m = -INFINITY;
  for (int c = tid; c < p.vocab; c += 256) m = fmaxf(m, (float)x[c]);
  m = join(red, m, [](float a, float b) { return fmaxf(a, b); });
  float s = 0.f, u = 0.f;
  for (int c = tid; c < p.vocab; c += 256) {
    const float t = (float)x[c] - m, e = expf(t);
    s += e;
    u += t == -INFINITY ? 0.f : e * t;
  }
  s = join(red, s, [](float a, float b) { return a + b; });
  u = join(red2, u, [](float a, float b) { return a + b; });
  const float ls = logf(s);
  if (tid == 0) {
    if (p.tokens) {
      const int tok = p.tokens[r];
      p.logprob[r] = tok < 0 ? 0.f : tok < p.vocab ? ((float)x[tok] - m) - ls : NAN;
    }
    if (p.entropy) p.entropy[r] = ls - u / s;
  }
  uint64_t below = ~0ull;
  for (int k = 0; k < p.top; ++k) {
    uint64_t best = 0;
    for (int c = tid; c < p.vocab; c += 256) {
      const uint64_t v = (uint64_t)order_of((float)x[c]) << 32 | (uint32_t)~c;
      if ((k == 0 || v < below) && v > best) best = v;
    }
    below = join(key, best, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
    if (tid == 0) {
      const int c = (int)~(uint32_t)below;
      p.ids[(int64_t)r * p.top + k] = c;
      p.top_logprobs[(int64_t)r * p.top + k] = ((float)x[c] - m) - ls;
    }
  }
}

kraken_status fail(kraken_status s, const char* msg) { return (kraken_status)set_error(s, msg); }

}  // namespace
}  // namespace kraken

using namespace kraken;

extern "C" {

int64_t kraken_token_logprobs_work_floats(int32_t rows, int32_t vocab, int32_t top) {
  if (rows < 0 || vocab < 1 || top < 0 || top > KRAKEN_MAX_TOP || top > vocab) return -1;
  return 0;
}

kraken_status kraken_op_token_logprobs(int32_t dtype, const void* logits, int64_t ld,
                                       int32_t rows, int32_t vocab, const int32_t* tokens,
                                       float* logprob, float* entropy, int32_t top,
                                       int32_t* top_ids, float* top_logprobs, float* work,
                                       int64_t work_floats, void* stream) {
  if (dtype < KRAKEN_DTYPE_F32 || dtype > KRAKEN_DTYPE_F16)
    return fail(KRAKEN_ERR_UNSUPPORTED, "unknown dtype");
  if (rows < 0 || vocab < 1 || ld < vocab)
    return fail(KRAKEN_ERR_INVALID_ARG, "bad rows, vocab or ld");
  if (top < 0 || top > KRAKEN_MAX_TOP || top > vocab)
    return fail(KRAKEN_ERR_INVALID_ARG, "top out of 0..min(vocab, KRAKEN_MAX_TOP)");
  if (!logits) return fail(KRAKEN_ERR_INVALID_ARG, "logits is NULL");
  if (reinterpret_cast<uintptr_t>(logits) % (dtype == KRAKEN_DTYPE_F32 ? 4 : 2) != 0)
    return fail(KRAKEN_ERR_INVALID_ARG, "logits is not aligned to an element");
  if (!tokens != !logprob) return fail(KRAKEN_ERR_INVALID_ARG, "tokens and logprob go together");
  if ((top > 0) != (top_ids != nullptr) || (top > 0) != (top_logprobs != nullptr))
    return fail(KRAKEN_ERR_INVALID_ARG, "top_ids and top_logprobs go with top > 0");
  if (work_floats < 0 || work_floats < kraken_token_logprobs_work_floats(rows, vocab, top))
    return fail(KRAKEN_ERR_INVALID_ARG, "work is smaller than the call needs");
  if (reinterpret_cast<uintptr_t>(work) % 16 != 0)
    return fail(KRAKEN_ERR_INVALID_ARG, "work is not 16-byte aligned");
  if (rows == 0) return KRAKEN_OK;
  LogprobParams p{logits, ld, rows, vocab, top, tokens, logprob, entropy, top_ids, top_logprobs};
  hipStream_t s = static_cast<hipStream_t>(stream);
  const dim3 grid((unsigned)rows);
  switch (dtype) {
    case KRAKEN_DTYPE_BF16:
      hipLaunchKernelGGL(logprob_kernel<bf16>, grid, dim3(256), 0, s, p);
      break;
    case KRAKEN_DTYPE_F16:
      hipLaunchKernelGGL(logprob_kernel<f16>, grid, dim3(256), 0, s, p);
      break;
    default: hipLaunchKernelGGL(logprob_kernel<float>, grid, dim3(256), 0, s, p);
  }
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? KRAKEN_OK : fail(KRAKEN_ERR_HIP, hipGetErrorString(e));
}

}  // extern "C"
