// Log probabilities of given tokens, the entropy and the most likely tokens of rows of logits.
//
// With m the largest logit, s = sum e^(x - m) and u = sum e^(x - m) (x - m):
//   log p(x) = (x - m) - log s,   entropy = log s - u / s.
// Both are formed from differences to m, so an offset of the row costs no precision.  One pass:
// every lane keeps its own (m, s, u), rescaled when its m grows; they are joined at the end.
//
// The most likely tokens, in the same pass: a logit and its index make a 64-bit key (larger
// logit, then lower index, first).  A wave collects the keys above a bound in LDS; when 64
// have come, it ranks them with its list and keeps the best `top`.  The bound is the best
// top-th key that any wave of the block has seen, to begin with the top-th largest of the 64
// lanes' maxima of a wave's first elements, so hardly more than the answer is ever collected,
// and a pass over most elements is one comparison each.  What the waves hold at the end is
// ranked once more.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>

#include "kraken_internal.hpp"
#include "../../include/kraken.h"

namespace kraken {
namespace {

constexpr int MAX_SPLITS = 32;

struct LogprobParams {
  const void* logits;
  int64_t ld;
  int rows, vocab, top;
  const int32_t* tokens;
  float *logprob, *entropy;
  int32_t* ids;
  float* top_logprobs;
  int splits;             // blocks that share a row
  float4* sums;           // [rows][splits]: m, s, u of a block's part (splits > 1)
  uint64_t* keys;         // [rows][splits][top]: its best keys, 0 behind the last
};

constexpr float LOG2E = 1.44269504088896341f;

// Order of logits as unsigned integers: larger means larger, a NaN above +inf, -0 = +0.  Never 0.
__device__ __forceinline__ uint32_t order_of(float x) {
  if (x != x) return 0xffffffffu;
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t order) {
  return __builtin_bit_cast(float, order & 0x80000000u ? order & 0x7fffffffu : ~order);
}

// Running sums over part of a row: s = sum e^(x - m), u = sum e^(x - m) (x - m).
struct Sums {
  float m, s, u;
};
// Differences to the largest are cut at -200, where e^d is 0 in fp32: no product with an
// infinity arises from a part that counts for nothing.  (A NaN stays in s.)
__device__ __forceinline__ Sums joined(Sums a, Sums b) {
  const float m = fmaxf(a.m, b.m);
  const float da = fmaxf(a.m - m, -200.f), db = fmaxf(b.m - m, -200.f);
  const float ea = __builtin_amdgcn_exp2f(da * LOG2E), eb = __builtin_amdgcn_exp2f(db * LOG2E);
  return {m, a.s * ea + b.s * eb, (a.u + a.s * da) * ea + (b.u + b.s * db) * eb};
}
__device__ __forceinline__ Sums wave_sums(Sums a) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1)
    a = joined(a, {__shfl_xor(a.m, o, 64), __shfl_xor(a.s, o, 64), __shfl_xor(a.u, o, 64)});
  return a;
}

// What a row's sums say (one thread).
__device__ __forceinline__ void write_row(const LogprobParams& p, int r, Sums a, float logit,
                                          int token) {
  const float ls = logf(a.s);
  if (p.tokens) p.logprob[r] = token < 0 ? 0.f : token < p.vocab ? (logit - a.m) - ls : NAN;
  if (p.entropy) p.entropy[r] = ls - a.u / a.s;
}

// A row's n best keys (its best `top` among them), ranked by the block and written.
template <int THREADS>
__device__ __forceinline__ void write_top(const LogprobParams& p, int r, const uint64_t* keys,
                                          int n, float m, float ls) {
  for (int e = threadIdx.x; e < n; e += THREADS) {
    const uint64_t mine = keys[e];
    int rank = 0;
    for (int k = 0; k < n; ++k) rank += keys[k] > mine ? 1 : 0;
    if (rank < p.top) {
      p.ids[(int64_t)r * p.top + rank] = (int)~(uint32_t)mine;
      p.top_logprobs[(int64_t)r * p.top + rank] = (value_of((uint32_t)(mine >> 32)) - m) - ls;
    }
  }
}

// Block: row r, or one of the equal shares of its vectors of 16 bytes.  NW waves take 64 GV
// vectors each in turn.
template <typename S, int NW, bool TOP>
__global__ __launch_bounds__(NW * 64) void logprob_kernel(LogprobParams p) {
  constexpr int VPT = 16 / sizeof(S), GV = 16 / VPT, E = 16;
  constexpr int LIST = TOP ? 128 : 1;
  __shared__ uint64_t list[NW][LIST];         // a wave's best and the keys it has collected
  __shared__ uint64_t last[TOP ? NW * 128 : 1];
  __shared__ unsigned long long bound;        // keys at or below are not among the row's best,
                                              // but for the key itself
  __shared__ float red[NW][3];
  __shared__ int n_last;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r = p.splits == 1 ? blockIdx.x : blockIdx.x / p.splits;
  const int share = p.splits == 1 ? 0 : blockIdx.x % p.splits;
  const S* row = static_cast<const S*>(p.logits) + r * p.ld;
  int token = -1;
  float logit = 0.f;
  if (tid == 0 && p.tokens && p.splits == 1) {
    token = p.tokens[r];
    if (token >= 0 && token < p.vocab) logit = (float)row[token];
  }
  if (TOP && tid == 0) {
    bound = 0;
    n_last = 0;
  }
  // vector v: the aligned 16 bytes with elements v VPT - off ...; vectors v0 .. v1 - 1 are ours
  const int off = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(S));
  const S* base = row - off;
  const int nv = (int)(((int64_t)off + p.vocab + VPT - 1) / VPT);
  const int per = (nv + p.splits - 1) / p.splits;
  const int v0 = share * per, v1 = min(v0 + per, nv);
  auto load = [&](int first, uint4* raw) {
#pragma unroll
    for (int g = 0; g < GV; ++g) {
      const int v = first + g * 64 + lane;
      if (v > 0 && v < nv - 1 && v < v1) {
        raw[g] = *reinterpret_cast<const uint4*>(base + (int64_t)v * VPT);
      } else {                                // an edge of the row, or nothing of ours
        alignas(16) S x[VPT];
#pragma unroll
        for (int e = 0; e < VPT; ++e) {
          const int64_t c = (int64_t)v * VPT + e - off;
          x[e] = v < v1 && c >= 0 && c < p.vocab ? row[c] : (S)(-INFINITY);
        }
        raw[g] = *reinterpret_cast<const uint4*>(x);
      }
    }
  };

  Sums a = {-INFINITY, 0.f, 0.f};
  uint64_t cut = 0;                           // as bound, of the wave
  float cut_f = -INFINITY;                    // its logit
  int have = 0, fresh = 0;                    // keys of the list, and behind it
  auto rank_list = [&]() {
    uint64_t* l = list[wave];
    const int n = have + fresh;
    const uint64_t k0 = lane < n ? l[lane] : 0, k1 = lane + 64 < n ? l[lane + 64] : 0;
    int r0 = 0, r1 = 0;
#pragma unroll 4
    for (int j = 0; j < n; ++j) {
      const uint64_t k = l[j];
      r0 += k > k0 ? 1 : 0;
      r1 += k > k1 ? 1 : 0;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (lane < n && r0 < p.top) l[r0] = k0;
    if (lane + 64 < n && r1 < p.top) l[r1] = k1;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    have = n < p.top ? n : p.top;
    fresh = 0;
    if (have == p.top) {
      const uint64_t k = l[p.top - 1];
      if (k > cut) {
        cut = k;
        if (lane == 0) atomicMax(&bound, (unsigned long long)k);
      }
    }
  };

  uint4 raw[GV];
  constexpr int STEP = NW * 64 * GV;
  int at = v0 + wave * 64 * GV;
  if (TOP) __syncthreads();
  load(at, raw);
  bool first = true;
  while (at < v1) {
    float x[E];
#pragma unroll
    for (int g = 0; g < GV; ++g) {
      const S* c = reinterpret_cast<const S*>(&raw[g]);
#pragma unroll
      for (int e = 0; e < VPT; ++e) x[g * VPT + e] = (float)c[e];
    }
    const int here = at;
    at += STEP;
    if (at < v1) load(at, raw);
    float mx = x[0];
#pragma unroll
    for (int e = 1; e < E; ++e) mx = fmaxf(mx, x[e]);
    {
      const float m = fmaxf(a.m, mx), d = fmaxf(a.m - m, -200.f);
      const float f = __builtin_amdgcn_exp2f(d * LOG2E), ref = m == -INFINITY ? 0.f : m;
      a.u = (a.u + a.s * d) * f;
      a.s *= f;
      a.m = m;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float t = x[e] - ref, w = __builtin_amdgcn_exp2f(t * LOG2E);
        a.s += w;
        a.u = fmaf(w, fmaxf(t, -200.f), a.u);
      }
    }
    if constexpr (TOP) {
      if (first) {
        // the top-th largest of the lanes' maxima: that many elements are at least as large
        first = false;
        const uint32_t o = order_of(mx);
        int rank = 0;
        for (int j = 0; j < 64; ++j) {
          const uint32_t k = (uint32_t)__builtin_amdgcn_readlane((int)o, j);
          rank += k > o || (k == o && j < lane) ? 1 : 0;
        }
        const int who = __ffsll((unsigned long long)__ballot(rank == p.top - 1)) - 1;
        const uint32_t t = (uint32_t)__builtin_amdgcn_readlane((int)o, who);
        cut = ((uint64_t)t << 32) - 1;
        if (lane == 0) atomicMax(&bound, (unsigned long long)cut);
      }
      const uint64_t b = *(volatile unsigned long long*)&bound;
      cut = b > cut ? b : cut;
      // (bounds that end in ones are of the order above: all that equals it may pass)
      cut_f = value_of((uint32_t)((cut + 1) >> 32));
      bool any = false;
#pragma unroll
      for (int e = 0; e < E; ++e) any |= !(x[e] < cut_f);
      if (__any(any)) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int v = here + (e / VPT) * 64 + lane;
          const int64_t c = (int64_t)v * VPT + e % VPT - off;
          const bool valid = v < v1 && c >= 0 && c < p.vocab;
          const uint64_t key = (uint64_t)order_of(x[e]) << 32 | (uint32_t)~(uint32_t)c;
          uint64_t pass = __ballot(valid && key > cut);
          if (!pass) continue;
          if (fresh + __popcll(pass) > 64) {
            rank_list();
            pass = __ballot(valid && key > cut);
          }
          if (pass >> lane & 1)
            list[wave][have + fresh + __popcll(pass & ((1ull << lane) - 1))] = key;
          fresh += __popcll(pass);
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
      }
    }
  }

  a = wave_sums(a);
  if (lane == 0) {
    red[wave][0] = a.m;
    red[wave][1] = a.s;
    red[wave][2] = a.u;
  }
  __syncthreads();
  a = {red[0][0], red[0][1], red[0][2]};
#pragma unroll
  for (int k = 1; k < NW; ++k) a = joined(a, {red[k][0], red[k][1], red[k][2]});
  if (tid == 0) {
    if (p.splits == 1) write_row(p, r, a, logit, token);
    else p.sums[blockIdx.x] = make_float4(a.m, a.s, a.u, 0.f);
  }
  if constexpr (TOP) {
    // the waves' keys that may be among the best, together
    const uint64_t b = bound;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int e = lane + 64 * h;
      const uint64_t key = e < have + fresh ? list[wave][e] : 0;
      const uint64_t keep = __ballot(key != 0 && key >= b);
      int to = 0;
      if (lane == 0 && keep) to = atomicAdd(&n_last, __popcll(keep));
      to = __builtin_amdgcn_readfirstlane(to);
      if (keep >> lane & 1) last[to + __popcll(keep & ((1ull << lane) - 1))] = key;
    }
    __syncthreads();
    const int n = n_last;
    if (p.splits == 1) {
      write_top<NW * 64>(p, r, last, n, a.m, logf(a.s));
    } else {
      uint64_t* out = p.keys + (int64_t)blockIdx.x * p.top;
      for (int e = n + tid; e < p.top; e += NW * 64) out[e] = 0;
      for (int e = tid; e < n; e += NW * 64) {
        const uint64_t mine = last[e];
        int rank = 0;
        for (int k = 0; k < n; ++k) rank += last[k] > mine ? 1 : 0;
        if (rank < p.top) out[rank] = mine;
      }
    }
  }
}

// Block: the shares of one row.
template <typename S>
__global__ __launch_bounds__(256) void logprob_join_kernel(LogprobParams p) {
  __shared__ uint64_t keys[MAX_SPLITS * KRAKEN_MAX_TOP];
  __shared__ unsigned long long bound;
  __shared__ int n_keys;
  const int r = blockIdx.x, tid = threadIdx.x;
  Sums a = {-INFINITY, 0.f, 0.f};
  for (int k = 0; k < p.splits; ++k) {
    const float4 v = p.sums[(int64_t)r * p.splits + k];
    a = joined(a, {v.x, v.y, v.z});
  }
  if (tid == 0) {
    int token = -1;
    float logit = 0.f;
    if (p.tokens) {
      token = p.tokens[r];
      if (token >= 0 && token < p.vocab)
        logit = (float)(static_cast<const S*>(p.logits) + r * p.ld)[token];
    }
    write_row(p, r, a, logit, token);
    bound = 0;
    n_keys = 0;
  }
  if (p.top == 0) return;
  const uint64_t* in = p.keys + (int64_t)r * p.splits * p.top;
  __syncthreads();
  for (int k = tid; k < p.splits; k += 256)
    atomicMax(&bound, (unsigned long long)in[(k + 1) * p.top - 1]);
  __syncthreads();
  const uint64_t b = bound;
  for (int e = tid; e < p.splits * p.top; e += 256) {
    const uint64_t key = in[e];
    if (key != 0 && key >= b) keys[atomicAdd(&n_keys, 1)] = key;
  }
  __syncthreads();
  write_top<256>(p, r, keys, n_keys, a.m, logf(a.s));
}

// Blocks per row.
int splits_of(int rows, int vocab) { return 1; }

template <typename S, int NW>
void launch_logprobs(const LogprobParams& p, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)p.rows * p.splits)), block(NW * 64);
  if (p.top > 0) hipLaunchKernelGGL((logprob_kernel<S, NW, true>), grid, block, 0, s, p);
  else hipLaunchKernelGGL((logprob_kernel<S, NW, false>), grid, block, 0, s, p);
}

template <typename S>
hipError_t launch_typed(const LogprobParams& p, hipStream_t s) {
  if (p.rows * (int64_t)p.splits >= 512) launch_logprobs<S, 4>(p, s);
  else launch_logprobs<S, 16>(p, s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  hipLaunchKernelGGL(logprob_join_kernel<S>, dim3((unsigned)p.rows), dim3(256), 0, s, p);
  return hipGetLastError();
}

kraken_status fail(kraken_status s, const char* msg) { return (kraken_status)set_error(s, msg); }

}  // namespace
}  // namespace kraken

using namespace kraken;

extern "C" {

int64_t kraken_token_logprobs_work_floats(int32_t rows, int32_t vocab, int32_t top) {
  if (rows < 0 || vocab < 1 || top < 0 || top > KRAKEN_MAX_TOP || top > vocab) return -1;
  const int splits = splits_of(rows, vocab);
  return splits == 1 ? 0 : (int64_t)rows * splits * (4 + 2 * top);
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
  const int64_t need = kraken_token_logprobs_work_floats(rows, vocab, top);
  if (work_floats < need || work_floats < 0 || (need > 0 && !work))
    return fail(KRAKEN_ERR_INVALID_ARG, "work is smaller than the call needs");
  if (reinterpret_cast<uintptr_t>(work) % 16 != 0)
    return fail(KRAKEN_ERR_INVALID_ARG, "work is not 16-byte aligned");
  if (rows == 0) return KRAKEN_OK;
  LogprobParams p{logits, ld, rows, vocab, top, tokens, logprob, entropy, top_ids, top_logprobs,
                  splits_of(rows, vocab), nullptr, nullptr};
  if (p.splits > 1) {
    p.sums = reinterpret_cast<float4*>(work);
    p.keys = reinterpret_cast<uint64_t*>(work + 4 * (int64_t)rows * p.splits);
  }
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e;
  switch (dtype) {
    case KRAKEN_DTYPE_BF16: e = launch_typed<bf16>(p, s); break;
    case KRAKEN_DTYPE_F16: e = launch_typed<f16>(p, s); break;
    default: e = launch_typed<float>(p, s);
  }
  return e == hipSuccess ? KRAKEN_OK : fail(KRAKEN_ERR_HIP, hipGetErrorString(e));
}

}  // extern "C"
