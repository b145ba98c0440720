// Log probabilities of given tokens, the entropy and the most likely tokens of rows of logits.
//
// With m the largest logit, s = sum e^(x - m) and u = sum e^(x - m) (x - m):
//   log p(x) = (x - m) - log s,   entropy = log s - u / s.
// Both are formed from differences to m, so an offset of the row costs no precision.  (c x - c m
// in one operation would: its products overflow at the lowest values that masks hold.)  One pass:
// every lane keeps its own (m, s, u), rescaled when its m grows; they are joined at the end.
//
// The most likely tokens: a logit and its index make a 64-bit key (larger logit, then lower
// index, first).  The pass over the row also keeps the largest logit of every lane in up to 8
// pieces of its elements.  The top-th largest of 256 groups of lanes' maxima is then a bound
// that at least `top` elements reach and few more: the pieces that reach it, about as many, are
// read again, their keys at or above the bound collected in LDS and ranked.  Where more keys
// come than fit (rows of many equal logits), the block looks for a better bound by counting
// (bisection over the 32-bit order of fp32), and takes equal logits by ascending index.
//
// What bounds it: many rows, the logits read once (2048 x 51200 fp32 with the likeliest token: 78
// us, 5.4 TB/s, as without it; with 64 alternatives 84 us).  Few rows, one block's pass over
// 50 000 logits: 10 us (7 us without alternatives; its CU issues vector instructions for 43% of
// that).  A list per wave, ranked as it fills, instead of the bound: 21 and 111 us.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>

#include "kraken_internal.hpp"
#include "../../include/kraken.h"

namespace kraken {
namespace {

constexpr int MAX_SPLITS = 8;
constexpr int JOIN_THREADS = MAX_SPLITS * KRAKEN_MAX_TOP;    // a key each

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

// Ranks n keys (a row's best `top` among them) and hands each of the best to put(rank, key).
template <int THREADS, class Put>
__device__ __forceinline__ void rank_keys(const uint64_t* keys, int n, int top, Put&& put) {
  for (int e = threadIdx.x; e < n; e += THREADS) {
    const uint64_t mine = keys[e];
    int rank = 0, k = 0;
    for (; k + 8 <= n; k += 8) {
#pragma unroll
      for (int x = 0; x < 8; ++x) rank += keys[k + x] > mine ? 1 : 0;
    }
    for (; k < n; ++k) rank += keys[k] > mine ? 1 : 0;
    if (rank < top) put(rank, mine);
  }
}
__device__ __forceinline__ void write_key(const LogprobParams& p, int r, int rank, uint64_t key,
                                          float m, float ls) {
  p.ids[(int64_t)r * p.top + rank] = (int)~(uint32_t)key;
  p.top_logprobs[(int64_t)r * p.top + rank] = (value_of((uint32_t)(key >> 32)) - m) - ls;
}
__device__ __forceinline__ uint64_t key_of(uint32_t order, int c) {
  return (uint64_t)order << 32 | (uint32_t)~(uint32_t)c;
}

// The largest t, of the upper 20 bits, that at least k of the wave's 256 values (four a lane)
// reach.  (16-bit logits have no others; of fp32 ones the bound lets a few more through.)
__device__ __forceinline__ uint32_t kth_of_256(const uint32_t* v, int k) {
  uint32_t t = 0;
#pragma unroll
  for (int bit = 31; bit >= 12; --bit) {
    const uint32_t c = t | 1u << bit;
    int n = 0;
#pragma unroll
    for (int x = 0; x < 4; ++x) n += __popcll(__ballot(v[x] >= c));
    t = n >= k ? c : t;
  }
  return t;
}

// Block: row r, or one of the equal shares of its vectors of 16 bytes.  A step takes GV vectors (16
// elements) of every lane.  A wave's are adjacent (2048 x 51200 fp32: 78 us; spread over the block's
// step, 80).  SPREAD: every lane has one before any has a second, so that a row of one step has
// as many lanes' maxima as vectors: 1000 fp32 in 63 lanes left 64 alternatives without a bound,
// for bisection (4096 rows: 61 us, now 22).
template <typename S, int NW, bool TOP, bool SPREAD>
__global__ __launch_bounds__(NW * 64) void logprob_kernel(LogprobParams p) {
  constexpr int VPT = 16 / sizeof(S), GV = 16 / VPT, E = 16, THREADS = NW * 64;
  constexpr int PIECES = TOP ? 8 : 1, CAP = 512;
  __shared__ float largest[PIECES][TOP ? THREADS : 1];   // of a lane's pieces
  __shared__ uint32_t lane_max[TOP ? THREADS : 1];
  __shared__ uint64_t keys[TOP ? CAP + THREADS : 1];
  __shared__ uint16_t pieces[TOP ? CAP : 1];             // that reach the bound: index * THREADS + tid
  __shared__ uint32_t bound;
  __shared__ int n_keys, n_pieces;
  __shared__ float red[NW][3];
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
  // vector v: the aligned 16 bytes with elements v VPT - off ...; vectors v0 .. v1 - 1 are ours
  const int off = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(S));
  const S* base = row - off;
  const int nv = (int)(((int64_t)off + p.vocab + VPT - 1) / VPT);
  const int per = (nv + p.splits - 1) / p.splits;
  const int v0 = share * per, v1 = min(v0 + per, nv);
  const int whole = min(nv - 1, v1);          // vectors 1 .. whole - 1 lie inside the row
  constexpr int STEP = THREADS * GV;
  const int steps = v1 > v0 ? (v1 - v0 + STEP - 1) / STEP : 0;
  // from a wave's first vector of a step to the next wave's, and from a lane's vector to its next
  constexpr int PER_WAVE = SPREAD ? 64 : 64 * GV, NEXT = SPREAD ? THREADS : 64;
  const int mine = v0 + wave * PER_WAVE;
  auto load = [&](int first, uint4* raw) {
    if (first > 0 && first + (GV - 1) * NEXT + 64 <= whole) {
      const uint4* from = reinterpret_cast<const uint4*>(base) + first + lane;
#pragma unroll
      for (int g = 0; g < GV; ++g) raw[g] = from[g * NEXT];
      return;
    }
#pragma unroll
    for (int g = 0; g < GV; ++g) {
      const int v = first + g * NEXT + lane;
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
  auto unpack = [&](const uint4* raw, float* x) {
#pragma unroll
    for (int g = 0; g < GV; ++g) {
      const S* c = reinterpret_cast<const S*>(&raw[g]);
#pragma unroll
      for (int e = 0; e < VPT; ++e) x[g * VPT + e] = (float)c[e];
    }
  };
  const int piece = (steps + PIECES - 1) / PIECES;     // steps of a piece

  Sums a = {-INFINITY, 0.f, 0.f};
  float top_piece = -INFINITY, top_lane = -INFINITY;
  uint4 raw[GV];
  load(mine, raw);
  int left = piece, at_piece = 0;
  for (int i = 0; i < steps; ++i) {
    float x[E];
    unpack(raw, x);
    if (i + 1 < steps) load(mine + (i + 1) * STEP, raw);
    float mx = x[0];
#pragma unroll
    for (int e = 1; e < E; ++e) mx = fmaxf(mx, x[e]);
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
    if constexpr (TOP) {
      top_piece = fmaxf(top_piece, mx);
      if (--left == 0 || i + 1 == steps) {
        largest[at_piece++][tid] = top_piece;
        top_lane = fmaxf(top_lane, top_piece);
        top_piece = -INFINITY;
        left = piece;
      }
    }
  }

  a = wave_sums(a);
  if (lane == 0) {
    red[wave][0] = a.m;
    red[wave][1] = a.s;
    red[wave][2] = a.u;
  }
  if constexpr (TOP) lane_max[tid] = order_of(top_lane);
  __syncthreads();
  a = {red[0][0], red[0][1], red[0][2]};
#pragma unroll
  for (int k = 1; k < NW; ++k) a = joined(a, {red[k][0], red[k][1], red[k][2]});
  if (tid == 0) {
    if (p.splits == 1) write_row(p, r, a, logit, token);
    else p.sums[blockIdx.x] = make_float4(a.m, a.s, a.u, 0.f);
  }
  if constexpr (TOP) {
    if (wave == NW - 1) {
      uint32_t v[4] = {0, 0, 0, 0};
#pragma unroll
      for (int k = 0; k < NW; ++k) v[k % 4] = max(v[k % 4], lane_max[k * 64 + lane]);
      const uint32_t t = kth_of_256(v, p.top);
      if (lane == 0) {
        bound = t;
        n_keys = n_pieces = 0;
      }
    }
    __syncthreads();
    uint32_t t = bound;
    // a vector's element c, if it is ours
    auto ours = [&](int v, int64_t c) { return v < v1 && c >= 0 && c < p.vocab; };
    auto push = [&](uint64_t key) {
      const int to = atomicAdd(&n_keys, 1);
      if (to < CAP) keys[to] = key;
    };
    // every element (x, its index) of steps i0 .. i1 - 1 of this lane
    auto each = [&](int i0, int i1, auto&& fn) {
      for (int i = i0; i < i1; ++i) {
        const int first = mine + i * STEP;
        uint4 again[GV];
        float x[E];
        load(first, again);
        unpack(again, x);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int v = first + (e / VPT) * NEXT + lane;
          const int64_t c = (int64_t)v * VPT + e % VPT - off;
          if (ours(v, c)) fn(order_of(x[e]), (int)c);
        }
      }
    };
    const bool plain = a.s == a.s;            // (a maximum passes over NaNs)
    if (plain) {
      for (int k = 0; k < at_piece; ++k)
        if (order_of(largest[k][tid]) >= t) {
          const int to = atomicAdd(&n_pieces, 1);
          if (to < CAP) pieces[to] = (uint16_t)(k * THREADS + tid);
        }
    }
    __syncthreads();
    const bool few = plain && n_pieces <= CAP;
    if (few) {
      // one vector of one of those pieces per thread and turn
      for (int i = 0; i < piece; ++i)
        for (int q = tid; q < n_pieces * GV; q += THREADS) {
          const int who = pieces[q / GV], of = who % THREADS, step = who / THREADS * piece + i;
          const int v = v0 + step * STEP + of / 64 * PER_WAVE + q % GV * NEXT + of % 64;
          if (step >= steps || v >= v1) continue;
          const int64_t c0 = (int64_t)v * VPT - off;
          if (v > 0 && v < nv - 1) {
            const uint4 again = *reinterpret_cast<const uint4*>(base + (int64_t)v * VPT);
            const S* x = reinterpret_cast<const S*>(&again);
#pragma unroll
            for (int e = 0; e < VPT; ++e) {
              const uint32_t o = order_of((float)x[e]);
              if (o >= t) push(key_of(o, (int)(c0 + e)));
            }
          } else {
            for (int e = 0; e < VPT; ++e)
              if (c0 + e >= 0 && c0 + e < p.vocab) {
                const uint32_t o = order_of((float)row[c0 + e]);
                if (o >= t) push(key_of(o, (int)(c0 + e)));
              }
          }
        }
    }
    __syncthreads();
    int n = n_keys;
    if (!few || n > CAP) {
      // A t that at least `top` elements reach and at most CAP exceed.  The first bound has the
      // former (or every element of a short share reaches it).
      auto above = [&](uint32_t o) {          // elements above o, for the whole block
        __syncthreads();
        if (tid == 0) n_keys = 0;
        __syncthreads();
        int count = 0;
        each(0, steps, [&](uint32_t x, int) { count += x > o ? 1 : 0; });
#pragma unroll
        for (int w = 1; w < 64; w <<= 1) count += __shfl_xor(count, w, 64);
        if (lane == 0) atomicAdd(&n_keys, count);
        __syncthreads();
        return n_keys;
      };
      if (above(t) > CAP) {
        uint32_t lo = t, hi = 0xffffffffu;    // above(lo) > CAP, above(hi) = 0
        t = hi;
        while (hi - lo > 1) {
          const uint32_t mid = lo + (hi - lo) / 2;
          const int c = above(mid);
          if (c > CAP) {
            lo = mid;
          } else {
            hi = mid;
            t = c >= p.top ? mid + 1 : mid;
            if (c >= p.top) break;
          }
        }
      }
      __syncthreads();
      if (tid == 0) n_keys = 0;
      __syncthreads();
      each(0, steps, [&](uint32_t o, int c) {
        if (o > t) push(key_of(o, c));
      });
      __syncthreads();
      n = n_keys;
      // what is missing, from the elements that equal it, in their order
      const int64_t c0 = max((int64_t)v0 * VPT - off, (int64_t)0);
      const int64_t c1 = min((int64_t)v1 * VPT - off, (int64_t)p.vocab);
      for (int64_t c = c0; c < c1 && n < p.top; c += THREADS) {
        __syncthreads();
        if (c + tid < c1 && order_of((float)row[c + tid]) == t) {
          const int to = atomicAdd(&n_keys, 1);
          keys[to] = key_of(t, (int)(c + tid));
        }
        __syncthreads();
        n = n_keys;
      }
    }
    if (p.splits == 1) {
      const float ls = logf(a.s);
      rank_keys<THREADS>(keys, n, p.top,
                         [&](int rank, uint64_t key) { write_key(p, r, rank, key, a.m, ls); });
    } else {
      uint64_t* out = p.keys + (int64_t)blockIdx.x * p.top;
      for (int e = n + tid; e < p.top; e += THREADS) out[e] = 0;
      rank_keys<THREADS>(keys, n, p.top, [&](int rank, uint64_t key) { out[rank] = key; });
    }
  }
}

// Block: the shares of one row.  Their keys are sorted, so a key's rank is the sum of what binary
// searches find in front of it in every share.
template <typename S>
__global__ __launch_bounds__(JOIN_THREADS) void logprob_join_kernel(LogprobParams p) {
  __shared__ uint64_t keys[JOIN_THREADS];
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
  }
  if (p.top == 0) return;
  const int total = p.splits * p.top;
  const uint64_t mine = tid < total ? p.keys[(int64_t)r * total + tid] : 0;    // 0: none
  keys[tid] = mine;
  __syncthreads();
  if (mine == 0) return;
  int before[MAX_SPLITS] = {};
  for (int step = 1 << (31 - __builtin_clz(p.top)); step > 0; step >>= 1) {
#pragma unroll
    for (int k = 0; k < MAX_SPLITS; ++k) {
      const int to = before[k] + step;          // the first `to` keys of share k
      const uint64_t key = keys[min(k * p.top + to, JOIN_THREADS) - 1];
      before[k] = to <= p.top && k < p.splits && key > mine ? to : before[k];
    }
  }
  int rank = 0;
#pragma unroll
  for (int k = 0; k < MAX_SPLITS; ++k) rank += before[k];
  if (rank < p.top) write_key(p, r, rank, mine, a.m, logf(a.s));
}

// Blocks per row.  A block of 8 waves takes 10 us for 51200 logits and 19 us for 160000 (fp32, the
// likeliest token; 12 and 21 us with 64), eight and the join of their parts 11 us for 160000 (14
// with 64), three 10.4 us for 64000 bf16 (one: 11.2).  So long rows are shared out where that
// leaves no block waiting for a CU.
int splits_of(int rows, int vocab) {
  if (vocab < 60000 || rows > 128 || rows < 1) return 1;
  return std::min({vocab / 20000, 256 / rows, MAX_SPLITS});
}

template <typename S, int NW, bool SPREAD>
void launch_logprobs(const LogprobParams& p, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)p.rows * p.splits)), block(NW * 64);
  if (p.top > 0) hipLaunchKernelGGL((logprob_kernel<S, NW, true, SPREAD>), grid, block, 0, s, p);
  else hipLaunchKernelGGL((logprob_kernel<S, NW, false, false>), grid, block, 0, s, p);
}

template <typename S>
hipError_t launch_typed(const LogprobParams& p, hipStream_t s) {
  // Many rows stream better in blocks of 4 waves (1000 x 16000 fp32 with the likeliest token: 16
  // us, of 8 waves 19), and rows that one step of such a block holds end sooner (511 x 2000: 6.4
  // and 7.8); few long ones with 8 (1 x 51200: 10.0, with 4 11.8, with 16 11.3; 511 x 30000 bf16:
  // 13, 15 and 19).
  if (p.vocab <= 4096) launch_logprobs<S, 4, true>(p, s);
  else if (p.rows * (int64_t)p.splits >= 512) launch_logprobs<S, 4, false>(p, s);
  else launch_logprobs<S, 8, false>(p, s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  hipLaunchKernelGGL(logprob_join_kernel<S>, dim3((unsigned)p.rows), dim3(JOIN_THREADS), 0, s, p);
  return hipGetLastError();
}

kraken_status fail(kraken_status s, const char* msg) { return (kraken_status)set_error(s, msg); }

}  // namespace
}  // namespace kraken

using namespace kraken;

extern "C" {

int64_t kraken_token_logprobs_work_floats(int32_t rows, int32_t vocab, int32_t top) {
  if (rows < 0 || rows > 1 << 22 || vocab < 1 || top < 0 || top > KRAKEN_MAX_TOP || top > vocab) return -1;
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
  if (rows > 1 << 22) return fail(KRAKEN_ERR_UNSUPPORTED, "rows above 4194304");
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
