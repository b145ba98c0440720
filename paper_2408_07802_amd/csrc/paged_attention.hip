// Attention of one new token per sequence over a paged KV cache.
//
// Work: a unit is one (sub-layer, key/value head, block of up to 16 of its query heads) of one
// sequence; its keys are cut into tiles of KT.  All tiles of all units stand in one list
// (sequence by sequence), which W waves share in equal runs, whatever the sequences' lengths are:
// the lengths are read on the device, so a replayed graph follows them.  A wave takes its run
// tile by tile with a running maximum and sum per query head (online softmax, base 2), writes
// the output of every unit that lies inside its run, and a partial (maximum, sum, output) of the
// unit that its run begins or ends in the middle of; the join kernel merges those.  Waves share
// nothing: there is no barrier.
//
// Tile: S^T = K Q^T and O^T += V^T P^T by 16 x 16 matrix instructions, keys x query heads and
// features x query heads, so a lane keeps one query head (lane % 16) throughout and the maximum,
// the sum and the rescaling are its own; the scores are the second product's operand as they
// lie in registers.  Only few of the 16 columns are used where few query heads share a
// key/value head; the products are cheap next to the tile's bytes all the same.
//
// Data: a tile's K and V rows (8 KB each) go from the pages straight into LDS, two tiles ahead
// (K rows as soon as the scores have left their place free), and the page numbers of a tile's
// rows do so two tiles before that.  Chunks of 16 bytes of a row are permuted so that the reads
// spread over all LDS banks; V is read transposed (ds_read_b64_tr).
//
// What bounds it: the cache, read once (counters: 537 MB fetched of 537).  8192 keys of 8
// sub-layers of 16 heads of 128 (fp16): 92 us, 5.8 TB/s, and 5 us for the join; eight
// conversations of 32 674 keys in all, 4 key/value heads (bf16): 93 + 5 us, 5.6 TB/s; 128 of 470
// on average, 4 sub-layers of 16 heads of 64: 163 + 5 us, 5.3 TB/s; 16 of 19 400 in 8 bits, 2
// heads for 32: 36 + 6 us, 4.4 TB/s (the waves' first tiles and the join are a fifth of it).  A
// block per (query head, sequence) that splits nothing took 587, 769, 171 and 1862 us.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "kraken_internal.hpp"
#include "paged.hpp"

namespace kraken {
namespace {

struct RowsView {
  void* data;
  int64_t sub, row;
};

struct PagedAttnParams {
  RowsView q, out;
  PagedView cache;
  const int32_t* lens;
  int32_t* fault;
  int4* desc;           // units that runs share (parts, first run, b, u); parts 0: nothing to join
  float* ml;            // [W][2][qh][2]: maximum and sum
  float* o;             // [W][2][qh][HD]: unnormalised output
  int heads, group, max_len, W;
  FastDiv per_run, per_seq, per_block, per_head;   // by W, units of a sequence, qblocks, kv heads
  int qblocks, qh;      // blocks of query heads per key/value head; query heads per block (<= 16)
  int whole;            // runs end where units end: nothing is shared
  int by_unit;          // desc has an entry per unit (of every sequence), not per run
  float scale;
};

typedef uint8_t e4m3;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) void* lds_ptr;

__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return (uint32_t)(uintptr_t)(lds_ptr)p;
}

// 16 (4) bytes per lane from global memory into LDS at `lds` + 16 (4) * lane; lds is uniform.
// Counted by vmcnt, which the kernel waits for itself.
__device__ __forceinline__ void dma16(uint32_t lds, uint64_t g) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               :: "s"(lds), "v"(g) : "memory", "m0");
}
__device__ __forceinline__ void dma4(uint32_t lds, const void* g) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
               :: "s"(lds), "v"(g) : "memory", "m0");
}
// What lies at an LDS address.
template <typename V>
__device__ __forceinline__ V lds_read(uint32_t at) {
  return *(const __attribute__((address_space(3))) V*)at;
}
// Waits until at most N of the wave's vector memory operations are outstanding (they complete
// in order).
template <int N>
__device__ __forceinline__ void wait_vm() {
  static_assert(N < 64, "vmcnt has 6 bits");
  asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory");
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// x of lane ^ 16 (^ 32) and the lane's own, in an order that both lanes share.
struct Both {
  float a, b;
};
template <bool BY32>
__device__ __forceinline__ Both with_other(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = BY32 ? __builtin_amdgcn_permlane32_swap(u, u, false, false)
                      : __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t a = r[0], b = r[1];
  return {__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)};
}
// Of the four lanes lane % 16 + 16 k: the maximum, and the sum.
__device__ __forceinline__ float max4(float x) {
  const Both p = with_other<false>(x);
  const Both q = with_other<true>(fmaxf(p.a, p.b));
  return fmaxf(q.a, q.b);
}
__device__ __forceinline__ float sum4(float x) {
  const Both p = with_other<false>(x);
  const Both q = with_other<true>(p.a + p.b);
  return q.a + q.b;
}

// Keys of a tile of rows of hd elements of es bytes: 8 KB, at most 128.  (Tiles of 4 KB with twice
// the waves: the same for 16-bit rows of 64, 2 to 8% slower for 8-bit rows, whose instructions
// per tile are many.)
constexpr int tile_keys(int hd, int es) { return 8192 / (hd * es) < 128 ? 8192 / (hd * es) : 128; }

// Sizes of a tile.  C: the cache's element type.
template <typename C, int HD>
struct Tile {
  static constexpr int RB = HD * (int)sizeof(C);               // bytes of a row
  static constexpr int NC = RB / 16;                           // 16-byte chunks of a row
  static constexpr int KT = tile_keys(HD, (int)sizeof(C));     // keys
  static constexpr int RPI = 64 / NC;                          // rows per DMA instruction
  static constexpr int NI = KT / RPI;                          // DMA instructions for K (for V)
  static constexpr int NT = (KT + 63) / 64;                    // and for the page numbers
  static constexpr int LINE = NC < 16 ? 16 / NC : 1;           // rows per 256 bytes of LDS
};

// Logical chunk c of row r lies at chunk c ^ key of its row.  K is read by 16 lanes that take
// the same chunk of 16 consecutive rows: those fall on 16 different chunks of a 256-byte line.
template <typename C, int HD>
__device__ __forceinline__ int k_key(int r) {
  using T = Tile<C, HD>;
  return (r / T::LINE) & (T::NC < 16 ? T::NC - 1 : 15);
}
// V by 32 lanes at a time.  16 bits: two chunks of 8 consecutive rows (the pair stays together);
// 8 bits: one chunk of rows r .. r + 7 and r + 16 .. r + 23; fp32: 16 chunks of one row.
template <typename C, int HD>
__device__ __forceinline__ int v_key(int r) {
  using T = Tile<C, HD>;
  if constexpr (sizeof(C) == 2) return ((r / T::LINE) & (T::NC / 2 - 1)) * 2;
  if constexpr (sizeof(C) == 1)
    return ((r / T::LINE) & (8 / T::LINE - 1)) | ((r >> 4) & 1) * (8 / T::LINE);
  return 0;
}

template <typename S>
using Vec8 = typename std::conditional<__is_same(S, bf16), bf16x8, f16x8>::type;

template <typename S>
__device__ __forceinline__ f32x4 mfma32(Vec8<S> a, Vec8<S> b, f32x4 c) {
  if constexpr (__is_same(S, bf16))
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Eight e4m3 values as S (exact: S has more bits and a wider range).
template <typename S>
__device__ __forceinline__ Vec8<S> from_e4m3(uint32_t lo, uint32_t hi) {
  Vec8<S> r;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t w = k < 2 ? lo : hi;
    if constexpr (__is_same(S, bf16)) {
      const bf16x2 x = k & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true)
                             : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false);
      r[2 * k] = x[0]; r[2 * k + 1] = x[1];
    } else {
      const f16x2 x = k & 1 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, true)
                            : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, false);
      r[2 * k] = x[0]; r[2 * k + 1] = x[1];
    }
  }
  return r;
}

// A wave's place in the list of tiles: tile j of the nt of unit u (sub-layer i, key/value head
// h, query block qb) of sequence b.
struct Place {
  int b, u, i, h, qb, j, nt, len, bad;
};

// Queries of a unit in LDS: rows of qh heads, in whole DMA instructions.
constexpr int q_slot(int qh, int row_bytes) { return (qh * row_bytes + 1023) / 1024 * 1024; }

template <typename S, typename C, int HD>
__global__ __launch_bounds__(64, 1) void paged_attn_kernel(PagedAttnParams p) {
  using T = Tile<C, HD>;
  constexpr bool F32 = sizeof(C) == 4, F8 = sizeof(C) == 1;
  constexpr int KT = T::KT, KB = KT / 16, FT = HD / 16, NT = T::NT, ND = 2 * T::NI;
  constexpr int RBQ = HD * (int)sizeof(S), STAGE = KT * T::RB;
  __shared__ __align__(1024) uint8_t kv[2][2][STAGE];          // [stage][K, V]
  __shared__ int pg[4][NT * 64];                               // pages of a tile's rows
  __shared__ uint64_t row_at[NT * 64];                         // and where its K rows lie
  __shared__ int s_len[KRAKEN_MAX_SEQS];                       // keys, -1: out of range
  extern __shared__ __align__(16) uint8_t q_rows[];            // a unit's queries

  const int lane = threadIdx.x, w = blockIdx.x, g = lane >> 4, col = lane & 15;
  const int B = p.cache.seqs, U = (int)p.per_seq.d;

  // lengths, and the tiles of sequences 0 .. b for the lane's four
  int total, incl[4];
  {
    int sum = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int b = lane * 4 + e;
      int len = b < B ? p.lens[b] : 0;
      if (len < 0 || len > p.max_len) len = -1;
      s_len[b] = len;
      sum += len > 0 ? (len + KT - 1) / KT : 0;
      incl[e] = sum;
    }
    int scan = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int up = __shfl_up(scan, d, 64);
      if (lane >= d) scan += up;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) incl[e] += scan - sum;
    total = uniform(__shfl(scan, 63, 64)) * U;
  }
  auto len_of = [&](int b) { return uniform(s_len[b]); };

  // rows without keys: zeros, or NaN for a length out of range
  for (int r = w; r < p.cache.n * B; r += gridDim.x) {
    const int i = r / B, b = r - i * B, len = len_of(b);
    if (len > 0) continue;
    if (p.by_unit)
      for (int u = lane; u < p.cache.heads * p.qblocks; u += 64)
        p.desc[b * U + i * p.cache.heads * p.qblocks + u] = make_int4(0, 0, 0, 0);
    if (len < 0 && p.fault && lane == 0) *p.fault = 1;
    S* out = static_cast<S*>(p.out.data) + i * p.out.sub + b * p.out.row;
    for (int c = lane; c < p.heads * HD; c += 64) out[c] = len < 0 ? (S)NAN : (S)0.f;
  }
  if (p.desc && !p.by_unit && lane == 0) p.desc[w] = make_int4(0, 0, 0, 0);

  // sequence, unit and tile of an item of the list
  auto place_of = [&](int item) {
    Place c;
    const int x = (int)div_of(p.per_seq, (uint32_t)item);
    int b = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) b += __popcll(__ballot(incl[e] <= x));
    b = uniform(b);
    c.b = b;
    c.len = len_of(b);
    c.nt = (c.len + KT - 1) / KT;
    // tiles before b: its own inclusive count less its tiles
    const int own = (b & 3) == 0 ? incl[0] : (b & 3) == 1 ? incl[1] : (b & 3) == 2 ? incl[2] : incl[3];
    const uint32_t rem = (uint32_t)(item - (uniform(__shfl(own, b >> 2, 64)) - c.nt) * U);
    c.u = uniform((int)(rem / (uint32_t)c.nt));
    c.j = (int)rem - c.u * c.nt;
    const int hq = (int)div_of(p.per_block, (uint32_t)c.u);
    c.qb = c.u - hq * p.qblocks;
    c.i = (int)div_of(p.per_head, (uint32_t)hq);
    c.h = hq - c.i * p.cache.heads;
    c.bad = 0;
    return c;
  };
  auto advance = [&](Place& c) {
    if (++c.j < c.nt) return;
    c.j = 0;
    ++c.u;
    if (++c.qb < p.qblocks) return;
    c.qb = 0;
    if (++c.h < p.cache.heads) return;
    c.h = 0;
    if (++c.i < p.cache.n) return;
    c.i = c.u = 0;
    do ++c.b; while (c.b < B - 1 && len_of(c.b) <= 0);
    c.len = len_of(min(c.b, B - 1));
    c.nt = (c.len + KT - 1) / KT;
  };

  // the run: items begin .. begin + cnt - 1, and the place of the next tile to look up.  Where
  // units are not shared, an edge inside a unit moves behind it.
  const int run = run_length(p.per_run, total);
  int begin = w * run;
  if (begin >= total) return;
  int end = min(begin + run, total);
  Place tp = place_of(begin);
  if (p.whole) {
    if (end < total) {
      const Place e = place_of(end);
      if (e.j > 0) end += e.nt - e.j;
    }
    if (tp.j > 0) {
      begin += tp.nt - tp.j;
      tp.j = tp.nt - 1;
      if (begin < end) advance(tp);
    }
  }
  const int cnt = end - begin;
  if (cnt <= 0) return;

  const uint32_t page_bytes = (uint32_t)p.cache.heads * p.cache.page.d * T::RB;
  const uint64_t v_off = (uint64_t)p.cache.pages * page_bytes;
  const uint32_t kv_at = lds_addr(kv), q_at = lds_addr(q_rows);
  // this lane's chunk of a DMA instruction's K and V rows: bytes behind the row's beginning
  uint32_t k_off[T::NI];
  uint64_t v_at[T::NI];
#pragma unroll
  for (int x = 0; x < T::NI; ++x) {
    const int r = x * T::RPI + lane / T::NC, pc = lane % T::NC;
    k_off[x] = (pc ^ k_key<C, HD>(r)) * 16;
    v_at[x] = v_off + (pc ^ v_key<C, HD>(r)) * 16;
  }

  // page numbers of a tile's rows; rows behind the last key are the last key's
  auto look_up = [&](const Place& c, int slot) {
    const int32_t* row = p.cache.table + (int64_t)c.b * p.cache.table_ld;
#pragma unroll
    for (int x = 0; x < NT; ++x) {
      const int key = min(c.j * KT + x * 64 + lane, c.len - 1);
      dma4(lds_addr(&pg[slot][x * 64]), row + div_of(p.cache.page, (uint32_t)key));
    }
  };
  // a unit's queries, adjacent rows
  auto fetch_q = [&](const Place& c) {
    const int bytes = min(16, p.group - c.qb * 16) * RBQ;
    const uint64_t src = reinterpret_cast<uint64_t>(
        static_cast<const S*>(p.q.data) + c.i * p.q.sub + c.b * p.q.row +
        (int64_t)(c.h * p.group + c.qb * 16) * HD);
    for (int x = 0; x < bytes; x += 1024)
      dma16(uniform((int)(q_at + x)), src + min(x + lane * 16, bytes - 16));
  };
  // a tile's K rows, and then (with the rows' places as they are) its V rows
  auto fetch_k = [&](Place& c, int slot, int stage) {
    const uint64_t base = reinterpret_cast<uint64_t>(p.cache.data) + 2 * c.i * v_off +
                          (uint64_t)((uint32_t)c.h * p.cache.page.d * T::RB);
    bool bad = false;
#pragma unroll
    for (int x = 0; x < NT; ++x) {
      const int key = min(c.j * KT + x * 64 + lane, c.len - 1);
      const uint32_t at = ((uint32_t)key - div_of(p.cache.page, (uint32_t)key) * p.cache.page.d) *
                          (uint32_t)T::RB;
      int page = pg[slot][x * 64 + lane];
      const bool ok = page >= 0 && page < p.cache.pages;
      bad |= !ok;
      page = ok ? page : 0;
      row_at[x * 64 + lane] = base + (uint64_t)(uint32_t)page * page_bytes + at;
    }
    c.bad = __any(bad);
    const uint32_t to = kv_at + stage * (2 * STAGE);
#pragma unroll
    for (int x = 0; x < T::NI; ++x) {
      const uint64_t at = row_at[x * T::RPI + lane / T::NC];
      dma16(to + x * 1024, at + k_off[x]);
    }
  };
  auto fetch_v = [&](int stage) {
    const uint32_t to = kv_at + stage * (2 * STAGE) + STAGE;
#pragma unroll
    for (int x = 0; x < T::NI; ++x)
      dma16(to + x * 1024, row_at[x * T::RPI + lane / T::NC] + v_at[x]);
  };

  // state of the unit at hand: the lane's query head col
  Vec8<typename std::conditional<F32, f16, S>::type> q[F32 ? 1 : HD / 32];
  f32x4 q4[F32 ? HD / 16 : 1];
  f32x4 acc[FT];
  float m_run = -INFINITY, l_run = 0.f, ks = 0.f, vs = 1.f;
  int h0 = 0, nh = 0, bad = 0;
  bool began = false;

  auto open_unit = [&](const Place& c) {
    h0 = c.h * p.group + c.qb * 16;
    nh = min(16, p.group - c.qb * 16);
    const uint32_t src = q_at + min(col, nh - 1) * RBQ;
    const bool mine = col < nh;
    if constexpr (F32) {
#pragma unroll
      for (int m = 0; m < HD / 16; ++m) {
        q4[m] = lds_read<f32x4>(src + (16 * m + 4 * g) * 4);
        if (!mine) q4[m] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
    } else {
#pragma unroll
      for (int m = 0; m < HD / 32; ++m) {
        // dimensions of k slot 8 g + e of product m: as the K operand's
        const int at = F8 && HD > 32 ? 64 * (m / 2) + 16 * g + 8 * (m % 2) : 32 * m + 8 * g;
        i32x4 v = lds_read<i32x4>(src + at * 2);
        if (!mine) v = i32x4{0, 0, 0, 0};
        q[m] = __builtin_bit_cast(Vec8<S>, v);
      }
    }
    ks = p.scale * 1.44269504088896341f;
    vs = 1.f;
    if constexpr (F8) {
      ks *= p.cache.scales[(c.i * 2) * p.cache.heads + c.h];
      vs = p.cache.scales[(c.i * 2 + 1) * p.cache.heads + c.h];
    }
    m_run = -INFINITY;
    l_run = 0.f;
    bad = 0;
    began = c.j == 0;
#pragma unroll
    for (int f = 0; f < FT; ++f) acc[f] = f32x4{0.f, 0.f, 0.f, 0.f};
  };

  // This lane's LDS addresses, all but constants: chunk (4 m + g) ^ key of K row col (the key of
  // rows col + 16 kb is the same), and its part of V rows.  (Chunks are permuted within the
  // aligned bytes of a row, so the permuted chunk of block f is one exclusive or away.)
  const uint32_t k_row = kv_at + col * T::RB;
  const int k_k = k_key<C, HD>(col);
  f32x4 sc[KB];                             // scores of the tile at hand
  auto score = [&](int stage) {
    const uint32_t K = k_row + stage * (2 * STAGE);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) sc[kb] = f32x4{0.f, 0.f, 0.f, 0.f};
    if constexpr (F32) {
#pragma unroll
      for (int m = 0; m < HD / 16; ++m) {
        const uint32_t at = K + ((4 * m + g) ^ k_k) * 16;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
          const f32x4 a = lds_read<f32x4>(at + kb * 16 * T::RB);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            sc[kb] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], q4[m][e], sc[kb], 0, 0, 0);
        }
      }
    } else if constexpr (F8 && HD == 32) {
      const uint32_t at = K + ((g / 2) ^ k_k) * 16 + g % 2 * 8;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const i32x2 a = lds_read<i32x2>(at + kb * 16 * T::RB);
        sc[kb] = mfma32<S>(from_e4m3<S>(a[0], a[1]), q[0], sc[kb]);
      }
    } else if constexpr (F8) {
#pragma unroll
      for (int m = 0; m < HD / 64; ++m) {
        const uint32_t at = K + ((4 * m + g) ^ k_k) * 16;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
          const i32x4 a = lds_read<i32x4>(at + kb * 16 * T::RB);
          sc[kb] = mfma32<S>(from_e4m3<S>(a[0], a[1]), q[2 * m], sc[kb]);
          sc[kb] = mfma32<S>(from_e4m3<S>(a[2], a[3]), q[2 * m + 1], sc[kb]);
        }
      }
    } else {
#pragma unroll
      for (int m = 0; m < HD / 32; ++m) {
        const uint32_t at = K + ((4 * m + g) ^ k_k) * 16;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
          sc[kb] = mfma32<S>(lds_read<Vec8<S>>(at + kb * 16 * T::RB), q[m], sc[kb]);
      }
    }
  };
  auto output = [&](const Place& c, int stage) {
    // scores in base-2 units, of keys 16 kb + 4 g + r
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) sc[kb] *= ks;
    const int left = c.len - c.j * KT;
    if (left < KT) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (kb * 16 + 4 * g + r >= left) sc[kb][r] = -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
      mx = fmaxf(mx, fmaxf(fmaxf(sc[kb][0], sc[kb][1]), fmaxf(sc[kb][2], sc[kb][3])));
    mx = max4(mx);
    if (__any(mx > m_run)) {
      const float m_new = fmaxf(m_run, mx);
      // (a head without a finite score yet has sums of zero, which any factor but NaN keeps)
      const float alpha = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m_new);
      l_run *= alpha;
#pragma unroll
      for (int f = 0; f < FT; ++f) acc[f] *= alpha;
      m_run = m_new;
    }
    const float mref = m_run == -INFINITY ? 0.f : m_run;
    f32x4 ps = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
      for (int r = 0; r < 4; ++r) sc[kb][r] = __builtin_amdgcn_exp2f(sc[kb][r] - mref);
      ps += sc[kb];
    }
    // of the lane's keys; the lanes join at the end
    l_run += (ps[0] + ps[1]) + (ps[2] + ps[3]);
    const uint32_t V = kv_at + stage * (2 * STAGE) + STAGE;
    if constexpr (F32) {
      constexpr int E = HD < 64 ? 2 : 4;      // features 16 E cc + E row + e of one LDS read
      const uint32_t at = V + 4 * g * T::RB + col * 4 * E;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int cc = 0; cc < FT / E; ++cc) {
            typedef float vec __attribute__((ext_vector_type(E)));
            const vec v = lds_read<vec>(at + (kb * 16 + r) * T::RB + cc * 64 * E);
#pragma unroll
            for (int e = 0; e < E; ++e)
              acc[cc * E + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e], sc[kb][r],
                                                                     acc[cc * E + e], 0, 0, 0);
          }
    } else {
      // the lane's row of block f's reads: 8 bits, of 8 rows; 16 bits, of 4 (and 16 further on)
      const int e = col / 2, r0 = F8 ? 16 * (e / 4) + 4 * g + e % 4 : 4 * g + col / 4;
      const uint32_t at = V + r0 * T::RB + (col & 1) * 8 +
                          ((F8 ? 0 : (col & 3) / 2) ^ v_key<C, HD>(r0)) * 16;
#pragma unroll
      for (int k2 = 0; k2 < KB / 2; ++k2) {
        // k slots 8 g + e: keys 4 g + e of block 2 k2, then of the next.  A weight goes into
        // the product as two terms, its rounding to S and what that leaves out: the output
        // keeps 16 bits of it and more, and the second product is free next to the loads.
        Vec8<S> hi, lo;
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const float v = sc[2 * k2 + x / 4][x % 4];
          hi[x] = (S)v;
          lo[x] = (S)(v - (float)hi[x]);
        }
#pragma unroll
        for (int f = 0; f < FT; ++f) {
          Vec8<S> a;
          if constexpr (F8) {
            const i32x2 x = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                (__attribute__((address_space(3))) i32x2*)((at ^ (f * 16)) + k2 * 32 * T::RB));
            a = from_e4m3<S>((uint32_t)x[0], (uint32_t)x[1]);
          } else {
            s16x4 x[2];
#pragma unroll
            for (int y = 0; y < 2; ++y)
              x[y] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                  (__attribute__((address_space(3))) s16x4*)((at ^ (f * 32)) +
                                                             (k2 * 32 + y * 16) * T::RB));
            typedef short s16x8 __attribute__((ext_vector_type(8)));
            const s16x8 both = __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7);
            a = __builtin_bit_cast(Vec8<S>, both);
          }
          acc[f] = mfma32<S>(a, hi, acc[f]);
          acc[f] = mfma32<S>(a, lo, acc[f]);
        }
      }
    }
    bad |= c.bad;
  };

  // four neighbouring features of the lane's query head, the n-th of HD / 16 times, and the
  // first of them
  auto four = [&](int n, int& feature) {
    if constexpr (F32 && HD == 32) {
      feature = 8 * g + 4 * n;
      return f32x4{acc[0][2 * n], acc[1][2 * n], acc[0][2 * n + 1], acc[1][2 * n + 1]};
    } else if constexpr (F32) {
      const int cc = n / 4, r = n % 4;
      feature = 64 * cc + 16 * g + 4 * r;
      return f32x4{acc[4 * cc][r], acc[4 * cc + 1][r], acc[4 * cc + 2][r], acc[4 * cc + 3][r]};
    } else {
      feature = 16 * n + 4 * g;
      return acc[n];
    }
  };

  // end of the unit (done) or of the wave's run in the middle of it
  auto close_unit = [&](const Place& c, int at) {
    const bool done = c.j == c.nt - 1;
    float l = sum4(l_run);
    if (bad) {
      l = NAN;
      if (p.fault && lane == 0) *p.fault = 1;
    }
    if (began && done) {
      if (p.by_unit && lane == 0) p.desc[c.b * U + c.u] = make_int4(0, 0, 0, 0);
      if (col < nh) {
        S* out = static_cast<S*>(p.out.data) + c.i * p.out.sub + c.b * p.out.row +
                 (int64_t)(h0 + col) * HD;
        const float inv = vs / l;
#pragma unroll
        for (int n = 0; n < FT; ++n) {
          int feature;
          const f32x4 v = four(n, feature);
          typedef S S4 __attribute__((ext_vector_type(4)));
          S4 x;
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = (S)(v[e] * inv);
          *reinterpret_cast<S4*>(out + feature) = x;
        }
      }
      return;
    }
    const int slot = 2 * w + (began ? 1 : 0);
    if (began && lane == 0) {
      const int last = (int)((uint32_t)(at + c.nt - 1 - c.j) / (uint32_t)run);
      p.desc[p.by_unit ? c.b * U + c.u : w] = make_int4(last - w + 1, w, c.b, c.u);
    }
    if (col < nh) {
      if (g == 0) {
        float* ml = p.ml + ((int64_t)slot * p.qh + col) * 2;
        ml[0] = m_run;
        ml[1] = l;
      }
      float* o = p.o + ((int64_t)slot * p.qh + col) * HD;
#pragma unroll
      for (int n = 0; n < FT; ++n) {
        int feature;
        const f32x4 v = four(n, feature);
        *reinterpret_cast<f32x4*>(o + feature) = v;
      }
    }
  };

  // The run.  Memory operations in order: pages of tiles 0 and 1, the first queries, then rows of
  // tile t and pages of tile t + 2, tile after tile; while tile t is computed, the rows of t + 1
  // and the pages of t + 2 and t + 3 may be outstanding.  The queries of a unit that begins with
  // tile t + 1 follow the pages of t + 3, once those of tile t's unit are in registers.
  Place cur, nxt, tp2;                       // tiles t, t + 1 and t + 2
  cur = tp;
  look_up(tp, 0);
  advance(tp);
  nxt = tp;
  if (cnt > 1) {
    look_up(tp, 1);
    advance(tp);
  }
  tp2 = tp;
  fetch_q(cur);
  wait_vm<0>();
  fetch_k(cur, 0, 0);
  fetch_v(0);
  if (cnt > 2) {
    look_up(tp, 2);
    advance(tp);
  }
  if (cnt > 1) {
    fetch_k(nxt, 1, 1);
    fetch_v(1);
  }
  if (cnt > 3) {
    look_up(tp, 3);
  }
  Place tp3 = tp;                            // tile t + 3
  for (int t = 0; t < cnt; ++t) {
    const int rem = cnt - t;
    const bool opens = t == 0 || cur.j == 0;
    if (rem > 3) {
      // (a unit's queries are older than the rows of t + 1 and the pages of t + 3 alone)
      if (opens) wait_vm<ND + NT>();
      else wait_vm<ND + 2 * NT>();
    } else if (rem > 1) {
      wait_vm<ND>();
    } else {
      wait_vm<0>();
    }
    if (opens) open_unit(cur);
    if (rem > 1 && nxt.j == 0) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // (the queries' reads)
      fetch_q(nxt);
    }
    score(t & 1);
    if (rem > 2) {
      // the K rows' reads are done, and the page numbers are there
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (rem > 3) wait_vm<ND + NT>();
      else wait_vm<ND>();
      fetch_k(tp2, (t + 2) & 3, t & 1);
    }
    output(cur, t & 1);
    if (cur.j == cur.nt - 1 || rem == 1) close_unit(cur, begin + t);
    if (rem > 2) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      fetch_v(t & 1);
    }
    cur = nxt;
    nxt = tp2;
    tp2 = tp3;
    if (rem > 4) {
      advance(tp3);
      look_up(tp3, t & 3);
    }
  }
}

// Joins the partials of a unit that several runs share: with M the largest maximum,
// out = sum o e^(m - M) / sum l e^(m - M).  Block (entry of desc, share of the query heads); a
// group of HD / 4 lanes takes a query head's partials, every gph-th of them where there are more
// groups than heads.
template <typename S, int HD, int THREADS>
__global__ __launch_bounds__(THREADS) void paged_join_kernel(PagedAttnParams p) {
  constexpr int LQ = HD / 4, NG = THREADS / LQ;
  __shared__ float sm[NG], sl[NG];
  __shared__ f32x4 so[NG][LQ];
  const int tid = threadIdx.x, grp = tid / LQ, f = tid % LQ;
  const int4 d = p.desc[blockIdx.x];
  const int parts = d.x, w = d.y, b = d.z, u = d.w;
  if (parts == 0) return;
  const int hq = u / p.qblocks, qb = u % p.qblocks;
  const int i = hq / p.cache.heads, h = hq % p.cache.heads;
  const int h0 = h * p.group + qb * 16, nh = min(16, p.group - qb * 16);
  const int share = (p.qh + gridDim.y - 1) / gridDim.y, end = min(nh, (int)(blockIdx.y + 1) * share);
  const float vs = p.cache.scales ? p.cache.scales[(i * 2 + 1) * p.cache.heads + h] : 1.f;
  // groups per head: a power of two
  int gph = 1;
  while (2 * gph * share <= NG) gph *= 2;
  for (int hb = blockIdx.y * share; hb < end; hb += NG / gph) {
    const int head = hb + grp / gph, sub = grp % gph;
    float m = -INFINITY, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    auto merge = [&](float mk, float lk, f32x4 ok) {
      const float mn = fmaxf(m, mk), ref = mn == -INFINITY ? 0.f : mn;
      const float a = __builtin_amdgcn_exp2f(m - ref), c = __builtin_amdgcn_exp2f(mk - ref);
      l = l * a + lk * c;
      o = o * a + ok * c;
      m = mn;
    };
    if (head < end) {
      for (int k0 = sub; k0 < parts; k0 += 4 * gph) {          // four loads in flight
        float mk[4], lk[4];
        f32x4 ok[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int k = min(k0 + x * gph, parts - 1);
          const int64_t slot = ((int64_t)(w + k) * 2 + (k == 0 ? 1 : 0)) * p.qh + head;
          mk[x] = p.ml[slot * 2];
          lk[x] = p.ml[slot * 2 + 1];
          ok[x] = *reinterpret_cast<const f32x4*>(p.o + slot * HD + 4 * f);
        }
#pragma unroll
        for (int x = 0; x < 4; ++x)
          if (k0 + x * gph < parts) merge(mk[x], lk[x], ok[x]);
      }
    }
    if (gph > 1) {
      if (f == 0) {
        sm[grp] = m;
        sl[grp] = l;
      }
      so[grp][f] = o;
      __syncthreads();
      if (sub == 0)
        for (int k = 1; k < gph; ++k) merge(sm[grp + k], sl[grp + k], so[grp + k][f]);
      __syncthreads();
    }
    if (head < end && sub == 0) {
      S* out = static_cast<S*>(p.out.data) + i * p.out.sub + b * p.out.row +
               (int64_t)(h0 + head) * HD + 4 * f;
      typedef S S4 __attribute__((ext_vector_type(4)));
      const float inv = vs / l;
      S4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = (S)(o[e] * inv);
      *reinterpret_cast<S4*>(out) = x;
    }
  }
}

int cache_es(int dtype) {
  return dtype == KRAKEN_DTYPE_E4M3 ? 1 : dtype == KRAKEN_DTYPE_F32 ? 4 : 2;
}

// How a call is shared out.
struct Shape {
  int qh, qblocks, q_bytes, waves, entries;      // entries of desc (0: whole units)
  int parts;                                     // of a unit, about, at most
  double tiles;                                  // at most
};
// Units of up to 4 tiles are not shared: a wave takes 1.2 us (16 bits) to 1.9 us a tile after 4.6
// us for the first, the join 5 us.
constexpr int WHOLE_TILES = 4;
// Tiles of a run, at least, once that leaves a wave for every CU (65536 keys of one head: 19 us,
// with runs of two tiles 41 us, most of it the join of a thousand parts).
constexpr int RUN_TILES = 4;
Shape shape_of(const kraken_paged_cache* c, int n_heads, int max_len) {
  Shape s;
  const int es = cache_es(c->dtype), kt = tile_keys(c->head_dim, es);
  const int group = n_heads / c->n_kv_heads;
  s.qh = std::min(16, group);
  s.qblocks = (group + 15) / 16;
  s.q_bytes = q_slot(s.qh, c->head_dim * std::max(es, 2));
  // as many waves as LDS holds: two stages of K and V, 4 KB at most of lengths, pages and places,
  // and the queries (four per CU; three with 16 fp32 queries of 128, seven with 8-bit heads of 32)
  const int most = 256 * (163840 / (4 * kt * c->head_dim * es + 4096 + s.q_bytes));
  const int64_t units = (int64_t)c->n_sub * c->n_kv_heads * s.qblocks * c->num_seqs;
  const int64_t per = (max_len + (int64_t)kt - 1) / kt;
  const bool whole = per <= WHOLE_TILES;
  s.tiles = (double)units * std::max<int64_t>(per, 1);
  const double items = (double)units * (whole ? 1 : per);    // (may be 0)
  const double want = whole ? items : std::max(std::min(items, 256.0), items / RUN_TILES);
  s.waves = want >= most ? most : std::max(1, (int)want);
  s.entries = whole ? 0 : (int)std::min<int64_t>(units, s.waves);
  s.parts = (int)std::min<double>(s.waves, per * (s.waves / items) + 2);
  return s;
}

template <typename S, typename C, int HD>
hipError_t launch_hd(const PagedAttnParams& p, const Shape& sh, hipStream_t s) {
  const dim3 grid((unsigned)p.W);
  hipLaunchKernelGGL((paged_attn_kernel<S, C, HD>), grid, dim3(64), (unsigned)sh.q_bytes, s, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.whole) return e;
  // about 2048 blocks (more wait for the rest to start and find nothing to do), and more threads
  // for each of few that have much to read
  const int y = std::max(1, std::min(sh.qh, 2048 / sh.entries));
  const dim3 joins((unsigned)sh.entries, (unsigned)y);
  if (sh.parts > 128)
    hipLaunchKernelGGL((paged_join_kernel<S, HD, 1024>), joins, dim3(1024), 0, s, p);
  else
    hipLaunchKernelGGL((paged_join_kernel<S, HD, 256>), joins, dim3(256), 0, s, p);
  return hipGetLastError();
}

template <typename S, typename C>
hipError_t launch_typed(const PagedAttnParams& p, const Shape& sh, int hd, hipStream_t s) {
  if (hd == 32) return launch_hd<S, C, 32>(p, sh, s);
  if (hd == 64) return launch_hd<S, C, 64>(p, sh, s);
  return launch_hd<S, C, 128>(p, sh, s);
}

kraken_status fail(kraken_status s, const char* msg) { return (kraken_status)set_error(s, msg); }

}  // namespace
}  // namespace kraken

using namespace kraken;

extern "C" {

int64_t kraken_paged_attention_work_floats(const kraken_paged_cache* cache, int32_t n_heads,
                                           int32_t max_len) {
  kraken_status st;
  if (paged_view(cache, false, nullptr, &st) || n_heads < 1 || n_heads > 65535 ||
      n_heads % cache->n_kv_heads != 0 || max_len < 0 ||
      max_len > (int64_t)cache->pages_per_seq * cache->page_size)
    return -1;
  const Shape sh = shape_of(cache, n_heads, max_len);
  if (sh.entries == 0) return 0;
  return 4 * (int64_t)sh.entries + 2 * (int64_t)sh.waves * sh.qh * (2 + cache->head_dim);
}

kraken_status kraken_op_paged_attention(int32_t dtype, const kraken_rows* q,
                                        const kraken_rows* out, int32_t n_heads,
                                        const kraken_paged_cache* cache, const int32_t* lens,
                                        int32_t max_len, float scale, float* work,
                                        int64_t work_floats, int32_t* fault, void* stream) {
  PagedAttnParams p;
  kraken_status st;
  if (const char* msg = paged_view(cache, true, &p.cache, &st)) return fail(st, msg);
  if (dtype < KRAKEN_DTYPE_F32 || dtype > KRAKEN_DTYPE_F16)
    return fail(KRAKEN_ERR_UNSUPPORTED, "unknown dtype");
  const bool e4m3_cache = cache->dtype == KRAKEN_DTYPE_E4M3;
  if (e4m3_cache ? dtype == KRAKEN_DTYPE_F32 : cache->dtype != dtype)
    return fail(KRAKEN_ERR_UNSUPPORTED,
                "the cache has the queries' dtype, or is E4M3 with BF16 or F16 queries");
  if (!q || !out || !lens) return fail(KRAKEN_ERR_INVALID_ARG, "q, out or lens is NULL");
  if (n_heads < 1 || n_heads > 65535 || n_heads % cache->n_kv_heads != 0)
    return fail(KRAKEN_ERR_INVALID_ARG, "n_kv_heads does not divide n_heads");
  if (max_len < 0 || max_len > (int64_t)cache->pages_per_seq * cache->page_size)
    return fail(KRAKEN_ERR_INVALID_ARG, "max_len out of 0..pages_per_seq * page_size");
  if (!isfinite(scale)) return fail(KRAKEN_ERR_INVALID_ARG, "scale is not finite");
  const Shape sh = shape_of(cache, n_heads, max_len);
  if (sh.tiles >= 1073741824.0)
    return fail(KRAKEN_ERR_UNSUPPORTED, "2^30 or more tiles of keys");
  const int es = dtype == KRAKEN_DTYPE_F32 ? 4 : 2;
  for (const kraken_rows* r : {q, out})
    if (const char* msg = check_rows(r, cache->n_sub, cache->num_seqs, es,
                                     r == out ? (int64_t)n_heads * cache->head_dim : 0))
      return fail(KRAKEN_ERR_INVALID_ARG, msg);
  const int64_t need = kraken_paged_attention_work_floats(cache, n_heads, max_len);
  if (work_floats < need || (need > 0 && !work) || work_floats < 0)
    return fail(KRAKEN_ERR_INVALID_ARG, "work is smaller than the call needs");
  if (reinterpret_cast<uintptr_t>(work) % 16 != 0)
    return fail(KRAKEN_ERR_INVALID_ARG, "work is not 16-byte aligned");
  const int hd = cache->head_dim;
  p.q = {q->data, q->sub_stride, q->row_stride};
  p.out = {out->data, out->sub_stride, out->row_stride};
  p.lens = lens; p.fault = fault;
  p.heads = n_heads; p.group = n_heads / cache->n_kv_heads; p.max_len = max_len;
  p.qblocks = sh.qblocks;
  p.per_run = fast_div((uint32_t)sh.waves);
  p.per_seq = fast_div((uint32_t)(cache->n_sub * cache->n_kv_heads * sh.qblocks));
  p.per_block = fast_div((uint32_t)sh.qblocks);
  p.per_head = fast_div((uint32_t)cache->n_kv_heads);
  p.qh = sh.qh;
  p.W = sh.waves;
  p.whole = sh.entries == 0;
  p.by_unit = 0;
  p.desc = nullptr;
  p.ml = p.o = nullptr;
  if (!p.whole) {
    p.by_unit = (int64_t)cache->n_sub * cache->n_kv_heads * sh.qblocks * cache->num_seqs <= p.W;
    p.desc = reinterpret_cast<int4*>(work);
    p.ml = work + 4 * (int64_t)sh.entries;
    p.o = p.ml + 4 * (int64_t)p.W * p.qh;
  }
  p.scale = scale != 0.f ? scale : (float)(1.0 / sqrt((double)hd));
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e;
  if (dtype == KRAKEN_DTYPE_F32) e = launch_typed<float, float>(p, sh, hd, s);
  else if (dtype == KRAKEN_DTYPE_BF16)
    e = e4m3_cache ? launch_typed<bf16, e4m3>(p, sh, hd, s) : launch_typed<bf16, bf16>(p, sh, hd, s);
  else e = e4m3_cache ? launch_typed<f16, e4m3>(p, sh, hd, s) : launch_typed<f16, f16>(p, sh, hd, s);
  if (e == hipSuccess) return KRAKEN_OK;
  return fail(KRAKEN_ERR_HIP, hipGetErrorString(e));
}

}  // extern "C"
