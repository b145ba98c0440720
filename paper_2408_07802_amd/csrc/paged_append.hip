// Appending keys and values to a paged KV cache, with the rotation of queries and keys by
// their positions on the way.
//
// Rotation: row t turns the pair (a, b) of dimensions j and j + rot / 2 (or 2 j and 2 j + 1) of
// every head by the angle pos f_j: (a cos - b sin, a sin + b cos).  At position 10^6 an fp32
// product pos f_j is off by up to 2^-5 radians, so the angle is formed in 64 bits, in turns, its
// whole turns are dropped there, and only the rest in [-1/2, 1/2] goes to fp32.
//
// What bounds it: every row read and written once.  8192 rows of 8 sub-layers of 16 query and 16
// key/value heads of 128 (fp16, rotated keys as rows too): 341 us, 5.5 TB/s, as much as a copy
// reaches; 17 228 rows of 4 x 20 heads of 64 into 8 bits: 218 us, 4.9 TB/s (the conversions and
// the addresses keep the vector units busy for half of that).  One row: 4 us.
#include <hip/hip_runtime.h>
#include <math.h>
#include <algorithm>

#include "kraken_internal.hpp"
#include "paged.hpp"

namespace kraken {
namespace {

constexpr int MAX_FREQ = 64;          // pairs of a head of 128

struct RowsView {
  void* data;
  int64_t sub, row;                   // elements between sub-layers and between rows
};

// The rows of one kind (queries, keys or values): where they come from, where they go as rows
// (data NULL: nowhere), and how blocks share them.
struct Part {
  RowsView in, out;
  int units, rows;                    // units of a row; rows of a block
  FastDiv per_row;                    // by units
  unsigned first;                     // block
};

struct AppendParams {
  Part part[3];                       // 0: queries (in.data NULL: none), 1: keys, 2: values
  PagedView cache;
  const int32_t* pos;
  const int32_t* seq;
  int32_t* fault;
  int T, hd, rot, neighbours;
  double turns[MAX_FREQ];             // inv_freq / (2 pi)
};

template <typename T, int N>
struct alignas(sizeof(T) * N) Vec {
  T v[N];
};

// Chunk of U elements as S, and in 8 bits.
template <typename S, int U>
__device__ __forceinline__ void store_chunk(S* p, const float* x) {
  Vec<S, U> c;
#pragma unroll
  for (int e = 0; e < U; ++e) c.v[e] = (S)x[e];
  *reinterpret_cast<Vec<S, U>*>(p) = c;
}
// (Nearest e4m3, ties to even, beyond +-448 the largest; a NaN stays one.  The conversion makes
// NaNs of values out of range, so those are clamped first, where there are any: a clamp that
// keeps NaNs costs four instructions an element.)
template <int U>
__device__ __forceinline__ void store_e4m3(uint8_t* p, float* x, float inv) {
  float most = 0.f;
#pragma unroll
  for (int e = 0; e < U; ++e) {
    x[e] *= inv;
    most = fmaxf(most, fabsf(x[e]));
  }
  if (most > 448.f) {
#pragma unroll
    for (int e = 0; e < U; ++e) x[e] = x[e] > 448.f ? 448.f : x[e] < -448.f ? -448.f : x[e];
  }
  Vec<int, U / 4> c;
#pragma unroll
  for (int e = 0; e < U / 4; ++e) {
    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * e], x[4 * e + 1], 0, false);
    c.v[e] = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * e + 2], x[4 * e + 3], w, true);
  }
  *reinterpret_cast<Vec<int, U / 4>*>(p) = c;
}

constexpr int MAX_ROWS = 8;           // per block

// Block (rows of one kind, sub-layer).  Unit: two chunks of U elements of one head.  Where pairs
// are (j, j + rot / 2), the chunks of the two halves of the rotated dimensions, which a thread
// turns together; of other dimensions, too, one of each half, so that neighbouring threads read
// and write neighbouring chunks.  What a thread reads first is on its way before the block looks
// positions and pages up and forms the angles.
template <typename S, bool E4M3, int U>
__global__ __launch_bounds__(256) void append_kernel(AppendParams p) {
  __shared__ float cs[MAX_ROWS][MAX_FREQ], sn[MAX_ROWS][MAX_FREQ];
  __shared__ int64_t s_at[MAX_ROWS];  // element of the row's place in the cache, head 0; -1: none
  const int i = blockIdx.y, tid = threadIdx.x;
  const int kind = blockIdx.x < p.part[1].first ? 0 : blockIdx.x < p.part[2].first ? 1 : 2;
  const Part& part = p.part[kind];
  const int t0 = (blockIdx.x - part.first) * part.rows;
  const int rows = min(part.rows, p.T - t0), half = p.rot / 2;
  const int per_head = p.hd / (2 * U), log_per_head = 31 - __builtin_clz(per_head);
  const int nkv = p.cache.heads;
  const bool all = kind == 2 || p.neighbours;          // halves of a head, whatever is turned
  const S* in = static_cast<const S*>(part.in.data) + i * part.in.sub + t0 * part.in.row;
  S* out = static_cast<S*>(part.out.data);
  if (out) out += i * part.out.sub + t0 * part.out.row;

  struct Unit {
    int row, h, ca, cb;               // the chunks' dimensions of head h
    float scale;                      // E4M3, of keys and values
    Vec<S, U> a, b;
  };
  auto fetch = [&](int x) {
    Unit u;
    u.row = (int)div_of(part.per_row, (uint32_t)x);
    const int in_row = x - u.row * part.units, w = in_row & (per_head - 1);
    u.h = in_row >> log_per_head;
    // the first and half the number of the dimensions that are shared out
    const bool turned = w * U < half;
    u.ca = all || turned ? w * U : p.rot + w * U - half;
    u.cb = u.ca + (all ? p.hd : turned ? p.rot : p.hd - p.rot) / 2;
    if constexpr (E4M3)
      if (kind != 0) u.scale = p.cache.scales[(i * 2 + kind - 1) * nkv + u.h];
    const S* src = in + u.row * part.in.row + u.h * p.hd;
    u.a = *reinterpret_cast<const Vec<S, U>*>(src + u.ca);
    u.b = *reinterpret_cast<const Vec<S, U>*>(src + u.cb);
    return u;
  };
  auto finish = [&](const Unit& u) {
    const int64_t at = s_at[u.row];
    if (at < 0) return;
    float a[U], b[U];
#pragma unroll
    for (int e = 0; e < U; ++e) {
      a[e] = (float)u.a.v[e];
      b[e] = (float)u.b.v[e];
    }
    if (kind != 2) {
      if (!p.neighbours) {
        if (u.ca < half) {
#pragma unroll
          for (int e = 0; e < U; ++e) {
            const float c = cs[u.row][u.ca + e], s = sn[u.row][u.ca + e], x = a[e], y = b[e];
            a[e] = x * c - y * s;
            b[e] = x * s + y * c;
          }
        }
      } else {
        auto turn = [&](float* x, int first) {
          if (first >= p.rot) return;
#pragma unroll
          for (int e = 0; e < U; e += 2) {
            const int j = (first + e) / 2;
            const float c = cs[u.row][j], s = sn[u.row][j], y = x[e], z = x[e + 1];
            x[e] = y * c - z * s;
            x[e + 1] = y * s + z * c;
          }
        };
        turn(a, u.ca);
        turn(b, u.cb);
      }
      if (out) {
        S* dst = out + u.row * part.out.row + u.h * p.hd;
        store_chunk<S, U>(dst + u.ca, a);
        store_chunk<S, U>(dst + u.cb, b);
      }
    }
    if (kind != 0) {
      const int64_t to = at + (uint32_t)u.h * p.cache.page.d * (uint32_t)p.hd;
      if constexpr (E4M3) {
        const float inv = 1.f / u.scale;
        uint8_t* dst = static_cast<uint8_t*>(p.cache.data) + to;
        store_e4m3<U>(dst + u.ca, a, inv);
        store_e4m3<U>(dst + u.cb, b, inv);
      } else {
        S* dst = static_cast<S*>(p.cache.data) + to;
        store_chunk<S, U>(dst + u.ca, a);
        store_chunk<S, U>(dst + u.cb, b);
      }
    }
  };

  const int total = rows * part.units;
  int x = tid;
  Unit u;
  if (x < total) u = fetch(x);
  // the rows' places, and the angles
  for (int a = tid; a < rows * MAX_FREQ; a += 256) {
    const int r = a / MAX_FREQ, j = a % MAX_FREQ, t = t0 + r;
    if (j > 0 && (kind == 2 || j >= half)) continue;
    const int pos = p.pos[t];
    if (j == 0) {
      int64_t at = -1;
      if (pos >= 0) {
        const int page = paged_page(p.cache, p.seq ? p.seq[t] : t, pos);
        if (page < 0 && p.fault) *p.fault = 1;
        const int place = pos - (int)(div_of(p.cache.page, (uint32_t)pos) * p.cache.page.d);
        if (page >= 0) at = (paged_row(p.cache, i, kind == 2, page, 0) + place) * p.hd;
      }
      s_at[r] = at;
    }
    if (j < half && pos >= 0 && kind != 2) {
      const double turns = (double)pos * p.turns[j];
      sincospif(2.f * (float)(turns - rint(turns)), &sn[r][j], &cs[r][j]);
    }
  }
  __syncthreads();
  while (x < total) {
    finish(u);
    x += 256;
    if (x < total) u = fetch(x);
  }
}

template <typename S, bool E4M3>
hipError_t launch_append(AppendParams p, int heads, hipStream_t s) {
  // 16 bytes of a 16-bit row at a time, unless half the rotated dimensions end inside of them
  // (heads of 104: 8 bytes)
  const int U = sizeof(S) == 2 && (p.neighbours || p.rot % 16 == 0) ? 8 : 4;
  // One unit per thread: rows for 256 units (8192 rows of 8 x 48 heads of 128, with 512 and 1024
  // units a block: 343, 351 and 359 us), fewer where not every CU had two blocks of each kind.
  const int spread = (int)std::max<int64_t>(1, (int64_t)p.T * p.cache.n / 512);
  unsigned blocks = 0;
  for (int k = 0; k < 3; ++k) {
    Part& part = p.part[k];
    part.first = blocks;
    part.units = (k == 0 ? heads : p.cache.heads) * (p.hd / (2 * U));
    part.per_row = fast_div((uint32_t)part.units);
    part.rows = std::max(1, std::min({MAX_ROWS, 256 / part.units, spread}));
    if (part.in.data) blocks += (unsigned)((p.T + part.rows - 1) / part.rows);
  }
  const dim3 grid(blocks, (unsigned)p.cache.n);
  if (U == 4) hipLaunchKernelGGL((append_kernel<S, E4M3, 4>), grid, dim3(256), 0, s, p);
  else if constexpr (sizeof(S) == 2)
    hipLaunchKernelGGL((append_kernel<S, E4M3, 8>), grid, dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace

const char* paged_view(const kraken_paged_cache* c, bool with_data, PagedView* view,
                       kraken_status* status) noexcept {
  *status = KRAKEN_ERR_INVALID_ARG;
  if (!c) return "cache is NULL";
  if (c->dtype < KRAKEN_DTYPE_F32 || c->dtype > KRAKEN_DTYPE_E4M3) {
    *status = KRAKEN_ERR_UNSUPPORTED;
    return "unknown dtype of the cache";
  }
  if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128) {
    *status = KRAKEN_ERR_UNSUPPORTED;
    return "head_dim must be 32, 64 or 128";
  }
  if (c->n_sub < 1 || c->n_sub > 65535 || c->n_kv_heads < 1 || c->n_kv_heads > 65535 ||
      c->num_pages < 1 || c->page_size < 1 || c->pages_per_seq < 1)
    return "non-positive (or too large) size in the cache";
  if (c->num_seqs < 1 || c->num_seqs > KRAKEN_MAX_SEQS)
    return "num_seqs out of 1..KRAKEN_MAX_SEQS";
  if (c->table_ld < c->pages_per_seq) return "table_ld is below pages_per_seq";
  if ((int64_t)c->pages_per_seq * c->page_size >= (1ll << 31))
    return "pages_per_seq * page_size must stay below 2^31";
  const int es = c->dtype == KRAKEN_DTYPE_E4M3 ? 1 : c->dtype == KRAKEN_DTYPE_F32 ? 4 : 2;
  if ((int64_t)c->n_kv_heads * c->head_dim * es * c->page_size >= (1ll << 31)) {
    *status = KRAKEN_ERR_UNSUPPORTED;
    return "a page of one sub-layer's keys must stay below 2^31 bytes";
  }
  // (elements of the cache must fit 62 bits)
  const double elems = 2.0 * c->n_sub * c->num_pages * c->n_kv_heads * (double)c->page_size *
                       c->head_dim;
  if (elems >= 4.0e18) return "the cache has too many elements";
  if (with_data) {
    if (!c->pages || !c->table) return "pages or table is NULL";
    if (reinterpret_cast<uintptr_t>(c->pages) % 16 != 0) return "pages is not 16-byte aligned";
    if ((c->dtype == KRAKEN_DTYPE_E4M3) != (c->scales != nullptr))
      return "scales go with a cache of E4M3, and with no other";
  }
  if (view) {
    view->data = c->pages;
    view->table = c->table;
    view->scales = c->scales;
    view->n = c->n_sub;
    view->heads = c->n_kv_heads;
    view->pages = c->num_pages;
    view->seqs = c->num_seqs;
    view->per_seq = c->pages_per_seq;
    view->table_ld = c->table_ld;
    view->page = fast_div((uint32_t)c->page_size);
  }
  *status = KRAKEN_OK;
  return nullptr;
}

const char* check_rows(const kraken_rows* r, int n, int64_t T, int es,
                       int64_t out_width) noexcept {
  if (!r || T == 0) return nullptr;
  if (!r->data) return "rows without data";
  const int64_t sub = n > 1 ? r->sub_stride : 0, row = T > 1 ? r->row_stride : 0;
  if (sub < 0 || row < 0) return "negative stride";
  if (reinterpret_cast<uintptr_t>(r->data) % 16 != 0 || sub % (16 / es) != 0 ||
      row % (16 / es) != 0)
    return "rows and their strides must be aligned to 16 bytes";
  if (out_width > 0 && rows_overlap(n, T, sub, row, out_width))
    return "the rows of an output overlap";
  return nullptr;
}

}  // namespace kraken

using namespace kraken;

namespace {

kraken_status fail(kraken_status s, const char* msg) { return (kraken_status)set_error(s, msg); }

RowsView rows_view(const kraken_rows* r) {
  return r ? RowsView{r->data, r->sub_stride, r->row_stride} : RowsView{nullptr, 0, 0};
}

}  // namespace

extern "C" {

size_t kraken_paged_cache_bytes(const kraken_paged_cache* c) {
  kraken_status st;
  if (paged_view(c, false, nullptr, &st)) return 0;
  const size_t es = c->dtype == KRAKEN_DTYPE_E4M3 ? 1 : c->dtype == KRAKEN_DTYPE_F32 ? 4 : 2;
  return (size_t)c->n_sub * 2 * c->num_pages * c->n_kv_heads * c->page_size * c->head_dim * es;
}

kraken_status kraken_op_paged_append(int32_t dtype, const kraken_rows* q, const kraken_rows* k,
                                     const kraken_rows* v, const kraken_rows* q_out,
                                     const kraken_rows* k_out, int32_t T, int32_t n_heads,
                                     const int32_t* pos, const int32_t* seq,
                                     const double* inv_freq, int32_t rot_dim, int32_t neighbours,
                                     const kraken_paged_cache* cache, int32_t* fault,
                                     void* stream) {
  AppendParams p;
  kraken_status st;
  if (const char* msg = paged_view(cache, true, &p.cache, &st)) return fail(st, msg);
  if (dtype < KRAKEN_DTYPE_F32 || dtype > KRAKEN_DTYPE_F16)
    return fail(KRAKEN_ERR_UNSUPPORTED, "unknown dtype");
  const bool e4m3 = cache->dtype == KRAKEN_DTYPE_E4M3;
  if (e4m3 ? dtype == KRAKEN_DTYPE_F32 : cache->dtype != dtype)
    return fail(KRAKEN_ERR_UNSUPPORTED,
                "the cache has the rows' dtype, or is E4M3 with BF16 or F16 rows");
  if (T < 0) return fail(KRAKEN_ERR_INVALID_ARG, "T is negative");
  if (T > 1 << 22) return fail(KRAKEN_ERR_UNSUPPORTED, "T above 4194304");
  if (T > 0 && (!k || !v || !pos)) return fail(KRAKEN_ERR_INVALID_ARG, "k, v or pos is NULL");
  if (!q != !q_out) return fail(KRAKEN_ERR_INVALID_ARG, "q and q_out go together");
  if (n_heads < 1 || n_heads > 65535 || n_heads % cache->n_kv_heads != 0)
    return fail(KRAKEN_ERR_INVALID_ARG, "n_kv_heads does not divide n_heads");
  if (!seq && T > cache->num_seqs)
    return fail(KRAKEN_ERR_INVALID_ARG, "more rows than sequences, and no seq");
  if (rot_dim < 0 || rot_dim > cache->head_dim || rot_dim % 8 != 0)
    return fail(KRAKEN_ERR_INVALID_ARG, "rot_dim must be a multiple of 8 in 0..head_dim");
  if (rot_dim > 0 && !inv_freq) return fail(KRAKEN_ERR_INVALID_ARG, "inv_freq is NULL");
  const int es = dtype == KRAKEN_DTYPE_F32 ? 4 : 2;
  for (const kraken_rows* r : {q, k, v, q_out, k_out}) {
    const int64_t width = r == q_out ? (int64_t)n_heads * cache->head_dim
                          : r == k_out ? (int64_t)cache->n_kv_heads * cache->head_dim : 0;
    if (const char* msg = check_rows(r, cache->n_sub, T, es, width))
      return fail(KRAKEN_ERR_INVALID_ARG, msg);
  }
  for (int j = 0; j < rot_dim / 2; ++j) {
    if (!isfinite(inv_freq[j])) return fail(KRAKEN_ERR_INVALID_ARG, "inv_freq is not finite");
    p.turns[j] = inv_freq[j] * 0.15915494309189533577;     // 1 / (2 pi)
  }
  if (T == 0) return KRAKEN_OK;
  p.part[0].in = rows_view(q); p.part[1].in = rows_view(k); p.part[2].in = rows_view(v);
  p.part[0].out = rows_view(q_out); p.part[1].out = rows_view(k_out);
  p.part[2].out = rows_view(nullptr);
  p.pos = pos; p.seq = seq; p.fault = fault;
  p.T = T; p.hd = cache->head_dim; p.rot = rot_dim;
  p.neighbours = neighbours != 0;
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e;
  if (dtype == KRAKEN_DTYPE_F32) e = launch_append<float, false>(p, n_heads, s);
  else if (dtype == KRAKEN_DTYPE_BF16)
    e = e4m3 ? launch_append<bf16, true>(p, n_heads, s) : launch_append<bf16, false>(p, n_heads, s);
  else e = e4m3 ? launch_append<f16, true>(p, n_heads, s) : launch_append<f16, false>(p, n_heads, s);
  if (e == hipSuccess) return KRAKEN_OK;
  return fail(KRAKEN_ERR_HIP, hipGetErrorString(e));
}

}  // extern "C"
