// Appending keys and values to a paged KV cache, with the rotation of queries and keys by
// their positions on the way.
//
// Rotation: row t turns the pair (a, b) of dimensions j and j + rot / 2 (or 2 j and 2 j + 1) of
// every head by the angle pos f_j: (a cos - b sin, a sin + b cos).  At position 10^6 an fp32
// product pos f_j is off by up to 2^-5 radians, so the angle is formed in 64 bits, in turns, its
// whole turns are dropped there, and only the rest in [-1/2, 1/2] goes to fp32.
#include <hip/hip_runtime.h>
#include <math.h>

#include "kraken_internal.hpp"
#include "paged.hpp"

namespace kraken {
namespace {

constexpr int MAX_FREQ = 64;          // pairs of a head of 128

struct RowsView {
  void* data;
  int64_t sub, row;                   // elements between sub-layers and between rows
};

struct AppendParams {
  RowsView q, k, v, q_out, k_out;     // (data NULL: absent)
  PagedView cache;
  const int32_t* pos;
  const int32_t* seq;
  int32_t* fault;
  int T, heads, hd, rot, neighbours;
  double turns[MAX_FREQ];             // inv_freq / (2 pi)
};

template <typename T, int N>
struct alignas(sizeof(T) * N) Vec {
  T v[N];
};

// Nearest e4m3 of x (ties to even), beyond +-448 the largest; a NaN stays one (the hardware's
// conversion of a NaN, which the clamp alone would lose).
__device__ __forceinline__ uint8_t to_e4m3(float x) {
  const float c = x != x ? x : fminf(fmaxf(x, -448.f), 448.f);
  return (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, c, 0, false);
}

// Chunk of U elements: as fp32, and back.
template <typename S, int U>
__device__ __forceinline__ void load_chunk(const S* p, float* x) {
  const Vec<S, U> c = *reinterpret_cast<const Vec<S, U>*>(p);
#pragma unroll
  for (int e = 0; e < U; ++e) x[e] = (float)c.v[e];
}
template <typename S, int U>
__device__ __forceinline__ void store_chunk(S* p, const float* x) {
  Vec<S, U> c;
#pragma unroll
  for (int e = 0; e < U; ++e) c.v[e] = (S)x[e];
  *reinterpret_cast<Vec<S, U>*>(p) = c;
}
template <int U>
__device__ __forceinline__ void store_e4m3(uint8_t* p, const float* x, float scale) {
  Vec<uint8_t, U> c;
#pragma unroll
  for (int e = 0; e < U; ++e) c.v[e] = to_e4m3(x[e] / scale);
  *reinterpret_cast<Vec<uint8_t, U>*>(p) = c;
}

// Block (row t, sub-layer i).  Unit u of a row: two chunks of U elements of one head, which a
// thread turns together: pairs (j, j + rot / 2) chunk by chunk, neighbouring pairs and the
// dimensions that are not turned as two consecutive chunks.
template <typename S, bool E4M3, int U>
__global__ __launch_bounds__(256) void append_kernel(AppendParams p) {
  __shared__ float cs[MAX_FREQ], sn[MAX_FREQ];
  const int t = blockIdx.x, i = blockIdx.y, tid = threadIdx.x;
  const int pos = p.pos[t];
  if (pos < 0) return;
  const int page = paged_page(p.cache, p.seq ? p.seq[t] : t, pos);
  if (page < 0) {
    if (tid == 0 && p.fault) *p.fault = 1;
    return;
  }
  if (tid < p.rot / 2) {
    const double turns = (double)pos * p.turns[tid];
    sincospif(2.f * (float)(turns - rint(turns)), &sn[tid], &cs[tid]);
  }
  __syncthreads();
  const int per_head = p.hd / (2 * U), half = p.rot / 2;
  const int nq = p.q.data ? p.heads : 0, nkv = p.cache.heads;
  const int place = pos - (int)div_of(p.cache.page, (uint32_t)pos) * (int)p.cache.page.d;
  for (int u = tid; u < (nq + 2 * nkv) * per_head; u += 256) {
    const int head = u / per_head, w = u % per_head;
    const int kind = head < nq ? 0 : head < nq + nkv ? 1 : 2;          // q, k, v
    const int h = kind == 0 ? head : kind == 1 ? head - nq : head - nq - nkv;
    const RowsView& src = kind == 0 ? p.q : kind == 1 ? p.k : p.v;
    const S* in = static_cast<const S*>(src.data) + i * src.sub + t * src.row + h * p.hd;
    const bool turn = kind != 2 && w * 2 * U < p.rot;
    const bool halves = turn && !p.neighbours;
    const int ca = halves ? w * U : w * 2 * U, cb = halves ? half + w * U : ca + U;
    float a[U], b[U];
    load_chunk<S, U>(in + ca, a);
    load_chunk<S, U>(in + cb, b);
    if (halves) {
#pragma unroll
      for (int e = 0; e < U; ++e) {
        const float c = cs[ca + e], s = sn[ca + e], x = a[e], y = b[e];
        a[e] = x * c - y * s;
        b[e] = x * s + y * c;
      }
    } else if (turn) {
#pragma unroll
      for (int e = 0; e < U; e += 2) {
        const int j = (ca + e) / 2, l = (cb + e) / 2;
        const float x = a[e], y = a[e + 1], z = b[e], r = b[e + 1];
        a[e] = x * cs[j] - y * sn[j];
        a[e + 1] = x * sn[j] + y * cs[j];
        b[e] = z * cs[l] - r * sn[l];
        b[e + 1] = z * sn[l] + r * cs[l];
      }
    }
    const RowsView& dst = kind == 0 ? p.q_out : p.k_out;
    if (kind != 2 && dst.data) {
      S* out = static_cast<S*>(dst.data) + i * dst.sub + t * dst.row + h * p.hd;
      store_chunk<S, U>(out + ca, a);
      store_chunk<S, U>(out + cb, b);
    }
    if (kind != 0) {
      const int64_t at = (paged_row(p.cache, i, kind - 1, page, h) + place) * p.hd;
      if constexpr (E4M3) {
        const float scale = p.cache.scales[(i * 2 + kind - 1) * nkv + h];
        uint8_t* out = static_cast<uint8_t*>(p.cache.data) + at;
        store_e4m3<U>(out + ca, a, scale);
        store_e4m3<U>(out + cb, b, scale);
      } else {
        S* out = static_cast<S*>(p.cache.data) + at;
        store_chunk<S, U>(out + ca, a);
        store_chunk<S, U>(out + cb, b);
      }
    }
  }
}

template <typename S, bool E4M3>
hipError_t launch_append(const AppendParams& p, hipStream_t s) {
  const dim3 grid((unsigned)p.T, (unsigned)p.cache.n);
  hipLaunchKernelGGL((append_kernel<S, E4M3, 4>), grid, dim3(256), 0, s, p);
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
  // (elements of the cache must fit 62 bits; the first three factors stay below 2^64)
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
  if (reinterpret_cast<uintptr_t>(r->data) % 16 != 0 || sub * es % 16 != 0 || row * es % 16 != 0)
    return "rows and their strides must be aligned to 16 bytes";
  if ((n > 1 && sub < out_width) || (T > 1 && row < out_width))
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
  p.q = rows_view(q); p.k = rows_view(k); p.v = rows_view(v);
  p.q_out = rows_view(q_out); p.k_out = rows_view(k_out);
  p.pos = pos; p.seq = seq; p.fault = fault;
  p.T = T; p.heads = n_heads; p.hd = cache->head_dim; p.rot = rot_dim;
  p.neighbours = neighbours != 0;
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e;
  if (dtype == KRAKEN_DTYPE_F32) e = launch_append<float, false>(p, s);
  else if (dtype == KRAKEN_DTYPE_BF16)
    e = e4m3 ? launch_append<bf16, true>(p, s) : launch_append<bf16, false>(p, s);
  else e = e4m3 ? launch_append<f16, true>(p, s) : launch_append<f16, false>(p, s);
  if (e == hipSuccess) return KRAKEN_OK;
  return fail(KRAKEN_ERR_HIP, hipGetErrorString(e));
}

}  // extern "C"
