// Attention of one new token per sequence over a paged KV cache.
#include <hip/hip_runtime.h>
#include <math.h>

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
  int heads, group, max_len;
  float scale;
};

typedef uint8_t e4m3;

template <typename C>
__device__ __forceinline__ void load8(const C* p, float* x) {
  if constexpr (sizeof(C) == 1) {
    const uint2 c = *reinterpret_cast<const uint2*>(p);
    x[0] = __builtin_amdgcn_cvt_f32_fp8(c.x, 0);
    x[1] = __builtin_amdgcn_cvt_f32_fp8(c.x, 1);
    x[2] = __builtin_amdgcn_cvt_f32_fp8(c.x, 2);
    x[3] = __builtin_amdgcn_cvt_f32_fp8(c.x, 3);
    x[4] = __builtin_amdgcn_cvt_f32_fp8(c.y, 0);
    x[5] = __builtin_amdgcn_cvt_f32_fp8(c.y, 1);
    x[6] = __builtin_amdgcn_cvt_f32_fp8(c.y, 2);
    x[7] = __builtin_amdgcn_cvt_f32_fp8(c.y, 3);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)p[e];
  }
}

// Block (head, sequence, sub-layer), 4 waves.  HD / 8 lanes take one key; every group of lanes
// keeps the running maximum, sum and output of its keys, which are joined at the end.
template <typename S, typename C, int HD>
__global__ __launch_bounds__(256) void paged_attn_kernel(PagedAttnParams p) {
  constexpr int L = HD / 8, KEYS = 256 / L;
  __shared__ float sm[KEYS], sl[KEYS], so[KEYS][HD];
  const int h = blockIdx.x, b = blockIdx.y, i = blockIdx.z, tid = threadIdx.x;
  const int hkv = h / p.group, c = tid % L, g = tid / L;
  S* out = static_cast<S*>(p.out.data) + i * p.out.sub + b * p.out.row + h * HD;
  const int len = p.lens[b];
  bool bad = len < 0 || len > p.max_len;
  float q[8], o[8] = {}, m = -INFINITY, l = 0.f;
  load8(static_cast<const S*>(p.q.data) + i * p.q.sub + b * p.q.row + h * HD + c * 8, q);
  float ks = 1.f, vs = 1.f;
  if (sizeof(C) == 1) {
    ks = p.cache.scales[(i * 2) * p.cache.heads + hkv];
    vs = p.cache.scales[(i * 2 + 1) * p.cache.heads + hkv];
  }
  for (int k = g; k < len && !bad; k += KEYS) {
    const int page = paged_page(p.cache, b, k);
    if (page < 0) {
      bad = true;
      break;
    }
    const int place = k - (int)div_of(p.cache.page, (uint32_t)k) * (int)p.cache.page.d;
    float x[8];
    const C* data = static_cast<const C*>(p.cache.data);
    load8(data + (paged_row(p.cache, i, 0, page, hkv) + place) * HD + c * 8, x);
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(q[e], x[e], s);
#pragma unroll
    for (int w = 1; w < L; w <<= 1) s += __shfl_xor(s, w, 64);
    s *= p.scale * ks;
    const float mn = fmaxf(m, s), ref = mn == -INFINITY ? 0.f : mn;
    const float alpha = __expf(m - ref), e1 = __expf(s - ref);
    load8(data + (paged_row(p.cache, i, 1, page, hkv) + place) * HD + c * 8, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = o[e] * alpha + e1 * x[e];
    l = l * alpha + e1;
    m = mn;
  }
  if (c == 0) {
    sm[g] = m;
    sl[g] = l;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) so[g][c * 8 + e] = o[e];
  bad = __syncthreads_or(bad);
  if (bad && tid == 0 && p.fault) *p.fault = 1;
  if (tid >= HD) return;
  float M = -INFINITY, sum = 0.f, v = 0.f;
  for (int k = 0; k < KEYS; ++k) M = fmaxf(M, sm[k]);
  for (int k = 0; k < KEYS; ++k) {
    const float w = sm[k] == -INFINITY ? 0.f : __expf(sm[k] - M);
    sum += sl[k] * w;
    v += so[k][tid] * w;
  }
  out[tid] = bad ? (S)NAN : len == 0 ? (S)0.f : (S)(v * vs / sum);
}

template <typename S, typename C>
hipError_t launch_typed(const PagedAttnParams& p, int hd, hipStream_t s) {
  const dim3 grid((unsigned)p.heads, (unsigned)p.cache.seqs, (unsigned)p.cache.n);
  if (hd == 32) hipLaunchKernelGGL((paged_attn_kernel<S, C, 32>), grid, dim3(256), 0, s, p);
  else if (hd == 64) hipLaunchKernelGGL((paged_attn_kernel<S, C, 64>), grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL((paged_attn_kernel<S, C, 128>), grid, dim3(256), 0, s, p);
  return hipGetLastError();
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
  return 0;
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
  const int es = dtype == KRAKEN_DTYPE_F32 ? 4 : 2;
  for (const kraken_rows* r : {q, out})
    if (const char* msg = check_rows(r, cache->n_sub, cache->num_seqs, es,
                                     r == out ? (int64_t)n_heads * cache->head_dim : 0))
      return fail(KRAKEN_ERR_INVALID_ARG, msg);
  if (work_floats < 0 || work_floats < kraken_paged_attention_work_floats(cache, n_heads, max_len))
    return fail(KRAKEN_ERR_INVALID_ARG, "work is smaller than the call needs");
  if (reinterpret_cast<uintptr_t>(work) % 16 != 0)
    return fail(KRAKEN_ERR_INVALID_ARG, "work is not 16-byte aligned");
  const int hd = cache->head_dim;
  p.q = {q->data, q->sub_stride, q->row_stride};
  p.out = {out->data, out->sub_stride, out->row_stride};
  p.lens = lens; p.fault = fault;
  p.heads = n_heads; p.group = n_heads / cache->n_kv_heads; p.max_len = max_len;
  p.scale = scale != 0.f ? scale : (float)(1.0 / sqrt((double)hd));
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e;
  if (dtype == KRAKEN_DTYPE_F32) e = launch_typed<float, float>(p, hd, s);
  else if (dtype == KRAKEN_DTYPE_BF16)
    e = e4m3_cache ? launch_typed<bf16, e4m3>(p, hd, s) : launch_typed<bf16, bf16>(p, hd, s);
  else e = e4m3_cache ? launch_typed<f16, e4m3>(p, hd, s) : launch_typed<f16, f16>(p, hd, s);
  if (e == hipSuccess) return KRAKEN_OK;
  return fail(KRAKEN_ERR_HIP, hipGetErrorString(e));
}

}  // extern "C"
