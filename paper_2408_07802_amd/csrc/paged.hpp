// Paged KV cache: where a position lies, and the checks of a cache's description.  The index
// arithmetic is plain C++ that the host compiler takes too.
#pragma once

#include <stdint.h>

#include "../../include/kraken.h"

#ifdef __HIPCC__
#define KRAKEN_HD __host__ __device__ __forceinline__
#else
#define KRAKEN_HD inline
#endif

namespace kraken {

// Division of a non-negative 32-bit integer by a fixed d >= 1 as one multiplication: with
// 2^l >= d and m = ceil(2^(31 + l) / d), x / d = (x m) >> (31 + l) for every x < 2^31 (m d
// exceeds 2^(31 + l) by less than d <= 2^l, so x m / 2^(31 + l) exceeds x / d by less than 1 / d).
struct FastDiv {
  uint32_t d, mul, shift;
};
KRAKEN_HD FastDiv fast_div(uint32_t d) {
  uint32_t l = 0;
  while ((1ull << l) < d) ++l;
  return {d, (uint32_t)(((1ull << (31 + l)) + d - 1) / d), 31 + l};
}
KRAKEN_HD uint32_t div_of(FastDiv f, uint32_t x) {
  return (uint32_t)(((uint64_t)x * f.mul) >> f.shift);
}

// A paged cache as its kernels see it.  One layer: [n][2 (K, V)][pages][heads][page][hd].
struct PagedView {
  void* data;
  const int32_t* table;
  const float* scales;          // [n][2][heads], E4M3 only
  int n, heads, pages, seqs, per_seq, table_ld;
  FastDiv page;                 // places per page
};

// Page of position pos >= 0 of sequence `seq`, or -1 where the sequence, the position or the
// page is out of range.
KRAKEN_HD int paged_page(const PagedView& c, int seq, int pos) {
  if (seq < 0 || seq >= c.seqs) return -1;
  const int j = (int)div_of(c.page, (uint32_t)pos);
  if (j >= c.per_seq) return -1;
  const int page = c.table[(int64_t)seq * c.table_ld + j];
  return page >= 0 && page < c.pages ? page : -1;
}

// Row (of hd elements) of place 0 of head h of a page: K (kv = 0) or V (1) of sub-layer i.
KRAKEN_HD int64_t paged_row(const PagedView& c, int i, int kv, int page, int h) {
  return ((((int64_t)i * 2 + kv) * c.pages + page) * c.heads + h) * (int64_t)c.page.d;
}

// Items of each run where a list of total >= 0 (below 2^31) items is cut into at most runs.d
// equal ones (the last may be shorter): item x lies in run x / that.
KRAKEN_HD int run_length(FastDiv runs, int total) {
  const int q = (int)div_of(runs, (uint32_t)total);
  return q + ((uint32_t)q * runs.d < (uint32_t)total || q == 0 ? 1 : 0);
}

// Whether two of n x T rows of `width` elements, row t of sub-layer i at i sub + t row (strides >=
// 0), share an element.  Rows of equal i or t are a multiple of one stride apart; of rows di
// sub-layers apart, the nearest are those whose rows lie di sub / row apart, rounded either way.
inline bool rows_overlap(int n, int64_t T, int64_t sub, int64_t row, int64_t width) {
  if ((n > 1 && T > 0 && sub < width) || (T > 1 && row < width)) return true;
  if (n < 2 || T < 2) return false;
  const __int128 rows_end = (__int128)(T - 1) * row + width, subs_end = (__int128)(n - 1) * sub + width;
  if (sub >= rows_end || row >= subs_end) return false;    // one inside a step of the other
  for (int di = 1; di < n; ++di) {
    const __int128 at = (__int128)di * sub, dt = at / row;
    if (dt < T && at - dt * row < width) return true;
    if (dt + 1 < T && (dt + 1) * row - at < width) return true;
  }
  return false;
}

// Checks a cache's description (with_data: its pointers, too) and fills view; a message and
// *status otherwise.
const char* paged_view(const kraken_paged_cache* cache, bool with_data, PagedView* view,
                       kraken_status* status) noexcept;

// Checks n x T rows of elements of es bytes (NULL: absent); nullptr or a message.  out_width > 0:
// rows of that many elements that are written, which must not share elements.
const char* check_rows(const kraken_rows* r, int n, int64_t T, int es, int64_t out_width) noexcept;

}  // namespace kraken
