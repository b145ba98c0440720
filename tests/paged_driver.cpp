// The index arithmetic of the paged-cache entry points on the host: division by a page size,
// where a position lies (bad pages, sequences and positions among them), rows that share
// elements, and the equal runs of a list of tiles.  Exits 0 when every result is the plain computation's.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "../paper_2408_07802_amd/csrc/paged.hpp"

using namespace kraken;

#define CHECK(x)                                                \
  do {                                                          \
    if (!(x)) {                                                 \
      std::fprintf(stderr, "line %d: %s\n", __LINE__, #x);      \
      std::exit(1);                                             \
    }                                                           \
  } while (0)

int main() {
  std::mt19937_64 rng(1);
  // division: small and large divisors, powers of two and their neighbours
  std::vector<uint32_t> divisors{1, 2, 3, 5, 7, 16, 48, 4099, (1u << 31) - 1};
  for (int l = 2; l < 31; ++l)
    for (int k = -1; k <= 1; ++k) divisors.push_back((1u << l) + k);
  for (uint32_t d : divisors) {
    const FastDiv f = fast_div(d);
    for (int k = 0; k < 2000; ++k) {
      uint32_t x = (uint32_t)(rng() >> (33 + rng() % 31));
      if (k % 3 == 0) x = (uint32_t)((uint64_t)x * d & 0x7fffffff) / d * d;   // multiples
      if (k % 3 == 1 && x >= d) x = x / d * d - 1;                            // and one less
      CHECK(div_of(f, x) == x / d);
    }
    CHECK(div_of(f, 0x7fffffffu) == 0x7fffffffu / d);
  }

  // positions: the table is exactly as large as said (the sanitizer sees a read past it)
  for (int k = 0; k < 500; ++k) {
    PagedView c{};
    c.seqs = 1 + (int)(rng() % 4);
    c.per_seq = 1 + (int)(rng() % 6);
    c.table_ld = c.per_seq + (int)(rng() % 3);
    c.pages = 1 + (int)(rng() % 10);
    c.page = fast_div(1 + (uint32_t)(rng() % 40));
    std::vector<int32_t> table((size_t)(c.seqs - 1) * c.table_ld + c.per_seq);
    for (auto& e : table) e = (int32_t)(rng() % (c.pages + 4)) - 2;
    c.table = table.data();
    const int ps = (int)c.page.d;
    for (int b = -2; b < c.seqs + 2; ++b)
      for (int pos : {0, 1, ps - 1, ps, c.per_seq * ps - 1, c.per_seq * ps, 0x7fffffff}) {
        int want = -1;
        if (b >= 0 && b < c.seqs && pos / ps < c.per_seq) {
          const int page = table[(size_t)b * c.table_ld + pos / ps];
          if (page >= 0 && page < c.pages) want = page;
        }
        CHECK(paged_page(c, b, pos) == want);
      }
  }

  // rows that share elements: as counted one by one; and strides whose products pass 64 bits
  for (int k = 0; k < 4000; ++k) {
    const int n = 1 + (int)(rng() % 5), T = 1 + (int)(rng() % 5), width = 1 + (int)(rng() % 6);
    const int sub = (int)(rng() % 30), row = (int)(rng() % 30);
    std::vector<int> used(30 * 10 + 8, 0);
    bool want = false;
    for (int i = 0; i < n; ++i)
      for (int t = 0; t < T; ++t)
        for (int c = 0; c < width; ++c) want |= used[i * sub + t * row + c]++ > 0;
    CHECK(rows_overlap(n, T, sub, row, width) == want);
  }
  CHECK(!rows_overlap(65535, 1 << 22, INT64_MAX / 2, 1024, 512));
  CHECK(rows_overlap(65535, 1 << 22, INT64_MAX / 2, INT64_MAX / 2, 512));

  // runs: no more than asked for, every item in the run of its quotient, and no run longer
  // than an even share rounded up
  for (int k = 0; k < 20000; ++k) {
    const int total = k % 3 ? (int)(rng() % 5000) : (int)(rng() >> 33);
    const int runs = (int)(1 + rng() % 1024);
    const int len = run_length(fast_div((uint32_t)runs), total);
    CHECK(len >= 1 && len == (total == 0 ? 1 : (total + (int64_t)runs - 1) / runs));
    CHECK(((int64_t)total + len - 1) / len <= runs);
  }
  std::puts("paged index arithmetic holds");
  return 0;
}
