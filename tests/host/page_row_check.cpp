// Every row of small pools and tables, entries that are no page, and the largest pools.
#include <cstdio>
#include <cstdlib>
#include <set>
#include <vector>
#include "page_row.h"

static void need(bool ok, const char* what) {
  if (ok) return;
  std::printf("wrong: %s\n", what);
  std::exit(1);
}

int main() {
  for (int shift : {4, 5, 7})
    for (int n_pages : {1, 3, 8})
      for (int max_pages : {1, 2, 5})
        for (int heads : {1, 3}) {
          const int32_t odd[] = {-1, n_pages, INT32_MAX, INT32_MIN, n_pages - 1, 0};
          for (int kind = 0; kind < 6; ++kind) {
            std::vector<int32_t> table(2 * max_pages);
            for (int i = 0; i < 2 * max_pages; ++i) table[i] = i % 2 ? odd[kind] : i / 2 % n_pages;
            PcPages p = {};
            p.table = table.data(); p.n_pages = n_pages; p.shift = shift; p.max_pages = max_pages;
            for (long long b = 0; b < 2; ++b)
              for (int g = 0; g < heads; ++g)
                for (long long row = -70; row < (long long)(max_pages + 2) << shift; ++row) {
                  const long long at = pc_page_row(p, b, row, g, heads);
                  const bool in = row >= 0 && row < (long long)max_pages << shift;
                  const int page = in ? table[b * max_pages + (row >> shift)] : -1;
                  if (!in || page < 0 || page >= n_pages) { need(at == -1, "a row that is not there"); continue; }
                  need(at >= 0 && at < (long long)n_pages * heads << shift, "inside of the pool");
                  need(at == ((long long)page * heads + g) * (1 << shift) + row % (1 << shift), "its place");
                }
          }
        }
  const int32_t last[] = {INT32_MAX - 1};
  PcPages p = {};
  p.table = last; p.n_pages = INT32_MAX; p.shift = 16; p.max_pages = 1;
  need(pc_page_row(p, 0, 65535, 65535, 65536) == ((long long)(INT32_MAX - 1) * 65536 + 65535) * 65536 + 65535, "the largest pool");
  need(pc_page_row(p, 0, 65536, 0, 1) == -1 && pc_page_row(p, 0, 1LL << 40, 0, 1) == -1 && pc_page_row(p, 0, -(1LL << 40), 0, 1) == -1, "rows far away");
  std::printf("ok\n");
}
