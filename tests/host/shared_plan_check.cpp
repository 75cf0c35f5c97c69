// Plans of pc_shared_attn calls over the sizes that the argument checks let through, built with the compiler's check for
// signed overflow: the estimates behind a plan stay numbers.  Prints the number of calls planned.
#include <initializer_list>
#include <stdio.h>
#include "parallelcomp_bench.h"

int main() {
  static const int segs[] = {0, 1, 7, 1 << 10, 1 << 20}, caps[] = {1, 33, 2048, 1 << 15, 1 << 20, 1 << 24};
  static const int fans[] = {1, 3, 300, 1 << 12, 1 << 20}, rows[] = {1, 8, 100, 1 << 15, 1 << 20}, heads[][2] = {{1, 1}, {8, 1}, {32, 8}, {32, 32}};
  const void* at = (const void*)256;                        // never followed
  int planned = 0;
  for (int eight = 0; eight < 4; ++eight)
    for (int s : segs) for (int c : caps) for (int t : caps) for (int f : fans) for (int n : rows) for (auto& h : heads) for (int p : {1, 5}) {
      const float* ks = eight & 1 ? (const float*)at : nullptr;
      const float* ts = eight & 2 ? (const float*)at : nullptr;
      const pc_row_cache prefix = {at, at, ks, ks, nullptr, 0, s, c}, tail = {at, at, ts, ts, nullptr, 0, 1, t};
      pc_shared_attn_plan_info info;
      if (pc_shared_attn_plan(s ? &prefix : nullptr, &tail, f * p, p, n, h[0], h[1], eight ? 128 : 64, &info) != PC_OK) continue;
      ++planned;
      const bool sane = info.alone || ((s == 0 || (info.prefix_rows > 0 && info.prefix_parts >= 1 && info.prefix_parts <= 64)) &&
                                       info.tail_rows > 0 && info.tail_parts >= 1 && info.tail_parts <= 64);
      if (!sane) { printf("a plan out of range\n"); return 1; }
    }
  printf("%d\n", planned);
  return 0;
}
