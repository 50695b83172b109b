// Every token of a sequence is in exactly one of its slices, and no range leaves [0, tokens].
#include <stdio.h>

#include <initializer_list>

#include "../paper_2510_16415_amd/csrc/loss_ranges.h"

using namespace mecefo;

int main() {
  const int64_t tokens = 1000, far = (int64_t)1 << 62;
  const int64_t at[] = {-far, -5, 0, 1, 63, 64, 65, 500, 999, 1000, 1001, far};
  for (int64_t a : at)
    for (int64_t b : at)
      for (int n : {1, 2, 3, 7, 64}) {
        const TokenRange r = token_range(a, b, tokens);
        if (r.lo < 0 || r.hi < r.lo || r.hi > tokens) return printf("range %lld %lld\n", (long long)a, (long long)b), 1;
        if (a >= 0 && a <= b && b <= tokens && (r.lo != a || r.hi != b)) return printf("changed %lld %lld\n", (long long)a, (long long)b), 1;
        int64_t next = r.lo;
        for (int j = 0; j < n; ++j) {
          const TokenRange s = token_slice(r, j, n);
          if (s.lo != next || s.hi < s.lo || s.hi > r.hi) return printf("slice %d of %d\n", j, n), 1;
          next = s.hi;
        }
        if (next != r.hi) return printf("slices end at %lld of %lld\n", (long long)next, (long long)r.hi), 1;
      }
  const TokenRange r = token_range(3, ((int64_t)1 << 29) - 1, ((int64_t)1 << 29) - 1);      // the longest
  int64_t next = r.lo;
  for (int j = 0; j < 64; ++j) {
    const TokenRange s = token_slice(r, j, 64);
    if (s.lo != next) return printf("long slice %d\n", j), 1;
    next = s.hi;
  }
  if (next != r.hi) return printf("long slices\n"), 1;
  puts("ok");
  return 0;
}
