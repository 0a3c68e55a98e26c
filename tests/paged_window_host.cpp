// Host run of the arithmetic that lets a row tile of windowed attention leave out entries (csrc/paged.h): in its own count of keys a
// tile meets every entry that one of its rows sees, once and in order, no entry outside the sequence, and no more keys than its launch was planned for.
#include <stdio.h>

#include "paged.h"

int main() {
  long cases = 0;
  for (int step : {16, 32, 64})
    for (int base : {-40, -1, 0, 1, 15, 16, 63, 64, 65, 200, 1000, 1023})
      for (int tokens : {1, 2, 7, 40})
        for (int window : {1, 2, 15, 16, 17, 31, 64, 65, 100, 500, 2000})
          for (int sinks : {0, 1, 4, 16, 17, 64, 65, 130, 900, 2000}) {
            const int end = base + tokens, len = end > 0 ? end : 0, max_len = 3000;  // entries up to the last row's own
            const qp::RowsGap g = qp::rows_gap(window, sinks, base, step);
            const int keys = len - g.gap, span = qp::rows_span(window, sinks, tokens, step, max_len);
            bool ok = g.gap >= 0 && g.jump >= 0 && g.gap % step == 0 && g.jump % step == 0 && keys >= 0 && keys <= span && (len == 0 || keys > 0);
            int next = 0;
            for (int e = 0; e < len && ok; ++e) {
              bool seen = false;  // by some row
              for (int p = base; p < end; ++p) seen = seen || (p >= 0 && e <= p && (e > p - window || e < sinks));
              const bool met = next < keys && g.entry(next) == e;
              ok = met || !seen;
              next += met;
            }
            ok = ok && next == keys;
            ++cases;
            if (!ok) {
              printf("FAILED step %d base %d tokens %d window %d sinks %d: jump %d gap %d\n", step, base, tokens, window, sinks, g.jump, g.gap);
              return 1;
            }
          }
  // the largest sizes
  const int most = 1 << 30;
  for (int first : {-most, -1, 0, most - 1})
    for (int window : {1, 17, most})
      for (int sinks : {0, 1, most - 1, most})
        for (int step : {16, 32, 64}) {
          const qp::RowsGap g = qp::rows_gap(window, sinks, first, step);
          const int span = qp::rows_span(window, sinks, most, step, most);
          const long long low = (long long)first - window + 1;
          if (g.gap < 0 || g.jump < 0 || span > most || span < 1 || (g.gap > 0 && (long long)g.jump + g.gap > low)) return printf("FAILED extremes\n"), 1;
        }
  printf("ALL OK %ld\n", cases);
  return 0;
}
