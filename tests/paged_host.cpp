// Host run of the arithmetic that keeps the paged cache's kernels inside their arrays (csrc/paged.h), over values that no caller
// should hand in: what the device arrays say, whatever it is, has to give rows, entries and pages inside the batch's limits.
#include <limits.h>
#include <stdio.h>

#include "paged.h"

int main() {
  const int odd[] = {INT_MIN, -1000000, -17, -1, 0, 1, 15, 16, 17, 300, 1 << 20, 1 << 30, INT_MAX};
  const int sizes[] = {1, 7, 64, 1000, 1 << 30};
  long cases = 0;
  for (int len : odd)
    for (int r0 : odd)
      for (int r1 : odd)
        for (int n_rows : sizes)
          for (int max_new : sizes)
            for (int max_len : sizes)
              for (int pages : {1, 3, 1 << 20, INT_MAX})
                for (int shift = 4; shift <= 8; ++shift) {
                  const qp::PagedSeq q = qp::paged_seq(len, r0, r1, n_rows, max_new, max_len, pages, shift);
                  const bool ok = q.len >= 0 && q.len <= max_len && (q.len == 0 || (long long)(q.len - 1) >> shift < pages) &&
                                  q.row0 >= 0 && q.n >= 0 && q.n <= max_new && (long long)q.row0 + q.n <= n_rows &&
                                  (long long)q.base + q.n <= (long long)q.len && q.base >= -n_rows;
                  ++cases;
                  if (!ok) {
                    printf("FAILED len %d rows %d..%d of %d, limits %d %d, %d pages\n", len, r0, r1, n_rows, max_new, max_len, pages);
                    return 1;
                  }
                }
  // ordinary ones: the last rows of a sequence are its last entries
  const qp::PagedSeq q = qp::paged_seq(100, 5, 9, 20, 8, 4096, 10, 4);
  if (q.len != 100 || q.row0 != 5 || q.n != 4 || q.base != 96) return printf("FAILED ordinary\n"), 1;
  if (qp::paged_seq(100, 5, 9, 20, 8, 4096, 3, 4).len != 48) return printf("FAILED table\n"), 1;
  if (qp::paged_seq(2, 0, 5, 20, 8, 4096, 3, 4).base != -3) return printf("FAILED rows without entries\n"), 1;
  for (int page : odd)
    if (qp::paged_page_ok(page, 17) != (page >= 0 && page < 17)) return printf("FAILED page %d\n", page), 1;
  if (qp::paged_row(1 << 20, 7, 255, 8, 8) != ((((size_t)1 << 20) * 8 + 7) << 8) + 255) return printf("FAILED row\n"), 1;
  printf("ALL OK %ld\n", cases);
  return 0;
}
