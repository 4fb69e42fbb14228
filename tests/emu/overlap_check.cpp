// Region::meets() against the bytes themselves: regions that share one are never taken apart; regions that share none are
// taken apart where their ranges lie apart, where their strides are equal, or where one of them is a single run of bytes.
#include <stdio.h>

#include <vector>

#include "../../paper_1412_2302_amd/csrc/overlap.h"

using namespace ax;

static void mark(std::vector<char>& m, long at, long rows, long stride, long bytes) {
  for (long r = 0; r < rows; ++r)
    for (long i = 0; i < bytes; ++i) m[at + r * stride + i] = 1;
}

int main() {
  const long base = 1 << 20;
  long pairs = 0;
  for (long rows_a : {0, 1, 2, 3})
    for (long stride_a : {4, 5, 9})
      for (long bytes_a : {1, 3, 4})
        for (long rows_b : {0, 1, 2, 4})
          for (long stride_b : {4, 5, 9, 12})
            for (long bytes_b : {1, 2, 4})
              for (long at = -60; at <= 60; ++at) {
                std::vector<char> a(400, 0), b(400, 0);
                mark(a, 150, rows_a, stride_a, bytes_a);
                mark(b, 150 + at, rows_b, stride_b, bytes_b);
                bool share = false;
                for (size_t i = 0; i < a.size(); ++i) share |= a[i] && b[i];
                const Region p((const void*)(base + 150), rows_a, stride_a, bytes_a), q((const void*)(base + 150 + at), rows_b, stride_b, bytes_b);
                const bool run = rows_a <= 1 || rows_b <= 1 || stride_a == bytes_a || stride_b == bytes_b;
                const bool meets = p.meets(q);
                if (meets != q.meets(p) || (share && !meets) || (!share && meets && (run || stride_a == stride_b))) {
                  printf("FAIL rows %ld %ld strides %ld %ld bytes %ld %ld at %ld: share %d, meets %d %d\n", rows_a, rows_b, stride_a, stride_b,
                         bytes_a, bytes_b, at, share, meets, q.meets(p));
                  return 1;
                }
                ++pairs;
              }
  // nothing, and strides past the address space
  const Region none(nullptr, 10, 4, 4), all((const void*)base, 1L << 40, 1L << 40, 4), far_off((const void*)(base + (1L << 50) + 8), 1, 4, 4);
  if (none.meets(all) || all.meets(none) || !all.meets(Region((const void*)(base + (1L << 50)), 1, 4, 4)) || all.meets(far_off)) {
    printf("FAIL ends\n");
    return 1;
  }
  printf("OK %ld pairs\n", pairs);
  return 0;
}
