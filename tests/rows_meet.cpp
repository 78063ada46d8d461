// Host program of tests/test_packed_edges.py.  Reads layouts from standard input, two to a line: address, bytes, dimensions, then count and stride of
// each; prints whether rows of the two meet and whether they are the same rows.
#include <stdio.h>

#include "../paper_2506_04708_b200/csrc/overlap.cuh"

static bool read(stand::RowSet& r) {
  long long at, bytes, count, stride;
  if (scanf("%lld %lld %d", &at, &bytes, &r.dims) != 3) return false;
  r.at = (const void*)at;
  r.bytes = bytes;
  for (int i = 0; i < r.dims; ++i) {
    if (scanf("%lld %lld", &count, &stride) != 2) return false;
    r.count[i] = count;
    r.stride[i] = stride;
  }
  return true;
}

int main() {
  stand::RowSet x, y;
  while (read(x) && read(y)) printf("%d%d\n", (int)stand::rows_meet(x, y), (int)stand::same_rows(x, y));
  return 0;
}
