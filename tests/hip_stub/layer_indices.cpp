// The index arithmetic of layer_index.h at the ends of the sizes that the calls take, under UBSan: what the kernels do with it, thread
// by thread, without memory.
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <vector>

#include "layer_index.h"

namespace {
int g_failures = 0;
void expect(bool ok, const char* what, long a = 0, long b = 0) {
  if (ok) return;
  std::fprintf(stderr, "%s (%ld, %ld)\n", what, a, b);
  ++g_failures;
}

// The rows of a chunk as a work-group that takes `at_once` of them walks them: every row once, none outside.
void walk(const svd::ChunkAt& c, int at_once) {
  std::vector<int> seen(c.row1 - c.row0);
  for (int mine = 0; mine < at_once; ++mine)
    for (int row = svd::row_behind(c.row0, mine, c.row1); row < c.row1; row = svd::row_behind(row, at_once, c.row1)) {
      expect(row >= c.row0, "row of the chunk", row, c.row0);
      if (row < c.row0) return;
      ++seen[row - c.row0];
    }
  expect(std::all_of(seen.begin(), seen.end(), [](int n) { return n == 1; }), "every row of a chunk once", c.row0, c.row1);
}

void rows() {
  for (int L : {1, 2, 15, 16, 17, 1000, INT32_MAX - 16, INT32_MAX - 15, INT32_MAX - 1, INT32_MAX})
    for (int first : {0, 1, L / 2, L - 1})
      for (int group : {0, 1, 7, 1 << 30, INT32_MAX})
        for (int per : {1, 16, 48, 256, 4096, 1 << 16}) {
          if (first >= L) continue;
          const int groups = svd::row_chunks(L, first, group, per).groups;
          if (per < 256 && L > 1000 && group > 0) continue;   // chunks past 2^31 / 256: refused by the grid's size
          const svd::RowChunks ch = svd::row_chunks(L, first, group, per);
          expect(groups >= 1 && ch.per_entry >= 1, "chunks", L, per);
          for (int id : {0, ch.per_entry / 2, ch.per_entry - 2, ch.per_entry - 1}) {
            if (id < 0 || id >= ch.per_entry) continue;
            const svd::ChunkAt c = svd::chunk_at(ch, id);
            expect(c.row0 >= 0 && c.row0 < c.row1 && c.row1 <= L && c.row1 - c.row0 <= per, "chunk", c.row0, c.row1);
            for (int at_once : {1, 4, 8, 16}) walk(c, at_once);
          }
          expect(svd::chunk_at(ch, ch.per_entry - 1).row1 == L, "the last row", L, per);
        }
}

}  // namespace

int main(int argc, char** argv) {
  const char* what = argc > 1 ? argv[1] : "";
  if (!std::strcmp(what, "rows")) rows();
  else expect(false, "which part?");
  if (!g_failures) std::printf("%s: ok\n", what);
  return g_failures != 0;
}
