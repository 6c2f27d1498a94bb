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

// Every token and head of every entry once, by the threads of a launch; the places of the partial sums.
void rope_of(int L, int B, int D, const std::vector<int>& heads) {
  const int n = (int)heads.size(), most = *std::max_element(heads.begin(), heads.end()), blocks = svd::rope_blocks(L, D), tokens = svd::rope_tokens(D);
  auto once = [&](const std::vector<int>& seen, const char* what) {
    expect(std::all_of(seen.begin(), seen.end(), [](int k) { return k == 1; }), what, L, D);
  };
  const int splits = svd::rope_forward_splits(L, B, D, n, most);
  expect(splits >= 1 && splits <= most && (int64_t)n * splits <= 65535, "parts of the heads", splits, most);
  const svd::RopeWalk walk = svd::rope_walk(L, B, D, most);
  expect(walk.splits >= 1 && walk.splits <= most && walk.groups >= 1 && walk.groups <= svd::kRopePartials, "walk", walk.splits, walk.groups);
  for (int t = 0; t < n; ++t) {
    const int H = heads[t];
    std::vector<int> forward((size_t)B * H * L), backward(forward.size());
    auto take = [&](std::vector<int>& seen, int b, int block, const svd::HeadRange& r) {
      for (int k = 0; k < tokens; ++k) {
        const int l = block * tokens + k;
        if (l >= L) continue;
        for (int h = r.first; h < r.last; ++h) {
          expect(b >= 0 && b < B && h >= 0 && h < H, "inside", b, h);
          ++seen[((size_t)b * H + h) * L + l];
        }
      }
    };
    for (int block = 0; block < blocks; ++block)
      for (int b = 0; b < B; ++b)
        for (int part = 0; part < splits; ++part) take(forward, b, block, svd::heads_of_part(H, splits, part));
    once(forward, "forward, every row once");
    const int64_t units = (int64_t)blocks * B * walk.splits;
    for (int group = 0; group < walk.groups; ++group)
      for (int64_t i = group; i < units; i += walk.groups) {
        const svd::RopeUnit u = svd::rope_unit(i, blocks, walk.splits);
        expect(u.block < blocks && u.part < walk.splits, "unit", (long)i, u.block);
        take(backward, u.b, u.block, svd::heads_of_part(H, walk.splits, u.part));
      }
    once(backward, "backward, every row once");
  }
}
void rope() {
  for (int D : {64, 128})
    for (int L : {1, 15, 16, 17, 33, 1000, 8191})
      for (int B : {1, 3})
        for (const std::vector<int>& heads : {std::vector<int>{1}, {3}, {5, 2}, {2, 40}, {48, 48}}) rope_of(L, B, D, heads);
  // the most rows: nothing passes 32 bits
  for (int D : {64, 128}) {
    const int L = 1 << 27, blocks = svd::rope_blocks(L, D);
    expect((int64_t)blocks * svd::kRopeThreads < (int64_t)1 << 32 && svd::rope_forward_splits(L, 15, D, 2, 40) == 1, "launch", blocks);
    const svd::RopeWalk walk = svd::rope_walk(L, 15, D, 65535);
    const int64_t units = (int64_t)blocks * 15 * walk.splits;
    const svd::RopeUnit u = svd::rope_unit(units - 1, blocks, walk.splits);
    expect(u.b == 14 && u.block == blocks - 1 && u.part == walk.splits - 1 && u.block * svd::rope_tokens(D) + svd::rope_tokens(D) - 1 == L - 1, "last unit", u.b, u.block);
  }
}

// Every 8 elements of every block once, every scale byte once; by columns every element read and written once.
void quantise() {
  for (int C : {1, 100, 128, 129, 200, 256, 257, 512, 1000})
    for (int R : {1, 31, 32, 33, 70}) {
      const int blocks = svd::quant_blocks(C), at_once = svd::quant_rows_at_once(blocks), wide = (C + blocks * 128 - 1) / (blocks * 128);
      std::vector<int> seen((size_t)R * wide * blocks * 16), scales((size_t)R * wide * blocks);
      for (int gx = 0; gx < (R + svd::kQuantRows - 1) / svd::kQuantRows; ++gx)
        for (int gy = 0; gy < wide; ++gy)
          for (int thread = 0; thread < 256; ++thread)
            for (int i = 0; i < 8 / at_once; ++i) {
              const svd::QuantAt at = svd::quant_at(thread, blocks);
              const int k = at.row + i * at_once, row = gx * svd::kQuantRows + k, block = gy * blocks + at.block;
              expect(at.block < blocks && k < svd::kQuantRows && at.column % 8 == 0 && at.column < 128, "lane", thread, i);
              expect(at.block == svd::quant_at(thread & ~15, blocks).block && at.row == svd::quant_at(thread & ~15, blocks).row, "16 lanes a block", thread);
              if (row >= R) continue;
              ++seen[((size_t)row * wide * blocks + block) * 16 + at.column / 8];
              if ((thread & 15) == 0) ++scales[(size_t)row * wide * blocks + block];
            }
      expect(std::all_of(seen.begin(), seen.end(), [](int n) { return n == 1; }), "every element once", R, C);
      expect(std::all_of(scales.begin(), scales.end(), [](int n) { return n == 1; }), "every scale once", R, C);
    }
  std::vector<int> read(128 * 64), written(128 * 64);
  for (int thread = 0; thread < 256; ++thread) {
    for (int step = 0; step < 4; ++step)
      for (int j = 0; j < 8; ++j) {
        const svd::QuantPlace at = svd::quant_read_at(thread, step);
        ++read[at.row * 64 + at.column + j];
      }
    const svd::QuantPlace at = svd::quant_write_at(thread);
    for (int i = 0; i < 32; ++i) ++written[(at.row + i) * 64 + at.column];
    expect(at.column == svd::quant_write_at(thread & ~3).column, "4 lanes a column", thread);
  }
  expect(std::all_of(read.begin(), read.end(), [](int n) { return n == 1; }), "read once");
  expect(std::all_of(written.begin(), written.end(), [](int n) { return n == 1; }), "written once");
}

// The joins of the sums: every group once, every chunk of a group once by the threads of a channel.
void joins() {
  for (int n : {1, 2, 32767, 32768, 32769, 70000}) {
    std::vector<int> seen(n);
    const int y = n < svd::kJoinRow ? n : svd::kJoinRow, z = (n + svd::kJoinRow - 1) / svd::kJoinRow;
    for (int k = 0; k < z; ++k)
      for (int j = 0; j < y; ++j)
        if (const int at = svd::join_at(j, k); at < n) ++seen[at];
    expect(std::all_of(seen.begin(), seen.end(), [](int k) { return k == 1; }), "every group once", n);
  }
  for (int lanes : {8, 32})
    for (int n : {1, 5, 64, 65, 255, 256, 257, 1000, 507}) {
      std::vector<int> seen(n);
      for (int lane = 0; lane < lanes; ++lane)
        for (int i = lane; i < n; i += svd::kSumAhead * lanes)
          for (int u = 0; u < svd::kSumAhead; ++u)
            if (const int at = svd::sum_at(i, u, lanes); at < n) ++seen[at];
      expect(std::all_of(seen.begin(), seen.end(), [](int k) { return k == 1; }), "every part once", n, lanes);
    }
  for (int rows : {1, 16, 64, 1000})
    for (int L : {1, 77, 5000}) {
      const int first = L / 7;
      for (int group : {0, 1, 300}) {
        const svd::RowChunks ch = svd::row_chunks(L, first, group, rows);
        int most = 0;
        for (int g = 0; g < ch.groups; ++g) most = std::max(most, svd::chunks_of(ch, g).second - svd::chunks_of(ch, g).first);
        expect(svd::join_lanes(ch) == (most > 64 ? 32 : most > 4 ? 8 : 1), "threads a channel", most, svd::join_lanes(ch));
      }
    }
}

}  // namespace

int main(int argc, char** argv) {
  const char* what = argc > 1 ? argv[1] : "";
  if (!std::strcmp(what, "rows")) rows();
  else if (!std::strcmp(what, "rope")) rope();
  else if (!std::strcmp(what, "quantise")) quantise();
  else if (!std::strcmp(what, "joins")) joins();
  else expect(false, "which part?");
  if (!g_failures) std::printf("%s: ok\n", what);
  return g_failures != 0;
}
