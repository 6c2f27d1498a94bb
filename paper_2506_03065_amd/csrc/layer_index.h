// Index arithmetic of the kernels around an attention, apart from them so that it also runs on the host: what a work-group,
// a wave or a lane takes.  (constexpr: usable on both sides.)
#pragma once

#include <cstdint>

namespace svd {

// ---- rows of a batch entry in chunks that lie within one group each ----

struct RowChunks {
  int L, first, group;             // rows; of the first group; of every group behind it, > 0
  int rows;                        // per chunk
  int first_chunks, group_chunks;  // of the first rows; of a whole group
  int per_entry, groups;           // chunks and groups of a batch entry
};

constexpr int rows_of_group(int L, int first_rows, int group_rows) {
  return group_rows > 0 && group_rows < L - first_rows ? group_rows : L - first_rows;
}
constexpr RowChunks row_chunks(int L, int first_rows, int group_rows, int rows) {
  RowChunks c{};
  const int rest = L - first_rows;
  c.L = L;
  c.first = first_rows;
  c.group = rows_of_group(L, first_rows, group_rows);
  c.rows = rows;
  c.first_chunks = c.first / rows + (c.first % rows > 0);
  c.group_chunks = c.group / rows + (c.group % rows > 0);
  const int whole = (rest - 1) / c.group, last = rest - whole * c.group;   // groups ahead of the last, and its rows
  c.per_entry = c.first_chunks + whole * c.group_chunks + last / rows + (last % rows > 0);
  c.groups = (c.first > 0 ? 1 : 0) + whole + 1;
  return c;
}

struct ChunkAt {
  int b, g, row0, row1;
};
constexpr ChunkAt chunk_at(const RowChunks& c, const int id) {
  const int b = id / c.per_entry, i = id % c.per_entry;
  if (i < c.first_chunks) return {b, 0, i * c.rows, c.first - i * c.rows < c.rows ? c.first : (i + 1) * c.rows};
  const int k = i - c.first_chunks, g = k / c.group_chunks, start = c.first + g * c.group, in = (k % c.group_chunks) * c.rows;
  const int end = c.L - start < c.group ? c.L - start : c.group;   // of the group, from its start
  return {b, g + (c.first > 0 ? 1 : 0), start + in, start + (end - in < c.rows ? end : in + c.rows)};
}

// The chunks of group g of an entry: [first, second).
struct ChunkRange {
  int first, second;
};
constexpr ChunkRange chunks_of(const RowChunks& c, const int g) {
  const int behind = g - (c.first > 0 ? 1 : 0);   // -1: the first rows
  if (behind < 0) return {0, c.first_chunks};
  const int c0 = c.first_chunks + behind * c.group_chunks;
  return {c0, behind + 1 + (c.first > 0 ? 1 : 0) < c.groups ? c0 + c.group_chunks : c.per_entry};
}

// The row `step` behind `row` in a chunk that ends at `end`, or `end` if there is none (row + step may itself be past 2^31).
constexpr int row_behind(int row, int step, int end) { return end - row > step ? row + step : end; }

// Lanes of a row: up to 1,024 channels a work-group of 256 takes several rows at once, a row to 16, 32 or 64 lanes, so that its sums
// need no barrier; above (0) it takes one row.  Pieces of 8 channels that a thread holds.  (A work-group a row at any width, 8
// channels a thread: 123,375 x 96 fp32: forward 66 us against 33, backward 356 against 63; 75,600 x 512 bf16: 63 against 61, and 200
// against 107; 75,600 x 768 bf16 with a norm of y: backward 230 against 159; without one, forward 91 against 93.)
constexpr int kLeastGroup = 3;   // rows; of smaller groups a work-group could hardly take several (30,000 x 768 of one row: 119 us for 87)
struct NormShape {
  int lanes, pieces, threads;
  int rows;   // at once
};
constexpr NormShape norm_shape(int C, int group) {
  if (C <= 1024 && group >= kLeastGroup) {
    const int lanes = C <= 128 ? 16 : C <= 256 ? 32 : 64;
    return {lanes, C <= 512 ? 1 : 2, 256, 256 / lanes};
  }
  const int pieces = C <= 2048 ? 1 : C <= 8192 ? 2 : 4;
  return {0, pieces, (C / 8 + 64 * pieces - 1) / (64 * pieces) * 64, 1};
}

// ---- sums of the groups ----

// Group of a work-group of the joining kernel: `y` is at most 32,768 of a launch, `z` the rest.
constexpr int kJoinRow = 32768;
constexpr int join_at(int y, int z) { return y + z * kJoinRow; }
// Threads a channel of it: as many as a group has chunks for (30,000 x 512 in groups of one row: 470 us of four threads a channel, 201 of one).
constexpr int join_lanes(const RowChunks& c) {
  const int chunks = c.group_chunks > c.first_chunks ? c.group_chunks : c.first_chunks;
  return chunks > 64 ? 32 : chunks > 4 ? 8 : 1;
}
// Number u of the eight that a thread of a column takes in a step from `i` on (n or more: none).
constexpr int kSumAhead = 8;
constexpr int sum_at(int i, int u, int lanes) { return i + u * lanes; }

// ---- rotary positions ----

constexpr int kRopeThreads = 256;
constexpr int rope_tokens(int D) { return kRopeThreads / (D / 8); }   // of a work-group: 8 channels of one to a thread
constexpr int rope_blocks(int L, int D) { return (L + rope_tokens(D) - 1) / rope_tokens(D); }

struct HeadRange {
  int first, last;   // [first, last)
};
constexpr HeadRange heads_of_part(int H, int splits, int part) {
  const int per = (H + splits - 1) / splits, first = part * per;
  return {first, first + per < H ? first + per : H};
}

// Parts of the heads, forward: few tokens share the heads out, until the chip has 2,048 work-groups or a thread one head.
constexpr int rope_forward_splits(int L, int B, int D, int n, int heads) {
  const int64_t splits = 2048 / ((int64_t)rope_blocks(L, D) * B * n);
  return (int)(splits < 1 ? 1 : splits > heads ? heads : splits);
}

// Backward: a unit is a block of tokens and a part of the heads; a work-group walks units in steps of the launch, so that the partial sums
// stay few.  Parts so that every work-group has 4 units or more: the last, partly filled round is then little of the whole.
// (48 heads of 64 x 21,825, q and k: 170 us for 4, 173 for 8, 177 for 16, 204 for a unit of all heads.)
constexpr int kRopePartials = 512;   // work-groups of a tensor, at most, that leave a partial sum
struct RopeWalk {
  int splits, groups;
};
constexpr RopeWalk rope_walk(int L, int B, int D, int heads) {
  const int64_t blocks = (int64_t)B * rope_blocks(L, D), want = (4 * kRopePartials + blocks - 1) / blocks;
  const int splits = (int)(want > heads ? heads : want);
  return {splits, (int)(blocks * splits < kRopePartials ? blocks * splits : kRopePartials)};
}
struct RopeUnit {
  int b, block, part;
};
constexpr RopeUnit rope_unit(int64_t i, int blocks, int splits) {
  const int at = (int)(i / splits);
  return {at / blocks, at % blocks, (int)(i % splits)};
}

struct Place {
  bool video;
  int frame, y, x;
};
// Of the token in row l: first other tokens, then frames x height x width.
constexpr Place place_of(int token, int frames, int height, int width, bool position_major) {
  const int N = height * width;
  if (token < 0 || token >= N * frames) return {false, 0, 0, 0};
  const int pos = position_major ? token / frames : token % N;
  return {true, position_major ? token % frames : token / N, pos / width, pos % width};
}

// ---- blocks of 128 ----

// By rows: a work-group takes 32 rows of `blocks` blocks, a wave 8 rows, 16 lanes a block, four or two rows at once where the rows are of
// one or two blocks (300,000 x 128 bf16: 17.5 us against 43; 75,600 x 256: 10.7 against 16.5).
constexpr int kQuantRows = 32;
constexpr int quant_blocks(int C) { return C <= 128 ? 1 : C <= 256 ? 2 : 4; }
constexpr int quant_rows_at_once(int blocks) { return 4 / blocks; }   // of a wave
struct QuantAt {
  int block, row, column;   // of the work-group; first row of the thread, its further ones quant_rows_at_once apart; of the block
};
constexpr QuantAt quant_at(int thread, int blocks) {
  const int quarter = (thread & 63) >> 4;
  return {quarter % blocks, (thread >> 6) * 8 + quarter / blocks, (thread & 15) * 8};
}
// By columns: 128 rows of 64 columns, read in four steps of 32 rows, 8 columns a thread; then a thread has 32 rows of a column.
struct QuantPlace {
  int row, column;
};
constexpr QuantPlace quant_read_at(int thread, int step) { return {step * 32 + thread / 8, (thread & 7) * 8}; }
constexpr QuantPlace quant_write_at(int thread) { return {(thread & 3) * 32, thread >> 2}; }

// ---- block-scaled products ----

// Work-group -> tile.  Work-groups go to the 8 XCDs in turn; each XCD takes a run of the tiles in an order that walks groups of
// kGroupTiles rows of tiles column by column, so that what its compute units work on at a time shares rows and columns in its L2.
// (75,600 x 5,120 x 5,120: groups of 4 1,630 us, 8 1,635, 16 1,765; 11,881 x 1,920 x 7,680: 181, 171, 168; column by column over the
// whole matrix, without regard to the XCDs, 2,480 against 1,930 of the kernel of that time.)
constexpr int kGroupTiles = 8;
struct TileAt {
  int m, n;
};
constexpr TileAt tile_at(const int at, const int m_tiles, const int n_tiles) {
  const int total = m_tiles * n_tiles, xcd = at & 7, each = total >> 3, more = total & 7;
  const int o = xcd * each + (xcd < more ? xcd : more) + (at >> 3);
  const int first = o / (kGroupTiles * n_tiles) * kGroupTiles, in = o % (kGroupTiles * n_tiles);
  const int rows = m_tiles - first < kGroupTiles ? m_tiles - first : kGroupTiles;
  return {first + in % rows, in / rows};
}

// Position of a row's 16-byte chunk in an LDS tile of 128-byte rows, in chunks.  A fragment read takes rows j * TILES + t,
// j = 0 .. 15, at the same chunk: inside the 256 bytes of a pair of rows the 16 positions are permuted with j, so that
// the 16 lanes spread over all banks.
constexpr int swizzle(int row, int tiles) { return (row / tiles) & 15; }

// Three forms of the product: 256 x 256 tiles, 128 x 128 with two work-groups to a compute unit, and 64 x 64 in four parts of K.
// The last for up to 64 rows, or where the chip's 256 units take the product in one round that way (two rounds, if K is long).
// Otherwise the rounds decide: one of large tiles counts 100, one of 512 small tiles 69, the rest of at most 256 small tiles 45.
// The large tiles behind the last full round go in quarters, as small tiles in a launch of its own (counted 12), if K is not
// short and that is to save a thirtieth part: over many rounds the units part anyway. us whole / cut, in turn on one card:
// 11,881 x 1,920 x 7,680: 167 / 156; 24,000 x 1,000 x 4,096: 93 / 88; 9,107 x 6,144 x 2,048: 111 / 108; 20,000 x 2,048 x 2,048: 85 / 82;
// not so 11,881 x 1,920 x 1,024: 33.1 / 33.7; 75,600 x 5,120 x 5,120: 1,556 / 1,578.
// us for 256 / 128 / 64, on the same card (another takes up to 6 % more or less):
// 75,600 x 5,120 x 5,120: 1,556 / 1,886 / 3,958;  9,107 x 6,144 x 2,048: 111 / 119 / 307;  11,881 x 1,920 x 7,680: 167 / 163 / 327;
// 7,680 x 1,920 x 11,881: 146 / 162 / 298;  6,000 x 3,300 x 4,096: 120 / 107 / 197;  1,920 x 1,920 x 30,000: 254 / 148 / 178;
// 800 x 1,536 x 8,192: 71 / 39.7 / 29.7;  800 x 1,536 x 2,048: 23.5 / 13.7 / 13.8;  1,000 x 1,920 x 1,920: 22.7 / 13.9 / 13.8;
// 300 x 1,920 x 1,920: 20.8 / 10.8 / 7.4;  128 x 5,120 x 5,120: 46.7 / 29.9 / 13.3;  17 x 4,096 x 4,096: 36.4 / 20.8 / 9.8;
// 2 x 30,720 x 5,120: 63 / 42.7 / 32.6.
enum { FORM_64 = 0, FORM_128 = 1, FORM_256 = 2 };
struct MatmulPlan {
  int form;
  int whole;   // FORM_256: tiles that run whole; the others in quarters
};
constexpr int64_t tiles_of(int M, int N, int size) { return (int64_t)((M + size - 1) / size) * ((N + size - 1) / size); }
constexpr int64_t small_cost(int64_t n) { return n / 512 * 69 + (n % 512 > 256 ? 69 : n % 512 > 0 ? 45 : 0); }
constexpr MatmulPlan matmul_plan(int M, int N, int K) {
  if (M <= 64 || tiles_of(M, N, 64) <= (K >= 4096 ? 512 : 256)) return {FORM_64, 0};
  const int64_t large = tiles_of(M, N, 256), full = large / 256 * 256, rest = large - full;
  const int64_t whole_cost = (large + 255) / 256 * 100, cut_cost = full / 256 * 100 + small_cost(4 * rest) + 12;
  const bool cut = full > 0 && rest > 0 && K >= 2048 && cut_cost * 30 < whole_cost * 29;
  if ((cut ? cut_cost : whole_cost) > small_cost(tiles_of(M, N, 128))) return {FORM_128, 0};
  return {FORM_256, (int)(cut ? full : large)};
}
// Work-group -> (large tile, quarter) behind the first `whole` tiles (a multiple of 8: a quarter runs on its tile's XCD).
struct QuarterAt {
  int tile, quarter;
};
constexpr QuarterAt quarter_at(int block, int whole) { return {whole + (block >> 5) * 8 + (block & 7), (block >> 3) & 3}; }
constexpr int64_t quarter_blocks(int64_t rest) { return (rest + 7) / 8 * 32; }

// Byte of a tile in memory that lane `lane` of slab `slab` (1 KB, 8 rows) brings to the slab's byte 16 * lane; past every range for
// bytes at or behind `left` of a row.
constexpr uint32_t slab_place(int slab, int lane, int tiles, uint32_t stride, int left) {
  const int at = slab * 64 + lane, pair = at >> 4, x = (at & 15) ^ swizzle(pair * 2, tiles);
  return (x & 7) * 16 < left ? (uint32_t)(pair * 2 + (x >> 3)) * stride + (x & 7) * 16 : 0x80000000u;
}
// Byte of the LDS tile that holds chunk `chunk` of row `row`.
constexpr int tile_byte(int row, int chunk, int tiles) { return (row >> 1) * 256 + ((((row & 1) * 8 + chunk) ^ swizzle(row, tiles)) << 4); }

}  // namespace svd
