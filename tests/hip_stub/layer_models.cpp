// Host models of the kernel launches behind layer_ops.h.  No arithmetic on values: the models touch, on the host, every row, vector,
// table entry, partial sum, tile and scale byte that a launch would address, the norms' and the product's through the kernels' own index
// arithmetic (layer_index.h), work-group by work-group.  (That of the rotary kernels, of the quantisation and of the joins of sums is
// walked in layer_indices.cpp.)  All of that memory is exact-size heap memory of the test, so an index that leaves its buffer is an
// AddressSanitizer report and a violation.
#include <algorithm>
#include <cstdint>
#include <cstring>
#include <vector>

#include "hip_stub.h"
#include "layer_ops.h"

namespace svd {

namespace {

volatile uint64_t g_sink;

void rd(const void* p, size_t bytes, const char* what) {
  if (!stub::in_device(p, bytes)) {
    stub::violation("%s: read of %zu bytes outside every device allocation", what, bytes);
    return;
  }
  const unsigned char* c = static_cast<const unsigned char*>(p);
  g_sink = g_sink + c[0] + c[bytes - 1];
}
void wr(void* p, size_t bytes, const char* what) {
  if (!stub::in_device(p, bytes)) {
    stub::violation("%s: write of %zu bytes outside every device allocation", what, bytes);
    return;
  }
  std::memset(p, 0x11, bytes);
}
void check(bool ok, const char* what, long a = 0, long b = 0) {
  if (!ok) stub::violation("%s (%ld, %ld)", what, a, b);
}
char* row(const RowsView& r, int b, int l, size_t size) { return static_cast<char*>(r.data) + ((int64_t)b * r.stride_b + (int64_t)l * r.stride_l) * size; }

void norm_vectors(const NormLaunch& p, int b, int g) {
  const int64_t mod = b * p.mod_stride_b + g * p.mod_stride_g;
  for (const float* v : {p.vec.weight, p.vec.bias, p.vec.post_weight})
    if (v) rd(v, p.C * 4, "vector");
  for (const float* v : {p.vec.gate, p.vec.scale, p.vec.shift})
    if (v) rd(v + mod, p.C * 4, "modulation");
}

// every row of every entry in one chunk, of its own group
template <class F>
void walk_chunks(const NormLaunch& p, F f) {
  const NormShape s = norm_shape(p.C, p.ch.group);
  check((s.lanes ? s.lanes : s.threads) * s.pieces * 8 >= p.C && s.threads <= (s.lanes || s.pieces == 1 ? 256 : 512) && s.threads % 64 == 0 &&
            (s.lanes == 0 || s.lanes * s.rows == s.threads), "threads of a row", s.threads, p.C);
  std::vector<int> seen((size_t)p.B * p.ch.L);
  for (int id = 0; id < p.B * p.ch.per_entry; ++id) {
    const ChunkAt c = chunk_at(p.ch, id);
    check(c.b >= 0 && c.b < p.B && c.g >= 0 && c.g < p.ch.groups && c.row0 < c.row1 && c.row1 <= p.ch.L, "chunk", id, c.row0);
    const ChunkRange range = chunks_of(p.ch, c.g);
    check(id % p.ch.per_entry >= range.first && id % p.ch.per_entry < range.second, "chunk of a group", id, c.g);
    norm_vectors(p, c.b, c.g);
    for (int l = c.row0; l < c.row1; ++l) {
      const int want = l < p.ch.first ? 0 : (p.ch.first > 0 ? 1 : 0) + (l - p.ch.first) / p.ch.group;
      check(want == c.g, "group of a row", l, c.g);
      ++seen[(size_t)c.b * p.ch.L + l];
      f(id, c.b, l);
    }
  }
  check(std::all_of(seen.begin(), seen.end(), [](int n) { return n == 1; }), "every row once", p.B, p.ch.L);
  int at = 0;
  for (int g = 0; g < p.ch.groups; ++g) {   // the groups' chunks follow one another
    const ChunkRange range = chunks_of(p.ch, g);
    check(range.first == at && range.second > range.first, "chunks of the groups", g, range.first);
    at = range.second;
  }
  check(at == p.ch.per_entry, "chunks of an entry", at, p.ch.per_entry);
}

void rope_rows(const RopeLaunch& p, bool backward) {
  for (int i = 0; i < p.n; ++i) {
    const RopeTensor& t = p.t[i];
    for (const float* v : {t.weight, t.bias})
      if (v) rd(v, p.D * 4, "vector");
    for (int b = 0; b < p.B; ++b)
      for (int l = 0; l < p.L; ++l) {
        const Place q = place_of(p.r.row_offset + l - p.r.first, p.r.frames, p.r.height, p.r.width, p.r.position_major != 0);
        if (q.video) {
          check(q.frame < p.r.frames && q.y < p.r.height && q.x < p.r.width, "place", q.frame, q.x);
          const int len[3] = {p.r.frames * p.r.pairs_t, p.r.height * p.r.pairs_h, p.r.width * p.r.pairs_w};
          const int at[3] = {q.frame * p.r.pairs_t, len[0] + q.y * p.r.pairs_h, len[0] + len[1] + q.x * p.r.pairs_w};
          const int n[3] = {p.r.pairs_t, p.r.pairs_h, p.r.pairs_w};
          for (int a = 0; a < 3; ++a)
            if (n[a]) rd(p.table + 2 * (int64_t)at[a], n[a] * 8, "table");
        }
        for (int h = 0; h < t.H; ++h) {
          if (t.x) rd(t.x + b * t.x_b + h * t.x_h + l * t.x_l, p.D * 2, "x row");
          if (backward) rd(t.dout + b * t.d_b + h * t.d_h + l * t.d_l, p.D * 2, "dout row");
          wr(t.out + b * t.o_b + h * t.o_h + l * t.o_l, p.D * 2, "out row");
        }
      }
  }
}

}  // namespace

hipError_t launch_norm_forward(const NormLaunch& p, hipStream_t stream) {
  stub::note_launch(stream, "norm forward");
  const size_t x = p.stream_type == SVD_F32 ? 4 : 2;
  walk_chunks(p, [&](int, int b, int l) {
    rd(row(p.x, b, l, x), p.C * x, "x");
    if (p.y.data) {
      rd(row(p.y, b, l, 2), p.C * 2, "y");
      wr(row(p.x_out, b, l, x), p.C * x, "x_out");
    }
    if (!p.h.data) return;
    wr(row(p.h, b, l, p.h_scales ? 1 : 2), p.C * (p.h_scales ? 1 : 2), "h");
    if (p.h_scales)
      for (int c = 0; c < p.C; c += 128) wr(p.h_scales + (int64_t)(c >> 7) * p.h_scale_stride + (int64_t)b * p.ch.L + l, 1, "h_scales");
  });
  return hipSuccess;
}

hipError_t launch_norm_backward(const NormLaunch& p, hipStream_t stream) {
  stub::note_launch(stream, "norm backward");
  const size_t x = p.stream_type == SVD_F32 ? 4 : 2;
  walk_chunks(p, [&](int id, int b, int l) {
    rd(row(p.x_out, b, l, x), p.C * x, "x_out");
    if (p.dx_out.data) rd(row(p.dx_out, b, l, x), p.C * x, "dx_out");
    if (p.dh.data) rd(row(p.dh, b, l, 2), p.C * 2, "dh");
    wr(row(p.dx, b, l, x), p.C * x, "dx");
    if (p.y.data) {
      rd(row(p.y, b, l, 2), p.C * 2, "y");
      wr(row(p.dy, b, l, 2), p.C * 2, "dy");
    }
    if (p.partial) wr(p.partial + (int64_t)id * 3 * p.C, 3 * p.C * 4, "partial sums");
  });
  if (!p.partial) return hipSuccess;
  const int n = p.B * p.ch.groups;
  for (int bg = 0; bg < n; ++bg) {
    for (float* v : {p.grads.gate, p.grads.scale, p.grads.shift})
      if (v) wr(v + (int64_t)bg * p.C, p.C * 4, "gradient of a modulation");
    if (n > 1 && (p.grads.weight || p.grads.bias || p.grads.post_weight)) wr(p.sums + (int64_t)bg * 3 * p.C, 3 * p.C * 4, "sums of a group");
  }
  for (float* v : {p.grads.weight, p.grads.bias, p.grads.post_weight})
    if (v) wr(v, p.C * 4, "gradient of a weight");
  return hipSuccess;
}

hipError_t launch_rope_table(const svd_rope_desc& r, double, const double*, const double*, float* table, hipStream_t stream) {
  stub::note_launch(stream, "rope table");
  wr(table, (size_t)(r.frames * r.pairs_t + r.height * r.pairs_h + r.width * r.pairs_w) * 8, "table");
  return hipSuccess;
}
hipError_t launch_rope_forward(const RopeLaunch& p, hipStream_t stream) {
  stub::note_launch(stream, "rope forward");
  rope_rows(p, false);
  return hipSuccess;
}
hipError_t launch_rope_backward(const RopeLaunch& p, hipStream_t stream) {
  stub::note_launch(stream, "rope backward");
  rope_rows(p, true);
  for (int i = 0; i < p.n; ++i) {
    if (p.partial) wr(p.partial + (int64_t)i * kRopePartials * 2 * p.D, (size_t)kRopePartials * 2 * p.D * 4, "partial sums");
    for (float* v : {p.t[i].dweight, p.t[i].dbias})
      if (v) wr(v, p.D * 4, "gradient of a weight");
  }
  return hipSuccess;
}

hipError_t launch_quantise_rows(const QuantLaunch& p, hipStream_t stream) {
  stub::note_launch(stream, "quantise rows");
  const size_t x = p.src_type == SVD_F32 ? 4 : 2;
  for (int r = 0; r < p.R; ++r) {
    rd(static_cast<const char*>(p.src) + (int64_t)r * p.src_stride * x, p.C * x, "src row");
    wr(p.dst + (int64_t)r * p.dst_stride, (p.C + 15) / 16 * 16, "row of values");
    for (int b = 0; b < (p.C + 127) / 128; ++b) wr(p.scales + (int64_t)b * p.scale_stride + r, 1, "scale");
  }
  return hipSuccess;
}
hipError_t launch_quantise_columns(const QuantLaunch& p, hipStream_t stream) {
  stub::note_launch(stream, "quantise columns");
  check((p.C + 63) / 64 <= 65535 && (p.R + 127) / 128 <= 65535, "grid", p.R, p.C);
  const size_t x = p.src_type == SVD_F32 ? 4 : 2;
  for (int r = 0; r < p.R; ++r) rd(static_cast<const char*>(p.src) + (int64_t)r * p.src_stride * x, p.C * x, "src row");
  for (int c = 0; c < p.C; ++c) {
    wr(p.dst + (int64_t)c * p.dst_stride, (p.R + 15) / 16 * 16, "row of values");
    for (int b = 0; b < (p.R + 127) / 128; ++b) wr(p.scales + (int64_t)b * p.scale_stride + c, 1, "scale");
  }
  return hipSuccess;
}

namespace {

// A tile's requests: every lane of every slab and step.  What starts inside the range of the rows is read; a row's own chunks
// have to be among it, each at the byte of LDS where the fragment reads look for it, and no byte of another row.
void model_operand(const uint8_t* base, int row0, int rows, int64_t stride, int size, int tiles, int K) {
  const int k16 = (K + 15) / 16 * 16, n = std::min(rows - row0, size);
  const uint8_t* const at = base + (int64_t)row0 * stride;
  const uint64_t range = (uint64_t)(n - 1) * stride + k16;
  check(range < (uint64_t{1} << 31), "range of a tile", (long)range, size);
  for (int step = 0; step * 128 < k16; ++step) {
    const bool tail = step * 128 + 128 > k16;
    std::vector<int> filled(size * 8);
    for (int slab = 0; slab < size / 8; ++slab)
      for (int lane = 0; lane < 64; ++lane) {
        const uint32_t place = slab_place(slab, lane, tiles, (uint32_t)stride, tail ? k16 % 128 : 128);
        const uint64_t off = (uint64_t)place + (uint64_t)step * 128;
        if (place >= range) continue;   // the lane's own offset alone decides
        check(off + 16 <= range, "inside the range", (long)off, (long)range);
        rd(at + off, 16, "operand");
        const int r = (int)(place / stride), chunk = (int)(place % stride) / 16;
        check(r < n && step * 128 + chunk * 16 < k16, "a chunk of the row itself", r, chunk);
        check(slab * 1024 + lane * 16 == tile_byte(r, chunk, tiles), "where a fragment looks for it", r, chunk);
        ++filled[r * 8 + chunk];
      }
    for (int r = 0; r < n; ++r)
      for (int c = 0; c < 8; ++c) check(filled[r * 8 + c] == (step * 128 + c * 16 < k16 ? 1 : 0), "every chunk once", r, c);
  }
}

}  // namespace

hipError_t launch_blockscale_matmul(const MatmulLaunch& p, hipStream_t stream) {
  stub::note_launch(stream, "product");
  const svd_blockscale_desc& d = p.d;
  const MatmulPlan plan = matmul_plan(d.M, d.N, d.K);
  const int form = plan.form, size = form == FORM_64 ? 64 : form == FORM_128 ? 128 : 256, mt = form == FORM_256 ? 4 : 2, nt = 2;
  const int m_tiles = (d.M + size - 1) / size, n_tiles = (d.N + size - 1) / size, blocks = (d.K + 127) / 128;
  std::vector<int> seen((size_t)m_tiles * n_tiles);
  const int total = m_tiles * n_tiles, whole = form == FORM_256 ? plan.whole : total;
  check(whole <= total && (whole == total || whole % 8 == 0), "whole tiles", whole, total);
  std::vector<int> quarters((size_t)total * 4);
  for (int block = 0; block < quarter_blocks(total - whole); ++block) {
    const QuarterAt q = quarter_at(block, whole);
    if (q.tile < total) ++quarters[(size_t)q.tile * 4 + q.quarter];
  }
  for (int i = 0; i < total * 4; ++i) check(quarters[i] == (i / 4 >= whole ? 1 : 0), "every quarter once", i, whole);
  for (int i = 0; i < total; ++i) {
    const TileAt t = tile_at(i, m_tiles, n_tiles);
    check(t.m >= 0 && t.m < m_tiles && t.n >= 0 && t.n < n_tiles, "tile", t.m, t.n);
    ++seen[(size_t)t.m * n_tiles + t.n];
  }
  check(std::all_of(seen.begin(), seen.end(), [](int n) { return n == 1; }), "every tile once", m_tiles, n_tiles);
  for (int m = 0; m < m_tiles; ++m) model_operand(p.a, m * size, d.M, d.a_stride, size, mt, d.K);
  for (int n = 0; n < n_tiles; ++n) model_operand(p.b, n * size, d.N, d.b_stride, size, nt, d.K);
  for (int i = whole; i < total; ++i)
    for (int q = 0; q < 4; ++q) {
      const TileAt t = tile_at(i, m_tiles, n_tiles);
      const int m0 = t.m * 256 + (q & 1) * 128, n0 = t.n * 256 + (q >> 1) * 128;
      if (m0 >= d.M || n0 >= d.N) continue;
      model_operand(p.a, m0, d.M, d.a_stride, 128, 2, d.K);
      model_operand(p.b, n0, d.N, d.b_stride, 128, 2, d.K);
    }
  rd(p.a_scales, (size_t)(blocks - 1) * d.a_scale_stride + (d.M + 15) / 16 * 16, "scales");   // the range of their buffers
  rd(p.b_scales, (size_t)(blocks - 1) * d.b_scale_stride + (d.N + 15) / 16 * 16, "scales");
  if (p.bias) rd(p.bias, d.N * 4, "bias");
  for (int m = 0; m < d.M; ++m) wr(p.out + (int64_t)m * d.out_stride, d.N * 2, "out row");
  return hipSuccess;
}

}  // namespace svd
