// Entry points of the operators around the attention of a layer: every argument is checked here, ahead of the first
// launch.  Index arithmetic that the kernels do in 32 bits is bounded here.
#include <cmath>
#include <cstddef>
#include <cstdint>
#include <initializer_list>

#include "layer_index.h"
#include "layer_ops.h"
#include "sparse_vdit.h"

namespace {

bool aligned16(const void* ptr) { return (reinterpret_cast<uintptr_t>(ptr) & 15u) == 0; }

svd_status status_of(hipError_t e) { return e == hipSuccess ? SVD_OK : SVD_ERR_HIP; }

constexpr int kMaxChannels = 16384;
constexpr int64_t kMaxStride = int64_t{1} << 40;   // of rows and entries: byte offsets stay inside 63 bits

// A tensor of rows; `unit`: elements in 16 bytes.  An axis of length 1 needs no stride.
svd_status check_rows(const svd_rows* r, int32_t B, int32_t L, int32_t C, int unit) {
  if (!aligned16(r->data)) return SVD_ERR_ALIGN;
  if ((L > 1 && (r->stride_l < C || r->stride_l > kMaxStride)) || (B > 1 && (r->stride_b < 1 || r->stride_b > kMaxStride)))
    return SVD_ERR_SHAPE;
  if ((L > 1 && r->stride_l % unit) || (B > 1 && r->stride_b % unit)) return SVD_ERR_ALIGN;
  return SVD_OK;
}

bool present(const svd_rows* r) { return r && r->data; }

svd::RowsView rows_view(const svd_rows* r) {
  return present(r) ? svd::RowsView{r->data, r->stride_b, r->stride_l} : svd::RowsView{nullptr, 0, 0};
}

svd_status check_norm_desc(const svd_norm_desc& d) {
  if (d.B < 1 || d.L < 1 || d.C < 8 || d.C > kMaxChannels) return SVD_ERR_SHAPE;
  if (d.C % 8) return SVD_ERR_ALIGN;
  if (static_cast<int64_t>(d.B) * d.L > INT32_MAX) return SVD_ERR_UNSUPPORTED;
  if (d.stream_type != SVD_BF16 && d.stream_type != SVD_F32) return SVD_ERR_DTYPE;
  if (d.norm != SVD_NORM_LAYER && d.norm != SVD_NORM_RMS) return SVD_ERR_PARAMS;
  if (d.post_norm < SVD_NORM_NONE || d.post_norm > SVD_NORM_RMS) return SVD_ERR_PARAMS;
  if (!(d.eps > 0.f) || !std::isfinite(d.eps)) return SVD_ERR_PARAMS;
  if (d.first_rows < 0 || d.first_rows >= d.L || d.group_rows < 0) return SVD_ERR_PARAMS;
  if (d.mod_stride_b < 0 || d.mod_stride_g < 0 || d.mod_stride_b > kMaxStride || d.mod_stride_g > kMaxStride) return SVD_ERR_SHAPE;
  if (d.mod_stride_b % 4 || d.mod_stride_g % 4) return SVD_ERR_ALIGN;
  return SVD_OK;
}

svd_status check_vectors(const svd_norm_desc& d, const svd_norm_vectors& v, bool y) {
  for (const float* p : {v.weight, v.bias, v.post_weight, v.gate, v.scale, v.shift})
    if (!aligned16(p)) return SVD_ERR_ALIGN;
  if (v.post_weight && (d.post_norm == SVD_NORM_NONE || !y)) return SVD_ERR_PARAMS;
  if (v.gate && !y) return SVD_ERR_PARAMS;
  return SVD_OK;
}

svd::NormShape norm_shape(const svd_norm_desc& d) {
  return svd::norm_shape(d.C, svd::rows_of_group(d.L, d.first_rows, d.group_rows));
}

int clamp_rows(int64_t rows, int most) { return static_cast<int>(rows < 1 ? 1 : rows > most ? most : rows); }

// Rows of a chunk.  Forward: eight rounds of the work-groups that a compute unit holds (20 waves of one piece a thread, 10 to 12 of
// more), 16 rows at most: a chunk's vectors and first loads are paid once, the last round is little of the whole.  us for 4, 8 and 32
// rows and for what this gives: 75,600 x 5,120 bf16: 679 / 603 / 631, 16: 597;  35,552 x 1,920 fp32: 158 / 167 / 183, 3: 156.  No fewer
// than 3 rows (4 of several pieces) where that leaves two work-groups to a unit (one and three rows: 9,107 x 2,048 bf16: 40 / 31;
// one and four: 5,000 x 5,120: 90 / 54).  Where a work-group takes several rows at once, rounds of five work-groups: four of them for a
// wave a row, two for less (75,600 x 512 bf16, one, two and four rounds: 70 / 66 / 61 us; 75,600 x 256: 33 / 30 / 34).
int norm_forward_rows(const svd_norm_desc& d) {
  const svd::NormShape s = norm_shape(d);
  const int64_t n = static_cast<int64_t>(d.B) * d.L;
  if (s.rows > 1) return s.rows * clamp_rows(n / s.rows / ((s.rows == 4 ? 4 : 2) * 256 * 5), 16);
  const int held = (s.pieces == 1 ? 20 : 10) / (s.threads / 64), least = s.pieces == 1 ? 3 : 4;
  const int many = clamp_rows(n / (8 * 256 * (held < 1 ? 1 : held)), 16), few = clamp_rows(n / (2 * 256), least);
  return many > few ? many : few;
}
// Backward: about 512 chunks, whose partial sums are few (75,600 x 5,120: 31 MB beside 2 GB), but no fewer than 256 for less
// than 4 rows each (or 4 times as many as a work-group takes at once).  1,024 where a work-group has three waves (75,600 x 1,152 bf16:
// 234 us against 293; 23,762 x 1,920, four waves: 203 against 182; 40,000 x 2,560, two pieces a thread: 275 against 263); 256 where one
// fills a compute unit (8,000 x 16,384: 456 us against 490).
int norm_backward_rows(const svd_norm_desc& d) {
  const svd::NormShape s = norm_shape(d);
  const int64_t chunks = s.pieces == 4 ? 256 : s.pieces == 1 && s.threads < 256 ? 1024 : 512;
  const int64_t n = (static_cast<int64_t>(d.B) * d.L + s.rows - 1) / s.rows;
  const int64_t most = (n + chunks - 1) / chunks, few = (n + 255) / 256;
  return s.rows * clamp_rows(most > (few < 4 ? few : 4) ? most : (few < 4 ? few : 4), 1 << 20);
}

svd::NormLaunch norm_launch(const svd_norm_desc& d, const svd_norm_vectors& v, int rows) {
  svd::NormLaunch p{};
  p.ch = svd::row_chunks(d.L, d.first_rows, d.group_rows, rows);
  p.B = d.B;
  p.C = d.C;
  p.stream_type = d.stream_type;
  p.norm = d.norm;
  p.post_norm = d.post_norm;
  p.eps = d.eps;
  p.mod_stride_b = d.mod_stride_b;
  p.mod_stride_g = d.mod_stride_g;
  p.vec = v;
  return p;
}

// A launch has less than 2^32 threads.
svd_status check_grid(const svd::NormLaunch& p) {
  return static_cast<uint64_t>(p.B) * p.ch.per_entry * svd::norm_shape(p.C, p.ch.group).threads < (uint64_t{1} << 32) ? SVD_OK : SVD_ERR_UNSUPPORTED;
}

size_t norm_partial_floats(const svd_norm_desc& d) {
  const svd::RowChunks ch = svd::row_chunks(d.L, d.first_rows, d.group_rows, norm_backward_rows(d));
  return static_cast<size_t>(d.B) * (static_cast<size_t>(ch.per_entry) + ch.groups) * 3 * d.C;
}

// Table entries (pairs of floats).
int64_t rope_entries(const svd_rope_desc& r) {
  return static_cast<int64_t>(r.frames) * r.pairs_t + static_cast<int64_t>(r.height) * r.pairs_h +
         static_cast<int64_t>(r.width) * r.pairs_w;
}

svd_status check_rope(const svd_rope_desc& r) {
  if (r.first < 0 || r.row_offset < 0 || r.frames < 1 || r.height < 1 || r.width < 1) return SVD_ERR_PARAMS;
  if (r.pairs_t < 0 || r.pairs_h < 0 || r.pairs_w < 0) return SVD_ERR_PARAMS;
  if (static_cast<int64_t>(r.pairs_t) + r.pairs_h + r.pairs_w > 64) return SVD_ERR_PARAMS;
  if (r.pairing != SVD_ROPE_ADJACENT && r.pairing != SVD_ROPE_HALVES) return SVD_ERR_PARAMS;
  if (r.position_major != 0 && r.position_major != 1) return SVD_ERR_PARAMS;
  const double tokens = static_cast<double>(r.frames) * r.height * r.width;   // the kernels index tokens and the table in 32 bits
  if (tokens + r.first >= 2147483648.0 || rope_entries(r) > INT32_MAX) return SVD_ERR_UNSUPPORTED;
  return SVD_OK;
}

// Heads of q or k: the rotary kernels form offsets in 64 bits, so the limits of the attention's tensors do not hold here.
constexpr int32_t kMaxRopeRows = 1 << 27;   // a launch has less than 2^32 threads an axis
svd_status check_heads(const svd_tensor_desc* t, int32_t B, int32_t L, int32_t D) {
  if (!t) return SVD_ERR_NULL;
  if (t->B < 1 || t->L < 1 || t->H < 1 || t->H > 65535 || (t->D != 64 && t->D != 128)) return SVD_ERR_SHAPE;
  if (t->B != B || t->L != L || t->D != D) return SVD_ERR_SHAPE;
  if (t->stride_l < t->D || t->stride_b < 1 || t->stride_h < 1) return SVD_ERR_SHAPE;
  if ((t->L > 1 && t->stride_l > kMaxStride) || (t->B > 1 && t->stride_b > kMaxStride) || (t->H > 1 && t->stride_h > kMaxStride)) return SVD_ERR_SHAPE;
  if (t->stride_b % 8 || t->stride_h % 8 || t->stride_l % 8) return SVD_ERR_ALIGN;
  return SVD_OK;
}

svd_status check_rope_call(const svd_rope_desc* rope, const float* table, int32_t norm, float eps, int32_t n,
                           const svd_tensor_desc* d, svd::RopeLaunch* p) {
  if (!d) return SVD_ERR_NULL;
  if (svd_status st = check_rope(*rope)) return st;
  if (svd_status st = check_heads(d, d->B, d->L, d->D)) return st;
  if (2 * (rope->pairs_t + rope->pairs_h + rope->pairs_w) > d->D) return SVD_ERR_PARAMS;
  if (!table && rope_entries(*rope) > 0) return SVD_ERR_NULL;
  if (!aligned16(table)) return SVD_ERR_ALIGN;
  if (norm < SVD_NORM_NONE || norm > SVD_NORM_RMS) return SVD_ERR_PARAMS;
  if (norm != SVD_NORM_NONE && (!(eps > 0.f) || !std::isfinite(eps))) return SVD_ERR_PARAMS;
  if (d->B > 65535 || d->L > kMaxRopeRows || static_cast<int64_t>(d->B) * d->L > INT32_MAX) return SVD_ERR_UNSUPPORTED;
  if (static_cast<int64_t>(rope->row_offset) + d->L > INT32_MAX) return SVD_ERR_UNSUPPORTED;
  p->r = *rope;
  p->table = table;
  p->norm = norm;
  p->eps = eps;
  p->B = d->B;
  p->L = d->L;
  p->D = d->D;
  p->n = n;
  return SVD_OK;
}

bool same_layout(const svd_tensor_desc& a, const svd_tensor_desc& b) {
  return a.stride_b == b.stride_b && a.stride_h == b.stride_h && a.stride_l == b.stride_l;
}

constexpr int32_t kMaxMatrix = 1 << 21;   // and grids of 64 columns within 65,535
constexpr int64_t kMaxMatrixStride = int64_t{1} << 22;   // 256 rows of a tile stay within 32-bit byte offsets

int64_t round16(int64_t n) { return (n + 15) / 16 * 16; }

}  // namespace

extern "C" {

svd_status svd_residual_norm_forward(const svd_norm_desc* desc, const svd_norm_vectors* vec, const svd_rows* x,
                                     const svd_rows* y, const svd_rows* x_out, const svd_rows* h, uint8_t* h_scales,
                                     int64_t h_scale_stride, void* hip_stream) {
  if (!desc || !vec || !present(x)) return SVD_ERR_NULL;
  if (!present(y) && !present(h)) return SVD_ERR_NULL;            // nothing to do
  if (present(y) != present(x_out)) return SVD_ERR_NULL;
  if (h_scales && !present(h)) return SVD_ERR_NULL;
  const svd_norm_desc& d = *desc;
  if (svd_status st = check_norm_desc(d)) return st;
  if (svd_status st = check_vectors(d, *vec, present(y))) return st;
  const int unit = d.stream_type == SVD_F32 ? 4 : 8;
  if (svd_status st = check_rows(x, d.B, d.L, d.C, unit)) return st;
  if (present(y)) {
    if (svd_status st = check_rows(y, d.B, d.L, d.C, 8)) return st;
    if (svd_status st = check_rows(x_out, d.B, d.L, d.C, unit)) return st;
    if (x_out->data == y->data || (x_out->data == x->data && ((d.L > 1 && x_out->stride_l != x->stride_l) ||
                                                               (d.B > 1 && x_out->stride_b != x->stride_b))))
      return SVD_ERR_UNSUPPORTED;
  }
  if (present(h)) {
    if (svd_status st = check_rows(h, d.B, d.L, d.C, h_scales ? 16 : 8)) return st;
    if (h->data == x->data || (present(y) && (h->data == y->data || h->data == x_out->data))) return SVD_ERR_UNSUPPORTED;
  }
  if (h_scales) {
    if (d.C % 16 || !aligned16(h_scales) || h_scale_stride % 16) return SVD_ERR_ALIGN;
    if (h_scale_stride < static_cast<int64_t>(d.B) * d.L || h_scale_stride > kMaxStride) return SVD_ERR_SHAPE;
  }
  svd::NormLaunch p = norm_launch(d, *vec, norm_forward_rows(d));
  if (svd_status st = check_grid(p)) return st;
  p.x = rows_view(x);
  p.y = rows_view(y);
  p.x_out = rows_view(x_out);
  p.h = rows_view(h);
  p.h_scales = h_scales;
  p.h_scale_stride = h_scale_stride;
  return status_of(svd::launch_norm_forward(p, static_cast<hipStream_t>(hip_stream)));
}

svd_status svd_residual_norm_backward_workspace_bytes(const svd_norm_desc* desc, size_t* bytes) {
  if (!desc || !bytes) return SVD_ERR_NULL;
  if (svd_status st = check_norm_desc(*desc)) return st;
  *bytes = norm_partial_floats(*desc) * sizeof(float);
  return SVD_OK;
}

svd_status svd_residual_norm_backward(const svd_norm_desc* desc, const svd_norm_vectors* vec, const svd_rows* x_out,
                                      const svd_rows* y, const svd_rows* dh, const svd_rows* dx_out,
                                      const svd_rows* dx, const svd_rows* dy, const svd_norm_grads* grads,
                                      void* device_workspace, size_t workspace_bytes, void* hip_stream) {
  if (!desc || !vec || !grads || !present(x_out) || !present(dx)) return SVD_ERR_NULL;
  if (!present(dh) && !present(dx_out)) return SVD_ERR_NULL;
  if (present(y) != present(dy)) return SVD_ERR_NULL;
  const svd_norm_desc& d = *desc;
  if (svd_status st = check_norm_desc(d)) return st;
  if (svd_status st = check_vectors(d, *vec, present(y))) return st;
  const int unit = d.stream_type == SVD_F32 ? 4 : 8;
  for (const svd_rows* r : {x_out, dx_out, dx})
    if (present(r))
      if (svd_status st = check_rows(r, d.B, d.L, d.C, unit)) return st;
  for (const svd_rows* r : {y, dh, dy})
    if (present(r))
      if (svd_status st = check_rows(r, d.B, d.L, d.C, 8)) return st;
  if (present(dx_out) && dx->data == dx_out->data &&
      ((d.L > 1 && dx->stride_l != dx_out->stride_l) || (d.B > 1 && dx->stride_b != dx_out->stride_b)))
    return SVD_ERR_UNSUPPORTED;
  for (const svd_rows* r : {x_out, y, dh})
    if (present(r) && (r->data == dx->data || (present(dy) && r->data == dy->data))) return SVD_ERR_UNSUPPORTED;
  if (present(dy) && (dy->data == dx->data || (present(dx_out) && dy->data == dx_out->data))) return SVD_ERR_UNSUPPORTED;
  for (const float* g : {grads->weight, grads->bias, grads->post_weight, grads->gate, grads->scale, grads->shift})
    if (!aligned16(g)) return SVD_ERR_ALIGN;
  // a gradient of what the forward pass did not have
  if ((grads->weight || grads->bias || grads->scale || grads->shift) && !present(dh)) return SVD_ERR_PARAMS;
  if ((grads->gate && !present(y)) || (grads->post_weight && (!present(y) || d.post_norm == SVD_NORM_NONE))) return SVD_ERR_PARAMS;
  const bool any = grads->weight || grads->bias || grads->post_weight || grads->gate || grads->scale || grads->shift;
  if (any && (!device_workspace || !aligned16(device_workspace) || workspace_bytes < norm_partial_floats(d) * sizeof(float)))
    return SVD_ERR_WORKSPACE;
  svd::NormLaunch p = norm_launch(d, *vec, norm_backward_rows(d));
  if (svd_status st = check_grid(p)) return st;
  p.x_out = rows_view(x_out);
  p.y = rows_view(y);
  p.dh = rows_view(dh);
  p.dx_out = rows_view(dx_out);
  p.dx = rows_view(dx);
  p.dy = rows_view(dy);
  p.grads = *grads;
  if (any) {
    p.partial = static_cast<float*>(device_workspace);
    p.sums = p.partial + static_cast<size_t>(d.B) * p.ch.per_entry * 3 * d.C;
  }
  return status_of(svd::launch_norm_backward(p, static_cast<hipStream_t>(hip_stream)));
}

svd_status svd_rope_table_bytes(const svd_rope_desc* rope, size_t* bytes) {
  if (!rope || !bytes) return SVD_ERR_NULL;
  if (svd_status st = check_rope(*rope)) return st;
  *bytes = static_cast<size_t>(rope_entries(*rope)) * 2 * sizeof(float);
  return SVD_OK;
}

svd_status svd_rope_table(const svd_rope_desc* rope, double base, const double* start, const double* step, float* table,
                          size_t table_bytes, void* hip_stream) {
  if (!rope || !start || !step || !table) return SVD_ERR_NULL;
  if (svd_status st = check_rope(*rope)) return st;
  if (!aligned16(table)) return SVD_ERR_ALIGN;
  if (!(base > 0.0) || !std::isfinite(base)) return SVD_ERR_PARAMS;
  for (int i = 0; i < 3; ++i)
    if (!std::isfinite(start[i]) || !std::isfinite(step[i])) return SVD_ERR_PARAMS;
  const int64_t n = rope_entries(*rope);
  if (n < 1) return SVD_ERR_SHAPE;
  if (table_bytes < static_cast<size_t>(n) * 2 * sizeof(float)) return SVD_ERR_WORKSPACE;
  return status_of(svd::launch_rope_table(*rope, base, start, step, table, static_cast<hipStream_t>(hip_stream)));
}

svd_status svd_rope_forward(const svd_rope_desc* rope, const float* table, int32_t norm, float eps,
                            const svd_rope_tensor* tensors, int32_t n_tensors, void* hip_stream) {
  if (!rope || !tensors) return SVD_ERR_NULL;
  if (n_tensors < 1 || n_tensors > 2) return SVD_ERR_SHAPE;
  svd::RopeLaunch p{};
  if (svd_status st = check_rope_call(rope, table, norm, eps, n_tensors, tensors[0].x_desc, &p)) return st;
  for (int i = 0; i < n_tensors; ++i) {
    const svd_rope_tensor& t = tensors[i];
    if (!t.x || !t.out) return SVD_ERR_NULL;
    if (svd_status st = check_heads(t.x_desc, p.B, p.L, p.D)) return st;
    if (svd_status st = check_heads(t.out_desc, p.B, p.L, p.D)) return st;
    if (t.out_desc->H != t.x_desc->H) return SVD_ERR_SHAPE;
    if (!aligned16(t.x) || !aligned16(t.out) || !aligned16(t.weight) || !aligned16(t.bias)) return SVD_ERR_ALIGN;
    if (norm == SVD_NORM_NONE && (t.weight || t.bias)) return SVD_ERR_PARAMS;
    if (t.x == t.out && !same_layout(*t.x_desc, *t.out_desc)) return SVD_ERR_UNSUPPORTED;
    const svd_tensor_desc &x = *t.x_desc, &o = *t.out_desc;
    p.t[i] = {static_cast<const __bf16*>(t.x), nullptr, static_cast<__bf16*>(t.out), x.H, x.stride_b, x.stride_h, x.stride_l,
              0, 0, 0, o.stride_b, o.stride_h, o.stride_l, t.weight, t.bias, nullptr, nullptr};
  }
  if (n_tensors == 2 && (tensors[0].out == tensors[1].out || tensors[0].out == tensors[1].x || tensors[1].out == tensors[0].x))
    return SVD_ERR_UNSUPPORTED;
  return status_of(svd::launch_rope_forward(p, static_cast<hipStream_t>(hip_stream)));
}

svd_status svd_rope_backward_workspace_bytes(int32_t B, int32_t L, int32_t D, size_t* bytes) {
  if (!bytes) return SVD_ERR_NULL;
  if (B < 1 || L < 1 || (D != 64 && D != 128)) return SVD_ERR_SHAPE;
  *bytes = static_cast<size_t>(2) * svd::kRopePartials * 2 * D * sizeof(float);
  return SVD_OK;
}

svd_status svd_rope_backward(const svd_rope_desc* rope, const float* table, int32_t norm, float eps,
                             const svd_rope_grad* tensors, int32_t n_tensors, void* device_workspace, size_t workspace_bytes,
                             void* hip_stream) {
  if (!rope || !tensors) return SVD_ERR_NULL;
  if (n_tensors < 1 || n_tensors > 2) return SVD_ERR_SHAPE;
  svd::RopeLaunch p{};
  if (svd_status st = check_rope_call(rope, table, norm, eps, n_tensors, tensors[0].dout_desc, &p)) return st;
  bool any = false;
  for (int i = 0; i < n_tensors; ++i) {
    const svd_rope_grad& t = tensors[i];
    if (!t.dout || !t.dx) return SVD_ERR_NULL;
    if (svd_status st = check_heads(t.dout_desc, p.B, p.L, p.D)) return st;
    if (svd_status st = check_heads(t.dx_desc, p.B, p.L, p.D)) return st;
    if (t.dx_desc->H != t.dout_desc->H) return SVD_ERR_SHAPE;
    svd_tensor_desc x{};
    if (norm != SVD_NORM_NONE) {
      if (!t.x) return SVD_ERR_NULL;
      if (svd_status st = check_heads(t.x_desc, p.B, p.L, p.D)) return st;
      if (t.x_desc->H != t.dout_desc->H) return SVD_ERR_SHAPE;
      x = *t.x_desc;
      if (!aligned16(t.x)) return SVD_ERR_ALIGN;
      if (t.dx == t.x) return SVD_ERR_UNSUPPORTED;
    } else if (t.weight || t.dweight || t.dbias) {
      return SVD_ERR_PARAMS;
    }
    if (!aligned16(t.dout) || !aligned16(t.dx) || !aligned16(t.weight) || !aligned16(t.dweight) || !aligned16(t.dbias))
      return SVD_ERR_ALIGN;
    if (t.dout == t.dx && !same_layout(*t.dout_desc, *t.dx_desc)) return SVD_ERR_UNSUPPORTED;
    any = any || t.dweight || t.dbias;
    const svd_tensor_desc &g = *t.dout_desc, &o = *t.dx_desc;
    p.t[i] = {static_cast<const __bf16*>(norm != SVD_NORM_NONE ? t.x : nullptr), static_cast<const __bf16*>(t.dout),
              static_cast<__bf16*>(t.dx), g.H, x.stride_b, x.stride_h, x.stride_l, g.stride_b, g.stride_h, g.stride_l,
              o.stride_b, o.stride_h, o.stride_l, t.weight, nullptr, t.dweight, t.dbias};
  }
  if (n_tensors == 2) {
    const svd_rope_grad &a = tensors[0], &b = tensors[1];
    if (a.dx == b.dx || a.dx == b.dout || b.dx == a.dout || (p.t[1].x && a.dx == b.x) || (p.t[0].x && b.dx == a.x))
      return SVD_ERR_UNSUPPORTED;
  }
  if (any) {
    const size_t need = static_cast<size_t>(2) * svd::kRopePartials * 2 * p.D * sizeof(float);
    if (!device_workspace || !aligned16(device_workspace) || workspace_bytes < need) return SVD_ERR_WORKSPACE;
    p.partial = static_cast<float*>(device_workspace);
  }
  return status_of(svd::launch_rope_backward(p, static_cast<hipStream_t>(hip_stream)));
}

svd_status svd_blockscale_quantise(const void* src, int32_t src_type, int32_t R, int32_t C, int64_t src_stride,
                                   int32_t transpose, void* dst, int64_t dst_stride, uint8_t* scales, int64_t scale_stride,
                                   void* hip_stream) {
  if (!src || !dst || !scales) return SVD_ERR_NULL;
  if (src_type != SVD_BF16 && src_type != SVD_F32) return SVD_ERR_DTYPE;
  if (R < 1 || C < 1 || R >= kMaxMatrix || C >= kMaxMatrix) return SVD_ERR_SHAPE;
  const int64_t rows = transpose ? C : R, cols = transpose ? R : C;
  if ((R > 1 && src_stride < C) || src_stride > kMaxStride || (rows > 1 && dst_stride < round16(cols)) || dst_stride > kMaxStride ||
      scale_stride < rows || scale_stride > kMaxStride)
    return SVD_ERR_SHAPE;
  if (!aligned16(src) || !aligned16(dst) || !aligned16(scales) || dst_stride % 16 || scale_stride % 16 ||
      (R > 1 && src_stride % (src_type == SVD_F32 ? 4 : 8)))
    return SVD_ERR_ALIGN;
  if (dst == src) return SVD_ERR_UNSUPPORTED;
  const svd::QuantLaunch p{src, src_type, R, C, src_stride, static_cast<uint8_t*>(dst), dst_stride, scales, scale_stride};
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  return status_of(transpose ? svd::launch_quantise_columns(p, stream) : svd::launch_quantise_rows(p, stream));
}

static svd_status check_matmul(const svd_blockscale_desc& d) {
  if (d.M < 1 || d.N < 1 || d.K < 1 || d.M >= kMaxMatrix || d.N >= kMaxMatrix || d.K >= kMaxMatrix) return SVD_ERR_SHAPE;
  const int64_t K16 = round16(d.K);
  if (d.a_stride < K16 || d.b_stride < K16 || d.out_stride < d.N || d.a_scale_stride < d.M || d.b_scale_stride < d.N)
    return SVD_ERR_SHAPE;
  if (d.a_stride >= kMaxMatrixStride || d.b_stride >= kMaxMatrixStride || d.out_stride > kMaxStride) return SVD_ERR_UNSUPPORTED;
  if (d.a_stride % 16 || d.b_stride % 16 || d.a_scale_stride % 16 || d.b_scale_stride % 16) return SVD_ERR_ALIGN;
  // the kernels address the scales of a matrix with 32-bit byte offsets
  const int64_t blocks = (d.K + 127) / 128;
  if (blocks > INT32_MAX / d.a_scale_stride || blocks > INT32_MAX / d.b_scale_stride) return SVD_ERR_UNSUPPORTED;
  return SVD_OK;
}

svd_status svd_blockscale_matmul(const svd_blockscale_desc* desc, const void* a, const uint8_t* a_scales, const void* b,
                                 const uint8_t* b_scales, const float* bias, void* out, void* hip_stream) {
  if (!desc || !a || !a_scales || !b || !b_scales || !out) return SVD_ERR_NULL;
  if (svd_status st = check_matmul(*desc)) return st;
  if (!aligned16(a) || !aligned16(b) || !aligned16(a_scales) || !aligned16(b_scales) || (reinterpret_cast<uintptr_t>(bias) & 3u) ||
      (reinterpret_cast<uintptr_t>(out) & 1u))
    return SVD_ERR_ALIGN;
  if (out == a || out == b) return SVD_ERR_UNSUPPORTED;
  const svd::MatmulLaunch p{*desc, static_cast<const uint8_t*>(a), a_scales, static_cast<const uint8_t*>(b), b_scales, bias,
                            static_cast<__bf16*>(out)};
  return status_of(svd::launch_blockscale_matmul(p, static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
