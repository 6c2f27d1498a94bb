// gfx950 kernels of the residual update and the norms around a block of a layer:
//   u = post_norm(y) * post_weight, x' = x + gate * u, h = (norm(x') * weight + bias) * (1 + scale) + shift,
// and their gradients.  Streaming kernels bound by HBM: a row is read once, kept in registers as 8 channels per thread
// (16 from 520 to 1,024 channels and above 2,048, 32 above 8,192), and everything that depends on it leaves in the same pass.
// (75,600 x 5,120 bf16 with y and gate: 597 us, 5.2 TB/s, a copy's 5.0.  Ahead of the joint reading of statistics below: 16 channels
// a thread and 256 registers 621; 8 a thread, ten waves to a row, 730; 16 a thread in 128 registers 742, they spill.)
//
// A work-group walks the rows of one chunk, which lies within one group, so its slices of gate, scale, shift and weights
// stay in registers, folded into three factors.  The next row's loads are in flight while a row is worked on.
//
// Statistics: a wave takes the mean of its part and the squares of the deviations from it, and the parts are joined with
// the deviations of their means (sum of squares = sum_w [M2_w + n_w (m_w - m)^2]): one barrier, and no cancellation.  What the
// waves tell one another is read all at once, and a backward pass takes the statistics of both its rows in one go: three
// barriers a row (20,000 x 5,120 with a norm of y: 285 us; read wave by wave, one norm after the other, 392).
#include <hip/hip_runtime.h>

#include "layer_ops.h"
#include "wave_ops.h"

namespace svd {
namespace {

constexpr int kMaxThreads = 512;
constexpr int waves_of(int pieces) { return pieces == 1 ? 4 : 8; }   // of a work-group, at most

// LANES > 0: a row's, of several that the work-group takes at once; 0: the work-group takes one row.
template <int NJ, int LANES>
struct Lanes {
  int at[NJ];                // first channel
  bool on[NJ];
  int count[waves_of(NJ)];   // channels of the work-group's waves
  __device__ __forceinline__ Lanes(int C) {
    const int T = LANES ? LANES : blockDim.x;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      at[j] = ((LANES ? threadIdx.x % LANES : threadIdx.x) + j * T) * 8;
      on[j] = at[j] < C;
    }
#pragma unroll
    for (int w = 0; w < waves_of(NJ); ++w) {
      count[w] = 0;
#pragma unroll
      for (int j = 0; j < NJ; ++j) count[w] += w * 64 < T ? min(max(C - (w * 64 + j * T) * 8, 0), 512) : 0;
    }
  }
};

// What the waves of a row have to say to one another: a float of each wave, zeros of those that the work-group does not have, so
// that all can be read at once.  Written by no other reduction until two barriers later.
template <int NJ>
struct __attribute__((aligned(16))) Slot {
  float of[waves_of(NJ)];
};
template <int NJ>
__device__ __forceinline__ void clear_slots(Slot<NJ>* slots, int n) {
  const int w = threadIdx.x % waves_of(NJ);
  if (w >= (int)blockDim.x >> 6)
    for (int i = threadIdx.x / waves_of(NJ); i < n; i += blockDim.x / waves_of(NJ)) slots[i].of[w] = 0.f;
}
__device__ __forceinline__ float sum8(const f32x8 v) { return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])); }
template <int N>
__device__ __forceinline__ float sum_of_waves(const float (&v)[N]) {
  const float s = (v[0] + v[1]) + (v[2] + v[3]);
  if constexpr (N == 8) return s + ((v[4] + v[5]) + (v[6] + v[7]));
  else return s;
}

// Sums over a row's values.
template <int LANES, int NV, int NJ>
__device__ __forceinline__ void row_sum(float (&v)[NV], Slot<NJ>* slot) {
#pragma unroll
  for (int i = 0; i < NV; ++i) v[i] = lane_sum<LANES ? LANES : 64>(v[i]);
  if (LANES) return;
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int i = 0; i < NV; ++i) slot[i].of[threadIdx.x >> 6] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NV; ++i) v[i] = sum_of_waves(slot[i].of);
}

// Mean (0 for RMS) and squared deviations from it, of a wave's part of a row, or of all of it (LANES > 0).
struct Part {
  float m, q;
};
template <int NJ, int LANES>
__device__ __forceinline__ Part part_of(const f32x8 (&v)[NJ], const Lanes<NJ, LANES>& ln, const int C, const int kind) {
  Part p = {0.f, 0.f};
  if (kind == SVD_NORM_LAYER) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) p.m += sum8(v[j]);
    int count = C;
    if (!LANES) {
      count = 0;
#pragma unroll
      for (int j = 0; j < NJ; ++j) count += min(max(C - (int)((threadIdx.x & ~63u) + j * blockDim.x) * 8, 0), 512);
    }
    p.m = lane_sum<LANES ? LANES : 64>(p.m) / (float)count;
  }
#pragma unroll
  for (int j = 0; j < NJ; ++j)
    if (ln.on[j])
#pragma unroll
      for (int i = 0; i < 8; ++i) p.q = __builtin_fmaf(v[j][i] - p.m, v[j][i] - p.m, p.q);
  p.q = lane_sum<LANES ? LANES : 64>(p.q);
  return p;
}
template <int NJ>
__device__ __forceinline__ void tell(const Part& p, Slot<NJ>* slot) {
  if ((threadIdx.x & 63) == 0) {
    slot[0].of[threadIdx.x >> 6] = p.m;
    slot[1].of[threadIdx.x >> 6] = p.q;
  }
}

struct Stats {
  float mean, rstd;
};
// Mean and 1 / sqrt(variance + eps) of a row from its parts.
template <int NJ, int LANES>
__device__ __forceinline__ Stats joined(Part p, const Slot<NJ>* slot, const Lanes<NJ, LANES>& ln, const int C, const int kind, const float eps) {
  if (!LANES) {
    constexpr int W = waves_of(NJ);
    float q[W];
#pragma unroll
    for (int w = 0; w < W; ++w) q[w] = slot[1].of[w];
    if (kind == SVD_NORM_LAYER) {
      float m[W], s[W];
#pragma unroll
      for (int w = 0; w < W; ++w) {
        m[w] = slot[0].of[w];
        s[w] = m[w] * (float)ln.count[w];
      }
      p.m = sum_of_waves(s) / (float)C;
#pragma unroll
      for (int w = 0; w < W; ++w) q[w] += (m[w] - p.m) * (m[w] - p.m) * (float)ln.count[w];
    }
    p.q = sum_of_waves(q);
  }
  return {p.m, 1.f / __builtin_sqrtf(p.q / (float)C + eps)};
}
template <int NJ, int LANES>
__device__ __forceinline__ Stats row_stats(const f32x8 (&v)[NJ], const Lanes<NJ, LANES>& ln, const int C, const int kind, const float eps, Slot<NJ>* slot) {
  const Part p = part_of(v, ln, C, kind);
  if (!LANES) {
    tell(p, slot);
    __syncthreads();
  }
  return joined(p, slot, ln, C, kind, eps);
}

template <typename XT>
__device__ __forceinline__ XT* row_of(const RowsView& r, int b, int row) {
  return static_cast<XT*>(r.data) + (int64_t)b * r.stride_b + (int64_t)row * r.stride_l;
}

template <int NJ, int LANES, typename XT>
__global__ void __launch_bounds__(NJ == 1 || LANES ? 256 : 512) norm_forward_kernel(const NormLaunch p) {
  __shared__ Slot<NJ> slots[2][2][2];   // [row parity][y, x'][mean, squares]
  const ChunkAt ch = chunk_at(p.ch, blockIdx.x);
  const Lanes<NJ, LANES> ln(p.C);
  constexpr int ROWS = LANES ? 256 / LANES : 1;   // at once
  const bool has_y = p.y.data != nullptr, has_h = p.h.data != nullptr;
  const int64_t mod = ch.b * p.mod_stride_b + ch.g * p.mod_stride_g;
  f32x8 gate[NJ], mul[NJ], add[NJ];   // gate * post_weight; (1 + scale) * weight; (1 + scale) * bias + shift
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const f32x8 zero = {0, 0, 0, 0, 0, 0, 0, 0}, one = zero + 1.f;
    auto vec = [&](const float* v, const f32x8 none) { return v && ln.on[j] ? load8(v + ln.at[j]) : none; };
    auto mod_vec = [&](const float* v, const f32x8 none) { return vec(v ? v + mod : v, none); };
    gate[j] = mod_vec(p.vec.gate, one) * vec(p.vec.post_weight, one);
    const f32x8 s = mod_vec(p.vec.scale, zero) + 1.f;
    mul[j] = s * vec(p.vec.weight, one);
    add[j] = s * vec(p.vec.bias, zero) + mod_vec(p.vec.shift, zero);
  }
  Raw8<XT> x_next[NJ];
  Raw8<__bf16> y_next[NJ];
  auto request = [&](int row) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      x_next[j].v = decltype(x_next[j].v){};
      y_next[j].v = decltype(y_next[j].v){};
      if (!ln.on[j]) continue;
      x_next[j].load(row_of<const XT>(p.x, ch.b, row) + ln.at[j]);
      if (has_y) y_next[j].load(row_of<const __bf16>(p.y, ch.b, row) + ln.at[j]);
    }
  };
  // a row at a time: row + 1 is at most ch.row1
  auto behind = [&](int row, int step) { return LANES ? row_behind(row, step, ch.row1) : row + step; };
  const int row0 = behind(ch.row0, LANES ? (int)threadIdx.x / LANES : 0);
  if (row0 < ch.row1) request(row0);
  if (!LANES) clear_slots(&slots[0][0][0], sizeof(slots) / sizeof(slots[0][0][0]));
  for (int row = row0; row < ch.row1; row = behind(row, ROWS)) {
    f32x8 x[NJ], y[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      x[j] = x_next[j].get();
      y[j] = y_next[j].get();
    }
    if (behind(row, ROWS) < ch.row1) request(behind(row, ROWS));
    Slot<NJ> (*slot)[2] = slots[row & 1];
    if (has_y) {
      Stats st = {0.f, 1.f};
      if (p.post_norm != SVD_NORM_NONE) st = row_stats(y, ln, p.C, p.post_norm, p.eps, slot[0]);
#pragma unroll
      for (int j = 0; j < NJ; ++j)
        if (ln.on[j]) {
          x[j] += gate[j] * ((y[j] - st.mean) * st.rstd);
          store8(row_of<XT>(p.x_out, ch.b, row) + ln.at[j], x[j]);
        }
    }
    if (!has_h) continue;
    const Stats st = row_stats(x, ln, p.C, p.norm, p.eps, slot[1]);
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const f32x8 h = (x[j] - st.mean) * st.rstd * mul[j] + add[j];
      if (!p.h_scales) {
        if (ln.on[j]) store8(row_of<__bf16>(p.h, ch.b, row) + ln.at[j], h);
        continue;
      }
      // 16 lanes hold a block of 128 channels (lanes past the last channel: nothing)
      int top = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, ln.on[j] ? magnitude(h[i]) : 0);
      const int byte = scale_byte(max16(top));
      const float f = scale_inverse(byte);
      if (!ln.on[j]) continue;
      u32x2 w = {(unsigned)pack_e4m3(h[0] * f, h[1] * f, h[2] * f, h[3] * f),
                 (unsigned)pack_e4m3(h[4] * f, h[5] * f, h[6] * f, h[7] * f)};
      *reinterpret_cast<u32x2*>(row_of<uint8_t>(p.h, ch.b, row) + ln.at[j]) = w;
      if ((threadIdx.x & 15) == 0) p.h_scales[(int64_t)(ln.at[j] >> 7) * p.h_scale_stride + (int64_t)ch.b * p.ch.L + row] = (uint8_t)byte;
    }
  }
}

// Gradients of a row, with n = norm(x'), a = (1 + scale) * weight, ny = post_norm(y):
//   dn = dh a,  dx = dx_out + r (dn - mean(dn) - n mean(dn n)),     (mean(dn): layer norms only)
//   dv = dx gate post_weight,  dy = ry (dv - mean(dv) - ny mean(dv ny)),  or dx gate without a norm of y.
// What the vectors need of a group's rows are three sums per channel: S1 = sum dh, S2 = sum dh n, T2 = sum dx ny; a
// work-group leaves those of its chunk, and the second kernel adds the chunks of a group in order, in 64 bits.
template <int NJ, int LANES, typename XT>
__global__ void __launch_bounds__(NJ == 1 || LANES ? 256 : 512) norm_backward_kernel(const NormLaunch p) {
  __shared__ Slot<NJ> slots[2][4][2];   // [row parity][x', y, sums of x', of y]
  const ChunkAt ch = chunk_at(p.ch, blockIdx.x);
  const Lanes<NJ, LANES> ln(p.C);
  constexpr int ROWS = LANES ? 256 / LANES : 1;   // at once
  const bool has_y = p.y.data != nullptr, has_h = p.dh.data != nullptr, has_up = p.dx_out.data != nullptr;
  const bool post = p.post_norm != SVD_NORM_NONE;
  const int64_t mod = ch.b * p.mod_stride_b + ch.g * p.mod_stride_g;
  const f32x8 zero = {0, 0, 0, 0, 0, 0, 0, 0}, one = zero + 1.f;
  const float inv_c = 1.f / (float)p.C;
  // Above 8,192 channels the three sums and a row do not fit the registers: two sums stay in LDS, the factors are read anew for
  // every row, and no row is requested ahead.  (8,000 x 16,384 bf16: 698 us where all in registers took 2,590, 556 of them spilled; 456 now.)
  constexpr bool kLean = NJ > 2;
  __shared__ f32x4 lds_sums[kLean ? 4 * NJ * kMaxThreads : 1];
  f32x8 sums[2][kLean ? 1 : NJ], t2[NJ], kept[2][kLean ? 1 : NJ];
  auto lds_sum = [&](int k, int j, int half) -> f32x4& { return lds_sums[kLean ? ((k * NJ + j) * 2 + half) * kMaxThreads + threadIdx.x : 0]; };
  auto sum_of = [&](int k, int j) -> f32x8 {
    if (!kLean) return sums[k][kLean ? 0 : j];
    const f32x4 a = lds_sum(k, j, 0), b = lds_sum(k, j, 1);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto set_sum = [&](int k, int j, const f32x8 v) {
    if (!kLean) {
      sums[k][kLean ? 0 : j] = v;
    } else {
      lds_sum(k, j, 0) = __builtin_shufflevector(v, v, 0, 1, 2, 3);
      lds_sum(k, j, 1) = __builtin_shufflevector(v, v, 4, 5, 6, 7);
    }
  };
  auto vec = [&](const float* v, int j, const f32x8 none) { return v && ln.on[j] ? load8(v + ln.at[j]) : none; };
  auto mod_vec = [&](const float* v, int j, const f32x8 none) { return vec(v ? v + mod : v, j, none); };
  auto gate_now = [&](int j) { return mod_vec(p.vec.gate, j, one) * vec(p.vec.post_weight, j, one); };
  auto mul_now = [&](int j) { return (mod_vec(p.vec.scale, j, zero) + 1.f) * vec(p.vec.weight, j, one); };
  auto gate = [&](int j) { return kLean ? gate_now(j) : kept[0][kLean ? 0 : j]; };
  auto mul = [&](int j) { return kLean ? mul_now(j) : kept[1][kLean ? 0 : j]; };
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    if (!kLean) {
      kept[0][kLean ? 0 : j] = gate_now(j);
      kept[1][kLean ? 0 : j] = mul_now(j);
    }
    t2[j] = zero;
    set_sum(0, j, zero);
    set_sum(1, j, zero);
  }
  Raw8<XT> x_next[NJ], up_next[NJ];
  Raw8<__bf16> y_next[NJ], dh_next[NJ];
  auto request = [&](int row) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      x_next[j].v = up_next[j].v = decltype(x_next[j].v){};
      y_next[j].v = dh_next[j].v = decltype(y_next[j].v){};
      if (!ln.on[j]) continue;
      x_next[j].load(row_of<const XT>(p.x_out, ch.b, row) + ln.at[j]);
      if (has_up) up_next[j].load(row_of<const XT>(p.dx_out, ch.b, row) + ln.at[j]);
      if (has_h) dh_next[j].load(row_of<const __bf16>(p.dh, ch.b, row) + ln.at[j]);
      if (has_y) y_next[j].load(row_of<const __bf16>(p.y, ch.b, row) + ln.at[j]);
    }
  };
  auto behind = [&](int row, int step) { return LANES ? row_behind(row, step, ch.row1) : row + step; };
  const int row0 = behind(ch.row0, LANES ? (int)threadIdx.x / LANES : 0);
  if (!kLean && row0 < ch.row1) request(row0);
  if (!LANES) clear_slots(&slots[0][0][0], sizeof(slots) / sizeof(slots[0][0][0]));
  for (int row = row0; row < ch.row1; row = behind(row, ROWS)) {
    f32x8 x[NJ], y[NJ], dh[NJ], dx[NJ];
    if (kLean) request(row);
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      x[j] = x_next[j].get();
      y[j] = y_next[j].get();
      dh[j] = dh_next[j].get();
      dx[j] = up_next[j].get();
    }
    if (!kLean && behind(row, ROWS) < ch.row1) request(behind(row, ROWS));
    Slot<NJ> (*slot)[2] = slots[row & 1];
    // the statistics of both rows in one go
    Part px = {0.f, 0.f}, py = {0.f, 0.f};
    if (has_h) px = part_of(x, ln, p.C, p.norm);
    if (has_y && post) py = part_of(y, ln, p.C, p.post_norm);
    if (!LANES && (has_h || (has_y && post))) {
      tell(px, slot[0]);
      tell(py, slot[1]);
      __syncthreads();
    }
    if (has_h) {
      const Stats st = joined(px, slot[0], ln, p.C, p.norm, p.eps);
      float c[2] = {0.f, 0.f};
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        x[j] = (x[j] - st.mean) * st.rstd;   // n
        if (ln.on[j]) {
          set_sum(0, j, sum_of(0, j) + dh[j]);
          set_sum(1, j, sum_of(1, j) + dh[j] * x[j]);
        }
        dh[j] *= mul(j);                     // dn (0 past the last channel)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          c[0] += dh[j][i];
          c[1] = __builtin_fmaf(dh[j][i], x[j][i], c[1]);
        }
      }
      row_sum<LANES>(c, slot[2]);
      const float c0 = p.norm == SVD_NORM_LAYER ? c[0] * inv_c : 0.f, c1 = c[1] * inv_c;
#pragma unroll
      for (int j = 0; j < NJ; ++j) dx[j] += (dh[j] - c0 - x[j] * c1) * st.rstd;
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j)
      if (ln.on[j]) store8(row_of<XT>(p.dx, ch.b, row) + ln.at[j], dx[j]);
    if (!has_y) continue;
    Stats st = {0.f, 1.f};
    if (post) st = joined(py, slot[1], ln, p.C, p.post_norm, p.eps);
    float c[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      y[j] = (y[j] - st.mean) * st.rstd;     // ny
      if (ln.on[j]) t2[j] += dx[j] * y[j];
      dx[j] *= gate(j);                      // dv
      if (!ln.on[j]) dx[j] = y[j] = zero;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        c[0] += dx[j][i];
        c[1] = __builtin_fmaf(dx[j][i], y[j][i], c[1]);
      }
    }
    if (post) {
      row_sum<LANES>(c, slot[3]);
      const float c0 = p.post_norm == SVD_NORM_LAYER ? c[0] * inv_c : 0.f, c1 = c[1] * inv_c;
#pragma unroll
      for (int j = 0; j < NJ; ++j) dx[j] = (dx[j] - c0 - y[j] * c1) * st.rstd;
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j)
      if (ln.on[j]) store8(row_of<__bf16>(p.dy, ch.b, row) + ln.at[j], dx[j]);
  }
  if (!p.partial) return;
  float* out = p.partial + (int64_t)blockIdx.x * 3 * p.C;
  if constexpr (LANES > 0) {   // of the rows that went at once, in order
    constexpr int CHANNELS = LANES * 8 * NJ;
    __shared__ __attribute__((aligned(16))) float parts[ROWS][3][CHANNELS];
    float (*mine)[CHANNELS] = parts[threadIdx.x / LANES];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      store8(mine[0] + ln.at[j], sum_of(0, j));
      store8(mine[1] + ln.at[j], sum_of(1, j));
      store8(mine[2] + ln.at[j], t2[j]);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 3 * CHANNELS; i += 256) {
      const int k = i / CHANNELS, c = i % CHANNELS;
      float s = 0.f;
      for (int r = 0; r < ROWS; ++r) s += parts[r][k][c];
      if (c < p.C) out[k * p.C + c] = s;
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < NJ; ++j)
    if (ln.on[j]) {
      store8(out + ln.at[j], sum_of(0, j));
      store8(out + p.C + ln.at[j], sum_of(1, j));
      store8(out + 2 * p.C + ln.at[j], t2[j]);
    }
}

// Work-group (32 channels, entry and group): the sums of the group's chunks, the gradients of its gate, scale and shift,
// and its share in those of the weights.  LANES = 1: 256 channels, a thread each.
template <int LANES>
__global__ void __launch_bounds__(LANES == 1 ? 256 : 32 * LANES) norm_group_kernel(const NormLaunch p) {
  constexpr int COLUMNS = LANES == 1 ? 256 : 32;
  const int column = threadIdx.x % COLUMNS, c = blockIdx.x * COLUMNS + column, bg = join_at(blockIdx.y, blockIdx.z);
  if (bg >= p.B * p.ch.groups) return;
  const int b = bg / p.ch.groups, g = bg % p.ch.groups;
  const ChunkRange chunks = chunks_of(p.ch, g);
  const float* in = p.partial + ((int64_t)b * p.ch.per_entry + chunks.first) * 3 * p.C + c;
  float s1, s2, t2;
  if constexpr (LANES == 1) {
    if (c >= p.C) return;
    double s[3] = {};
    for (int i = chunks.first; i < chunks.second; ++i, in += (int64_t)3 * p.C)
#pragma unroll
      for (int k = 0; k < 3; ++k) s[k] += (double)in[k * p.C];
    s1 = (float)s[0], s2 = (float)s[1], t2 = (float)s[2];
  } else {
    __shared__ double slots[3][LANES][32];
    __shared__ float sums[3][32];
    const double s = column_sums<LANES, 3>(in, p.C, (int64_t)3 * p.C, chunks.second - chunks.first, c < p.C, slots);
    if (threadIdx.x < 96) sums[threadIdx.x / 32][column] = (float)s;
    __syncthreads();
    if (c >= p.C || threadIdx.x >= 32) return;
    s1 = sums[0][column], s2 = sums[1][column], t2 = sums[2][column];
  }
  const int64_t mod = b * p.mod_stride_b + g * p.mod_stride_g + c, at = (int64_t)bg * p.C + c;
  const float w = p.vec.weight ? p.vec.weight[c] : 1.f, bias = p.vec.bias ? p.vec.bias[c] : 0.f;
  const float pw = p.vec.post_weight ? p.vec.post_weight[c] : 1.f;
  const float scale = 1.f + (p.vec.scale ? p.vec.scale[mod] : 0.f), gate = p.vec.gate ? p.vec.gate[mod] : 1.f;
  if (p.grads.shift) p.grads.shift[at] = s1;
  if (p.grads.scale) p.grads.scale[at] = __builtin_fmaf(w, s2, bias * s1);
  if (p.grads.gate) p.grads.gate[at] = pw * t2;
  if (p.B * p.ch.groups == 1) {
    if (p.grads.weight) p.grads.weight[c] = scale * s2;
    if (p.grads.bias) p.grads.bias[c] = scale * s1;
    if (p.grads.post_weight) p.grads.post_weight[c] = gate * t2;
  } else if (p.grads.weight || p.grads.bias || p.grads.post_weight) {
    float* out = p.sums + (int64_t)bg * 3 * p.C + c;
    out[0] = scale * s2;
    out[p.C] = scale * s1;
    out[2 * p.C] = gate * t2;
  }
}

// Work-group (32 channels, weight): the groups' shares.
template <int LANES>
__global__ void __launch_bounds__(32 * LANES) norm_weight_kernel(const NormLaunch p) {
  __shared__ double slots[1][LANES][32];
  const int c = blockIdx.x * 32 + threadIdx.x % 32, k = blockIdx.y;
  float* out = k == 0 ? p.grads.weight : k == 1 ? p.grads.bias : p.grads.post_weight;
  if (!out) return;
  const double s = column_sums<LANES, 1>(p.sums + (int64_t)k * p.C + c, 0, (int64_t)3 * p.C, p.B * p.ch.groups, c < p.C, slots);
  if (c < p.C && threadIdx.x < 32) out[c] = (float)s;
}

template <typename Launch>
void with_type(int stream_type, Launch launch) {
  if (stream_type == SVD_F32) launch(float{});
  else launch(__bf16{});
}

}  // namespace

// Launches KERNEL<pieces, lanes, type of the stream> for p.C channels.
#define SVD_NORM_LAUNCH(KERNEL)                                                                                                    \
  with_type(p.stream_type, [&](auto type) {                                                                                        \
    using T = decltype(type);                                                                                                      \
    const NormShape s = norm_shape(p.C, p.ch.group);                                                                               \
    const auto kernel = s.lanes == 16 ? KERNEL<1, 16, T> : s.lanes == 32 ? KERNEL<1, 32, T>                                        \
                        : s.lanes == 64 ? (s.pieces == 1 ? KERNEL<1, 64, T> : KERNEL<2, 64, T>)                                    \
                        : s.pieces == 1 ? KERNEL<1, 0, T> : s.pieces == 2 ? KERNEL<2, 0, T> : KERNEL<4, 0, T>;                     \
    hipLaunchKernelGGL(kernel, dim3((unsigned)p.B * p.ch.per_entry), dim3(s.threads), 0, stream, p);                               \
  })

hipError_t launch_norm_forward(const NormLaunch& p, hipStream_t stream) {
  SVD_NORM_LAUNCH(norm_forward_kernel);
  return hipGetLastError();
}

hipError_t launch_norm_backward(const NormLaunch& p, hipStream_t stream) {
  SVD_NORM_LAUNCH(norm_backward_kernel);
  if (hipError_t e = hipGetLastError(); e != hipSuccess || !p.partial) return e;
  const int n = p.B * p.ch.groups, columns = (p.C + 31) / 32;
  dim3 groups(columns, n < kJoinRow ? n : kJoinRow, (n + kJoinRow - 1) / kJoinRow);
  const int lanes = join_lanes(p.ch);
  if (lanes == 32) hipLaunchKernelGGL(norm_group_kernel<32>, groups, dim3(1024), 0, stream, p);
  else if (lanes == 8) hipLaunchKernelGGL(norm_group_kernel<8>, groups, dim3(256), 0, stream, p);
  else {
    groups.x = (p.C + 255) / 256;
    hipLaunchKernelGGL(norm_group_kernel<1>, groups, dim3(256), 0, stream, p);
  }
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if (n > 1 && (p.grads.weight || p.grads.bias || p.grads.post_weight))
    hipLaunchKernelGGL(norm_weight_kernel<32>, dim3(columns, 3), dim3(1024), 0, stream, p);
  return hipGetLastError();
}

}  // namespace svd
