// gfx950 kernels of the per-head norm of q and k with the rotary positions of time, height and width, and their
// gradients.  Streaming kernels bound by HBM.
//
// A thread owns one token and 8 channels of a head (4 pairs): it forms the token's frame, row and column and reads its 4
// cosines and sines once, then walks the heads, whose norm is a sum over the 8 or 16 lanes of the head's row.
#include <hip/hip_runtime.h>

#include "layer_ops.h"
#include "wave_ops.h"

namespace svd {
namespace {

constexpr int kThreads = kRopeThreads;

// A thread's 8 channels: 8 in a row (pairs of neighbours), or 4 from either half.
template <bool HALVES>
struct Piece {
  static __device__ __forceinline__ bf16x8 raw(const __bf16* row, int c, int D) {
    if (!HALVES) return *reinterpret_cast<const bf16x8*>(row + 8 * c);
    const bf16x4 a = *reinterpret_cast<const bf16x4*>(row + 4 * c), b = *reinterpret_cast<const bf16x4*>(row + D / 2 + 4 * c);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  static __device__ __forceinline__ f32x8 load(const float* row, int c, int D) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(row + (HALVES ? 4 * c : 8 * c));
    const f32x4 b = *reinterpret_cast<const f32x4*>(row + (HALVES ? D / 2 + 4 * c : 8 * c + 4));
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  static __device__ __forceinline__ void store(__bf16* row, int c, int D, const f32x8 v) {
    const bf16x8 w = __builtin_convertvector(v, bf16x8);
    if (!HALVES) {
      *reinterpret_cast<bf16x8*>(row + 8 * c) = w;
    } else {
      *reinterpret_cast<bf16x4*>(row + 4 * c) = __builtin_shufflevector(w, w, 0, 1, 2, 3);
      *reinterpret_cast<bf16x4*>(row + D / 2 + 4 * c) = __builtin_shufflevector(w, w, 4, 5, 6, 7);
    }
  }
  static __device__ __forceinline__ void store(float* row, int c, int D, const f32x8 v) {
    *reinterpret_cast<f32x4*>(row + (HALVES ? 4 * c : 8 * c)) = __builtin_shufflevector(v, v, 0, 1, 2, 3);
    *reinterpret_cast<f32x4*>(row + (HALVES ? D / 2 + 4 * c : 8 * c + 4)) = __builtin_shufflevector(v, v, 4, 5, 6, 7);
  }
  // pair i of the piece: channels (2i, 2i + 1) of it, or (i, i + 4)
  static constexpr int first(int i) { return HALVES ? i : 2 * i; }
  static constexpr int second(int i) { return HALVES ? i + 4 : 2 * i + 1; }
};

struct Angles {
  float cos[4], sin[4];
};
// Of pairs 4c .. 4c + 3 of the token in row l.
__device__ __forceinline__ Angles angles_of(const RopeLaunch& p, const int l, const int c) {
  Angles a;
  const svd_rope_desc& r = p.r;
  const Place q = place_of(r.row_offset + l - r.first, r.frames, r.height, r.width, r.position_major != 0);
  const int at_t = q.frame * r.pairs_t, at_h = r.frames * r.pairs_t + q.y * r.pairs_h;
  const int at_w = r.frames * r.pairs_t + r.height * r.pairs_h + q.x * r.pairs_w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    int j = 4 * c + i, at = at_t + j;
    bool turns = j < r.pairs_t;
    j -= r.pairs_t;
    if (!turns && j < r.pairs_h) {
      at = at_h + j;
      turns = true;
    }
    if (!turns) {
      j -= r.pairs_h;
      at = at_w + j;
      turns = j < r.pairs_w;
    }
    a.cos[i] = 1.f;
    a.sin[i] = 0.f;
    if (turns && q.video) {
      const float2 cs = reinterpret_cast<const float2*>(p.table)[at];
      a.cos[i] = cs.x;
      a.sin[i] = cs.y;
    }
  }
  return a;
}

template <bool HALVES>
__device__ __forceinline__ f32x8 turn(const f32x8 v, const Angles& a, const float sign) {
  typedef Piece<HALVES> P;
  f32x8 o;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float x = v[P::first(i)], y = v[P::second(i)], s = sign * a.sin[i];
    // What does not turn keeps its bits, zeros' signs too, whatever stands beside it: 1 * 0 is subtracted, -1 * 0 added.
    const bool turns = s != 0.f;
    const float one = __builtin_copysignf(1.f, s), xs = turns ? x : -one, ys = turns ? y : one;
    o[P::first(i)] = __builtin_fmaf(x, a.cos[i], -(ys * s));
    o[P::second(i)] = __builtin_fmaf(xs, s, y * a.cos[i]);
  }
  return o;
}

__device__ __forceinline__ float sum8(const f32x8 v) { return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])); }

// Normalised channels of a head in place; returns 1 / sqrt(variance + eps).
template <int LANES>
__device__ __forceinline__ float normalise(f32x8& v, const int kind, const float eps) {
  constexpr float inv = 1.f / (8 * LANES);
  if (kind == SVD_NORM_LAYER) v -= lane_sum<LANES>(sum8(v)) * inv;
  const float r = 1.f / __builtin_sqrtf(lane_sum<LANES>(sum8(v * v)) * inv + eps);
  v *= r;
  return r;
}

// grid: tokens / (kThreads / LANES), entry, tensor * splits + part of the heads.
template <int D, bool HALVES>
__global__ void __launch_bounds__(kThreads) rope_forward_kernel(const RopeLaunch p, const int splits) {
  constexpr int LANES = D / 8;
  typedef Piece<HALVES> P;
  const RopeTensor& t = p.t[blockIdx.z / splits];
  const int c = threadIdx.x % LANES, l = blockIdx.x * (kThreads / LANES) + threadIdx.x / LANES, b = blockIdx.y;
  if (l >= p.L) return;
  const HeadRange heads = heads_of_part(t.H, splits, blockIdx.z % splits);
  const Angles a = angles_of(p, l, c);
  const f32x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
  const f32x8 w = t.weight ? P::load(t.weight, c, D) : zero + 1.f, bias = t.bias ? P::load(t.bias, c, D) : zero;
  const __bf16* x = t.x + (int64_t)b * t.x_b + (int64_t)l * t.x_l;
  __bf16* o = t.out + (int64_t)b * t.o_b + (int64_t)l * t.o_l;
  for (int h = heads.first; h < heads.last; ++h) {
    f32x8 v = __builtin_convertvector(P::raw(x + (int64_t)h * t.x_h, c, D), f32x8);
    if (p.norm != SVD_NORM_NONE) {
      normalise<LANES>(v, p.norm, p.eps);
      v = v * w + bias;
    }
    P::store(o + (int64_t)h * t.o_h, c, D, turn<HALVES>(v, a, 1.f));
  }
}

// d = turned back dout; dweight = sum d n, dbias = sum d over all rows; dx = r (dn - mean(dn) - n mean(dn n)), dn = d w.
// A work-group walks units of a block of tokens and a part of the heads.  The next head's loads are in flight while a head is worked on.
template <int D, bool HALVES>
__global__ void __launch_bounds__(kThreads) rope_backward_kernel(const RopeLaunch p, const int splits) {
  constexpr int LANES = D / 8, TOKENS = kThreads / LANES;
  typedef Piece<HALVES> P;
  const int tensor = blockIdx.y;
  const RopeTensor& t = p.t[tensor];
  const int c = threadIdx.x % LANES;
  const bool normed = p.norm != SVD_NORM_NONE;
  const f32x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
  const f32x8 w = t.weight ? P::load(t.weight, c, D) : zero + 1.f;
  f32x8 dw = zero, db = zero;
  const int blocks = rope_blocks(p.L, D);
  const int64_t units = (int64_t)blocks * p.B * splits;
  for (int64_t i = blockIdx.x; i < units; i += gridDim.x) {
    const RopeUnit unit = rope_unit(i, blocks, splits);
    const int b = unit.b, l = unit.block * TOKENS + threadIdx.x / LANES;
    const HeadRange heads = heads_of_part(t.H, splits, unit.part);
    const int h0 = heads.first, h1 = heads.last;
    if (l >= p.L || h0 >= h1) continue;
    const __bf16* x = normed ? t.x + (int64_t)b * t.x_b + (int64_t)l * t.x_l : nullptr;
    const __bf16* g = t.dout + (int64_t)b * t.d_b + (int64_t)l * t.d_l;
    __bf16* o = t.out + (int64_t)b * t.o_b + (int64_t)l * t.o_l;
    bf16x8 d_next = P::raw(g + (int64_t)h0 * t.d_h, c, D), x_next = {};
    if (normed) x_next = P::raw(x + (int64_t)h0 * t.x_h, c, D);
    const Angles a = angles_of(p, l, c);
    for (int h = h0; h < h1; ++h) {
      f32x8 d = turn<HALVES>(__builtin_convertvector(d_next, f32x8), a, -1.f), n = __builtin_convertvector(x_next, f32x8);
      if (h + 1 < h1) {
        d_next = P::raw(g + (int64_t)(h + 1) * t.d_h, c, D);
        if (normed) x_next = P::raw(x + (int64_t)(h + 1) * t.x_h, c, D);
      }
      if (normed) {
        const float r = normalise<LANES>(n, p.norm, p.eps);
        dw += d * n;
        db += d;
        d *= w;
        constexpr float inv = 1.f / D;
        const float c1 = lane_sum<LANES>(sum8(d * n)) * inv;
        const float c0 = p.norm == SVD_NORM_LAYER ? lane_sum<LANES>(sum8(d)) * inv : 0.f;
        d = (d - c0 - n * c1) * r;
      }
      P::store(o + (int64_t)h * t.o_h, c, D, d);
    }
  }
  if (!p.partial) return;
  __shared__ __attribute__((aligned(16))) float sums[TOKENS][2][D];
  P::store(sums[threadIdx.x / LANES][0], c, D, dw);
  P::store(sums[threadIdx.x / LANES][1], c, D, db);
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
    float s = 0.f;
    for (int k = 0; k < TOKENS; ++k) s += sums[k][i / D][i % D];
    p.partial[(((int64_t)tensor * gridDim.x + blockIdx.x) * 2 + i / D) * D + i % D] = s;
  }
}

// Work-group (32 channels, weight or bias of a tensor): the sum of the parts.
__global__ void __launch_bounds__(1024) rope_weight_kernel(const RopeLaunch p, const int groups) {
  __shared__ double slots[1][32][32];
  const int tensor = blockIdx.y >> 1, k = blockIdx.y & 1, c = blockIdx.x * 32 + threadIdx.x % 32;
  float* out = k == 0 ? p.t[tensor].dweight : p.t[tensor].dbias;
  if (!out) return;
  const double s = column_sums<32, 1>(p.partial + ((int64_t)tensor * groups * 2 + k) * p.D + c, 0, (int64_t)2 * p.D, groups, true, slots);
  if (threadIdx.x < 32) out[c] = (float)s;
}

struct TableArgs {
  svd_rope_desc r;
  double base, start[3], step[3];
};
__global__ void __launch_bounds__(kThreads) rope_table_kernel(const TableArgs a, float2* __restrict__ table, const int n) {
  const int i = blockIdx.x * kThreads + threadIdx.x;
  if (i >= n) return;
  const int len[3] = {a.r.frames * a.r.pairs_t, a.r.height * a.r.pairs_h, a.r.width * a.r.pairs_w};
  const int axis = i < len[0] ? 0 : i < len[0] + len[1] ? 1 : 2;
  const int k = i - (axis > 0 ? len[0] : 0) - (axis > 1 ? len[1] : 0);
  const int pairs = axis == 0 ? a.r.pairs_t : axis == 1 ? a.r.pairs_h : a.r.pairs_w;
  const double angle = (a.start[axis] + (double)(k / pairs) * a.step[axis]) * pow(a.base, -(double)(k % pairs) / (double)pairs);
  table[i] = make_float2((float)cos(angle), (float)sin(angle));
}

int most_heads(const RopeLaunch& p) { return p.n == 2 && p.t[1].H > p.t[0].H ? p.t[1].H : p.t[0].H; }

}  // namespace

hipError_t launch_rope_table(const svd_rope_desc& r, double base, const double start[3], const double step[3], float* table,
                             hipStream_t stream) {
  TableArgs a{r, base, {start[0], start[1], start[2]}, {step[0], step[1], step[2]}};
  const int n = r.frames * r.pairs_t + r.height * r.pairs_h + r.width * r.pairs_w;
  hipLaunchKernelGGL(rope_table_kernel, dim3((unsigned)(((int64_t)n + kThreads - 1) / kThreads)), dim3(kThreads), 0, stream, a,
                     reinterpret_cast<float2*>(table), n);
  return hipGetLastError();
}

hipError_t launch_rope_forward(const RopeLaunch& p, hipStream_t stream) {
  const int splits = rope_forward_splits(p.L, p.B, p.D, p.n, most_heads(p));
  const dim3 grid(rope_blocks(p.L, p.D), p.B, (unsigned)(p.n * splits));
  const bool halves = p.r.pairing == SVD_ROPE_HALVES;
#define SVD_ROPE_LAUNCH(D, H) hipLaunchKernelGGL((rope_forward_kernel<D, H>), grid, dim3(kThreads), 0, stream, p, splits)
  if (p.D == 64) {
    if (halves) SVD_ROPE_LAUNCH(64, true);
    else SVD_ROPE_LAUNCH(64, false);
  } else {
    if (halves) SVD_ROPE_LAUNCH(128, true);
    else SVD_ROPE_LAUNCH(128, false);
  }
#undef SVD_ROPE_LAUNCH
  return hipGetLastError();
}

hipError_t launch_rope_backward(const RopeLaunch& p, hipStream_t stream) {
  const RopeWalk walk = rope_walk(p.L, p.B, p.D, most_heads(p));
  const dim3 grid(walk.groups, p.n);
  const bool halves = p.r.pairing == SVD_ROPE_HALVES;
#define SVD_ROPE_LAUNCH(D, H) hipLaunchKernelGGL((rope_backward_kernel<D, H>), grid, dim3(kThreads), 0, stream, p, walk.splits)
  if (p.D == 64) {
    if (halves) SVD_ROPE_LAUNCH(64, true);
    else SVD_ROPE_LAUNCH(64, false);
  } else {
    if (halves) SVD_ROPE_LAUNCH(128, true);
    else SVD_ROPE_LAUNCH(128, false);
  }
#undef SVD_ROPE_LAUNCH
  if (hipError_t e = hipGetLastError(); e != hipSuccess || !p.partial) return e;
  hipLaunchKernelGGL(rope_weight_kernel, dim3(p.D / 32, 2 * p.n), dim3(1024), 0, stream, p, walk.groups);
  return hipGetLastError();
}

}  // namespace svd
