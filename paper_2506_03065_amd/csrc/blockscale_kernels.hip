// gfx950 kernels of matrices held in E4M3 with a power-of-two scale for each row and block of 128 columns: the
// quantisation of rows and of columns, and the product out[m][n] = sum_k a[m][k] b[n][k] + bias[n].
//
// The product runs on v_mfma_scale_f32_32x32x64_f8f6f4, which multiplies every 32 elements of an operand's row by a scale byte
// that the lane holds: the scales cost no vector instruction and the accumulators stay with the matrix pipe.  (The 16x16x128
// form takes the same bytes per product from LDS, but its results are not tied to its addends: the compiler moves
// accumulators about and spills; 256 x 256 tiles, 8,192^3: 527 us against 445.)  Inside an instruction products that lie more than 13 bits below the largest
// beside them are dropped (a property of all FP8 matrix instructions of this chip: 1.5e-5 of a result over normal data,
// whatever K); across instructions the sum is fp32.
//
// Roles: b (columns n of the result) is the instruction's first operand, a (rows m) its second, so that a lane holds, for
// one m, consecutive n.  Row j of operand tile t of a wave is row j * TILES + t of the wave's part of the matrix: a lane's
// scale bytes of all its tiles are then consecutive (one load, the byte chosen by the instruction), and so are its
// results of all tiles (16 bytes to a store).
#include <hip/hip_runtime.h>

#include <type_traits>
#include <utility>

#include "layer_index.h"
#include "layer_ops.h"
#include "wave_ops.h"

namespace svd {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void* lds_ptr;

// ---- quantisation ----

// Work-group: 32 rows by BLOCKS blocks of 128 columns.  The scale bytes of a block's 32 rows go out together.
template <typename T, int BLOCKS>
__global__ void __launch_bounds__(256) quantise_rows_kernel(const QuantLaunch p) {
  constexpr int ROWS = quant_rows_at_once(BLOCKS);
  __shared__ __attribute__((aligned(16))) uint8_t bytes[BLOCKS][kQuantRows];
  const QuantAt at = quant_at(threadIdx.x, BLOCKS);
  const int r0 = blockIdx.x * kQuantRows, c = (blockIdx.y * BLOCKS + at.block) * 128 + at.column;
  const int c16 = (p.C + 15) / 16 * 16;
#pragma unroll
  for (int i = 0; i < 8 / ROWS; ++i) {
    const int k = at.row + i * ROWS, row = r0 + k;
    const T* src = static_cast<const T*>(p.src) + (int64_t)row * p.src_stride + c;
    f32x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
    if (row < p.R && c + 8 <= p.C) {
      Raw8<T> raw;
      raw.load(src);
      v = raw.get();
    } else if (row < p.R) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (c + j < p.C) v[j] = (float)src[j];
    }
    int top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, magnitude(v[j]));
    const int byte = scale_byte(max16(top));
    const float f = scale_inverse(byte);
    if (row < p.R && c < c16) {
      const u32x2 w = {(unsigned)pack_e4m3(v[0] * f, v[1] * f, v[2] * f, v[3] * f),
                       (unsigned)pack_e4m3(v[4] * f, v[5] * f, v[6] * f, v[7] * f)};
      *reinterpret_cast<u32x2*>(p.dst + (int64_t)row * p.dst_stride + c) = w;
    }
    if ((threadIdx.x & 15) == 0) bytes[at.block][k] = (uint8_t)byte;
  }
  __syncthreads();
  const int b = threadIdx.x / kQuantRows, k = threadIdx.x % kQuantRows;
  if (b < BLOCKS && (blockIdx.y * BLOCKS + b) * 128 < p.C && r0 + k < p.R)
    p.scales[(int64_t)(blockIdx.y * BLOCKS + b) * p.scale_stride + r0 + k] = bytes[b][k];
}

// Work-group: 128 rows (one block) by 64 columns of src, turned round in LDS; a thread then holds 32 rows of a column.  Neighbouring
// work-groups read neighbouring columns of the same rows (75,600 x 5,120 bf16: 272 us, 4.3 TB/s; the other way round 333).
template <typename T>
__global__ void __launch_bounds__(256) quantise_columns_kernel(const QuantLaunch p) {
  constexpr int PAD = 66;
  __shared__ float tile[128 * PAD];
  const int r0 = blockIdx.y * 128, c0 = blockIdx.x * 64;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const QuantPlace at = quant_read_at(threadIdx.x, i);
    const int k = at.row, c = at.column, row = r0 + k;
    const T* src = static_cast<const T*>(p.src) + (int64_t)row * p.src_stride + c0 + c;
    f32x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
    if (row < p.R && c0 + c + 8 <= p.C) {
      Raw8<T> raw;
      raw.load(src);
      v = raw.get();
    } else if (row < p.R) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (c0 + c + j < p.C) v[j] = (float)src[j];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) tile[k * PAD + c + j] = v[j];
  }
  __syncthreads();
  const QuantPlace at = quant_write_at(threadIdx.x);
  const int col = at.column, part = threadIdx.x & 3;
  float v[32];
  int top = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    v[i] = tile[(at.row + i) * PAD + col];
    top = max(top, magnitude(v[i]));
  }
  top = max(top, dpp<kXor1>(top));
  top = max(top, dpp<kXor2>(top));
  const int byte = scale_byte(top);
  const float f = scale_inverse(byte);
  if (c0 + col >= p.C) return;
  const int r16 = (p.R + 15) / 16 * 16;
  uint8_t* dst = p.dst + (int64_t)(c0 + col) * p.dst_stride + r0 + at.row;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      w[j] = (unsigned)pack_e4m3(v[16 * q + 4 * j] * f, v[16 * q + 4 * j + 1] * f, v[16 * q + 4 * j + 2] * f, v[16 * q + 4 * j + 3] * f);
    if (r0 + at.row + 16 * q < r16) *reinterpret_cast<u32x4*>(dst + 16 * q) = w;
  }
  if (part == 0) p.scales[(int64_t)blockIdx.y * p.scale_stride + c0 + col] = (uint8_t)byte;
}

// ---- product ----

template <class F, int... I>
__device__ __forceinline__ void unrolled(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void unrolled(F&& f) {
  unrolled(f, std::make_integer_sequence<int, N>{});
}

// What a buffer load reads depends on the range of its resource and the lane's own offset alone: the offset that the lanes share is
// never past the range, and a step behind the last has a range of 0.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t resource(const uint8_t* base, unsigned bytes) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (int)bytes, 0x00020000);
}
// Bytes of rows row0 .. of a matrix, at most `most` of them: rows past the last one lie past the range and arrive as zeros.
__device__ __forceinline__ unsigned rows_range(int row0, int rows, int64_t stride, int most, int bytes) {
  return (unsigned)(min(rows - row0, most) - 1) * (unsigned)stride + bytes;
}
// Requests 16 bytes a lane from a range of memory into LDS.
__device__ __forceinline__ void request16(const uint8_t* base, unsigned range, unsigned at, int offset, uint8_t* lds) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(resource(base, range), (lds_ptr)lds, 16, (int)at, offset, 0, 0);
}
// The scales of `rows` rows: up to the next multiple of 16 in the last block (base and stride are multiples of 16), and no further: a
// part of a larger matrix may end where its memory does.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t scales_resource(const uint8_t* base, int blocks, int64_t stride, int rows) {
  return resource(base, (unsigned)(blocks - 1) * (unsigned)stride + (rows + 15) / 16 * 16);
}
// The scale bytes of a lane's TILES consecutive rows; at: of the first, in the block.
template <int TILES>
__device__ __forceinline__ void load_scales(const __amdgpu_buffer_rsrc_t r, unsigned at, int (&s)[(TILES + 3) / 4]) {
  static_assert(TILES == 2 || TILES % 4 == 0, "");
  if constexpr (TILES == 2) {
    s[0] = (int)__builtin_amdgcn_raw_buffer_load_b16(r, (int)at, 0, 0);
  } else {
#pragma unroll
    for (int i = 0; i < TILES / 4; ++i) s[i] = (int)__builtin_amdgcn_raw_buffer_load_b32(r, (int)(at + 4 * i), 0, 0);
  }
}

// Every wave's requests into LDS have landed, and its reads of LDS are over.  (The barrier alone waits for no request: the
// compiler only holds a wave's own reads back until its own requests are there.)
__device__ __forceinline__ void landed_barrier() {
  __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
  __syncthreads();
}

// The same for LDS that a wave has to itself.
__device__ __forceinline__ void landed_wave() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0) lgkmcnt(0)
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// WM x WN waves of MT x NT tiles of 32 x 32.  KG > 1: KG single waves that each take a part of K for the same tile, with LDS of
// their own; their sums are added in LDS, in order.
template <int WM, int WN, int MT, int NT, int KG>
__device__ __forceinline__ void matmul_tile(const MatmulLaunch& p, const int m0, const int n0) {
  constexpr int BM = WM * MT * 32, BN = WN * NT * 32, WAVES = WM * WN;
  static_assert(KG == 1 || (KG == 4 && WAVES == 1 && MT == 2 && NT == 2), "");
  // one object per buffer: a request into one then does not hold up reads of the other
  __shared__ __attribute__((aligned(1024))) uint8_t sA0[KG * BM * 128], sA1[KG * BM * 128], sB0[KG * BN * 128], sB1[KG * BN * 128];
  const int lane = threadIdx.x & 63, j = lane & 31, half = lane >> 5;
  const int wave = KG > 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), kg = KG > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
  const int wm = wave % WM, wn = wave / WM;
  const svd_blockscale_desc& d = p.d;
  const int k16 = (d.K + 15) / 16 * 16, blocks = (d.K + 127) / 128;
  const int whole = k16 / 128, first = whole * kg / KG, steps = whole * (kg + 1) / KG;   // whole steps, and this wave's

  const uint8_t *const base_a = p.a + (int64_t)m0 * d.a_stride, *const base_b = p.b + (int64_t)n0 * d.b_stride;
  const unsigned range_a = rows_range(m0, d.M, d.a_stride, BM, k16), range_b = rows_range(n0, d.N, d.b_stride, BN, k16);
  const __amdgpu_buffer_rsrc_t rsa = scales_resource(p.a_scales, blocks, d.a_scale_stride, d.M), rsb = scales_resource(p.b_scales, blocks, d.b_scale_stride, d.N);

  // A wave fills slabs of 1 KB (8 rows), 16 bytes a lane.  Of a block that ends early, the bytes behind a row's end (the
  // next row's) start past every range and arrive as zeros.
  constexpr int LA = BM / 8 / WAVES, LB = BN / 8 / WAVES;
  unsigned ga[LA], gb[LB];
  auto places = [&](int left) {
#pragma unroll
    for (int u = 0; u < LA; ++u) ga[u] = slab_place(wave * LA + u, lane, MT, (unsigned)d.a_stride, left);
#pragma unroll
    for (int u = 0; u < LB; ++u) gb[u] = slab_place(wave * LB + u, lane, NT, (unsigned)d.b_stride, left);
  };
  struct Source {
    unsigned a, b;   // ranges
    int offset;      // of the step in a row's bytes
  };
  auto source_of = [&](int step, int end) {   // behind the last: nothing is read
    const bool on = step < end;
    return Source{on ? range_a : 0, on ? range_b : 0, on ? step * 128 : 0};
  };
  auto request_one = [&](auto buf_tag, auto u_tag, const Source& s) {   // slab u of a's, then of b's
    constexpr int u = decltype(u_tag)::value;
    if constexpr (u < LA)
      request16(base_a, s.a, ga[u], s.offset, (decltype(buf_tag)::value ? sA1 : sA0) + kg * BM * 128 + (wave * LA + u) * 1024);
    else
      request16(base_b, s.b, gb[u - LA], s.offset, (decltype(buf_tag)::value ? sB1 : sB0) + kg * BN * 128 + (wave * LB + u - LA) * 1024);
  };
  auto request = [&](auto buf_tag, const Source& s) {
    unrolled<LA + LB>([&](auto u_tag) { request_one(buf_tag, u_tag, s); });
  };

  f32x16 acc[MT][NT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[m][n][i] = 0.f;

  const int m_lane = m0 + (wm * 32 + j) * MT, n_lane = n0 + (wn * 32 + j) * NT;   // first of the lane's rows
  // byte offsets of a fragment's two chunks, for even and odd tiles and the two halves of a step; the rest is an immediate
  int fa[2][2][2], fb[2][2][2];
#pragma unroll
  for (int odd = 0; odd < 2; ++odd)
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int at = ((odd * 8 + k * 4 + half * 2 + c) ^ (j & 15)) << 4;
        fa[odd][k][c] = kg * BM * 128 + (wm * 32 + j) * MT * 128 + at;
        fb[odd][k][c] = kg * BN * 128 + (wn * 32 + j) * NT * 128 + at;
      }
  auto fragment = [&](const uint8_t* s, const int (&at)[2][2][2], int tile, int k) {
    const i32x4 lo = *reinterpret_cast<const i32x4*>(s + (tile >> 1) * 256 + at[tile & 1][k][0]);
    const i32x4 hi = *reinterpret_cast<const i32x4*>(s + (tile >> 1) * 256 + at[tile & 1][k][1]);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  struct Scales {
    int m[(MT + 3) / 4], n[(NT + 3) / 4];
  };
  auto scales_of = [&](int step) {
    Scales s;
    load_scales<MT>(rsa, m_lane + step * (unsigned)d.a_scale_stride, s.m);
    load_scales<NT>(rsb, n_lane + step * (unsigned)d.b_scale_stride, s.n);
    return s;
  };
  typedef std::integral_constant<int, 0> Zero;
  typedef std::integral_constant<int, 1> One;

  i32x8 fn[2][NT], fm[3];   // b's fragments of either half of a step, and three of a's
  Scales scales[2];         // of the step in either buffer
  auto product = [&](auto buf_tag, auto m_tag, auto n_tag, auto k_tag, const i32x8& f) {
    const Scales& s = scales[decltype(buf_tag)::value];
    constexpr int m = decltype(m_tag)::value, n = decltype(n_tag)::value, k = decltype(k_tag)::value;
    acc[m][n] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fn[k][n], f, acc[m][n], 0, 0, n % 4, s.n[n / 4], m % 4, s.m[m / 4]);
  };
  auto landed = [&] {
    if constexpr (KG > 1) landed_wave();
    else landed_barrier();
  };
  places(128);
  if (steps > first) {
    request(Zero{}, source_of(first, steps));
    scales[0] = scales_of(first);
    landed();
    request(One{}, source_of(first + 1, steps));
    scales[1] = scales_of(first + 1);
#pragma unroll
    for (int n = 0; n < NT; ++n) fn[0][n] = fragment(sB0, fb, n, 0);
    fm[0] = fragment(sA0, fa, 0, 0);
  }

  // One step of 128 in units of one tile of a's rows and one half of the step; a unit's fragment is read under the products
  // of the one before.  Ahead of the last two units the step's LDS reads are over: one barrier, after which the buffer takes the
  // step after the next and the next step's first fragments are read under the last products.
  constexpr int UNITS = 2 * MT;
  auto stage = [&](auto buf_tag, const int step) {
    constexpr int buf = decltype(buf_tag)::value;
    const uint8_t *a = buf ? sA1 : sA0, *b = buf ? sB1 : sB0, *a_next = buf ? sA0 : sA1, *b_next = buf ? sB0 : sB1;
    const Source source = source_of(step + 2, steps);
    auto unit = [&](auto u_tag) {
      constexpr int u = decltype(u_tag)::value;
      unrolled<NT>([&](auto n_tag) {
        product(buf_tag, std::integral_constant<int, u % MT>{}, n_tag, std::integral_constant<int, u / MT>{}, fm[u % 3]);
      });
      __builtin_amdgcn_sched_barrier(0);
    };
    unrolled<UNITS - 2>([&](auto u_tag) {
      constexpr int u = decltype(u_tag)::value;
      fm[(u + 1) % 3] = fragment(a, fa, (u + 1) % MT, (u + 1) / MT);
      if constexpr (u < NT) fn[1][u] = fragment(b, fb, u, 1);
      if constexpr (u == UNITS - 3) fm[(u + 2) % 3] = fragment(a, fa, (u + 2) % MT, (u + 2) / MT);
      unit(u_tag);
    });
    landed();
    // Tiles of 2 request the scales first, and a copy then waits for these alone (24,000 x 1,000 x 4,096: 89.8 us; behind the last
    // product, where the registers are free and no copy is needed, 91.9; 2 x 30,720 x 5,120: 33 and 38).  Tiles of 4 do the latter.
    Scales after;
    if constexpr (MT <= 2) {
      after = scales_of(step + 2);
      __builtin_amdgcn_sched_barrier(0);
    }
    constexpr int all = LA + LB, part = (all + 2 * NT - 1) / (2 * NT);
    if constexpr (MT <= 2) {   // all requests first: the compute unit's other work-group fills the gap
      request(buf_tag, source);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int n = 0; n < NT; ++n) fn[0][n] = fragment(b_next, fb, n, 0);
      fm[UNITS % 3] = fragment(a_next, fa, 0, 0);
      unit(std::integral_constant<int, UNITS - 2>{});
      unit(std::integral_constant<int, UNITS - 1>{});
    } else {   // the requests among the products, which go on at once (75,600 x 5,120 x 5,120: 1,660 -> 1,585 us; 128 x 128 tiles lose 3 %)
      unrolled<2 * NT>([&](auto i_tag) {
        constexpr int i = decltype(i_tag)::value;
        product(buf_tag, std::integral_constant<int, (UNITS - 2 + i / NT) % MT>{}, std::integral_constant<int, i % NT>{}, One{}, fm[(UNITS - 2 + i / NT) % 3]);
        if constexpr (i == 0) {
#pragma unroll
          for (int n = 0; n < NT; ++n) fn[0][n] = fragment(b_next, fb, n, 0);
          fm[UNITS % 3] = fragment(a_next, fa, 0, 0);
        }
        unrolled<part>([&](auto q_tag) {
          constexpr int q = i * part + decltype(q_tag)::value;
          if constexpr (q < all) request_one(buf_tag, std::integral_constant<int, q>{}, source);
        });
        __builtin_amdgcn_sched_barrier(0);
      });
    }
    fm[0] = fm[UNITS % 3];
    if constexpr (MT <= 2) scales[buf] = after;
    else scales[buf] = scales_of(step + 2);
  };
  static_assert(NT <= MT, "the second half's fragments of b are read in the first half");
  int step = first;
  for (; step + 1 < steps; step += 2) {
    stage(Zero{}, step);
    stage(One{}, step + 1);
  }
  if (step < steps) stage(Zero{}, step);
  if (k16 % 128 && kg == KG - 1) {   // a last block that ends early, on its own
    landed();
    places(k16 % 128);
    request(Zero{}, source_of(whole, whole + 1));
    scales[0] = scales_of(whole);
    landed();
    unrolled<2>([&](auto k_tag) {
      constexpr int k = decltype(k_tag)::value;
#pragma unroll
      for (int n = 0; n < NT; ++n) fn[k][n] = fragment(sB0, fb, n, k);
      unrolled<MT>([&](auto m_tag) {
        constexpr int m = decltype(m_tag)::value;
        const i32x8 f = fragment(sA0, fa, m, k);
        unrolled<NT>([&](auto n_tag) { product(Zero{}, m_tag, n_tag, k_tag, f); });
      });
    });
  }
  // no request may be on its way when the work-group ends: its LDS is the next one's
  landed_barrier();

  // result i of tile n: column (wn * 32 + 8 * (i / 4) + 4 * half + i % 4) * NT + n
  const bool wide = ((reinterpret_cast<uintptr_t>(p.out) | (uintptr_t)(d.out_stride * 2)) & 15) == 0;
  auto store = [&](const int row, const int col, const bf16x8 v) {   // 8 columns
    __bf16* o = p.out + (int64_t)row * d.out_stride + col;
    if (wide && col + 8 <= d.N) {
      *reinterpret_cast<bf16x8*>(o) = v;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (col + i < d.N) o[i] = v[i];
    }
  };
  auto bias_of = [&](const int col) {
    f32x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
    if (p.bias)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = col + i < d.N ? p.bias[col + i] : 0.f;
    return v;
  };
  static_assert(NT == 2, "a wave's rows of results: 128 bytes");
  if constexpr (KG > 1) {
    // every part's tile (m, n) in the memory of one buffer, [part][16][64 lanes]; wave kg then adds half of a row of tiles
    float* const sums[4] = {reinterpret_cast<float*>(sA0), reinterpret_cast<float*>(sA1), reinterpret_cast<float*>(sB0), reinterpret_cast<float*>(sB1)};
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) sums[t][(kg * 16 + i) * 64 + lane] = acc[t >> 1][t & 1][i];
    __syncthreads();
    const int m = kg >> 1, row = m_lane + m;
    const float* const of[2] = {m ? sums[2] : sums[0], m ? sums[3] : sums[1]};
    if (row >= d.M) return;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int g = 2 * (kg & 1) + h, col = n0 + (8 * g + 4 * half) * NT;
      f32x8 v = bias_of(col);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < KG; ++w) s += of[i % 2][(w * 16 + 4 * g + i / 2) * 64 + lane];
        v[i] += s;
      }
      store(row, col, __builtin_convertvector(v, bf16x8));
    }
  } else {
    // A wave's results through the LDS of a buffer (no longer in use), so that a store covers whole rows of 128 bytes, not 32 bytes
    // in each of 32 rows (75,600 x 5,120 x 5,120: 1,634 -> 1,555 us; 9,107 x 6,144 x 2,048: 117.7 -> 113.9).  The chunks lie in
    // the order of the operand tiles (swizzle).
    constexpr int ROWS = MT * 32;
    uint8_t* const mine = (wave >> 1 == 0 ? sA0 : wave >> 1 == 1 ? sA1 : wave >> 1 == 2 ? sB0 : sB1) + (wave & 1) * ROWS * 128;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x8 bias = bias_of(n0 + (wn * 32 + 8 * g + 4 * half) * NT);
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        f32x8 v = bias;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += acc[m][i % 2][4 * g + i / 2];
        *reinterpret_cast<bf16x8*>(mine + tile_byte(j * MT + m, 2 * g + half, MT)) = __builtin_convertvector(v, bf16x8);
      }
    }
    landed_wave();
    const int row0 = m0 + wm * ROWS, col = n0 + wn * 64 + (lane & 7) * 8;
#pragma unroll
    for (int i = 0; i < ROWS / 8; ++i) {
      const int r = i * 8 + (lane >> 3);
      const bf16x8 v = *reinterpret_cast<const bf16x8*>(mine + tile_byte(r, lane & 7, MT));
      if (row0 + r < d.M && col < d.N) store(row0 + r, col, v);
    }
  }
}

template <int WM, int WN, int MT, int NT, int KG>
__global__ void __launch_bounds__(WM * WN * KG * 64) blockscale_matmul_kernel(const MatmulLaunch p, const int m_tiles, const int n_tiles) {
  const TileAt tile = tile_at(blockIdx.x, m_tiles, n_tiles);
  matmul_tile<WM, WN, MT, NT, KG>(p, tile.m * (WM * MT * 32), tile.n * (WN * NT * 32));
}

// The tiles of 256 x 256 behind the first `whole`, in quarters.
__global__ void __launch_bounds__(256) blockscale_quarters_kernel(const MatmulLaunch p, const int m_tiles, const int n_tiles, const int whole) {
  const QuarterAt q = quarter_at(blockIdx.x, whole);
  if (q.tile >= m_tiles * n_tiles) return;
  const TileAt tile = tile_at(q.tile, m_tiles, n_tiles);
  const int m0 = tile.m * 256 + (q.quarter & 1) * 128, n0 = tile.n * 256 + (q.quarter >> 1) * 128;
  if (m0 < p.d.M && n0 < p.d.N) matmul_tile<2, 2, 2, 2, 1>(p, m0, n0);
}

template <int WM, int WN, int MT, int NT, int KG>
void launch_tiles(const MatmulLaunch& p, int tiles, hipStream_t stream) {
  const int m_tiles = (p.d.M + WM * MT * 32 - 1) / (WM * MT * 32), n_tiles = (p.d.N + WN * NT * 32 - 1) / (WN * NT * 32);
  hipLaunchKernelGGL((blockscale_matmul_kernel<WM, WN, MT, NT, KG>), dim3(tiles ? tiles : m_tiles * n_tiles), dim3(WM * WN * KG * 64), 0, stream, p,
                     m_tiles, n_tiles);
}

}  // namespace

hipError_t launch_quantise_rows(const QuantLaunch& p, hipStream_t stream) {
  const int blocks = quant_blocks(p.C);
  const dim3 grid((p.R + kQuantRows - 1) / kQuantRows, (p.C + blocks * 128 - 1) / (blocks * 128));
  auto launch = [&](auto type) {
    using T = decltype(type);
    const auto kernel = blocks == 1 ? quantise_rows_kernel<T, 1> : blocks == 2 ? quantise_rows_kernel<T, 2> : quantise_rows_kernel<T, 4>;
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, p);
  };
  if (p.src_type == SVD_F32) launch(float{});
  else launch(__bf16{});
  return hipGetLastError();
}

hipError_t launch_quantise_columns(const QuantLaunch& p, hipStream_t stream) {
  const dim3 grid((p.C + 63) / 64, (p.R + 127) / 128);
  if (p.src_type == SVD_F32) hipLaunchKernelGGL(quantise_columns_kernel<float>, grid, dim3(256), 0, stream, p);
  else hipLaunchKernelGGL(quantise_columns_kernel<__bf16>, grid, dim3(256), 0, stream, p);
  return hipGetLastError();
}

// What bounds large products is power and the end of a tile: 75,600 x 5,120 x 5,120 over and over draws the card's 1,400 W at 1.70 to
// 1.82 of its 2.4 GHz (1,618 and 1,547 us by card), the matrix pipe busy 68 % of the cycles, no LDS bank conflicts; all tiles of a round end together, and their 128 KB of results each take 4 us to leave
// (6 % of 5,120 deep products).  Resident work-groups that request the next tile ahead of their stores are 5 % slower; starting
// the units apart in time gains 2 to 4 % where the last round is nearly empty and costs as much where it is full.  Two groups of
// four waves on halves of K: 6 to 20 % for products of one round of small tiles, but the same code without them loses 13 %.
hipError_t launch_blockscale_matmul(const MatmulLaunch& p, hipStream_t stream) {
  const MatmulPlan plan = matmul_plan(p.d.M, p.d.N, p.d.K);
  if (plan.form == FORM_64) {
    launch_tiles<1, 1, 2, 2, 4>(p, 0, stream);
  } else if (plan.form == FORM_128) {
    launch_tiles<2, 2, 2, 2, 1>(p, 0, stream);
  } else {
    launch_tiles<2, 4, 4, 2, 1>(p, plan.whole, stream);
    const int m_tiles = (p.d.M + 255) / 256, n_tiles = (p.d.N + 255) / 256, rest = m_tiles * n_tiles - plan.whole;
    if (rest > 0) {
      if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
      hipLaunchKernelGGL(blockscale_quarters_kernel, dim3((unsigned)quarter_blocks(rest)), dim3(256), 0, stream, p, m_tiles, n_tiles, plan.whole);
    }
  }
  return hipGetLastError();
}

}  // namespace svd
