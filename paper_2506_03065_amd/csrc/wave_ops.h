// Reductions over the lanes of a wave without LDS, and the 16-byte loads and stores of rows.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "layer_index.h"

namespace svd {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

template <int CTRL>
__device__ __forceinline__ int dpp(int x) {
  return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xf, 0xf, true);
}
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __builtin_bit_cast(float, dpp<CTRL>(__builtin_bit_cast(int, x)));
}
constexpr int kXor1 = 0xb1, kXor2 = 0x4e, kHalfMirror = 0x141, kMirror = 0x140;   // within 2, 4, 8 and 16 lanes

// Sum over groups of LANES lanes, the same bits in each of them (every step adds the same two numbers on both sides).
template <int LANES>
__device__ __forceinline__ float lane_sum(float x) {
  x += dpp<kXor1>(x);
  x += dpp<kXor2>(x);
  x += dpp<kHalfMirror>(x);
  if (LANES >= 16) x += dpp<kMirror>(x);
  if (LANES >= 32) {
    const unsigned a = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane16_swap(a, a, false, false);
    const unsigned r0 = r[0], r1 = r[1];
    x = __builtin_bit_cast(float, r0) + __builtin_bit_cast(float, r1);
  }
  if (LANES >= 64) {
    const unsigned a = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane32_swap(a, a, false, false);
    const unsigned r0 = r[0], r1 = r[1];
    x = __builtin_bit_cast(float, r0) + __builtin_bit_cast(float, r1);
  }
  return x;
}

// Maximum of non-negative integers over groups of 16 lanes.
__device__ __forceinline__ int max16(int x) {
  x = max(x, dpp<kXor1>(x));
  x = max(x, dpp<kXor2>(x));
  x = max(x, dpp<kHalfMirror>(x));
  return max(x, dpp<kMirror>(x));
}

// Eight elements as they lie in memory, and as floats.
template <typename T>
struct Raw8;
template <>
struct Raw8<__bf16> {
  bf16x8 v;
  __device__ __forceinline__ void load(const __bf16* p) { v = *reinterpret_cast<const bf16x8*>(p); }
  __device__ __forceinline__ f32x8 get() const { return __builtin_convertvector(v, f32x8); }
};
template <>
struct Raw8<float> {
  f32x8 v;
  __device__ __forceinline__ void load(const float* p) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
    v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  __device__ __forceinline__ f32x8 get() const { return v; }
};

__device__ __forceinline__ f32x8 load8(const float* p) {
  Raw8<float> r;
  r.load(p);
  return r.get();
}
__device__ __forceinline__ void store8(__bf16* p, const f32x8 v) {
  *reinterpret_cast<bf16x8*>(p) = __builtin_convertvector(v, bf16x8);
}
__device__ __forceinline__ void store8(float* p, const f32x8 v) {
  *reinterpret_cast<f32x4*>(p) = __builtin_shufflevector(v, v, 0, 1, 2, 3);
  *reinterpret_cast<f32x4*>(p + 4) = __builtin_shufflevector(v, v, 4, 5, 6, 7);
}

// NV sums of n numbers `stride` apart, the k-th from in + k * next, by the LANES threads of a column (thread = lane * 32 + column), in
// 64 bits and a fixed order; lane k of a column returns the k-th.  Every thread of the work-group calls it; those without a column
// (`on` false) add nothing.
template <int LANES, int NV>
__device__ __forceinline__ double column_sums(const float* in, int64_t next, int64_t stride, int n, bool on, double (*slots)[LANES][32]) {
  constexpr int AHEAD = kSumAhead;
  const int lane = threadIdx.x / 32, column = threadIdx.x % 32;
  double s[NV] = {};
  if (on)
    for (int i = lane; i < n; i += AHEAD * LANES) {   // all of a step's loads at once; behind the last number, it again, not added
      float v[AHEAD][NV];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
#pragma unroll
        for (int k = 0; k < NV; ++k) v[u][k] = in[(int64_t)min(sum_at(i, u, LANES), n - 1) * stride + k * next];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
#pragma unroll
        for (int k = 0; k < NV; ++k) s[k] += sum_at(i, u, LANES) < n ? (double)v[u][k] : 0.0;
    }
#pragma unroll
  for (int k = 0; k < NV; ++k) slots[k][lane][column] = s[k];
  __syncthreads();
  double sum = 0.0;
  if (lane < NV)
#pragma unroll
    for (int l = 0; l < LANES; ++l) sum += slots[lane][l][column];
  return sum;
}

// ---- E4M3 with a power-of-two scale for each block of 128 ----

// Scale byte e + 127 of a block from the bits of its largest magnitude: the least e >= -127 with max <= 448 * 2^e.
// 448 = 1.75 * 2^8, so e is the exponent of the maximum less 8, one more where its mantissa is over 1.75.  An infinity
// or NaN (exponent 255; its bits are larger than a finite number's, so the integer maximum finds it) gives 255.
__device__ __forceinline__ int scale_byte(int max_bits) {
  const int e = max_bits >> 23;
  return e == 255 ? 255 : max(e - 8 + ((max_bits & 0x7fffff) > 0x600000 ? 1 : 0), 0);
}
// 2^-e for a scale byte below 255: exact, and in the normal range (e <= 120 for any float, -e <= 127).
__device__ __forceinline__ float scale_inverse(int byte) {
  return __builtin_bit_cast(float, byte >= 254 ? 0 : (254 - byte) << 23);
}
__device__ __forceinline__ int magnitude(float x) { return __builtin_bit_cast(int, x) & 0x7fffffff; }

// Four floats within +-448 to four E4M3 bytes, the first in the lowest, to nearest even.
__device__ __forceinline__ int pack_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

}  // namespace svd
