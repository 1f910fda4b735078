// Number formats and small vector types that the kernels share.
#pragma once

#include "eep_internal.hpp"

namespace eep {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ inline float bf16_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ inline float bf16_hi(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }

// Two binary32 -> two bfloat16 in one dword, round to nearest even, NaN stays (quiet) NaN: one
// v_cvt_pk_bf16_f32.  Compared with the integer form of the rule (add 0x7fff and the kept
// bit, shift) over all 2^32 inputs, NaNs and subnormals included: no difference.
__device__ inline uint32_t pack_bf16x2(float lo, float hi) {
  const f32x2 v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// Maximum over aligned groups of n lanes (n a power of two <= 64), in every lane of the group.
__device__ __forceinline__ uint32_t group_max(uint32_t v, int n) {
  auto larger = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
  if (n > 1) v = larger(v, __builtin_amdgcn_update_dpp(0u, v, 0xB1, 0xf, 0xf, false));   // lane ^ 1
  if (n > 2) v = larger(v, __builtin_amdgcn_update_dpp(0u, v, 0x4E, 0xf, 0xf, false));   // lane ^ 2
  if (n > 4) v = larger(v, __builtin_amdgcn_update_dpp(0u, v, 0x141, 0xf, 0xf, false));  // half row mirrored
  if (n > 8) v = larger(v, __builtin_amdgcn_update_dpp(0u, v, 0x140, 0xf, 0xf, false));  // row mirrored
  for (int m = 16; m < n; m <<= 1) v = larger(v, __shfl_xor(v, m, 64));
  return v;
}

// One of 16 (a row of lanes) or all 64 lanes' values, in every lane: op joins two, in any order.
template <int LANES, class T, class Op>
__device__ __forceinline__ T fold(T v, Op op) {
  static_assert(sizeof(T) == 4 && (LANES == 16 || LANES == 64), "");
  const auto bits = [&]() { return __builtin_bit_cast(uint32_t, v); };
  const auto join = [&](uint32_t other) { v = op(v, __builtin_bit_cast(T, other)); };
  join(__builtin_amdgcn_update_dpp(0u, bits(), 0xB1, 0xf, 0xf, false));   // lane ^ 1
  join(__builtin_amdgcn_update_dpp(0u, bits(), 0x4E, 0xf, 0xf, false));   // lane ^ 2
  join(__builtin_amdgcn_update_dpp(0u, bits(), 0x141, 0xf, 0xf, false));  // half row mirrored
  join(__builtin_amdgcn_update_dpp(0u, bits(), 0x140, 0xf, 0xf, false));  // row mirrored
  if constexpr (LANES == 64) {
    const auto rows = __builtin_amdgcn_permlane16_swap(bits(), bits(), false, false);  // both of a pair of rows
    const uint32_t even = rows[0], odd = rows[1];
    v = op(__builtin_bit_cast(T, even), __builtin_bit_cast(T, odd));
    const auto halves = __builtin_amdgcn_permlane32_swap(bits(), bits(), false, false);
    const uint32_t low = halves[0], high = halves[1];
    v = op(__builtin_bit_cast(T, low), __builtin_bit_cast(T, high));
  }
  return v;
}

// Eight neighbouring values of an array, fp32 or bf16.
template <bool BF16>
__device__ __forceinline__ void load8(const void* base, int64_t vec, float (&v)[8]) {
  if constexpr (BF16) {
    const u32x4 d = ((const u32x4*)base)[vec];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = bf16_lo(d[i]);
      v[2 * i + 1] = bf16_hi(d[i]);
    }
  } else {
    const f32x4 a = ((const f32x4*)base)[2 * vec], b = ((const f32x4*)base)[2 * vec + 1];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = a[i];
      v[4 + i] = b[i];
    }
  }
}

template <bool BF16>
__device__ __forceinline__ void store8(void* base, int64_t vec, const float (&v)[8]) {
  if constexpr (BF16) {
    u32x4 d;
#pragma unroll
    for (int i = 0; i < 4; ++i) d[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
    __builtin_nontemporal_store(d, &((u32x4*)base)[vec]);
  } else {
    __builtin_nontemporal_store(f32x4{v[0], v[1], v[2], v[3]}, &((f32x4*)base)[2 * vec]);
    __builtin_nontemporal_store(f32x4{v[4], v[5], v[6], v[7]}, &((f32x4*)base)[2 * vec + 1]);
  }
}

// The sum over groups of 16 or all 64 lanes, in every lane.
template <int LANES>
__device__ __forceinline__ float lane_sum(float v) {
  return fold<LANES>(v, [](float a, float b) { return a + b; });
}

// The largest magnitude of N fp32 values as its bits, which are ordered as the values are, NaN above everything.
template <int N>
__device__ __forceinline__ uint32_t top_magnitude(const float (&v)[N]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t m = __float_as_uint(v[i]) & 0x7fffffffu;
    top = m > top ? m : top;
  }
  return top;
}

// The scale of a group of that largest magnitude.
__device__ __forceinline__ float scale_of(uint32_t top) {
  const float scale = __uint_as_float(top) / 448.0f;
  return scale == 0.0f ? 1.0f : scale;
}

// v / scale, saturating at +-448 (NaN stays NaN), which the conversion by itself does not: it gives NaN above 464.  A normal scale
// leaves no quotient above 448 but for its roundings, a subnormal one of up to 13 units of 2^-149 is rounded so far that there are some of 671.
__device__ __forceinline__ float quotient(float v, float scale) {
  return __builtin_elementwise_maximum(__builtin_elementwise_minimum(v / scale, 448.0f), -448.0f);
}

// e4m3(v / scale) of four values, round to nearest even, saturating.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float scale) {
  const int low = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(a, scale), quotient(b, scale), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(quotient(c, scale), quotient(d, scale), low, true);
}

}  // namespace eep
