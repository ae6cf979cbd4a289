// Device helpers that the kernels of several files share (kf_rows.hip,
// kf_budget.hip).
#pragma once

#include "kf_internal.h"

namespace kf {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }
__device__ __forceinline__ float qnan() { return __builtin_nanf(""); }
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  bf16x2 v = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, v);
}

// Slice index of (page, KV head) in a pool of either layout.
__device__ __forceinline__ size_t slice_of(int page, int g, int H, int P, int32_t head_major) {
  return head_major ? (size_t)g * P + page : (size_t)page * H + g;
}

template <class T>
__device__ __forceinline__ u32x4 ld16(const T* p) {
  return *reinterpret_cast<const u32x4*>(p);
}

// E4M3FN codes of two floats, round to nearest even, clamped to +-448, the
// sign bit the input's (a NaN becomes 448), in the low half.
__device__ __forceinline__ uint32_t e4m3_pair(float x, float y) {
  x = __builtin_copysignf(fminf(fabsf(x), 448.0f), x);
  y = __builtin_copysignf(fminf(fabsf(y), 448.0f), y);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, y, 0, false) & 0xFFFFu;
}

// Values of the two codes in the low half (exact).
__device__ __forceinline__ f32x2 e4m3_values(uint32_t codes) {
  const uint32_t b = __builtin_bit_cast(
      uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.0f, false));
  return f32x2{__builtin_bit_cast(float, b << 16), __builtin_bit_cast(float, b & 0xFFFF0000u)};
}

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) x = fmaxf(x, __shfl_xor(x, m));
  return x;
}

__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Tables that no kernel of the launch writes, read through the scalar cache.
template <class T>
__device__ __forceinline__ const __attribute__((address_space(4))) T* fixed(const T* p) {
  return (const __attribute__((address_space(4))) T*)(uintptr_t)p;
}

// 16 E4M3 codes -> two times 8 bf16, exactly.
__device__ __forceinline__ void widen(u32x4 codes, u32x4& lo, u32x4& hi) {
  uint32_t o[8];
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    o[2 * w] = __builtin_bit_cast(
        uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[w], 1.0f, false));
    o[2 * w + 1] = __builtin_bit_cast(
        uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[w], 1.0f, true));
  }
  lo = u32x4{o[0], o[1], o[2], o[3]};
  hi = u32x4{o[4], o[5], o[6], o[7]};
}

}  // namespace
}  // namespace kf
