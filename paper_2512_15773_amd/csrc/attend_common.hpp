// Device pieces that the cache and attention kernels share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "attend_plan.hpp"

namespace tsdp {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr int HELD_F32 = 0, HELD_BF16 = 1, HELD_MX8 = 2;
constexpr int STATUS_ROWS = 1 << 5, STATUS_PAGE = 1 << 6;      // tsdp_status bits of these kernels

__device__ __forceinline__ void report(int32_t* status, int bit) { atomicOr(status, bit); }

// How many i in 1..n (n = B) have f(i) <= x, f growing: 64 probes a step, all lanes of the wave together (x uniform).
template <class F>
__device__ __forceinline__ int count_upto(int B, int x, F f) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = B;
  while (n > 64) {
    const int step = (n + 63) / 64, at = (lane + 1) * step;
    const bool in = at <= n && f(lo + at) <= x;
    lo += __popcll(__ballot(in)) * step;
    n = min(step, B - lo);
  }
  const bool in = lane < n && f(lo + lane + 1) <= x;
  return lo + __popcll(__ballot(in));
}

__device__ __forceinline__ float as_f32(uint32_t b) { return __builtin_bit_cast(float, b); }
__device__ __forceinline__ uint32_t as_u32(float f) { return __builtin_bit_cast(uint32_t, f); }
__device__ __forceinline__ float scale_of(uint32_t byte) { return as_f32(byte << 23); }   // 2^(byte - 127), byte 1 .. 254

// four e4m3 values of a word, times a power of two, as bf16 (exact)
__device__ __forceinline__ u32x2 mx8_to_bf16(uint32_t w, float scale) {
  u32x2 r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true));
  return r;
}

// NaN where one of them is (v_maximum3_f32: needs no quieting of its operands, as fmaxf does)
__device__ __forceinline__ float max3(float a, float b, float c) {
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}
// largest / sum over the four groups of 16 lanes, and over the two halves of the wave
__device__ __forceinline__ float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(as_u32(x), as_u32(x), false, false);
  return __builtin_elementwise_maximum(as_f32(r[0]), as_f32(r[1]));
}
__device__ __forceinline__ float sum_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(as_u32(x), as_u32(x), false, false);
  return as_f32(r[0]) + as_f32(r[1]);
}
__device__ __forceinline__ float max_groups(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(as_u32(x), as_u32(x), false, false);
  return max_halves(__builtin_elementwise_maximum(as_f32(r[0]), as_f32(r[1])));
}
__device__ __forceinline__ float sum_groups(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(as_u32(x), as_u32(x), false, false);
  return sum_halves(as_f32(r[0]) + as_f32(r[1]));
}

// a bf16 that is not finite: exponent bits all ones (either half of a word)
__device__ __forceinline__ bool not_finite_bf16(uint32_t w) {
  return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u;
}
__device__ __forceinline__ uint32_t not_finite_halves(uint32_t w) {   // bit 0: the low half, bit 1: the high one
  return ((w & 0x7F80u) == 0x7F80u ? 1u : 0u) | ((w & 0x7F800000u) == 0x7F800000u ? 2u : 0u);
}
// whether one of eight is not finite
__device__ __forceinline__ bool some_not_finite(u32x4 w) {
  typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
  u16x2 most = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, w[i] & 0x7FFF7FFFu));
  return most[0] >= 0x7F80u || most[1] >= 0x7F80u;
}
// both halves: 0 where finite, 1.0 where not; and the word with such halves taken out
__device__ __forceinline__ uint32_t marks_bf16(uint32_t w) {
  return ((w & 0x7F80u) == 0x7F80u ? 0x3F80u : 0u) | ((w & 0x7F800000u) == 0x7F800000u ? 0x3F800000u : 0u);
}
__device__ __forceinline__ uint32_t finite_bf16(uint32_t w) {
  return ((w & 0x7F80u) == 0x7F80u ? 0u : w & 0xFFFFu) | ((w & 0x7F800000u) == 0x7F800000u ? 0u : w & 0xFFFF0000u);
}
__device__ __forceinline__ bool not_finite_f32(float f) { return (as_u32(f) & 0x7F800000u) == 0x7F800000u; }

// A query's maximum is that of its first keys, and moves only where a score is 2^48 times its weight above it (each query by its
// own scores): weights up to 2^48 lose nothing in floating types, and leave 2^59 to the values before a sum of 2^20 of them
// overflows.
constexpr float MOST_RISE = 48.f;
// what a sum of weights exceeds if one of them rose further (or was infinite); any does if the first keys gave no maximum at all
__device__ __forceinline__ float most_sum(float m) { return m == -INFINITY ? -1.f : __builtin_amdgcn_exp2f(MOST_RISE); }
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

}  // namespace tsdp
