// The paged key / value cache: rows of new tokens written into its pages (quantised on the way) and read back.
//
// Both kernels are one pass over the data, bound by HBM: a wave takes one token's row of keys and values (several, where they
// are short), finds the environment that the row belongs to and the page of its position, and moves 8 elements a lane and step.
// Measured: 8 sequences of 9001..16384 tokens, 8 heads of 128, bf16 rows into 8 bits 137 us = 4.5 TB/s, and back 125 us = 5.0 TB/s (a
// large copy: 5.1); 65536 rows of one head of 32: 8.7 us and 7.2 (19.3 and 16.9 with a row a wave).
//
// 8 bits (gfx950 converts to and from them in one instruction): blocks of 32 elements along a head share one power of two,
// the smallest 2^e with max|x| <= 448 * 2^e, and are held as e4m3 of x * 2^-e, rounded to the nearest, ties to even.  The
// power of two makes x * 2^-e exact, so each value is rounded once; it costs no relative precision, e4m3 being a floating
// type itself.  e starts at -111: what is held is then a normal bf16 or zero when read back, whatever its element.  An
// infinity or NaN is held as NaN and does not enter its block's scale.
#pragma once
#include "attend_common.hpp"

namespace tsdp {

struct CacheRows {
  CacheView c;
  int B, R_cap;
  const int32_t* row_ptr; const int32_t* start;
  void* k; void* v;                          // packed rows
  int64_t k_row, v_row;                      // elements from one row to the next
  int per_wave;                              // rows a wave takes
  int32_t* status;
};

// A lane's row, first unit of 8 elements, page and place; page -1: outside.  False: no live row.
__device__ __forceinline__ bool place_of(const CacheRows& a, int units, int lane, int& r, int& u, int& page, int& token) {
  const int first = __builtin_amdgcn_readfirstlane((blockIdx.x * 4 + (threadIdx.x >> 6)) * a.per_wave);
  if (first >= a.R_cap) return false;
  if (first == 0 && lane == 0 && a.row_ptr[a.B] > a.R_cap) report(a.status, STATUS_ROWS);
  int b = count_upto(a.B, first, [&](int i) { return a.row_ptr[i]; });
  r = first; u = lane;
  if (a.per_wave > 1) {
    const int n = lane / units;
    if (n >= a.per_wave || first + n >= a.R_cap) return false;
    r += n; u -= n * units;
    while (b < a.B && a.row_ptr[b + 1] <= r) ++b;
  }
  if (b >= a.B) return false;
  const int start = a.row_ptr[b];
  if (r < start) return false;
  const long pos = (long)a.start[b] + (r - start);
  page = pos < 0 ? -1 : page_of(a.c, b, pos >> a.c.page_shift);
  token = (int)(pos & ((1L << a.c.page_shift) - 1));
  if (page < 0 && u == 0) report(a.status, STATUS_PAGE);
  return true;
}

__device__ __forceinline__ void load8(const float* p, float* x) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
}
__device__ __forceinline__ void load8(const __bf16* p, float* x) {
  const bf16x8 a = *reinterpret_cast<const bf16x8*>(p);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (float)a[i];
}
__device__ __forceinline__ void store8(float* p, const float* x) {
  *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]};
  *reinterpret_cast<f32x4*>(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
}
__device__ __forceinline__ void store8(__bf16* p, const float* x) {
  bf16x8 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = (__bf16)x[i];
  *reinterpret_cast<bf16x8*>(p) = r;
}

// scale byte of a block whose largest finite magnitude is amax
__device__ __forceinline__ uint32_t scale_byte(float amax) {
  const uint32_t b = as_u32(amax);
  const int e = (int)(b >> 23) - 8 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return (uint32_t)min(max(e, 16), 254);
}

template <int STEP>
__device__ __forceinline__ float quad_max(float x) {
  const int y = __builtin_amdgcn_update_dpp(0, (int)as_u32(x), STEP == 1 ? 0xB1 : 0x4E, 0xF, 0xF, true);   // lane ^ 1, lane ^ 2
  return fmaxf(x, as_f32((uint32_t)y));
}

template <typename In, int HELD, int D>
__global__ __launch_bounds__(256) void k_cache_write(CacheRows a) {
  const int lane = threadIdx.x & 63, units = a.c.kv_heads * (D / 8);
  int r, u, page, token;
  if (!place_of(a, 2 * units, lane, r, u, page, token) || page < 0) return;
  for (; u < 2 * units; u += 64) {
    const bool val = u >= units;
    const int e = (val ? u - units : u) * 8, head = e / D, off = e % D;
    const In* src = val ? static_cast<const In*>(a.v) + r * a.v_row : static_cast<const In*>(a.k) + r * a.k_row;
    const int64_t row = pool_row(a.c, page, head, token);
    float x[8];
    load8(src + e, x);
    void* pool = val ? a.c.v : a.c.k;
    if constexpr (HELD == HELD_F32) {
      store8(static_cast<float*>(pool) + row * D + off, x);
    } else if constexpr (HELD == HELD_BF16) {
      store8(static_cast<__bf16*>(pool) + row * D + off, x);
    } else {
      float amax = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) amax = fmaxf(amax, not_finite_f32(x[i]) ? 0.f : fabsf(x[i]));
      amax = quad_max<2>(quad_max<1>(amax));                       // four lanes hold a block
      const uint32_t byte = scale_byte(amax);
      const float inv = scale_of(254 - byte);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = not_finite_f32(x[i]) ? as_f32(0x7FC00000u) : x[i] * inv;
      u32x2 q;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * j], x[4 * j + 1], 0, false);
        q[j] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * j + 2], x[4 * j + 3], w, true);
      }
      *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(pool) + row * D + off) = q;
      if ((lane & 3) == 0) (val ? a.c.v_scale : a.c.k_scale)[row * (D / MX_BLOCK) + off / MX_BLOCK] = (uint8_t)byte;
    }
  }
}

// A position outside the pages reads as zeros.
template <typename Out, int HELD, int D>
__global__ __launch_bounds__(256) void k_cache_read(CacheRows a) {
  const int lane = threadIdx.x & 63, units = a.c.kv_heads * (D / 8);
  int r, u, page, token;
  if (!place_of(a, 2 * units, lane, r, u, page, token)) return;
  for (; u < 2 * units; u += 64) {
    const bool val = u >= units;
    const int e = (val ? u - units : u) * 8, head = e / D, off = e % D;
    Out* dst = val ? static_cast<Out*>(a.v) + r * a.v_row : static_cast<Out*>(a.k) + r * a.k_row;
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (page >= 0) {
      const int64_t row = pool_row(a.c, page, head, token);
      const void* pool = val ? a.c.v : a.c.k;
      if constexpr (HELD == HELD_F32) {
        load8(static_cast<const float*>(pool) + row * D + off, x);
      } else if constexpr (HELD == HELD_BF16) {
        load8(static_cast<const __bf16*>(pool) + row * D + off, x);
      } else {
        const u32x2 q = *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(pool) + row * D + off);
        const float s = scale_of((val ? a.c.v_scale : a.c.k_scale)[row * (D / MX_BLOCK) + off / MX_BLOCK]);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(q[j], s, false);
          const auto hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(q[j], s, true);
          x[4 * j] = lo[0]; x[4 * j + 1] = lo[1]; x[4 * j + 2] = hi[0]; x[4 * j + 3] = hi[1];
        }
      }
    }
    store8(dst + e, x);
  }
}

}  // namespace tsdp
