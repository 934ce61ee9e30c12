// Attention of many columns over the same keys where weights must not be rounded to bf16: prompts in fp32, and more than 16 columns
// (queries x heads of a group) over the paged cache.
//
// A workgroup takes 64 columns and all keys of them (of its chunk), 32 keys at a time: they are loaded into registers some tiles
// ahead, turned into bf16 once for all columns and put into LDS; each of four waves owns 16 columns.  Prompts have two such groups
// of waves, which take tiles in turns and join at the end: half the way from the first key to the last (64 us, 71 with one, for four prompts
// of 301..1501 tokens, 8 heads of 64; over the cache, whose chunks are short, one group is faster by 14 % on ragged lengths).  fp32 becomes
// three bf16 parts that add up to it to 2^-24, and a product of fp32 six products of parts (what is left out is 2^-25 of it each): 6 passes of
// the bf16 matrix pipe take 3/8 of the time of one of the fp32 pipe.  8 bits are one part, their scale included.  Weights are three parts
// for outputs in fp32, two for bf16.
//
// Bound by the vector and LDS pipes of workgroups that run for different times (ragged lengths), not by memory: 64 queries of 32
// sequences of 501..4000 tokens, 12 / 4 heads of 64 in 8 bits, outputs in fp32: 60.5 us = 240 TFLOP/s of the two products (each weight is
// multiplied in three parts; vector pipe busy 40 %, 1.8 of 4 waves a SIMD resident on average); the fp32 prompts
// above, now 61 us = 91 TFLOP/s (matrix 22 %, vector 37 %).
//
// The operand layouts are those of the narrow kernel: S^T = K Q^T, O^T = V^T P^T in tiles of 16, P in registers throughout.
// The maximum is that of the first keys, as everywhere; a rise is noticed from the sums, and the workgroup starts over with
// maxima that move.
#pragma once
#include "attend_paged.hpp"
#include "attend_prompt.hpp"

namespace tsdp {

constexpr float BF16_MOST = 3.3895313892515355e38f;

// fp32 data as NK bf16 parts; a value next to the largest fp32 does not round to infinity
template <int NK>
__device__ __forceinline__ void split_data(float x, float y, bf16x2 (&p)[NK]) {
  p[0] = bf16x2{(__bf16)__builtin_amdgcn_fmed3f(x, -BF16_MOST, BF16_MOST), (__bf16)__builtin_amdgcn_fmed3f(y, -BF16_MOST, BF16_MOST)};
  const uint32_t w = __builtin_bit_cast(uint32_t, p[0]);
  bf16x2 rest[NK - 1];
  split<NK - 1>(x - as_f32(w << 16), y - as_f32(w & 0xFFFF0000u), rest);
#pragma unroll
  for (int i = 1; i < NK; ++i) p[i] = rest[i - 1];
}

// D / 8 elements of one key's row, as a thread loads them: `row` is the first of 16 rows (the same for a wave: their page is), place
// the thread's 8 parts a row from there
template <int D, int HELD> struct WideRow;
template <int D> struct WideRow<D, HELD_F32> {
  static constexpr int E = D / 8, NK = 3;
  f32x4 x[E / 4];
  __device__ __forceinline__ void load(const void* pool, const uint8_t*, int64_t row, uint32_t place) {
    at(static_cast<const char*>(pool) + row * (4 * D), place * (4 * E));
  }
  __device__ __forceinline__ void at(const char* base, uint32_t off) {
#pragma unroll
    for (int i = 0; i < E / 4; ++i) x[i] = *reinterpret_cast<const f32x4*>(base + off + 16 * i);
  }
  // words of element pairs, [part][pair]; bits of elements that are not finite
  __device__ __forceinline__ void parts(uint32_t (&w)[NK][E / 2]) const {
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {
      bf16x2 p[NK];
      split_data<NK>(x[i / 2][2 * (i % 2)], x[i / 2][2 * (i % 2) + 1], p);
#pragma unroll
      for (int z = 0; z < NK; ++z) w[z][i] = __builtin_bit_cast(uint32_t, p[z]);
    }
  }
  __device__ __forceinline__ uint32_t unusual() {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (not_finite_f32(x[i / 4][i % 4])) { m |= 1u << i; x[i / 4][i % 4] = 0.f; }
    return m;
  }
};
template <int D> struct WideRow<D, HELD_BF16> {
  static constexpr int E = D / 8, NK = 1;
  uint32_t x[E / 2];
  __device__ __forceinline__ void load(const void* pool, const uint8_t*, int64_t row, uint32_t place) {
    __builtin_memcpy(x, __builtin_assume_aligned(static_cast<const char*>(pool) + row * (2 * D) + place * (2 * E), 2 * E < 16 ? 2 * E : 16), 2 * E);
  }
  __device__ __forceinline__ void parts(uint32_t (&w)[NK][E / 2]) const {
#pragma unroll
    for (int i = 0; i < E / 2; ++i) w[0][i] = x[i];
  }
  __device__ __forceinline__ uint32_t unusual() {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < E / 2; ++i) { m |= not_finite_halves(x[i]) << (2 * i); x[i] = finite_bf16(x[i]); }
    return m;
  }
};
template <int D> struct WideRow<D, HELD_MX8> {
  static constexpr int E = D / 8, NK = 1;
  uint32_t x[E / 4];
  uint8_t scale;                             // as loaded: nothing may wait for it before it is used
  __device__ __forceinline__ void load(const void* pool, const uint8_t* scales, int64_t row, uint32_t place) {
    __builtin_memcpy(x, __builtin_assume_aligned(static_cast<const char*>(pool) + row * D + place * E, E), E);
    scale = (scales + row * (D / MX_BLOCK))[place * E / MX_BLOCK];
  }
  __device__ __forceinline__ void parts(uint32_t (&w)[NK][E / 2]) const {
#pragma unroll
    for (int i = 0; i < E / 4; ++i) {
      const u32x2 y = mx8_to_bf16(x[i], scale_of(scale));
      w[0][2 * i] = y[0]; w[0][2 * i + 1] = y[1];
    }
  }
  __device__ __forceinline__ uint32_t unusual() {
    // judged by what they widen to: memory that nobody wrote may hold any scale
    if (scale == 255) {
#pragma unroll
      for (int i = 0; i < E / 4; ++i) x[i] = 0;
      scale = 127;
      return (1u << E) - 1;
    }
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < E / 4; ++i) {
      const u32x2 y = mx8_to_bf16(x[i], scale_of(scale));
      const uint32_t bad = not_finite_halves(y[0]) | not_finite_halves(y[1]) << 2;
      m |= bad << (4 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[i] &= bad >> e & 1 ? ~(255u << (8 * e)) : ~0u;
    }
    return m;
  }
};

// Rows of a tile are CH chunks of 16 bytes.  Keys are read by 16 rows at one chunk (key_swizzle), values by 8 rows at 32 bytes at a time.
template <int CH> __device__ __forceinline__ int wide_swizzle(int row) { return CH >= 16 ? (row & 7) << 1 : CH == 8 ? ((row >> 1) & 3) << 1 : ((row >> 2) & 1) << 1; }

template <int D, int HELD, bool QF32, int NP>
struct Wide {
  typedef WideRow<D, HELD> Row;
  static constexpr int KT = 32, NK = Row::NK, NQ = QF32 ? 3 : 1, F = D / 16, CH = D / 8, E = Row::E, PLANE = KT * D * 2;
  static constexpr int BYTES = 2 * NK * PLANE;                   // keys, values
  // Two buffers save a barrier a tile where LDS has room for as many workgroups (64 queries of 32 sequences of 2000 tokens, 12 / 4 heads
  // of 64 in 8 bits: 51.5 us, 52.8 with one; prompts of 32 x 200, 8 heads of 32 in fp32: 23.8 and 25.0).
  static constexpr int BUFFERS = BYTES <= 16 * 1024 ? 2 : 1;
  // Tiles in registers on their way: one in fp32, whose conversion leaves no registers, otherwise four (51.5 us, 52.9 with two; 8
  // sequences of 2000, 64 queries, 32 / 8 heads of 128 in bf16: 50.9 and 53.2).
  static constexpr int AHEAD = NK == 1 ? 4 : 1;
  // Over the cache, tiles without masks: the scores of the next tile while the weights of this one are made, so that the matrix pipe does
  // not wait for the exponentials.  Keys go to LDS a tile before values, into the other buffer (64 queries of 32 sequences of 501..4000
  // tokens, 12 / 4 heads of 64 in 8 bits: 60.5 us, 64.2 one after the other; 4 of 16000, 32 / 8 heads of 128 in bf16: 169 and 187).
  static constexpr bool PIPE = NK == 1;
  static_assert(!PIPE || (AHEAD % 2 == 0 && BUFFERS == 2), "buffers go in turns with the tiles");

  f32x4 o[F];
  bf16x8 q[NQ][D / 32];
  float m, l;
  uint32_t gone;                             // outputs that a visible value makes NaN: bit 4 f + x is o[f][x]

  __device__ __forceinline__ void start(const void* at, int64_t off, int g) {
#pragma unroll
    for (int x = 0; x < D / 32; ++x) {
      if constexpr (QF32) {
        const float* p = static_cast<const float*>(at) + off + 32 * x + 8 * g;
#pragma unroll
        for (int y = 0; y < 8; y += 2) {
          bf16x2 parts[3];
          split_data<3>(p[y], p[y + 1], parts);
#pragma unroll
          for (int z = 0; z < 3; ++z) { q[z][x][y] = parts[z][0]; q[z][x][y + 1] = parts[z][1]; }
        }
      } else {
        q[0][x] = *reinterpret_cast<const bf16x8*>(static_cast<const __bf16*>(at) + off + 32 * x + 8 * g);
      }
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int f = 0; f < F; ++f) o[f] = f32x4{};
    m = -INFINITY; l = 0.f; gone = 0;
  }

  // a thread's part of row `row` into the planes of keys or values
  static __device__ __forceinline__ void put(const Row& r, uint8_t* planes, int row, int part, bool value) {
    uint32_t w[NK][E / 2];
    r.parts(w);
    const int byte = part * E * 2, chunk = (byte >> 4) ^ (value ? wide_swizzle<CH>(row) : key_swizzle<CH>(row));
    uint8_t* at = planes + row * (D * 2) + (byte & 15);
#pragma unroll
    for (int z = 0; z < NK; ++z) {
      if constexpr (E == 16) {               // two chunks: next to each other, in one order or the other
        *reinterpret_cast<u32x4*>(at + z * PLANE + (chunk << 4)) = u32x4{w[z][0], w[z][1], w[z][2], w[z][3]};
        *reinterpret_cast<u32x4*>(at + z * PLANE + ((chunk ^ 1) << 4)) = u32x4{w[z][4], w[z][5], w[z][6], w[z][7]};
      } else if constexpr (E == 8) {
        *reinterpret_cast<u32x4*>(at + z * PLANE + (chunk << 4)) = u32x4{w[z][0], w[z][1], w[z][2], w[z][3]};
      } else {
        *reinterpret_cast<u32x2*>(at + z * PLANE + (chunk << 4)) = u32x2{w[z][0], w[z][1]};
      }
    }
  }

  // of the 32 keys of a tile
  __device__ __forceinline__ void scores(f32x4 (&s)[2], const uint8_t* keys, int lane) const {
    const int r = lane & 15, g = lane >> 4;
    s[0] = f32x4{}; s[1] = f32x4{};
#pragma unroll
    for (int x = 0; x < D / 32; ++x)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        bf16x8 k[NK];
#pragma unroll
        for (int z = 0; z < NK; ++z)
          k[z] = *reinterpret_cast<const bf16x8*>(keys + z * PLANE + (16 * u + r) * (D * 2) + (((4 * x + g) ^ key_swizzle<CH>(16 * u + r)) << 4));
#pragma unroll
        for (int sum = NK + NQ - 2 < 2 ? NK + NQ - 2 : 2; sum >= 0; --sum)       // smallest products first
#pragma unroll
          for (int z = 0; z < NK; ++z)
            if (sum - z >= 0 && sum - z < NQ) s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[z], q[sum - z][x], s[u], 0, 0, 0);
      }
  }
  static __device__ __forceinline__ float largest(const f32x4 (&s)[2]) {
    const float top = max3(max3(s[0][0], s[0][1], s[0][2]), s[0][3], s[1][0]);
    return max_groups(max3(max3(top, s[1][1], s[1][2]), s[1][3], s[1][3]));
  }
  // A tile's scores, weights and product.  careful: some keys are masked (sees), or maxima have to be looked at.
  template <class Sees>
  __device__ __forceinline__ void step(const uint8_t* keys, const uint8_t* values, float c, int lane, bool careful, bool masked, Sees sees) {
    const int g = lane >> 4;
    f32x4 s[2];
    scores(s, keys, lane);
    if (careful) {
      if (masked) {
#pragma unroll
        for (int x = 0; x < 8; ++x)
          if (!sees(16 * (x / 4) + 4 * g + x % 4)) s[x / 4][x % 4] = -INFINITY;
      }
      const float top = largest(s) * c;
      const float to = top > m + MOST_RISE ? top : m, f = to == m ? 1.f : __builtin_amdgcn_exp2f(m - to);
      m = to;
      l *= f;
#pragma unroll
      for (int y = 0; y < F; ++y)
#pragma unroll
        for (int x = 0; x < 4; ++x) o[y][x] *= f;
    }
    product(s, values, c, lane);
  }
  // value operand f: one read turns 4 keys x 16 dims for 16 lanes, each of which names 4 dims of one key
  static __device__ __forceinline__ void operand(bf16x8 (&v)[NK], const uint8_t* values, int f, int lane) {
    typedef __attribute__((ext_vector_type(4))) short s16x4;
    typedef __attribute__((address_space(3))) s16x4* at;
    const int r = lane & 15, g = lane >> 4, row = 4 * g + (r >> 2), dim = 16 * f + (r & 3) * 4;
#pragma unroll
    for (int z = 0; z < NK; ++z) {
      const uint8_t* base = values + z * PLANE + (dim & 7) * 2;
      const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)(base + row * (D * 2) + (((dim >> 3) ^ wide_swizzle<CH>(row)) << 4))));
      const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)(base + (row + 16) * (D * 2) + (((dim >> 3) ^ wide_swizzle<CH>(row + 16)) << 4))));
      v[z] = __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
    }
  }
  // Weights of scores, and their product with the values.  Where registers allow, two operands are read before the weights are made (8
  // sequences of 4096, 16 queries, 32 / 8 heads of 128 in 8 bits: 34.0 us, 37.9 without).
  static constexpr int EARLY = NK == 1 ? 2 : 0;
  __device__ __forceinline__ void product(const f32x4 (&s)[2], const uint8_t* values, float c, int lane) {
    bf16x8 v[F][NK];
#pragma unroll
    for (int f = 0; f < EARLY; ++f) operand(v[f], values, f, lane);
    if (EARLY) __builtin_amdgcn_sched_barrier(0);
    const float sub = m == -INFINITY ? 0.f : m;
    bf16x8 p[NP];
#pragma unroll
    for (int x = 0; x < 8; x += 2) {
      const float e0 = __builtin_amdgcn_exp2f(fmaf(s[x / 4][x % 4], c, -sub)), e1 = __builtin_amdgcn_exp2f(fmaf(s[x / 4][x % 4 + 1], c, -sub));
      l += e0;
      l += e1;
      bf16x2 parts[NP];
      split<NP>(e0, e1, parts);
#pragma unroll
      for (int z = 0; z < NP; ++z) { p[z][x] = parts[z][0]; p[z][x + 1] = parts[z][1]; }
    }
#pragma unroll
    for (int f = 0; f < F; ++f) {
      if (f + EARLY < F) operand(v[f + EARLY], values, f + EARLY, lane);
#pragma unroll
      for (int sum = NK + NP - 2 < 2 ? NK + NP - 2 : 2; sum >= 0; --sum)
#pragma unroll
        for (int z = 0; z < NK; ++z)
          if (sum - z >= 0 && sum - z < NP) o[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[f][z], p[sum - z], o[f], 0, 0, 0);
    }
  }
};

template <class W>
__device__ __forceinline__ void wide_out(const W& w, float* out, float l, int g) {
#pragma unroll
  for (int f = 0; f < W::F; ++f) {
    f32x4 y;
#pragma unroll
    for (int x = 0; x < 4; ++x) y[x] = w.gone >> (4 * f + x) & 1 ? NAN : l == 0.f ? 0.f : w.o[f][x] / l;
    *reinterpret_cast<f32x4*>(out + 16 * f + 4 * g) = y;
  }
}
template <class W>
__device__ __forceinline__ void wide_out(const W& w, __bf16* out, float l, int g) {
#pragma unroll
  for (int f = 0; f < W::F; ++f) {
    bf16x4 y;
#pragma unroll
    for (int x = 0; x < 4; ++x) y[x] = (__bf16)(w.gone >> (4 * f + x) & 1 ? NAN : l == 0.f ? 0.f : w.o[f][x] / l);
    *reinterpret_cast<bf16x4*>(out + 16 * f + 4 * g) = y;
  }
}

// PAGED: the columns of a kv head over a chunk of the cache; otherwise those of a sequence over its rows.
// Waves a SIMD: as many as registers allow; heads of 64 over the cache are held to the 128 of four (64 queries of 32 sequences of 4000
// tokens, 12 / 4 heads in 8 bits, the call: 79.7 us, 83.2 with the 130 of three), but for queries of three parts, which need 146.
template <bool PAGED> constexpr int WIDE_GROUPS = PAGED ? 1 : 2;
template <int D, int HELD, bool QF32, int NP, typename Out, bool PAGED, typename Args>
__global__ __launch_bounds__(256 * WIDE_GROUPS<PAGED>, (D == 128 ? 2 : PAGED && QF32 ? 3 : 4)) void k_wide(Args a) {
  constexpr int GROUPS = WIDE_GROUPS<PAGED>, WAVES = 4 * GROUPS;
  typedef Wide<D, HELD, QF32, NP> W;
  constexpr int COLS = 64;
  typedef typename W::Row Row;
  constexpr int F = W::F, KT = W::KT;
  __shared__ __align__(16) uint8_t lds_all[GROUPS][W::BUFFERS][W::BYTES];
  __shared__ uint8_t where_all[GROUPS][W::BUFFERS][KT * 8];           // D / 8 elements a byte or two: values of the tile that are not finite
  __shared__ uint8_t where_hi_all[GROUPS][D == 128 ? W::BUFFERS : 1][D == 128 ? KT * 8 : 1];
  __shared__ uint32_t unusual[WAVES], rises[WAVES];
  const int lane = threadIdx.x & 63, wave8 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  const int group = GROUPS == 1 ? 0 : wave8 >> 2, wave = wave8 & 3, tid = threadIdx.x & 255;
  const int my_row = tid >> 3, part = tid & 7;                   // what this thread loads of a tile
  auto& lds = lds_all[group];
  auto& where = where_all[group];
  auto& where_hi = where_hi_all[group];
  if (lane == 0) { unusual[wave8] = 0; rises[wave8] = 0; }

  int mine, tiles, plain;                    // keys that this lane's column sees, tiles at all, tiles that all columns see
  W w;
  // PAGED: place of the chunk; otherwise: of the queries
  int kvh, b, col, chunks = 1, chunk = 0, len = 0, pages = 0, G = 1;
  long lo = 0;
  PromptTile t;
  if constexpr (PAGED) {
    const int kv = a.cache.kv_heads, ct = (a.cols + COLS - 1) / COLS;
    kvh = blockIdx.x % kv; chunk = blockIdx.y;
    const int rest = blockIdx.x / kv;
    const int col0 = (rest % ct) * COLS;
    b = rest / ct;
    len = paged_len(a, b);
    const int shift = chunk_shift(len, a.cols, a.fp32);
    chunks = chunks_of(len, a.cols, a.fp32);
    if (chunk > 0 && chunk >= chunks) return;
    G = a.heads / kv;
    lo = (long)chunk << shift;
    const long hi = min(lo + (1L << shift), (long)len);
    if (lo + 16 * lane < hi) {               // pages of the chunk's keys, 16 a lane
      pages = page_of(a.cache, b, (lo + 16 * lane) >> a.cache.page_shift);
      if (pages < 0) report(a.status, STATUS_PAGE);
    }
    const long all = min((long)seen(col0 / G, a.tokens, len, a.causal), hi) - lo;
    tiles = lo < hi ? (int)((hi - lo + KT - 1) / KT) : 0;
    plain = __any(pages < 0) ? 0 : (int)(max(all, 0L) / KT);
    col = col0 + 16 * wave + r;
    const int token = min(col, a.cols - 1) / G;
    mine = col < a.cols ? (int)max(0L, min((long)seen(token, a.tokens, len, a.causal), hi) - lo) : 0;
  } else {
    if (!prompt_tile<COLS>(a, t)) return;
    kvh = t.kv_head; b = t.b;
    G = a.group;
    tiles = (seen(query_of(min(t.i0 + COLS, t.columns) - 1, G), t.nq, t.nk, a.causal) + KT - 1) / KT;
    plain = seen(query_of(t.i0, G), t.nq, t.nk, a.causal) / KT;
    col = t.i0 + 16 * wave + r;
    mine = col < t.columns ? seen(query_of(col, G), t.nq, t.nk, a.causal) : 0;
  }

  constexpr int AHEAD = W::AHEAD;
  Row rk[AHEAD], rv[AHEAD];                  // tiles on their way
  uint32_t k_off = 0, v_off = 0;             // !PAGED: this thread's bytes of a tile (a row is at most 2^24 elements)
  if constexpr (!PAGED) { k_off = (my_row * (uint32_t)a.k_row + part * W::E) * 4; v_off = (my_row * (uint32_t)a.v_row + part * W::E) * 4; }
  // keys or values of tile n of the cache
  auto load_one = [&](Row& r, const void* pool, const uint8_t* scales, int n) __attribute__((always_inline)) {
    if constexpr (PAGED) {
      if (n >= tiles) return;
      const int page = max(__builtin_amdgcn_readlane(pages, 2 * n + (wave >> 1)), 0);
      r.load(pool, scales, pool_row(a.cache, page, kvh, (int)((lo + KT * n + 16 * (wave >> 1)) & ((1 << a.cache.page_shift) - 1))), tid & 127);
    }
  };
  // the group's tile i is tile GROUPS i + group
  auto load = [&](Row& rk, Row& rv, int i) __attribute__((always_inline)) {
    const int n = GROUPS * i + group;
    if (n >= tiles) return;
    if constexpr (PAGED) {
      load_one(rk, a.cache.k, a.cache.k_scale, n);
      load_one(rv, a.cache.v, a.cache.v_scale, n);
    } else {
      const char* ka = reinterpret_cast<const char*>(static_cast<const float*>(a.k) + (int64_t)(t.k_lo + KT * n) * a.k_row + kvh * D);
      const char* va = reinterpret_cast<const char*>(static_cast<const float*>(a.v) + (int64_t)(t.k_lo + KT * n) * a.v_row + kvh * D);
      uint32_t ko = k_off, vo = v_off;
      if (KT * (n + 1) > t.nk) {             // rows behind the sequence: its last one, masked
        const int over = max(KT * n + my_row - (t.nk - 1), 0);
        ko -= over * (uint32_t)a.k_row * 4; vo -= over * (uint32_t)a.v_row * 4;
      }
      rk.at(ka, ko);
      rv.at(va, vo);
    }
  };
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) load(rk[u], rv[u], u);
  if constexpr (PAGED) {
    const int at = min(col, a.cols - 1);
    w.start(a.q, ((int64_t)b * a.tokens + at / G) * a.q_row + (kvh * G + at % G) * D, g);
  } else {
    const int at = min(col, t.columns - 1);
    const int query = query_of(at, G);
    w.start(a.q, (int64_t)(t.q_lo + query) * a.q_row + (kvh * G + at - query * G) * D, g);
  }
  w.clear();

  bool careful = false, rose = false;
  auto tile = [&](Row& rk, Row& rv, int i, int buffer) __attribute__((always_inline)) {
    const int n = GROUPS * i + group;
    uint8_t* keys = lds[buffer];
    uint8_t* values = keys + W::BYTES / 2;
    const bool masked = n >= plain;
    if (W::BUFFERS == 1 && i > 0) __syncthreads();               // the last tile has been read by all
    if (n < tiles) {
      if (masked) {
        const uint32_t m = rv.unusual();
        where[buffer][tid] = (uint8_t)m;
        if constexpr (D == 128) where_hi[buffer][tid] = (uint8_t)(m >> 8);
        if (__any(m != 0) && lane == 0) unusual[wave8] = 1;
      }
      W::put(rk, keys, my_row, part, false);
      W::put(rv, values, my_row, part, true);
      load(rk, rv, i + AHEAD);
    }
    __syncthreads();
    if (n >= tiles) return;
    bool ok0 = true, ok1 = true;
    if constexpr (PAGED) { ok0 = __builtin_amdgcn_readlane(pages, 2 * n) >= 0; ok1 = __builtin_amdgcn_readlane(pages, 2 * n + 1) >= 0; }
    auto sees = [&](int key) __attribute__((always_inline)) { return (key < 16 ? ok0 : ok1) && KT * n + key < mine; };
    w.step(keys, values, a.c, lane, masked || careful || i == 0, masked, sees);
    if (n < plain && n + GROUPS >= plain) rose = w.l > most_sum(w.m); // in the tiles without masks a maximum would have had to move
    if (masked && any_of<WAVES>(unusual)) {
#pragma unroll 1
      for (int key = 0; key < KT; ++key) {
        uint32_t gone = 0;
        // row 4 g + x of operand f: dim 16 f + 4 g + x
#pragma unroll
        for (int f = 0; f < F; ++f) {
          const int dim = 16 * f + 4 * g, at = key * 8 + dim / W::E;
          uint32_t bits = where[buffer][at];
          if constexpr (D == 128) bits |= (uint32_t)where_hi[buffer][at] << 8;
          gone |= (bits >> (dim % W::E) & 15u) << (4 * f);
        }
        if (sees(key)) w.gone |= gone;
      }
    }
  };
  int from = 0;                              // first tile of the loop that looks at masks and maxima
  if constexpr (W::PIPE && PAGED) if (plain > 0) {
    f32x4 s[2][2];
    W::put(rk[0], lds[0], my_row, part, false);
    load_one(rk[0], a.cache.k, a.cache.k_scale, AHEAD);
    __syncthreads();
    w.scores(s[0], lds[0], lane);
    const float top = W::largest(s[0]) * a.c;
    w.m = top > -INFINITY ? top : -INFINITY;
    for (int n = 0; n < plain; n += AHEAD) {
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        if (n + u >= plain) break;
        W::put(rv[u], lds[u % 2] + W::BYTES / 2, my_row, part, true);
        load_one(rv[u], a.cache.v, a.cache.v_scale, n + u + AHEAD);
        if (n + u + 1 < plain) {
          W::put(rk[(u + 1) % AHEAD], lds[(u + 1) % 2], my_row, part, false);
          load_one(rk[(u + 1) % AHEAD], a.cache.k, a.cache.k_scale, n + u + 1 + AHEAD);
          __syncthreads();
          w.scores(s[(u + 1) % 2], lds[(u + 1) % 2], lane);
        } else {
          __syncthreads();
        }
        w.product(s[u % 2], lds[u % 2] + W::BYTES / 2, a.c, lane);
      }
    }
    careful = true;
    from = plain;
    if (__any(w.l > most_sum(w.m)) && lane == 0) rises[wave8] = 1;
    __syncthreads();
    if (any_of<WAVES>(rises)) {                // once more, with maxima that move
      w.clear();
      from = 0;
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) load(rk[u], rv[u], from + u);
  }
  const int steps = (tiles + GROUPS - 1) / GROUPS, steps_plain = (plain + GROUPS - 1) / GROUPS;
  for (int i = from; i < steps; i += AHEAD) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (i + u >= steps) break;
      tile(rk[u], rv[u], i + u, AHEAD % W::BUFFERS == 0 ? u % W::BUFFERS : (i + u) % W::BUFFERS);
    }
    if (!careful && plain > 0 && i + AHEAD >= steps_plain) {
      careful = true;
      if (__any(rose) && lane == 0) rises[wave8] = 1;
      __syncthreads();
      if (any_of<WAVES>(rises)) {                // once more, with maxima that move
        w.clear();
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) load(rk[u], rv[u], u);
        i = -AHEAD;
      }
    }
  }

  if constexpr (GROUPS == 2) {               // the second group's share to the first one
    f32x4* from = reinterpret_cast<f32x4*>(&lds_all[0][0][0]) + wave * (F * 64) + lane;
    __shared__ float ml[4][64][2];
    __shared__ uint32_t lost[4][64];
    static_assert(4 * F * 64 * 16 <= (int)sizeof(lds_all), "a group's outputs fit the tiles");
    __syncthreads();
    if (group == 1) {
#pragma unroll
      for (int f = 0; f < F; ++f) from[f * 64] = w.o[f];
      ml[wave][lane][0] = w.m; ml[wave][lane][1] = w.l; lost[wave][lane] = w.gone;
    }
    __syncthreads();
    if (group == 1) return;
    const float m = ml[wave][lane][0], top = fmaxf(w.m, m), sub = top == -INFINITY ? 0.f : top;
    const float f0 = __builtin_amdgcn_exp2f(w.m - sub), f1 = __builtin_amdgcn_exp2f(m - sub);
    w.l = w.l * f0 + ml[wave][lane][1] * f1;
    w.m = top;
    w.gone |= lost[wave][lane];
#pragma unroll
    for (int f = 0; f < F; ++f) {
      const f32x4 y = from[f * 64];
#pragma unroll
      for (int x = 0; x < 4; ++x) w.o[f][x] = w.o[f][x] * f0 + y[x] * f1;
    }
  }
  const float l = sum_groups(w.l);
  int64_t row;                               // of the outputs
  int head;
  if constexpr (PAGED) {
    if (col >= a.cols) return;
    head = kvh * G + col % G;
    row = (int64_t)b * a.tokens + col / G;
    if (chunks > 1) {
      const int64_t at = (((int64_t)b * a.cache.kv_heads + kvh) * a.cols + col) * a.max_chunks + chunk;
#pragma unroll
      for (int f = 0; f < F; ++f) {
        f32x4 y;
#pragma unroll
        for (int x = 0; x < 4; ++x) y[x] = w.gone >> (4 * f + x) & 1 ? NAN : w.o[f][x];
        *reinterpret_cast<f32x4*>(a.part + at * D + 16 * f + 4 * g) = y;
      }
      if (g == 0) { a.part_ml[2 * at] = w.m; a.part_ml[2 * at + 1] = l; }
      return;
    }
  } else {
    if (col >= t.columns) return;
    const int query = query_of(col, G);
    head = kvh * G + col - query * G;
    row = t.q_lo + query;
  }
  wide_out(w, static_cast<Out*>(a.out) + row * a.out_row + head * D, l, g);
  if (a.lse && g == 0) a.lse[row * a.heads + head] = (w.m + __builtin_amdgcn_logf(l)) * LN2;
}

}  // namespace tsdp
