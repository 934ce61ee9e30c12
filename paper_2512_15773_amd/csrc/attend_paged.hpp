// Attention of new tokens over the paged cache, split over the cache's length and joined.
//
// Bound by the stream of keys and values out of HBM: every byte is loaded once per 16 columns (queries x heads of a group),
// straight from the pages into registers.  A workgroup takes one chunk of one environment's sequence and one kv head; its
// four waves take 32 keys at a time, each with a running softmax of its own, and join through LDS.  A sequence of more than
// one chunk leaves (output, maximum, sum) per chunk in the scratch, which k_paged_join adds up in the order of the chunks.
//
// As in the prompt kernels both products are transposed.  S^T = K Q^T with 16 keys x 16 columns; the score registers of the
// two halves of a tile are keys 4 g + i and 16 + 4 g + i of lane group g = l / 16, which is the operand of P^T as it is
// when the value operand takes its keys in that order.  A lane loads D / 16 neighbouring values of those eight keys (whole
// rows per 16 lanes) and turns them with byte permutes into D / 16 operands, operand f holding dims (D / 16) r + f.
//
// Measured: 8 sequences of 20001..131072 tokens, 32 / 8 heads of 128 in 8 bits, 259 us = 5.2 TB/s (a large read reaches 5.9); 256 of
// 1..2001, 8 / 2 heads of 64 in bf16, 26 us = 5.1 TB/s; the join 4 to 6 us.
//
// Fewer than 32 bits enter a matrix product only without loss: keys and values as they are held (8 bits widen exactly to
// bf16 with their scale), fp32 queries as three bf16 parts, and the weights P as two or three (to 2^-16 or 2^-24 of each).
#pragma once
#include "attend_common.hpp"

namespace tsdp {

struct PagedArgs {
  CacheView cache;
  int B, heads, tokens, cols, max_len, max_chunks, causal, fp32;   // cols = tokens * heads / kv_heads; fp32: type of the queries
  float c;
  const int32_t* len;
  const void* q; void* out;
  int64_t q_row, out_row;
  float* lse;                                // [B * tokens][heads] or null
  float* part;                               // scratch: [B][kv][cols][max_chunks][D], then as many (maximum, sum)
  float* part_ml;
  int32_t* status;
};

__device__ __forceinline__ int paged_len(const PagedArgs& a, int b) {
  const long room = min((long)a.max_len, (long)a.cache.columns << a.cache.page_shift);
  const int n = a.len[b];
  if (n > room && threadIdx.x == 0) report(a.status, STATUS_ROWS);
  return n < 0 ? 0 : (int)min((long)n, room);
}

// 32 keys and values of a kv head in registers, as they are held
template <int D, int HELD> struct PagedTile;

template <int D> struct PagedTile<D, HELD_BF16> {
  u32x4 k[2][D / 32];
  uint32_t v[8][D / 32];
  static constexpr int q_dim(int ks, int g) { return 32 * ks + 8 * g; }   // first of the 8 dims of lane group g in k-step ks
  __device__ __forceinline__ void load(const CacheView& c, const int64_t* row, int lane) {
    const int r = lane & 15, g = lane >> 4;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const uint8_t* kp = static_cast<const uint8_t*>(c.k) + row[s] * (2 * D) + r * (2 * D) + g * 16;
#pragma unroll
      for (int x = 0; x < D / 32; ++x) k[s][x] = *reinterpret_cast<const u32x4*>(kp + 64 * x);
      const uint8_t* vp = static_cast<const uint8_t*>(c.v) + row[s] * (2 * D) + (4 * g) * (2 * D) + r * (D / 8);
#pragma unroll
      for (int i = 0; i < 4; ++i) __builtin_memcpy(v[4 * s + i], __builtin_assume_aligned(vp + i * (2 * D), D / 8), D / 8);
    }
  }
  __device__ __forceinline__ bf16x8 key(int s, int ks, int) const { return __builtin_bit_cast(bf16x8, k[s][ks]); }
  __device__ __forceinline__ void values(uint32_t (&w)[8][D / 32], int) const {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int x = 0; x < D / 32; ++x) w[i][x] = v[i][x];
  }
};

template <int D> struct PagedTile<D, HELD_MX8> {
  static constexpr int NB = D / MX_BLOCK, KV = D >= 64 ? D / 64 : 1;      // scales a row, key loads a row
  static constexpr int KW = D >= 64 ? 4 : 2;                              // words of a key load
  uint32_t k[2][KV][KW], ks[2];
  uint32_t v[8][D / 64 ? D / 64 : 1], vs[2][NB];                          // D = 32: two values a key, in the low half
  static constexpr int q_dim(int s, int g) { return D >= 64 ? 64 * (s / 2) + 16 * g + 8 * (s % 2) : 8 * g; }
  __device__ __forceinline__ void load(const CacheView& c, const int64_t* row, int lane) {
    const int r = lane & 15, g = lane >> 4;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const uint8_t* kp = static_cast<const uint8_t*>(c.k) + (row[s] + r) * D + g * (4 * KW);
#pragma unroll
      for (int x = 0; x < KV; ++x) __builtin_memcpy(k[s][x], __builtin_assume_aligned(kp + 64 * x, 4 * KW), 4 * KW);
      ks[s] = 0;
      __builtin_memcpy(&ks[s], __builtin_assume_aligned(c.k_scale + (row[s] + r) * NB, NB), NB);
      const uint8_t* vp = static_cast<const uint8_t*>(c.v) + (row[s] + 4 * g) * D + r * (D / 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[4 * s + i][0] = 0;
        __builtin_memcpy(v[4 * s + i], __builtin_assume_aligned(vp + i * D, D / 16), D / 16);
      }
      __builtin_memcpy(vs[s], __builtin_assume_aligned(c.v_scale + (row[s] + 4 * g) * NB, 4 * NB), 4 * NB);
    }
  }
  __device__ __forceinline__ bf16x8 key(int s, int x, int lane) const {
    const int g = lane >> 4;
    const float f = D >= 64 ? scale_of((ks[s] >> (8 * (2 * (x / 2) + g / 2))) & 255) : scale_of(ks[s] & 255);
    const int at = D >= 64 ? 2 * (x % 2) : 0;
    const u32x2 lo = mx8_to_bf16(k[s][x / 2][at], f), hi = mx8_to_bf16(k[s][x / 2][at + 1], f);
    return __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
  }
  __device__ __forceinline__ void values(uint32_t (&w)[8][D / 32], int lane) const {
    const int r = lane & 15;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // byte of key i % 4's scale of the block that dims (D / 16) r .. lie in
      const int block = r * (D / 16) / MX_BLOCK, byte = (i % 4) * NB;
      const uint32_t word = D == 128 ? vs[i / 4][i % 4] : D == 64 ? vs[i / 4][(i % 4) / 2] : vs[i / 4][0];
      const float f = scale_of((word >> (8 * (byte % 4 + block))) & 255);
      if constexpr (D == 32) {
        w[i][0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[i][0], f, false));
      } else {
#pragma unroll
        for (int x = 0; x < D / 64; ++x) {
          const u32x2 y = mx8_to_bf16(v[i][x], f);
          w[i][2 * x] = y[0]; w[i][2 * x + 1] = y[1];
        }
      }
    }
  }
};

template <int D> struct PagedTile<D, HELD_F32> {
  f32x4 k[2][D / 16];
  float v[8][D / 16];
  __device__ __forceinline__ void load(const CacheView& c, const int64_t* row, int lane) {
    const int r = lane & 15, g = lane >> 4;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const float* kp = static_cast<const float*>(c.k) + (row[s] + r) * D + g * 4;
#pragma unroll
      for (int x = 0; x < D / 16; ++x) k[s][x] = *reinterpret_cast<const f32x4*>(kp + 16 * x);
      const float* vp = static_cast<const float*>(c.v) + (row[s] + 4 * g) * D + r * (D / 16);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        __builtin_memcpy(v[4 * s + i], __builtin_assume_aligned(vp + i * D, D / 4 < 16 ? D / 4 : 16), D / 4);
    }
  }
};

// x as NP bf16 parts whose sum it is to 2^-8 (1), 2^-16 (2), 2^-24 (3) of it; an infinity has parts that are NaN
template <int NP>
__device__ __forceinline__ void split(float x, float y, bf16x2 (&p)[NP]) {
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    p[i] = bf16x2{(__bf16)x, (__bf16)y};
    const uint32_t w = __builtin_bit_cast(uint32_t, p[i]);
    x -= as_f32(w << 16);
    y -= as_f32(w & 0xFFFF0000u);
  }
}

// One wave's share: 16 columns, with a softmax of their own.
// QF32: queries are fp32.  NP: bf16 parts of P (unused where the cache is fp32).
template <int D, int HELD, bool QF32, int NP>
struct PagedWave {
  static constexpr bool F32 = HELD == HELD_F32;
  static constexpr int NQ = QF32 && !F32 ? 3 : 1, F = D / 16;
  typedef PagedTile<D, HELD> Tile;
  bf16x8 q[F32 ? 1 : NQ][F32 ? 1 : D / 32];
  f32x4 qx[F32 ? F : 1];
  f32x4 o[F];
  float m, l;
  int mine;                                  // keys that this lane's column sees
  uint32_t gone;                             // outputs that a visible value makes NaN: bit 4 f + x is o[f][x]

  __device__ __forceinline__ void start(const void* at, int64_t off, int g) {
    if constexpr (F32) {
#pragma unroll
      for (int x = 0; x < F; ++x) qx[x] = *reinterpret_cast<const f32x4*>(static_cast<const float*>(at) + off + 16 * x + 4 * g);
    } else {
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {
        const int d = Tile::q_dim(x, g);
        if constexpr (QF32) {
          const float* p = static_cast<const float*>(at) + off + d;
#pragma unroll
          for (int y = 0; y < 8; y += 2) {
            bf16x2 parts[3];
            split<3>(p[y], p[y + 1], parts);
#pragma unroll
            for (int z = 0; z < 3; ++z) { q[z][x][y] = parts[z][0]; q[z][x][y + 1] = parts[z][1]; }
          }
        } else {
          q[0][x] = *reinterpret_cast<const bf16x8*>(static_cast<const __bf16*>(at) + off + d);
        }
      }
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int f = 0; f < F; ++f) o[f] = f32x4{};
    m = -INFINITY; l = 0.f; gone = 0;
  }

  __device__ __forceinline__ void scores(const Tile& t, f32x4 (&s)[2], int lane) const {
    s[0] = f32x4{}; s[1] = f32x4{};
    if constexpr (F32) {
#pragma unroll
      for (int x = 0; x < F; ++x)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int u = 0; u < 2; ++u) s[u] = __builtin_amdgcn_mfma_f32_16x16x4f32(t.k[u][x][j], qx[x][j], s[u], 0, 0, 0);
    } else {
#pragma unroll
      for (int x = 0; x < D / 32; ++x)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const bf16x8 key = t.key(u, x, lane);
#pragma unroll
          for (int z = NQ - 1; z >= 0; --z) s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key, q[z][x], s[u], 0, 0, 0);
        }
    }
  }
  static __device__ __forceinline__ float largest(const f32x4 (&s)[2]) {
    const float top = max3(max3(s[0][0], s[0][1], s[0][2]), s[0][3], s[1][0]);
    return max_groups(max3(max3(top, s[1][1], s[1][2]), s[1][3], s[1][3]));
  }
  __device__ __forceinline__ void weights(const f32x4 (&s)[2], float c, float (&p)[8]) {
    const float sub = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      p[x] = __builtin_amdgcn_exp2f(fmaf(s[x / 4][x % 4], c, -sub));
      l += p[x];
    }
  }

  // 32 keys that every column sees.  FIRST: their maximum is taken; afterwards it stays, and a rise above it shows in the sums.
  template <bool FIRST>
  __device__ __forceinline__ void step(const Tile& t, float c, int lane) {
    float p[8];
    f32x4 s[2];
    scores(t, s, lane);
    if (FIRST) {
      const float top = largest(s) * c;
      m = top > -INFINITY ? top : -INFINITY;
    }
    weights(s, c, p);
    if constexpr (F32) {
      product_f32(t.v, p);
    } else {
      uint32_t w[8][D / 32];
      t.values(w, lane);
      product_bf16(w, p);
    }
  }
  __device__ __forceinline__ bool rose() const { return __any(l > most_sum(m)); }

  // Any 32 keys from position k0 on.  ok: their halves' pages are inside the pool.
  __device__ __forceinline__ void masked_step(Tile& t, long k0, bool ok0, bool ok1, float c, int lane) {
    const int g = lane >> 4;
    float p[8];
    f32x4 s[2];
    scores(t, s, lane);
#pragma unroll
    for (int x = 0; x < 8; ++x)
      if (!sees(x, k0, ok0, ok1, g)) s[x / 4][x % 4] = -INFINITY;
    const float top = largest(s) * c, to = top > m + MOST_RISE ? top : m, by = to == m ? 1.f : __builtin_amdgcn_exp2f(m - to);
    m = to;
    l *= by;
#pragma unroll
    for (int y = 0; y < F; ++y)
#pragma unroll
      for (int x = 0; x < 4; ++x) o[y][x] *= by;
    weights(s, c, p);
    // Values that are not finite are taken out of the product, and noted for the columns that see them.
    bool bad = false;
    if constexpr (F32) {
#pragma unroll
      for (int x = 0; x < 8; ++x)
#pragma unroll
        for (int f = 0; f < F; ++f) bad |= not_finite_f32(t.v[x][f]);
      if (__any(bad)) {
#pragma unroll
        for (int f = 0; f < F; ++f) {
          f32x4 marks = f32x4{};
#pragma unroll
          for (int x = 0; x < 8; ++x)
            marks = __builtin_amdgcn_mfma_f32_16x16x4f32(not_finite_f32(t.v[x][f]) ? 1.f : 0.f, sees(x, k0, ok0, ok1, g) ? 1.f : 0.f, marks, 0, 0, 0);
#pragma unroll
          for (int x = 0; x < 4; ++x) gone |= marks[x] != 0.f ? 1u << (4 * f + x) : 0u;
        }
#pragma unroll
        for (int x = 0; x < 8; ++x)
#pragma unroll
          for (int f = 0; f < F; ++f) t.v[x][f] = not_finite_f32(t.v[x][f]) ? 0.f : t.v[x][f];
      }
      product_f32(t.v, p);
    } else {
      uint32_t w[8][D / 32];
      t.values(w, lane);
#pragma unroll
      for (int x = 0; x < 8; ++x)
#pragma unroll
        for (int y = 0; y < D / 32; ++y) bad |= not_finite_bf16(w[x][y]);
      if (__any(bad)) {
        bf16x8 one;
#pragma unroll
        for (int x = 0; x < 8; ++x) one[x] = (__bf16)(sees(x, k0, ok0, ok1, g) ? 1.f : 0.f);
#pragma unroll
        for (int f = 0; f < F; ++f) {
          u32x4 mark = turned(w, f / 2, f % 2);
#pragma unroll
          for (int x = 0; x < 4; ++x) mark[x] = marks_bf16(mark[x]);
          const f32x4 marks = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, mark), one, f32x4{}, 0, 0, 0);
#pragma unroll
          for (int x = 0; x < 4; ++x) gone |= marks[x] != 0.f ? 1u << (4 * f + x) : 0u;
        }
#pragma unroll
        for (int x = 0; x < 8; ++x)
#pragma unroll
          for (int y = 0; y < D / 32; ++y) w[x][y] = finite_bf16(w[x][y]);
      }
      product_bf16(w, p);
    }
  }

  __device__ __forceinline__ bool sees(int x, long k0, bool ok0, bool ok1, int g) const {
    return (x < 4 ? ok0 : ok1) && k0 + 16 * (x / 4) + 4 * g + x % 4 < mine;
  }

  __device__ __forceinline__ void product_f32(const float (&v)[8][F], const float (&p)[8]) {
#pragma unroll
    for (int x = 0; x < 8; ++x)
#pragma unroll
      for (int f = 0; f < F; ++f) o[f] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[x][f], p[x], o[f], 0, 0, 0);
  }
  // low (h = 0) or high halves of word y of eight keys: operand 2 y + h
  static __device__ __forceinline__ u32x4 turned(const uint32_t (&w)[8][D / 32], int y, int h) {
    u32x4 v;
#pragma unroll
    for (int x = 0; x < 4; ++x) v[x] = __builtin_amdgcn_perm(w[2 * x + 1][y], w[2 * x][y], h ? 0x07060302u : 0x05040100u);
    return v;
  }
  __device__ __forceinline__ void product_bf16(const uint32_t (&w)[8][D / 32], const float (&p)[8]) {
    bf16x8 pf[NP];
#pragma unroll
    for (int x = 0; x < 8; x += 2) {
      bf16x2 parts[NP];
      split<NP>(p[x], p[x + 1], parts);
#pragma unroll
      for (int z = 0; z < NP; ++z) { pf[z][x] = parts[z][0]; pf[z][x + 1] = parts[z][1]; }
    }
#pragma unroll
    for (int f = 0; f < F; ++f) {
      const bf16x8 v = __builtin_bit_cast(bf16x8, turned(w, f / 2, f % 2));
#pragma unroll
      for (int z = NP - 1; z >= 0; --z) o[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pf[z], o[f], 0, 0, 0);
    }
  }
};

template <int D, int HELD, bool QF32, int NP, typename Out>
__global__ __launch_bounds__(256, 2) void k_paged(PagedArgs a) {
  constexpr int F = D / 16, OP = D + 4;
  // The next tile is loaded ahead where registers hold two (12 heads on one of 64 in fp32, 32 sequences of 2000: 16.1 us, 18.1 without;
  // 8 sequences of 20001..131072, 32 / 8 heads of 128 in 8 bits: 259 and 263; 256 of 1..2001, 8 / 2 heads of 64 in bf16: 25.8 and 26.5).
  constexpr bool AHEAD = !(HELD == HELD_F32 && D == 128);
  __shared__ __align__(16) float o_lds[4][16][OP];
  __shared__ float ml_lds[4][16][2];
  const int kv = a.cache.kv_heads, kvh = blockIdx.x % kv, b = blockIdx.x / kv, chunk = blockIdx.y;
  const int len = paged_len(a, b);
  const int shift = chunk_shift(len, a.cols, a.fp32), chunks = chunks_of(len, a.cols, a.fp32);
  if (chunk > 0 && chunk >= chunks) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  const int G = a.heads / kv, per_wave = 1 << (shift - 2);       // keys of a wave
  const long lo = ((long)chunk << shift) + wave * per_wave, hi = min(lo + per_wave, (long)len);
  // pages of the wave's keys, 16 a lane: 16 keys lie in one page
  int pages = 0;
  if (lo + 16 * lane < hi) {
    pages = page_of(a.cache, b, (lo + 16 * lane) >> a.cache.page_shift);
    if (pages < 0) report(a.status, STATUS_PAGE);
  }
  const long all = seen(0, a.tokens, len, a.causal);             // keys that every column sees
  typedef PagedWave<D, HELD, QF32, NP> Wave;
  typedef typename Wave::Tile Tile;
  Wave w;
  const int page_mask = (1 << a.cache.page_shift) - 1;
  bool ok[2];                                // the pages of the halves of the tile loaded last are inside the pool
  auto load = [&](Tile& t, int n) __attribute__((always_inline)) {
    int64_t row[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int page = __builtin_amdgcn_readlane(pages, 2 * n + s);
      ok[s] = page >= 0;
      row[s] = pool_row(a.cache, max(page, 0), kvh, (int)((lo + 32 * n + 16 * s) & page_mask));
    }
    t.load(a.cache, row, lane);
  };
  const int tiles = lo < hi ? (int)((hi - lo + 31) >> 5) : 0;
  int plain = __any(pages < 0) ? 0 : min(tiles, (int)((max(all - lo, 0L)) >> 5));   // tiles that every column sees in full
  Tile t[2];
  if (tiles > 0) load(t[0], 0);
  const int at = min(r, a.cols - 1), token = at / G;
  w.mine = r < a.cols ? seen(token, a.tokens, len, a.causal) : 0;
  w.start(a.q, ((int64_t)b * a.tokens + token) * a.q_row + (kvh * G + at % G) * D, g);
  w.clear();
  if (plain > 0) {
    if constexpr (AHEAD) {                   // the next tile's loads before this one's products
      if (1 < tiles) load(t[1], 1);
      w.template step<true>(t[0], a.c, lane);
      int n = 1;
      for (; n + 1 < plain; n += 2) {
        load(t[0], n + 1);
        w.template step<false>(t[1], a.c, lane);
        if (n + 2 < tiles) load(t[1], n + 2);
        w.template step<false>(t[0], a.c, lane);
      }
      if (n < plain) {
        if (n + 1 < tiles) load(t[0], n + 1);
        w.template step<false>(t[1], a.c, lane);
      } else if (n < tiles) {
        t[0] = t[1];
      }
    } else {
      w.template step<true>(t[0], a.c, lane);
      for (int n = 1; n < plain; ++n) {
        load(t[0], n);
        w.template step<false>(t[0], a.c, lane);
      }
      if (plain < tiles) load(t[0], plain);
    }
    if (w.rose()) {                          // once more, with maxima that move
      plain = 0;
      w.clear();
      load(t[0], 0);
    }
  }
  for (int n = plain; n < tiles; ++n) {
    w.masked_step(t[0], lo + 32 * n, ok[0], ok[1], a.c, lane);
    if (n + 1 < tiles) load(t[0], n + 1);
  }
  const float l = sum_groups(w.l);
  if (g == 0) { ml_lds[wave][r][0] = w.m; ml_lds[wave][r][1] = l; }
#pragma unroll
  for (int x = 0; x < 4; ++x)                                    // accumulator row 4 g + x of operand f: dim F (4 g + x) + f
#pragma unroll
    for (int f = 0; f < F; ++f) o_lds[wave][r][F * (4 * g + x) + f] = w.gone >> (4 * f + x) & 1 ? NAN : w.o[f][x];
  __syncthreads();

  const int col = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * F; // 16 threads a column, D / 16 dims each
  if (col >= a.cols) return;
  float top = -INFINITY, total = 0.f, y[F];
#pragma unroll
  for (int v = 0; v < 4; ++v) top = fmaxf(top, ml_lds[v][col][0]);
#pragma unroll
  for (int f = 0; f < F; ++f) y[f] = 0.f;
  const float sub = top == -INFINITY ? 0.f : top;
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    const float f = __builtin_amdgcn_exp2f(ml_lds[v][col][0] - sub);
    total = fmaf(ml_lds[v][col][1], f, total);
#pragma unroll
    for (int x = 0; x < F; ++x) y[x] = fmaf(o_lds[v][col][d0 + x], f, y[x]);
  }
  const int head = kvh * G + col % G;
  if (chunks > 1) {
    const int64_t place = (((int64_t)b * kv + kvh) * a.cols + col) * a.max_chunks + chunk;
#pragma unroll
    for (int x = 0; x < F; ++x) a.part[place * D + d0 + x] = y[x];
    if (d0 == 0) { a.part_ml[2 * place] = top; a.part_ml[2 * place + 1] = total; }
  } else {
    const int64_t row = (int64_t)b * a.tokens + col / G;
    Out* out = static_cast<Out*>(a.out) + row * a.out_row + head * D + d0;
#pragma unroll
    for (int x = 0; x < F; ++x) out[x] = (Out)(total == 0.f ? 0.f : y[x] / total);
    if (a.lse && d0 == 0) a.lse[row * a.heads + head] = (top + __builtin_amdgcn_logf(total)) * LN2;
  }
}

// Adds up the chunks of a column, 16 bytes a lane: D / 4 lanes hold an output.  Up to join_one chunks are added one after the other by
// the same lanes (64 queries of 32 sequences of 501..4000 tokens, 12 heads of 64: 5.8 us; 11.2 with a wave a column); more by the lanes
// of four waves, so many chunks at a time.  Which, goes by the sequence's own length.
template <int D>
struct PagedJoin {
  static constexpr int LANES = D / 4, SETS = 64 / LANES;         // chunks that a wave's load covers
  f32x4 y = f32x4{};
  float top = -INFINITY, total = 0.f;
  __device__ __forceinline__ void few(const PagedArgs& a, int64_t at, int chunks, int lane) {
    const f32x2* ml = reinterpret_cast<const f32x2*>(a.part_ml) + at;
    const float* p = a.part + at * D + lane * 4;
    for (int n = 0; n < chunks; n += 4) {
      f32x2 w[4];
      f32x4 v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int c = min(n + u, chunks - 1);
        w[u] = ml[c];
        v[u] = *reinterpret_cast<const f32x4*>(p + (int64_t)c * D);
      }
      float to = top;
#pragma unroll
      for (int u = 0; u < 4; ++u) to = fmaxf(to, w[u][0]);
      const float sub = to == -INFINITY ? 0.f : to, by = __builtin_amdgcn_exp2f(top - sub);
      total *= by;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] *= by;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (n + u >= chunks) break;
        const float f = __builtin_amdgcn_exp2f(w[u][0] - sub);
        total = fmaf(w[u][1], f, total);
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = fmaf(v[u][e], f, y[e]);
      }
      top = to;
    }
  }
  // every SETS * 4-th of many chunks
  __device__ __forceinline__ void many(const PagedArgs& a, int64_t at, int chunks, int wave, int lane) {
    const float* ml = a.part_ml + 2 * at;
    for (int n = lane; n < chunks; n += 64) top = fmaxf(top, ml[2 * n]);
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor(top, s));
    const float sub = top == -INFINITY ? 0.f : top;
    const float* p = a.part + at * D + (lane % LANES) * 4;
#pragma unroll 4
    for (int n = wave * SETS + lane / LANES; n < chunks; n += 4 * SETS) {
      const float f = __builtin_amdgcn_exp2f(ml[2 * n] - sub);
      const f32x4 v = *reinterpret_cast<const f32x4*>(p + (int64_t)n * D);
      total = fmaf(ml[2 * n + 1], f, total);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = fmaf(v[e], f, y[e]);
    }
#pragma unroll
    for (int s = 32; s >= LANES; s >>= 1) {
      total += __shfl_xor(total, s);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] += __shfl_xor(y[e], s);
    }
  }
  template <typename Out>
  __device__ __forceinline__ void out(const PagedArgs& a, int b, int kvh, int col, int lane) const {
    const int G = a.heads / a.cache.kv_heads, head = kvh * G + col % G;
    const int64_t row = (int64_t)b * a.tokens + col / G;
    Out* to = static_cast<Out*>(a.out) + row * a.out_row + head * D + lane * 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) to[e] = (Out)(total == 0.f ? 0.f : y[e] / total);
    if (a.lse && lane == 0) a.lse[row * a.heads + head] = (top + __builtin_amdgcn_logf(total)) * LN2;
  }
};

// FEW: no sequence of the call can have more than join_one chunks; a workgroup takes as many columns as it has lanes for.  Otherwise
// one column.
template <int D, typename Out, bool FEW>
__global__ __launch_bounds__(256) void k_paged_join(PagedArgs a) {
  typedef PagedJoin<D> Join;
  const int kv = a.cache.kv_heads, lane = threadIdx.x % Join::LANES;
  const int64_t column = FEW ? (int64_t)blockIdx.x * join_columns(D) + threadIdx.x / Join::LANES : blockIdx.x;
  if (column >= (int64_t)a.B * kv * a.cols) return;
  const int col = (int)(column % a.cols), bk = (int)(column / a.cols), b = bk / kv;
  const int chunks = chunks_of(paged_len(a, b), a.cols, a.fp32);
  if (chunks <= 1) return;
  const int64_t at = column * a.max_chunks;
  Join j;
  if (FEW || chunks <= join_one(a.cols)) {
    if (!FEW && threadIdx.x >= Join::LANES) return;
    j.few(a, at, chunks, lane);
  } else {
    __shared__ __align__(16) float lds[4][D + 4];
    const int wave = threadIdx.x >> 6;
    j.many(a, at, chunks, wave, threadIdx.x & 63);
    if ((threadIdx.x & 63) < Join::LANES) *reinterpret_cast<f32x4*>(&lds[wave][4 * lane]) = j.y;
    if ((threadIdx.x & 63) == 0) lds[wave][D] = j.total;
    __syncthreads();
    if (threadIdx.x >= Join::LANES) return;
    j.y = f32x4{}; j.total = 0.f;
    for (int w = 0; w < 4; ++w) {
      j.total += lds[w][D];
      j.y += *reinterpret_cast<const f32x4*>(&lds[w][4 * lane]);
    }
  }
  j.template out<Out>(a, b, bk % kv, col, lane);
}

}  // namespace tsdp
