// Attention of whole prompts: packed sequences, grouped heads, causal (aligned at the last key) or not.
//
//   o_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(scale <q_i, k_j> - m_i) over the keys that query i sees
//
// One pass over the keys with a running maximum m_i, sum and output (all fp32), so scores never leave the registers.  A wave
// owns 32 columns (a query of one head each); the waves of a workgroup share the tiles of keys and values in LDS.  Both products are taken
// transposed, S^T = K Q^T and O^T = V^T P^T: a lane then holds scores of one query only (column l % 32), so the softmax
// needs one exchange between the wave's halves per tile, and the accumulator layout of S^T is the operand layout of P^T as it
// is, up to the order of the keys, which the value operand follows: P stays in registers.
//
// Measured: two prompts of 5003..8192 tokens, 32 / 8 heads of 128, 880 us = 1.08 PFLOP/s (a large library product: 1.19 to 1.36; the
// matrix pipe is busy 55 % of the time, the exponentials and their conversion fill the vector pipe meanwhile); 16 chunks of
// 65..257 queries behind 2000 tokens, 16 / 4 heads of 128, 63 us = 0.71 PFLOP/s (few workgroups, of unequal length); 256 prompts of 1..191
// tokens, 8 heads of 64, 36 us = 2.8 TB/s (each is a chain of look-up, loads, two to three tiles and stores).
#pragma once
#include "attend_common.hpp"

namespace tsdp {

struct PromptArgs {
  int B, q_cap, k_cap, heads, kv_heads, group, causal;         // group = heads / kv_heads
  float c;                                   // scale * log2 e: exponentials are powers of two
  const int32_t* q_ptr; const int32_t* k_ptr;
  const void* q; const void* k; const void* v; void* out;
  int64_t q_row, k_row, v_row, out_row;      // elements from one row to the next
  float* lse;                                // [q_cap][heads] or null
  int slots;                                 // tiles of columns that the row bound allows
  int32_t* status;
};

// (most calls have no group: the division takes 1 of 37 us of 256 short prompts)
__device__ __forceinline__ int query_of(int column, int group) { return group == 1 ? column : column / group; }

// The tile of a workgroup: TQ columns of one kv head, a column being a query of one of the heads that share its keys (heads of a query
// next to each other), so that short sequences fill it with all of them (180 prompts of 5 tokens, 32 / 4 heads of 128: 16.3 us in
// bf16, 64.4 with a workgroup a head; in fp32 35.3 and 161; 32 of 300, 32 / 8 heads of 128 in bf16: 67.7 and 82.7).  With G heads in
// a group, sequence b owns the slots from G q_ptr[b] / TQ + b on, which no other does since floor(x) + ceil(n) <= floor(x + n) + 1.
// Late tiles of late sequences come first: causal ones have the most keys.
struct PromptTile { int b, kv_head, q_lo, nq, i0, columns, k_lo, nk; };
template <int TQ>
__device__ __forceinline__ bool prompt_tile(const PromptArgs& a, PromptTile& t) {
  // neighbours in the order of the kv heads: tiles of the same keys share an XCD's L2
  const int slot = a.slots - 1 - (int)(blockIdx.x / a.kv_heads);
  t.kv_head = blockIdx.x % a.kv_heads;
  t.b = count_upto(a.B, slot, [&](int i) { return min(max(a.q_ptr[i], 0), a.q_cap) * a.group / TQ + i; });
  if (t.b >= a.B) return false;
  int hi;
  rows_of(a.q_ptr, t.b, a.q_cap, t.q_lo, hi);
  if (a.q_ptr[t.b + 1] > a.q_cap && threadIdx.x == 0) report(a.status, STATUS_ROWS);
  t.nq = hi - t.q_lo;
  t.columns = t.nq * a.group;
  t.i0 = (slot - (t.q_lo * a.group / TQ + t.b)) * TQ;
  if (t.i0 < 0 || t.i0 >= t.columns) return false;
  rows_of(a.k_ptr, t.b, a.k_cap, t.k_lo, hi);
  if (a.k_ptr[t.b + 1] > a.k_cap && threadIdx.x == 0) report(a.status, STATUS_ROWS);
  t.nk = hi - t.k_lo;
  return true;
}

template <int NW>
__device__ __forceinline__ bool any_of(const uint32_t* flags) {
  uint32_t f = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) f |= flags[w];
  return __builtin_amdgcn_readfirstlane(f) != 0;
}

// 16 bytes a lane from global memory into LDS: lane l of the wave lands at lds + 16 l.
__device__ __forceinline__ void to_lds(const void* g, void* lds) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)g, (__attribute__((address_space(3))) void*)lds, 16, 0, 0);
}

// Rows of both tiles are CH chunks of 16 bytes in LDS.  A key operand is read by 16 rows at one chunk at a time, a value
// operand by 4 rows at 64 bytes: chunks are stored where these fall into different banks (64 banks of 4 bytes).
template <int CH> __device__ __forceinline__ int key_swizzle(int row) { return CH >= 16 ? row & 15 : CH == 8 ? (row >> 1) & 7 : (row >> 2) & 3; }
template <int CH> __device__ __forceinline__ int value_swizzle(int row) { return CH >= 16 ? (row & 3) << 2 : CH == 8 ? ((row >> 1) & 1) << 2 : 0; }

// Until all of this wave's loads into LDS have landed.  (The builtin: the compiler counts with it.)
__device__ __forceinline__ void wait_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0F70);        // vmcnt(0)
  asm volatile("" ::: "memory");
}

// bf16.  A wave owns 32 columns.  Keys go by 32 (half a tile) through three stages that do not depend on each other and are
// issued into each other: scores of the next 32 keys (matrix pipe), softmax of these (vector pipe), product of the last 32
// with their values (matrix pipe).  Key tiles are two buffers, and so are value tiles, a tile behind: one barrier a tile, in
// its middle, where the tiles requested at the last one have landed and the oldest buffers are free again.  Each buffer is a
// variable of its own, so that the compiler sees that reads of one need not wait for loads into another.
// Tiles that are masked for some query of the workgroup come last and go through the stages one by one -- and so does
// everything, once more, where a maximum would have had to move on the way, which the overlapped loop only notices.
// A weight of zero does not hide a value that is not finite from a matrix product.  Where some query does not see all of a
// tile, such values are therefore zeroed in LDS by the wave that loaded them and noted in a bitmap (a byte for 8 dims), from which each
// query that sees them collects the outputs that become NaN.
template <int D, int NW>
struct PromptBf16 {
  static constexpr int KT = 64, CH = D / 8, DT = D / 32, TILE_B = KT * D * 2, ROUNDS = KT * CH / (NW * 64);
  static constexpr int RPR = NW * 64 / CH;   // rows a round of loads
  static constexpr int TQ = 32 * NW;
  static_assert(ROUNDS >= 1 && KT * CH % (NW * 64) == 0 && RPR % 16 == 0, "a tile is whole rounds of the workgroup's loads, swizzled alike");

  f32x16 o[DT];
  bf16x8 q[D / 16];
  float m, l;

  static __device__ __forceinline__ bf16x8 key(const uint8_t* tile, int row, int chunk) {
    return *reinterpret_cast<const bf16x8*>(tile + row * (D * 2) + ((chunk ^ key_swizzle<CH>(row)) << 4));
  }
  // values of 8 keys as a transposed operand: lane l gets dim 32 d + l % 32 of keys 16 x + 4 h + {0..3, 8..11} of the 32 keys
  // from row0 on (h = l / 32).  One read turns 4 keys x 16 dims for 16 lanes, each of which names 4 dims of one key.
  static __device__ __forceinline__ u32x4 values(const uint8_t* tile, int row0, int x, int d, int lane) {
    typedef __attribute__((ext_vector_type(4))) short s16x4;
    typedef __attribute__((address_space(3))) s16x4* at;
    const int row = row0 + 16 * x + 4 * (lane >> 5) + ((lane & 15) >> 2), dim = 32 * d + ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
    const uint8_t* p = tile + row * (D * 2) + (((dim >> 3) ^ value_swizzle<CH>(row)) << 4) + (dim & 7) * 2;
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)p));
    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)(p + 8 * (D * 2))));
    return u32x4{lo[0], lo[1], hi[0], hi[1]};
  }

  __device__ __forceinline__ f32x16 scores(const uint8_t* kt, int row0, int lane) const {
    f32x16 s = f32x16{};
#pragma unroll
    for (int x = 0; x < D / 16; ++x) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key(kt, row0 + (lane & 31), 2 * x + (lane >> 5)), q[x], s, 0, 0, 0);
    return s;
  }

  // f: what sums and outputs so far have to be scaled by
  __device__ __forceinline__ bool maximum(const f32x16& s, float c, float& f) {
    float top = -INFINITY;
#pragma unroll
    for (int x = 0; x < 16; x += 2) top = max3(top, s[x], s[x + 1]);
    top = max_halves(top) * c;
    const bool moves = top > m + MOST_RISE;
    const float to = moves ? top : m;
    f = moves ? __builtin_amdgcn_exp2f(m - to) : 1.f;
    l *= f;
    m = to;
    return moves;
  }
  // weight of the key of register x
  __device__ __forceinline__ void weight(const f32x16& s, float c, float sub, int x, bf16x8 (&p)[2]) {
    const float e = __builtin_amdgcn_exp2f(fmaf(s[x], c, -sub));
    l += e;
    p[x / 8][x % 8] = (__bf16)e;             // rounded for the matrix cores: by at most 2^-8 of each weight
  }
  __device__ __forceinline__ float subtrahend() const { return m == -INFINITY ? 0.f : m; }

  __device__ __forceinline__ void scale(float f) {
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int x = 0; x < 16; ++x) o[d][x] *= f;
  }

  __device__ __forceinline__ void product(const bf16x8 (&p)[2], const uint8_t* vt, int row0, int lane) {
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int d = 0; d < DT; ++d)
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, values(vt, row0, x, d, lane)), p[x], o[d], 0, 0, 0);
  }

  // The three stages of 32 keys, step by step: `next` = scores of the keys at k_row of kt, weights of `s`, product of `last` with
  // the values at v_row of vt; as many steps of the one product as of the other, in turns, their operands read AHEAD steps
  // before -- those of the first steps by the call before (READY), where that is not on the other side of a barrier; MORE: the
  // next call continues at rows + 32 of the same tiles.
  static constexpr int KS = D / 16, STEPS = 2 * KS, AHEAD = 3, RING = AHEAD + 1;
  template <bool FIRST, bool LAST, bool READY, bool MORE>
  __device__ __forceinline__ void half_tile(bf16x8 (&ring)[RING], f32x16& next, const f32x16& s, bf16x8 (&p)[2], const bf16x8 (&last)[2], float c,
                                            const uint8_t* kt, int k_row, const uint8_t* vt, int v_row, int lane) {
    static_assert(STEPS % RING == 0 || !(READY || MORE), "the ring goes on from one call to the next");
    auto fetch = [&](int st) __attribute__((always_inline)) {
      const int more = st >= STEPS ? 32 : 0, x = (st % STEPS) / 2;
      if (more && !MORE) return;
      if (st % 2 == 0) {
        if (!LAST || more) ring[st % RING] = key(kt, k_row + more + (lane & 31), 2 * x + (lane >> 5));
      } else {
        if (!FIRST || more) ring[st % RING] = __builtin_bit_cast(bf16x8, values(vt, v_row + more, x / DT, x % DT, lane));
      }
    };
    const float sub = subtrahend();
    if (!READY) {
#pragma unroll
      for (int st = 0; st < AHEAD; ++st) fetch(st);
    }
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
      fetch(st + AHEAD);
#pragma unroll
      for (int x = st * 16 / STEPS; x < (st + 1) * 16 / STEPS; ++x) {
        weight(s, c, sub, x, p);
        asm volatile("" : "+v"(l));                                    // computed here, not where it is used
        if (x % 8 == 7) asm volatile("" : "+v"(p[x / 8]));
      }
      const int i = st / 2;
      if (st % 2 == 0) {
        if constexpr (!LAST) next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[st % RING], q[i], i == 0 ? f32x16{} : next, 0, 0, 0);
      } else {
        if constexpr (!FIRST) o[i % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[st % RING], last[i / DT], o[i % DT], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
};

// OVERLAP: with the overlapped loop, 2 waves a SIMD; without it (the same results, bit for bit) there is room for more waves to
// hide each other's loads, which pays where sequences are short.
template <int D, int NW, int WAVES, bool OVERLAP>
__global__ __launch_bounds__(NW * 64, WAVES) void k_prompt_bf16(PromptArgs a) {
  typedef PromptBf16<D, NW> C;
  constexpr int KT = C::KT, CH = C::CH;
  __shared__ __align__(16) uint8_t k0[C::TILE_B], k1[C::TILE_B], v0[C::TILE_B], v1[C::TILE_B];   // tiles of even and odd number
  __shared__ uint32_t unusual[NW];           // some value of a masked tile is not finite, as each wave has seen it
  __shared__ uint8_t where[2][KT * CH];      // which, a bit for each
  __shared__ uint32_t rises[NW];             // some maximum would have had to move in the overlapped loop
  PromptTile t;
  if (!prompt_tile<C::TQ>(a, t)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int i0 = t.i0 + wave * 32, i = i0 + col, G = a.group;  // the wave's first column, this lane's
  const int query = query_of(min(i, t.columns - 1), G), head = t.kv_head * G + min(i, t.columns - 1) - query * G;
  const auto sees = [&](int column) { return seen(query_of(column, G), t.nq, t.nk, a.causal); };
  // tiles that every column of the workgroup sees in full, and that some column sees
  const int full = OVERLAP ? sees(t.i0) / KT : 0;
  const int tiles = (sees(min(t.i0 + C::TQ, t.columns) - 1) + KT - 1) / KT;
  const int mine = i < t.columns ? seen(query, t.nq, t.nk, a.causal) : 0;                     // keys that this lane's column sees
  const int some = i0 < t.columns ? sees(min(i0 + 31, t.columns - 1)) : 0;                    // and that some column of the wave sees
  const int least = sees(i0);                // and that every column of it sees
  if (lane == 0) { unusual[wave] = 0; rises[wave] = 0; }

  const __bf16* kb = static_cast<const __bf16*>(a.k) + (int64_t)t.k_lo * a.k_row + t.kv_head * D;
  const __bf16* vb = static_cast<const __bf16*>(a.v) + (int64_t)t.k_lo * a.v_row + t.kv_head * D;
  const int sr = wave * (64 / CH) + lane / CH, pc = lane % CH;
  // this lane's bytes of the first round of a tile; rounds and tiles are whole rows further
  const uint32_t k_off = (uint32_t)(sr * (int)a.k_row + (pc ^ key_swizzle<CH>(sr)) * 8) * 2;
  const uint32_t v_off = (uint32_t)(sr * (int)a.v_row + (pc ^ value_swizzle<CH>(sr)) * 8) * 2;
  auto stage = [&](const __bf16* base, int64_t row, uint32_t off, int tile, uint8_t* to) __attribute__((always_inline)) {
    if (tile >= tiles) return;
    const char* at = reinterpret_cast<const char*>(base + (int64_t)tile * KT * row);
    const int left = t.nk - tile * KT;
    if (left >= KT) {
#pragma unroll
      for (int n = 0; n < C::ROUNDS; ++n) to_lds(at + (int64_t)n * C::RPR * row * 2 + off, to + (n * NW + wave) * 1024);
    } else {                                 // rows behind the sequence: its last one, masked
#pragma unroll 1
      for (int n = 0; n < C::ROUNDS; ++n) {
        const int over = max(n * C::RPR + sr - (left - 1), 0);
        to_lds(at + ((int64_t)n * C::RPR - over) * row * 2 + off, to + (n * NW + wave) * 1024);
      }
    }
  };
#define TSDP_KEYS(N, TO) stage(kb, a.k_row, k_off, N, TO)
#define TSDP_VALUES(N, TO) stage(vb, a.v_row, v_off, N, TO)
  TSDP_KEYS(0, k0);
  TSDP_KEYS(1, k1);
  TSDP_VALUES(0, v0);

  C w;
  const __bf16* q = static_cast<const __bf16*>(a.q) + (int64_t)(t.q_lo + query) * a.q_row + head * D;
#pragma unroll
  for (int x = 0; x < D / 16; ++x) w.q[x] = *reinterpret_cast<const bf16x8*>(q + 16 * x + 8 * half);
  auto clear = [&]() __attribute__((always_inline)) {
    w.m = -INFINITY; w.l = 0.f;
#pragma unroll
    for (int d = 0; d < C::DT; ++d) w.o[d] = f32x16{};
  };
  clear();

  int from = 0;                              // first tile of the plain loop
  if constexpr (OVERLAP) if (full > 0) {
    f32x16 s[2];
    bf16x8 p[2][2], ring[C::RING];
    float f;
    wait_loads();
    __syncthreads();
    // first and second half of a tile: K, V its buffers, KN the next tile's keys, VL the last one's values
#define TSDP_FIRST(FIRST, K, VL) w.template half_tile<FIRST, false, !(FIRST), false>(ring, s[1], s[0], p[0], p[1], a.c, K, 32, VL, 32, lane)
#define TSDP_SECOND(LAST, KN, V) w.template half_tile<false, LAST, false, !(LAST)>(ring, s[0], s[1], p[1], p[0], a.c, KN, 0, V, 0, lane)
    // between them, in tile N with keys in K and the other buffer of values VN
#define TSDP_MIDDLE(N, K, VN)                                                                                     \
  do {                                                                                                            \
    wait_loads();                                                                                                 \
    __syncthreads();                                                                                              \
    TSDP_KEYS((N) + 2, K);                                                                                        \
    TSDP_VALUES((N) + 1, VN);                                                                                     \
  } while (0)
    if (some == 0) {                         // a wave behind the last query only loads
      for (int n = 0; n < full; n += 2) {
        TSDP_MIDDLE(n, k0, v1);
        if (n + 1 < full) TSDP_MIDDLE(n + 1, k1, v0);
      }
    } else {
    s[0] = w.scores(k0, 0, lane);
    w.maximum(s[0], a.c, f);
    TSDP_FIRST(true, k0, v1);
    TSDP_MIDDLE(0, k0, v1);
    int n = 0;
    while (n + 1 < full) {
      TSDP_SECOND(false, k1, v0);
      TSDP_FIRST(false, k1, v0);
      TSDP_MIDDLE(n + 1, k1, v0);
      if (++n + 1 >= full) break;
      TSDP_SECOND(false, k0, v1);
      TSDP_FIRST(false, k0, v1);
      TSDP_MIDDLE(n + 1, k0, v1);
      ++n;
    }
    if (n & 1) {
      TSDP_SECOND(true, k0, v1);
      w.product(p[1], v1, 32, lane);
    } else {
      TSDP_SECOND(true, k1, v0);
      w.product(p[1], v0, 32, lane);
    }
    }
#undef TSDP_FIRST
#undef TSDP_SECOND
#undef TSDP_MIDDLE
    if (some > 0 && __any(w.l > most_sum(w.m)) && lane == 0) rises[wave] = 1;
    __syncthreads();
    from = full;
    if (any_of<NW>(rises)) {                 // once more from the start
      from = 0;
      wait_loads();
      __syncthreads();                       // nobody's loads land behind the new ones
      TSDP_KEYS(0, k0);
      TSDP_KEYS(1, k1);
      TSDP_VALUES(0, v0);
      clear();
    }
  }
  uint32_t gone[C::DT];                      // outputs that a visible value makes NaN: bit 8 j + e of word d is o[d][4 j + e]
#pragma unroll
  for (int d = 0; d < C::DT; ++d) gone[d] = 0;
  auto plain = [&](int n, uint8_t* k, uint8_t* kn, uint8_t* v, uint8_t* vn) __attribute__((always_inline)) {
    wait_loads();
    bool bad = false;
#pragma unroll
    for (int x = 0; x < C::ROUNDS; ++x) {
      u32x4* at = reinterpret_cast<u32x4*>(v + (x * NW + wave) * 1024 + lane * 16);
      u32x4 y = *at;
      uint32_t marks = 0;
      if (__any(some_not_finite(y))) {
        bad = true;
#pragma unroll
        for (int z = 0; z < 4; ++z) marks |= not_finite_halves(y[z]) << (2 * z);
        if (marks) {
#pragma unroll
          for (int z = 0; z < 4; ++z) y[z] = finite_bf16(y[z]);
          *at = y;
        }
      }
      where[n & 1][(x * C::RPR + sr) * CH + (pc ^ value_swizzle<CH>(sr))] = (uint8_t)marks;
    }
    if (bad && lane == 0) unusual[wave] = 1;
    __syncthreads();
    if (n > from) TSDP_KEYS(n + 1, kn);
    TSDP_VALUES(n + 1, vn);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int left = mine - (n * KT + 32 * u);
      if (n * KT + 32 * u >= some) continue;
      f32x16 s = w.scores(k, 32 * u, lane);
      bf16x8 p[2];
      if (n * KT + 32 * u + 32 > least) {
#pragma unroll
        for (int x = 0; x < 16; ++x)
          if (8 * (x / 4) + 4 * half + x % 4 >= left) s[x] = -INFINITY;
      }
      float f;
      if (__any(w.maximum(s, a.c, f))) w.scale(f);
      const float sub = w.subtrahend();
#pragma unroll
      for (int x = 0; x < 16; ++x) w.weight(s, a.c, sub, x, p);
      w.product(p, v, 32 * u, lane);
    }
    if (any_of<NW>(unusual)) {
      const int left = min(mine - n * KT, KT);
#pragma unroll 1
      for (int j = 0; j < left; ++j)
#pragma unroll
        for (int d = 0; d < C::DT; ++d) gone[d] |= *reinterpret_cast<const uint32_t*>(&where[n & 1][j * CH + 4 * d]) >> (4 * half) & 0x0F0F0F0Fu;
    }
  };
  for (int n = from; n < tiles; ++n) {
    if (n & 1) plain(n, k1, k0, v1, v0);
    else plain(n, k0, k1, v0, v1);
  }
#undef TSDP_KEYS
#undef TSDP_VALUES
  const float l = sum_halves(w.l);
  const float r = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;      // no key seen: zeros; NaN stays
  __bf16* out = static_cast<__bf16*>(a.out) + (int64_t)(t.q_lo + query) * a.out_row + head * D + 8 * half;
#pragma unroll
  for (int d = 0; d < C::DT; ++d)
#pragma unroll
    for (int x = 0; x < 4; x += 2) {         // the halves of the wave hold dims 0..3 and 4..7 of each eight: one takes all of the first
      u32x2 y[2];                            // eight, the other of the second
#pragma unroll
      for (int z = 0; z < 2; ++z)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int at = 4 * (x + z) + 2 * e, bit = 8 * (x + z) + 2 * e;
          const float lo = gone[d] >> bit & 1 ? NAN : w.o[d][at] * r, hi = gone[d] >> (bit + 1) & 1 ? NAN : w.o[d][at + 1] * r;
          y[z][e] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)lo, (__bf16)hi});
        }
      const auto s0 = __builtin_amdgcn_permlane32_swap(y[0][0], y[1][0], false, false);
      const auto s1 = __builtin_amdgcn_permlane32_swap(y[0][1], y[1][1], false, false);
      if (i < t.columns) *reinterpret_cast<u32x4*>(out + 32 * d + 8 * x) = u32x4{s0[0], s1[0], s0[1], s1[1]};
    }
  if (a.lse && half == 0 && i < t.columns) a.lse[(int64_t)(t.q_lo + query) * a.heads + head] = (w.m + __builtin_amdgcn_logf(l)) * LN2;
}

}  // namespace tsdp
