// Attention of whole prompts: packed sequences, grouped heads, causal (aligned at the last key) or not.
//
//   o_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(scale <q_i, k_j> - m_i) over the keys that query i sees
//
// One pass over the keys with a running maximum m_i, sum and output (all fp32), so scores never leave the registers.  A wave
// owns 32 queries of one head; the waves of a workgroup share the tiles of keys and values in LDS.  Both products are taken
// transposed, S^T = K Q^T and O^T = V^T P^T: a lane then holds scores of one query only (column l % 32), so the softmax
// needs one exchange between the wave's halves per tile, and the accumulator layout of S^T is the operand layout of P^T as it
// is, up to the order of the keys, which the value operand follows: P stays in registers.
#pragma once
#include "attend_common.hpp"

namespace tsdp {

struct PromptArgs {
  int B, q_cap, k_cap, heads, kv_heads, causal;
  float c;                                   // scale * log2 e: exponentials are powers of two
  const int32_t* q_ptr; const int32_t* k_ptr;
  const void* q; const void* k; const void* v; void* out;
  int64_t q_row, k_row, v_row, out_row;      // elements from one row to the next
  float* lse;                                // [q_cap][heads] or null
  int slots;                                 // tiles of queries that the row bound allows
  int32_t* status;
};

// The tile of queries of a workgroup: sequence b owns the slots from q_ptr[b] / TQ + b on, which no other does since
// floor(x) + ceil(n) <= floor(x + n) + 1.  Late tiles of late sequences come first: causal ones have the most keys.
struct PromptTile { int b, head, kv_head, q_lo, nq, i0, k_lo, nk; };
template <int TQ>
__device__ __forceinline__ bool prompt_tile(const PromptArgs& a, PromptTile& t) {
  // heads of one group of queries read the same keys: neighbours in the order of the kv heads share an XCD's L2
  const int h = blockIdx.x % a.heads, slot = a.slots - 1 - (int)(blockIdx.x / a.heads);
  t.kv_head = h % a.kv_heads;
  t.head = t.kv_head * (a.heads / a.kv_heads) + h / a.kv_heads;
  t.b = count_upto(a.B, slot, [&](int i) { return max(a.q_ptr[i], 0) / TQ + i; });
  if (t.b >= a.B) return false;
  int hi;
  rows_of(a.q_ptr, t.b, a.q_cap, t.q_lo, hi);
  if (a.q_ptr[t.b + 1] > a.q_cap && threadIdx.x == 0) report(a.status, STATUS_ROWS);
  t.nq = hi - t.q_lo;
  t.i0 = (slot - (t.q_lo / TQ + t.b)) * TQ;
  if (t.i0 < 0 || t.i0 >= t.nq) return false;
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

template <int D, int NW>
struct PromptBf16 {
  static constexpr int KT = 64, CH = D / 8, TILE_B = KT * D * 2, ROUNDS = KT * CH / (NW * 64);
  static constexpr int RPR = NW * 64 / CH;   // rows a round of loads
  static_assert(ROUNDS >= 1 && KT * CH % (NW * 64) == 0, "a tile is whole rounds of the workgroup's loads");

  static __device__ __forceinline__ bf16x8 read_key(const uint8_t* tile, int row, int chunk) {
    return *reinterpret_cast<const bf16x8*>(tile + row * (D * 2) + ((chunk ^ key_swizzle<CH>(row)) << 4));
  }
  // values of keys row .. row + 3 (row: of this lane's quarter) as a transposed operand of 4 keys: lane l gets dim l % 16
  // of its group's 16 dims
  static __device__ __forceinline__ u32x2 read_value(const uint8_t* tile, int row, int dim) {
    const int chunk = dim >> 3;
    const uint8_t* p = tile + row * (D * 2) + ((chunk ^ value_swizzle<CH>(row)) << 4) + (dim & 7) * 2;
    typedef __attribute__((ext_vector_type(4))) short s16x4;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p));
  }
};

template <int D, int NW>
__global__ __launch_bounds__(NW * 64) void k_prompt_bf16(PromptArgs a) {
  typedef PromptBf16<D, NW> C;
  constexpr int KT = C::KT, CH = C::CH, DT = D / 32, TQ = 32 * NW;
  __shared__ __align__(16) uint8_t lds[2][2][C::TILE_B];
  __shared__ uint32_t unusual[NW];           // some value of a masked tile is not finite, as each wave has seen it
  PromptTile t;
  if (!prompt_tile<TQ>(a, t)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int i0 = t.i0 + wave * 32, i = i0 + col;               // this lane's query
  const int mine = i < t.nq ? seen(i, t.nq, t.nk, a.causal) : 0;
  // keys that all / some queries of the wave see, and that some / all of the workgroup see
  const int all = i0 >= t.nq ? 0 : seen(i0, t.nq, t.nk, a.causal);
  const int some = i0 >= t.nq ? 0 : seen(min(i0 + 31, t.nq - 1), t.nq, t.nk, a.causal);
  const int last = seen(min(t.i0 + TQ, t.nq) - 1, t.nq, t.nk, a.causal);
  const int first = seen(t.i0, t.nq, t.nk, a.causal);
  const int tiles = (last + KT - 1) / KT;
  if (lane == 0) unusual[wave] = 0;

  const __bf16* q = static_cast<const __bf16*>(a.q) + (int64_t)(t.q_lo + min(i, t.nq - 1)) * a.q_row + t.head * D;
  bf16x8 qf[D / 16];
#pragma unroll
  for (int s = 0; s < D / 16; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(q + 16 * s + 8 * half);

  const __bf16* kb = static_cast<const __bf16*>(a.k) + (int64_t)t.k_lo * a.k_row + t.kv_head * D;
  const __bf16* vb = static_cast<const __bf16*>(a.v) + (int64_t)t.k_lo * a.v_row + t.kv_head * D;
  const int sr = wave * (64 / CH) + lane / CH, pc = lane % CH;
  auto stage = [&](int tile, int buf) {
#pragma unroll
    for (int n = 0; n < C::ROUNDS; ++n) {
      const int r = n * C::RPR + sr;
      const int64_t row = min(tile * KT + r, t.nk - 1);        // rows behind the sequence: its last one, masked
      uint8_t* at = &lds[buf][0][0] + (n * NW + wave) * 1024;
      to_lds(kb + row * a.k_row + (pc ^ key_swizzle<CH>(r)) * 8, at);
      to_lds(vb + row * a.v_row + (pc ^ value_swizzle<CH>(r)) * 8, at + C::TILE_B);
    }
  };

  f32x16 o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) o[d] = f32x16{};
  float m = -INFINITY, l = 0.f;
  if (tiles > 0) stage(0, 0);
  for (int n = 0; n < tiles; ++n) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    const uint8_t* kt = &lds[n & 1][0][0];
    const uint8_t* vt = kt + C::TILE_B;
    if ((n + 1) * KT > first) {              // masked for some wave: what this wave has loaded of the values is looked at
      bool bad = false;
#pragma unroll
      for (int x = 0; x < C::ROUNDS; ++x) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(vt + (x * NW + wave) * 1024 + lane * 16);
#pragma unroll
        for (int y = 0; y < 4; ++y) bad |= not_finite_bf16(w[y]);
      }
      if (__ballot(bad) && lane == 0) unusual[wave] = 1;
    }
    __syncthreads();                         // the tile is there for all, and the other buffer read by all
    if (n + 1 < tiles) stage(n + 1, (n + 1) & 1);
    if (n * KT >= some) continue;
    f32x16 s[2] = {f32x16{}, f32x16{}};
#pragma unroll
    for (int x = 0; x < D / 16; ++x)
#pragma unroll
      for (int u = 0; u < 2; ++u)
        s[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(C::read_key(kt, 32 * u + col, 2 * x + half), qf[x], s[u], 0, 0, 0);
    const bool masked = (n + 1) * KT > all;
    if (masked) {
      const int left = mine - n * KT;        // keys of the tile that this query sees
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int x = 0; x < 16; ++x)
          if (32 * u + 8 * (x / 4) + 4 * half + x % 4 >= left) s[u][x] = -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int x = 0; x < 16; ++x) top = fmaxf(top, s[u][x]);
    top = max_halves(top) * a.c;
    // the running maximum moves only where it would grow by more than 2^8: powers stay below 2^8, and sums far from overflow
    if (__any(top > m + 8.f)) {
      const float to = top > m + 8.f ? top : m, f = to == m ? 1.f : __builtin_amdgcn_exp2f(m - to);   // each query by its own scores
      m = to;
      l *= f;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int x = 0; x < 16; ++x) o[d][x] *= f;
    }
    const float sub = m == -INFINITY ? 0.f : m;
    bf16x8 p[4];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        const float e = __builtin_amdgcn_exp2f(fmaf(s[u][x], a.c, -sub));
        l += e;
        p[2 * u + x / 8][x % 8] = (__bf16)e;  // P rounded to bf16 for the matrix cores: at most 2^-8 of each weight
      }
    const int vrow = 4 * half + (lane & 15) / 4, vdim = ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
    if (masked && any_of<NW>(unusual)) {
      // values that are not finite are taken out of the product, and set the outputs of the queries that see them
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        f32x16 marks = f32x16{};
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const u32x2 lo = C::read_value(vt, 16 * x + vrow, 32 * d + vdim), hi = C::read_value(vt, 16 * x + 8 + vrow, 32 * d + vdim);
          const u32x4 w = {lo[0], lo[1], hi[0], hi[1]};
          u32x4 fin, mark;
#pragma unroll
          for (int y = 0; y < 4; ++y) { fin[y] = finite_bf16(w[y]); mark[y] = marks_bf16(w[y]); }
          bf16x8 sees;
#pragma unroll
          for (int y = 0; y < 8; ++y)
            sees[y] = (__bf16)(n * KT + 16 * x + 8 * (y / 4) + 4 * half + y % 4 < mine ? 1.f : 0.f);
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fin), p[x], o[d], 0, 0, 0);
          marks = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, mark), sees, marks, 0, 0, 0);
        }
#pragma unroll
        for (int x = 0; x < 16; ++x)
          if (marks[x] != 0.f) o[d][x] = NAN;
      }
    } else {
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const u32x2 lo = C::read_value(vt, 16 * x + vrow, 32 * d + vdim), hi = C::read_value(vt, 16 * x + 8 + vrow, 32 * d + vdim);
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]}), p[x], o[d], 0, 0, 0);
        }
    }
  }
  l = sum_halves(l);
  if (i >= t.nq) return;
  const float r = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;      // no key seen: zeros; NaN stays
  __bf16* out = static_cast<__bf16*>(a.out) + (int64_t)(t.q_lo + i) * a.out_row + t.head * D;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      bf16x4 y;
#pragma unroll
      for (int z = 0; z < 4; ++z) y[z] = (__bf16)(o[d][4 * x + z] * r);
      *reinterpret_cast<bf16x4*>(out + 32 * d + 8 * x + 4 * half) = y;
    }
  if (a.lse && half == 0) a.lse[(int64_t)(t.q_lo + i) * a.heads + t.head] = (m + __builtin_amdgcn_logf(l)) * LN2;
}

// fp32: the same walk with mfma_f32_32x32x2_f32.  A lane's 16-byte chunk of a key feeds four of them (MFMA j contracts dims
// 8 s + j and 8 s + 4 + j); the score register x feeds the value product at key 8 (x / 4) + 4 half + x % 4.
template <int D, int NW>
__global__ __launch_bounds__(NW * 64) void k_prompt_f32(PromptArgs a) {
  constexpr int KT = 32, CH = D / 4, DT = D / 32, TQ = 32 * NW, TILE = KT * D, ROUNDS = KT * CH / (NW * 64), RPR = NW * 64 / CH;
  static_assert(ROUNDS >= 1 && KT * CH % (NW * 64) == 0, "a tile is whole rounds of the workgroup's loads");
  __shared__ __align__(16) float lds[2][2][TILE];
  __shared__ uint32_t unusual[NW];
  PromptTile t;
  if (!prompt_tile<TQ>(a, t)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int i0 = t.i0 + wave * 32, i = i0 + col;
  const int mine = i < t.nq ? seen(i, t.nq, t.nk, a.causal) : 0;
  const int all = i0 >= t.nq ? 0 : seen(i0, t.nq, t.nk, a.causal);
  const int some = i0 >= t.nq ? 0 : seen(min(i0 + 31, t.nq - 1), t.nq, t.nk, a.causal);
  const int last = seen(min(t.i0 + TQ, t.nq) - 1, t.nq, t.nk, a.causal);
  const int first = seen(t.i0, t.nq, t.nk, a.causal);
  const int tiles = (last + KT - 1) / KT;
  if (lane == 0) unusual[wave] = 0;

  const float* q = static_cast<const float*>(a.q) + (int64_t)(t.q_lo + min(i, t.nq - 1)) * a.q_row + t.head * D;
  f32x4 qf[D / 8];
#pragma unroll
  for (int s = 0; s < D / 8; ++s) qf[s] = *reinterpret_cast<const f32x4*>(q + 8 * s + 4 * half);

  const float* kb = static_cast<const float*>(a.k) + (int64_t)t.k_lo * a.k_row + t.kv_head * D;
  const float* vb = static_cast<const float*>(a.v) + (int64_t)t.k_lo * a.v_row + t.kv_head * D;
  const int sr = wave * (64 / CH) + lane / CH, pc = lane % CH;
  auto stage = [&](int tile, int buf) {
#pragma unroll
    for (int n = 0; n < ROUNDS; ++n) {
      const int r = n * RPR + sr;
      const int64_t row = min(tile * KT + r, t.nk - 1);
      float* at = &lds[buf][0][0] + (n * NW + wave) * 256;
      to_lds(kb + row * a.k_row + (pc ^ key_swizzle<CH>(r)) * 4, at);
      to_lds(vb + row * a.v_row + pc * 4, at + TILE);
    }
  };

  f32x16 o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) o[d] = f32x16{};
  float m = -INFINITY, l = 0.f;
  if (tiles > 0) stage(0, 0);
  for (int n = 0; n < tiles; ++n) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    const float* kt = &lds[n & 1][0][0];
    const float* vt = kt + TILE;
    if ((n + 1) * KT > first) {
      bool bad = false;
#pragma unroll
      for (int x = 0; x < ROUNDS; ++x) {
        const f32x4 w = *reinterpret_cast<const f32x4*>(vt + (x * NW + wave) * 256 + lane * 4);
#pragma unroll
        for (int y = 0; y < 4; ++y) bad |= not_finite_f32(w[y]);
      }
      if (__ballot(bad) && lane == 0) unusual[wave] = 1;
    }
    __syncthreads();
    if (n + 1 < tiles) stage(n + 1, (n + 1) & 1);
    if (n * KT >= some) continue;
    f32x16 s = f32x16{};
#pragma unroll
    for (int x = 0; x < D / 8; ++x) {
      const f32x4 k = *reinterpret_cast<const f32x4*>(kt + col * D + (((2 * x + half) ^ key_swizzle<CH>(col)) << 2));
#pragma unroll
      for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_32x32x2f32(k[j], qf[x][j], s, 0, 0, 0);
    }
    const bool masked = (n + 1) * KT > all;
    if (masked) {
      const int left = mine - n * KT;
#pragma unroll
      for (int x = 0; x < 16; ++x)
        if (8 * (x / 4) + 4 * half + x % 4 >= left) s[x] = -INFINITY;
    }
    float top = s[0];
#pragma unroll
    for (int x = 1; x < 16; ++x) top = fmaxf(top, s[x]);
    top = max_halves(top) * a.c;
    if (__any(top > m + 8.f)) {
      const float to = top > m + 8.f ? top : m, f = to == m ? 1.f : __builtin_amdgcn_exp2f(m - to);   // each query by its own scores
      m = to;
      l *= f;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int x = 0; x < 16; ++x) o[d][x] *= f;
    }
    const float sub = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      s[x] = __builtin_amdgcn_exp2f(fmaf(s[x], a.c, -sub));
      l += s[x];
    }
    if (masked && any_of<NW>(unusual)) {
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        f32x16 marks = f32x16{};
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const int key = 8 * (x / 4) + 4 * half + x % 4;
          const float v = vt[key * D + 32 * d + col];
          const bool bad = not_finite_f32(v);
          o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(bad ? 0.f : v, s[x], o[d], 0, 0, 0);
          marks = __builtin_amdgcn_mfma_f32_32x32x2f32(bad ? 1.f : 0.f, n * KT + key < mine ? 1.f : 0.f, marks, 0, 0, 0);
        }
#pragma unroll
        for (int x = 0; x < 16; ++x)
          if (marks[x] != 0.f) o[d][x] = NAN;
      }
    } else {
#pragma unroll
      for (int x = 0; x < 16; ++x)
#pragma unroll
        for (int d = 0; d < DT; ++d)
          o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(vt[(8 * (x / 4) + 4 * half + x % 4) * D + 32 * d + col], s[x], o[d], 0, 0, 0);
    }
  }
  l = sum_halves(l);
  if (i >= t.nq) return;
  float* out = static_cast<float*>(a.out) + (int64_t)(t.q_lo + i) * a.out_row + t.head * D;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      f32x4 y;
#pragma unroll
      for (int z = 0; z < 4; ++z) y[z] = l == 0.f ? 0.f : o[d][4 * x + z] / l;
      *reinterpret_cast<f32x4*>(out + 32 * d + 8 * x + 4 * half) = y;
    }
  if (a.lse && half == 0) a.lse[(int64_t)(t.q_lo + i) * a.heads + t.head] = (m + __builtin_amdgcn_logf(l)) * LN2;
}

}  // namespace tsdp
