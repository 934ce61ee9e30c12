// Rules of attention and of the key / value cache that host and device share: which sequence a packed row belongs to,
// where a token lies in the pages, how a length is split into chunks.  Plain C++: the CPU tests compile this file alone.
#pragma once
#include <stdint.h>
#include <initializer_list>

#ifdef __HIPCC__
#define TSDP_HD __host__ __device__ __forceinline__
#else
#define TSDP_HD inline
#endif

namespace tsdp {

constexpr int MX_BLOCK = 32;                 // elements that share a scale in the 8-bit cache
constexpr int MIN_PAGE_SHIFT = 4, MAX_PAGE_SHIFT = 12;

struct CacheView {                           // tsdp_kv_cache, checked
  void* k; void* v; uint8_t* k_scale; uint8_t* v_scale;
  const int32_t* table;                      // [B][columns]
  int32_t pages, columns, kv_heads, page_shift;
};

// Page of column `col` of environment b, -1 where the column or the table's entry lies outside (nothing is read through
// such an entry).
TSDP_HD int page_of(const CacheView& c, int b, long col) {
  if (col < 0 || col >= c.columns) return -1;
  const int32_t p = c.table[(long)b * c.columns + col];
  return p < 0 || p >= c.pages ? -1 : p;
}

// Row of `token` (its place in the page) of a head in the pools, counted in rows of head_dim elements: past 32 bits in
// a long cache.
TSDP_HD int64_t pool_row(const CacheView& c, int page, int head, int token) {
  return ((((int64_t)page * c.kv_heads + head) << c.page_shift) + token);
}

// Live rows b .. of a packed table: [lo, hi) clipped to 0 .. cap; an entry that points backwards owns no rows.
TSDP_HD void rows_of(const int32_t* ptr, int b, int cap, int& lo, int& hi) {
  lo = ptr[b]; hi = ptr[b + 1];
  if (lo < 0 || lo > cap) { lo = 0; hi = 0; }
  if (hi > cap) hi = cap;
  if (hi < lo) hi = lo;
}

// Keys that query i of nq sees of nk: all, or (causal) those up to its own place, the last query at the last key.
TSDP_HD int seen(int i, int nq, int nk, bool causal) {
  if (!causal) return nk;
  const long n = (long)nk - nq + 1 + i;
  return n < 0 ? 0 : n > nk ? nk : (int)n;
}

// Chunk of a sequence that one workgroup of the paged kernel takes, from the sequence's own length and the columns
// (queries x heads of a group) and type alone, so that a result does not depend on the batch around it.  Short chunks spread one short
// sequence over the chip (700 keys in fp32, 8 heads of 64: 8.0 us in chunks of 256, 11.2 in chunks of 512, without the join);
// long ones leave fewer partial results (16 sequences of 4096, 32 / 8 heads of 128 in 8 bits, the call: 29.8 us in chunks of
// 512, 34.2 in chunks of 256).  Many columns take longer for a key, with queries in fp32 twice as long again (32 sequences of 8000,
// 64 queries, 12 / 4 heads of 64 in 8 bits: 157 us in chunks of 1024, 178 in chunks of 512; in fp32, 32 of 1000, 12 / 3 heads of 64:
// 56.1 in chunks of 512, 67.4 in one of 1024; 32 of 4000: 203 in both; 32 of 4000 with 8 bits held: 103 and 94, 5 of 3000: 26.7 and 29.6).
TSDP_HD int chunk_shift(int len, int cols, bool fp32 = false) {
  int s = cols <= 16 ? 8 : fp32 ? 9 : 10;
  if (len > (1 << 10) && s < 9) s = 9;
  if (len > (1 << 14) && s < 10) s = 10;
  if (len > (1 << 16) && cols <= 16) s = 11;
  return s;
}
TSDP_HD int chunks_of(int len, int cols, bool fp32 = false) {
  const int s = chunk_shift(len, cols, fp32);
  return (int)(((long)len + (1L << s) - 1) >> s);
}
// the most chunks that a length of at most max_len has
inline int most_chunks(int max_len, int cols, bool fp32 = false) {
  int n = chunks_of(max_len, cols, fp32);
  for (int at : {1 << 10, 1 << 14, 1 << 16})     // where chunks grow
    if (max_len > at && chunks_of(at, cols, fp32) > n) n = chunks_of(at, cols, fp32);
  return n;
}

// Chunks that the same lanes add up one after the other; more are dealt to the lanes of a workgroup.  Few columns leave the chip
// idle meanwhile (64 sequences of 8000 tokens, 8 / 2 heads of 64, the call: 44.7 us with 4 chunks at most, 49.0 with 16), many do
// not (64 queries of 32 sequences of 8000, 12 / 4 heads of 64: 156 us with 16, 180 with 4).
TSDP_HD constexpr int join_one(int cols) { return cols <= 16 ? 4 : 16; }
TSDP_HD constexpr int join_columns(int head_dim) { return 256 / (head_dim / 4); }   // columns of a workgroup of such lanes

// Workgroups of the launches of a call: rows of the cache, queries of a prompt, the larger of the two over the cache.
inline int rows_per_wave(int kv_heads, int head_dim) {           // as many as 64 lanes of 8 elements hold, one at least
  const int n = 64 / (2 * kv_heads * (head_dim / 8));
  return n > 1 ? n : 1;
}
inline int64_t cache_blocks(int64_t rows, int kv_heads, int head_dim) {
  const int64_t n = 4 * rows_per_wave(kv_heads, head_dim);
  return (rows + n - 1) / n;
}
inline int64_t prompt_slots(int64_t rows, int group, int64_t B, int tq) { return rows * group / tq + B; }   // columns: rows x heads of a group
inline int64_t paged_blocks(int64_t bk, int cols) { return cols <= 16 ? bk : bk * ((cols + 63) / 64); }
inline int64_t join_blocks(int64_t bk, int cols, int chunks, int head_dim) {
  const int64_t columns = bk * cols, per = join_columns(head_dim);
  return chunks <= 1 ? 0 : chunks <= join_one(cols) ? (columns + per - 1) / per : columns;
}

}  // namespace tsdp
