// Argument checks of the cache and attention entry points: plain C++, the CPU tests compile this file alone.
#pragma once
#include <stddef.h>
#include <stdint.h>
#include <cmath>
#include "../../include/tsdp.h"
#include "attend_plan.hpp"

namespace tsdp {

struct Fault { int code; const char* msg; };         // code TSDP_OK: none
constexpr Fault NO_FAULT{TSDP_OK, nullptr};

constexpr int64_t MOST_ROW = int64_t(1) << 24;       // elements from one row to the next
constexpr int MOST_HEADS = 1024, MOST_TOKENS = 1024, MOST_GRID_Y = 65535;
constexpr int64_t MOST_GRID = 0xFFFFFFFF / 512;       // workgroups: a launch has fewer than 2^32 threads, a workgroup up to 512
constexpr int MOST_LENGTH = 0x7FFFFF00;              // keys: whole tiles of them are counted in 32 bits

inline bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool head_dim_ok(int d) { return d == 32 || d == 64 || d == 128; }

inline Fault heads_fault(const tsdp_heads* h) {
  if (!h) return {TSDP_E_INVAL, "null heads"};
  if (h->type != 0 && h->type != 1) return {TSDP_E_INVAL, "heads: type must be 0 (fp32) or 1 (bf16)"};
  if (!head_dim_ok(h->head_dim)) return {TSDP_E_SHAPE, "heads: head_dim must be 32, 64 or 128"};
  if (h->kv_heads < 1 || h->q_heads < h->kv_heads || h->q_heads > MOST_HEADS || h->q_heads % h->kv_heads)
    return {TSDP_E_SHAPE, "heads: q_heads must be a multiple of kv_heads, at most 1024"};
  if (h->causal != 0 && h->causal != 1) return {TSDP_E_INVAL, "heads: causal must be 0 or 1"};
  if (!(h->scale > 0.f) || !std::isfinite(h->scale * 1.4426950408889634f)) return {TSDP_E_INVAL, "heads: scale must be positive and finite"};
  return NO_FAULT;
}

inline Fault cache_fault(const tsdp_kv_cache* k, int B) {
  if (!k) return {TSDP_E_INVAL, "null cache"};
  if (k->type < 0 || k->type > 2) return {TSDP_E_INVAL, "cache: type must be 0 (fp32), 1 (bf16) or 2 (8 bits)"};
  if (!head_dim_ok(k->head_dim)) return {TSDP_E_SHAPE, "cache: head_dim must be 32, 64 or 128"};
  if (k->kv_heads < 1 || k->kv_heads > MOST_HEADS) return {TSDP_E_SHAPE, "cache: kv_heads outside 1..1024"};
  const int n = k->page_tokens;
  if (n < (1 << MIN_PAGE_SHIFT) || n > (1 << MAX_PAGE_SHIFT) || (n & (n - 1))) return {TSDP_E_SHAPE, "cache: page_tokens must be a power of two, 16..4096"};
  if (k->pages < 1 || k->columns < 1 || k->B < 1) return {TSDP_E_SHAPE, "cache: pages, columns and B must be positive"};
  if (B < 0 || B > k->B) return {TSDP_E_SHAPE, "B is negative or more than the page table has rows"};
  if (!k->d_k || !k->d_v || !k->d_page_table) return {TSDP_E_INVAL, "cache: null pointer"};
  if (!aligned(k->d_k, 16) || !aligned(k->d_v, 16) || !aligned(k->d_page_table, 4)) return {TSDP_E_INVAL, "cache: pools must start at multiples of 16 bytes"};
  if (k->type == 2 && (!k->d_k_scale || !k->d_v_scale || !aligned(k->d_k_scale, 16) || !aligned(k->d_v_scale, 16)))
    return {TSDP_E_INVAL, "cache: 8 bits need both scale pools, at multiples of 16 bytes"};
  return NO_FAULT;
}

// rows of `width` elements of a type (0 fp32, 1 bf16), `row` elements apart
inline Fault rows_fault(const void* p, int64_t row, int64_t width, int type) {
  if (!p) return {TSDP_E_INVAL, "null pointer passed for packed rows"};
  if (!aligned(p, 16)) return {TSDP_E_INVAL, "packed rows must start at a multiple of 16 bytes"};
  if (row < width || row > MOST_ROW || row % (type == 0 ? 4 : 8) != 0)
    return {TSDP_E_SHAPE, "packed rows: distance less than a row, more than 2^24 elements or not a multiple of 16 bytes"};
  return NO_FAULT;
}

// A call whose fault is none and whose work is none returns at once.
inline Fault cache_rows_fault(const tsdp_kv_cache* cache, int B, int R_cap, int type, const int32_t* row_ptr, const int32_t* start,
                              const void* k, int64_t k_row, const void* v, int64_t v_row) {
  Fault f = cache_fault(cache, B);
  if (f.code) return f;
  if (R_cap < 0) return {TSDP_E_SHAPE, "R_cap must not be negative"};
  if (cache_blocks(R_cap, cache->kv_heads, cache->head_dim) > MOST_GRID) return {TSDP_E_SHAPE, "too many rows for one launch"};
  if (type != 0 && type != 1) return {TSDP_E_INVAL, "rows are fp32 (0) or bf16 (1)"};
  if (B == 0 || R_cap == 0) return NO_FAULT;
  if (!row_ptr || !start) return {TSDP_E_INVAL, "null row table"};
  const int64_t width = (int64_t)cache->kv_heads * cache->head_dim;
  f = rows_fault(k, k_row, width, type);
  return f.code ? f : rows_fault(v, v_row, width, type);
}

inline Fault prompt_fault(const tsdp_heads* h, int B, int q_cap, int k_cap, const int32_t* q_ptr, const int32_t* k_ptr,
                          const void* q, int64_t q_row, const void* k, int64_t k_row, const void* v, int64_t v_row,
                          const void* out, int64_t out_row) {
  Fault f = heads_fault(h);
  if (f.code) return f;
  if (B < 0 || q_cap < 0 || k_cap < 0) return {TSDP_E_SHAPE, "B, q_cap and k_cap must not be negative"};
  if (h->kv_heads * prompt_slots(q_cap, h->q_heads / h->kv_heads, B, 64) > MOST_GRID || k_cap > MOST_LENGTH) return {TSDP_E_SHAPE, "too many rows times heads for one launch"};
  if (B == 0 || q_cap == 0) return NO_FAULT;
  if (!q_ptr) return {TSDP_E_INVAL, "null row table"};
  if (!k_ptr && k_cap != q_cap) return {TSDP_E_INVAL, "without a row table of the keys k_cap must equal q_cap"};
  const int64_t qw = (int64_t)h->q_heads * h->head_dim, kw = (int64_t)h->kv_heads * h->head_dim;
  if ((f = rows_fault(q, q_row, qw, h->type)).code || (f = rows_fault(out, out_row, qw, h->type)).code) return f;
  if (k_cap == 0) return NO_FAULT;
  f = rows_fault(k, k_row, kw, h->type);
  return f.code ? f : rows_fault(v, v_row, kw, h->type);
}

// scratch of one call in bytes, -1 where the sizes are outside what one launch takes (heads: checked)
inline int64_t scratch_bytes(const tsdp_heads* h, int B, int tokens, int max_len) {
  if (B < 0 || tokens < 1 || tokens > MOST_TOKENS || max_len < 0) return -1;
  const int cols = tokens * (h->q_heads / h->kv_heads), n = most_chunks(max_len, cols, h->type == 0);
  const int64_t bk = (int64_t)B * h->kv_heads;
  if (n > MOST_GRID_Y || paged_blocks(bk, cols) > MOST_GRID || join_blocks(bk, cols, n, h->head_dim) > MOST_GRID) return -1;
  return n <= 1 ? 0 : (int64_t)B * h->kv_heads * cols * n * (h->head_dim + 2) * 4;
}

inline Fault paged_fault(const tsdp_heads* h, const tsdp_kv_cache* cache, int B, int tokens, int max_len, const int32_t* len,
                         const void* q, int64_t q_row, int out_type, const void* out, int64_t out_row, const void* scratch_at, int64_t scratch) {
  Fault f = heads_fault(h);
  if (f.code || (f = cache_fault(cache, B)).code) return f;
  if (cache->kv_heads != h->kv_heads || cache->head_dim != h->head_dim) return {TSDP_E_INVAL, "heads and cache differ in kv_heads or head_dim"};
  if (cache->type != 2 && cache->type != h->type) return {TSDP_E_INVAL, "queries must be of the cache's type, or the cache of 8 bits"};
  if (out_type != 0 && out_type != h->type) return {TSDP_E_INVAL, "outputs are fp32 or of the queries' type"};
  const int64_t need = scratch_bytes(h, B, tokens, max_len);
  if (need < 0) return {TSDP_E_SHAPE, "tokens (1..1024), max_len or their product with B and the heads outside what one launch takes"};
  if (B == 0) return NO_FAULT;
  if (!len) return {TSDP_E_INVAL, "null lengths"};
  const int64_t qw = (int64_t)h->q_heads * h->head_dim;
  if ((f = rows_fault(q, q_row, qw, h->type)).code || (f = rows_fault(out, out_row, qw, out_type)).code) return f;
  if (need > 0 && (!scratch_at || scratch < need || !aligned(scratch_at, 16)))
    return {TSDP_E_SHAPE, "scratch: null, too small or not at a multiple of 16 bytes"};
  return NO_FAULT;
}

}  // namespace tsdp
