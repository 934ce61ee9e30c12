// C ABI of attention over observation histories: the paged key / value cache, attention of whole prompts, attention of new
// tokens over the cache.  Argument checks and launches; nothing here allocates, synchronises or keeps state.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <algorithm>

#include "ctx_access.hpp"
#include "attend_check.hpp"
#include "attend_common.hpp"
#include "cache_kernels.hpp"
#include "attend_prompt.hpp"
#include "attend_paged.hpp"
#include "attend_wide.hpp"

using namespace tsdp;

namespace {

// the context's device is current (its status word and the kernels are that device's)
int check_device(tsdp_ctx* c) {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev != ctx_device(c)) return ctx_fail(c, TSDP_E_STATE, "the context's device is not current");
  return TSDP_OK;
}

int launched(tsdp_ctx* c) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? TSDP_OK : ctx_fail(c, TSDP_E_HIP, hipGetErrorString(e));
}

CacheView view_of(const tsdp_kv_cache* k) {
  return CacheView{k->d_k, k->d_v, k->d_k_scale, k->d_v_scale, k->d_page_table, k->pages, k->columns, k->kv_heads,
                   __builtin_ctz(k->page_tokens)};
}

template <template <typename, int, int> class Kernel, int HELD, int D>
void launch_cache(int type, const CacheRows& a, hipStream_t s) {
  const dim3 grid((unsigned)cache_blocks(a.R_cap, a.c.kv_heads, D));
  if (type == 0) hipLaunchKernelGGL((Kernel<float, HELD, D>::fn), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((Kernel<__bf16, HELD, D>::fn), grid, dim3(256), 0, s, a);
}
template <typename T, int HELD, int D> struct Write { static constexpr auto fn = k_cache_write<T, HELD, D>; };
template <typename T, int HELD, int D> struct Read { static constexpr auto fn = k_cache_read<T, HELD, D>; };
template <template <typename, int, int> class Kernel, int D>
void launch_cache_held(int held, int type, const CacheRows& a, hipStream_t s) {
  if (held == 0) launch_cache<Kernel, HELD_F32, D>(type, a, s);
  else if (held == 1) launch_cache<Kernel, HELD_BF16, D>(type, a, s);
  else launch_cache<Kernel, HELD_MX8, D>(type, a, s);
}

template <template <typename, int, int> class Kernel>
int cache_rows(tsdp_ctx* c, const tsdp_kv_cache* cache, int B, int R_cap, int type, const int32_t* row_ptr, const int32_t* start,
               void* k, int64_t k_row, void* v, int64_t v_row, void* stream) {
  if (!c) return TSDP_E_INVAL;
  const Fault f = cache_rows_fault(cache, B, R_cap, type, row_ptr, start, k, k_row, v, v_row);
  if (f.code) return ctx_fail(c, f.code, f.msg);
  if (B == 0 || R_cap == 0) return TSDP_OK;
  if (int rc = check_device(c)) return rc;
  CacheRows a{};
  a.c = view_of(cache);
  a.B = B; a.R_cap = R_cap; a.row_ptr = row_ptr; a.start = start;
  a.k = k; a.v = v; a.k_row = k_row; a.v_row = v_row; a.status = ctx_status(c);
  a.per_wave = rows_per_wave(cache->kv_heads, cache->head_dim);
  const hipStream_t s = (hipStream_t)stream;
  if (cache->head_dim == 32) launch_cache_held<Kernel, 32>(cache->type, type, a, s);
  else if (cache->head_dim == 64) launch_cache_held<Kernel, 64>(cache->type, type, a, s);
  else launch_cache_held<Kernel, 128>(cache->type, type, a, s);
  return launched(c);
}

template <int TQ>
dim3 prompt_grid(PromptArgs& a) {
  a.slots = (int)prompt_slots(a.q_cap, a.group, a.B, TQ);
  return dim3((unsigned)((int64_t)a.slots * a.kv_heads));
}

template <int D>
void launch_prompt(int type, PromptArgs a, hipStream_t s) {
  if (type == 0) {
    const dim3 grid = prompt_grid<64>(a);
    hipLaunchKernelGGL((k_wide<D, HELD_F32, true, 3, float, false, PromptArgs>), grid, dim3(256 * WIDE_GROUPS<false>), 0, s, a);
    return;
  }
  // Sequences of at most 320 keys on average: three waves a SIMD instead of the overlapped loop (256 of 96 tokens, 8 heads of
  // 64: 37 against 46 us; 32 of 512, 32 heads: 94 against 96; 128 x 128 queries on 512 keys: 133 against 110).  Heads of 128 have no
  // registers for it.
  const dim3 grid = prompt_grid<128>(a);
  if constexpr (D <= 64) {
    if (a.k_cap <= 320 * (int64_t)a.B) {
      hipLaunchKernelGGL((k_prompt_bf16<D, 4, 3, false>), grid, dim3(256), 0, s, a);
      return;
    }
  }
  hipLaunchKernelGGL((k_prompt_bf16<D, 4, 2, true>), grid, dim3(256), 0, s, a);
}

// Up to 16 columns a kv head (one matrix operand) keys and values go straight into registers; more share them through LDS, which
// also takes fewer, only slower (16 sequences of 4096, 32 heads on 2 of 128 in 8 bits: 16.0 against 32.7 us; 32 of 2000, 12 heads on one
// of 64 in fp32: 16.1 against 46.8).
template <int D, int HELD, bool QF32, int NP, typename Out>
void launch_paged(const PagedArgs& a, hipStream_t s) {
  const int64_t bk = (int64_t)a.B * a.cache.kv_heads;
  if (a.cols <= 16)
    hipLaunchKernelGGL((k_paged<D, HELD, QF32, NP, Out>), dim3((unsigned)paged_blocks(bk, a.cols), a.max_chunks), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((k_wide<D, HELD, QF32, NP, Out, true, PagedArgs>), dim3((unsigned)paged_blocks(bk, a.cols), a.max_chunks), dim3(256 * WIDE_GROUPS<true>), 0, s, a);
  if (a.max_chunks <= 1) return;
  const dim3 join((unsigned)join_blocks(bk, a.cols, a.max_chunks, D));
  if (a.max_chunks <= join_one(a.cols)) hipLaunchKernelGGL((k_paged_join<D, Out, true>), join, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((k_paged_join<D, Out, false>), join, dim3(256), 0, s, a);
}

template <int D>
void launch_paged_held(int held, int type, int out_type, const PagedArgs& a, hipStream_t s) {
  if (held == 0) launch_paged<D, HELD_F32, true, 3, float>(a, s);
  else if (held == 1 && out_type == 0) launch_paged<D, HELD_BF16, false, 3, float>(a, s);
  else if (held == 1) launch_paged<D, HELD_BF16, false, 2, __bf16>(a, s);
  else if (type == 0) launch_paged<D, HELD_MX8, true, 3, float>(a, s);
  else if (out_type == 0) launch_paged<D, HELD_MX8, false, 3, float>(a, s);
  else launch_paged<D, HELD_MX8, false, 2, __bf16>(a, s);
}

}  // namespace

extern "C" {

int tsdp_cache_write(tsdp_ctx* c, const tsdp_kv_cache* cache, int B, int R_cap, int type, const int32_t* d_row_ptr,
                     const int32_t* d_start, const void* d_k, int64_t k_row, const void* d_v, int64_t v_row, void* stream) {
  return cache_rows<Write>(c, cache, B, R_cap, type, d_row_ptr, d_start, const_cast<void*>(d_k), k_row, const_cast<void*>(d_v), v_row, stream);
}

int tsdp_cache_read(tsdp_ctx* c, const tsdp_kv_cache* cache, int B, int R_cap, int type, const int32_t* d_row_ptr,
                    const int32_t* d_start, void* d_k, int64_t k_row, void* d_v, int64_t v_row, void* stream) {
  return cache_rows<Read>(c, cache, B, R_cap, type, d_row_ptr, d_start, d_k, k_row, d_v, v_row, stream);
}

int tsdp_attend_prompt(tsdp_ctx* c, const tsdp_heads* h, int B, int q_cap, int k_cap, const int32_t* d_q_ptr, const int32_t* d_k_ptr,
                       const void* d_q, int64_t q_row, const void* d_k, int64_t k_row, const void* d_v, int64_t v_row,
                       void* d_out, int64_t out_row, float* d_lse, void* stream) {
  if (!c) return TSDP_E_INVAL;
  const Fault f = prompt_fault(h, B, q_cap, k_cap, d_q_ptr, d_k_ptr, d_q, q_row, d_k, k_row, d_v, v_row, d_out, out_row);
  if (f.code) return ctx_fail(c, f.code, f.msg);
  if (B == 0 || q_cap == 0) return TSDP_OK;
  if (int rc = check_device(c)) return rc;
  PromptArgs a{};
  a.B = B; a.q_cap = q_cap; a.k_cap = k_cap; a.heads = h->q_heads; a.kv_heads = h->kv_heads; a.group = h->q_heads / h->kv_heads; a.causal = h->causal;
  a.c = h->scale * LOG2E; a.q_ptr = d_q_ptr; a.k_ptr = d_k_ptr ? d_k_ptr : d_q_ptr;
  a.q = d_q; a.k = d_k; a.v = d_v; a.out = d_out; a.q_row = q_row; a.k_row = k_row; a.v_row = v_row; a.out_row = out_row;
  a.lse = d_lse; a.status = ctx_status(c);
  const hipStream_t s = (hipStream_t)stream;
  if (h->head_dim == 32) launch_prompt<32>(h->type, a, s);
  else if (h->head_dim == 64) launch_prompt<64>(h->type, a, s);
  else launch_prompt<128>(h->type, a, s);
  return launched(c);
}

int64_t tsdp_attend_scratch(const tsdp_heads* h, int B, int tokens, int max_len) {
  const Fault f = heads_fault(h);
  if (f.code) return f.code;
  const int64_t n = scratch_bytes(h, B, tokens, max_len);
  return n < 0 ? TSDP_E_SHAPE : n;
}

int tsdp_attend_paged(tsdp_ctx* c, const tsdp_heads* h, const tsdp_kv_cache* cache, int B, int tokens, int max_len,
                      const int32_t* d_len, const void* d_q, int64_t q_row, int out_type, void* d_out, int64_t out_row,
                      float* d_lse, void* d_scratch, int64_t scratch, void* stream) {
  if (!c) return TSDP_E_INVAL;
  const Fault f = paged_fault(h, cache, B, tokens, max_len, d_len, d_q, q_row, out_type, d_out, out_row, d_scratch, scratch);
  if (f.code) return ctx_fail(c, f.code, f.msg);
  if (B == 0) return TSDP_OK;
  if (int rc = check_device(c)) return rc;
  PagedArgs a{};
  a.cache = view_of(cache);
  a.B = B; a.heads = h->q_heads; a.tokens = tokens; a.cols = tokens * (h->q_heads / h->kv_heads); a.max_len = max_len; a.fp32 = h->type == 0;
  a.max_chunks = std::max(1, most_chunks(max_len, a.cols, a.fp32)); a.causal = h->causal; a.c = h->scale * LOG2E;
  a.len = d_len; a.q = d_q; a.out = d_out; a.q_row = q_row; a.out_row = out_row; a.lse = d_lse; a.status = ctx_status(c);
  a.part = static_cast<float*>(d_scratch);
  a.part_ml = a.part + (int64_t)B * h->kv_heads * a.cols * a.max_chunks * h->head_dim;
  const hipStream_t s = (hipStream_t)stream;
  if (h->head_dim == 32) launch_paged_held<32>(cache->type, h->type, out_type, a, s);
  else if (h->head_dim == 64) launch_paged_held<64>(cache->type, h->type, out_type, a, s);
  else launch_paged_held<128>(cache->type, h->type, out_type, a, s);
  return launched(c);
}

}  // extern "C"
