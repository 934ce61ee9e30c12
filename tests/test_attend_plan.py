"""Host-side rules of attention and of the key / value cache (csrc/attend_plan.hpp, csrc/attend_check.hpp, plain C++), compiled
here and checked without a GPU: positions and bad pages, masks, chunks, tiles of packed rows, refused arguments."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

from tests import attend_oracle as ao

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2512_15773_amd", "csrc")
SHIM = """
#include "attend_check.hpp"
using namespace tsdp;
extern "C" {
int page(const int32_t* table, int pages, int columns, int b, long col) {
  CacheView c{}; c.table = table; c.pages = pages; c.columns = columns;
  return page_of(c, b, col);
}
int64_t row(int kv, int shift, int page, int head, int token) { CacheView c{}; c.kv_heads = kv; c.page_shift = shift; return pool_row(c, page, head, token); }
void rows(const int32_t* ptr, int b, int cap, int* lo, int* hi) { rows_of(ptr, b, cap, *lo, *hi); }
int sees(int i, int nq, int nk, int causal) { return seen(i, nq, nk, causal != 0); }
int chunks(int len, int cols, int fp32) { return chunks_of(len, cols, fp32 != 0); }
int chunk(int len, int cols, int fp32) { return 1 << chunk_shift(len, cols, fp32 != 0); }
int most(int max_len, int cols, int fp32) { return most_chunks(max_len, cols, fp32 != 0); }
int refuse_rows(const tsdp_kv_cache* c, int B, int R, int type, const int32_t* p, const int32_t* s, const void* k, int64_t kr, const void* v, int64_t vr) {
  return cache_rows_fault(c, B, R, type, p, s, k, kr, v, vr).code;
}
int refuse_prompt(const tsdp_heads* h, int B, int qc, int kc, const int32_t* qp, const int32_t* kp, const void* q, int64_t qr, const void* k, int64_t kr, const void* v, int64_t vr, const void* o, int64_t orow) {
  return prompt_fault(h, B, qc, kc, qp, kp, q, qr, k, kr, v, vr, o, orow).code;
}
int refuse_paged(const tsdp_heads* h, const tsdp_kv_cache* c, int B, int t, int n, const int32_t* len, const void* q, int64_t qr, int ot, const void* o, int64_t orow, const void* s, int64_t sb) {
  return paged_fault(h, c, B, t, n, len, q, qr, ot, o, orow, s, sb).code;
}
int64_t scratch(const tsdp_heads* h, int B, int t, int n) { return scratch_bytes(h, B, t, n); }
}
"""
OK, INVAL, SHAPE = 0, -1, -2


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    out = tmp_path_factory.mktemp("attend_plan")
    src, lib = str(out / "shim.cpp"), str(out / "shim.so")
    with open(src, "w") as f:
        f.write(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, src, "-o", lib], check=True)
    plan = C.CDLL(lib)
    i32, i64, vp = C.c_int, C.c_int64, C.c_void_p
    plan.page.argtypes = [vp, i32, i32, i32, C.c_long]
    plan.row.restype = i64
    plan.rows.argtypes = [vp, i32, i32, C.POINTER(i32), C.POINTER(i32)]
    plan.refuse_rows.argtypes = [vp, i32, i32, i32, vp, vp, vp, i64, vp, i64]
    plan.refuse_prompt.argtypes = [vp, i32, i32, i32, vp, vp] + [vp, i64] * 4
    plan.refuse_paged.argtypes = [vp, vp, i32, i32, i32, vp, vp, i64, i32, vp, i64, vp, i64]
    plan.scratch.argtypes, plan.scratch.restype = [vp, i32, i32, i32], i64
    return plan


def test_pages_outside_the_pool_or_the_table_are_never_followed(plan):
    table = np.array([[0, 3, -1], [4, 2 ** 31 - 1, -2 ** 31]], np.int32)
    for b in range(2):
        for col in (-2 ** 40, -1, 0, 1, 2, 3, 2 ** 40):
            want = int(table[b, col]) if 0 <= col < 3 and 0 <= table[b, col] < 4 else -1
            assert plan.page(table.ctypes.data, 4, 3, b, col) == want, (b, col)


def test_rows_of_the_pools_pass_32_bits(plan):
    assert plan.row(8, 8, 2 ** 20, 7, 255) == ((2 ** 20 * 8 + 7) << 8) + 255 > 2 ** 31
    assert plan.row(1024, 12, 2 ** 31 - 1, 1023, 4095) == (((2 ** 31 - 1) * 1024 + 1023) << 12) + 4095


def test_packed_rows_are_clipped_to_their_bound(plan):
    for ptr in ([0, 5, 5, 9], [0, 5, 3, 40], [-3, 4, 12, 12], [11, 12, 2 ** 31 - 1, 0]):
        p = np.array(ptr, np.int32)
        for b in range(3):
            lo, hi = C.c_int(), C.c_int()
            plan.rows(p.ctypes.data, b, 10, C.byref(lo), C.byref(hi))
            assert 0 <= lo.value <= hi.value <= 10
            if 0 <= ptr[b] <= ptr[b + 1] <= 10:
                assert (lo.value, hi.value) == (ptr[b], ptr[b + 1])


def test_keys_that_a_query_sees(plan):
    for nq, nk in ((1, 1), (1, 7), (5, 5), (5, 2), (3, 0), (4, 9)):
        for i in range(nq):
            assert plan.sees(i, nq, nk, 0) == nk
            assert plan.sees(i, nq, nk, 1) == sum(j <= nk - nq + i for j in range(nk))
    assert plan.sees(0, 2 ** 31 - 1, 0, 1) == 0 and plan.sees(2 ** 31 - 2, 2 ** 31 - 1, 2 ** 31 - 1, 1) == 2 ** 31 - 1


@pytest.mark.parametrize("fp32", (0, 1))
def test_chunks_cover_a_length_and_their_bound_holds(plan, fp32):
    rng = np.random.default_rng(0)
    for cols in (1, 8, 16, 17, 33, 64, 65, 1024):
        lens = [0, 1, 255, 256, 257, 1024, 1025, 16383, 16384, 16385, 65536, 65537, 131072] + rng.integers(0, 300000, 50).tolist()
        for n in lens:
            c = plan.chunk(n, cols, fp32)
            assert c >= 128 and c % 128 == 0                          # four waves of whole tiles
            assert c <= (2048 if cols <= 16 else 1024)                # 64 lanes hold the pages of 16 tokens each, of a wave or of all four
            assert plan.chunks(n, cols, fp32) == -(-n // c)
        for most in lens:
            bound = plan.most(most, cols, fp32)
            for n in [x for x in lens if x <= most] + [min(most, 1024), min(most, 16384), min(most, 65536)]:
                assert plan.chunks(n, cols, fp32) <= bound, (n, most, cols)


@pytest.mark.parametrize("tq", (32, 64, 128))
@pytest.mark.parametrize("group", (1, 3, 8))
def test_every_query_has_one_slot(tq, group):
    """The rule by which a workgroup of the prompt kernel finds its columns (queries x heads of a group): sequence b owns slots
    group * ptr[b] / tq + b and on."""
    rng = np.random.default_rng(tq)
    for _ in range(200):
        n = group * (rng.integers(0, 300, rng.integers(1, 70)) * rng.integers(0, 2))
        ptr = np.concatenate([[0], np.cumsum(n)])
        B, slots = len(n), int(ptr[-1]) // tq + len(n)
        first = ptr[:-1] // tq + np.arange(B)
        done = np.zeros(int(ptr[-1]), int)
        for slot in range(slots):
            b = int(((ptr[1:] // tq + np.arange(1, B + 1)) <= slot).sum())
            if b >= B:
                continue
            i0 = (slot - first[b]) * tq
            if 0 <= i0 < n[b]:
                done[ptr[b] + i0:ptr[b] + min(i0 + tq, n[b])] += 1
        assert (done == 1).all()


def _good():
    from paper_2512_15773_amd import binding as b
    at = 1 << 20
    heads = dict(type=1, q_heads=8, kv_heads=2, head_dim=64, causal=1, scale=0.125)
    cache = dict(type=2, kv_heads=2, head_dim=64, page_tokens=64, pages=10, B=4, columns=5, d_k=at, d_v=at, d_k_scale=at, d_v_scale=at, d_page_table=at)
    return b, at, heads, cache


def test_refused_heads(plan):
    b, at, heads, cache = _good()
    for bad, code in ((dict(type=2), INVAL), (dict(type=-1), INVAL), (dict(head_dim=48), SHAPE), (dict(head_dim=256), SHAPE), (dict(q_heads=7), SHAPE),
                      (dict(kv_heads=0), SHAPE), (dict(q_heads=0), SHAPE), (dict(q_heads=2048, kv_heads=1), SHAPE), (dict(causal=2), INVAL),
                      (dict(scale=0.0), INVAL), (dict(scale=-1.0), INVAL), (dict(scale=float("nan")), INVAL), (dict(scale=3e38), INVAL)):
        h = b.TsdpHeads(**{**heads, **bad})
        assert plan.refuse_prompt(C.byref(h), 4, 100, 100, at, None, at, 512, at, 128, at, 128, at, 512) == code, bad
        c = b.TsdpKvCache(**cache)
        assert plan.refuse_paged(C.byref(h), C.byref(c), 4, 1, 100, at, at, 512, 1, at, 512, None, 0) == code, bad
    assert plan.refuse_prompt(None, 4, 100, 100, at, None, at, 512, at, 128, at, 128, at, 512) == INVAL
    lib = b.load_library()
    assert lib.tsdp_attend_scratch(b.TsdpHeads(**{**heads, "head_dim": 48}), 4, 1, 100) == SHAPE
    assert lib.tsdp_attend_scratch(None, 4, 1, 100) == INVAL


def test_refused_caches_and_rows(plan):
    b, at, heads, cache = _good()
    good = (4, 100, 1, at, at, at, 128, at, 128)
    call = lambda c, a=good: plan.refuse_rows(C.byref(c), *a)
    assert call(b.TsdpKvCache(**cache)) == OK
    for bad, code in ((dict(type=3), INVAL), (dict(head_dim=96), SHAPE), (dict(kv_heads=0), SHAPE), (dict(page_tokens=8), SHAPE), (dict(page_tokens=48), SHAPE),
                      (dict(page_tokens=8192), SHAPE), (dict(page_tokens=0), SHAPE), (dict(pages=0), SHAPE), (dict(columns=0), SHAPE), (dict(B=3), SHAPE), (dict(d_k=None), INVAL),
                      (dict(d_v=at + 8), INVAL), (dict(d_page_table=None), INVAL), (dict(d_k_scale=None), INVAL), (dict(d_v_scale=at + 4), INVAL)):
        assert call(b.TsdpKvCache(**{**cache, **bad})) == code, bad
    assert plan.refuse_rows(None, *good) == INVAL
    c = b.TsdpKvCache(**cache)
    for i, value, code in ((0, -1, SHAPE), (1, -1, SHAPE), (2, 2, INVAL), (2, -1, INVAL), (3, None, INVAL), (4, None, INVAL), (5, None, INVAL), (5, at + 2, INVAL),
                           (6, 127, SHAPE), (6, 132, SHAPE), (6, (1 << 24) + 8, SHAPE), (7, None, INVAL), (8, 64, SHAPE)):
        assert call(c, good[:i] + (value,) + good[i + 1:]) == code, (i, value)
    assert call(c, (0, 0, 1, None, None, None, 0, None, 0)) == OK              # nothing to do
    assert call(c, (4, 100, 0, at, at, at, 132, at, 128)) == OK                # fp32: multiples of four elements


def test_refused_prompts(plan):
    b, at, heads, _ = _good()
    h = b.TsdpHeads(**heads)
    good = (4, 100, 100, at, None, at, 512, at, 128, at, 128, at, 512)
    call = lambda a: plan.refuse_prompt(C.byref(h), *a)
    assert call(good) == OK
    for i, value, code in ((0, -1, SHAPE), (1, -1, SHAPE), (2, -5, SHAPE), (2, 99, INVAL), (3, None, INVAL), (5, None, INVAL), (6, 511, SHAPE), (7, at + 8, INVAL), (8, 120, SHAPE),
                           (9, None, INVAL), (10, 129, SHAPE), (11, None, INVAL), (12, 256, SHAPE), (0, 2 ** 31 - 1, SHAPE)):
        assert call(good[:i] + (value,) + good[i + 1:]) == code, (i, value)
    assert call((0, 0, 0, None, None) + (None, 0) * 4) == OK
    assert call((4, 100, 0, at, at, at, 512, None, 0, None, 0, at, 512)) == OK   # no keys at all


def test_refused_paged_calls(plan):
    b, at, heads, cache = _good()
    h, c = b.TsdpHeads(**heads), b.TsdpKvCache(**cache)
    need = plan.scratch(C.byref(h), 4, 1, 1000)
    assert need == 4 * 2 * 4 * 4 * 66 * 4
    good = (4, 1, 1000, at, at, 512, 1, at, 512, at, need)
    call = lambda a, h=h, c=c: plan.refuse_paged(C.byref(h), C.byref(c), *a)
    assert call(good) == OK
    for i, value, code in ((0, -1, SHAPE), (0, 5, SHAPE), (1, 0, SHAPE), (1, 1025, SHAPE), (2, -1, SHAPE), (2, 2 ** 31 - 1, SHAPE), (3, None, INVAL), (4, None, INVAL), (5, 8, SHAPE),
                           (6, 2, INVAL), (6, -1, INVAL), (7, None, INVAL), (8, 8, SHAPE), (9, None, SHAPE), (9, at + 4, SHAPE), (10, need - 1, SHAPE)):
        assert call(good[:i] + (value,) + good[i + 1:]) == code, (i, value)
    assert call((4, 1, 200, at, at, 512, 0, at, 512, None, 0)) == OK            # one chunk: no scratch
    for bad in (dict(type=0), dict(kv_heads=4), dict(head_dim=32)):
        assert call(good, c=b.TsdpKvCache(**{**cache, **bad})) == INVAL, bad
    assert call(good, h=b.TsdpHeads(**{**heads, "type": 0})) == INVAL           # fp32 queries with bf16 outputs


def test_refused_launches(plan):
    """A launch has fewer than 2^32 threads: calls that would need more are refused, not left to the launch."""
    b, at, heads, cache = _good()
    most = (2 ** 32 - 1) // 512
    c, one = b.TsdpKvCache(**{**cache, "B": 2 ** 31 - 1}), b.TsdpHeads(**{**heads, "q_heads": 2})
    rows = lambda n: plan.refuse_rows(C.byref(c), 4, n, 1, at, at, at, 128, at, 128)
    assert rows(2 * 4 * most) == OK and rows(2 * 4 * most + 1) == SHAPE          # two rows a wave, four waves
    prompt = lambda B, q, k: plan.refuse_prompt(C.byref(one), B, q, k, at, at, at, 512, at, 128, at, 128, at, 512)
    assert prompt(4, 64 * (most // 2 - 4), 100) == OK and prompt(4, 64 * (most // 2 - 3), 100) == SHAPE
    assert prompt(most // 2, 63, 100) == OK and prompt(most // 2, 64, 100) == SHAPE
    assert prompt(4, 100, 2 ** 31 - 256) == OK and prompt(4, 100, 2 ** 31 - 255) == SHAPE
    scratch = lambda B, tokens, n: plan.scratch(C.byref(one), B, tokens, n)      # two kv heads, a column a token
    assert scratch(most // 2, 16, 256) == 0 and scratch(most // 2 + 1, 16, 256) < 0
    assert scratch(most // 4, 65, 1024) == 0 and scratch(most // 4 + 1, 65, 1024) < 0
    assert scratch(most // 2, 16, 300) > 0 and scratch(most // 2 + 1, 16, 300) < 0
    assert scratch(most // 2, 1, 10000) > 0 and scratch(most // 4, 2, 10000) > 0 and scratch(most // 4 + 1, 2, 10000) < 0


def test_oracle_of_8_bits():
    x = ao.e4m3_values()
    assert np.nanmax(x) == 448 and np.isnan(x[[127, 255]]).all() and x[8] == 2.0 ** -6 and x[1] == 2.0 ** -9
    v = np.zeros(64)
    v[:3], v[3], v[32:36] = (448.0, 447.0, 24.5), np.inf, (1e-40, 465.0, -17.0, 2.0 ** -11)
    codes, scale = ao.mx8(v)
    assert scale.tolist() == [127, 128]
    back = ao.mx8_values(codes, scale)
    assert back[:3].tolist() == [448, 448, 24] and np.isnan(back[3]) and back[32:36].tolist() == [0, 480, -16, 0]
