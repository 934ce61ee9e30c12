"""Attention over observation histories against a plain implementation in 64 bits (needs an MI355X): whole prompts, the cache
written and read back, new tokens over the cache, and all of them as they are used together."""
import numpy as np
import pytest

import tsdp_inputs as ti
from tests import attend_oracle as ao
from tests.helpers import kernels

pytestmark = pytest.mark.gpu
WEIGHTS = {"prompt": {"fp32": 0.0, "bf16": 2.0 ** -8}, "paged": {"fp32": 2.0 ** -24, "bf16": 2.0 ** -16}}   # by type / type of the outputs
POISON = 0x7FC1                                          # a NaN


@pytest.fixture(scope="module")
def ctx():
    from paper_2512_15773_amd import Tsdp
    c = Tsdp.from_workload(ti.C1)
    yield c
    c.close()


def torch_dtype(name):
    import torch
    return {"fp32": torch.float32, "bf16": torch.bfloat16}[name]


def draw(rng, shape, dtype, spread=1.0):
    """A device tensor of normal values of the type."""
    import torch
    return torch.from_numpy((rng.standard_normal(shape) * spread).astype(np.float32)).to(torch_dtype(dtype)).cuda()


def f64(t):
    return t.double().cpu().numpy()


def i32(x):
    import torch
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def nans(shape, dtype):
    import torch
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda")


def check(got, lse, ref, dim, n, out_type, weights, what):
    out, ref_lse, mean, size = ref
    err, lim = np.abs(f64(got) - out), ao.bound(out, mean, size, dim, n, out_type, weights)
    assert (err <= lim).all(), f"{what}: {np.nanmax(err / lim):.3f} of the bound, {np.isnan(err).sum()} NaN"
    if lse is not None:
        a, lim = f64(lse), ao.lse_bound(ref_lse, size, dim, n)[..., 0]
        gone = np.isinf(ref_lse)
        assert np.array_equal(a[gone], ref_lse[gone]), what
        assert (np.abs(a[~gone] - ref_lse[~gone]) <= lim[~gone]).all(), what


# ---- whole prompts

SEQUENCES = {                                            # (queries, keys) of each environment
    "edges": [(1, 1), (0, 0), (33, 33), (64, 64), (5, 0), (7, 3), (0, 9), (2, 1), (31, 63), (32, 65)],
    "tiles": [(128, 128), (129, 129), (1, 130), (97, 257)],
    "history": [(3, 200), (130, 191), (70, 64)],
}


@pytest.mark.parametrize("dtype", ("fp32", "bf16"))
@pytest.mark.parametrize("dim,heads,kv", ((32, 4, 4), (64, 6, 2), (128, 8, 1)))
@pytest.mark.parametrize("causal", (True, False))
@pytest.mark.parametrize("which", sorted(SEQUENCES))
def test_prompt(ctx, dtype, dim, heads, kv, causal, which):
    import torch
    rng = np.random.default_rng(dim * 7 + heads + len(which))
    seqs = SEQUENCES[which]
    qp, kp = (np.concatenate([[0], np.cumsum([s[i] for s in seqs])]) for i in (0, 1))
    # rows of wider projections: q beside something else, k and v next to each other; NaN in every row that nobody owns
    spare = 5
    q = nans((qp[-1] + spare, heads + 1, dim), torch_dtype(dtype))
    kvs = nans((kp[-1] + spare, 2 * kv, dim), torch_dtype(dtype))
    q[:qp[-1], :heads] = draw(rng, (qp[-1], heads, dim), dtype, 1.5)
    kvs[:kp[-1]] = draw(rng, (kp[-1], 2 * kv, dim), dtype, 1.5)
    out = torch.full((qp[-1] + spare, heads, dim), 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full((qp[-1] + spare, heads), 7.0, device="cuda")
    got = ctx.tsdp_attend_prompt(q[:, :heads], kvs[:, :kv], kvs[:, kv:], i32(qp), i32(kp), causal=causal, scale=0.11, out=out, lse=lse)
    assert got is out
    for b, (nq, nk) in enumerate(seqs):
        rq, rk = slice(qp[b], qp[b + 1]), slice(kp[b], kp[b + 1])
        ref = ao.attend(f64(q[rq, :heads]), f64(kvs[rk, :kv]), f64(kvs[rk, kv:]), 0.11, causal)
        check(out[rq], lse[rq], ref, dim, nk, dtype, WEIGHTS["prompt"][dtype], (which, b))
    assert (out[qp[-1]:] == 7).all() and (lse[qp[-1]:] == 7).all()             # rows behind the last sequence
    assert ctx.tsdp_status() == 0


@pytest.mark.parametrize("dtype", ("fp32", "bf16"))
@pytest.mark.parametrize("n,dim", ((300, 64), (700, 64), (700, 128)))
def test_prompt_over_large_scores_and_far_maxima(ctx, dtype, n, dim):
    """Scores of some hundreds, growing and falling along the keys: the running maximum moves often, or never."""
    rng = np.random.default_rng(1)
    k = rng.standard_normal((n, 1, dim)) * 0.2
    k[:, 0, 0] = np.concatenate([np.linspace(-30, 30, n // 2), np.linspace(30, -30, n // 2)])
    q = rng.standard_normal((n, 2, dim)) * 0.2
    q[:, 0, 0], q[:, 1, 0] = 10.0, -10.0
    import torch
    to = lambda x: torch.from_numpy(x.astype(np.float32)).to(torch_dtype(dtype)).cuda()
    q, k, v = to(q), to(k), draw(rng, (n, 1, dim), dtype)
    for causal in (True, False):
        got = ctx.tsdp_attend_prompt(q, k, v, i32([0, n]), causal=causal, scale=1.0)
        check(got, None, ao.attend(f64(q), f64(k), f64(v), 1.0, causal), dim, n, dtype, WEIGHTS["prompt"][dtype], causal)


@pytest.mark.parametrize("dtype", ("fp32", "bf16"))
@pytest.mark.parametrize("n,dim", ((200, 32), (200, 64), (200, 128), (500, 32), (500, 64)))
def test_prompt_hides_what_is_masked_and_shows_what_is_not(ctx, dtype, n, dim):
    """NaN and infinities in keys and values: queries before them are bit-equal to a run without them, those from them on are not
    finite (values) or NaN (keys)."""
    rng = np.random.default_rng(2)
    at = n - 123
    q, k, v = (draw(rng, (n, 2, dim), dtype) for _ in range(3))
    clean = ctx.tsdp_attend_prompt(q, k, v, i32([0, n]), causal=True)
    for bad in (float("nan"), float("inf"), -float("inf")):
        for x, name in ((v, "v"), (k, "k")):
            y = x.clone()
            y[at, 0, 3] = bad
            got = ctx.tsdp_attend_prompt(q, y if name == "k" else k, y if name == "v" else v, i32([0, n]), causal=True)
            assert (got[:at] == clean[:at]).all(), (bad, name)
            assert (got[:, 1] == clean[:, 1]).all()
            if name == "v":
                assert not np.isfinite(f64(got[at:, 0, 3])).any()
                rest = [i for i in range(dim) if i != 3]
                assert (got[:, 0, rest] == clean[:, 0, rest]).all()
            elif np.isnan(bad):
                assert np.isnan(f64(got[at:, 0])).all()


@pytest.mark.parametrize("dtype", ("fp32", "bf16"))
def test_prompt_rows_do_not_depend_on_their_batch(ctx, dtype):
    import torch
    rng = np.random.default_rng(3)
    n = [190, 1, 333, 64, 1300]                          # on average more than 320 keys, some less: another kernel alone
    ptr = np.concatenate([[0], np.cumsum(n)])
    dim = 64
    q, k, v = draw(rng, (ptr[-1], 4, dim), dtype), draw(rng, (ptr[-1], 2, dim), dtype), draw(rng, (ptr[-1], 2, dim), dtype)
    whole = ctx.tsdp_attend_prompt(q, k, v, i32(ptr))
    for b in range(5):
        r = slice(ptr[b], ptr[b + 1])
        one = ctx.tsdp_attend_prompt(q[r], k[r], v[r], i32([0, n[b]]))
        assert torch.equal(one, whole[r]), b


def test_prompt_row_tables_beyond_their_bound_are_clipped_and_reported(ctx):
    import torch
    rng = np.random.default_rng(4)
    q, k, v = (draw(rng, (100, 2, 32), "fp32") for _ in range(3))
    out = torch.full((150, 2, 32), 7.0, device="cuda")
    ctx.tsdp_attend_prompt(q, k, v, i32([0, 60, 140]), causal=False, out=out[:100])
    assert ctx.tsdp_status() == 32
    check(out[:60], None, ao.attend(f64(q[:60]), f64(k[:60]), f64(v[:60]), 32 ** -0.5, False), 32, 60, "fp32", 0.0, "first")
    check(out[60:100], None, ao.attend(f64(q[60:]), f64(k[60:]), f64(v[60:]), 32 ** -0.5, False), 32, 40, "fp32", 0.0, "clipped")
    assert (out[100:] == 7).all()
    for ptr in ([0, -5, 30], [90, 20, 10], [2 ** 31 - 1, 5, 5]):
        ctx.tsdp_attend_prompt(q, k, v, i32(ptr), causal=True, out=out[:100])
    ctx.tsdp_status()
    assert (out[100:] == 7).all()


# ---- the cache

HELD = {"fp32": "float32", "bf16": "bfloat16", "mx8": "uint8"}


def new_cache(rng, held, B, columns, kv, page, dim, poison=True):
    """Pages in random order; what nobody writes holds NaN."""
    import torch
    from paper_2512_15773_amd import KvCache
    pages = B * columns + 3
    table = i32(rng.permutation(pages)[:B * columns].reshape(B, columns))
    c = KvCache.alloc(getattr(torch, HELD[held]), pages, kv, page, dim, table)
    if poison:
        for x in (c.k, c.v):
            x.fill_(127 if held == "mx8" else float("nan"))
        if held == "mx8":
            c.k_scale.fill_(127); c.v_scale.fill_(127)
    return c


def unusual_rows(rng, shape, dtype):
    """Normal rows of all sizes, with blocks of zeros, borders of the 8-bit grid, infinities and NaN."""
    x = rng.standard_normal(shape) * np.exp2(rng.integers(-20, 20, shape[:2] + (1,)))
    flat = x.reshape(-1, 32)
    flat[0] = 0.0
    if len(flat) > 8:
        flat[1, :4] = (np.inf, -np.inf, np.nan, 3.0)
        flat[2] = 448.0 - np.arange(32)
        flat[3] = np.exp2(-np.arange(32)) * 448.0
        flat[4, 0] = 449.0
        flat[5] = -0.0
        flat[6] = np.linspace(-1, 1, 32) * 2.0 ** -125
    import torch
    return torch.from_numpy(x.astype(np.float32)).to(torch_dtype(dtype)).cuda()


def equal(a, b):
    a, b = np.asarray(a), np.asarray(b)
    return np.array_equal(a, b, equal_nan=a.dtype.kind == "f")


@pytest.mark.parametrize("held", ("fp32", "bf16", "mx8"))
@pytest.mark.parametrize("dtype", ("fp32", "bf16"))
@pytest.mark.parametrize("dim,kv,page", ((32, 1, 16), (64, 3, 64), (128, 8, 32)))
def test_cache_written_and_read_back(ctx, held, dtype, dim, kv, page):
    import torch
    rng = np.random.default_rng(dim + kv)
    n, start = [1, 0, 37, 5, 70], [0, 9, page - 1, 2 * page, 3]
    B, columns, ptr = len(n), -(-80 // page) + 3, np.concatenate([[0], np.cumsum(n)])
    c = new_cache(rng, held, B, columns, kv, page, dim)
    wide = nans((ptr[-1] + 4, 2 * kv, dim), torch_dtype(dtype))                # rows behind the last one: never written anywhere
    wide[:ptr[-1]] = unusual_rows(rng, (ptr[-1], 2 * kv, dim), dtype)
    before = [x.clone() for x in (c.k, c.v)]
    ctx.tsdp_cache_write(c, i32(ptr), i32(start), wide[:, :kv], wide[:, kv:])
    table = c.page_table.cpu().numpy()
    pool = lambda x: (x if held == "mx8" else x.float()).cpu().numpy()
    want = [pool(x).copy() for x in before]
    scales = [np.full((c.k.shape[0], kv, page, dim // 32), 127, np.uint8) for _ in "kv"] if held == "mx8" else None
    rows = [f64(wide[:, :kv]), f64(wide[:, kv:])]
    values = []
    for which, x in enumerate(rows):
        if held == "mx8":
            codes, scale = ao.mx8(x)
            values.append(ao.mx8_values(codes, scale))
        else:
            codes = torch.from_numpy(x).to(torch_dtype(held)).float().numpy()
            values.append(codes.astype(np.float64))
        for b in range(B):
            for i in range(n[b]):
                pos = start[b] + i
                p, t = table[b, pos // page], pos % page
                want[which][p, :, t] = codes[ptr[b] + i]
                if held == "mx8":
                    scales[which][p, :, t] = scale[ptr[b] + i]
    for which, (x, s) in enumerate(((c.k, c.k_scale), (c.v, c.v_scale))):
        got = pool(x)
        if held == "mx8":
            nan = (want[which] & 127) == 127                                    # either sign of NaN
            assert np.array_equal(np.where(nan, 127, got & np.where(nan, 127, 255)), np.where(nan, 127, want[which])) and np.array_equal(s.cpu().numpy(), scales[which])
        else:
            assert equal(got, want[which])
    for out_type in ("fp32", "bf16"):
        out = tuple(torch.full((ptr[-1] + 4, kv, dim), 7.0, dtype=torch_dtype(out_type), device="cuda") for _ in "kv")
        ctx.tsdp_cache_read(c, i32(ptr), i32(start), ptr[-1] + 4, torch_dtype(out_type), out=out)
        for which in (0, 1):
            w = torch.from_numpy(values[which][:ptr[-1]]).to(torch_dtype(out_type))
            assert equal(out[which][:ptr[-1]].float().cpu().numpy(), w.float().numpy()), (out_type, which)
            assert (out[which][ptr[-1]:] == 7).all()
    assert ctx.tsdp_status() == 0


def test_cache_positions_outside_are_left_out_and_reported(ctx):
    import torch
    rng = np.random.default_rng(6)
    c = new_cache(rng, "bf16", 3, 2, 2, 16, 64, poison=False)
    c.page_table[1, 0] = c.k.shape[0]                                           # one behind the pool
    c.page_table[2, 1] = -1
    n, start = [4, 4, 8], [30, 14, -4]                                          # past the table, half on a bad page, before the first
    ptr = np.concatenate([[0], np.cumsum(n)])
    k, v = draw(rng, (16, 2, 64), "bf16"), draw(rng, (16, 2, 64), "bf16")
    ctx.tsdp_cache_write(c, i32(ptr), i32(start), k, v)
    assert ctx.tsdp_status() == 64
    table = c.page_table.cpu().numpy()
    seen = torch.zeros(16, dtype=torch.bool)
    for b in range(3):
        for i in range(n[b]):
            pos = start[b] + i
            page = table[b, pos // 16] if 0 <= pos < 32 else -1
            if 0 <= page < c.k.shape[0]:
                seen[ptr[b] + i] = True
                assert torch.equal(c.k[page, :, pos % 16], k[ptr[b] + i])
    assert int((c.k != 0).any(-1).any(1).sum()) == int(seen.sum()) == 8
    out = ctx.tsdp_cache_read(c, i32(ptr), i32(start), 16, torch.bfloat16)
    assert ctx.tsdp_status() == 64
    assert torch.equal(out[0][seen.cuda()], k[seen.cuda()]) and (out[0][~seen.cuda()] == 0).all()
    ctx.tsdp_cache_read(c, i32([0, 4, 8, 99]), i32([0, 0, 0]), 16, torch.bfloat16)   # row table beyond its bound
    assert ctx.tsdp_status() & 32


# ---- new tokens over the cache

def filled(rng, held, lens, kv, page, dim, spread=1.0):
    """A cache with random values at the first lens[b] positions; everything else NaN.  Also those values in 64 bits."""
    import torch
    columns = -(-max(max(lens), 1) // page)
    c = new_cache(rng, held, len(lens), columns, kv, page, dim)
    table, values = c.page_table.cpu().numpy(), []
    for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)):
        per = []
        for b, n in enumerate(lens):
            y = rng.standard_normal((n, kv, dim)) * spread
            at = (torch.from_numpy(table[b, np.arange(n) // page]).long().cuda(), torch.from_numpy(np.arange(n) % page).cuda())
            if held == "mx8":
                codes, scale = ao.mx8(y)
                x[at[0], :, at[1]] = torch.from_numpy(codes).cuda()
                s[at[0], :, at[1]] = torch.from_numpy(scale).cuda()
                per.append(ao.mx8_values(codes, scale))
            else:
                y = torch.from_numpy(y.astype(np.float32)).to(x.dtype)
                x[at[0], :, at[1]] = y.cuda()
                per.append(y.double().numpy())
        values.append(per)
    return c, values


@pytest.mark.parametrize("dtype,held,out", (("fp32", "fp32", "fp32"), ("bf16", "bf16", "bf16"), ("bf16", "bf16", "fp32"), ("fp32", "mx8", "fp32"),
                                            ("bf16", "mx8", "bf16"), ("bf16", "mx8", "fp32")))
@pytest.mark.parametrize("dim,heads,kv,page", ((32, 6, 6, 16), (64, 8, 2, 64), (128, 24, 2, 32)))
@pytest.mark.parametrize("tokens,causal", ((1, True), (3, True), (7, False)))
def test_paged(ctx, dtype, held, out, dim, heads, kv, page, tokens, causal):
    import torch
    rng = np.random.default_rng(dim + tokens)
    lens = [0, 1, 2, 15, 16, 17, 33, 64, 255, 256, 257, 300, 700]
    c, values = filled(rng, held, lens, kv, page, dim, 1.3)
    B = len(lens)
    q = draw(rng, (B * tokens, heads + 1, dim), dtype, 1.3)[:, 1:]
    lse = torch.full((B * tokens, heads), 7.0, device="cuda")
    wide = torch.full((B * tokens, heads + 2, dim), 7.0, dtype=torch_dtype(out), device="cuda")
    ctx.tsdp_attend_paged(q, c, i32(lens), max(lens), tokens=tokens, causal=causal, scale=0.13, out=wide[:, 1:-1], lse=lse)
    for b, n in enumerate(lens):
        r = slice(b * tokens, (b + 1) * tokens)
        ref = ao.attend(f64(q[r]), values[0][b], values[1][b], 0.13, causal)
        check(wide[r, 1:-1], lse[r], ref, dim, n, out, WEIGHTS["paged"][out], (b, n))
    assert (wide[:, 0] == 7).all() and (wide[:, -1] == 7).all()
    assert ctx.tsdp_status() == 0


@pytest.mark.parametrize("dtype,held", (("fp32", "fp32"), ("bf16", "mx8")))
def test_paged_long(ctx, dtype, held):
    """Lengths around the one at which chunks grow; a row's result is the same alone and with another bound of the lengths."""
    import torch
    rng = np.random.default_rng(8)
    lens = [16383, 20001, 16385, 1025]
    c, values = filled(rng, held, lens, 1, 256, 64)
    q = draw(rng, (4, 4, 64), dtype)
    got = ctx.tsdp_attend_paged(q, c, i32(lens), 20001)
    for b, n in enumerate(lens):
        check(got[b:b + 1], None, ao.attend(f64(q[b:b + 1]), values[0][b], values[1][b], 0.125, True), 64, n, dtype, WEIGHTS["paged"][dtype], n)
    from paper_2512_15773_amd import KvCache
    for b in range(4):
        one = KvCache(c.k, c.v, c.page_table[b:b + 1], c.k_scale, c.v_scale)
        for most in (lens[b], 200000):
            assert torch.equal(ctx.tsdp_attend_paged(q[b:b + 1], one, i32([lens[b]]), most), got[b:b + 1])
    assert ctx.tsdp_status() == 0


@pytest.mark.parametrize("dtype,held", (("fp32", "fp32"), ("bf16", "mx8")))
def test_paged_long_many_columns(ctx, dtype, held):
    """As above for 36 columns, on both sides of the chunks that one set of lanes joins."""
    import torch
    rng = np.random.default_rng(18)
    lens, tokens = [16384, 17500, 16385, 5, 1025], 9
    c, values = filled(rng, held, lens, 1, 256, 64)
    q = draw(rng, (len(lens) * tokens, 4, 64), dtype)
    lse = torch.zeros(len(lens) * tokens, 4, device="cuda")
    got = ctx.tsdp_attend_paged(q, c, i32(lens), 17500, tokens=tokens, lse=lse)
    for b, n in enumerate(lens):
        r = slice(b * tokens, (b + 1) * tokens)
        check(got[r], lse[r], ao.attend(f64(q[r]), values[0][b], values[1][b], 0.125, True), 64, n, dtype, WEIGHTS["paged"][dtype], n)
    from paper_2512_15773_amd import KvCache
    for b in (0, 2, 4):
        one, r = KvCache(c.k, c.v, c.page_table[b:b + 1], c.k_scale, c.v_scale), slice(b * tokens, (b + 1) * tokens)
        for most in (lens[b], 60000):
            assert torch.equal(ctx.tsdp_attend_paged(q[r], one, i32([lens[b]]), most, tokens=tokens), got[r]), (b, most)
    assert ctx.tsdp_status() == 0


@pytest.mark.parametrize("held", ("bf16", "mx8"))
def test_pools_past_32_bits(ctx, held):
    """The last pages of pools of more than 2^32 bytes (8 bits) and 2^32 elements' bytes: written, attended to and read back."""
    import torch
    from paper_2512_15773_amd import KvCache
    kv, page, dim = 8, 256, 128
    pages = (1 << 32) // (kv * page * dim) + 5
    table = torch.tensor([[pages - 1, pages - 3], [0, pages - 2]], dtype=torch.int32, device="cuda")
    shape = (pages, kv, page, dim)
    if held == "mx8":
        pools = [torch.empty(shape, dtype=torch.uint8, device="cuda") for _ in "kv"] + [torch.empty(shape[:3] + (4,), dtype=torch.uint8, device="cuda") for _ in "kv"]
    else:
        pools = [torch.empty(shape, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    c = KvCache(pools[0], pools[1], table, *pools[2:])
    rng = np.random.default_rng(9)
    lens = [400, 512]
    ptr = i32([0, 400, 912])
    k, v = draw(rng, (912, kv, dim), "bf16"), draw(rng, (912, kv, dim), "bf16")
    ctx.tsdp_cache_write(c, ptr, i32([0, 0]), k, v)
    bk, bv = ctx.tsdp_cache_read(c, ptr, i32([0, 0]), 912, torch.float32)
    if held == "bf16":
        assert torch.equal(bk, k.float()) and torch.equal(bv, v.float())
    q = draw(rng, (2, kv, dim), "bf16")
    got = ctx.tsdp_attend_paged(q, c, i32(lens), 512)
    for b, r in ((0, slice(0, 400)), (1, slice(400, 912))):
        check(got[b:b + 1], None, ao.attend(f64(q[b:b + 1]), f64(bk[r]), f64(bv[r]), dim ** -0.5, True), dim, lens[b], "bf16", WEIGHTS["paged"]["bf16"], b)
    assert ctx.tsdp_status() == 0


@pytest.mark.parametrize("dtype,held", (("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "mx8")))
def test_paged_hides_what_is_masked(ctx, dtype, held):
    """A value that is not finite at the third of four new tokens: the first two are bit-equal to a run without it, the others
    are not finite there.  A page outside the pool is not attended to."""
    import torch
    rng = np.random.default_rng(10)
    n, tokens, dim = 301, 4, 64
    c, values = filled(rng, held, [n], 2, 64, dim)
    q = draw(rng, (tokens, 4, dim), dtype)
    clean = ctx.tsdp_attend_paged(q, c, i32([n]), n, tokens=tokens)
    page, t = int(c.page_table[0, 299 // 64]), 299 % 64
    old = c.v[page, 1, t, 5].clone()
    c.v[page, 1, t, 5] = 127 if held == "mx8" else float("inf")
    got = ctx.tsdp_attend_paged(q, c, i32([n]), n, tokens=tokens)
    c.v[page, 1, t, 5] = old
    assert torch.equal(got[:2], clean[:2]) and torch.equal(got[:, :2], clean[:, :2])
    assert not np.isfinite(f64(got[2:, 2:, 5])).any()
    assert torch.equal(got[2:, 2:, 6:], clean[2:, 2:, 6:]) and torch.equal(got[2:, 2:, :5], clean[2:, 2:, :5])
    c.page_table[0, 1] = -7
    got = ctx.tsdp_attend_paged(q[:1], c, i32([n]), n)
    assert ctx.tsdp_status() == 64
    keep = [i for i in range(n) if i // 64 != 1]
    check(got, None, ao.attend(f64(q[:1]), values[0][0][keep], values[1][0][keep], dim ** -0.5, True), dim, n, dtype, WEIGHTS["paged"][dtype], "page")


def test_paged_lengths_beyond_their_bound_are_clipped_and_reported(ctx):
    rng = np.random.default_rng(11)
    c, values = filled(rng, "bf16", [64, 64, 64], 2, 16, 32)
    q = draw(rng, (3, 2, 32), "bf16")
    got = ctx.tsdp_attend_paged(q, c, i32([50, 2 ** 31 - 1, -4]), 60)
    assert ctx.tsdp_status() == 32
    for b, n in ((0, 50), (1, 60), (2, 0)):
        check(got[b:b + 1], None, ao.attend(f64(q[b:b + 1]), values[0][b][:n], values[1][b][:n], 32 ** -0.5, True), 32, n, "bf16", WEIGHTS["paged"]["bf16"], b)
    got = ctx.tsdp_attend_paged(q, c, i32([64, 64, 2000]), 100000)              # past the table: 64 positions
    assert ctx.tsdp_status() == 32
    check(got[2:], None, ao.attend(f64(q[2:]), values[0][2], values[1][2], 32 ** -0.5, True), 32, 64, "bf16", WEIGHTS["paged"]["bf16"], "table")


# ---- what the above leaves open: many columns over several chunks, maxima that move, hidden memory, extremes

def put(c, which, b, rows):
    """rows [n, kv, dim] (float64) to positions 0 .. of environment b, as the cache holds them; returns the held values."""
    import torch
    page, n = c.k.shape[2], rows.shape[0]
    x, s = ((c.k, c.k_scale), (c.v, c.v_scale))[which]
    table = c.page_table.cpu().numpy()
    at = (torch.from_numpy(table[b, np.arange(n) // page]).long().cuda(), torch.from_numpy(np.arange(n) % page).cuda())
    if s is None:
        y = torch.from_numpy(rows.astype(np.float32)).to(x.dtype)
        x[at[0], :, at[1]] = y.cuda()
        return y.double().numpy()
    codes, scale = ao.mx8(rows)
    x[at[0], :, at[1]] = torch.from_numpy(codes).cuda()
    s[at[0], :, at[1]] = torch.from_numpy(scale).cuda()
    return ao.mx8_values(codes, scale)


KINDS = (("fp32", "fp32", "fp32"), ("bf16", "bf16", "bf16"), ("bf16", "bf16", "fp32"), ("fp32", "mx8", "fp32"), ("bf16", "mx8", "bf16"), ("bf16", "mx8", "fp32"))


@pytest.mark.parametrize("dtype,held,out", KINDS)
@pytest.mark.parametrize("dim,heads,kv,tokens,page", ((32, 6, 2, 9, 16), (64, 4, 1, 33, 64), (128, 8, 4, 9, 128)))
@pytest.mark.parametrize("causal", (True, False))
def test_paged_many_columns(ctx, dtype, held, out, dim, heads, kv, tokens, page, causal):
    """18, 27 and 132 columns of a kv head, over lengths of none to several chunks."""
    import torch
    rng = np.random.default_rng(dim * 3 + tokens)
    lens = [0, 1, tokens - 1, tokens + 1, 31, 32, 33, 130, 1023, 1024, 1025, 2100]
    c, values = filled(rng, held, lens, kv, page, dim, 1.3)
    B = len(lens)
    q = draw(rng, (B * tokens, heads, dim), dtype, 1.3)
    lse = torch.full((B * tokens, heads), 7.0, device="cuda")
    got = ctx.tsdp_attend_paged(q, c, i32(lens), max(lens), tokens=tokens, causal=causal, scale=0.13, out_dtype=torch_dtype(out), lse=lse)
    for b, n in enumerate(lens):
        r = slice(b * tokens, (b + 1) * tokens)
        check(got[r], lse[r], ao.attend(f64(q[r]), values[0][b], values[1][b], 0.13, causal), dim, n, out, WEIGHTS["paged"][out], (b, n))
    from paper_2512_15773_amd import KvCache
    for b in (3, 9, 11):                                     # alone, and with another bound of the lengths
        one, r = KvCache(c.k, c.v, c.page_table[b:b + 1], c.k_scale, c.v_scale), slice(b * tokens, (b + 1) * tokens)
        for most in (lens[b], 40000):
            again = ctx.tsdp_attend_paged(q[r], one, i32([lens[b]]), most, tokens=tokens, causal=causal, scale=0.13, out_dtype=torch_dtype(out))
            assert torch.equal(again, got[r]), (b, most)
    assert ctx.tsdp_status() == 0


@pytest.mark.parametrize("dtype,held,out", KINDS)
@pytest.mark.parametrize("dim", (32, 64, 128))
@pytest.mark.parametrize("tokens", (1, 9))
@pytest.mark.parametrize("n", (300, 1400))
def test_paged_over_large_scores_and_far_maxima(ctx, dtype, held, out, dim, tokens, n):
    """Scores of some hundreds that grow and fall along the keys: maxima move often for one head and never for the other."""
    rng = np.random.default_rng(n + dim)
    k = rng.standard_normal((n, 1, dim)) * 0.2
    k[:, 0, 0] = np.concatenate([np.linspace(-30, 30, n // 2), np.linspace(30, -30, n - n // 2)])
    q = rng.standard_normal((tokens, 2, dim)) * 0.2
    q[:, 0, 0], q[:, 1, 0] = 10.0, -10.0
    c = new_cache(rng, held, 1, -(-n // 64), 1, 64, dim)
    import torch
    k, v = put(c, 0, 0, k), put(c, 1, 0, rng.standard_normal((n, 1, dim)))
    q = torch.from_numpy(q.astype(np.float32)).to(torch_dtype(dtype)).cuda()
    for causal in (True, False):
        lse = torch.zeros(tokens, 2, device="cuda")
        got = ctx.tsdp_attend_paged(q, c, i32([n]), n, tokens=tokens, causal=causal, scale=1.0, out_dtype=torch_dtype(out), lse=lse)
        check(got, lse, ao.attend(f64(q), k, v, 1.0, causal), dim, n, out, WEIGHTS["paged"][out], causal)


LOST = 70                                                    # first keys whose scores are all -infinity


def lost_keys(rng, n, dim):
    """Queries and keys: the first scores overflow to -infinity, the others are near -300 (a power of two that fp32 does not hold)."""
    k = rng.standard_normal((n, 1, dim)) * 0.3
    k[:LOST, 0, 0], k[LOST:, 0, 0], k[:, 0, 1] = -1e20, 0.0, -300.0
    q = rng.standard_normal((n, 2, dim)) * 0.3
    q[:, :, 0], q[:, :, 1] = 1e20, 1.0
    return q, k


@pytest.mark.parametrize("dtype", ("fp32", "bf16"))
@pytest.mark.parametrize("n,dim", ((200, 32), (200, 64), (500, 64), (300, 128)))
def test_prompt_whose_first_scores_overflow(ctx, dtype, n, dim):
    """Weights of zero: the result is that of the other keys."""
    import torch
    rng = np.random.default_rng(n + dim)
    to = lambda x: torch.from_numpy(x.astype(np.float32)).to(torch_dtype(dtype)).cuda()
    q, k = (to(x) for x in lost_keys(rng, n, dim))
    v, lse = draw(rng, (n, 1, dim), dtype), torch.zeros(n, 2, device="cuda")
    got = ctx.tsdp_attend_prompt(q, k, v, i32([0, n]), causal=False, scale=1.0, lse=lse)
    check(got, lse, ao.attend(f64(q), f64(k)[LOST:], f64(v)[LOST:], 1.0, False), dim, n, dtype, WEIGHTS["prompt"][dtype], n)


@pytest.mark.parametrize("dtype,held,out", KINDS)
@pytest.mark.parametrize("dim", (32, 64, 128))
@pytest.mark.parametrize("tokens,n", ((1, 300), (1, 1400), (9, 300), (9, 1400)))
def test_paged_whose_first_scores_overflow(ctx, dtype, held, out, dim, tokens, n):
    import torch
    rng = np.random.default_rng(n + dim + tokens)
    q, k = lost_keys(rng, n, dim)
    if held == "mx8":                                        # next to 1e20 a block holds nothing else, -300 is lost there: no key but
        k[:LOST, 0, 2:] = 0.0                                # the first ones has to be exact
    c = new_cache(rng, held, 1, -(-n // 64), 1, 64, dim)
    k, v = put(c, 0, 0, k), put(c, 1, 0, rng.standard_normal((n, 1, dim)))
    q, lse = torch.from_numpy(q[:tokens].astype(np.float32)).to(torch_dtype(dtype)).cuda(), torch.zeros(tokens, 2, device="cuda")
    got = ctx.tsdp_attend_paged(q, c, i32([n]), n, tokens=tokens, causal=False, scale=1.0, out_dtype=torch_dtype(out), lse=lse)
    check(got, lse, ao.attend(f64(q), k[LOST:], v[LOST:], 1.0, False), dim, n, out, WEIGHTS["paged"][out], n)


@pytest.mark.parametrize("dtype,held,out", KINDS)
@pytest.mark.parametrize("dim", (32, 64, 128))
@pytest.mark.parametrize("tokens", (2, 12))
def test_paged_memory_behind_a_length_stays_hidden(ctx, dtype, held, out, dim, tokens):
    """Whatever the places behind a sequence in its last page hold, the result is bit-equal."""
    import torch
    rng = np.random.default_rng(dim + tokens)
    n = 1024 + 70                                            # ends inside a page, 6 places into a tile
    c, _ = filled(rng, held, [n], 2, 256, dim)
    q = draw(rng, (tokens, 4, dim), dtype)
    run = lambda: ctx.tsdp_attend_paged(q, c, i32([n]), n, tokens=tokens, out_dtype=torch_dtype(out))
    clean, page = run(), int(c.page_table[0, n // 256])
    assert torch.isfinite(clean).all()
    pools = [x[page][:, n % 256:] for x in (c.k, c.v)]
    if held == "mx8":
        scales = [x[page][:, n % 256:] for x in (c.k_scale, c.v_scale)]
        for code, scale in ((0x7E, 255), (0x7E, 254), (0xFE, 248), (0, 255), (0x7F, 0), (0x7E, 246), (1, 255)):
            for x, s in zip(pools, scales):
                x.fill_(code); s.fill_(scale)
            assert torch.equal(run(), clean), (code, scale)
    else:
        for bad in (float("inf"), -float("inf"), float("nan"), torch.finfo(pools[0].dtype).max, torch.finfo(pools[0].dtype).min):
            for x in pools:
                x.fill_(bad)
            assert torch.equal(run(), clean), bad


@pytest.mark.parametrize("dtype,held", (("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "mx8"), ("fp32", "mx8")))
@pytest.mark.parametrize("dim", (32, 64, 128))
def test_paged_many_columns_hide_what_is_masked(ctx, dtype, held, dim):
    """As for few columns: a value that is not finite reaches the tokens from its own on, at its own element; a page outside the
    pool is not attended to."""
    import torch
    rng = np.random.default_rng(dim)
    n, tokens, heads, own = 1024 + 301, 12, 4, 5             # the value is that of the sixth of twelve new tokens
    c, values = filled(rng, held, [n], 2, 64, dim)
    q = draw(rng, (tokens, heads, dim), dtype)
    run = lambda: ctx.tsdp_attend_paged(q, c, i32([n]), n, tokens=tokens)
    clean, pos = run(), n - tokens + own
    page, t = int(c.page_table[0, pos // 64]), pos % 64
    for e in (0, 13, dim - 1):
        old = c.v[page, 1, t, e].clone()
        c.v[page, 1, t, e] = 127 if held == "mx8" else float("inf")
        got = run()
        c.v[page, 1, t, e] = old
        rest = [i for i in range(dim) if i != e]
        assert torch.equal(got[:own], clean[:own]) and torch.equal(got[:, :2], clean[:, :2])
        assert not np.isfinite(f64(got[own:, 2:, e])).any() and torch.equal(got[own:, 2:][..., rest], clean[own:, 2:][..., rest])
    for column in (1, 17, 20):
        old = c.page_table[0, column].clone()
        c.page_table[0, column] = c.k.shape[0] + 5
        got = run()
        c.page_table[0, column] = old
        assert ctx.tsdp_status() == 64
        keep = np.array([i for i in range(n) if i // 64 != column])
        for token in (0, own, tokens - 1):
            see = keep[keep < n - tokens + 1 + token]
            check(got[token:token + 1], None, ao.attend(f64(q[token:token + 1]), values[0][0][see], values[1][0][see], dim ** -0.5, False),
                  dim, n, dtype, WEIGHTS["paged"][dtype], (column, token))


@pytest.mark.parametrize("where", ("prompt", "few", "many"))
@pytest.mark.parametrize("dim", (32, 64, 128))
def test_values_next_to_the_largest(ctx, where, dim):
    """fp32 values of +-3.4e38 at equal weights of a fourth: nothing overflows on the way to a bf16 part."""
    import torch
    rng = np.random.default_rng(dim)
    most = float(np.finfo(np.float32).max)
    n, tokens = 4, 1 if where == "few" else 4
    k = np.zeros((n, 1, dim)); v = np.zeros((n, 1, dim))
    v[0], v[2] = most, rng.standard_normal((1, dim))
    q = torch.zeros(tokens, 8, dim, device="cuda")
    if where == "prompt":
        to = lambda x: torch.from_numpy(x.astype(np.float32)).cuda()
        got = ctx.tsdp_attend_prompt(q, to(k), to(v), i32([0, 4]), causal=False)
    else:
        c = new_cache(rng, "fp32", 1, 1, 1, 16, dim)
        put(c, 0, 0, k); put(c, 1, 0, v)
        got = ctx.tsdp_attend_paged(q, c, i32([4]), 4, tokens=tokens, causal=False)
    check(got, None, ao.attend(f64(q), k, v, dim ** -0.5, False), dim, n, "fp32", WEIGHTS["paged"]["fp32"], where)


def test_memory_of_a_call_on_another_stream_is_that_streams(ctx):
    """Outputs and scratch that a call allocates for a stream it is given: nothing that the current stream still uses."""
    import torch
    rng = np.random.default_rng(20)
    c, _ = filled(rng, "bf16", [5000], 2, 64, 64)
    q, length = draw(rng, (1, 8, 64), "bf16"), i32([5000])
    p = [draw(rng, (700, h, 64), "bf16") for h in (8, 2, 2)]
    ptr, rows, zero = i32([0, 700]), i32([0, 100]), i32([0])
    calls = (lambda s: ctx.tsdp_attend_paged(q, c, length, 5000, stream=s), lambda s: ctx.tsdp_attend_prompt(*p, ptr, stream=s),
             lambda s: ctx.tsdp_cache_read(c, rows, zero, 100, torch.bfloat16, stream=s)[0])
    want = [f(None) for f in calls]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    allocated = []
    for f in calls:
        allocated.append(f(side))
        mine = [s for s in torch.cuda.memory_snapshot() if s["stream"] == side.cuda_stream]
        at = allocated[-1].data_ptr()
        assert any(s["address"] <= at < s["address"] + s["total_size"] for s in mine)
    torch.cuda.synchronize()
    for x, y in zip(allocated, want):
        assert torch.equal(x, y)


# ---- together

def test_an_episode(ctx):
    """A history as it is used: the first observations through the prompt kernel into an 8-bit cache, a chunk of later ones behind
    the history read back, a step of one token, and the observation tokens that condition a network, pooled from the history in
    fp32 -- each against 64 bits on the values the cache holds, and the conditioned network against one that is given the same tokens."""
    import torch
    from paper_2512_15773_amd import Tsdp
    rng = np.random.default_rng(12)
    wl = ti.small_variant(ti.C4, B=3, base=ti.NetShape(1, 512, 8), draft=ti.NetShape(1, 256, 8))
    B, heads, kv, dim, page = 3, 12, 4, 64, 32
    assert heads * dim == wl.cond_dim
    net = Tsdp.from_workload(wl)
    for which, name in ((0, "base"), (1, "draft")):
        net.tsdp_load_weights(which, ti.pack_blob(ti.make_weights(wl, name, b_std=0.02)))
    n = [70, 33, 129]
    held = [[], []]                                      # values of every environment as the cache holds them
    c = new_cache(rng, "mx8", B, 8, kv, page, dim)
    scale = dim ** -0.5

    def project(rows):
        qkv = draw(rng, (rows, heads + 2 * kv, dim), "bf16")
        return qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:]

    # the first observations
    ptr = np.concatenate([[0], np.cumsum(n)])
    q, k, v = project(ptr[-1])
    out = net.tsdp_attend_prompt(q, k, v, i32(ptr))
    for b in range(B):
        r = slice(ptr[b], ptr[b + 1])
        check(out[r], None, ao.attend(f64(q[r]), f64(k[r]), f64(v[r]), scale, True), dim, n[b], "bf16", WEIGHTS["prompt"]["bf16"], b)
    net.tsdp_cache_write(c, i32(ptr), i32([0] * B), k, v)
    for which, x in enumerate((k, v)):
        held[which] = [ao.mx8_values(*ao.mx8(f64(x[ptr[b]:ptr[b + 1]]))) for b in range(B)]
    # a chunk of 20 tokens each behind the history read back
    more = [20] * B
    mptr, now = np.concatenate([[0], np.cumsum(more)]), [x + 20 for x in n]
    kptr = np.concatenate([[0], np.cumsum(now)])
    q, k, v = project(60)
    net.tsdp_cache_write(c, i32(mptr), i32(n), k, v)
    for which, x in enumerate((k, v)):
        for b in range(B):
            held[which][b] = np.concatenate([held[which][b], ao.mx8_values(*ao.mx8(f64(x[20 * b:20 * b + 20])))])
    hk, hv = net.tsdp_cache_read(c, i32(kptr), i32([0] * B), int(kptr[-1]), torch.bfloat16)
    out = net.tsdp_attend_prompt(q, hk, hv, i32(mptr), i32(kptr))
    for b in range(B):
        r = slice(20 * b, 20 * b + 20)
        assert np.array_equal(f64(hk[kptr[b]:kptr[b + 1]]), held[0][b])
        check(out[r], None, ao.attend(f64(q[r]), held[0][b], held[1][b], scale, True), dim, now[b], "bf16", WEIGHTS["prompt"]["bf16"], b)
    # the same chunk over the cache itself
    paged = net.tsdp_attend_paged(q, c, i32(now), 256, tokens=20)
    for b in range(B):
        r = slice(20 * b, 20 * b + 20)
        check(paged[r], None, ao.attend(f64(q[r]), held[0][b], held[1][b], scale, True), dim, now[b], "bf16", WEIGHTS["paged"]["bf16"], b)
    # the observation tokens that condition the network, and a round on them
    q = draw(rng, (B * wl.cond_tokens, heads, dim), "bf16")
    cond = net.tsdp_attend_paged(q, c, i32(now), 256, tokens=wl.cond_tokens, causal=False, out_dtype=torch.float32)
    for b in range(B):
        r = slice(64 * b, 64 * b + 64)
        check(cond[r], None, ao.attend(f64(q[r]), held[0][b], held[1][b], scale, False), dim, now[b], "fp32", WEIGHTS["paged"]["fp32"], b)
    cond = cond.view(B, wl.cond_tokens, wl.cond_dim)
    assert net.tsdp_status() == 0
    ends = []
    for tokens in (cond, torch.from_numpy(cond.cpu().numpy()).cuda()):
        net.tsdp_set_cond(tokens)
        x, t = torch.from_numpy(ti.make_latents(wl, B)).cuda(), i32([50, 20, 3])
        net.tsdp_round(x, t, i32([4] * B), torch.ones(B, device="cuda"), None)
        ends.append((x.cpu().numpy(), t.cpu().numpy()))
    assert np.isfinite(ends[0][0]).all() and np.array_equal(ends[0][0], ends[1][0]) and np.array_equal(ends[0][1], ends[1][1])
    assert kernels(net)[0] in ("tiles", "k_flow", "k_few")
    net.close()


def test_a_step_captured_and_replayed(ctx):
    """Write, attend and read of one step as a graph: every replay against the eager calls on that step's inputs, with eager work
    and synchronizations in between."""
    import torch
    rng = np.random.default_rng(13)
    B, heads, kv, dim, page, most = 4, 8, 2, 64, 16, 600
    # four steps' room behind the first lengths: those positions hold numbers that a step overwrites
    caches = [filled(np.random.default_rng(14), "mx8", [564, 294, 21, 260], kv, page, dim)[0] for _ in range(2)]
    ptr, start, length = i32([0, 1, 2, 3, 4]), i32([560, 290, 17, 256]), i32([561, 291, 18, 257])
    q, k, v = (torch.zeros(B, h, dim, dtype=torch.bfloat16, device="cuda") for h in (heads, kv, kv))
    out, back = torch.zeros_like(q), (torch.zeros_like(k), torch.zeros_like(v))
    scratch = ctx.alloc_scratch(caches[0], heads, 1, most)

    def step(c, q, k, v, out, back, scratch):
        ctx.tsdp_cache_write(c, ptr, start, k, v)
        ctx.tsdp_attend_paged(q, c, length, most, out=out, scratch=scratch)
        ctx.tsdp_cache_read(c, ptr, start, B, torch.bfloat16, out=back)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(caches[0], q, k, v, out, back, scratch)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(caches[0], q, k, v, out, back, scratch)
    for turn in range(4):
        new = [draw(rng, x.shape, "bf16") for x in (q, k, v)]
        want, wback = torch.zeros_like(out), (torch.zeros_like(k), torch.zeros_like(v))
        step(caches[1], *new, want, wback, ctx.alloc_scratch(caches[1], heads, 1, most))
        for x, y in zip((q, k, v), new):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(back[0], wback[0]) and torch.equal(back[1], wback[1]), turn
        assert torch.isfinite(want).all() and torch.equal(caches[0].k, caches[1].k) and torch.equal(caches[0].v_scale, caches[1].v_scale)
        start += 1; length += 1
    assert ctx.tsdp_status() == 0


def test_calls_on_two_streams(ctx):
    """Prompts and steps on two streams at once, each with memory of its own: the results of the calls one after the other."""
    import torch
    rng = np.random.default_rng(16)
    c, _ = filled(rng, "bf16", [900, 300], 2, 64, 64)
    q = draw(rng, (2, 8, 64), "bf16")
    p = [draw(rng, (700, h, 64), "bf16") for h in (8, 2, 2)]
    lens, ptr = i32([900, 300]), i32([0, 200, 700])
    want = ctx.tsdp_attend_paged(q, c, lens, 900), ctx.tsdp_attend_prompt(*p, ptr)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.zeros_like(want[0]) for _ in range(8)], [torch.zeros_like(want[1]) for _ in range(8)]]
    scratch = [ctx.alloc_scratch(c, 8, 1, 900) for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(8):
        ctx.tsdp_attend_paged(q, c, lens, 900, out=outs[0][i], scratch=scratch[0], stream=streams[0])
        ctx.tsdp_attend_prompt(*p, ptr, out=outs[1][i], stream=streams[1])
    torch.cuda.synchronize()
    for which in (0, 1):
        for o in outs[which]:
            assert torch.equal(o, want[which])


def test_refusals_reach_the_caller(ctx):
    import torch
    from paper_2512_15773_amd import TsdpError
    rng = np.random.default_rng(17)
    c, _ = filled(rng, "bf16", [300], 2, 64, 64)
    q = draw(rng, (1, 4, 64), "bf16")
    for call, code in ((lambda: ctx.tsdp_attend_prompt(draw(rng, (3, 2, 48), "fp32"), draw(rng, (3, 2, 48), "fp32"), draw(rng, (3, 2, 48), "fp32"), i32([0, 3])), -2),
                       (lambda: ctx.tsdp_attend_paged(q, c, i32([300]), 300, scale=-1.0), -1),
                       (lambda: ctx.tsdp_attend_paged(q, c, i32([300]), 300, scratch=torch.empty(16, dtype=torch.uint8, device="cuda")), -2),
                       (lambda: ctx.tsdp_attend_paged(q.float(), c, i32([300]), 300), -1),
                       (lambda: ctx.alloc_scratch(c, 4, 2000, 300), -2)):
        with pytest.raises(TsdpError) as e:
            call()
        assert e.value.code == code
    for call in (lambda: ctx.tsdp_cache_write(c, i32([0, 1]), i32([0]), q.transpose(1, 2), q), lambda: ctx.tsdp_cache_write(c, i32([0, 1]), i32([0, 0]), q[:, :2], q[:, :2]),
                 lambda: ctx.tsdp_attend_prompt(q, q.cpu(), q, i32([0, 1]))):
        with pytest.raises(AssertionError):
            call()
    # nothing to do: no rows, no environments
    assert ctx.tsdp_attend_prompt(q[:0], q[:0], q[:0], i32([0])).shape == (0, 4, 64)
    ctx.tsdp_cache_write(c, i32([0, 0]), i32([0]), q[:0, :2], q[:0, :2])
    assert ctx.tsdp_status() == 0
