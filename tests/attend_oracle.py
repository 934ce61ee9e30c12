"""Attention, the cache's positions and its 8-bit values in 64 bits on the CPU, with the error bounds of the GPU tests."""
import numpy as np

U = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}              # half a step, relative


def attend(q, k, v, scale, causal):
    """q [nq, heads, dim], k / v [nk, kv, dim] in float64 -> out, lse [nq, heads], and what the bounds need: the mean of |v|
    under the weights, and the largest sum of |q k| scale of a score."""
    nq, heads, dim = q.shape
    nk, kv = k.shape[:2]
    out, lse, mean, size = np.zeros((nq, heads, dim)), np.full((nq, heads), -np.inf), np.zeros((nq, heads, dim)), np.zeros((nq, heads, 1))
    for i in range(nq):
        n = nk if not causal else min(max(nk - nq + 1 + i, 0), nk)
        if n == 0:
            continue
        for h in range(heads):
            kk, vv = k[:n, h // (heads // kv)], v[:n, h // (heads // kv)]
            s = kk @ q[i, h] * scale
            top = s.max()
            p = np.exp(s - top)
            out[i, h], lse[i, h] = p @ vv / p.sum(), top + np.log(p.sum())
            mean[i, h] = p @ np.abs(vv) / p.sum()
            size[i, h] = (np.abs(kk) @ np.abs(q[i, h])).max() * scale
    return out, lse, mean, size


def bound(out, mean, size, dim, n, out_type, weights):
    """Elementwise error bound.  weights: relative rounding of a weight for its product with the values.  A score is a sum of dim
    products in fp32 (dim + 4 roundings of sums as large as `size`, among them the scale's), its exponential doubles nothing but
    adds a few roundings and that of its argument (the distance to a maximum, at most twice the largest score); sums over n keys
    round once per key and join; the quotient and the output round once each."""
    u = 2.0 ** -24
    weight = weights + 2 * ((dim + 4) * u * size + 2 * u * (size + 12)) + 8 * u
    return U[out_type] * np.abs(out) + mean * (1 + U[out_type]) * (weight * 2 + 2 * (n + 16) * u) + 1e-30


def lse_bound(lse, size, dim, n):
    u = 2.0 ** -24
    return (dim + 4) * u * size + 2 * u * (size + 12) + (n + 24) * u + 4 * u * np.abs(np.where(np.isfinite(lse), lse, 0.0))[..., None]


def e4m3_values():
    """The 256 codes' values."""
    c = np.arange(256)
    p, f = (c >> 3) & 15, c & 7
    x = np.where(p > 0, (1 + f / 8.0) * 2.0 ** (p - 7.0), f * 2.0 ** -9)
    x = np.where((c & 127) == 127, np.nan, x)
    return np.where(c & 128, -x, x)


def mx8(x):
    """x [..., dim] (float64) -> (codes, scale bytes), from the definition: the nearest code, ties to the even one."""
    b = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    fin = np.isfinite(b)
    amax = np.where(fin, np.abs(b), 0.0).max(-1)
    e = np.full(amax.shape, -111)
    while True:
        over = amax > 448.0 * 2.0 ** e.astype(np.float64)
        if not over.any():
            break
        e = e + over
    y = np.where(fin, b, 0.0) * 2.0 ** -e[..., None].astype(np.float64)
    codes = e4m3_values()[:127]                              # the non-negative ones, growing
    at = np.searchsorted(codes, np.abs(y))
    hi = np.minimum(at, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = np.abs(y) - codes[lo], codes[hi] - np.abs(y)
    c = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    c = np.where(np.abs(y) == codes[hi], hi, c)
    c = c | np.where(np.signbit(b) & fin, 128, 0)
    c = np.where(fin, c, 127)
    return c.reshape(x.shape).astype(np.uint8), (e + 127).astype(np.uint8)


def mx8_values(codes, scale):
    x = e4m3_values()[codes].reshape(*scale.shape, 32) * 2.0 ** (scale.astype(np.float64) - 127)[..., None]
    return x.reshape(codes.shape)
