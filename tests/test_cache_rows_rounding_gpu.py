"""Rows read from the 4-bit cache are m + s code rounded once, for every s and m."""
import numpy as np
import pytest
import torch

from attention_cache_forms import DT

pytestmark = pytest.mark.gpu


def nearest_bf16(x):
    """float64 numbers rounded to bf16 (ties to even), as float64."""
    f, e = np.frexp(x)                                  # |f| in [1/2, 1)
    step = np.exp2(np.maximum(e, -125) - 8.0)           # (the least bf16 number is 2^-133)
    y = np.rint(x / step) * step                        # (powers of two: exact)
    return np.where(np.abs(y) >= 2.0 ** 128, np.copysign(np.inf, x), y)


def nearest(x, dtype):
    if dtype == "bf16":
        return nearest_bf16(x)
    with np.errstate(over="ignore"):
        return x.astype({"fp16": np.float16, "fp32": np.float32}[dtype]).astype(np.float64)


def test_the_plain_rounding():
    x = np.array([1.0, 1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, -(1 + 2.0 ** -8 + 2.0 ** -40), 2.0 ** -133, 2.0 ** -134, 3e38, 3.4e38])
    want = [1.0, 1.0, 1 + 2.0 ** -6, -(1 + 2.0 ** -7), 2.0 ** -133, 0.0]
    got = nearest_bf16(x)
    assert got[:6].tolist() == want and got[-1] == np.inf and np.isfinite(got[-2])


def cache_of(s, m, codes):
    """A cache of one head x 64 channels that holds codes (tokens, 64) with s, m (tokens,) for keys and
    values (uint16 arrays of bf16 bits)."""
    import paper_2609_04910_gb300 as gs
    n = len(s)
    cache = gs.attention_cache(1, n, 1, 64)
    pair = np.stack([s, m], -1).astype("<u2").view(np.uint8).reshape(n, 4)
    words = {"k": np.zeros((n, 32), np.uint8), "v": np.zeros((n, 32), np.uint8)}
    for ch in range(64):
        j, inside = ch // 32, ch % 32
        t, p = inside // 8, inside % 8
        words["k"][:, (t * 2 + j) * 4 + p // 2] |= codes[:, ch] << (4 * (p % 2))
        g, p = inside // 4, inside % 4
        words["v"][:, (g * 2 + j) * 2 + p // 2] |= codes[:, ch] << (4 * (p % 2))
    block = np.concatenate([words[x].reshape(n // 16, 512) for x in "kv"] + [pair.reshape(n // 16, 64)] * 2, -1)
    cache.data.copy_(torch.from_numpy(block).view(1, 1, n // 16, 1152).cuda())
    return cache


def bits(x):
    return (np.asarray(x, dtype=np.float32).view(np.uint32) >> 16).astype(np.uint16)


def pairs(rng, n):
    """Steps and least values (bits), near and far from each other and from the types' ends."""
    e = rng.integers(-30, 13, n)
    s = np.ldexp(1 + rng.integers(0, 128, n) / 128.0, e)
    near = np.ldexp(1 + rng.integers(0, 128, n) / 128.0, e + rng.integers(-40, 12, n))
    m = np.where(rng.random(n) < 0.1, 0.0, near * rng.choice([-1.0, 1.0], n))
    m = np.where(rng.random(n) < 0.2, -8.0 * s, m)
    s, m = np.concatenate([s[:-5], [139 * 2.0 ** -11, 0.0, 2.0 ** -126, 2.0 ** 100, 4384.0]]), \
        np.concatenate([m[:-5], [2.0 ** -40, 3.0, -2.0 ** -126, -2.0 ** 101, 0.0]])
    return bits(s), bits(m)


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
def test_rows_are_rounded_once(dtype):
    import paper_2609_04910_gb300 as gs
    rng = np.random.default_rng(7)
    n = 1 << 14
    s, m = pairs(rng, n)
    codes = rng.integers(0, 16, (n, 64), dtype=np.uint8)
    codes[:, :16] = np.arange(16)
    cache = cache_of(s, m, codes)
    value = [(x.astype(np.uint32) << 16).view(np.float32).astype(np.float64)[:, None] for x in (s, m)]
    # (Exact in float64: at most 12 bits of s code and 8 of m, or so far apart that the smaller one only breaks ties.)
    want = nearest(value[1] + value[0] * codes, dtype)
    for rows in gs.gauss_sum_cache_read(cache, n, DT[dtype]):
        got = rows[0, :, 0].double().cpu().numpy()
        bad = (got != want).any(-1)
        assert not bad.any(), (int(bad.sum()), s[bad][:4], m[bad][:4])
