"""The 4-bit cache where sizes of numbers change within a call: values that grow along a
sequence, scores that vanish, rows that see few keys of a cache with much room."""
import math

import pytest
import torch

from attention_cache_forms import DT, attention64, quantise, values, within
from test_attention_cache_gpu import Store, filled, path_of
from test_attention_gpu import ints, points

pytestmark = pytest.mark.gpu


def sizes_of(k, v):
    """|m| + s code of keys and |m| + 15 s of values, as Store keeps them."""
    kq, vq = quantise(k), quantise(v)
    size = vq[2].double().abs() + 15 * vq[1].double()
    return values(kq[0], kq[1], kq[2].abs()), size[..., torch.arange(v.shape[-1], device=v.device) // 64]


def check(s, k, v, q, tau, causal=True, kl=None, path=None, dims=None):
    """Writes k and v into s and holds attention over it against float64."""
    import paper_2609_04910_gb300 as gs
    s.write(k, v, kl=kl)
    k_size, size = sizes_of(k, v)
    B, M, H, D = q.shape
    path = path or path_of(M, H, s.Hk, D, s.C, dims)
    want = attention64(q, s.k, s.v, k_size, size, tau, causal, k_lengths=ints(kl), path=path)
    out, lse = gs.gauss_sum_attention_cached(q, s.cache, tau, causal=causal, k_lengths=ints(kl), page_table=s.table)
    gs.gauss_sum_device_status()
    worst = within(held(out, want["out"]), want["out"]), within(lse, want["lse"])
    assert max(worst) <= 1, worst


def held(out, want):
    """out, with the exact value for an infinity that a right result may be: fp16 numbers end at 65504,
    and from 65520 on the nearest one is infinity."""
    value, bound = want
    if out.dtype != torch.float16:
        return out
    past = out.isinf() & (value.abs() + bound >= 65520) & (out.sign() == value.sign())
    return torch.where(past, value, out.double())


@pytest.mark.parametrize("first,then", [(None, 30), (None, 90), (-110, 30), (-120, 100), (-60, 60), (90, -90)])
@pytest.mark.parametrize("M", [1, 3, 40, 300])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_values_that_grow(first, then, M, dtype):
    """Tokens of zeros (or very small values), then tokens of 2^30 and more: the weights of
    the first ones stay in the sum."""
    B, N, H, Hk, D = 2, 1024, 4, 2, 64
    s = Store(B, N, Hk, D, D, 32, seed=1)
    k, v = points((B, N, Hk, D), "fp32", 2), points((B, N, Hk, D), "fp32", 3)
    v[:, :600] *= 0.0 if first is None else 2.0 ** first
    v[:, 600:] *= 2.0 ** then
    check(s, k, v, points((B, M, H, D), dtype, 4), 0.125, dims=dtype)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("q_scale,k_scale", [(0.0, 0.0), (2.0 ** -12, 0.0), (0.0, 1.0), (1.0, 0.0), (2.0 ** -60, 2.0 ** -60),
                                             (2.0 ** -14, 2.0 ** -110)])
@pytest.mark.parametrize("M", [1, 40, 300])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_scores_that_vanish(q_scale, k_scale, M, dtype, causal):
    """Queries and keys of zeros, or whose products are below float32's least number: all keys
    that a query sees weigh the same, the others nothing."""
    B, N, H, Hk, D = 3, 700, 4, 2, 64
    s = Store(B, N, Hk, D, D, 32, seed=1)
    k, v = points((B, N, Hk, D), "fp32", 2) * k_scale, points((B, N, Hk, D), "fp32", 3)
    check(s, k, v, points((B, M, H, D), dtype, 4, scale=q_scale), 0.125, causal, [700, 650, 333], dims=dtype)


@pytest.mark.parametrize("M", [1, 40, 300])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_an_empty_cache_as_it_is_made(M, dtype):
    """Values 0 wherever a query looks: out 0, lse the logarithm of the number of keys."""
    import paper_2609_04910_gb300 as gs
    cache = gs.attention_cache(2, 1024, 2, 64)
    q = torch.zeros(2, M, 4, 64, dtype=DT[dtype], device="cuda")
    q[:, M // 2:] = 2.0 ** -12
    out, lse = gs.gauss_sum_attention_cached(q, cache, 0.125, causal=True, k_lengths=ints([1000, 321]))
    gs.gauss_sum_device_status()
    assert not bool(out.any())
    for b, n in enumerate((1000, 321)):
        for m in range(M):
            seen = n - M + m + 1
            want = math.log(seen)
            assert bool(((lse[b, :, m].double() - want).abs() <= 2.0 ** -21 + 2.0 ** -22 * want).all()), (b, m)


def test_weights_of_a_long_run_of_zero_values():
    """1.7e8 keys (a table that repeats a page) whose scores are 5.9 log2 units above the first ones':
    a warp's sum of some 1e5 weights of 2^5.9 stays in float32's range.  lse is off by at most
    2^-24 for each of the 2^14 additions of a lane."""
    import paper_2609_04910_gb300 as gs
    T, D, pages = 4096, 32, 41800
    cache = gs.attention_cache(2, T, 1, D)
    score = 4.09375                                     # (a bf16 number)
    rows = torch.full((1, T, 1, D), score, device="cuda")
    high = ints([1])[None]
    gs.gauss_sum_cache_write(cache, rows, torch.zeros_like(rows), page_table=high)
    table = torch.ones(1, pages, dtype=torch.int32, device="cuda")
    table[0, 0] = 0
    q = torch.ones(1, 1, 1, D, device="cuda")
    out, lse = gs.gauss_sum_attention_cached(q, cache, 1 / D, page_table=table)
    gs.gauss_sum_device_status()
    want = math.log(T + (pages - 1) * T * math.exp(score))
    assert not bool(out.any())
    assert abs(float(lse) - want) <= 2.0 ** -10, (float(lse), want)


@pytest.mark.parametrize("k_exp,q_exp,v_scale", [(20, -20, 1.0), (90, -20, 1.0), (-60, 12, 1.0), (0, 0, 3e5), (0, 0, 1e-6)])
@pytest.mark.parametrize("M", [1, 20, 200])
@pytest.mark.parametrize("D,C", [(160, 160), (256, 64), (64, 200)])
def test_fp16_queries_of_wide_heads(D, C, M, k_exp, q_exp, v_scale):
    """Keys and values outside fp16 numbers' range: what is read back of them is scaled."""
    B, N, H, Hk = 2, 700, 4, 2
    s = Store(B, N, Hk, D, C, 32, seed=1)
    k, v = points((B, N, Hk, D), "fp32", 2) * 2.0 ** k_exp, points((B, N, Hk, C), "fp32", 3) * v_scale
    q = points((B, M, H, D), "fp16", 4, scale=2.0 ** q_exp)
    check(s, k, v, q, D ** -0.5 * 2.0 ** -(k_exp + q_exp), False, [700, 650], path="many")


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("M,H,held,room", [(17, 2, 17, 8192), (9, 4, 20, 300), (64, 8, 70, 4096), (130, 4, 130, 272),
                                           (250, 4, 250, 8192), (40, 4, 260, 8192), (250, 4, 1000, 1008)])
@pytest.mark.parametrize("D,C", [(64, 64), (128, 128), (100, 36), (33, 128)])
def test_few_keys_in_a_wide_cache(M, H, held, room, D, C, dtype):
    """The log-sum-exp of rows that see few keys, whatever the cache has room for: no rounding of
    a key is left to average away (2^-21 of the sizes of a score's terms, as for few rows)."""
    import paper_2609_04910_gb300 as gs
    s = filled(2, room, 2, D, C, 16, M, [held, (held + 1) // 2])
    kl = ints([held, (held + 1) // 2])
    q = points((2, M, H, D), dtype, M)
    tau = D ** -0.5
    out, lse = gs.gauss_sum_attention_cached(q, s.cache, tau, causal=True, k_lengths=kl, page_table=s.table)
    gs.gauss_sum_device_status()
    want = attention64(q, s.k, s.v, s.k_size, s.size, tau, True, k_lengths=kl, path="many")
    exact = attention64(q, s.k, s.v, s.k_size, s.size, tau, True, k_lengths=kl, path="few")
    worst = within(out, want["out"]), within(lse, exact["lse"])
    assert max(worst) <= 1, worst


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("B,M,H,Hk,D,N", [(2, 300, 4, 2, 64, 300), (1, 600, 8, 2, 128, 700), (2, 520, 4, 2, 33, 1000),
                                          (3, 257, 16, 4, 100, 2000)])
def test_few_keys_of_calls_that_fit_the_card(B, M, H, Hk, D, N, dtype):
    """More than 512 rows, but few enough tiles that nothing is read back: keys are exact, and so
    is lse of the first rows of a prompt."""
    import paper_2609_04910_gb300 as gs
    kl = [M + b for b in range(B)]
    s = filled(B, N, Hk, D, D, 16, M, kl)
    q = points((B, M, H, D), dtype, M)
    tau = D ** -0.5
    out, lse = gs.gauss_sum_attention_cached(q, s.cache, tau, causal=True, k_lengths=ints(kl), page_table=s.table)
    gs.gauss_sum_device_status()
    args = q, s.k, s.v, s.k_size, s.size, tau, True, None, ints(kl)
    want, exact = attention64(*args, path="many"), attention64(*args, path="few")
    worst = within(out, want["out"]), within(lse, exact["lse"])
    assert max(worst) <= 1, worst


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("M,H,D,ql,kl", [(700, 64, 64, [700, 300], [700, 300]), (600, 64, 128, [600, 411], [600, 17]),
                                         (2500, 16, 100, [2500, 0], [2500, 256])])
def test_rows_read_back_of_short_sequences(M, H, D, ql, kl, causal, dtype):
    """Calls with more tiles than that, some of whose rows see few keys (rounded to 11 bits)."""
    import paper_2609_04910_gb300 as gs
    s = filled(2, M, 2, D, D, 16, M, kl)
    q = points((2, M, H, D), dtype, M)
    out, lse = gs.gauss_sum_attention_cached(q, s.cache, 0.1, causal=causal, q_lengths=ints(ql), k_lengths=ints(kl),
                                             page_table=s.table)
    gs.gauss_sum_device_status()
    want = attention64(q, s.k, s.v, s.k_size, s.size, 0.1, causal, ints(ql), ints(kl), path="many")
    worst = within(out, want["out"]), within(lse, want["lse"])
    assert max(worst) <= 1, worst
