"""Each of the three ways that attention over the 4-bit cache is computed (few rows, tiles, rows read
back first), on caches with room for more than 256 tokens."""
import pytest
import torch

from attention_cache_forms import attention64, within
from test_attention_cache_gpu import Store, filled, path_of
from test_attention_gpu import ints, points

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("M,kl", [(1, 600), (40, 600), (300, 600), (300, 300)])
@pytest.mark.parametrize("side", ["k", "v"])
def test_nan_tokens(side, M, kl, dtype, causal):
    """A token with a NaN makes the queries that see it NaN; other heads and problems are untouched."""
    import paper_2609_04910_gb300 as gs
    s = Store(2, 600, 2, 64, 64, 16, seed=3)
    x = {"k": points((2, 600, 2, 64), dtype, 1), "v": points((2, 600, 2, 64), dtype, 2)}
    x[side][1, kl - 50, 0, 3] = float("nan")
    s.write(x["k"], x["v"], kl=[600, 600])
    q = points((2, M, 4, 64), dtype, 5)
    args = dict(causal=causal, k_lengths=ints([kl, kl]), page_table=s.table)
    out, lse = gs.gauss_sum_attention_cached(q, s.cache, 0.125, **args)
    gs.gauss_sum_device_status()
    assert bool(out[0].isfinite().all()) and bool(out[1, :, 2:].isfinite().all())
    assert bool(lse[0].isfinite().all()) and bool(lse[1, 2:].isfinite().all())
    sees = slice(max(0, M - 50), M) if causal else slice(0, M)
    assert bool(out[1, sees, :2].isnan().all())
    if side == "k":
        assert bool(lse[1, :2, sees].isnan().all())
    # Past the lengths the token is not looked at.
    args["k_lengths"] = ints([kl, kl - 50])
    out, lse = gs.gauss_sum_attention_cached(q[:, :M], s.cache, 0.125, **args)
    assert bool(out.isfinite().all()) and not bool(lse.isnan().any())


@pytest.mark.parametrize("M", [1, 33, 300])
def test_slices_of_a_pool(M):
    """A cache whose pages and heads are a part of a larger array."""
    import paper_2609_04910_gb300 as gs
    whole = gs.attention_cache(10, 320, 6, 64, 32)
    part = gs.AttentionCache(whole.data[2:8:2, 1:5], 64, 32)
    plain = gs.attention_cache(3, 320, 4, 64, 32)
    k, v = points((3, 320, 4, 64), "fp16", 1), points((3, 320, 4, 32), "fp16", 2)
    for c in (part, plain):
        gs.gauss_sum_cache_write(c, k, v)
    assert torch.equal(part.data, plain.data)
    q = points((3, M, 8, 64), "fp16", M)
    got = [gs.gauss_sum_attention_cached(q, c, 0.125, causal=True) for c in (part, plain)]
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


@pytest.mark.parametrize("M", [1, 40, 300])
def test_no_tokens(M):
    import paper_2609_04910_gb300 as gs
    c = gs.attention_cache(2, 320, 2, 64)
    c.data.fill_(0xFF)                                  # (NaN groups that nothing may look at)
    q = points((2, M, 4, 64), "bf16", 3)
    for kl in ([0, 0], [-5, 0]):
        out, lse = gs.gauss_sum_attention_cached(q, c, 0.125, causal=True, k_lengths=ints(kl))
        assert not bool(out.any()) and bool((lse == -float("inf")).all())
    gs.gauss_sum_device_status()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_a_longer_run_of_rotary_writes_and_attention(dtype):
    """Two prompts, then tokens one by one and in parts, through all three kernels."""
    import paper_2609_04910_gb300 as gs
    B, H, Hk, D, T = 2, 8, 2, 128, 64
    prompt, steps = [400, 290], [1, 1, 5, 40, 1, 200, 1, 130, 1]
    total = max(prompt) + sum(steps)
    freqs, scale = gs.rotary_frequencies(64, scaling="yarn", factor=4.0, original_length=1024)
    q, k, v = (points((B, total, h, D), dtype, i) for i, h in enumerate((H, Hk, Hk)))
    s = Store(B, total, Hk, D, D, T, fill=0xFF)
    held, done = ints([0] * B), [0, 0]
    for i, M in enumerate([max(prompt)] + steps):
        ql = ints(prompt if i == 0 else [M] * B)
        at = torch.tensor([[d + m for m in range(M)] for d in done], device="cuda")
        rows = [x.gather(1, at.clamp_max(total - 1)[:, :, None, None].expand(-1, -1, *x.shape[2:])) for x in (q, k, v)]
        qr, kr = gs.gauss_sum_rotary(rows[0], at, freqs, k=rows[1], scale=scale)
        held += ql
        gs.gauss_sum_cache_write(s.cache, kr, rows[2], q_lengths=ql, k_lengths=held, page_table=s.table)
        out, lse = gs.gauss_sum_attention_cached(qr, s.cache, D ** -0.5, causal=True, q_lengths=ql, k_lengths=held,
                                                 page_table=s.table)
        done = [d + n for d, n in zip(done, ql.tolist())]
        kc, vc = gs.gauss_sum_cache_read(s.cache, s.N, torch.float32, q_lengths=held, k_lengths=held,
                                         page_table=s.table)
        # (The rows themselves, float32 of the stored numbers to 2^-24, and a size that bounds
        # their parts: the tokens' quantised ranges are at most twice 16 values' |v|.)
        big = [x.abs().amax(-1, keepdim=True).expand_as(x).double() * 3 for x in (kc, vc)]
        want = attention64(qr, kc.double(), vc.double(), big[0], big[1], D ** -0.5, True, ql, held,
                           path=path_of(M, H, Hk, D, D, dtype))
        assert within(out, want["out"]) <= 1 and within(lse, want["lse"]) <= 1, (i, M)
    assert held.tolist() == done
    gs.gauss_sum_device_status()


@pytest.mark.parametrize("M", [1, 40, 300])
def test_results_repeat_in_other_rooms(M):
    """The same tokens in a cache with room for few and for many: the same results to the bounds of the
    kernels, and the same bits from call to call."""
    import paper_2609_04910_gb300 as gs
    B, n, H, Hk, D = 2, 250, 8, 2, 64
    q = points((B, M, H, D), "bf16", 4)
    for room in (256, 272, 4096):
        s = filled(B, room, Hk, D, D, 16, 2, [n, n - 70])
        kl = ints([n, n - 70])
        want = attention64(q, s.k, s.v, s.k_size, s.size, 0.125, True, k_lengths=kl, path="many")
        exact = attention64(q, s.k, s.v, s.k_size, s.size, 0.125, True, k_lengths=kl, path="few")
        got = [gs.gauss_sum_attention_cached(q, s.cache, 0.125, causal=True, k_lengths=kl, page_table=s.table)
               for _ in range(2)]
        assert within(got[0][0], want["out"]) <= 1 and within(got[0][1], exact["lse"]) <= 1
        assert all(torch.equal(x, y) for x, y in zip(*got))
    gs.gauss_sum_device_status()


def test_many_problems():
    """More than 2^31 / 64 sets of rows for the tile kernel (problems x key heads)."""
    import math
    import paper_2609_04910_gb300 as gs
    B, Hk, H, T = (1 << 22) + 1, 8, 136, 272
    cache = gs.attention_cache(1, T, Hk, 1)
    k = torch.full((1, T, Hk, 1), 2.0, device="cuda")
    gs.gauss_sum_cache_write(cache, k, k)
    table = torch.zeros(1, 1, dtype=torch.int32, device="cuda").expand(B, 1)
    q = torch.ones(1, 1, H, 1, dtype=torch.float16, device="cuda").expand(B, 1, H, 1)
    kl = torch.full((B,), 3, dtype=torch.int32, device="cuda")
    out, lse = gs.gauss_sum_attention_cached(q, cache, 0.5, causal=True, k_lengths=kl, page_table=table)
    gs.gauss_sum_device_status()
    assert bool((out == 2.0).all())
    assert float((lse - (1 + math.log(3))).abs().max()) <= 2.0 ** -20
