"""Attention over many key tiles to a block: rings that wrap, maxima that move, repeats.

Enough problems and heads that one block streams all keys of its rows (blocks
that do not fill the GPU split them: more than 76 blocks of the kernels that
keep an SM to themselves, more than 152 of those that share one)."""
import pytest
import torch

from attention_forms import DT, attention64, within
from test_attention_gpu import points, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("causal,ql,kl", [(True, None, None), (True, [700, 513], [1700, 1409]),
                                          (False, [650, 700], [1537, 1700])])
@pytest.mark.parametrize("D,C", [(128, 128), (64, 64), (128, 64), (72, 104)])
def test_many_key_tiles(D, C, causal, ql, kl, dtype):
    run(2, 700, 1700, 32, 16, D, C, dtype, causal, ql=ql, kl=kl, seed=D + C, g_lse=True)


@pytest.mark.parametrize("rising", [True, False])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("M", [1, 100, 130, 300])
@pytest.mark.parametrize("D,C", [(64, 64), (128, 128), (64, 128)])
def test_maximum_moves_at_every_tile(D, C, M, dtype, rising):
    # 200 nats over 1500 keys: 12 log2 units in 64 of them, and a maximum that
    # is moved as soon as a tile exceeds it by 8.
    import paper_2609_04910_gb300 as gs
    B, H, N, tau = 2, 48, 1500, 0.125
    ramp = torch.linspace(-100, 100, N, device="cuda")
    ramp = (ramp if rising else ramp.flip(0)) / (tau * D)
    q = torch.ones(B, M, H, D, device="cuda").to(DT[dtype])
    q[1] *= 0.5                           # (a slope of its own: six units a tile)
    k = ramp[None, :, None, None].expand(B, N, H, D).to(DT[dtype])
    v = points((B, N, H, C), dtype, 4)
    want = attention64(q, k, v, tau)
    out, lse = gs.gauss_sum_attention(q, k, v, tau)
    gs.gauss_sum_device_status()
    assert within(out, want["out"]) <= 1 and within(lse, want["lse"]) <= 1


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("M", [1, 100, 130, 300])
@pytest.mark.parametrize("D,C", [(64, 64), (128, 128)])
def test_sharp_scores_over_many_tiles(D, C, M, dtype):
    # Nearly one-hot rows whose winner lies anywhere: the maximum jumps late in some rows.
    run(2, M, 1500, 48, 48, D, C, dtype, scale=3.0, seed=M + D, grads=M >= 130)


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("M", [1, 90, 700])
@pytest.mark.parametrize("D", [64, 128])
def test_same_bits_every_call(D, M, dtype):
    import paper_2609_04910_gb300 as gs
    N, H, Hk = 1700, 32, 8
    q, k, v, g = (points((4, n, h, D), dtype, i) for i, (n, h) in enumerate(
        [(M, H), (N, Hk), (N, Hk), (M, H)]))
    ql = torch.tensor([M, max(1, M - 100), M, M // 2], dtype=torch.int32, device="cuda")
    kl = torch.tensor([N, N - 77, 900, 1], dtype=torch.int32, device="cuda")
    masks = dict(causal=True, q_lengths=ql, k_lengths=kl)
    first = None
    for _ in range(12 if dtype == "fp32" else 40):
        out, lse = gs.gauss_sum_attention(q, k, v, 0.1, **masks)
        got = (out, lse, *gs.gauss_sum_attention_vjp(q, k, v, out, lse, g, 0.1, **masks))
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(first, got))
    gs.gauss_sum_device_status()
