"""The attention example: training on the squared MMD, and decoding."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_training_lowers_the_mmd():
    import attention_mmd
    import paper_2609_04910_gb300 as gs
    losses = attention_mmd.train(steps=80)
    gs.gauss_sum_device_status()
    # The clouds start apart and end near the sampling floor of 512 points
    # (squared MMD of order 2 / 512).
    assert losses[-1] < 0.2 * losses[0] and losses[-1] > -1e-3, losses[::10]


def test_weight_gradients_against_differences():
    """The whole backward chain along random directions of each weight."""
    import attention_mmd
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    block = attention_mmd.Block(16, 4, 2, 64, 4, gen)
    positions = torch.arange(150, device="cuda", dtype=torch.int32)
    z = torch.randn(2, 150, 16, generator=gen, device="cuda")
    target = torch.randn(2, 150, 4, generator=gen, device="cuda") + 1
    y, kept = block.forward(z, positions)
    _, dy = attention_mmd.mmd2_and_gradient(y, target, 1 / 4)
    grads = block.backward(dy, kept)

    def loss(name, d, h):
        old = block.w[name]
        block.w[name] = old + h * d
        value = float(plain_loss(block, z, positions, target, 1 / 4))
        block.w[name] = old
        return value

    for name, g in grads.items():
        d = torch.randn(g.shape, generator=gen, device="cuda")
        h = 1e-4
        slope = (loss(name, d, h) - loss(name, d, -h)) / (2 * h)
        mine = float((g * d).sum())
        # bf16 attention (2^-8 per operand, a few of them) against float64 differences, of the
        # magnitude that the terms of this inner product add up to.
        size = float((g * d).norm()) * 3
        assert abs(mine - slope) <= 0.03 * size + 1e-6, (name, mine, slope, size)


def plain_loss(block, z, positions, target, tau):
    """The same loss in float64 torch operations."""
    import torch
    from attention_forms import rotary64
    from paper_2609_04910_gb300.rotary import angular_frequencies
    z, w = z.double(), {n: x.double() for n, x in block.w.items()}
    B, N, _ = z.shape
    H, Hk, D = block.heads, block.key_heads, block.head_dim
    freqs, scale = angular_frequencies(D // 2, scaling="yarn", factor=4.0, original_length=1024)
    q, k, v = ((z @ w[n]).view(B, N, h, D) for n, h in (("q", H), ("k", Hk), ("v", Hk)))
    q, k = (rotary64(x, positions, freqs, scale=scale) for x in (q, k))
    k, v = (x.repeat_interleave(H // Hk, 2) for x in (k, v))
    p = torch.softmax(torch.einsum("bmhd,bnhd->bhmn", q, k) * block.tau, -1)
    y = torch.einsum("bhmn,bnhd->bmhd", p, v).flatten(2) @ w["o"] + z @ w["s"]
    both = torch.cat([y, target.double()], 1)
    s = torch.cat([torch.full((N,), 1.0 / N), torch.full((N,), -1.0 / N)]).double().cuda()
    kernel = torch.exp(-tau / 2 * torch.cdist(both, both) ** 2)
    return torch.einsum("m,bmn,n->b", s, kernel, s).sum()


def test_decoding_gives_the_rows_of_the_full_pass():
    import attention_mmd
    import paper_2609_04910_gb300 as gs
    # Same probabilities and values, rounded differently on the way: a few
    # bf16 units of outputs of order one.
    assert attention_mmd.decode() <= 0.05
    gs.gauss_sum_device_status()
