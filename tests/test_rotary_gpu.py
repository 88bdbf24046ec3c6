"""Rotary positions on the GPU against float64."""
import pytest
import torch

from attention_forms import DT, UNIT, rotary64
from test_attention_gpu import points

pytestmark = pytest.mark.gpu


def check(B, M, H, Hk, D, R, dtype, interleaved=False, transpose=False, start=0, layout="bmhd",
          pos_dtype=torch.int32, seed=0, **scaling):
    import paper_2609_04910_gb300 as gs
    from paper_2609_04910_gb300.rotary import angular_frequencies
    freqs, scale = angular_frequencies(R, **scaling)
    table, scale2 = gs.rotary_frequencies(R, **scaling)
    assert scale == scale2
    q = points((B, M, H, D), dtype, seed, layout)
    k = points((B, M, Hk, D), dtype, seed + 1, layout) if Hk else None
    pos = (start + torch.arange(M, device="cuda")[None] +
           torch.arange(B, device="cuda")[:, None] * 17).to(pos_dtype)
    got = gs.gauss_sum_rotary(q, pos, table, k=k, interleaved=interleaved, transpose=transpose,
                              scale=scale)
    got = got if Hk else (got,)
    for x, y in zip((q, k), got):
        want = rotary64(x, pos, freqs, interleaved, transpose, scale)
        # One rounding to the type; cos and sin to 4 units of fp32 plus the
        # float64 form's own angle error (2^-52 of the angle, in radians).
        size = scale * x.double().abs().amax(-1, keepdim=True) * 2
        far = float(pos.abs().max()) * 2.0 ** -51 if M else 0.0
        bound = UNIT[dtype] * want.abs() + (2.0 ** -21 + far) * size + 1e-30
        if dtype == "fp16":
            bound = bound + 2.0 ** -25   # subnormal results
        assert ((y.double() - want).abs() <= bound).all()
        assert torch.equal(y[..., R:], x[..., R:])
    return q, k, got, pos, table, scale


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("D,R", [(128, 128), (64, 32), (96, 64), (80, 80), (80, 40), (20, 12), (7, 2),
                                 (64, 0), (24, 16), (40, 16)])
def test_widths(D, R, dtype, interleaved, transpose):
    check(2, 37, 5, 2, D, R, dtype, interleaved, transpose)


@pytest.mark.parametrize("layout", ["bhmd", "wide", "odd"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("M", [1, 300])
def test_layouts(layout, interleaved, M):
    for dtype in ("fp32", "fp16", "bf16"):
        check(3, M, 8, 2, 64, 48, dtype, interleaved, layout=layout)


@pytest.mark.parametrize("start", [0, 1000003, 2 ** 31 - 500, -70000])
@pytest.mark.parametrize("pos_dtype", [torch.int32, torch.int64])
def test_far_positions_keep_their_angles(start, pos_dtype):
    # Far from zero fp32 angles would be off by whole turns.
    check(2, 100, 2, 1, 64, 64, "fp32", start=start, pos_dtype=pos_dtype)


def test_positions_past_32_bits():
    check(2, 100, 2, 1, 64, 64, "fp32", start=2 ** 33 + 12345, pos_dtype=torch.int64)


@pytest.mark.parametrize("scaling", [
    dict(scaling="linear", factor=8.0), dict(scaling="ntk", factor=8.0),
    dict(scaling="yarn", factor=8.0, original_length=8192), dict(base=500000.0)])
def test_scaled_contexts(scaling):
    for dtype in ("fp32", "bf16"):
        check(2, 65, 6, 2, 128, 128, dtype, start=60000, **scaling)


def test_many_heads_and_long_rows():
    check(2, 2100, 33, 7, 128, 128, "bf16")
    check(1, 700, 40, 0, 96, 64, "fp16", True)
    check(70, 1, 32, 8, 128, 128, "bf16", start=5000)
    check(2, 700, 3, 1, 4096, 4096, "fp32")
    check(1, 900, 2, 0, 4100, 4090, "fp16", True)


def test_in_place_and_transpose_is_the_gradient():
    import paper_2609_04910_gb300 as gs
    for dtype in ("fp32", "fp16", "bf16"):
        for interleaved in (False, True):
            q, k, (qo, ko), pos, table, scale = check(2, 50, 4, 2, 96, 64, dtype, interleaved,
                                                      scaling="yarn", factor=4.0,
                                                      original_length=1024)
            q2, k2 = q.clone(), k.clone()
            a, b = gs.gauss_sum_rotary(q2, pos, table, k=k2, interleaved=interleaved, scale=scale,
                                       q_out=q2, k_out=k2)
            assert a is q2 and torch.equal(q2, qo) and torch.equal(k2, ko)
            # <g, R x> = <R^T g, x>: both sides to the type's rounding of their terms.
            g = points(tuple(q.shape), dtype, 40)
            back = gs.gauss_sum_rotary(g, pos, table, interleaved=interleaved, scale=scale,
                                       transpose=True)
            lhs, rhs = (g.double() * qo.double()).sum(), (back.double() * q.double()).sum()
            size = (g.double() * qo.double()).abs().sum() + (back.double() * q.double()).abs().sum()
            assert abs(float(lhs - rhs)) <= (UNIT[dtype] + 2.0 ** -20) * float(size)


def test_shared_and_strided_positions():
    import paper_2609_04910_gb300 as gs
    q = points((3, 40, 4, 64), "bf16", 1)
    table, _ = gs.rotary_frequencies(64)
    pos = torch.arange(40, device="cuda") + 9
    a = gs.gauss_sum_rotary(q, pos, table)
    b = gs.gauss_sum_rotary(q, pos[None].expand(3, 40), table)
    wide = torch.zeros(3, 80, dtype=torch.int64, device="cuda")
    wide[:, ::2] = pos
    c = gs.gauss_sum_rotary(q, wide[:, ::2], table)
    assert torch.equal(a, b) and torch.equal(a, c)


def test_empty():
    import paper_2609_04910_gb300 as gs
    table, _ = gs.rotary_frequencies(64)
    for B, M in ((0, 3), (2, 0)):
        q = points((B, M, 4, 64), "bf16", 1)
        assert gs.gauss_sum_rotary(q, torch.zeros(B, M, dtype=torch.int32, device="cuda"),
                                   table).shape == q.shape
