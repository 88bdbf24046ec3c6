"""Accuracy of attention and its gradient where a bound over whole heads says little."""
import math

import pytest
import torch

from attention_forms import UNIT, within
from attention_terms import heads64
from test_attention_gpu import points

pytestmark = pytest.mark.gpu


def forward64(q, k, v, tau, heads):
    out = torch.zeros(*q.shape[:3], v.shape[3], dtype=torch.float64, device=q.device)
    lse = torch.zeros(q.shape[0], q.shape[2], q.shape[1], dtype=torch.float64, device=q.device)
    for x in heads:
        out[x["b"], :, x["h"]], lse[x["b"], x["h"]] = x["out"], x["lse"]
    return out, lse


@pytest.mark.parametrize("side", ["queries", "values"])
@pytest.mark.parametrize("ratio", [1e-5, 1e-7])
@pytest.mark.parametrize("M,N", [(600, 600), (333, 700), (700, 450)])
@pytest.mark.parametrize("D,C", [(64, 64), (128, 96)])
def test_fp16_gradients_of_rows_far_apart(D, C, M, N, ratio, side):
    """dS keeps the precision of fp16 down to 2^-29 of the largest |g||v| + |delta|
    among the pairs that the causal mask shows of the same key (grad_k) or of the
    same query (grad_q): rows that it hides do not count, however large.

    The early queries have large upstream gradients and the late keys are seen by
    the others only; or the late values are large and the early queries see the
    others only.  An entry is off by |dS| (u + 2 eS) + p eD, and by half of 2^-24
    where its scaled value is below fp16's normal range: the scale brings the bound
    to 2^14 .. 2^15, so that is 2^-39 of the bound."""
    import paper_2609_04910_gb300 as gs
    H, Hk, tau, u = 4, 2, 1 / math.sqrt(D), UNIT["fp16"]
    q, k = points((1, M, H, D), "fp16", 1), points((1, N, Hk, D), "fp16", 2)
    v, g = points((1, N, Hk, C), "fp16", 3), points((1, M, H, C), "fp16", 4)
    if side == "queries":
        split = min(300, M // 2)
        g[:, :split] *= 1e4
        g[:, split:] *= 1e4 * ratio
    else:
        split = N // 2
        g *= 2
        v[:, :split] *= 1e4 * ratio
        v[:, split:] *= 1e4
    heads = list(heads64(q, k, v, g, tau, True))
    out, lse = forward64(q, k, v, tau, heads)
    want = {"q": torch.zeros_like(q, dtype=torch.float64), "k": torch.zeros_like(k, dtype=torch.float64)}
    err = {x: torch.zeros_like(t) for x, t in want.items()}
    top = torch.zeros(2, Hk, N, dtype=torch.float64, device="cuda")   # |g|, |delta| seen by a key
    for x in heads:
        gn = x["G"].norm(dim=-1, keepdim=True)
        top[0, x["j"]] = torch.maximum(top[0, x["j"]], (gn * x["seen"]).amax(0))
        top[1, x["j"]] = torch.maximum(top[1, x["j"]], (x["delta"].abs() * x["seen"]).amax(0))
    for x in heads:
        j, h, gn, vn = x["j"], x["h"], x["G"].norm(dim=-1), x["V"].norm(dim=-1)
        eD = 2.0 ** -21 * (x["G"].abs() @ x["V"].abs().T + x["delta"].abs()) + \
            u * (x["G"].abs() * x["out"].abs()).sum(-1, keepdim=True)
        eds = x["p"] * eD + x["ds"].abs() * (u + 2 * x["eS"])
        of_key = top[0, j] * vn + top[1, j]
        of_query = gn * (vn[None] * x["seen"]).amax(1) + x["delta"][:, 0].abs()
        want["q"][0, :, h] = tau * x["ds"] @ x["K"]
        want["k"][0, :, j] += tau * x["ds"].T @ x["Q"]
        err["q"][0, :, h] = tau * (eds + 2.0 ** -39 * of_query[:, None] * x["seen"]) @ x["K"].abs()
        err["k"][0, :, j] += tau * (eds + 2.0 ** -39 * of_key[None] * x["seen"]).T @ x["Q"].abs()
    got = gs.gauss_sum_attention_vjp(q, k, v, out.half(), lse.float(), g, tau, causal=True,
                                     want=("q", "k"))
    gs.gauss_sum_device_status()
    assert all(float(t.abs().max()) < 65504 for t in want.values())      # (of the inputs)
    worst = {x: within(t, (want[x], 1.02 * (err[x] + u * want[x].abs()) + 2.0 ** -25))
             for x, t in zip("qk", got)}
    assert all(w <= 1 for w in worst.values()), worst


@pytest.mark.parametrize("layout", ["bmhd", "odd"])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("M,N,causal", [(70, 2, False), (33, 7, False), (40, 24, False), (24, 24, True),
                                        (30, 9, True)])
@pytest.mark.parametrize("D,C", [(64, 64), (128, 40), (192, 130)])
def test_gradients_of_few_keys_do_not_carry_the_rounding_of_out(D, C, M, N, causal, dtype, layout):
    """Rows of at most 24 keys take delta from the keys, on the tensor cores and
    on the fp32 pipe: the bound has no term for the rounding of ``out``, whose
    share of such rows is the largest when one key has nearly all the weight."""
    import paper_2609_04910_gb300 as gs
    H, Hk, tau, u = 4, 2, 1 / math.sqrt(D), UNIT[dtype]
    q, k = (points((2, n, h, D), dtype, i, layout, 2.5) for i, (n, h) in enumerate([(M, H), (N, Hk)]))
    v, g = (points((2, n, h, C), dtype, i + 5, layout) for i, (n, h) in enumerate([(N, Hk), (M, H)]))
    z = points((2, H, M, 1), "fp32", 9)[..., 0].contiguous()
    heads = list(heads64(q, k, v, g, tau, causal, z))
    out, lse = forward64(q, k, v, tau, heads)
    want = {x: torch.zeros_like(t, dtype=torch.float64) for x, t in (("q", q), ("k", k))}
    err = {x: torch.zeros_like(t) for x, t in want.items()}
    for x in heads:
        b, j, h, a = x["b"], x["j"], x["h"], x["G"].abs() @ x["V"].abs().T
        # delta from fp32 probabilities: 2 eS of each term, and fp32 products and sums.
        eD = 2.0 ** -21 * (a + x["delta"].abs() + (x["p"] * a).sum(-1, keepdim=True)) + \
            2 * x["eS"] * (x["p"] * x["dp"].abs()).sum(-1, keepdim=True)
        least = 2.0 ** -38 * (x["G"].norm(dim=-1).max() * x["V"].norm(dim=-1).max() + x["delta"].abs().max())
        eds = x["p"] * eD + x["ds"].abs() * (u + 2 * x["eS"]) + least * x["seen"]
        want["q"][b, :, h] = tau * x["ds"] @ x["K"]
        want["k"][b, :, j] += tau * x["ds"].T @ x["Q"]
        err["q"][b, :, h] = tau * eds @ x["K"].abs()
        err["k"][b, :, j] += tau * eds.T @ x["Q"].abs()
    given = points((2, M, H, C), dtype, 11, layout)
    given.copy_(out)
    got = gs.gauss_sum_attention_vjp(q, k, v, given, lse.float(), g, tau, g_lse=z, causal=causal,
                                     want=("q", "k"))
    gs.gauss_sum_device_status()
    least = 2.0 ** -25 if dtype == "fp16" else 1e-30
    worst = {x: within(t, (want[x], 1.02 * (err[x] + u * want[x].abs()) + least)) for x, t in zip("qk", got)}
    assert all(w <= 1 for w in worst.values()), worst


@pytest.mark.parametrize("M", [1, 30])
@pytest.mark.parametrize("size", [256, 4096, 262144])
def test_fp32_exponents_of_large_scores(size, M):
    """Scores tau s of up to 30 size / 64 whose products are exact: the exponent
    c s - m is rounded once, so that its error goes with its own size and not
    with that of the scores.

    c = tau log2 e is off by 2^-24 of itself, the exponent x by 2^-24 |x| once more,
    ex2 by 2^-22, the sums of N terms by (N + 2) 2^-24 of their magnitude, and m
    (rounded) is common to all: an error of 2^-23 |x| + 2^-22 + N 2^-24 in each p, with
    |x| p <= 0.54 where p < 1 counts."""
    import paper_2609_04910_gb300 as gs
    N, H, D, tau = 40, 2, 4, 1.0 / 64
    q = torch.zeros(1, M, H, D, device="cuda")
    q[0, :, :, 1] = (1 + torch.arange(M, device="cuda") % 30)[:, None].float()
    k = torch.zeros(1, N, H, D, device="cuda")
    order = torch.randperm(N, generator=torch.Generator().manual_seed(3)).cuda()
    k[0, :, :, 1] = (size + 32 * order)[:, None].float()     # half a nat apart for the first row
    v = points((1, N, H, 8), "fp32", 5)
    heads = list(heads64(q, k, v, torch.zeros(1, M, H, 8, device="cuda"), tau))
    assert float((q[..., 1].max() * k[..., 1].max())) < 2.0 ** 24
    want, lse64 = forward64(q, k, v, tau, heads)
    bound = torch.zeros_like(want)
    for x in heads:
        p = x["p"]
        e = p * (2.0 ** -23 * -torch.log2(p.clamp_min(1e-300)) + 2.0 ** -22 + (N + 4) * 2.0 ** -24)
        e = e + p * e.sum(-1, keepdim=True)                    # the sum that divides
        bound[0, :, x["h"]] = e @ x["V"].abs() + 2.0 ** -23 * x["out"].abs()
    out, lse = gs.gauss_sum_attention(q, k, v, tau)
    gs.gauss_sum_device_status()
    assert within(out, (want, 1.05 * bound + 1e-30)) <= 1
    assert within(lse, (lse64, 2.0 ** -21 * (1 + lse64.abs()))) <= 1
