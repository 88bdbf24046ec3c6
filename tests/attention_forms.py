"""Float64 forms of the attention operators, written from the definitions,
with the error bounds that the tests allow.

Bounds (first order, worst case, elementwise).  With u the unit roundoff of
the element type (fp32: 2^-24, fp16: 2^-11, bf16: 2^-8), fp32
accumulation of a D-term product is allowed 2^-21 of the sum of magnitudes:

  score error      eS   = 2^-21 (tau max_n |q|.|k_n| + 1) per row (also covers
                          the exponential's own error)
  out              (u + 2 eS) sum_n p |v_n| + u |out|
  lse              eS + 2^-22 |lse|
  dP - delta       eD   = 2^-21 (|g|.|v_n| + |delta|) + u |g|.|out| (out is given rounded)
  dS               eS'  = p eD + |dS| (u + 2 eS)
  grad_q           tau eS' |k| + u |grad_q|;  grad_k with |q|;
  grad_v           (u + 2 eS) p^T |g| + u |grad_v|

The u in the out, dS and grad_v terms is the rounding of p and dS as
tensor-core operands (fp32 arrays do without, which only tightens it).
fp16 operands are scaled so that they lose nothing above 2^-28 of a row's
largest value; the bounds carry that as an absolute term.
"""
import torch

DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}


def attention64(q, k, v, tau, causal=False, q_lengths=None, k_lengths=None, g=None, g_lse=None,
                out=None):
    """out, lse and, with g, the gradients in float64, with their error bounds.

    Returns {name: (value, bound)}.  ``out`` (rounded) enters only the bound of
    the gradients."""
    f64 = {"dtype": torch.float64, "device": q.device}
    u = {torch.float32: UNIT["fp32"], torch.float16: UNIT["fp16"],
         torch.bfloat16: UNIT["bf16"]}[q.dtype]
    B, M, H, D = q.shape
    N, Hk, C = k.shape[1], k.shape[2], v.shape[3]
    r = {"out": torch.zeros(B, M, H, C, **f64), "lse": torch.full((B, H, M), -float("inf"), **f64),
         "q": torch.zeros(B, M, H, D, **f64), "k": torch.zeros(B, N, Hk, D, **f64),
         "v": torch.zeros(B, N, Hk, C, **f64)}
    e = {x: torch.zeros_like(t) for x, t in r.items()}
    tiny = 2.0 ** -28
    for b in range(B):
        ql = M if q_lengths is None else min(max(int(q_lengths[b]), 0), M)
        kl = N if k_lengths is None else min(max(int(k_lengths[b]), 0), N)
        seen = torch.ones(ql, kl, dtype=torch.bool, device=q.device)
        if causal:
            seen = torch.arange(kl, device=q.device)[None, :] <= \
                torch.arange(ql, device=q.device)[:, None] + (kl - ql)
        for h in range(H):
            j = h // (H // Hk)
            Q, K, V = q[b, :ql, h].double(), k[b, :kl, j].double(), v[b, :kl, j].double()
            if ql == 0 or kl == 0:
                continue
            s = (tau * Q @ K.T).masked_fill(~seen, -float("inf"))
            z = torch.logsumexp(s, -1)
            some = torch.isfinite(z)[:, None]
            p = torch.where(some & seen, torch.exp(s - torch.where(some, z[:, None], 0.0)), 0.0)
            mag = (tau * Q.abs() @ K.abs().T).masked_fill(~seen, 0).amax(-1, keepdim=True)
            eS = 2.0 ** -21 * (mag + 1)
            o = p @ V
            r["out"][b, :ql, h], r["lse"][b, h, :ql] = o, z
            e["out"][b, :ql, h] = (u + 2 * eS) * (p @ V.abs()) + u * o.abs() + \
                tiny * V.abs().amax(0) * seen.sum(-1, keepdim=True)
            e["lse"][b, h, :ql] = eS[:, 0] + 2.0 ** -22 * torch.where(some[:, 0], z.abs(), 0.0)
            if g is None:
                continue
            G = g[b, :ql, h].double()
            dp = G @ V.T
            delta = (G * o).sum(-1, keepdim=True)
            if g_lse is not None:
                delta = delta - g_lse[b, h, :ql, None].double()
            ds = p * (dp - delta)
            eD = 2.0 ** -21 * (G.abs() @ V.abs().T + delta.abs()) + \
                u * (G.abs() * o.abs()).sum(-1, keepdim=True)
            top = ((G * G).sum(-1).sqrt().max() * (V * V).sum(-1).sqrt().max() +
                   delta.abs().max())
            eds = p * eD + ds.abs() * (u + 2 * eS) + tiny * top * seen
            ep = (u + 2 * eS) * p + tiny * seen
            r["q"][b, :ql, h] = tau * ds @ K
            e["q"][b, :ql, h] = tau * eds @ K.abs()
            r["k"][b, :kl, j] += tau * ds.T @ Q
            e["k"][b, :kl, j] += tau * eds.T @ Q.abs()
            r["v"][b, :kl, j] += p.T @ G
            e["v"][b, :kl, j] += ep.T @ G.abs()
    for x in "qkv":
        e[x] += u * r[x].abs()
    # fp16 results below 2^-14 are rounded to multiples of 2^-24.
    least = 2.0 ** -25 if q.dtype == torch.float16 else 1e-30
    return {x: (r[x], 1.02 * e[x] + (1e-30 if x == "lse" else least)) for x in r}


def rotary64(x, positions, freqs, interleaved=False, transpose=False, scale=1.0):
    """The rotation in float64; freqs are radians per position."""
    R = 2 * len(freqs)
    pos = positions.double()
    pos = pos[None, :] if pos.dim() == 1 else pos
    angle = pos[..., None] * torch.tensor(freqs, dtype=torch.float64, device=x.device)
    c, s = angle.cos()[:, :, None, :], angle.sin()[:, :, None, :]
    s = -s if transpose else s
    y = x.double().clone()
    a, b = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    xa, xb = x[..., a].double(), x[..., b].double()
    y[..., a], y[..., b] = scale * (xa * c - xb * s), scale * (xa * s + xb * c)
    return y


def within(got, want):
    """Largest error over its bound; infinities have to agree."""
    value, bound = want
    got = got.double()
    if got.numel() == 0:
        return 0.0
    inf = torch.isinf(value)
    assert torch.equal(torch.isinf(got) & (got < 0), inf & (value < 0)), "infinities differ"
    assert torch.isfinite(got[~inf]).all(), "non-finite result"
    err = (got - value)[~inf].abs() / bound[~inf]
    return float(err.max()) if err.numel() else 0.0
