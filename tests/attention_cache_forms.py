"""Float64 and integer forms of the 4-bit cache, written from its definition,
with the error bounds that the tests allow.

Bounds (first order, worst case, elementwise).  u is the unit roundoff of the
element type (fp32 2^-24, fp16 2^-11, bf16 2^-8); fp32 accumulation is allowed
2^-21 of the sum of magnitudes, as for gauss_sum_attention:

  read back        u |value|  (+ 2^-24 |value| for the sum m + s code in fp32)
  score error      eS = 2^-21 (tau max_n sum |q||k_n| + 1)
                        + r tau max_n sum |q||k| + z tau |q|_1 max |k|
  out              (w + 2 eS) sum_n p |v_n| + z max |v| + u |out|

with, for the three ways a call is computed,

  few    (few rows)    codes as they are: r = z = 0, w the rounding of a probability times a
                       step (fp16: 2^-11; two fp16 numbers for fp32 queries: 2^-21)
  many   (16-bit)      values as fp16 numbers of a tile whose largest step is scaled to 2^-9 ..
                       2^-8: r = 2^-11, and below 2^-14 multiples of 2^-24, at most 2^-15 of
                       the step, off by half of that: z = 2^-16 / 15 (a step is a 15th of
                       |m| + 15 s at most); w = 2 x 2^-11 (a probability and a value)
  rows   (the rest)    values in the element type: r = u, z = 0, w = 2 u
  lse              eS + 2^-22 |lse|

|k_n| and |v_n| stand for |m| + s code and |m| + 15 s of their group: the two terms
of a value are summed apart, sum_n (s code) q + m sum q, so that what rounds is the
size of these terms and not of their sum (least values are mostly negative and
cancel against the codes: |m| + s code is up to 3.3 |k| on average over a normal
group, more for a value near zero).
"""
import torch

DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def bf16_down(x):
    """Largest bf16 number <= x, of finite float32 numbers."""
    y = x.bfloat16()
    lower = torch.nextafter(y, torch.full_like(y, -float("inf")))
    return torch.where(y.float() > x, lower, y)


def quantise(x):
    """codes (long), s and m (bf16) per group of rows x (..., D) (a CPU or CUDA tensor)."""
    codes, steps, lows = [], [], []
    for c in range(0, x.shape[-1], 64):
        g = x[..., c:c + 64].float()
        ok = torch.isfinite(g).all(-1)
        m = bf16_down(torch.where(ok, g.amin(-1), 0.0))
        span = (torch.where(ok, g.amax(-1), 0.0) - m.float()).double()
        s = (span / 15).float().bfloat16()
        s = torch.where(s.double() < 2.0 ** -126, torch.zeros_like(s), s)
        ok &= torch.isfinite(s.float()) & torch.isfinite(m.float())
        y = (g - m.float()[..., None]).double()
        q = torch.round(y / torch.where(s > 0, s, torch.ones_like(s)).double()[..., None]).clamp(0, 15)
        q = torch.where((ok & (s > 0))[..., None], q, 0.0)
        nan = torch.full_like(s, float("nan"))
        codes.append(q.long())
        steps.append(torch.where(ok, s, nan))
        lows.append(torch.where(ok, m, nan))
    return torch.cat(codes, -1), torch.stack(steps, -1), torch.stack(lows, -1)


def values(codes, s, m):
    """float64 values of codes (..., D) with groups (..., groups)."""
    group = torch.arange(codes.shape[-1], device=codes.device) // 64
    return m.double()[..., group] + s.double()[..., group] * codes.double()


def row_bytes(codes, is_key):
    """The bytes of one row of codes (D,), from the definition of the layout, as a list."""
    D = len(codes)
    W = (D + 31) // 32
    out = [0] * (16 * W)
    for ch, code in enumerate(codes):
        j, inside = ch // 32, ch % 32
        if is_key:
            t, p = inside // 8, inside % 8
            at = (t * W + j) * 4 + p // 2
        else:
            g, p = inside // 4, inside % 4
            at = (g * W + j) * 2 + p // 2
        out[at] |= int(code) << (4 * (p % 2))
    return out


def attention64(q, k, v, k_size, v_size, tau, causal=False, q_lengths=None, k_lengths=None, path="rows"):
    """out and lse in float64 with their bounds: {name: (value, bound)}.

    k (B, N, Hk, D), v (B, N, Hk, C) float64 values of the cache, k_size |m| + s code and
    v_size |m| + 15 s of each."""
    u = UNIT[q.dtype]
    f64 = {"dtype": torch.float64, "device": q.device}
    B, M, H, D = q.shape
    N, Hk, C = k.shape[1], k.shape[2], v.shape[3]
    out, lse = torch.zeros(B, M, H, C, **f64), torch.full((B, H, M), -float("inf"), **f64)
    e_out, e_lse = torch.zeros_like(out), torch.zeros_like(lse)
    r, z, w = {"few": (0, 0, 2.0 ** -21 if q.dtype == torch.float32 else 2.0 ** -11),
               "many": (2.0 ** -11, 2.0 ** -16 / 15, 2.0 ** -10), "rows": (u, 0, 2 * u)}[path]
    for b in range(B):
        ql = M if q_lengths is None else min(max(int(q_lengths[b]), 0), M)
        kl = N if k_lengths is None else min(max(int(k_lengths[b]), 0), N)
        if ql == 0 or kl == 0:
            continue
        seen = torch.ones(ql, kl, dtype=torch.bool, device=q.device)
        if causal:
            seen = torch.arange(kl, device=q.device)[None, :] <= \
                torch.arange(ql, device=q.device)[:, None] + (kl - ql)
        some = seen.any(-1, keepdim=True)
        for h in range(H):
            j = h // (H // Hk)
            Q, K, V, S = q[b, :ql, h].double(), k[b, :kl, j], v[b, :kl, j], v_size[b, :kl, j]
            s = (tau * Q @ K.T).masked_fill(~seen, -float("inf"))
            top = torch.where(some, torch.logsumexp(s, -1, keepdim=True), 0.0)
            p = torch.where(seen, torch.exp(s - top), 0.0)
            mag, size = ((tau * Q.abs() @ x.abs().T).masked_fill(~seen, 0).amax(-1, keepdim=True)
                         for x in (K, k_size[b, :kl, j]))
            biggest = k_size[b, :kl, j].max()
            eS = 2.0 ** -21 * (size + 1) + r * mag + z * biggest * tau * Q.abs().sum(-1, keepdim=True)
            out[b, :ql, h] = p @ V
            lse[b, h, :ql] = torch.where(some, top, -float("inf"))[:, 0]
            # (Products of a probability and a step keep 2^-32 of the largest |v|, rows of
            # 16 bits 2^-28 of it.)
            e_out[b, :ql, h] = (w + 2 * eS) * (p @ S) + u * (p @ V).abs() + \
                2.0 ** -28 * S.amax(0) * seen.sum(-1, keepdim=True) + z * S.max() * seen.any(-1, keepdim=True)
            e_lse[b, h, :ql] = eS[:, 0] + 2.0 ** -22 * top[:, 0].abs()
    least = 2.0 ** -25 if q.dtype == torch.float16 else 1e-30
    return {"out": (out, 1.02 * e_out + least), "lse": (lse, 1.02 * e_lse + 1e-30)}


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
