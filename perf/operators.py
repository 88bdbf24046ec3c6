"""Measured cases of the attention operators: softmax attention with its
log-sum-exp, its vector-Jacobian product, and rotary positions.

``run`` computes them in plain 32-bit torch operations, or, where ``own`` is
true, through the package's entry points.  Shapes: q (B, M, H, D),
k (B, N, Hk, D), v (B, N, Hk, C); query head h reads key head h // (H / Hk);
with ``causal`` query m sees the keys n <= m + (k_length - q_length).
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "fp16": 2, "bf16": 2}


def _attn(op, name, B, M, N, H, Hk, D, dtype, causal=False, ragged="no", layout="bmhd", C=None,
          g_lse=False):
    case = {"op": op, "B": B, "M": M, "N": N, "H": H, "Hk": Hk, "D": D, "C": D if C is None else C,
            "dtype": dtype, "causal": causal, "ragged": ragged, "layout": layout}
    if op == "vjp":
        case["g_lse"] = g_lse
    if name:
        case["name"] = name
    return case


def _rot(name, B, M, H, Hk, D, R, dtype, interleaved=False, transpose=False, scaling="none",
         start=0):
    case = {"op": "rotary", "B": B, "M": M, "H": H, "Hk": Hk, "D": D, "R": R, "dtype": dtype,
            "interleaved": interleaved, "transpose": transpose, "scaling": scaling, "start": start}
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # One new token of each of 16 sequences against caches of uneven length.
        _attn("attention", "token_bf16", 16, 1, 8191, 32, 8, 128, "bf16", True, "keys", "bhmd"),
        # One new token of a single sequence, short cache: latency alone.
        _attn("attention", "token_short_fp16", 1, 1, 333, 8, 8, 64, "fp16", True),
        # A padded batch of prompts, uneven lengths in queries and keys.
        _attn("attention", "prompts_fp16", 3, 1027, 1027, 16, 4, 64, "fp16", True, "both"),
        # The forward pass of a training step on long sequences.
        _attn("attention", "train_bf16", 2, 8192, 8192, 16, 16, 128, "bf16", True),
        # Point clouds attending to point clouds in full precision.
        _attn("attention", "points_fp32", 2, 700, 1501, 4, 4, 32, "fp32"),
        # A small model's gradient step: latency and few tiles.
        _attn("vjp", "vjp_small_fp16", 1, 200, 200, 4, 2, 64, "fp16", True),
        # Cross attention over uneven sources, with a gradient on the log-sum-exp as well.
        _attn("vjp", "vjp_cross_fp16", 4, 1500, 1111, 12, 12, 64, "fp16", False, "keys", "bhmd",
              None, True),
        # The gradient of a training step with shared key heads.
        _attn("vjp", "vjp_train_bf16", 2, 4096, 4096, 32, 8, 128, "bf16", True),
        # Gradients of point clouds in full precision.
        _attn("vjp", "vjp_points_fp32", 1, 500, 900, 4, 4, 32, "fp32"),
        # Queries and keys of one new token per sequence, far into a stretched context.
        _rot("rotary_token_bf16", 32, 1, 32, 8, 128, 128, "bf16", False, False, "yarn", 100000),
        # Queries and keys of a training batch.
        _rot("rotary_train_bf16", 2, 8192, 32, 8, 128, 128, "bf16"),
        # The gradient through interleaved positions on part of an odd-sized batch.
        _rot("rotary_grad_fp16", 3, 2777, 12, 12, 96, 64, "fp16", True, True, "linear", 5),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        kind = c["op"] + ("32" if c["dtype"] == "fp32" else "")
        for x in ("bytes", "flops"):
            most[kind, x] = max(w[x], most.get((kind, x), 0))
    while True:
        op = rng.choice(["attention", "attention", "vjp", "vjp", "rotary"])
        D = rng.choice([32, 64, 80, 96, 128, 128])
        Hk = rng.choice([1, 2, 4, 8, 12])
        H = Hk * rng.choice([1, 1, 2, 4, 7])
        if op == "rotary":
            dtype = rng.choice(["bf16", "fp16", "fp32"])
            M = rng.choice([1, _log_int(rng, 2, 8192)])
            c = _rot(None, _log_int(rng, 1, 64), M, H, Hk, D, rng.choice([D, D, 16, D // 2]), dtype,
                     rng.random() < 0.5, rng.random() < 0.5,
                     rng.choice(["none", "linear", "ntk", "yarn"]), _log_int(rng, 1, 500000))
        else:
            dtype = rng.choice(["bf16", "bf16", "fp16", "fp16", "fp32"])
            N = _log_int(rng, 16, 16384)
            causal = rng.random() < 0.6
            M = rng.choice([1, _log_int(rng, 2, N)]) if op == "attention" else \
                N if rng.random() < 0.6 else _log_int(rng, 16, 8192)
            if dtype == "fp32":
                D = rng.choice([16, 32, 64])
            c = _attn(op, None, _log_int(rng, 1, 32), M, N, H, Hk, D, dtype, causal,
                      rng.choice(["no", "keys", "both"]), rng.choice(["bmhd", "bhmd"]),
                      rng.choice([D, D, D // 2]), op == "vjp" and rng.random() < 0.3)
        w = work(c)
        kind = op + ("32" if dtype == "fp32" and op != "rotary" else "")
        if all(w[x] <= most[kind, x] for x in ("bytes", "flops")):
            return c


def _lengths(case):
    """(q_lengths, k_lengths) as lists: the first problem is full, later ones shorter, some odd."""
    B, M, N = case["B"], case["M"], case["N"]
    short = [b / (2.0 * B) for b in range(B)]
    ql = [M - int(M * s) for s in short] if case["ragged"] == "both" else [M] * B
    kl = [N - int(N * s) for s in short] if case["ragged"] != "no" else [N] * B
    return ql, kl


def _visible(case):
    """Pairs (m, n) that the masks leave, over the batch."""
    pairs = 0
    for ql, kl in zip(*_lengths(case)):
        if not case["causal"]:
            pairs += ql * kl
            continue
        off = kl - ql                       # row m sees max(0, m + off + 1) keys
        first = max(0, -off)
        rows = max(0, ql - first)
        pairs += rows * (first + off + 1) + rows * (rows - 1) // 2
    return pairs


def work(case):
    B, M, H, Hk, D = (case[x] for x in ("B", "M", "H", "Hk", "D"))
    es = BYTES[case["dtype"]]
    if case["op"] == "rotary":
        elems = B * M * (H + Hk) * D
        return {"bytes": 2 * elems * es + 4 * B * M,
                "flops": 3.0 * B * M * (H + Hk) * case["R"]}
    C = case["C"]
    ql, kl = _lengths(case)
    q, k, rows = sum(ql) * H * D * es, sum(kl) * Hk * D * es, sum(ql) * H
    v, o = sum(kl) * Hk * C * es, rows * C * es
    if case["op"] == "attention":
        return {"bytes": q + k + v + o + 4 * rows, "flops": 2.0 * _visible(case) * H * (D + C)}
    return {"bytes": 2 * (q + k + v) + 2 * o + 4 * rows * (2 if case["g_lse"] else 1),
            "flops": 2.0 * _visible(case) * H * (3 * D + 2 * C)}


def _wavelengths(case):
    """Angle per position of each pair of the rotated part, and the factor on both outputs.

    Scaled contexts stretch by 8 from 8192 positions: 'linear' divides every angle; 'ntk' raises
    the base; 'yarn' divides the angles that turn less than once over the original context, keeps
    those that turn more than 32 times, blends between, and multiplies by 0.1 ln 8 + 1.
    """
    R, factor, original, base = case["R"], 8.0, 8192.0, 10000.0
    if case["scaling"] == "ntk":
        base *= factor ** (R / max(1.0, R - 2.0))
    freqs = [base ** (-2.0 * i / R) for i in range(R // 2)]
    if case["scaling"] == "linear":
        freqs = [f / factor for f in freqs]
    if case["scaling"] != "yarn":
        return freqs, 1.0

    def where(turns):
        return R * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base))
    low, high = max(0.0, math.floor(where(32.0))), min(R - 1.0, math.ceil(where(1.0)))
    high = high + 0.001 if low == high else high
    out = []
    for i, f in enumerate(freqs):
        ramp = min(1.0, max(0.0, (i - low) / (high - low)))
        out.append(f * (1 - ramp) + f / factor * ramp)
    return out, 0.1 * math.log(factor) + 1.0


def _fixed_point(freqs):
    """Turns per position as 64-bit fractions of a turn (what the entry point takes)."""
    whole = []
    for f in freqs:
        t = int(round(f / (2 * math.pi) * 2.0 ** 64)) % (1 << 64)
        whole.append(t - (1 << 64) if t >= 1 << 63 else t)
    return torch.tensor(whole, dtype=torch.int64)


def _points(case, gen, rows, heads, width, scale=1.0):
    """(B, rows, heads, width) normal points, in the case's storage order."""
    shape = (case["B"], heads, rows, width) if case.get("layout") == "bhmd" else \
        (case["B"], rows, heads, width)
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * scale
    x = x.to(DTYPES[case["dtype"]])
    return x.transpose(1, 2) if case.get("layout") == "bhmd" else x


def _spoil(x, lengths):
    """What a padded buffer holds past its lengths is anything at all."""
    at = torch.arange(x.shape[1], device="cuda")[None, :] >= lengths[:, None]
    x.masked_fill_(at[:, :, None, None], float("nan"))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    st = {"case": case}
    if case["op"] == "rotary":
        st["q"] = _points(case, gen, case["M"], case["H"], case["D"])
        st["k"] = _points(case, gen, case["M"], case["Hk"], case["D"])
        first = torch.randint(0, 64, (case["B"], 1), generator=gen, device="cuda")
        st["positions"] = (case["start"] + first +
                           torch.arange(case["M"], device="cuda")[None, :]).to(torch.int32)
        freqs, st["scale"] = _wavelengths(case)
        st["frequencies"] = _fixed_point(freqs).cuda()
        return st
    M, N, H, Hk, D, C = (case[x] for x in ("M", "N", "H", "Hk", "D", "C"))
    st["q"] = _points(case, gen, M, H, D)
    st["k"] = _points(case, gen, N, Hk, D)
    st["v"] = _points(case, gen, N, Hk, C)
    st["tau"] = 1.0 / math.sqrt(D)
    ql, kl = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in _lengths(case))
    st["q_lengths"] = ql if case["ragged"] == "both" else None
    st["k_lengths"] = kl if case["ragged"] != "no" else None
    if case["op"] == "vjp":
        st["g"] = _points(case, gen, M, H, C)
        st["g_lse"] = torch.randn((case["B"], H, M), generator=gen, device="cuda") \
            if case["g_lse"] else None
        out, st["lse"] = _plain_attention(st)
        kept = torch.empty_like(st["g"])
        kept.copy_(out)
        st["out"] = kept
    _spoil(st["q"], ql)
    _spoil(st["k"], kl)
    _spoil(st["v"], kl)
    return st


def _grouped(st, dtype):
    """q as (B, Hk, G, M, D), k and v as (B, Hk, 1, N, .) with zeros past the lengths, and the
    mask (B, 1, 1, M, N) of visible pairs."""
    case, q, k, v = st["case"], st["q"], st["k"], st["v"]
    B, M, N, H, Hk = (case[x] for x in ("B", "M", "N", "H", "Hk"))
    ql, kl = (torch.tensor(x, device=q.device) for x in _lengths(case))
    rows, cols = torch.arange(M, device=q.device), torch.arange(N, device=q.device)
    in_q, in_k = rows[None, :] < ql[:, None], cols[None, :] < kl[:, None]
    seen = in_q[:, :, None] & in_k[:, None, :]
    if case["causal"]:
        seen &= cols[None, None, :] <= rows[None, :, None] + (kl - ql)[:, None, None]
    q = q.to(dtype).masked_fill(~in_q[:, :, None, None], 0)
    k = k.to(dtype).masked_fill(~in_k[:, :, None, None], 0)
    v = v.to(dtype).masked_fill(~in_k[:, :, None, None], 0)
    q = q.reshape(B, M, Hk, H // Hk, -1).permute(0, 2, 3, 1, 4)
    return q, k.permute(0, 2, 1, 3)[:, :, None], v.permute(0, 2, 1, 3)[:, :, None], \
        seen[:, None, None]


def _plain_attention(st):
    case = st["case"]
    B, M, H, C = (case[x] for x in ("B", "M", "H", "C"))
    q, k, v, seen = _grouped(st, torch.float32)
    s = torch.matmul(q, k.transpose(-1, -2))
    s.mul_(st["tau"]).masked_fill_(~seen, float("-inf"))
    top = s.amax(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).min)
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / total.masked_fill(total == 0, 1)
    lse = (top + total.log())[..., 0].masked_fill(total[..., 0] == 0, float("-inf"))
    out = out.permute(0, 3, 1, 2, 4).reshape(B, M, H, C)
    return out.to(DTYPES[case["dtype"]]), lse.reshape(B, H, M)


def _plain_vjp(st):
    case = st["case"]
    B, M, N, H, Hk, D, C = (case[x] for x in ("B", "M", "N", "H", "Hk", "D", "C"))
    q, k, v, seen = _grouped(st, torch.float32)
    g = st["g"].float().reshape(B, M, Hk, H // Hk, C).permute(0, 2, 3, 1, 4)
    lse = st["lse"].reshape(B, Hk, H // Hk, M, 1)
    s = torch.matmul(q, k.transpose(-1, -2))
    p = s.mul_(st["tau"]).sub_(lse).masked_fill_(~seen, float("-inf")).exp_()
    grad_v = torch.matmul(p.transpose(-1, -2), g).sum(2)
    dp = torch.matmul(g, v.transpose(-1, -2))
    delta = (p * dp).sum(-1, keepdim=True)
    if st["g_lse"] is not None:
        delta = delta - st["g_lse"].reshape(B, Hk, H // Hk, M, 1)
    ds = dp.sub_(delta).mul_(p).mul_(st["tau"])
    grad_q = torch.matmul(ds, k)
    grad_k = torch.matmul(ds.transpose(-1, -2), q).sum(2)
    to = DTYPES[case["dtype"]]
    return {"q": grad_q.permute(0, 3, 1, 2, 4).reshape(B, M, H, D).to(to),
            "k": grad_k.permute(0, 2, 1, 3).contiguous().to(to),
            "v": grad_v.permute(0, 2, 1, 3).contiguous().to(to)}


def _turn(x, case, cos, sin, scale):
    R = case["R"]
    x = x.to(cos.dtype)
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if case["interleaved"] else \
        (x[..., :R // 2], x[..., R // 2:R])
    sin = -sin if case["transpose"] else sin
    ya, yb = (a * cos - b * sin) * scale, (a * sin + b * cos) * scale
    y = torch.stack([ya, yb], -1).flatten(-2) if case["interleaved"] else torch.cat([ya, yb], -1)
    return torch.cat([y, x[..., R:]], -1)


def _plain_rotary(st):
    case = st["case"]
    turns = (st["positions"].long()[..., None] * st["frequencies"]).float() * 2.0 ** -64
    angle = (turns * (2 * math.pi))[:, :, None, :]
    cos, sin = angle.cos(), angle.sin()
    to = DTYPES[case["dtype"]]
    return {"q": _turn(st["q"], case, cos, sin, st["scale"]).to(to),
            "k": _turn(st["k"], case, cos, sin, st["scale"]).to(to)}


def run(st):
    case = st["case"]
    if not own:
        if case["op"] == "rotary":
            return _plain_rotary(st)
        if case["op"] == "vjp":
            return _plain_vjp(st)
        out, lse = _plain_attention(st)
        return {"out": out, "lse": lse}
    import paper_2609_04910_gb300 as gs
    if case["op"] == "rotary":
        q, k = gs.gauss_sum_rotary(st["q"], st["positions"], st["frequencies"], k=st["k"],
                                   interleaved=case["interleaved"], transpose=case["transpose"],
                                   scale=st["scale"])
        return {"q": q, "k": k}
    masks = {"causal": case["causal"], "q_lengths": st["q_lengths"], "k_lengths": st["k_lengths"]}
    if case["op"] == "vjp":
        grads = gs.gauss_sum_attention_vjp(st["q"], st["k"], st["v"], st["out"], st["lse"],
                                           st["g"], st["tau"], g_lse=st["g_lse"], **masks)
        return dict(zip("qkv", grads))
    out, lse = gs.gauss_sum_attention(st["q"], st["k"], st["v"], st["tau"], **masks)
    return {"out": out, "lse": lse}


def exact(case, seed):
    if case["op"] != "rotary" and work(case)["flops"] > 6e12:
        return None
    st = prepare(case, seed)
    if case["op"] == "rotary":
        freqs, scale = _wavelengths(case)
        angle = st["positions"].double()[..., None] * torch.tensor(freqs, dtype=torch.float64,
                                                                   device="cuda")
        angle = angle[:, :, None, :]
        return {x: _turn(st[x].double(), case, angle.cos(), angle.sin(), scale) for x in "qk"}
    B, M, N, H, Hk, D, C = (case[x] for x in ("B", "M", "N", "H", "Hk", "D", "C"))
    f64 = {"dtype": torch.float64, "device": "cuda"}
    out, lse = torch.zeros(B, M, H, C, **f64), torch.full((B, H, M), float("-inf"), **f64)
    dq, dk, dv = (torch.zeros(B, *x, **f64) for x in ((M, H, D), (N, Hk, D), (N, Hk, C)))
    for b, (ql, kl) in enumerate(zip(*_lengths(case))):
        hidden = None
        if case["causal"]:
            hidden = torch.arange(kl, device="cuda")[None, :] > \
                torch.arange(ql, device="cuda")[:, None] + (kl - ql)
        for h in range(H):
            j = h // (H // Hk)
            q, k, v = st["q"][b, :ql, h].double(), st["k"][b, :kl, j].double(), \
                st["v"][b, :kl, j].double()
            s = st["tau"] * (q @ k.T)
            if hidden is not None:
                s = s.masked_fill(hidden, float("-inf"))
            z = torch.logsumexp(s, -1)
            p = torch.exp(s - z.clamp_min(-1e300)[:, None])
            lse[b, h, :ql], out[b, :ql, h] = z, p @ v
            if case["op"] != "vjp":
                continue
            g = st["g"][b, :ql, h].double()
            dp = g @ v.T
            extra = 0.0 if st["g_lse"] is None else st["g_lse"][b, h, :ql, None].double()
            ds = p * (dp - (p * dp).sum(-1, keepdim=True) + extra) * st["tau"]
            dq[b, :ql, h] = ds @ k
            dk[b, :kl, j] += ds.T @ q
            dv[b, :kl, j] += p.T @ g
    if case["op"] == "vjp":
        return {"q": dq, "k": dk, "v": dv}
    return {"out": out, "lse": lse}
