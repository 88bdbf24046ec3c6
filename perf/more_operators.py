"""Measured cases of the 4-bit attention cache: writing tokens into it, reading
them back, and attention over it.

``run`` computes them in plain 32-bit torch operations, or, where ``own`` is
true, through the package's entry points.  Shapes: q (B, M, H, D), new keys and
values (B, M, Hk, D) and (B, M, Hk, C); token m of problem b is token
m + k_length - q_length of its sequence, and with ``causal`` sees the keys up to
itself; query head h reads key head h // (H / Hk).

The cache is one array of bytes (pages, Hk, tokens of a page / 16, block bytes).
A block holds 16 tokens of one head: their key codes, their value codes, their
key groups, their value groups, each token after token.  Up to 64 channels are a
group with two bf16 numbers, the step s and the least value m:

    m = the least value, rounded down,   s = (the largest - m) / 15,
    code = (x - m) / s to the nearest whole number (ties to even), 0 .. 15,

where x - m, largest - m and the quotient by 15 are float32 numbers and a step
below 2^-126 counts as 0 (all codes 0); a token's value is m + s code.  Codes of
a key row lie in four chunks t = 0 .. 3, each a 32-bit word for every 32
channels j: channel 32 j + 8 t + p in bits 4 p .. 4 p + 3; codes of a value row in
eight chunks g = 0 .. 7, each a 16-bit word for every j: channel 32 j + 4 g + p.
A page table (B, pages of a problem) gives the page of every run of tokens; -1 is
no page.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "fp16": 2, "bf16": 2}


def _case(op, name, B, M, N, H, Hk, D, dtype, page=0, ragged="no", causal=False, layout="bmhd"):
    case = {"op": op, "B": B, "M": M, "N": N, "Hk": Hk, "D": D, "dtype": dtype, "page": page,
            "ragged": ragged, "layout": layout}
    if op == "attention":
        case.update({"H": H, "causal": causal})
    if name:
        case["name"] = name
    return case


def _write(name, B, M, N, Hk, D, dtype, page=0, ragged="no", layout="bmhd"):
    return _case("write", name, B, M, N, Hk, Hk, D, dtype, page, ragged, layout=layout)


def _read(name, B, M, N, Hk, D, dtype, page=0, ragged="no"):
    return _case("read", name, B, M, N, Hk, Hk, D, dtype, page, ragged)


def _attend(name, B, M, N, H, Hk, D, dtype, page=0, ragged="no", causal=True, layout="bmhd"):
    return _case("attention", name, B, M, N, H, Hk, D, dtype, page, ragged, causal, layout)


def listed():
    return [
        # The new token of each of 64 sequences goes into its page: latency alone.
        _write("write_token_bf16", 64, 1, 2048, 8, 128, "bf16", 64, "keys"),
        # A padded batch of prompts into caches of their own.
        _write("write_prompts_fp16", 3, 1027, 1027, 4, 64, "fp16", 0, "both", "bhmd"),
        # Long prompts of a whole batch.
        _write("write_batch_bf16", 8, 4096, 4096, 8, 128, "bf16", 128),
        # Points kept in full precision until now.
        _write("write_points_fp32", 2, 700, 1501, 4, 32, "fp32"),
        # A kept prefix comes back, to be attended to or trained on in 16 bits.
        _read("read_prefix_bf16", 4, 8192, 8192, 8, 128, "bf16", 64),
        # The last tokens of uneven sequences in small pages, heads of 80 channels.
        _read("read_last_fp16", 5, 333, 1500, 6, 80, "fp16", 16, "both"),
        # One new token of each of 16 sequences against caches of uneven length.
        _attend("token_bf16", 16, 1, 8191, 32, 8, 128, "bf16", 64, "keys"),
        # One new token of a single sequence, short cache: latency alone.
        _attend("token_short_fp16", 1, 1, 333, 8, 8, 64, "fp16"),
        # One new token of a single very long sequence.
        _attend("token_long_bf16", 1, 1, 131071, 32, 8, 128, "bf16", 256),
        # A few drafted tokens of each sequence, checked in one pass.
        _attend("drafts_fp16", 8, 5, 4097, 28, 4, 128, "fp16", 32, "keys", True, "bhmd"),
        # The next part of two prompts against what is already in the cache.
        _attend("chunk_bf16", 2, 1024, 8192, 32, 8, 128, "bf16", 128),
        # One query of each point cloud in full precision.
        _attend("token_points_fp32", 2, 1, 1501, 4, 4, 32, "fp32", 0, "keys", False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        for x in ("bytes", "flops"):
            most[c["op"], x] = max(w[x], most.get((c["op"], x), 0))
    while True:
        op = rng.choice(["write", "read", "attention", "attention", "attention"])
        D = rng.choice([32, 64, 80, 96, 128, 128])
        Hk = rng.choice([1, 2, 4, 8, 12])
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp16", "fp32"])
        page = rng.choice([0, 16, 32, 64, 128, 256])
        B = _log_int(rng, 1, 64)
        if op == "attention":
            N = _log_int(rng, 16, 131072)
            M = rng.choice([1, 1, 1, _log_int(rng, 2, 16), _log_int(rng, 16, 1024)])
            H = Hk * rng.choice([1, 1, 2, 4, 7, 8])
            if dtype == "fp32":
                D = rng.choice([16, 32, 64])
            c = _attend(None, B, min(M, N), N, H, Hk, D, dtype, page,
                        rng.choice(["no", "keys", "both"]), rng.random() < 0.7,
                        rng.choice(["bmhd", "bhmd"]))
        else:
            N = _log_int(rng, 16, 8192)
            M = rng.choice([1, _log_int(rng, 2, N), N])
            make = _write if op == "write" else _read
            c = make(None, B, M, N, Hk, D, dtype, page, rng.choice(["no", "keys", "both"]))
        w = work(c)
        if all(w[x] <= most[op, x] for x in ("bytes", "flops")) and _stored(c) <= 1 << 30:
            return c


def _stored(case):
    """Tokens x heads x channels that the caches have room for."""
    return case["B"] * case["N"] * case["Hk"] * case["D"]


def _lengths(case):
    """(q_lengths, k_lengths) as lists: the first problem is full, later ones shorter, some odd."""
    B, M, N = case["B"], case["M"], case["N"]
    short = [b / (2.0 * B) for b in range(B)]
    ql = [M - int(M * s) for s in short] if case["ragged"] == "both" else [M] * B
    kl = [N - int(N * s) for s in short] if case["ragged"] != "no" else [N] * B
    return ql, kl


def _row_bytes(D):
    """Bytes of a row's codes, and groups of a row."""
    return (D + 31) // 32 * 16, (D + 63) // 64


def work(case):
    B, M, Hk, D, es = case["B"], case["M"], case["Hk"], case["D"], BYTES[case["dtype"]]
    ql, kl = _lengths(case)
    token = 2 * Hk * (0.5 * D + 4 * _row_bytes(D)[1])         # bytes of a token's codes and groups
    if case["op"] != "attention":
        taken = sum(min(q, k) for q, k in zip(ql, kl))
        wide = 2 * Hk * D * es
        read = taken * wide if case["op"] == "write" else 0
        per_value = 8.0 if case["op"] == "write" else 2.0
        return {"bytes": read + taken * token + B * M * wide,
                "flops": per_value * taken * 2 * Hk * D}
    H = case["H"]
    pairs = 0
    for q, k in zip(ql, kl):
        if not case["causal"]:
            pairs += q * k
        else:
            first = max(0, q - k)
            rows = max(0, q - first)
            pairs += rows * (first + k - q + 1) + rows * (rows - 1) // 2
    rows = sum(ql) * H
    return {"bytes": 2 * rows * D * es + 4 * rows + sum(kl) * token, "flops": 4.0 * pairs * H * D}


# ---------------------------------------------------------------- the stored form, in plain operations

def _groups(x):
    """x (..., D) in groups: (..., groups, 64), the last one filled with its first value."""
    D = x.shape[-1]
    n = (D + 63) // 64
    if D == n * 64:
        return x.unflatten(-1, (n, 64))
    fill = x[..., (n - 1) * 64:(n - 1) * 64 + 1].expand(*x.shape[:-1], n * 64 - D)
    return torch.cat([x, fill], -1).unflatten(-1, (n, 64))


def _down_bf16(x):
    """float32 values rounded down to bf16 numbers, still float32."""
    bits = x.view(torch.int32)
    low = bits & 0xFFFF
    return torch.where((bits < 0) & (low != 0), bits - low + 0x10000, bits - low).view(torch.float32)


def _quantise(x):
    """Codes (uint8, (..., D)), s and m (bf16, (..., groups)) of rows x (..., D)."""
    D = x.shape[-1]
    x = _groups(x.float())
    fine = torch.isfinite(x).all(-1)
    x = torch.where(fine[..., None], x, 0.0)
    m = _down_bf16(x.amin(-1))
    s = ((x.amax(-1) - m) / torch.full_like(m, 15.0)).bfloat16()    # (a scalar would be inverted)
    s = torch.where(s.float() < 2.0 ** -126, torch.zeros_like(s), s)
    fine &= torch.isfinite(s)
    step = torch.where(s > 0, s, torch.ones_like(s)).double()[..., None]
    code = torch.round((x - m[..., None]).double() / step).clamp(0, 15)
    code = torch.where((s > 0)[..., None] & fine[..., None], code, 0.0).to(torch.uint8)
    nan = torch.full_like(s, float("nan"))
    return code.flatten(-2)[..., :D], torch.where(fine, s, nan), torch.where(fine, m.bfloat16(), nan)


def _pack(code, chunks):
    """Bytes (..., 16 W) of codes (..., D): four chunks (keys) or eight (values)."""
    D = code.shape[-1]
    W = (D + 31) // 32
    if D < 32 * W:
        code = torch.nn.functional.pad(code, (0, 32 * W - D))
    x = code.unflatten(-1, (W, chunks, 16 // chunks, 2))
    return (x[..., 0] | (x[..., 1] << 4)).transpose(-3, -2).flatten(-3)


def _unpack(data, D, chunks):
    W = (D + 31) // 32
    x = data.unflatten(-1, (chunks, W, 16 // chunks)).transpose(-3, -2)
    return torch.stack([x & 15, x >> 4], -1).flatten(-4)[..., :D]


def _parts(data, D):
    """Views of the cache's bytes: key codes, value codes, key groups, value groups, each
    (pages, Hk, blocks, 16, bytes)."""
    row, n = _row_bytes(D)
    at, out = 0, []
    for size in (row, row, 4 * n, 4 * n):
        out.append(data[..., at:at + 16 * size].unflatten(-1, (16, size)))
        at += 16 * size
    return out


def _stored_rows(x, chunks):
    """Bytes of the codes and of the groups of rows x (..., D)."""
    code, s, m = _quantise(x)
    groups = torch.stack([s, m], -1).flatten(-2).contiguous().view(torch.uint8)
    return _pack(code, chunks), groups


def _values(codes, groups, D, chunks, dtype):
    """Rows (..., D) that stored codes and groups stand for."""
    pair = groups.contiguous().view(torch.bfloat16).to(dtype).unflatten(-1, (-1, 2))
    code = _unpack(codes, D, chunks).to(dtype)
    per = pair.repeat_interleave(64, -2)[..., :D, :]
    return per[..., 1] + per[..., 0] * code


def _place(case, table, b, token):
    """(page, block, row) of tokens of problems b."""
    if table is None:
        return b, token // 16, token % 16
    T = case["page"]
    return table.long()[b, token // T], token % T // 16, token % 16


def _store(case, data, table, b, token, k, v):
    """Rows k and v (n, Hk, D) of tokens into the cache."""
    kc, vc, kg, vg = _parts(data, case["D"])
    page, block, row = _place(case, table, b, token)
    for x, codes, groups, chunks in ((k, kc, kg, 4), (v, vc, vg, 8)):
        new_codes, new_groups = _stored_rows(x, chunks)
        codes[page, :, block, row] = new_codes
        groups[page, :, block, row] = new_groups


def _new_tokens(case):
    """Index tensors (b, m, token) of the new tokens that have a place."""
    ql, kl = (np.array(x) for x in _lengths(case))
    first = np.maximum(0, ql - kl)
    b = np.repeat(np.arange(case["B"]), ql - first)
    m = np.concatenate([np.arange(f, q) for f, q in zip(first, ql)])
    index = torch.from_numpy(np.stack([b, m, m + (kl - ql)[b]])).cuda()
    return index.unbind(0)


def _fetch(case, data, table, b, token, dtype):
    """Rows k and v (n, Hk, D) of tokens from the cache."""
    D = case["D"]
    kc, vc, kg, vg = _parts(data, D)
    at = _place(case, table, b, token)
    page, block, row = at
    return [_values(codes[page, :, block, row], groups[page, :, block, row], D, chunks, dtype)
            for codes, groups, chunks in ((kc, kg, 4), (vc, vg, 8))]


# ---------------------------------------------------------------- inputs

def _points(case, gen, rows, heads, width):
    shape = (case["B"], heads, rows, width) if case["layout"] == "bhmd" else \
        (case["B"], rows, heads, width)
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    x = x.to(DTYPES[case["dtype"]])
    return x.transpose(1, 2) if case["layout"] == "bhmd" else x


def _spoil(x, lengths):
    """What a padded buffer holds past its lengths is anything at all."""
    at = torch.arange(x.shape[1], device="cuda")[None, :] >= lengths[:, None]
    x.masked_fill_(at[:, :, None, None], float("nan"))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    B, M, N, Hk, D, page = (case[x] for x in ("B", "M", "N", "Hk", "D", "page"))
    st = {"case": case}
    ql, kl = _lengths(case)
    qt, kt = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (ql, kl))
    st["q_lengths"] = qt if case["ragged"] == "both" else None
    st["k_lengths"] = kt        # a cache has room for more than it holds
    row, n = _row_bytes(D)
    block = 16 * 2 * (row + 4 * n)
    if page:
        # Pages in no order, some of the pool not in use, none where a problem has no tokens.
        per = (N + page - 1) // page
        pool = B * per + 3
        table = torch.randperm(pool, generator=gen, device="cuda")[:B * per].view(B, per)
        used = torch.arange(per, device="cuda")[None, :] * page < kt[:, None]
        st["table"] = torch.where(used, table, -1).to(torch.int32)
    else:
        pool, st["table"] = B, None
    blocks = (page or (N + 15) // 16 * 16) // 16
    st["cache"] = torch.randint(0, 256, (pool, Hk, blocks, block), generator=gen, device="cuda",
                                dtype=torch.uint8)      # whatever the pool held before
    if case["op"] == "write":
        st["k"], st["v"] = _points(case, gen, M, Hk, D), _points(case, gen, M, Hk, D)
        _spoil(st["k"], qt)
        _spoil(st["v"], qt)
        return st
    for b in range(B):
        for t0 in range(0, kl[b], 16384):
            token = torch.arange(t0, min(kl[b], t0 + 16384), device="cuda")
            k, v = (torch.randn(token.numel(), Hk, D, generator=gen, device="cuda")
                    for _ in range(2))
            k *= 1 + (torch.arange(D, device="cuda") % 29 == 7) * 3.0      # channels that stand out
            _store(case, st["cache"], st["table"], torch.full_like(token, b), token, k, v)
    if case["op"] == "attention":
        st["q"] = _points(case, gen, M, case["H"], D)
        st["tau"] = 1.0 / math.sqrt(D)
        _spoil(st["q"], qt)
    return st


# ---------------------------------------------------------------- one pass

def _plain_read(st):
    case = st["case"]
    b, m, token = _new_tokens(case)
    shape = (case["B"], case["M"], case["Hk"], case["D"])
    out = {}
    for name, rows in zip("kv", _fetch(case, st["cache"], st["table"], b, token, torch.float32)):
        out[name] = torch.zeros(shape, dtype=DTYPES[case["dtype"]], device="cuda")
        out[name][b, m] = rows.to(DTYPES[case["dtype"]])
    return out


def _plain_write(st):
    case = st["case"]
    b, m, token = _new_tokens(case)
    _store(case, st["cache"], st["table"], b, token, st["k"][b, m], st["v"][b, m])
    return _plain_read(st)


def _plain_attention(st):
    case = st["case"]
    B, M, N, H, Hk, D = (case[x] for x in ("B", "M", "N", "H", "Hk", "D"))
    parts = _parts(st["cache"], D)
    if st["table"] is None:
        rows = [x.flatten(2, 3)[:, :, :N] for x in parts]
    else:
        at = st["table"].long().clamp_min(0)
        rows = [x[at].transpose(1, 2).flatten(2, 4)[:, :, :N] for x in parts]
    ql, kl = (torch.tensor(x, device="cuda") for x in _lengths(case))
    r, c = torch.arange(M, device="cuda"), torch.arange(N, device="cuda")
    in_q, in_k = r[None, :] < ql[:, None], c[None, :] < kl[:, None]
    seen = in_q[:, :, None] & in_k[:, None, :]
    if case["causal"]:
        seen &= c[None, None, :] <= r[None, :, None] + (kl - ql)[:, None, None]
    seen = seen[:, None, None]
    hide = ~in_k[:, None, :, None]
    k = _values(rows[0], rows[2], D, 4, torch.float32).masked_fill_(hide, 0)[:, :, None]
    q = st["q"].float().masked_fill(~in_q[:, :, None, None], 0)
    q = q.reshape(B, M, Hk, H // Hk, D).permute(0, 2, 3, 1, 4)
    s = torch.matmul(q, k.transpose(-1, -2))
    del k
    s.mul_(st["tau"]).masked_fill_(~seen, float("-inf"))
    top = s.amax(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).min)
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    v = _values(rows[1], rows[3], D, 8, torch.float32).masked_fill_(hide, 0)[:, :, None]
    out = torch.matmul(p, v) / total.masked_fill(total == 0, 1)
    lse = (top + total.log())[..., 0].masked_fill(total[..., 0] == 0, float("-inf"))
    out = out.permute(0, 3, 1, 2, 4).reshape(B, M, H, D)
    return {"out": out.to(DTYPES[case["dtype"]]), "lse": lse.reshape(B, H, M)}


def run(st):
    case = st["case"]
    if not own:
        return {"write": _plain_write, "read": _plain_read, "attention": _plain_attention}[case["op"]](st)
    import paper_2609_04910_gb300 as gs
    cache = gs.AttentionCache(st["cache"], case["D"])
    where = {"q_lengths": st["q_lengths"], "k_lengths": st["k_lengths"], "page_table": st["table"]}
    if case["op"] == "attention":
        out, lse = gs.gauss_sum_attention_cached(st["q"], cache, st["tau"], causal=case["causal"],
                                                 **where)
        return {"out": out, "lse": lse}
    if case["op"] == "write":
        gs.gauss_sum_cache_write(cache, st["k"], st["v"], **where)
    k, v = gs.gauss_sum_cache_read(cache, case["M"], DTYPES[case["dtype"]], **where)
    return {"k": k, "v": v}


# ---------------------------------------------------------------- the definition in 64 bits

def _round_trip64(x):
    """What rows x (..., D) become in the cache, group by group."""
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    for c in range(0, x.shape[-1], 64):
        y = x[..., c:c + 64].double()
        low, high = y.min(-1, keepdim=True).values, y.max(-1, keepdim=True).values
        # 8 significant bits, towards minus infinity (numbers of ordinary size).
        unit = torch.exp2(torch.floor(torch.log2(low.abs().clamp_min(1e-30))) - 7)
        m = torch.where(low == 0, low, torch.floor(low / unit) * unit)
        s = ((high - m).float().double() / 15).float().bfloat16().double()
        code = torch.round((y - m).float().double() / s.clamp_min(1e-30)).clamp(0, 15)
        out[..., c:c + 64] = m + s * code
    return out


def _nibbles64(codes, groups, D, chunk_bytes):
    """Rows of stored bytes as float64, channel by channel: chunk_bytes bytes of each chunk belong
    to one run of 32 channels."""
    row = codes.long()
    W = row.shape[-1] // 16
    chan = torch.arange(D, device="cuda")
    j, inside = chan // 32, chan % 32
    chunk, p = inside // (2 * chunk_bytes), inside % (2 * chunk_bytes)
    at = (chunk * W + j) * chunk_bytes + p // 2
    code = (row[..., at] >> (4 * (p % 2))) & 15
    # The upper 16 bits of a float32 number are the bf16 number.
    word = groups.long().unflatten(-1, (-1, 2))
    half = ((word[..., 0] | (word[..., 1] << 8)) << 16).to(torch.int32)
    half = half.view(torch.float32).double()
    return half[..., 2 * (chan // 64) + 1] + half[..., 2 * (chan // 64)] * code.double()


def exact(case, seed):
    if case["op"] == "attention" and work(case)["flops"] > 1e12:
        return None
    st = prepare(case, seed)
    B, M, Hk, D = (case[x] for x in ("B", "M", "Hk", "D"))
    ql, kl = _lengths(case)
    f64 = {"dtype": torch.float64, "device": "cuda"}

    def tokens(b, h, first, last):
        """k and v of tokens first .. last - 1 of one problem and head."""
        t = torch.arange(first, last, device="cuda")
        T = st["cache"].shape[2] * 16
        page = torch.full_like(t, b) if st["table"] is None else st["table"].long()[b, t // T]
        block = st["cache"][page, h, t % T // 16]
        row, n = _row_bytes(D)
        each = []
        for size, start in ((row, 0), (row, 16 * row), (4 * n, 32 * row), (4 * n, 32 * row + 64 * n)):
            col = start + (t % 16)[:, None] * size + torch.arange(size, device="cuda")[None, :]
            each.append(block.gather(1, col))
        return _nibbles64(each[0], each[2], D, 4), _nibbles64(each[1], each[3], D, 2)

    if case["op"] != "attention":
        out = {x: torch.zeros(B, M, Hk, D, **f64) for x in "kv"}
        for b in range(B):
            first = max(0, ql[b] - kl[b])
            if case["op"] == "write":
                for x in "kv":
                    out[x][b, first:ql[b]] = _round_trip64(st[x][b, first:ql[b]])
                continue
            for h in range(Hk):
                out["k"][b, first:ql[b], h], out["v"][b, first:ql[b], h] = \
                    tokens(b, h, first + kl[b] - ql[b], kl[b])
        return out
    H = case["H"]
    out, lse = torch.zeros(B, M, H, D, **f64), torch.full((B, H, M), float("-inf"), **f64)
    for b in range(B):
        hidden = None
        if case["causal"]:
            hidden = torch.arange(kl[b], device="cuda")[None, :] > \
                torch.arange(ql[b], device="cuda")[:, None] + (kl[b] - ql[b])
        for j in range(Hk):
            k, v = tokens(b, j, 0, kl[b])
            for h in range(j * (H // Hk), (j + 1) * (H // Hk)):
                s = st["tau"] * (st["q"][b, :ql[b], h].double() @ k.T)
                if hidden is not None:
                    s = s.masked_fill(hidden, float("-inf"))
                z = torch.logsumexp(s, -1)
                p = torch.exp(s - z.clamp_min(-1e300)[:, None])
                lse[b, h, :ql[b]], out[b, :ql[b], h] = z, p @ v
    return {"out": out, "lse": lse}
