"""Softmax attention and its gradients on the GPU against float64."""
import math

import pytest
import torch

from attention_forms import DT, attention64, within

pytestmark = pytest.mark.gpu

NAN = float("nan")


def points(shape, dtype, seed, layout="bmhd", scale=1.0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    B, rows, heads, width = shape
    if layout == "bmhd":
        x = torch.randn(B, rows, heads, width, generator=gen, device="cuda")
        return (x * scale).to(DT[dtype])
    if layout == "bhmd":
        x = torch.randn(B, heads, rows, width, generator=gen, device="cuda")
        return (x * scale).to(DT[dtype]).transpose(1, 2)
    if layout == "wide":       # a slice of wider rows, 16-byte aligned
        x = torch.randn(B, rows, heads, width + 24, generator=gen, device="cuda")
        return (x * scale).to(DT[dtype])[..., 8:8 + width]
    if layout == "odd":        # a slice off every alignment but the element's
        x = torch.randn(B, rows, heads, width + 3, generator=gen, device="cuda")
        return (x * scale).to(DT[dtype])[..., 1:1 + width]
    raise ValueError(layout)


def spoil(x, lengths):
    if lengths is not None:
        for b, n in enumerate(lengths.tolist()):
            x[b, max(n, 0):] = NAN
    return x


def ints(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


def run(B, M, N, H, Hk, D, C, dtype, causal=False, ql=None, kl=None, layout="bmhd", seed=0,
        g_lse=False, tau=None, scale=1.0, g_scale=1.0, grads=True):
    import paper_2609_04910_gb300 as gs
    tau = 1 / math.sqrt(D) if tau is None else tau
    ql, kl = ints(ql), ints(kl)
    q = points((B, M, H, D), dtype, seed, layout, scale)
    k = points((B, N, Hk, D), dtype, seed + 1, layout, scale)
    v = points((B, N, Hk, C), dtype, seed + 2, layout)
    g = points((B, M, H, C), dtype, seed + 3, layout, g_scale)
    z = points((B, H, M, 1), "fp32", seed + 4, scale=g_scale)[..., 0].contiguous() if g_lse else None
    want = attention64(q, k, v, tau, causal, ql, kl, g, z)
    spoil(q, ql), spoil(k, kl), spoil(v, kl), spoil(g, ql)
    if z is not None and ql is not None:
        spoil(z.transpose(1, 2), ql)
    masks = dict(causal=causal, q_lengths=ql, k_lengths=kl)
    out, lse = gs.gauss_sum_attention(q, k, v, tau, **masks)
    gs.gauss_sum_device_status()
    assert out.dtype == q.dtype and lse.dtype == torch.float32
    worst = {"out": within(out, want["out"]), "lse": within(lse, want["lse"])}
    if grads:
        given = want["out"][0].to(q.dtype)
        spoil(given, ql)
        got = gs.gauss_sum_attention_vjp(q, k, v, given, want["lse"][0].float(), g, tau, g_lse=z,
                                         **masks)
        gs.gauss_sum_device_status()
        worst.update({x: within(t, want[x]) for x, t in zip("qkv", got)})
    assert all(w <= 1 for w in worst.values()), worst
    return worst


SIZES = [(1, 1, 1), (1, 1, 129), (2, 3, 1), (1, 64, 64), (1, 65, 63), (2, 127, 130), (1, 128, 128),
         (1, 129, 257), (1, 300, 515), (2, 513, 200), (1, 1, 4100), (3, 5, 1000)]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("B,M,N", SIZES)
def test_sizes(B, M, N, dtype, causal):
    run(B, M, N, 4, 2, 64, 64, dtype, causal, seed=M + N)


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("D,C", [(1, 1), (8, 24), (20, 36), (32, 32), (64, 128), (72, 40), (96, 48),
                                 (128, 64), (128, 128), (130, 16), (192, 128), (256, 256)])
def test_widths(D, C, dtype):
    run(2, 140, 150, 2, 1, D, C, dtype, True, ql=[140, 77], kl=[150, 131], seed=D + C)


@pytest.mark.parametrize("H,Hk", [(1, 1), (5, 5), (7, 1), (12, 4), (40, 8)])
@pytest.mark.parametrize("M", [1, 2, 9, 200])
def test_head_groups(H, Hk, M):
    run(2, M, 333, H, Hk, 64, 64, "bf16", True, kl=[333, 290], seed=H + M)


@pytest.mark.parametrize("layout", ["bmhd", "bhmd", "wide", "odd"])
@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("M", [1, 150])
def test_layouts(layout, dtype, M):
    run(2, M, 260, 4, 2, 64, 64, dtype, True, kl=[260, 199], layout=layout, seed=5)


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("ql,kl", [([0, 5, 200], [300, 0, 1]), ([200, 130, 1], [1, 129, 300]),
                                   ([200, 200, 200], [128, 127, 0]), ([999, -4, 200], [300, 300, 9999])])
def test_lengths_leave_rows_empty(ql, kl, causal, dtype):
    # Padding holds NaN, causal rows past the keys see nothing, lengths clamp.
    run(3, 200, 300, 4, 2, 64, 64, dtype, causal, ql=ql, kl=kl, seed=11, g_lse=True)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("N", [2, 8, 9, 24, 25, 33])
@pytest.mark.parametrize("D,C", [(64, 64), (40, 20), (128, 96), (100, 128)])
def test_rows_of_few_keys(D, C, N, causal, dtype):
    run(2, 140, N, 4, 2, D, C, dtype, causal, kl=[N, N // 2], seed=N + D, g_lse=True)
    run(2, 70, 300, 2, 1, D, C, dtype, causal, ql=[70, 33], kl=[300, N], seed=N + D + 1)


@pytest.mark.parametrize("D,C", [(64, 64), (128, 72), (16, 128)])
@pytest.mark.parametrize("N", [1, 128, 129, 256, 384, 385, 2500])
@pytest.mark.parametrize("M", [1, 3, 40, 127])
def test_few_tokens(M, N, D, C):
    # One key tile or several to a block, one split or several, rows with
    # keys in one stream only.
    run(2, M, N, 12, 3, D, C, "fp16", True, ql=[M, M // 2], kl=[N, (N + 1) // 2], seed=M + N,
        grads=False)


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
def test_more_queries_than_keys(dtype):
    run(1, 400, 130, 2, 2, 64, 64, dtype, True, seed=3, g_lse=True)


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
def test_sharp_and_flat_scores(dtype):
    run(1, 200, 700, 2, 2, 64, 64, dtype, scale=3.0, seed=1)       # nearly one-hot rows
    run(1, 200, 700, 2, 2, 64, 64, dtype, scale=0.01, seed=2)      # nearly uniform rows
    run(1, 130, 9000, 2, 2, 64, 64, dtype, seed=3)


@pytest.mark.parametrize("g_scale", [1e-4, 1.0, 300.0])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_gradient_range(dtype, g_scale):
    # Upstream gradients far from one keep their relative precision.
    run(1, 150, 2000, 2, 1, 64, 64, dtype, seed=9, g_scale=g_scale, g_lse=True)


@pytest.mark.parametrize("rising", [False, True])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_running_maximum(dtype, rising):
    # Scores that keep rising (or falling) along the keys move the maximum at every tile.
    import paper_2609_04910_gb300 as gs
    N, D = 1500, 64
    q = torch.full((1, 130, 1, D), 1.0, device="cuda").to(DT[dtype])
    ramp = torch.linspace(-30, 30, N, device="cuda")
    ramp = ramp if rising else ramp.flip(0)
    k = (ramp[None, :, None, None] / 8).expand(1, N, 1, D).contiguous().to(DT[dtype])
    v = points((1, N, 1, D), dtype, 4)
    want = attention64(q, k, v, 0.125)
    out, lse = gs.gauss_sum_attention(q, k, v, 0.125)
    gs.gauss_sum_device_status()
    assert within(out, want["out"]) <= 1 and within(lse, want["lse"]) <= 1


def test_all_scores_far_below_zero():
    # exp of every score underflows in fp32: the running maximum keeps the result.
    import paper_2609_04910_gb300 as gs
    for dtype in ("fp32", "fp16", "bf16"):
        q = torch.full((1, 3, 2, 64), -8.0, device="cuda").to(DT[dtype])
        k = points((1, 300, 2, 64), dtype, 1, scale=0.01) + 8
        v = points((1, 300, 2, 64), dtype, 2)
        want = attention64(q, k, v, 1.0)
        out, lse = gs.gauss_sum_attention(q, k, v, 1.0)
        assert within(out, want["out"]) <= 1 and within(lse, want["lse"]) <= 1


def test_broadcast_keys():
    # Keys and values shared by the problems of a batch, as a stride of zero.
    import paper_2609_04910_gb300 as gs
    for dtype in ("fp32", "fp16", "bf16"):
        q = points((3, 70, 4, 64), dtype, 1)
        k = points((1, 200, 2, 64), dtype, 2).expand(3, 200, 2, 64)
        v = points((1, 200, 2, 64), dtype, 3).expand(3, 200, 2, 64)
        g = points((3, 70, 4, 64), dtype, 4)
        want = attention64(q, k, v, 0.125, g=g)
        out, lse = gs.gauss_sum_attention(q, k, v, 0.125)
        assert within(out, want["out"]) <= 1 and within(lse, want["lse"]) <= 1
        got = gs.gauss_sum_attention_vjp(q, k, v, want["out"][0].to(q.dtype), lse, g, 0.125)
        for x, t in zip("qkv", got):
            assert within(t, want[x]) <= 1, x


def test_gradient_against_differences():
    # Central differences of the float64 forward along a random direction.
    import paper_2609_04910_gb300 as gs
    B, M, N, H, Hk, D, C, tau = 2, 37, 45, 4, 2, 24, 16, 0.3
    q, k, v = (points(s, "fp32", i) for i, s in enumerate(
        [(B, M, H, D), (B, N, Hk, D), (B, N, Hk, C)]))
    g, z = points((B, M, H, C), "fp32", 7), points((B, H, M, 1), "fp32", 8)[..., 0].contiguous()
    kl = ints([45, 30])

    def loss(t):
        moved = [x.double() + t * d for x, d in zip((q, k, v), dirs)]
        r = plain64(*moved, tau, kl)
        return float((r[0] * g).sum() + (r[1] * z).sum())

    def plain64(q, k, v, tau, kl):
        s = torch.einsum("bmjgd,bnjd->bjgmn", q.reshape(B, M, Hk, H // Hk, D), k) * tau
        n = torch.arange(N, device="cuda")
        m = torch.arange(M, device="cuda")
        seen = (n[None, None] < kl[:, None, None]) & \
            (n[None, None] <= m[None, :, None] + (kl - M)[:, None, None])
        s = s.masked_fill(~seen[:, None, None], -float("inf"))
        lse = torch.logsumexp(s, -1)
        p = torch.where(torch.isfinite(lse)[..., None], torch.exp(s - lse[..., None]), 0.0)
        o = torch.einsum("bjgmn,bnjc->bmjgc", p, v).reshape(B, M, H, C)
        return o, torch.where(torch.isfinite(lse), lse, 0.0).reshape(B, H, M)

    out, lse = gs.gauss_sum_attention(q, k, v, tau, causal=True, k_lengths=kl)
    grads = gs.gauss_sum_attention_vjp(q, k, v, out, lse, g, tau, g_lse=z, causal=True,
                                       k_lengths=kl)
    for x in range(3):
        dirs = [points(t.shape, "fp32", 20 + i).double() if i == x else torch.zeros_like(t).double()
                for i, t in enumerate((q, k, v))]
        h = 1e-4
        slope = (loss(h) - loss(-h)) / (2 * h)
        mine = float((grads[x].double() * dirs[x]).sum())
        # Differences: h^2 / 6 of a third derivative of order one, and 1e-15 / h of the loss.
        size = float((grads[x].double() * dirs[x]).abs().sum())
        assert abs(mine - slope) <= 1e-5 * size, (x, mine, slope)


def test_gauss_sum_through_attention():
    # Alg. 1: the Gauss sum is out e^lse e^(-tau/2 |q|^2) of values scaled by e^(-tau/2 |k|^2).
    import paper_2609_04910_gb300 as gs
    M, N, D, tau = 200, 333, 16, 1.0 / 16
    q, k, v = (points((1, n, 1, w), "fp32", i) for i, (n, w) in enumerate(
        [(M, D), (N, D), (N, 3)]))
    s = gs.gauss_sum(q[0, :, 0].contiguous(), k[0, :, 0].contiguous(), v[0, :, 0].contiguous(), tau)
    vs = v * torch.exp(-tau / 2 * (k * k).sum(-1, keepdim=True))
    out, lse = gs.gauss_sum_attention(q, k, vs, tau)
    mine = out[0, :, 0] * torch.exp(lse[0, 0] - tau / 2 * (q[0, :, 0] ** 2).sum(-1))[:, None]
    mass = gs.gauss_sum(q[0, :, 0].contiguous(), k[0, :, 0].contiguous(),
                        v[0, :, 0].abs().contiguous(), tau)
    # Both sides carry 1e-5 of the absolute mass at most (fp32, exponents below 8).
    assert float(((mine - s).abs() / mass).max()) <= 2e-5


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
def test_outputs_given_and_wanted(dtype):
    import paper_2609_04910_gb300 as gs
    q, k, v, g = (points((2, n, h, 64), dtype, i, "bhmd") for i, (n, h) in enumerate(
        [(90, 4), (140, 2), (140, 2), (90, 4)]))
    ref, ref_lse = gs.gauss_sum_attention(q, k, v, 0.1)
    out = points((2, 90, 4, 64), dtype, 9, "wide")
    lse = torch.empty(2, 4, 90, device="cuda")
    a, b = gs.gauss_sum_attention(q, k, v, 0.1, out=out, lse=lse)
    assert a is out and b is lse and torch.equal(out, ref) and torch.equal(lse, ref_lse)
    all_three = gs.gauss_sum_attention_vjp(q, k, v, ref, lse, g, 0.1)
    for i, x in enumerate("qkv"):
        one = gs.gauss_sum_attention_vjp(q, k, v, ref, lse, g, 0.1, want=(x,))
        assert [t is not None for t in one] == [y == x for y in "qkv"]
        assert torch.equal(one[i], all_three[i])
    to = points((2, 140, 2, 64), dtype, 9, "bhmd")
    got = gs.gauss_sum_attention_vjp(q, k, v, ref, lse, g, 0.1, want=(), grad_k=to)
    assert got[0] is None and got[1] is to and torch.equal(to, all_three[1])


def test_same_results_every_call():
    import paper_2609_04910_gb300 as gs
    q, k, v, g = (points((2, n, h, 128), "bf16", i) for i, (n, h) in enumerate(
        [(700, 8), (900, 2), (900, 2), (700, 8)]))
    first = None
    for _ in range(4):
        out, lse = gs.gauss_sum_attention(q, k, v, 0.1, causal=True)
        got = (out, lse, *gs.gauss_sum_attention_vjp(q, k, v, out, lse, g, 0.1, causal=True))
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(first, got))


def test_other_stream_and_empty_sizes():
    import paper_2609_04910_gb300 as gs
    q, k, v, g = (points((1, 300, 4, 64), "fp16", i) for i in range(4))
    out, lse = gs.gauss_sum_attention(q, k, v, 0.1)
    grads = gs.gauss_sum_attention_vjp(q, k, v, out, lse, g, 0.1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o2, l2 = gs.gauss_sum_attention(q, k, v, 0.1, stream=side)
    g2 = gs.gauss_sum_attention_vjp(q, k, v, o2, l2, g, 0.1, stream=side)
    side.synchronize()
    assert torch.equal(out, o2) and torch.equal(lse, l2)
    assert all(torch.equal(a, b) for a, b in zip(grads, g2))
    for B, M, N in ((0, 4, 4), (2, 0, 4), (2, 4, 0)):
        q, g = points((B, M, 4, 64), "fp16", 1), points((B, M, 4, 64), "fp16", 1)
        k = points((B, N, 2, 64), "fp16", 2)
        out, lse = gs.gauss_sum_attention(q, k, k, 0.1, causal=True)
        assert not out.any() and torch.isinf(lse).all()
        for t in gs.gauss_sum_attention_vjp(q, k, k, out, lse, g, 0.1, causal=True):
            assert not t.any()
    gs.gauss_sum_device_status()


def test_captured_in_a_graph():
    import paper_2609_04910_gb300 as gs
    q, k, v, g = (points((2, 260, h, 128), "bf16", i) for i, h in enumerate((8, 2, 2, 8)))
    out, lse = gs.gauss_sum_attention(q, k, v, 0.1, causal=True)
    grads = gs.gauss_sum_attention_vjp(q, k, v, out, lse, g, 0.1, causal=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o2, l2 = gs.gauss_sum_attention(q, k, v, 0.1, causal=True)
        g2 = gs.gauss_sum_attention_vjp(q, k, v, o2, l2, g, 0.1, causal=True)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, o2) and torch.equal(lse, l2)
    assert all(torch.equal(a, b) for a, b in zip(grads, g2))


def test_failed_workspace_is_reported():
    import paper_2609_04910_gb300 as gs
    from paper_2609_04910_gb300._binding import testing_fail_allocations
    q, k = points((1, 1, 4, 64), "bf16", 1), points((1, 5000, 4, 64), "bf16", 2)
    out, lse = gs.gauss_sum_attention(q, k, k, 0.1)
    testing_fail_allocations(True)
    try:
        with pytest.raises(gs.GaussSumError) as err:
            gs.gauss_sum_attention_vjp(q, k, k, out, lse, out, 0.1)
        assert err.value.status == 3
    finally:
        testing_fail_allocations(False)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("M", [1, 150])
def test_offsets_past_32_bits(dtype, M):
    # The second problem lies more than 2^31 elements (and 2^32 bytes) past the first.
    import paper_2609_04910_gb300 as gs
    N, H, Hk, D, far = 300, 4, 2, 64, 2 ** 31 + 64
    store = torch.empty(far + N * H * D * 8, dtype=DT[dtype], device="cuda")
    at = [0]

    def place(x):
        rows, heads = x.shape[1], x.shape[2]
        y = store[at[0]:].as_strided((2, rows, heads, D), (far, heads * D, D, 1))
        at[0] += rows * heads * D
        y.copy_(x)
        return y

    q, k, v, g = (place(points((2, n, h, D), dtype, i)) for i, (n, h) in enumerate(
        [(M, H), (N, Hk), (N, Hk), (M, H)]))
    want = attention64(q, k, v, 0.125, causal=True, g=g)
    out, lse = gs.gauss_sum_attention(q, k, v, 0.125, causal=True, out=place(torch.zeros_like(g)))
    assert within(out, want["out"]) <= 1 and within(lse, want["lse"]) <= 1
    to = {x: place(torch.zeros_like(t)) for x, t in zip("qkv", (q, k, v))}
    gs.gauss_sum_attention_vjp(q, k, v, place(want["out"][0].to(q.dtype)), lse, g, 0.125, causal=True,
                               grad_q=to["q"], grad_k=to["k"], grad_v=to["v"])
    gs.gauss_sum_device_status()
    for x in "qkv":
        assert within(to[x], want[x]) <= 1, x


def test_binding_refusals():
    import paper_2609_04910_gb300 as gs
    q, k = points((2, 30, 4, 64), "bf16", 1), points((2, 50, 2, 64), "bf16", 2)
    out, lse = gs.gauss_sum_attention(q, k, k, 0.1)
    good = dict(q=q, k=k, v=k, tau=0.1)
    bad = [dict(k=k.half()), dict(v=k.float()), dict(k=k[:1]), dict(v=k[:, :49]), dict(k=k[..., :32]),
           dict(q=q.transpose(2, 3)), dict(k_lengths=ints([1, 2]).long()), dict(k_lengths=ints([1])),
           dict(q_lengths=torch.ones(2, dtype=torch.int32)), dict(out=out[:, :29]), dict(out=out.float()),
           dict(lse=lse.double()), dict(lse=lse.transpose(1, 2)), dict(q=q.cpu())]
    for change in bad:
        with pytest.raises(ValueError):
            gs.gauss_sum_attention(**{**good, **change})
    for change in (dict(tau=0.0), dict(tau=float("nan")), dict(out=out[:, :1].expand(2, 30, 4, 64)),
                   dict(q=points((2, 30, 3, 64), "bf16", 1))):
        with pytest.raises(gs.GaussSumError):
            gs.gauss_sum_attention(**{**good, **change})
    grad = dict(good, out=out, lse=lse, g=out)
    for change in (dict(lse=None), dict(g=out[:1]), dict(g_lse=lse.half()), dict(grad_k=q), dict(out=out.half())):
        with pytest.raises(ValueError):
            gs.gauss_sum_attention_vjp(**{**grad, **change})
    table, _ = gs.rotary_frequencies(64)
    pos = torch.arange(30, device="cuda")
    gs.gauss_sum_rotary(q, pos, table)
    for change in (dict(positions=pos.float()), dict(positions=pos[:29]), dict(positions=pos.cpu()),
                   dict(frequencies=table.int()), dict(frequencies=table[None]), dict(k=k), dict(q_out=q.half())):
        with pytest.raises(ValueError):
            gs.gauss_sum_rotary(**{**dict(q=q, positions=pos, frequencies=table), **change})
    with pytest.raises(gs.GaussSumError):      # more rotated channels than there are
        gs.gauss_sum_rotary(q[..., :32], pos, table)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("M", [1, 150])
@pytest.mark.parametrize("D,C", [(20, 36), (100, 7), (1, 128), (66, 64)])
def test_odd_widths_in_aligned_rows(D, C, M, dtype):
    # Rows of 16-byte multiples that are not full: the tensor-core kernels take them.
    import paper_2609_04910_gb300 as gs
    wide = [points((2, n, h, 128), dtype, i) for i, (n, h) in enumerate(
        [(M, 4), (260, 2), (260, 2), (M, 4), (M, 4)])]
    q, k, v, g, out = (x[..., :w] for x, w in zip(wide, (D, D, C, C, C)))
    kl = ints([260, 131])
    spoil(wide[0][..., D:], ints([0, 0])), spoil(wide[1][..., D:], ints([0, 0]))
    spoil(wide[2][..., C:], ints([0, 0])), spoil(wide[3][..., C:], ints([0, 0]))
    want = attention64(q, k, v, 0.2, True, None, kl, g)
    kept = wide[4][..., C:].clone()
    _, lse = gs.gauss_sum_attention(q, k, v, 0.2, causal=True, k_lengths=kl, out=out)
    assert within(out, want["out"]) <= 1 and within(lse, want["lse"]) <= 1
    assert torch.equal(wide[4][..., C:], kept)        # nothing written past the width
    given = torch.zeros_like(wide[4])[..., :C]
    given.copy_(want["out"][0])
    got = gs.gauss_sum_attention_vjp(q, k, v, given, lse, g, 0.2, causal=True, k_lengths=kl)
    gs.gauss_sum_device_status()
    for x, t in zip("qkv", got):
        assert within(t, want[x]) <= 1, x


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("M", [3, 200])
def test_nan_and_overflow_are_not_hidden(dtype, M):
    import paper_2609_04910_gb300 as gs
    q, k, v = (points((1, n, 2, 64), dtype, i) for i, n in enumerate((M, 300, 300)))
    q[0, 1, 0, 5] = NAN                               # a query: its own row
    out, lse = gs.gauss_sum_attention(q, k, v, 0.1)
    assert torch.isnan(out[0, 1, 0]).all() and torch.isnan(lse[0, 0, 1])
    rest = torch.ones(1, M, 2, dtype=torch.bool, device="cuda")
    rest[0, 1, 0] = False
    assert torch.isfinite(out[rest]).all() and torch.isfinite(lse.transpose(1, 2)[rest]).all()
    q[0, 1, 0, 5] = 0
    v[0, 7, 1, 3] = NAN                               # a value: its channel in every row
    out, lse = gs.gauss_sum_attention(q, k, v, 0.1)
    assert torch.isnan(out[0, :, 1, 3]).all() and torch.isfinite(lse).all()
    assert torch.isfinite(out[0, :, 0]).all()
    if dtype == "fp16":                               # gradients past 65504 round to infinity
        v[0, 7, 1, 3] = 0
        g = torch.full((1, M, 2, 64), 60000.0, device="cuda").half()
        out, lse = gs.gauss_sum_attention(q, k, v, 0.1)
        dv = gs.gauss_sum_attention_vjp(q, k[:, :1], v[:, :1], v[:, :1].expand(1, M, 2, 64).contiguous(),
                                        (0.1 * (q * k[:, :1]).float().sum(-1)).transpose(1, 2).contiguous(),
                                        g, 0.1, want=("v",))[2]
        assert torch.isinf(dv).all()                  # M times 60000
