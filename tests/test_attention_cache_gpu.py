"""The 4-bit cache on the GPU: stored bytes against the definition of the
format, rows read back and attention over the cache against float64."""
import math

import pytest
import torch

from attention_cache_forms import DT, UNIT, attention64, quantise, row_bytes, values, within
from test_attention_gpu import ints, points, spoil

pytestmark = pytest.mark.gpu


def lengths_of(x, default, B):
    return [default] * B if x is None else [min(max(int(n), 0), default) for n in x]


class Store:
    """A cache with its page table, and the codes and groups that its tokens should have."""

    def __init__(self, B, N, Hk, D, C, page=0, seed=0, spare=3, fill=None):
        import paper_2609_04910_gb300 as gs
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.B, self.Hk, self.D, self.C = B, Hk, D, C
        if page:
            per = -(-N // page)
            pool = B * per + spare
            self.table = torch.randperm(pool, generator=gen, device="cuda")[:B * per].view(B, per).int()
            self.cache = gs.attention_cache(pool, page, Hk, D, C)
            self.N = per * page
        else:
            self.table, self.N = None, -(-N // 16) * 16
            self.cache = gs.attention_cache(B, self.N, Hk, D, C)
        self.cache.data.random_(0, 256, generator=gen) if fill is None else self.cache.data.fill_(fill)
        self.k = torch.zeros(B, self.N, Hk, D, dtype=torch.float64, device="cuda")
        self.v = torch.zeros(B, self.N, Hk, C, dtype=torch.float64, device="cuda")
        self.size = torch.zeros_like(self.v)

    def write(self, k, v, ql=None, kl=None):
        """Through the library, and into the float64 copy."""
        import paper_2609_04910_gb300 as gs
        gs.gauss_sum_cache_write(self.cache, k, v, q_lengths=ints(ql), k_lengths=ints(kl),
                                 page_table=self.table)
        M = k.shape[1]
        want = [quantise(x) for x in (k, v)]
        rows = [values(*x) for x in want]
        size = want[1][2].double().abs() + 15 * want[1][1].double()
        size = size[..., torch.arange(self.C, device="cuda") // 64]
        for b, (q, n) in enumerate(zip(lengths_of(ql, M, self.B), lengths_of(kl, self.N, self.B))):
            first = max(0, q - n)
            self.k[b, first + n - q:n] = rows[0][b, first:q]
            self.v[b, first + n - q:n] = rows[1][b, first:q]
            self.size[b, first + n - q:n] = size[b, first:q]

    def row(self, b, h, token):
        """The stored bytes of one token and head: key codes, value codes, key groups, value groups."""
        T = self.cache.page_tokens
        page = b if self.table is None else int(self.table[b, token // T])
        block = self.cache.data[page, h, token % T // 16]
        r, at, out = token % 16, 0, []
        for size in (-(-self.D // 32) * 16, -(-self.C // 32) * 16, -(-self.D // 64) * 4,
                     -(-self.C // 64) * 4):
            out.append(block[at + r * size:at + (r + 1) * size].tolist())
            at += 16 * size
        return out


def group_bytes(s, m):
    out = []
    for x, y in zip(s, m):
        out += torch.stack([x, y]).view(torch.uint8).tolist()
    return out


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("page", [0, 16, 48])
@pytest.mark.parametrize("D,C", [(1, 7), (8, 32), (33, 64), (64, 64), (80, 100), (128, 128), (130, 256)])
def test_stored_bytes(D, C, page, dtype):
    s = Store(2, 40, 3, D, C, page, seed=D)
    k, v = points((2, 21, 3, D), dtype, D, scale=3.0), points((2, 21, 3, C), dtype, D + 1)
    before = s.cache.data.clone()
    s.write(k, v, ql=[21, 5], kl=[37, 5])
    kq, vq = quantise(k.cpu()), quantise(v.cpu())
    touched = torch.zeros_like(before, dtype=torch.bool)
    for b, q, n in ((0, 21, 37), (1, 5, 5)):
        for m in range(q):
            for h in range(3):
                got = s.row(b, h, m + n - q)
                assert got[0] == row_bytes(kq[0][b, m, h].tolist(), True)
                assert got[1] == row_bytes(vq[0][b, m, h].tolist(), False)
                assert got[2] == group_bytes(kq[1][b, m, h], kq[2][b, m, h])
                assert got[3] == group_bytes(vq[1][b, m, h], vq[2][b, m, h])
    # Nothing else changed: write the old rows' places back and compare.
    T = s.cache.page_tokens
    sizes = (-(-D // 32) * 16, -(-C // 32) * 16, -(-D // 64) * 4, -(-C // 64) * 4)
    for b, q, n in ((0, 21, 37), (1, 5, 5)):
        for token in range(n - q, n):
            page_at = b if s.table is None else int(s.table[b, token // T])
            at = 0
            for size in sizes:
                row = at + token % 16 * size
                touched[page_at, :, token % T // 16, row:row + size] = True
                at += 16 * size
    assert torch.equal(s.cache.data[~touched], before[~touched])


def check_read(s, M, dtype, ql=None, kl=None):
    import paper_2609_04910_gb300 as gs
    k, v = gs.gauss_sum_cache_read(s.cache, M, DT[dtype], q_lengths=ints(ql), k_lengths=ints(kl),
                                   page_table=s.table, B=s.B)
    u = UNIT[DT[dtype]]
    for got, want in ((k, s.k), (v, s.v)):
        assert got.dtype == DT[dtype]
        full = torch.zeros(got.shape, dtype=torch.float64, device="cuda")
        for b, (q, n) in enumerate(zip(lengths_of(ql, M, s.B), lengths_of(kl, s.N, s.B))):
            first = max(0, q - n)
            full[b, first:q] = want[b, first + n - q:n]
        # (float32 holds m + s code to 2^-24; 2^-25: half the least fp16 number.)
        bound = full.abs() * (u + 2.0 ** -24) * 1.01 + (2.0 ** -25 if dtype == "fp16" else 0)
        assert bool(((got.double() - full).abs() <= bound).all())


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("layout", ["bmhd", "bhmd", "wide", "odd"])
@pytest.mark.parametrize("D,C", [(1, 1), (20, 36), (32, 32), (64, 128), (96, 80), (128, 128), (256, 200)])
def test_written_rows_come_back(D, C, layout, dtype):
    for page, Hk in ((0, 2), (32, 5), (16, 1)):
        s = Store(3, 70, Hk, D, C, page, seed=C)
        M = 61
        k, v = points((3, M, Hk, D), dtype, 5, layout), points((3, M, Hk, C), dtype, 6, layout, 100.0)
        ql, kl = [61, 0, 33], [64, 9, 33]
        spoil(k, ints(ql)), spoil(v, ints(ql))
        s.write(k, v, ql, kl)
        check_read(s, M, dtype, ql, kl)
        check_read(s, 1, dtype, None, [64, 0, 33])


@pytest.mark.parametrize("Hk", [1, 2, 7, 300])
@pytest.mark.parametrize("M", [1, 3, 64, 500])
def test_sizes_of_writes(M, Hk):
    s = Store(2, 512, Hk, 64, 64, 64)
    k, v = points((2, M, Hk, 64), "bf16", M), points((2, M, Hk, 64), "bf16", M + 1)
    s.write(k, v, None, [M, 510])
    check_read(s, M, "bf16", None, [M, 510])


def test_tokens_before_the_first_have_no_place():
    s = Store(2, 64, 2, 64, 64, 16)
    k, v = points((2, 30, 2, 64), "fp16", 1), points((2, 30, 2, 64), "fp16", 2)
    before = s.cache.data.clone()
    s.write(k, v, [30, 30], [10, 0])
    check_read(s, 30, "fp16", [30, 30], [10, 0])
    for page in s.table[1].tolist():
        assert torch.equal(s.cache.data[page], before[page])


def test_lengths_are_clamped():
    s = Store(2, 64, 2, 32, 32)
    k, v = points((2, 70, 2, 32), "fp16", 1), points((2, 70, 2, 32), "fp16", 2)
    s.write(k, v, [999, -5], [9999, 64])
    check_read(s, 70, "fp16", [999, -5], [9999, -3])


def special(dtype):
    """Rows of 128 channels with groups where the quantiser could go wrong."""
    big = torch.finfo(DT[dtype]).max
    tiny = torch.finfo(DT[dtype]).tiny
    rows = torch.zeros(12, 128)
    rows[0] = 3.25                                          # constant
    rows[1] = torch.arange(128) % 16 - 7.5                  # ties with zeros between
    rows[1, 3] = rows[1, 70] = 0.0
    rows[2, 5] = float("nan")
    rows[3, 100] = float("inf")
    rows[4, 0], rows[4, 1] = big, -big                      # the span may overflow
    rows[5] = torch.linspace(0, tiny, 128)                  # steps near the least normal number
    rows[6] = 1000 + torch.arange(128) % 7 * 0.25           # far from zero
    rows[7, 9] = -float("inf")
    rows[8] = torch.arange(128) * (big / 200)
    rows[9] = -rows[8]
    rows[10] = torch.linspace(-1, 1, 128) ** 9
    rows[11, 64:] = torch.linspace(-3e-5, 2e-5, 64)
    return rows.to(DT[dtype]).view(1, 12, 1, 128).cuda()


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
def test_special_groups(dtype):
    import paper_2609_04910_gb300 as gs
    x = special(dtype)
    s = Store(1, 16, 1, 128, 128)
    gs.gauss_sum_cache_write(s.cache, x, x, k_lengths=ints([12]))
    codes, step, low = quantise(x.cpu())
    for m in range(12):
        got = s.row(0, 0, m)
        assert got[0] == row_bytes(codes[0, m, 0].tolist(), True), m
        assert got[1] == row_bytes(codes[0, m, 0].tolist(), False), m
        # (Any NaN will do for a group that is not finite.)
        for have in (got[2], got[3]):
            pair = torch.tensor(have, dtype=torch.uint8).view(torch.bfloat16).view(-1, 2)
            want = torch.stack([step[0, m, 0], low[0, m, 0]], -1)
            assert torch.equal(pair.isnan(), want.isnan()), m
            assert torch.equal(pair.nan_to_num(), want.nan_to_num()), m
    k, v = gs.gauss_sum_cache_read(s.cache, 12, torch.float32, k_lengths=ints([12]))
    want = values(codes, step, low).cuda()
    for got in (k, v):
        assert torch.equal(got.isnan(), want.isnan())
        err = (got.double() - want).nan_to_num().abs()
        assert bool((err <= want.nan_to_num().abs() * 2.0 ** -23).all())


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
def test_codes_next_to_a_border(dtype):
    """Rows whose quotients lie on and around halves."""
    import paper_2609_04910_gb300 as gs
    gen = torch.Generator().manual_seed(2)
    x = torch.randint(-30, 31, (1, 400, 2, 64), generator=gen).float() / 2     # halves: many exact ties
    x[..., 0], x[..., 1] = -7.5, 7.5
    x = x.clamp(-7.5, 7.5)
    if dtype == "fp32":
        x[0, 200:] = torch.nextafter(x[0, 200:], torch.tensor(float("inf")))
    x = x.to(DT[dtype])
    s = Store(1, 400, 2, 64, 64)
    gs.gauss_sum_cache_write(s.cache, x.cuda(), x.cuda(), k_lengths=ints([400]))
    want = values(*quantise(x))
    k, v = gs.gauss_sum_cache_read(s.cache, 400, torch.float32, k_lengths=ints([400]))
    assert torch.equal(k.cpu().double(), want) and torch.equal(v.cpu().double(), want)


# ---------------------------------------------------------------- attention

def filled(B, N, Hk, D, C, page, seed, kl=None, scale=1.0):
    """A Store whose problems hold their k_lengths tokens (NaN groups everywhere else)."""
    s = Store(B, N, Hk, D, C, page, seed, fill=0xFF)
    k = points((B, s.N, Hk, D), "fp32", seed + 1, scale=scale)
    v = points((B, s.N, Hk, C), "fp32", seed + 2)
    v += points((B, 1, Hk, C), "fp32", seed + 3)            # values that are not centred
    for b, n in enumerate(lengths_of(kl, s.N, B)):
        if n:
            at = None if s.table is None else s.table
            import paper_2609_04910_gb300 as gs
            cache = s.cache if at is not None else gs.AttentionCache(s.cache.data[b:b + 1], D, C)
            gs.gauss_sum_cache_write(cache, k[b:b + 1, :n], v[b:b + 1, :n], k_lengths=ints([n]),
                                     page_table=None if at is None else at[b:b + 1])
    kq, vq = quantise(k), quantise(v)
    s.k, s.v = values(*kq), values(*vq)
    s.k_size = values(kq[0], kq[1], kq[2].abs())
    s.size = (vq[2].double().abs() + 15 * vq[1].double())[..., torch.arange(C, device="cuda") // 64]
    return s


def path_of(M, H, Hk, D, C, dtype):
    """Which kernels take a call."""
    words = -(-D // 32), -(-C // 32)
    if (M * (H // Hk) <= 16 or dtype == "fp32") and words[0] == words[1] <= 4:
        return "few"
    return "many" if dtype != "fp32" and max(words) <= 4 else "rows"


def attend(B, M, N, H, Hk, D, C, dtype, causal=True, ql=None, kl=None, page=0, layout="bmhd", seed=0,
           scale=1.0, tau=None):
    import paper_2609_04910_gb300 as gs
    tau = 1 / math.sqrt(D) if tau is None else tau
    kl = [N] * B if kl is None else kl
    s = filled(B, N, Hk, D, C, page, seed, kl, scale)
    q = points((B, M, H, D), dtype, seed + 4, layout)
    want = attention64(q, s.k, s.v, s.k_size, s.size, tau, causal, ints(ql), ints(kl),
                       path=path_of(M, H, Hk, D, C, dtype))
    spoil(q, ints(ql))
    out, lse = gs.gauss_sum_attention_cached(q, s.cache, tau, causal=causal, q_lengths=ints(ql),
                                             k_lengths=ints(kl), page_table=s.table)
    gs.gauss_sum_device_status()
    assert out.dtype == q.dtype and lse.dtype == torch.float32
    worst = {"out": within(out, want["out"]), "lse": within(lse, want["lse"])}
    assert all(w <= 1 for w in worst.values()), worst
    return worst


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("B,M,N", [(1, 1, 1), (2, 1, 15), (1, 1, 16), (3, 1, 17), (1, 2, 100), (2, 1, 700),
                                   (1, 4, 4100), (2, 9, 300), (1, 40, 260), (2, 130, 130), (1, 300, 515)])
def test_sizes(B, M, N, dtype, causal):
    attend(B, M, N, 4, 2, 64, 64, dtype, causal, page=32 if N % 2 else 0, seed=M + N)


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("M", [1, 6, 70])
@pytest.mark.parametrize("D,C", [(1, 1), (8, 24), (20, 36), (32, 32), (33, 33), (64, 128), (64, 64), (80, 80),
                                 (96, 96), (100, 128), (128, 64), (128, 128), (130, 16), (256, 256)])
def test_widths(D, C, M, dtype):
    attend(2, M, 150, 4, 2, D, C, dtype, True, ql=[M, (M + 1) // 2], kl=[150, 131], page=16, seed=D + C)


@pytest.mark.parametrize("H,Hk", [(1, 1), (5, 5), (7, 1), (12, 4), (40, 8), (32, 2), (64, 1)])
@pytest.mark.parametrize("M", [1, 2, 5, 17])
def test_head_groups(H, Hk, M):
    attend(2, M, 333, H, Hk, 64, 64, "bf16", True, kl=[333, 290], seed=H + M, page=48)


@pytest.mark.parametrize("layout", ["bmhd", "bhmd", "wide", "odd"])
@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("M", [1, 150])
def test_layouts(layout, dtype, M):
    attend(2, M, 260, 4, 2, 64, 64, dtype, True, kl=[260, 199], layout=layout, seed=5)


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("M", [3, 40, 200])
@pytest.mark.parametrize("ql,kl", [([0, 5, 200], [300, 0, 1]), ([200, 130, 1], [1, 129, 300]),
                                   ([200, 200, 200], [128, 127, 0]), ([999, -4, 200], [300, 300, 9999])])
def test_lengths_leave_rows_empty(ql, kl, M, causal, dtype):
    attend(3, M, 304, 4, 2, 64, 64, dtype, causal, ql=ql, kl=kl, page=16, seed=11)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("scale", [0.01, 5.0, 40.0])
def test_score_ranges(scale, dtype):
    """From nearly equal weights to one key that takes all."""
    for M in (1, 3, 30):
        attend(2, M, 500, 8, 2, 128, 128, dtype, True, kl=[500, 37], page=32, seed=M, scale=scale)


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("M,H", [(1, 8), (1, 64), (40, 8), (200, 8)])
@pytest.mark.parametrize("B", [1, 3, 300])
def test_many_uneven_problems(B, M, H, dtype):
    """Lengths from none on, more problems than a block has threads."""
    if B == 300 and M > 1:
        pytest.skip("as B = 3")
    gen = torch.Generator().manual_seed(B + M)
    kl = torch.randint(0, 700, (B,), generator=gen).tolist()
    ql = [min(M, n + 2) if i % 3 else M for i, n in enumerate(kl)]
    if B >= 3:
        kl[1], kl[2] = 0, 704
    attend(B, M, 704, H, 2, 64, 64, dtype, True, ql=ql, kl=kl, page=32, seed=M)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("M", [1, 3, 20, 80])
def test_long_sequences(M, dtype):
    """Many blocks to a problem, one of them alone and beside short ones."""
    attend(1, M, 20000, 4, 2, 128, 128, dtype, True, page=64, seed=M)
    attend(3, M, 9000, 8, 2, 64, 64, dtype, True, kl=[9000, 1, 77], page=16, seed=M)


@pytest.mark.parametrize("N", [1500, 120000])
def test_fp32_sums_of_many_tokens(N):
    """Centred values, whose weighted mean is far smaller than they are.

    An error of a score changes a probability by as much, |error| <= eS = 2^-21 (size + 1)
    (attention_cache_forms); the changes of independent tokens add up like the tokens' values
    do, so that the 2-norm of the result is off by at most eS of its own, up to a factor of
    two for the values' own roundings (2^-21 |v| in every sum of 32 tokens)."""
    import paper_2609_04910_gb300 as gs
    s = Store(1, N, 2, 32, 32, 256, seed=N)
    k, v = points((1, s.N, 2, 32), "fp32", 1), points((1, s.N, 2, 32), "fp32", 2)
    s.write(k, v)
    size = quantise(k)
    k_size = values(size[0], size[1], size[2].abs())
    q = points((1, 2, 4, 32), "fp32", 3)
    tau = 32 ** -0.5
    want = attention64(q, s.k, s.v, k_size, s.size, tau, path="few")["out"][0]
    out, _ = gs.gauss_sum_attention_cached(q, s.cache, tau, page_table=s.table)
    sizes = tau * torch.einsum("bmhd,bnhd->bmhn", q.double().abs(), k_size.repeat_interleave(2, 2)).amax()
    rel = float((out.double() - want).norm() / want.norm())
    assert rel <= 2 * 2.0 ** -21 * (float(sizes) + 1), rel


@pytest.mark.parametrize("v_scale", [1e-6, 1e-3, 3e3])
@pytest.mark.parametrize("M", [1, 40, 200])
def test_value_sizes(v_scale, M):
    """Values far from one, and tokens 300 times larger than the others, in bf16."""
    import paper_2609_04910_gb300 as gs
    B, N, H, Hk, D = 2, 300, 4, 2, 64
    s = Store(B, N, Hk, D, D, 32, seed=1)
    k, v = points((B, s.N, Hk, D), "fp32", 2), points((B, s.N, Hk, D), "fp32", 3) * v_scale
    k[:, 5] *= 30
    v[:, 170] *= 300
    s.write(k, v)
    size = quantise(k)
    k_size = values(size[0], size[1], size[2].abs())
    q = points((B, M, H, D), "bf16", 4)
    want = attention64(q, s.k, s.v, k_size, s.size, 0.125, True, path=path_of(M, H, Hk, D, D, "bf16"))
    out, lse = gs.gauss_sum_attention_cached(q, s.cache, 0.125, causal=True, page_table=s.table)
    gs.gauss_sum_device_status()
    assert within(out, want["out"]) <= 1 and within(lse, want["lse"]) <= 1


@pytest.mark.parametrize("M", [1, 7, 70, 300])
@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
def test_missing_pages(M, dtype):
    """Queries that see a token without a page are NaN, other problems are as they were."""
    import paper_2609_04910_gb300 as gs
    B, N, H, Hk, D = 3, 400, 4, 2, 64
    s = filled(B, N, Hk, D, D, 16, 1)
    q = points((B, M, H, D), dtype, 9)
    kl = ints([400, 330, 390])
    whole, lse = gs.gauss_sum_attention_cached(q, s.cache, 0.125, k_lengths=kl, page_table=s.table)
    for bad in (-1, s.cache.data.shape[0], 1 << 30, -(1 << 31)):
        table = s.table.clone()
        table[1, 20] = bad               # tokens 320 .. 335 of problem 1, 320 .. 329 of them counted
        table[2, 24] = bad               # 384 .. 399, 384 .. 389 counted
        table[0, 25:] = bad
        out, z = gs.gauss_sum_attention_cached(q, s.cache, 0.125, k_lengths=kl, page_table=table)
        assert bool(out[1:].isnan().all()) and bool(z[1:].isnan().all())
        assert torch.equal(out[0], whole[0]) and torch.equal(z[0], lse[0])
        # Past the lengths an entry is not looked at.
        out, z = gs.gauss_sum_attention_cached(q, s.cache, 0.125, k_lengths=ints([400, 320, 384]),
                                               page_table=table)
        same, zs = gs.gauss_sum_attention_cached(q, s.cache, 0.125, k_lengths=ints([400, 320, 384]),
                                                 page_table=s.table)
        assert torch.equal(out, same) and torch.equal(z, zs)
        k, v = gs.gauss_sum_cache_read(s.cache, 30, DT[dtype], k_lengths=kl, page_table=table)
        k0, v0 = gs.gauss_sum_cache_read(s.cache, 30, DT[dtype], k_lengths=kl, page_table=s.table)
        for x, y in ((k, k0), (v, v0)):
            assert torch.equal(x[0], y[0]) and torch.equal(x[1, :20], y[1, :20])
            assert bool(x[1, 20:].isnan().all()) and bool(x[2, 24:].isnan().all())
            assert torch.equal(x[2, :24], y[2, :24])
        before = s.cache.data.clone()
        gs.gauss_sum_cache_write(s.cache, k0[:, 20:].contiguous(), v0[:, 20:].contiguous(), k_lengths=kl,
                                 page_table=torch.full_like(table, bad))
        assert torch.equal(s.cache.data, before)
    gs.gauss_sum_device_status()


@pytest.mark.parametrize("M", [1, 40, 300])
def test_nan_tokens(M):
    """A token with a NaN makes the queries that see it NaN, without a mask all of its head."""
    import paper_2609_04910_gb300 as gs
    for side in "kv":
        s = Store(2, 200, 2, 64, 64, 16, seed=3)
        x = {"k": points((2, 200, 2, 64), "bf16", 1), "v": points((2, 200, 2, 64), "bf16", 2)}
        x[side][1, 150, 0, 3] = float("nan")
        s.write(x["k"], x["v"], kl=[200, 200])
        q = points((2, M, 4, 64), "bf16", 5)
        out, _ = gs.gauss_sum_attention_cached(q, s.cache, 0.125, k_lengths=ints([200, 200]), page_table=s.table)
        assert bool(out[0].isfinite().all()) and bool(out[1, :, 2:].isfinite().all())
        # (In v only the channels of the token's group.)
        assert bool(out[1, :, :2].isnan().all())


def test_offsets_past_32_bits():
    """Pages beyond 4 GiB of the pool and heads far apart, in every kernel."""
    import paper_2609_04910_gb300 as gs
    B, T, Hk, D = 2, 256, 8, 128
    page_bytes = Hk * T // 16 * 2304
    pages = (5 << 30) // page_bytes + 8
    cache = gs.attention_cache(pages, T, Hk, D)
    assert cache.data.numel() > 1 << 32
    per = 3
    far = (torch.arange(B * per, dtype=torch.int32) + pages - B * per).view(B, per).cuda()
    small = gs.attention_cache(B * per, T, Hk, D)
    near = torch.arange(B * per, dtype=torch.int32).view(B, per).cuda()
    k, v = points((B, T * per, Hk, D), "bf16", 1), points((B, T * per, Hk, D), "bf16", 2)
    kl = ints([T * per, T * per - 100])
    for c, table in ((cache, far), (small, near)):
        gs.gauss_sum_cache_write(c, k, v, k_lengths=ints([T * per] * B), page_table=table)
    assert torch.equal(cache.data[far.long()], small.data[near.long()])
    # Heads far apart: one head in the front of the pool, the other past 4 GiB.
    wide = torch.as_strided(cache.data, (1, 2, 48, 2304), (0, (1 << 32) // 2304 * 2304 + 2304 * 16, 2304, 1))
    heads = gs.AttentionCache(wide, D)
    gs.gauss_sum_cache_write(heads, k[:1, :, :2], v[:1, :, :2])
    small2 = gs.attention_cache(1, T * per, 2, D)
    gs.gauss_sum_cache_write(small2, k[:1, :, :2].contiguous(), v[:1, :, :2].contiguous())
    assert torch.equal(wide, small2.data)
    gs.gauss_sum_cache_write(cache, k, v, k_lengths=ints([T * per] * B), page_table=far)
    for M in (1, 5, 100):
        q = points((B, M, 32, D), "bf16", M)
        got = [gs.gauss_sum_attention_cached(q, c, 0.1, causal=True, k_lengths=kl, page_table=t)
               for c, t in ((cache, far), (small, near))]
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
        got = [gs.gauss_sum_attention_cached(q[:1, :, :8], c, 0.1) for c in (heads, small2)]
        assert torch.equal(got[0][0], got[1][0])
    rows = [gs.gauss_sum_cache_read(c, T, torch.float16, k_lengths=kl, page_table=t)
            for c, t in ((cache, far), (small, near))]
    assert all(torch.equal(x, y) for x, y in zip(*rows))
    gs.gauss_sum_device_status()


def test_slices_of_a_pool():
    """A cache whose pages and heads are a part of a larger array."""
    import paper_2609_04910_gb300 as gs
    whole = gs.attention_cache(10, 64, 6, 64, 32)
    part = gs.AttentionCache(whole.data[2:8:2, 1:5], 64, 32)
    plain = gs.attention_cache(3, 64, 4, 64, 32)
    k, v = points((3, 64, 4, 64), "fp16", 1), points((3, 64, 4, 32), "fp16", 2)
    for c in (part, plain):
        gs.gauss_sum_cache_write(c, k, v)
    assert torch.equal(part.data, plain.data)
    whole.data[2:8:2, 1:5] = 0
    assert not bool(whole.data.any())
    gs.gauss_sum_cache_write(part, k, v)
    for M in (1, 33, 300):
        q = points((3, M, 8, 64), "fp16", M)
        got = [gs.gauss_sum_attention_cached(q, c, 0.125, causal=True) for c in (part, plain)]
        assert torch.equal(got[0][0], got[1][0])


@pytest.mark.parametrize("M", [1, 3, 60, 270])
def test_results_repeat(M):
    """The same bits from call to call, also on two streams at once."""
    import paper_2609_04910_gb300 as gs
    s = filled(4, 3000, 4, 128, 128, 64, 5, kl=[3000, 2999, 17, 1500])
    kl = ints([3000, 2999, 17, 1500])
    q = points((4, M, 16, 128), "bf16", 6)
    args = dict(causal=True, k_lengths=kl, page_table=s.table)
    first = gs.gauss_sum_attention_cached(q, s.cache, 0.09, **args)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for i in range(12):
        got.append(gs.gauss_sum_attention_cached(q, s.cache, 0.09, stream=streams[i % 2], **args))
    torch.cuda.synchronize()
    for out, lse in got:
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
    gs.gauss_sum_device_status()


def test_captured_steps_follow_the_lengths():
    """One captured step (write the new token, attend) replayed as the sequence grows, beside another
    graph of the same cache."""
    import paper_2609_04910_gb300 as gs
    B, H, Hk, D, T = 3, 8, 2, 64, 32
    s = Store(B, 320, Hk, D, D, T, fill=0xFF)
    k, v = points((B, 300, Hk, D), "bf16", 1), points((B, 300, Hk, D), "bf16", 2)
    q = points((B, 300, H, D), "bf16", 3)
    start = 250
    gs.gauss_sum_cache_write(s.cache, k[:, :start], v[:, :start], k_lengths=ints([start] * B), page_table=s.table)
    lengths = ints([start] * B)
    kn, vn, qn = (torch.empty_like(x[:, :1]) for x in (k, v, q))
    side = torch.cuda.Stream()

    def step(out, lse):
        lengths.add_(1)
        gs.gauss_sum_cache_write(s.cache, kn, vn, k_lengths=lengths, page_table=s.table)
        gs.gauss_sum_attention_cached(qn, s.cache, 0.125, causal=True, k_lengths=lengths, page_table=s.table,
                                      out=out, lse=lse)

    out, lse = torch.empty_like(qn), torch.empty(B, H, 1, device="cuda")
    out2 = torch.empty(B, 40, H, D, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    with torch.cuda.graph(graphs[0], stream=side):
        step(out, lse)
    with torch.cuda.graph(graphs[1], stream=side):
        gs.gauss_sum_attention_cached(q[:, 100:140], s.cache, 0.125, k_lengths=lengths, page_table=s.table, out=out2)
    kept = []
    for t in range(start, 300):
        for x, y in ((kn, k), (vn, v), (qn, q)):
            x.copy_(y[:, t:t + 1])
        for g in graphs:
            g.replay()
        kept.append(out.clone())
    assert lengths.tolist() == [300] * B
    whole = Store(B, 320, Hk, D, D, T)
    whole.write(k, v, kl=[300] * B)
    codes = quantise(torch.cat([k, k[:, :20]], 1))
    k_size = values(codes[0], codes[1], codes[2].abs())
    want = attention64(q[:, start:], whole.k, whole.v, k_size, whole.size, 0.125, True, k_lengths=ints([300] * B),
                       path="few")
    assert within(torch.cat(kept, 1), want["out"]) <= 1
    want = attention64(q[:, 100:140], whole.k, whole.v, k_size, whole.size, 0.125, k_lengths=ints([300] * B),
                       path="many")
    assert within(out2, want["out"]) <= 1
    gs.gauss_sum_device_status()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_a_run_of_rotary_writes_and_attention(dtype):
    """A prompt, then tokens one by one and a few at a time, as a network would use the operators: the
    results are those of attention on the rows that the cache holds."""
    import paper_2609_04910_gb300 as gs
    B, H, Hk, D, T = 2, 8, 2, 128, 64
    prompt, steps = [150, 90], [1, 1, 1, 4, 1, 9, 1, 40, 1]
    total = max(prompt) + sum(steps)
    freqs, scale = gs.rotary_frequencies(64, scaling="yarn", factor=4.0, original_length=1024)
    q, k, v = (points((B, total, h, D), dtype, i) for i, h in enumerate((H, Hk, Hk)))
    s = Store(B, total, Hk, D, D, T, fill=0xFF)
    held = ints([0] * B)
    done = [0, 0]
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


@pytest.mark.parametrize("layout", ["bmhd", "bhmd", "wide", "odd"])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("M,H,Hk,D,C", [(40, 40, 2, 64, 64), (90, 28, 4, 128, 128), (33, 17, 1, 100, 36),
                                        (530, 3, 3, 33, 128), (300, 2, 1, 20, 8)])
def test_rows_read_back_first(M, H, Hk, D, C, dtype, layout):
    """More rows than the tiles take: heads that are no multiple of a warp's, odd widths and strides."""
    attend(2, M, 700, H, Hk, D, C, dtype, True, ql=[M, M - 7], kl=[700, 555], page=48, layout=layout, seed=M)


@pytest.mark.parametrize("ql,kl", [([0, 300, 300], [300, 0, 1]), ([300, 130, 1], [1, 129, 300]),
                                   ([999, -4, 300], [304, 300, 9999])])
def test_rows_read_back_of_uneven_problems(ql, kl):
    attend(3, 300, 304, 4, 2, 64, 64, "bf16", True, ql=ql, kl=kl, page=16, seed=7)


@pytest.mark.parametrize("B,Hk,columns", [(2, 4, 512), (1, 4, 256), (5, 1, 256)])
def test_more_room_than_one_workspace(B, Hk, columns):
    """Tables of so many columns that problems, or their heads, are read back in several groups."""
    import paper_2609_04910_gb300 as gs
    M, H, D, page = 300, 2 * Hk, 128, 4096
    kl = [1000 + 77 * b for b in range(B)]
    s = filled(B, 4096, Hk, D, D, page, 3, kl)
    table = torch.full((B, columns), -1, dtype=torch.int32, device="cuda")
    table[:, 0] = s.table[:, 0]
    q = points((B, M, H, D), "bf16", 4)
    want = attention64(q, s.k, s.v, s.k_size, s.size, 0.09, True, k_lengths=ints(kl), path="many")
    out, lse = gs.gauss_sum_attention_cached(q, s.cache, 0.09, causal=True, k_lengths=ints(kl), page_table=table)
    assert within(out, want["out"]) <= 1 and within(lse, want["lse"]) <= 1
    gs.gauss_sum_device_status()


def test_more_room_than_one_workspace_without_a_table():
    import paper_2609_04910_gb300 as gs
    B, M, H, D, n = 5, 530, 1, 128, 900
    cache = gs.attention_cache(B, 1 << 20, 1, D)
    s = filled(B, n, 1, D, D, 0, 5, [n] * B)
    k, v = (x[:, :n].float() for x in (s.k, s.v))
    gs.gauss_sum_cache_write(cache, k, v, k_lengths=ints([n] * B))
    small = gs.attention_cache(B, 912, 1, D)
    gs.gauss_sum_cache_write(small, k, v, k_lengths=ints([n] * B))
    assert torch.equal(cache.data[:, :, :57], small.data)
    k, v = quantise(k), quantise(v)
    size = (v[2].double().abs() + 15 * v[1].double())[..., torch.arange(D, device="cuda") // 64]
    q = points((B, M, H, D), "fp16", 4)
    want = attention64(q, values(*k), values(*v), values(k[0], k[1], k[2].abs()), size, 0.09, True,
                       k_lengths=ints([n] * B), path="many")
    out, lse = gs.gauss_sum_attention_cached(q, cache, 0.09, causal=True, k_lengths=ints([n] * B))
    assert within(out, want["out"]) <= 1 and within(lse, want["lse"]) <= 1


@pytest.mark.parametrize("M", [1, 3, 60, 300])
def test_problems_that_share_pages(M):
    """A prefix that two problems read from the same pages, and a table whose rows are one row."""
    import paper_2609_04910_gb300 as gs
    s = filled(2, 640, 2, 64, 64, 64, 9)
    table = s.table.clone()
    table[1, :5] = table[0, :5]
    kl = ints([640, 500])
    q = points((2, M, 8, 64), "bf16", M)
    k, v = s.k.clone(), s.v.clone()
    for x, y in ((k, s.k), (v, s.v)):
        x[1, :320] = y[0, :320]
    k_size, size = s.k_size.clone(), s.size.clone()
    k_size[1, :320], size[1, :320] = s.k_size[0, :320], s.size[0, :320]
    path = path_of(M, 8, 2, 64, 64, "bf16")
    want = attention64(q, k, v, k_size, size, 0.125, True, k_lengths=kl, path=path)
    got = gs.gauss_sum_attention_cached(q, s.cache, 0.125, causal=True, k_lengths=kl, page_table=table)
    assert within(got[0], want["out"]) <= 1 and within(got[1], want["lse"]) <= 1
    got = gs.gauss_sum_attention_cached(q, s.cache, 0.125, page_table=s.table[:1].expand(2, -1))
    one = [x[:1].expand(2, -1, -1, -1) for x in (s.k, s.v, s.k_size, s.size)]
    want = attention64(q, *one, 0.125, False, path=path)
    assert within(got[0], want["out"]) <= 1 and within(got[1], want["lse"]) <= 1


def test_captured_rows_read_back():
    """Calls whose rows are read back, in two graphs of one cache, replayed as the lengths change."""
    import paper_2609_04910_gb300 as gs
    B, M, H, Hk, D = 2, 300, 4, 2, 64
    s = filled(B, 900, Hk, D, D, 64, 3)
    lengths = ints([900, 850])
    q = [points((B, M, H, D), "fp16", i) for i in range(2)]
    out = [torch.empty_like(x) for x in q]
    lse = [torch.empty(B, H, M, device="cuda") for _ in q]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in q]
    for g, x, o, l in zip(graphs, q, out, lse):
        with torch.cuda.graph(g, stream=side):
            gs.gauss_sum_attention_cached(x, s.cache, 0.125, causal=True, k_lengths=lengths, page_table=s.table,
                                          out=o, lse=l)
    for kl in ([900, 850], [17, 500], [0, 901]):
        lengths.copy_(ints(kl))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for x, o, l in zip(q, out, lse):
            want = attention64(x, s.k, s.v, s.k_size, s.size, 0.125, True, k_lengths=ints(kl), path="many")
            assert within(o, want["out"]) <= 1 and within(l, want["lse"]) <= 1, kl
    gs.gauss_sum_device_status()


def test_rows_read_back_past_32_bits():
    """Pages beyond 4 GiB of the pool: the scan of sizes and the rows read back."""
    import paper_2609_04910_gb300 as gs
    B, T, Hk, D, per = 2, 256, 8, 128, 3
    pages = (5 << 30) // (Hk * T // 16 * 2304) + 8
    far = (torch.arange(B * per, dtype=torch.int32) + pages - B * per).view(B, per).cuda()
    near = torch.arange(B * per, dtype=torch.int32).view(B, per).cuda()
    k, v = points((B, T * per, Hk, D), "bf16", 1), points((B, T * per, Hk, D), "bf16", 2)
    q = points((B, 200, 32, D), "bf16", 3)
    got = []
    for table, n in ((far, pages), (near, B * per)):
        cache = gs.attention_cache(n, T, Hk, D)
        gs.gauss_sum_cache_write(cache, k, v, page_table=table)
        got.append(gs.gauss_sum_attention_cached(q, cache, 0.1, causal=True, page_table=table))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    gs.gauss_sum_device_status()


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("M", [30, 70, 300])
@pytest.mark.parametrize("D,C", [(1, 1), (8, 24), (20, 36), (32, 32), (33, 33), (64, 128), (64, 64), (80, 80),
                                 (96, 96), (100, 128), (128, 64), (128, 128)])
def test_widths_of_longer_caches(D, C, M, dtype):
    """Of the kernels that round keys, which short caches do not take."""
    attend(2, M, 450, 4, 2, D, C, dtype, True, ql=[M, (M + 1) // 2], kl=[450, 333], page=16, seed=D + C)


@pytest.mark.parametrize("M,H", [(17, 4), (130, 8), (256, 16)])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("N", [17, 100, 256])
def test_short_caches_are_exact(N, M, H, dtype):
    """Few keys do not average a key's rounding away: their scores, and so lse, are those of
    32-bit arithmetic (2^-21 of the sizes of their terms and 2^-22 of lse) at every number of rows."""
    import paper_2609_04910_gb300 as gs
    s = filled(2, N, 2, 64, 64, 16, N, [N, (N + 1) // 2])
    q = points((2, M, H, 64), dtype, M)
    kl = ints([N, (N + 1) // 2])
    out, lse = gs.gauss_sum_attention_cached(q, s.cache, 0.125, causal=True, k_lengths=kl, page_table=s.table)
    want = attention64(q, s.k, s.v, s.k_size, s.size, 0.125, True, k_lengths=kl, path="few")
    assert within(out, want["out"]) <= 1 and within(lse, want["lse"]) <= 1


@pytest.mark.parametrize("q_exp,k_exp,v_exp", [(0, 0, 90), (0, 0, -90), (100, -100, 0), (-90, 90, -60)])
@pytest.mark.parametrize("M", [1, 40, 300])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_far_exponents(q_exp, k_exp, v_exp, M, dtype):
    """Queries, keys and values far from one (times powers of two, so that the bounds scale with them)."""
    import paper_2609_04910_gb300 as gs
    B, N, H, Hk, D = 2, 300, 4, 2, 64
    s = Store(B, N, Hk, D, D, 32, seed=1)
    k, v = (points((B, s.N, Hk, D), "fp32", i) * 2.0 ** e for i, e in ((2, k_exp), (3, v_exp)))
    v[:, 170] *= 300
    s.write(k, v)
    size = quantise(k)
    k_size = values(size[0], size[1], size[2].abs())
    q = points((B, M, H, D), dtype, 4) * 2.0 ** q_exp
    want = attention64(q, s.k, s.v, k_size, s.size, 0.125, True, path=path_of(M, H, Hk, D, D, dtype))
    out, lse = gs.gauss_sum_attention_cached(q, s.cache, 0.125, causal=True, page_table=s.table)
    gs.gauss_sum_device_status()
    assert within(out, want["out"]) <= 1 and within(lse, want["lse"]) <= 1


def test_allocation_failure_is_reported():
    import paper_2609_04910_gb300 as gs
    from paper_2609_04910_gb300 import _binding
    s = filled(1, 4000, 2, 64, 64, 64, 5)
    for M in (1, 40, 300):
        q = points((1, M, 4, 64), "bf16", 6)
        want = gs.gauss_sum_attention_cached(q, s.cache, 0.125, page_table=s.table)
        _binding.testing_fail_allocations(True)
        try:
            with pytest.raises(gs.GaussSumError) as e:
                gs.gauss_sum_attention_cached(q, s.cache, 0.125, page_table=s.table)
        finally:
            _binding.testing_fail_allocations(False)
        assert e.value.status == 3
        again = gs.gauss_sum_attention_cached(q, s.cache, 0.125, page_table=s.table)
        assert torch.equal(again[0], want[0])


def test_binding_checks():
    import paper_2609_04910_gb300 as gs
    c = gs.attention_cache(4, 32, 2, 64, 32)
    k, v = points((2, 3, 2, 64), "bf16", 1), points((2, 3, 2, 32), "bf16", 2)
    q = points((2, 3, 4, 64), "bf16", 3)
    table = torch.zeros(2, 2, dtype=torch.int32, device="cuda")
    for bad in (dict(page_table=table.long()), dict(page_table=table[:1]), dict(page_table=table[0]),
                dict(page_table=table.cpu()), dict(k_lengths=ints([1])), dict(q_lengths=ints([1, 2]).long()),
                dict(page_table=torch.zeros(2, 4, dtype=torch.int32, device="cuda")[:, ::2])):
        with pytest.raises(ValueError):
            gs.gauss_sum_cache_write(c, k, v, **bad)
        with pytest.raises(ValueError):
            gs.gauss_sum_cache_read(c, 3, torch.bfloat16, B=2, **bad)
        with pytest.raises(ValueError):
            gs.gauss_sum_attention_cached(q, c, 0.125, **bad)
    with pytest.raises(ValueError):
        gs.gauss_sum_cache_write(c, k, v.half())
    with pytest.raises(ValueError):
        gs.gauss_sum_cache_write(c, k[:, :, :1], v)
    with pytest.raises(ValueError):
        gs.gauss_sum_attention_cached(q[..., :32], c, 0.125)
    with pytest.raises(TypeError):
        gs.gauss_sum_cache_read(c, 3, torch.float64)
    with pytest.raises(gs.GaussSumError):
        gs.gauss_sum_attention_cached(q[:, :, :3], c, 0.125)
    assert gs.gauss_sum_cache_read(c, 3, torch.float32, want=("v",))[0] is None


def test_empty_calls():
    import paper_2609_04910_gb300 as gs
    c = gs.attention_cache(2, 32, 2, 64)
    none = torch.empty(2, 0, dtype=torch.int32, device="cuda")
    for M in (1, 40, 300):
        q = points((2, M, 4, 64), "bf16", 3)
        out, lse = gs.gauss_sum_attention_cached(q, c, 0.125, page_table=none)
        assert not bool(out.any()) and bool((lse == -float("inf")).all())
        out, lse = gs.gauss_sum_attention_cached(q, c, 0.125, k_lengths=ints([0, 0]))
        assert not bool(out.any()) and bool((lse == -float("inf")).all())
    k, v = gs.gauss_sum_cache_read(c, 5, torch.float16, page_table=none)
    assert k.shape == (2, 5, 2, 64) and not bool(k.any()) and not bool(v.any())
    gs.gauss_sum_cache_write(c, k, v, page_table=none)
    assert gs.gauss_sum_attention_cached(q[:0], c, 0.125, k_lengths=ints([]))[0].shape == (0, 300, 4, 64)
    gs.gauss_sum_device_status()
