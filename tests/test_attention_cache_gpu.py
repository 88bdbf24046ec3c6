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
    if M * (H // Hk) <= 16 and words[0] == words[1] <= 4:
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
