"""Host logic of the 4-bit cache: exported symbols, refusals (all before any
CUDA work), and the layout that the header states."""
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PTR = 4096   # an aligned address that is never dereferenced
BLOCK = 16 * (32 + 16 + 4 + 4)      # D = 64, C = 32


@pytest.fixture(scope="module")
def lib():
    from paper_2609_04910_gb300._binding import load_library
    from paper_2609_04910_gb300.build import build_library
    build_library()
    return load_library()


def test_every_declared_symbol_is_exported(lib):
    from paper_2609_04910_gb300._binding import CACHE_EXPORTS
    src = open(os.path.join(ROOT, "include", "gauss_sum", "attention_cache.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    declared = sorted(set(re.findall(r"\b(gauss_sum\w*)\s*\(", src)))
    assert declared == sorted(CACHE_EXPORTS)
    for name in declared:
        assert hasattr(lib, name)


def cache(**kw):
    from paper_2609_04910_gb300._binding import _CACHE
    a = dict(data=PTR, sp=2 * 4 * BLOCK, sh=4 * BLOCK, pages=8, tokens=64, heads=2, D=64, C=32, table=PTR,
             per=3, st=3)
    a.update(kw)
    return _CACHE.pack(*a.values())


def rows(**kw):
    from paper_2609_04910_gb300._binding import _CACHE_ROWS
    a = dict(dtype=1, B=2, M=4, ql=0, kl=0, k=(PTR, 512, 128, 64), v=(PTR, 256, 64, 32))
    a.update(kw)
    return _CACHE_ROWS.pack(*(a[x] for x in ("dtype", "B", "M", "ql", "kl")), *a["k"], *a["v"])


def attention(**kw):
    from paper_2609_04910_gb300._binding import _CACHED_ATTENTION
    a = dict(dtype=1, B=2, M=4, H=4, tau=1.0, causal=1, ql=0, kl=0, q=(PTR, 1024, 256, 64),
             out=(PTR, 512, 128, 32), lse=PTR)
    a.update(kw)
    return _CACHED_ATTENTION.pack(*(a[x] for x in ("dtype", "B", "M", "H", "tau", "causal", "ql", "kl")),
                                  *a["q"], *a["out"], a["lse"])


BAD_CACHE = [(dict(pages=-1), 1), (dict(heads=-1), 1), (dict(D=0), 1), (dict(C=0), 1), (dict(tokens=0), 1),
             (dict(tokens=24), 1), (dict(tokens=-16), 1), (dict(per=-1), 1), (dict(st=-1), 1), (dict(D=257), 2),
             (dict(C=257), 2), (dict(pages=1 << 31), 2), (dict(tokens=1 << 31), 2), (dict(per=1 << 26), 2),
             (dict(table=0, pages=1), 1), (dict(table=PTR + 2), 1), (dict(data=0), 1), (dict(data=PTR + 8), 1),
             (dict(sp=2 * 4 * BLOCK + 8), 1), (dict(sh=4 * BLOCK + 4), 1), (dict(sp=-4096), 1),
             (dict(sh=-4096), 1), (dict(sp=1 << 61), 1), (dict(st=1 << 60), 1)]


@pytest.mark.parametrize("case,status", BAD_CACHE + [(dict(heads=65536), 2)])
def test_refused_caches(lib, case, status):
    n = lib.gauss_sum_kernel_launches()
    assert lib.gauss_sum_cache_write(cache(**case), rows(), None) == status
    assert lib.gauss_sum_last_error()
    assert lib.gauss_sum_cache_read(cache(**case), rows(), None) == status
    if "heads" not in case:
        assert lib.gauss_sum_attention_cached(attention(), cache(**case), None) == status
    assert lib.gauss_sum_cache_write(None, rows(), None) == 1
    assert lib.gauss_sum_cache_read(None, rows(), None) == 1
    assert lib.gauss_sum_attention_cached(attention(), None, None) == 1
    assert lib.gauss_sum_kernel_launches() == n


@pytest.mark.parametrize("case", [dict(sh=4 * BLOCK - 16), dict(sp=0), dict(sp=4 * BLOCK, sh=4 * BLOCK),
                                  dict(sp=16, sh=4 * BLOCK)])
def test_written_caches_must_not_overlap_themselves(lib, case):
    assert lib.gauss_sum_cache_write(cache(**case), rows(), None) == 1
    assert b"overlap" in lib.gauss_sum_last_error()


BAD_ROWS = [(dict(dtype=7), 1), (dict(B=-1), 1), (dict(M=-1), 1), (dict(B=1 << 31), 2), (dict(M=1 << 31), 2),
            (dict(ql=PTR + 2), 1), (dict(kl=PTR + 1), 1), (dict(k=(PTR + 1, 512, 128, 64)), 1),
            (dict(v=(PTR, -256, 64, 32)), 1), (dict(k=(PTR, 1 << 61, 128, 64)), 1)]


@pytest.mark.parametrize("case,status", BAD_ROWS)
def test_refused_rows(lib, case, status):
    n = lib.gauss_sum_kernel_launches()
    assert lib.gauss_sum_cache_write(cache(), rows(**case), None) == status
    assert lib.gauss_sum_last_error()
    assert lib.gauss_sum_cache_read(cache(), rows(**case), None) == status
    assert lib.gauss_sum_cache_write(cache(), None, None) == 1
    assert lib.gauss_sum_cache_read(cache(), None, None) == 1
    assert lib.gauss_sum_kernel_launches() == n


def test_rows_that_only_one_direction_refuses(lib):
    none = (0, 0, 0, 0)
    assert lib.gauss_sum_cache_write(cache(), rows(k=none), None) == 1
    assert lib.gauss_sum_cache_write(cache(), rows(v=none), None) == 1
    assert lib.gauss_sum_cache_read(cache(), rows(k=none, v=none), None) == 0       # nothing wanted
    assert lib.gauss_sum_cache_read(cache(), rows(k=(PTR, 512, 0, 64)), None) == 1  # overlaps itself
    assert lib.gauss_sum_cache_read(cache(), rows(v=(PTR, 256, 64, 16)), None) == 1


BAD = [(dict(dtype=9), 1), (dict(B=-1), 1), (dict(M=-1), 1), (dict(H=-2), 1), (dict(H=3), 1), (dict(tau=0.0), 1),
       (dict(tau=-1.0), 1), (dict(tau=float("nan")), 1), (dict(tau=float("inf")), 1), (dict(tau=1e300), 1),
       (dict(tau=1e-300), 1), (dict(causal=2), 1), (dict(ql=PTR + 2), 1), (dict(kl=PTR + 1), 1),
       (dict(lse=PTR + 2), 1), (dict(q=(0, 1, 1, 1)), 1), (dict(out=(0, 1, 1, 1)), 1),
       (dict(q=(PTR + 1, 1024, 256, 64)), 1), (dict(out=(PTR, 0, 128, 32)), 1), (dict(M=1 << 31), 2),
       (dict(M=1 << 30, H=8), 2), (dict(B=1 << 31), 2)]


@pytest.mark.parametrize("case,status", BAD)
def test_refused_attention(lib, case, status):
    n = lib.gauss_sum_kernel_launches()
    assert lib.gauss_sum_attention_cached(attention(**case), cache(), None) == status
    assert lib.gauss_sum_last_error()
    assert lib.gauss_sum_attention_cached(None, cache(), None) == 1
    assert lib.gauss_sum_attention_cached(attention(H=0), cache(heads=0), None) == 1
    assert lib.gauss_sum_kernel_launches() == n


def test_empty_calls_need_no_gpu(lib):
    none = (0, 0, 0, 0)
    assert lib.gauss_sum_cache_write(cache(), rows(B=0, k=none, v=none), None) == 0
    assert lib.gauss_sum_cache_write(cache(), rows(M=0, k=none, v=none), None) == 0
    assert lib.gauss_sum_cache_write(cache(per=0), rows(), None) == 0               # room for no token
    assert lib.gauss_sum_cache_write(cache(pages=0, data=0), rows(), None) == 0
    assert lib.gauss_sum_cache_read(cache(), rows(M=0), None) == 0
    assert lib.gauss_sum_attention_cached(attention(B=0, q=none, out=none), cache(), None) == 0
    assert lib.gauss_sum_attention_cached(attention(M=0, q=none, out=none), cache(), None) == 0


def test_block_bytes_are_the_headers():
    from paper_2609_04910_gb300._binding import cache_block_bytes
    assert cache_block_bytes(64, 32) == BLOCK
    assert cache_block_bytes(128, 128) == 16 * 144
    assert cache_block_bytes(80, 80) == 16 * 112
    assert cache_block_bytes(1, 256) == 16 * (16 + 128 + 4 + 16)


def test_binding_refuses_before_the_library_runs():
    import torch
    import paper_2609_04910_gb300 as gs
    data = torch.zeros(3, 2, 4, BLOCK, dtype=torch.uint8)
    with pytest.raises(ValueError):
        gs.AttentionCache(data.int(), 64, 32)
    with pytest.raises(ValueError):
        gs.AttentionCache(data[0], 64, 32)
    with pytest.raises(ValueError):
        gs.AttentionCache(data, 64, 64)
    with pytest.raises(ValueError):
        gs.AttentionCache(data[:, :, ::2], 64, 32)
    with pytest.raises(ValueError):
        gs.AttentionCache(data.transpose(2, 3).contiguous().transpose(2, 3), 64, 32)
    for tokens in (0, 8, 40):
        with pytest.raises(ValueError):
            gs.attention_cache(3, tokens, 2, 64, 32, device="cpu")
    with pytest.raises(ValueError):
        gs.attention_cache(3, 16, 2, 0, device="cpu")
    c = gs.attention_cache(3, 64, 2, 64, 32, device="cpu")
    assert c.data.shape == data.shape and c.page_tokens == 64 and (c.D, c.C) == (64, 32)
    x = torch.zeros(1, 2, 2, 64)
    with pytest.raises(ValueError):
        gs.gauss_sum_cache_write(c, x, x)
    with pytest.raises(ValueError):
        gs.gauss_sum_cache_write(c, x[0], x)
    with pytest.raises(ValueError):
        gs.gauss_sum_cache_read(c, 2, torch.float32)
    with pytest.raises(ValueError):
        gs.gauss_sum_attention_cached(x, c, 1.0)
    with pytest.raises(ValueError):
        gs.gauss_sum_attention_cached(x[0], c, 1.0)


def test_forms_agree_on_hand_made_groups():
    """The test form of the quantiser on groups whose codes are known."""
    import torch
    from attention_cache_forms import quantise, row_bytes, values
    x = torch.arange(16.0).repeat(4)[None]                  # steps of one
    codes, s, m = quantise(x)
    assert s.tolist() == [[1.0]] and m.tolist() == [[0.0]]
    assert torch.equal(values(codes, s, m)[0], x[0].double())
    codes, s, m = quantise(torch.tensor([[-7.5, 7.5, 0.0, 0.5, -0.5]]))   # ties go to even codes
    assert s.item() == 1.0 and codes.tolist() == [[0, 15, 8, 8, 7]]
    codes, s, m = quantise(torch.tensor([[1.0, float("inf")], [2.0, 2.0], [1e30, -1e-30]]))
    assert s[0].isnan().all() and codes[0].tolist() == [0, 0]
    assert s[1].item() == 0.0 and m[1].item() == 2.0
    assert codes[2].tolist() == [15, 0]
    row = [0] * 64
    row[32 + 8 + 3] = 9                                     # word j = 1 of chunk t = 1, nibble 3
    assert row_bytes(row, True)[8 + 4 + 1] == 0x90
    assert row_bytes(row, False)[2 * 4 + 2 + 1] == 0x90     # word j = 1 of chunk g = 2, nibble 3
