"""Host logic of the attention operators: exported symbols, refusals (all
before any CUDA work), and the rotary frequency table."""
import math
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PTR = 4096   # an aligned address that is never dereferenced


@pytest.fixture(scope="module")
def lib():
    from paper_2609_04910_gb300._binding import load_library
    from paper_2609_04910_gb300.build import build_library
    build_library()
    return load_library()


def test_every_declared_symbol_is_exported(lib):
    from paper_2609_04910_gb300._binding import ATTENTION_EXPORTS
    src = open(os.path.join(ROOT, "include", "gauss_sum", "attention.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    declared = sorted(set(re.findall(r"\b(gauss_sum\w*)\s*\(", src)))
    assert declared == sorted(ATTENTION_EXPORTS)
    for name in declared:
        assert hasattr(lib, name)


def attention(**kw):
    from paper_2609_04910_gb300._binding import _ATTENTION
    a = dict(dtype=1, B=2, M=4, N=6, H=4, Hk=2, D=64, C=32, tau=1.0, causal=1, ql=0, kl=0, lse=PTR)
    a.update({x: y for x, y in kw.items() if x not in ("q", "k", "v", "out")})
    arrays = {"q": (PTR, 1024, 256, 64), "k": (PTR, 768, 128, 64), "v": (PTR, 384, 64, 32),
              "out": (PTR, 512, 128, 32)}
    arrays.update({x: y for x, y in kw.items() if x in arrays})
    return _ATTENTION.pack(*(a[x] for x in ("dtype", "B", "M", "N", "H", "Hk", "D", "C", "tau", "causal",
                                            "ql", "kl")),
                           *arrays["q"], *arrays["k"], *arrays["v"], *arrays["out"], a["lse"])


BAD = [(dict(dtype=7), 1), (dict(B=-1), 1), (dict(M=-1), 1), (dict(N=-2), 1), (dict(H=3), 1),
       (dict(Hk=0), 1), (dict(D=0), 1), (dict(C=0), 1), (dict(tau=0.0), 1), (dict(tau=-1.0), 1),
       (dict(tau=float("nan")), 1), (dict(tau=float("inf")), 1), (dict(tau=1e300), 1), (dict(causal=2), 1),
       (dict(D=257), 2), (dict(C=300), 2), (dict(M=1 << 31), 2), (dict(N=1 << 31), 2),
       (dict(M=1 << 30, H=8), 2), (dict(ql=PTR + 2), 1), (dict(kl=PTR + 1), 1), (dict(lse=PTR + 2), 1),
       (dict(q=(0, 1, 1, 1)), 1), (dict(k=(0, 1, 1, 1)), 1), (dict(v=(0, 1, 1, 1)), 1),
       (dict(out=(0, 512, 128, 32)), 1), (dict(q=(PTR + 1, 1024, 256, 64)), 1),
       (dict(k=(PTR, -768, 128, 64)), 1), (dict(q=(PTR, 1 << 61, 256, 64)), 1),
       (dict(out=(PTR, 0, 128, 32)), 1), (dict(out=(PTR, 512, 128, 31)), 1),
       (dict(out=(PTR, 128, 128, 32)), 1)]


@pytest.mark.parametrize("case,status", BAD)
def test_refused_arguments(lib, case, status):
    n = lib.gauss_sum_kernel_launches()
    assert lib.gauss_sum_attention(attention(**case), None) == status
    assert lib.gauss_sum_last_error()
    assert lib.gauss_sum_kernel_launches() == n
    assert lib.gauss_sum_attention(None, None) == 1


def grads(**kw):
    from paper_2609_04910_gb300._binding import _ATTENTION_GRAD
    a = {"g": (PTR, 512, 128, 32), "g_lse": 0, "q": (PTR, 1024, 256, 64), "k": (PTR, 768, 128, 64),
         "v": (PTR, 384, 64, 32)}
    a.update(kw)
    return _ATTENTION_GRAD.pack(*a["g"], a["g_lse"], *a["q"], *a["k"], *a["v"])


@pytest.mark.parametrize("case,grad", [
    (dict(dtype=9), {}), (dict(lse=0), {}), (dict(out=(0, 1, 1, 1)), {}), ({}, dict(g=(0, 1, 1, 1))),
    ({}, dict(g_lse=PTR + 1)), ({}, dict(q=(PTR, 0, 256, 64))), ({}, dict(k=(PTR + 1, 768, 128, 64))),
    ({}, dict(v=(PTR, 384, 64, 16)))])
def test_refused_gradient_arguments(lib, case, grad):
    n = lib.gauss_sum_kernel_launches()
    assert lib.gauss_sum_attention_vjp(attention(**case), grads(**grad), None) == 1
    assert lib.gauss_sum_last_error()
    assert lib.gauss_sum_attention_vjp(attention(), None, None) == 1
    assert lib.gauss_sum_kernel_launches() == n


def test_empty_calls_need_no_gpu(lib):
    none = (0, 0, 0, 0)
    assert lib.gauss_sum_attention(attention(B=0, q=none, k=none, v=none, out=none), None) == 0
    assert lib.gauss_sum_attention(attention(M=0, q=none, out=none), None) == 0
    assert lib.gauss_sum_attention_vjp(attention(), grads(q=none, k=none, v=none), None) == 0


def rotary(**kw):
    from paper_2609_04910_gb300._binding import _ROTARY
    a = dict(dtype=2, B=2, M=3, H=4, Hk=1, D=64, R=32, scale=1.0, il=0, tr=0, pos=PTR, p64=0, sb=3, sm=1,
             freq=PTR, q=(PTR, 768, 256, 64), k=(0, 0, 0, 0), qo=(2 * PTR, 768, 256, 64),
             ko=(0, 0, 0, 0))
    a.update(kw)
    return _ROTARY.pack(*(a[x] for x in ("dtype", "B", "M", "H", "Hk", "D", "R", "scale", "il", "tr", "pos",
                                         "p64", "sb", "sm", "freq")),
                        *a["q"], *a["k"], *a["qo"], *a["ko"])


@pytest.mark.parametrize("case", [
    dict(dtype=5), dict(B=-1), dict(R=31), dict(R=66), dict(R=-2), dict(scale=float("nan")),
    dict(scale=1e300), dict(il=2), dict(tr=-1), dict(p64=3), dict(pos=0), dict(freq=0), dict(pos=PTR + 2),
    dict(freq=PTR + 4), dict(sb=-1), dict(q=(0, 1, 1, 1)), dict(qo=(0, 768, 256, 64)),
    dict(qo=(PTR, 768, 64, 192)), dict(qo=(2 * PTR, 768, 0, 64)), dict(k=(PTR, 192, 64, 64)),
    dict(q=(PTR + 1, 768, 256, 64))])
def test_refused_rotary_arguments(lib, case):
    n = lib.gauss_sum_kernel_launches()
    assert lib.gauss_sum_rotary(rotary(**case), None) == 1
    assert lib.gauss_sum_last_error()
    assert lib.gauss_sum_rotary(None, None) == 1
    assert lib.gauss_sum_kernel_launches() == n


def test_rotated_part_has_a_limit(lib):
    assert lib.gauss_sum_rotary(rotary(D=8192, R=4098), None) == 2


def test_empty_rotary_needs_no_gpu(lib):
    none = (0, 0, 0, 0)
    assert lib.gauss_sum_rotary(rotary(B=0, q=none, qo=none), None) == 0
    assert lib.gauss_sum_rotary(rotary(M=0, pos=0), None) == 0


def test_binding_refuses_before_the_library_runs():
    import torch
    import paper_2609_04910_gb300 as gs
    x = torch.zeros(1, 2, 3, 4)
    with pytest.raises(ValueError):
        gs.gauss_sum_attention(x, x, x, 1.0)
    with pytest.raises(ValueError):
        gs.gauss_sum_attention(x[0], x, x, 1.0)
    with pytest.raises(ValueError):
        gs.gauss_sum_attention_vjp(x, x, x, x, x, x, 1.0)
    with pytest.raises(ValueError):
        gs.gauss_sum_rotary(x, torch.zeros(1, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int64))


def turns(t):
    return [(x % (1 << 64)) / 2.0 ** 64 for x in t]


def test_frequency_table():
    from paper_2609_04910_gb300.rotary import angular_frequencies, fixed_point
    f, scale = angular_frequencies(8)
    assert scale == 1.0 and f == pytest.approx([1.0, 0.1, 0.01, 0.001])
    assert turns(fixed_point(f)) == pytest.approx([x / (2 * math.pi) for x in f], rel=1e-15)
    # Positions wrap exactly: 2^40 steps of a table entry, modulo one turn.
    t = fixed_point([1.0])[0]
    whole = (t << 40) % (1 << 64)
    assert whole / 2.0 ** 64 == pytest.approx((t / 2.0 ** 24) % 1.0, abs=1e-15)
    # A frequency of half a turn or more keeps its sign bit.
    assert turns(fixed_point([4.0]))[0] == pytest.approx(4.0 / (2 * math.pi))


def test_scaled_frequencies():
    from paper_2609_04910_gb300.rotary import angular_frequencies
    plain, _ = angular_frequencies(64)
    linear, s = angular_frequencies(64, scaling="linear", factor=4.0)
    assert s == 1.0 and linear == pytest.approx([f / 4 for f in plain])
    ntk, _ = angular_frequencies(64, scaling="ntk", factor=4.0)
    assert ntk[0] == plain[0] and ntk[-1] == pytest.approx(plain[-1] / 4)
    yarn, s = angular_frequencies(64, scaling="yarn", factor=4.0, original_length=4096)
    assert s == pytest.approx(0.1 * math.log(4.0) + 1)
    for f, y in zip(plain, yarn):
        n = 4096 * f / (2 * math.pi)   # turns over the original context
        if n > 40:
            assert y == f
        elif n < 0.7:
            assert y == pytest.approx(f / 4)
        else:
            assert f / 4 <= y <= f
    assert angular_frequencies(64, scaling="yarn", factor=1.0, original_length=4096)[0] == \
        pytest.approx(plain)
    assert angular_frequencies(0) == ([], 1.0)


@pytest.mark.parametrize("bad", [
    dict(rotary_dim=3), dict(rotary_dim=-2), dict(rotary_dim=8, scaling="cubic"),
    dict(rotary_dim=8, base=1.0), dict(rotary_dim=8, base=float("inf")),
    dict(rotary_dim=8, factor=0.5), dict(rotary_dim=8, scaling="yarn", factor=2.0),
    dict(rotary_dim=8, scaling="yarn", factor=2.0, original_length=0),
    dict(rotary_dim=8, scaling="yarn", factor=2.0, original_length=99, fast=1.0)])
def test_refused_frequencies(bad):
    from paper_2609_04910_gb300.rotary import angular_frequencies
    with pytest.raises(ValueError):
        angular_frequencies(**bad)
