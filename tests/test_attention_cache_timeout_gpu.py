"""Waits of the cached attention's kernels that run out (after 2 s), without faulting the GPU: the call
is reported as timed out, nothing is read that was not written, and the next call is as ever."""
import pytest
import torch

from test_attention_cache_gpu import filled
from test_attention_gpu import ints, points

pytestmark = pytest.mark.gpu


def stalled(call):
    """The call's results, the status of the same call with a wait that runs out, its results after."""
    import paper_2609_04910_gb300 as gs
    from paper_2609_04910_gb300 import _binding
    gs.gauss_sum_device_status()
    want = call()
    gs.gauss_sum_device_status()
    _binding.testing_stall_cached_attention(True)
    try:
        call()                                          # (the launches succeed)
    finally:
        _binding.testing_stall_cached_attention(False)
    with pytest.raises(gs.GaussSumError) as e:
        gs.gauss_sum_device_status()
    assert e.value.status == 5 and "block (0, 0)" in e.value.message
    for _ in range(3):
        got = call()
        gs.gauss_sum_device_status()
        assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B,long", [(1, 0), (64, 4000), (64, 100), (3, 6000)])
def test_few_rows(B, long, dtype):
    """One set of rows to a block; blocks that would have gone on to further sets (64 problems of which
    one is long: 12 units a block, 8 a short set); sets over many blocks."""
    import paper_2609_04910_gb300 as gs
    kl = [100 + b % 7 for b in range(B)]
    kl[-1] = long or kl[-1]
    s = filled(B, 6000 if long else 112, 8, 64, 64, 16, B, kl)
    q = points((B, 1, 32, 64), dtype, 3)
    stalled(lambda: gs.gauss_sum_attention_cached(q, s.cache, 0.125, causal=True, k_lengths=ints(kl), page_table=s.table))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("B,M,held", [(1, 9, 272), (2, 40, 700), (40, 64, 1500), (1, 33, 20000)])
def test_tiles(B, M, held, dtype):
    """Key tiles of one trip round the ring of copies or of many, one block to a set of rows or a split of its keys."""
    import paper_2609_04910_gb300 as gs
    kl = [held - 3 * (b % 5) for b in range(B)]
    s = filled(B, held, 2, 128, 128, 64, B, kl)
    q = points((B, M, 8, 128), dtype, 3)
    stalled(lambda: gs.gauss_sum_attention_cached(q, s.cache, 0.09, causal=True, k_lengths=ints(kl), page_table=s.table))
