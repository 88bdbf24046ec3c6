"""Pinned values of the frequency table of stretched contexts."""
import pytest


@pytest.mark.parametrize("rotary_dim,base,length,factor,pairs", [
    # low = floor(10.47), high = ceil(22.51): pair 16 keeps 1 - (3/4)(6/13) of 0.01.
    (64, 10000.0, 4096, 4.0, {0: 1.0, 10: 0.0562341325, 11: 0.0421696503 * 49 / 52, 16: 0.01 * 34 / 52,
                              22: 0.00177827941 * 16 / 52, 23: 0.00133352143 / 4, 31: 0.000133352143 / 4}),
    # floor(18.08), ceil(34.98): pair 26 keeps 1 - (7/8)(8/17) of e^(-26 ln 500000 / 64).
    (128, 500000.0, 8192, 8.0, {18: 0.0249554087, 26: 0.00483942135 * 10 / 17, 35: 0.000764496988 / 8}),
    # A context of 128: the first bound lies below pair 0; ceil(10.47).
    (64, 10000.0, 128, 4.0, {0: 1.0, 1: 0.749894209 * (1 - 0.75 / 11), 11: 0.0421696503 / 4})])
def test_yarn_blend_is_linear_in_the_pair_index(rotary_dim, base, length, factor, pairs):
    from paper_2609_04910_gb300.rotary import angular_frequencies
    freqs, scale = angular_frequencies(rotary_dim, base, "yarn", factor, length)
    for i, f in pairs.items():
        assert freqs[i] == pytest.approx(f, rel=1e-8), i
    assert scale == pytest.approx({4.0: 1.13862944, 8.0: 1.20794415}[factor], rel=1e-8)
