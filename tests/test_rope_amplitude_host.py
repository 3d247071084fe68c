"""The amplitude of MSA_ROPE_SCALE_PAIRS: 0.1 ln(factor) + 1 for contexts that are stretched, 1 for others."""
import math

import numpy as np
import pytest

import paper_2606_02964_amd as msa


@pytest.mark.parametrize("factor", [1e-300, 1e-5, 0.5, 1.0 - 2.0 ** -53, 1.0, 1.0 + 2.0 ** -52, 1.5, 4.0, 1e6])
def test_amplitude(factor):
    freq, amplitude = msa.msa_rope_freqs(64, 10000.0, msa.MSA_ROPE_SCALE_PAIRS, factor, 4096.0, 1.0, 32.0)
    assert amplitude == np.float32(0.1 * math.log(factor) + 1.0 if factor > 1.0 else 1.0)
    assert np.isfinite(freq).all()


@pytest.mark.parametrize("original_len", [1.0, 6.0, 60.0, 150.0, 1e30])
def test_ends_of_the_mixture(original_len):
    """Pairs are taken within 0 .. rotary_dim - 1: the fastest one keeps its frequency, and where both ends are the
    same pair all behind it are divided."""
    R, base, factor, low, high = 64, 10000.0, 8.0, 1.0, 32.0
    freq, _ = msa.msa_rope_freqs(R, base, msa.MSA_ROPE_SCALE_PAIRS, factor, original_len, low, high)
    plain = np.array([base ** (-2.0 * i / R) for i in range(R // 2)])
    pair = lambda turns: R * math.log(original_len / (2 * math.pi * turns)) / (2 * math.log(base))  # noqa: E731
    start, stop = (min(max(x, 0), R - 1) for x in (math.floor(pair(high)), math.ceil(pair(low))))
    for i in range(R // 2):
        s = (1.0 if i <= start else 0.0) if start == stop else min(1.0, max(0.0, (stop - i) / (stop - start)))
        assert freq[i] == pytest.approx(plain[i] * s + plain[i] / factor * (1 - s), rel=1e-13)
