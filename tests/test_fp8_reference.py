"""The numpy references of the 8-bit operators against torch's own E4M3 conversion and by their definitions (CPU)."""
import numpy as np
import pytest
import torch

import fp8_reference as R


def test_values_and_nearest_match_torch():
    codes = np.arange(256, dtype=np.uint8)
    t = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(R.e4m3_value(codes), t, equal_nan=True)
    rng = np.random.default_rng(0)
    y = np.concatenate([rng.uniform(-448, 448, 20000), rng.normal(0, 2.0 ** -7, 20000), R.E4M3, -R.E4M3,
                        (R.E4M3[1:] + R.E4M3[:-1]) / 2]).astype(np.float32)
    want = torch.from_numpy(y).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(R.e4m3_nearest(y), want)


def test_stochastic_rounding_is_unbiased_to_its_bits_and_keeps_the_grid():
    for y in (0.0, 2.0 ** -9, 0.013, 2.0 ** -6, 0.3, 17.7, 447.9, 448.0):
        r = np.arange(65536)
        v = R.e4m3_value(R.e4m3_stochastic(np.full(65536, y, np.float32), r))
        step = 2.0 ** (np.frexp(max(y, 2.0 ** -6))[1] - 4.0)
        assert abs(v.mean() - np.float32(y)) <= step * 2.0 ** -16
        assert len(set(v)) <= 2
        if y in R.E4M3:
            assert set(v) == {y}


@pytest.mark.parametrize("a,k", [(448.0, 0), (np.nextafter(448.0, 449.0), 1), (896.0, 1), (1.0, -8), (1.75, -8),
                                 (1.7500001, -7), (0.0, 0), (1e-45, -127), (3.4028234663852886e38, 120)])
def test_exponent(a, k):
    assert R.exponent(a) == k


def test_philox_matches_its_published_vectors():
    # Random123's known answers: counter and key all zero, and all ones
    z = R.philox(np.array([0]), 0, 0, 0)[0]
    assert [int(x) for x in z] == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    one = (1 << 64) - 1
    assert [int(x) for x in R.philox(np.array([one], np.uint64), 0, one, one)[0]] == \
        [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
