"""Lists whose arrays overlap are refused by Muon, before any CUDA call (no GPU needed): a step would write both."""
import pytest

from paper_2607_10611_gb300 import builder as B

ROWS, COLS = 16, 8
SIZE = ROWS * COLS  # elements: 4 bytes of weights and 2 of momentum and copies each


@pytest.fixture(scope="module")
def N():
    B.build()
    from paper_2607_10611_gb300 import _native
    return _native


def _create(N, tensors):
    cfg = N.mpadam_muon_config(momentum=0.95, weight_decay=0.01, nesterov=1, steps=5, scale=0, weight_dtype=N.MPADAM_F32,
                               grad_dtype=N.MPADAM_BF16, momentum_dtype=N.MPADAM_BF16, rounding=0, reserved=0, seed=0)
    return N.mpadam_muon_create(tensors, cfg)


@pytest.mark.parametrize("second", [
    (0x10000, 0x50000, 0x60000), (0x10000 + 4 * SIZE - 4, 0x50000, 0x60000), (0x10000 - 4 * SIZE + 4, 0x50000, 0x60000),
    (0x40000, 0x20000, 0x60000), (0x40000, 0x20000 + 2 * SIZE - 2, 0x60000), (0x40000, 0x50000, 0x30000),
    (0x20000, 0x50000, 0x60000), (0x40000, 0x10002, 0x60000), (0x40000, 0x40000, 0x60000), (0x40000, 0x50000, 0x40010)])
def test_overlapping_arrays(N, second):
    with pytest.raises(N.MPAdamError, match="overlap") as ei:
        _create(N, [(0x10000, 0x20000, 0x30000, ROWS, COLS), (*second, ROWS, COLS)])
    assert ei.value.status == N.MPADAM_EINVAL


def test_arrays_side_by_side_and_empty_ones_do_not_overlap(N):
    """(What comes after the check needs a GPU, or is made of these addresses with one: only the list is looked at here.)"""
    import torch
    if torch.cuda.is_available():
        pytest.skip("the addresses are made up")
    w, m, c = 0x10000, 0x20000, 0x30000
    for second in ((w + 4 * SIZE, m + 2 * SIZE, c + 2 * SIZE, ROWS, COLS), (w, m, c, 0, COLS), (w, m, 0, ROWS, 0)):
        with pytest.raises(N.MPAdamError) as ei:
            _create(N, [(w, m, c, ROWS, COLS), second])
        assert ei.value.status != N.MPADAM_EINVAL and "overlap" not in str(ei.value)
