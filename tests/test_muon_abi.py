"""Refusals of the orthogonalisation's and Muon's entry points that are decided on the host, before any CUDA call (no GPU
needed)."""
import math

import pytest

from paper_2607_10611_gb300 import builder as B


@pytest.fixture(scope="module")
def N():
    B.build()
    from paper_2607_10611_gb300 import _native
    return _native


def refused(N, f, *args, **kw):
    with pytest.raises(N.MPAdamError) as ei:
        f(*args, **kw)
    assert ei.value.status == N.MPADAM_EINVAL and N.mpadam_last_error()


@pytest.mark.parametrize("shapes,dtype,steps", [
    ([(4, -1)], 1, 5), ([(-1, 4)], 1, 5), ([(4, 4), (1, (1 << 20) + 1)], 1, 5), ([((1 << 20) + 1, 1)], 1, 5), ([(1 << 62, 4)], 0, 5),
    ([(4, 4)], 2, 5), ([(4, 4)], -1, 5), ([(4, 4)], 1, 0), ([(4, 4)], 1, 33), ([(4, 4)], 1, -1)])
def test_orthogonalisation_refuses(N, shapes, dtype, steps):
    refused(N, N.mpadam_orthogonal_create, shapes, dtype, steps)


def _config(N, **kw):
    d = dict(momentum=0.95, weight_decay=0.01, nesterov=1, steps=5, scale=0, weight_dtype=N.MPADAM_F32, grad_dtype=N.MPADAM_BF16,
             momentum_dtype=N.MPADAM_BF16, rounding=0, reserved=0, seed=0)
    return N.mpadam_muon_config(**{**d, **kw})


GOOD = (0x1000, 0x2000, 0x3000, 16, 8)


@pytest.mark.parametrize("bad", [
    dict(momentum=1.0), dict(momentum=-0.1), dict(momentum=math.nan), dict(weight_decay=-1.0), dict(weight_decay=math.inf),
    dict(nesterov=2), dict(nesterov=-1), dict(steps=0), dict(steps=33), dict(scale=2), dict(scale=-1), dict(weight_dtype=2),
    dict(grad_dtype=2), dict(momentum_dtype=-1), dict(rounding=2), dict(reserved=1),
    dict(weight_dtype=1)])  # (a BF16 weight has no compute copy)
def test_muon_refuses_bad_configs(N, bad):
    refused(N, N.mpadam_muon_create, [GOOD], _config(N, **bad))


@pytest.mark.parametrize("at,value", [(0, 0), (1, 0), (0, 0x1002), (1, 0x2001), (2, 0x3001), (3, -1), (4, -1), (3, (1 << 20) + 1),
                                      (4, (1 << 20) + 1)])
def test_muon_refuses_bad_matrices(N, at, value):
    t = list(GOOD)
    t[at] = value
    refused(N, N.mpadam_muon_create, [GOOD, tuple(t)], _config(N))


def test_null_handles_are_refused_and_their_destruction_is_not(N):
    refused(N, N.mpadam_orthogonalize, 0, [0x1000], [0x2000])
    refused(N, N.mpadam_orthogonal_status, 0)
    refused(N, N.mpadam_muon_step, 0, [0x1000], 1, 1e-3)
    refused(N, N.mpadam_muon_status, 0)
    N.mpadam_orthogonal_destroy(0)
    N.mpadam_muon_destroy(0)


def test_lists_that_muon_does_not_take(N):
    """By the torch side, on what it is given, here without a GPU."""
    import torch
    from paper_2607_10611_gb300 import Muon
    w = [torch.zeros(3, 4, dtype=torch.bfloat16)]
    with pytest.raises(ValueError, match="CUDA"):
        Muon(w, **Muon.init_state(w))
    with pytest.raises(ValueError, match="one entry"):
        Muon(w, [])
    with pytest.raises(KeyError):
        Muon(w, w, scale="fan")
