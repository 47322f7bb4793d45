"""Where the AdamW step leaves its common ranges: arrays on 16-byte boundaries."""
import numpy as np
import pytest
import torch

from test_gpu_adamw import HP, Problem

pytestmark = pytest.mark.gpu

from paper_2607_10611_gb300.adamw import AdamW  # noqa: E402


@pytest.mark.parametrize("grads", ["f32", "bf16"])
@pytest.mark.parametrize("weights,state", [("f32", "f32"), ("bf16", "f32"), ("f32", "e4m3")])
def test_arrays_on_16_byte_boundaries_bit_for_bit(weights, state, grads):
    """Binary32 arrays at multiples of 16 bytes, not of 32 (BF16 ones of 8, 8-bit ones of 4)."""
    p = Problem([1, 7, 8, 128, 4000, 3841, 40000, 5], weights, grads, state, seed=22, offset=4, compute=weights == "f32")
    assert all(t.data_ptr() % 32 == 16 for t in p.gw if t.dtype == torch.float32)
    opt = p.optimizer()
    for t in (1, 2):
        host, dev = p.grads()
        opt.step(dev, t, HP["lr"])
        p.reference_step(host, t, 0, "nearest", "stochastic")
        p.check()


def test_arrays_on_16_byte_boundaries_are_stored_in_vectors():
    """60 M binary32 weights and moments, 16 bytes off a 32-byte boundary: single words took 1.9 times as long as whole
    sectors, two vectors of 16 bytes take hardly longer."""
    n, times = 60 << 20, {}
    g = torch.full((n,), 1e-3, dtype=torch.bfloat16, device="cuda")
    for offset in (0, 4):
        w, m, v = (torch.full((n + 4,), 1e-2, device="cuda")[offset:offset + n] for _ in range(3))
        opt = AdamW([w], [m], [v], weight_dtype="f32")
        start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        for t in range(1, 24):
            if t == 4:
                start.record()
            opt.step([g], t, 1e-3)
        end.record()
        end.synchronize()
        times[offset] = start.elapsed_time(end)
        assert opt.device_status() == 0
    assert times[4] < 1.3 * times[0], times
