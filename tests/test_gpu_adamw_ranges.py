"""Where the AdamW step and the norm leave their common ranges: arrays on 16-byte boundaries, long lists, small betas,
quotients at either end."""
import numpy as np
import pytest
import torch

from test_gpu_adamw import HP, Problem, probe  # noqa: F401

pytestmark = pytest.mark.gpu

from paper_2607_10611_gb300.adamw import AdamW, GradNorm  # noqa: E402


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


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_of_a_long_list(dtype):
    """Sixteen times the same 2^28 gradients, 4.3 10^9 in all.  Eight squares at most are added in binary32 (each with the
    square's own rounding, fused), their eight sums in three levels, and the rest in binary64: a sum of squares within 11
    units of 2^-24 of itself, so a norm within 6, and its own rounding to binary32, half of one."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    x = torch.randn(1 << 28, generator=gen, device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    total = sum(float(part.double().square().sum()) for part in x.split(1 << 25)) * 16
    norm = GradNorm([x.numel()] * 16, dtype)
    got = norm([x] * 16, 1.0).cpu().double()
    want = total ** 0.5
    print(f"{dtype}: relative error {float(got[0]) / want - 1:.2e}")
    assert abs(float(got[0]) - want) <= 6.5 * 2.0 ** -24 * want
    assert abs(float(got[1]) - 1.0 / want) <= 7 * 2.0 ** -24 / want


@pytest.mark.parametrize("kw", [dict(beta1=0.5, beta2=1.234567e-12, eps=1e-30), dict(beta1=0.5, beta2=3e-11, eps=1e-30),
                                dict(beta1=0.5, beta2=2.0 ** -30, eps=1e-30), dict(beta2=1e-30, eps=1e-30), dict(beta1=1e-30), dict(beta1=2.0 ** -81), dict(beta1=2.0 ** -30),
                                dict(beta1=1e-38, beta2=1e-38)])
def test_small_betas_bit_for_bit(kw):
    """Old scales down to 2^-47 times betas that make the product subnormal: gradients of the first step put the scales
    there, the second step's are zero, so that all there is comes of the decayed moments."""
    hp = {**HP, "weight_decay": 0.0, **kw}
    p = Problem([128 * 48, 1000], "f32", "f32", "e4m3", seed=21)
    opt = p.optimizer(seed=3, **{k: v for k, v in hp.items() if k != "lr"})
    for t in (1, 2, 3):
        host, dev = p.grads()
        for i, n in enumerate(p.sizes):
            scale = np.exp2(-np.arange(-(-n // 128)) % 44.0).repeat(128)[:n] if t == 1 else np.zeros(n)
            host[i] = (host[i] * scale).astype(np.float32)
            dev[i].copy_(torch.from_numpy(host[i]))
        opt.step(dev, t, hp["lr"])
        p.reference_step(host, t, 3, "nearest", "stochastic", hp=hp)
        p.check()


@pytest.mark.parametrize("near", [False, True])
def test_quotients_over_the_whole_range_of_the_step(probe, near):
    """Denominators in [2^-100, 2^25), numerators from 2^-100 up to where the quotient is still below 2^127; near: mantissas
    at either end, where quotients come closest to ties."""
    g = torch.Generator(device="cuda").manual_seed(1)
    n = 1 << 26
    below = lambda top: (torch.rand(n, generator=g, device="cuda", dtype=torch.float64) * top).to(torch.int32)

    def value(exponent):
        mantissa = torch.where(below(2) == 1, below(64), (1 << 23) - 1 - below(64)) if near else below(1 << 23)
        return ((exponent + 127) << 23 | mantissa).view(torch.float32)

    e = below(125) - 100
    top = (e + 125).clamp(max=126)
    a, d = value(-100 + below(top + 101)), value(e)
    assert float(a.min()) >= 2.0 ** -100 and float((a.double() / d.double()).min()) >= 2.0 ** -126
    wrong = torch.zeros(1, dtype=torch.int64, device="cuda")
    assert probe.quotient_probe(a.data_ptr(), d.data_ptr(), n, wrong.data_ptr()) == 0
    assert int(wrong) == 0, int(wrong)
