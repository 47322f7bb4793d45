"""Host logic around the training operators that needs no GPU: which device a handle's calls are made on, sizes that no list
can have, and what makes a build stale."""
import contextlib

import pytest
import torch


@pytest.fixture
def devices(monkeypatch):
    """Devices that torch.cuda.device makes current, innermost last."""
    stack = [torch.device("cuda", 0)]

    @contextlib.contextmanager
    def device(d):
        stack.append(torch.device(d))
        yield
        stack.pop()

    monkeypatch.setattr(torch.cuda, "device", device)
    return stack


def test_a_handles_calls_are_made_on_its_own_device(monkeypatch, devices):
    """The library refuses a status on another device, and waits for the current one before it frees."""
    from paper_2607_10611_gb300 import adamw
    seen = []
    for name in ("mpadam_adamw_status", "mpadam_adamw_destroy", "mpadam_grad_norm_destroy"):
        monkeypatch.setattr(adamw.N, name, lambda state, name=name: seen.append((name, state, devices[-1].index)) or 0)
    opt, norm = object.__new__(adamw.AdamW), object.__new__(adamw.GradNorm)
    opt.state, norm.state, opt.device, norm.device = 11, 12, torch.device("cuda", 1), torch.device("cuda", 2)
    assert opt.device_status() == 0
    opt.close()
    norm.close()
    opt.close()  # once is enough
    assert seen == [("mpadam_adamw_status", 11, 1), ("mpadam_adamw_destroy", 11, 1), ("mpadam_grad_norm_destroy", 12, 2)]
    assert opt.state is None and norm.state is None
