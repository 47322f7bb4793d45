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


def test_a_failed_link_of_the_torch_module_is_not_a_finished_build(monkeypatch, tmp_path):
    """An older module beside a new library would read the library's structs by their old layout."""
    from pathlib import Path
    from types import SimpleNamespace
    from paper_2607_10611_gb300 import builder as B
    for name, file in (("OUT_DIR", "."), ("LIB", B.LIB.name), ("EXT", B.EXT.name), ("EXT_TORCH", B.EXT_TORCH.name)):
        monkeypatch.setattr(B, name, tmp_path / file)
    state = {"fails": False, "made": 0}

    def run(cmd, **kw):
        out = Path(cmd[cmd.index("-o") + 1])
        if state["fails"] and "-ltorch_python" in cmd:
            return SimpleNamespace(returncode=1, stdout="", stderr="no space left")
        state["made"] += 1
        out.write_text(str(state["made"]))
        return SimpleNamespace(returncode=0, stdout="", stderr="")

    monkeypatch.setattr(B.subprocess, "run", run)
    B.build()
    assert not B.needs_build()
    old = B.EXT.read_text()
    state["fails"] = True
    with pytest.raises(RuntimeError, match="no space left"):
        B.build(force=True)
    assert B.EXT.read_text() == old and B.needs_build()
    with pytest.raises(RuntimeError, match="no space left"):
        B.build()
    state["fails"] = False
    B.build()
    assert B.EXT.read_text() != old and not B.needs_build()


TOP = (1 << 63) - 1


@pytest.mark.parametrize("sizes", [[TOP], [TOP - 500], [5, TOP - 3000], [1 << 62] * 3, [TOP - 3000, 1 << 62, 5],
                                   [(1 << 31) * 4000], [1 << 41] * 8, [-(-TOP // 4), -(-TOP // 4), -(-TOP // 4), -(-TOP // 4), 7]])
def test_sizes_that_no_list_can_have_are_refused(sizes):
    """Before any arithmetic on them could overflow."""
    from paper_2607_10611_gb300 import _native as N, build
    build()
    cfg = N.mpadam_adamw_config(0.9, 0.999, 1e-8, 0.0, N.MPADAM_BF16, N.MPADAM_F32, N.MPADAM_E4M3, 0, 0, 0, 0)
    for create in (lambda: N.mpadam_grad_norm_create(sizes, N.MPADAM_F32),
                   lambda: N.mpadam_adamw_create([(0x1000, 0x2000, 0x3000, 0x4000, 0x5000, 0, n) for n in sizes], cfg)):
        with pytest.raises(N.MPAdamError) as e:
            create()
        assert e.value.status == N.MPADAM_EINVAL and "too many elements" in str(e.value)
