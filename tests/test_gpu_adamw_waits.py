"""What the AdamW step does when a bounded wait gives up in one lane of a warp: the whole warp leaves its elements as they
were, all others are stepped, and the status says so.  In this build the wait has in fact been met and only says that it was
not, so that nothing is in flight that the kernel does not know of."""
import ctypes
import subprocess
from pathlib import Path

import numpy as np
import pytest
import torch

from test_gpu_adamw import HP, Problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    from paper_2607_10611_gb300 import builder as B
    from paper_2607_10611_gb300 import _native as N
    N.lib()
    out = tmp_path_factory.mktemp("waits") / "libadamw_wait_probe.so"
    objects = [str(B.OUT_DIR / (Path(s).stem + ".o")) for s in B.SOURCES if s != "adamw.cu"]
    subprocess.run([B.nvcc(), *B.NVCC_FLAGS, '-DPROBE_SOURCE="adamw.cu"', "-shared", "-Xlinker", "-Bsymbolic",
                    str(Path(__file__).parent / "cuda" / "wait_probe.cu"), *objects, "-o", str(out)], check=True)
    lib = ctypes.CDLL(str(out))
    P, i32 = ctypes.c_void_p, ctypes.c_int32
    lib.mpadam_adamw_create.argtypes = [P, i32, P, P]
    lib.mpadam_adamw_step.argtypes = [P, P, ctypes.c_int64, ctypes.c_float, P, P]
    lib.mpadam_adamw_status.argtypes = [P, P]
    lib.mpadam_adamw_destroy.argtypes = [P]
    lib.give_up.argtypes = [i32, i32, i32, ctypes.c_uint32]
    return lib


@pytest.mark.parametrize("state", ["f32", "e4m3"])
@pytest.mark.parametrize("lane", [-1, 0, 7])
def test_a_warp_gives_up_as_a_whole(probe, state, lane):
    """Tensors of one tile each, a CTA each: the second one's third warp gives up."""
    from paper_2607_10611_gb300 import _native as N
    sizes = [2000, 2500, 300]
    p = Problem(sizes, "f32", "f32", state, seed=5)
    low = state == "e4m3"
    before = [[t.view(torch.uint8).clone() for t in (w, m, v)] for w, m, v in zip(p.gw, p.gm, p.gv)]
    rows = [N.mpadam_adamw_tensor(w.data_ptr(), m.data_ptr(), v.data_ptr(), p.gms[i].data_ptr() if low else None,
                                  p.gvs[i].data_ptr() if low else None, None, n)
            for i, (w, m, v, n) in enumerate(zip(p.gw, p.gm, p.gv, sizes))]
    cfg = N.mpadam_adamw_config(HP["beta1"], HP["beta2"], HP["eps"], HP["weight_decay"], N.MPADAM_F32, N.MPADAM_F32,
                                N.MPADAM_E4M3 if low else N.MPADAM_F32, 0, 0, 0, 0)
    state_p, code = ctypes.c_void_p(), ctypes.c_int32()
    host, dev = p.grads()
    assert probe.mpadam_adamw_create((N.mpadam_adamw_tensor * 3)(*rows), 3, ctypes.addressof(cfg), ctypes.byref(state_p)) == 0
    try:
        assert probe.give_up(1, 2, lane, 0) == 0
        pointers = (ctypes.c_void_p * 3)(*[g.data_ptr() for g in dev])
        stream = torch.cuda.current_stream().cuda_stream
        assert probe.mpadam_adamw_step(state_p, pointers, 1, HP["lr"], None, stream) == 0
        assert probe.mpadam_adamw_status(state_p, ctypes.byref(code)) == 0 and code.value == 2
    finally:
        probe.give_up(-1, 0, 0, 0)
        probe.mpadam_adamw_destroy(state_p)
    p.reference_step(host, 1, 0, "nearest", "nearest")
    mine = slice(512, 768)  # 256 elements a warp
    for i, tensors in enumerate(zip(p.gw, p.gm, p.gv)):
        for got, old, want in zip(tensors, before[i], (p.w[i], p.m[i], p.v[i])):
            got, want = got.view(torch.uint8).cpu().numpy().copy(), np.ascontiguousarray(want).view(np.uint8).copy()
            if i == 1:
                size = len(got) // sizes[1]
                at = slice(mine.start * size, mine.stop * size)
                assert np.array_equal(got[at], old.cpu().numpy()[at])
                got[at] = want[at]
            assert np.array_equal(got, want)


def test_a_warp_that_gives_up_waits_for_the_stages_ahead(probe):
    """200 tensors of one tile on 152 CTAs: block 1 has tiles 1 and 153 in its ring when its third warp gives up, and leaves
    both; everything else is stepped."""
    from paper_2607_10611_gb300 import _native as N
    n, count = 1000, 200
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert sms < count - 1 < 2 * sms
    w, m, v, g = (torch.full((count, 1024), x, device="cuda") for x in (0.5, 0.0, 0.0, 1.0))
    rows = [N.mpadam_adamw_tensor(w[i].data_ptr(), m[i].data_ptr(), v[i].data_ptr(), None, None, None, n) for i in range(count)]
    cfg = N.mpadam_adamw_config(0.9, 0.999, 1e-8, 0.0, N.MPADAM_F32, N.MPADAM_F32, N.MPADAM_F32, 0, 0, 0, 0)
    state, code = ctypes.c_void_p(), ctypes.c_int32()
    assert probe.mpadam_adamw_create((N.mpadam_adamw_tensor * count)(*rows), count, ctypes.addressof(cfg), ctypes.byref(state)) == 0
    try:
        assert probe.give_up(1, 2, 7, 0) == 0
        pointers = (ctypes.c_void_p * count)(*[x.data_ptr() for x in g])
        assert probe.mpadam_adamw_step(state, pointers, 1, 0.25, None, torch.cuda.current_stream().cuda_stream) == 0
        assert probe.mpadam_adamw_status(state, ctypes.byref(code)) == 0 and code.value == 2
    finally:
        probe.give_up(-1, 0, 0, 0)
        probe.mpadam_adamw_destroy(state)
    left = torch.zeros(count, 1024, dtype=torch.bool, device="cuda")
    left[:, n:] = True
    left[[1, 1 + sms], 512:768] = True
    assert torch.equal(w == 0.5, left) and torch.equal(m == 0.0, left) and torch.equal(v == 0.0, left)
