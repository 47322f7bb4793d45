"""What the Newton-Schulz products do when one of their bounded waits gives up: nothing is written out, the status says so,
and the next call is whole.  In this build the wait has in fact been met and only says that it was not."""
import ctypes
import subprocess
from pathlib import Path

import pytest
import torch

pytestmark = pytest.mark.gpu

PRODUCER, ISSUER, EPILOGUE = 0, 1, 5  # warps


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    from paper_2607_10611_gb300 import builder as B
    from paper_2607_10611_gb300 import _native as N
    N.lib()
    out = tmp_path_factory.mktemp("waits") / "libnewton_probe.so"
    objects = [str(B.OUT_DIR / (Path(s).stem + ".o")) for s in B.SOURCES if s != "muon_products.cu"]
    subprocess.run([B.nvcc(), *B.NVCC_FLAGS, '-DPROBE_SOURCE="muon_products.cu"', "-shared", "-Xlinker", "-Bsymbolic",
                    str(Path(__file__).parent / "cuda" / "wait_probe.cu"), *objects, "-o", str(out)], check=True)
    lib = ctypes.CDLL(str(out))
    P = ctypes.c_void_p
    lib.mpadam_orthogonal_create.argtypes = [P, P, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, P]
    lib.mpadam_orthogonalize.argtypes = [P, P, P, P]
    lib.mpadam_orthogonal_status.argtypes = [P, P]
    lib.mpadam_orthogonal_destroy.argtypes = [P]
    lib.give_up.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_uint32]
    return lib


# Which tiles a pair of CTAs (blocks 2 i and 2 i + 1) takes differs from call to call, and so whether it comes to the wait that
# gives up: a call that does not is whole, and of twenty some do (of 118 tiles a step a pair takes seven or eight in all).
# What an epilogue waits for with this barrier is X's second part or A.
@pytest.mark.parametrize("block,warp,lane,parity", [(0, ISSUER, -1, 0), (0, ISSUER, 7, 1), (0, PRODUCER, 0, 0), (1, PRODUCER, 0, 0),
                                                    (3, PRODUCER, 0, 0), (0, EPILOGUE, -1, 0), (1, EPILOGUE, 3, 0), (2, EPILOGUE, 0, 1)])
def test_nothing_is_written_when_a_wait_gives_up(probe, block, warp, lane, parity):
    shapes = [(1500, 1600), (300, 300), (1000, 520)]
    x = [torch.randn(s, device="cuda", generator=torch.Generator(device="cuda").manual_seed(i)) for i, s in enumerate(shapes)]
    n = len(shapes)
    rows, cols = (ctypes.c_int64 * n)(*(r for r, _ in shapes)), (ctypes.c_int64 * n)(*(c for _, c in shapes))
    state = ctypes.c_void_p()
    assert probe.mpadam_orthogonal_create(rows, cols, n, 0, 5, ctypes.byref(state)) == 0
    stream = torch.cuda.current_stream().cuda_stream

    def call():
        out = [torch.full_like(t, 8.0) for t in x]
        xs, ys = (ctypes.c_void_p * n)(*(t.data_ptr() for t in x)), (ctypes.c_void_p * n)(*(t.data_ptr() for t in out))
        assert probe.mpadam_orthogonalize(state, xs, ys, stream) == 0
        code = ctypes.c_int32()
        assert probe.mpadam_orthogonal_status(state, ctypes.byref(code)) == 0
        return out, code.value

    try:
        assert probe.give_up(-1, 0, 0, 0) == 0
        want, code = call()
        assert code == 0 and all(float(t.abs().max()) < 1.5 for t in want)
        assert probe.give_up(block, warp, lane, parity) == 0
        codes = []
        while not codes or (not codes[-1] and len(codes) < 20):
            out, code = call()
            codes.append(code)
            assert all(bool((t == 8.0).all()) if code else torch.equal(t, w) for t, w in zip(out, want))
        assert probe.give_up(-1, 0, 0, 0) == 0
        assert codes[-1] != 0
        out, code = call()
        assert code == 0 and all(torch.equal(a, b) for a, b in zip(out, want))
    finally:
        assert probe.give_up(-1, 0, 0, 0) == 0
        probe.mpadam_orthogonal_destroy(state)
