"""What the Newton-Schulz products do when one of their bounded waits runs out with copies and products in flight, early or
late in a launch, in any role (among them the one that takes tiles and waits for their rows): the launch ends, nothing is
written out, the status says so, and the next call is whole."""
import ctypes
import subprocess
from pathlib import Path

import pytest
import torch

pytestmark = pytest.mark.gpu

PRODUCER, ISSUER, TAKER, MAPS, EPILOGUE = 0, 1, 2, 3, 4  # warps; the epilogue's are 4 to 11
SHAPES = [(1500, 1600), (300, 300), (1000, 520)]


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    from paper_2607_10611_gb300 import builder as B
    from paper_2607_10611_gb300 import _native as N
    N.lib()
    out = tmp_path_factory.mktemp("limits") / "libnewton_limits.so"
    objects = [str(B.OUT_DIR / (Path(s).stem + ".o")) for s in B.SOURCES if s != "muon_products.cu"]
    subprocess.run([B.nvcc(), *B.NVCC_FLAGS, "-shared", "-Xlinker", "-Bsymbolic",
                    str(Path(__file__).parent / "cuda" / "newton_limit_probe.cu"), *objects, "-o", str(out)], check=True)
    lib = ctypes.CDLL(str(out))
    P = ctypes.c_void_p
    lib.mpadam_orthogonal_create.argtypes = [P, P, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, P]
    lib.mpadam_orthogonalize.argtypes = [P, P, P, P]
    lib.mpadam_orthogonal_status.argtypes = [P, P]
    lib.mpadam_orthogonal_destroy.argtypes = [P]
    lib.run_out.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_uint32]
    return lib


@pytest.mark.parametrize("block,warp", [(0, TAKER), (2, TAKER), (0, MAPS), (3, MAPS), (0, ISSUER), (6, ISSUER), (0, PRODUCER), (1, PRODUCER), (7, PRODUCER),
                                        (0, EPILOGUE), (1, EPILOGUE + 5), (4, EPILOGUE + 7)])
def test_a_wait_that_runs_out_ends_the_launch(probe, block, warp):
    x = [torch.randn(s, device="cuda", generator=torch.Generator(device="cuda").manual_seed(i)) for i, s in enumerate(SHAPES)]
    n = len(SHAPES)
    rows, cols = (ctypes.c_int64 * n)(*(r for r, _ in SHAPES)), (ctypes.c_int64 * n)(*(c for _, c in SHAPES))
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
        assert probe.run_out(-1, 0, 0) == 0
        want, code = call()
        assert code == 0 and all(float(t.abs().max()) < 1.5 for t in want)
        ended = 0
        for looks in (0, 1, 2, 3, 5, 8, 13, 21, 34, 55, 89, 144, 233, 377, 610, 987, 1597, 2584, 4181, 6765, 10946):
            assert probe.run_out(block, warp, looks) == 0
            out, code = call()  # (a launch whose warp looks less often is whole)
            assert all(bool((t == 8.0).all()) if code else torch.equal(t, w) for t, w in zip(out, want)), looks
            ended += code != 0
            assert probe.run_out(-1, 0, 0) == 0
            out, code = call()
            assert code == 0 and all(torch.equal(a, b) for a, b in zip(out, want)), looks
        assert ended >= 8
    finally:
        assert probe.run_out(-1, 0, 0) == 0
        probe.mpadam_orthogonal_destroy(state)
