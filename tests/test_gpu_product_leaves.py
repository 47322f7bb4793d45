"""What an 8-bit product does when a block's epilogue leaves before its products are done: the block waits for them all the
same, the tile is left as it was, all others are right, the status says so, and the next product is whole."""
import ctypes
import subprocess
from pathlib import Path

import pytest

from test_gpu_product_waits import Product

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    from paper_2607_10611_gb300 import builder as B
    from paper_2607_10611_gb300 import _native as N
    N.lib()
    out = tmp_path_factory.mktemp("leaves") / "libleave_probe.so"
    objects = [str(B.OUT_DIR / (Path(s).stem + ".o")) for s in B.SOURCES if s != "fp8_matmul.cu"]
    subprocess.run([B.nvcc(), *B.NVCC_FLAGS, "-shared", "-Xlinker", "-Bsymbolic",
                    str(Path(__file__).parent / "cuda" / "product_leave_probe.cu"), *objects, "-o", str(out)], check=True)
    lib = ctypes.CDLL(str(out))
    lib.mpadam_e4m3_matmul.argtypes = [ctypes.c_void_p, ctypes.c_void_p]
    lib.mpadam_e4m3_status.argtypes = [ctypes.c_void_p, ctypes.POINTER(ctypes.c_int32)]
    lib.give_up.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_uint32]
    return lib


@pytest.mark.parametrize("m,n,k,block", [(100, 512, 384, 2), (128, 12800, 16384, 57), (16, 300, 500, 1)])
def test_a_block_waits_for_its_products(probe, m, n, k, block):
    p = Product(probe, m, n, k)
    assert p.N.mpadam_debug_e4m3_plan(m, n, k)[1:] == (1, False) and p.whole()
    for _ in range(5):
        d, status = p(block)
        cols = slice(128 * block, min(128 * block + 128, n))
        assert status == 4 and bool((d[:, cols] == 8.0).all()) and p.rest_is_right(d, slice(None), cols)
        assert p.whole()


@pytest.mark.parametrize("rank", [0, 1])
@pytest.mark.parametrize("m,n,k", [(1280, 2048, 512), (2048, 2048, 8192)])
def test_a_pair_waits_for_its_products(probe, m, n, k, rank):
    p = Product(probe, m, n, k)
    rows, _, pair = p.N.mpadam_debug_e4m3_plan(m, n, k)
    tiles = -(-m // rows)
    assert pair and tiles * -(-n // 256) <= 76 and tiles <= 8 and p.whole()
    t = 17
    for _ in range(5):
        d, status = p(2 * t + rank)
        r, first = slice(rows * (t % tiles), min(rows * (t % tiles) + rows, m)), 256 * (t // tiles) + 128 * rank
        c = slice(first, first + 128)
        assert status == 4 and bool((d[r, c] == 8.0).all()) and p.rest_is_right(d, r, c)
        assert p.whole()
