"""What a product does when one of its bounded waits gives up: the tiles whose sums are not known to be whole leave d as it
was, all others are right, the status says so, and the next product is whole again.  In these builds the wait has in fact
been met and only says that it was not, so that nothing is in flight that the kernel does not know of."""
import ctypes
import subprocess
from pathlib import Path

import pytest
import torch

from test_gpu_fp8 import _as_matrix, _exact_operands, _value

pytestmark = pytest.mark.gpu

ISSUER = 1  # the warp that issues the products; the epilogue's are 4 to 11


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    from paper_2607_10611_gb300 import builder as B
    from paper_2607_10611_gb300 import _native as N
    N.lib()
    out = tmp_path_factory.mktemp("waits") / "libwait_probe.so"
    objects = [str(B.OUT_DIR / (Path(s).stem + ".o")) for s in B.SOURCES if s != "fp8_matmul.cu"]
    subprocess.run([B.nvcc(), *B.NVCC_FLAGS, "-shared", "-Xlinker", "-Bsymbolic", str(Path(__file__).parent / "cuda" / "wait_probe.cu"),
                    *objects, "-o", str(out)], check=True)
    lib = ctypes.CDLL(str(out))
    lib.mpadam_e4m3_matmul.argtypes = [ctypes.c_void_p, ctypes.c_void_p]
    lib.mpadam_e4m3_status.argtypes = [ctypes.c_void_p, ctypes.POINTER(ctypes.c_int32)]
    lib.give_up.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_uint32]
    return lib


class Product:
    """d = 8 + a b^T of whole numbers, by the probe's kernels."""

    def __init__(self, probe, m, n, k):
        from paper_2607_10611_gb300 import _native as N
        (va, ea), (vb, eb) = _exact_operands(m, n, k, m + n + k)
        self.probe, self.N, self.shape = probe, N, (m, n, k)
        self.a, self.b = _as_matrix(va, ea), _as_matrix(vb, eb)
        self.want = (_value(va, ea) @ _value(vb, eb).t() + 8.0).float().cuda()
        assert not bool((self.want == 8.0).all())

    def __call__(self, block=-1, warp=ISSUER, lane=-1, parity=0):
        """(d, the status)"""
        N, (m, n, k) = self.N, self.shape
        assert self.probe.give_up(block, warp, lane, parity) == 0
        d = torch.full((m, n), 8.0, device="cuda")
        ptr = lambda t: t.data_ptr()
        p = N.mpadam_e4m3_product(ptr(self.a.codes), ptr(self.a.scales), self.a.codes.stride(0), ptr(self.b.codes),
                                  ptr(self.b.scales), self.b.codes.stride(0), ptr(d), n, m, n, k, N.MPADAM_F32, 1)
        stream = torch.cuda.current_stream().cuda_stream
        assert self.probe.mpadam_e4m3_matmul(ctypes.addressof(p), stream) == 0
        code = ctypes.c_int32()
        assert self.probe.mpadam_e4m3_status(stream, ctypes.byref(code)) == 0
        assert self.probe.give_up(-1, 0, 0, 0) == 0
        return d, code.value

    def whole(self):
        d, status = self()
        return status == 0 and torch.equal(d, self.want)

    def rest_is_right(self, d, rows, cols):
        """All of d but these rows and columns."""
        d = d.clone()
        d[rows, cols] = self.want[rows, cols]
        return torch.equal(d, self.want)


@pytest.mark.parametrize("lane", [-1, 7])
@pytest.mark.parametrize("m,n,k,block,parity", [(100, 512, 384, 2, 0), (100, 12800, 640, 57, 1), (16, 300, 500, 1, 0),
                                                (40, 500, 500, 3, 0)])
def test_a_tile_whose_operands_are_given_up_is_left_alone(probe, m, n, k, block, parity, lane):
    p = Product(probe, m, n, k)
    assert p.N.mpadam_debug_e4m3_plan(m, n, k)[1:] == (1, False) and p.whole()
    d, status = p(block, lane=lane, parity=parity)
    cols = slice(128 * block, min(128 * block + 128, n))
    assert status == 1 and bool((d[:, cols] == 8.0).all()) and p.rest_is_right(d, slice(None), cols)
    assert p.whole()


@pytest.mark.parametrize("lane", [-1, 7])
@pytest.mark.parametrize("rank", [0, 3])
def test_a_tile_of_which_one_share_is_given_up_is_left_alone(probe, rank, lane):
    m, n, k = 10, 500, 2048
    p = Product(probe, m, n, k)
    assert p.N.mpadam_debug_e4m3_plan(m, n, k) == (16, 4, False) and p.whole()
    d, status = p(4 * 2 + rank, lane=lane)
    assert status == 1 and bool((d[:, 256:384] == 8.0).all()) and p.rest_is_right(d, slice(None), slice(256, 384))
    assert p.whole()


@pytest.mark.parametrize("lane", [-1, 7])
@pytest.mark.parametrize("m,n,k,parity", [(1280, 2048, 512, 0), (1280, 2048, 1024, 1), (1290, 2000, 500, 0),
                                          (2048, 2048, 512, 0)])
def test_a_pair_whose_operands_are_given_up_leaves_its_tile_alone(probe, m, n, k, parity, lane):
    p = Product(probe, m, n, k)
    rows, _, pair = p.N.mpadam_debug_e4m3_plan(m, n, k)
    tiles = -(-m // rows)
    assert pair and tiles * -(-n // 256) <= 76 and tiles <= 8 and p.whole()
    t = 17
    d, status = p(2 * t, lane=lane, parity=parity)
    r, c = slice(rows * (t % tiles), min(rows * (t % tiles) + rows, m)), slice(256 * (t // tiles), min(256 * (t // tiles) + 256, n))
    assert status & 1 and bool((d[r, c] == 8.0).all()) and p.rest_is_right(d, r, c)
    assert p.whole()


@pytest.mark.parametrize("lane", [-1, 3])
def test_an_epilogue_warp_that_gives_up_stores_nothing(probe, lane):
    """Its 32 columns of d in half of the rows stay as they were; the tile's other warps may or may not have seen it."""
    p = Product(probe, 100, 512, 384)
    d, status = p(1, warp=5, lane=lane)
    mine, tile = (slice(0, 64), slice(160, 192)), d[:, 128:256]
    assert status == 4 and bool((d[mine] == 8.0).all())
    assert bool(((tile == 8.0) | (tile == p.want[:, 128:256])).all()) and p.rest_is_right(d, slice(None), slice(128, 256))
    assert p.whole()
