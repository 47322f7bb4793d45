"""The tensor maps that a block of the Newton-Schulz products acquires before any copy uses one (no GPU needed): every map of
the matrices that the launch works on, once, and nothing else."""
import re
import subprocess
from pathlib import Path

import pytest

from paper_2607_10611_gb300 import builder as B


@pytest.fixture(scope="module")
def reached(tmp_path_factory):
    exe = tmp_path_factory.mktemp("newton") / "maps"
    source = Path(__file__).parent / "cuda" / "newton_maps_check.cu"
    subprocess.run([B.nvcc(), "-std=c++17", "-O1", f"-I{B.INCLUDE}", f"-I{B.CSRC}", str(source), "-o", str(exe)], check=True)
    return lambda *a: subprocess.run([str(exe), *map(str, a)], check=True, capture_output=True, text=True).stdout.splitlines()


@pytest.mark.parametrize("all_of,first,members", [(1, 0, 1), (5, 0, 5), (40, 7, 20), (3, 2, 1), (4, 1, 0)])
def test_every_map_of_the_launch_once(reached, all_of, first, members):
    *maps, others = reached(all_of, first, members)
    assert others == "others 0" and len(maps) == 13 * all_of
    for line in maps:
        matrix, _, times = line.split()
        assert int(times) == (first <= int(matrix) < first + members), line


def test_acquired_before_the_first_use():
    """In the kernel's source: all blocks acquire all maps, and meet, before anything is prefetched or copied by one."""
    source = (B.CSRC / "muon_products.cu").read_text()
    kernel = source[source.index("newton_kernel("):]
    acquired = kernel.index("acquire_map(newton_map(")
    met = kernel.index("__syncthreads()", acquired)
    uses = [m.start() for m in re.finditer(r"\b(prefetch_map|pair_load_2d|tma_load_2d|tma_store_2d)\(", kernel)]
    assert uses and min(uses) > met
