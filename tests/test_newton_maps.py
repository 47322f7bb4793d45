"""The tensor maps that a block of the Newton-Schulz products acquires when it comes to a product of a matrix (no GPU needed):
all that its tiles copy by, before the block's copies or anything else uses one."""
import re
import subprocess
from pathlib import Path

from paper_2607_10611_gb300 import builder as B


def test_every_map_that_a_tile_copies_by(tmp_path):
    """A = X X^T; B = a I + b A + c A A, of A as it lies and turned, A added; X = B X, of B as it lies and turned and X along
    its rows, into the other X, with X's second part added and stored."""
    exe = tmp_path / "maps"
    source = Path(__file__).parent / "cuda" / "newton_maps_check.cu"
    subprocess.run([B.nvcc(), "-std=c++17", "-O1", f"-I{B.INCLUDE}", f"-I{B.CSRC}", str(source), "-o", str(exe)], check=True)
    lines = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines()
    got = {tuple(line.split()[:2]): set(line.split()[2:]) for line in lines}
    want = {}
    for x in "01":
        want["1", x] = {f"x{x}", "a_patch"}
        want["2", x] = {"a", "a_along", "a_patch", "b_patch"}
        want["3", x] = {"b", "b_along", f"x_along{x}", f"x_patch{1 - int(x)}", "lo_patch"}
    assert got == want


def test_acquired_before_the_first_use():
    """In the kernel's source: the maps' warp acquires before it fetches, and says that a tile is ready behind both; every other
    use of a map is behind the read of a slot that waits for that."""
    source = (B.CSRC / "muon_products.cu").read_text()
    kernel = source[source.index("newton_kernel("):]
    own = kernel[kernel.index("} else if (warp == 3) {"):kernel.index("} else if (warp == 1 && rank == 0) {")]
    acquired, ready = own.index("acquire_map("), own.index("mbar_arrive_cluster(peer_addr(slot_ready(s), rank))")
    fetched = [m.start() for m in re.finditer(r"prefetch_map\(", own)]
    assert fetched and acquired < min(fetched) and max(fetched) < ready
    rest = kernel.replace(own, "")
    uses = [m.start() for m in re.finditer(r"\b(prefetch_map|pair_load_2d|tma_load_2d|tma_store_2d)\(", rest)]
    read = rest[rest.index("auto read_slot"):]
    assert "wait_cluster(slot_ready(s)" in read[:read.index("};")] and "prefetch_map(" not in rest
    assert uses and all(rest.rindex("read_slot(", 0, at) > rest.index("auto read_slot") + 20 for at in uses)
