"""How a pair of CTAs of the Newton-Schulz products ends when its producers and its issuer leave at any time (no GPU needed):
what the leader makes up for on the stages' barriers lets its waits end, and not before every copy has landed."""
import subprocess
from pathlib import Path

import pytest

from paper_2607_10611_gb300 import builder as B


@pytest.fixture(scope="module")
def played(tmp_path_factory):
    exe = tmp_path_factory.mktemp("newton") / "end"
    source = Path(__file__).parent / "cuda" / "newton_end_check.cu"
    subprocess.run([B.nvcc(), "-std=c++17", "-O2", f"-I{B.INCLUDE}", f"-I{B.CSRC}", str(source), "-o", str(exe)], check=True)
    return lambda *a: subprocess.run([str(exe), *map(str, a)], capture_output=True, text=True).stdout.strip()


@pytest.mark.parametrize("stages", [1, 2, 5])
def test_copies_have_landed_and_waits_end_whoever_leaves_first(played, stages):
    assert played(stages, 1000 * stages, 50000) == "ok"
