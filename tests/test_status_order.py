"""What a state's status call has done when it returns (no GPU needed, the runtime's calls are fakes): the error word is read
with the device idle and cleared, and the clear is over.  A clear runs on the legacy stream, which the next call's stream need
not wait for; a call that still saw the old bits would write nothing."""
import subprocess
from pathlib import Path

import pytest

from paper_2607_10611_gb300 import builder as B


@pytest.fixture(scope="module")
def calls(tmp_path_factory):
    B.build()
    out, built = tmp_path_factory.mktemp("status"), {}

    def run(source, of):
        if source not in built:
            built[source] = out / source
            objects = [str(B.OUT_DIR / f"{Path(s).stem}.o") for s in B.SOURCES if Path(s).stem != source]
            flags = [f for f in B.NVCC_FLAGS if f not in ("-O3", "-lineinfo")]
            subprocess.run([B.nvcc(), *flags, f'-DSTATUS_SOURCE="{source}.cu"', f"-DOF_{source}",
                            str(Path(__file__).parent / "cuda" / "status_order_check.cu"), *objects, "-o", str(built[source])], check=True)
        return subprocess.run([str(built[source]), of], check=True, capture_output=True, text=True).stdout.splitlines()
    return run


@pytest.mark.parametrize("source,of", [("muon_api", "orthogonal"), ("muon_api", "muon"), ("train_api", "adamw"), ("mpadam_api", "step"),
                                       ("mpadam_api", "toy"), ("mpadam_api", "grid"), ("mpadam_api", "pool")])
def test_the_clear_is_over(calls, source, of):
    *made, last = calls(source, of)
    assert last == "returned 0, code 4"
    assert made[0] == "wait for the device" and (of in ("grid", "pool") or made[1] == "copy") and "clear" in made
    after = made[len(made) - made[::-1].index("clear"):]
    assert "wait for the device" in after or "wait for the legacy stream" in after
