"""The order in which the Newton-Schulz products' tiles are taken, by the library's own host code (no GPU needed): every tile of
every product once, each behind all that it is made of, and none before the last reader of what it writes over."""
import subprocess
from pathlib import Path

import pytest

from paper_2607_10611_gb300 import builder as B

SIGNALS = 16  # a tile's stores, in the unit of what tiles wait for


@pytest.fixture(scope="module")
def schedule(tmp_path_factory):
    exe = tmp_path_factory.mktemp("newton") / "schedule"
    source = Path(__file__).parent / "cuda" / "newton_schedule_check.cu"
    subprocess.run([B.nvcc(), "-std=c++17", "-O1", f"-I{B.INCLUDE}", f"-I{B.CSRC}", str(source), "-o", str(exe)], check=True)

    def run(shapes, steps):
        sides = [str(n) for r, c in shapes for n in (min(r, c), max(r, c))]
        out = subprocess.run([str(exe), str(steps), *sides], check=True, capture_output=True, text=True).stdout
        return [tuple(int(v) for v in line.split()) for line in out.splitlines()]
    return run


def _across(n):
    return -(-n // 256)


@pytest.mark.parametrize("steps", [1, 2, 5])
@pytest.mark.parametrize("shapes", [
    [], [(1, 1)], [(256, 256)], [(257, 300)], [(1500, 1501)], [(2000, 5000)], [(1, 3000), (700, 3), (64, 64)],
    [(768, 2304), (768, 768), (768, 2304), (2304, 768)] * 3, [(1 + i, 1 + 7 * i) for i in range(100)]])
def test_every_tile_is_behind_what_it_is_made_of(schedule, shapes, steps):
    made = {}   # (matrix, product of the steps' 3) -> its tiles so far
    rows = [[0] * _across(min(s)) for s in shapes]  # tiles stored in every 256 rows
    for matrix, which, tm, tn, k, need, first, adds, keep in schedule(shapes, steps):
        r, c = min(shapes[matrix]), max(shapes[matrix])
        down, across = _across(r), _across(c)
        step, rest = divmod(need // SIGNALS, 2 * down + across)
        assert need % SIGNALS == 0 and rest == (which - 1) * down and step < steps and first == step % 2
        assert k == -(-(c if which == 1 else r) // 64)
        assert adds == (which == 2 or (which == 3 and step + 1 < steps)) and keep == (which == 3 and step + 2 < steps)
        tiles = made.setdefault((matrix, 3 * step + which), set())
        assert (tm, tn) not in tiles and 0 <= tm < down and 0 <= tn < (across if which == 3 else tm + 1)
        tiles.add((tm, tn))
        # what it waits for is ahead of it in the list: X's rows tm and tn, A's rows tm and tn, or B's row tm
        waits = {tm} if which == 3 else {tm, tn}
        assert all(rows[matrix][i] * SIGNALS >= need for i in waits)
        if which == 3:  # and with B's row all of X, which it reads a column of, and the readers of the X that it writes over
            assert len(made[matrix, 3 * step + 1]) == down * (down + 1) // 2
            assert step == 0 or len(made[matrix, 3 * step]) == down * across
        else:  # A or B is written over: the last step's readers of these rows
            if step:
                reader = made[matrix, 3 * (step - 1) + which + 1]
                done = {(i, j) for i, j in reader if i in waits or (which == 1 and j in waits)}
                of = {(i, j) for i in range(down) for j in range(across if which == 2 else i + 1)
                      if i in waits or (which == 1 and j in waits)}
                assert done == of
        for i in {tm} if which == 3 else {tm, tn}:
            rows[matrix][i] += 1
    for m, (a, b) in enumerate(shapes):
        down, across = _across(min(a, b)), _across(max(a, b))
        for step in range(steps):
            assert [len(made[m, 3 * step + w]) for w in (1, 2, 3)] == [down * (down + 1) // 2] * 2 + [down * across]
        assert rows[m] == [steps * (2 * down + across)] * down
