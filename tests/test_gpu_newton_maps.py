"""Lists whose tables and workspaces take the place of others that were destroyed: their tensor maps lie where others lay."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2607_10611_gb300 import Orthogonalizer  # noqa: E402


def test_a_list_in_the_place_of_another():
    """The same number of matrices, so that tables have the same size; other sides, so that bases and extents differ."""
    lists = [[(300, 700), (64, 900), (513, 200)], [(520, 530), (700, 300), (40, 40)], [(100, 1100), (257, 255), (800, 90)]]
    xs = [[torch.randn(s, device="cuda", generator=torch.Generator(device="cuda").manual_seed(10 * i + k)) for k, s in enumerate(shapes)]
          for i, shapes in enumerate(lists)]
    held = [Orthogonalizer(shapes, "f32") for shapes in lists]
    want = [o(x) for o, x in zip(held, xs)]
    torch.cuda.synchronize()
    for o in held:
        o.close()
    for turn in range(30):
        i = turn % len(lists)
        o = Orthogonalizer(lists[i], "f32")
        got = o(xs[i])
        assert o.device_status() == 0
        assert all(torch.equal(a, b) for a, b in zip(got, want[i])), turn
        o.close()
