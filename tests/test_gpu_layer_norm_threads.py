"""Layer norms of several widths from several host threads at once, by the C entry points: no call's launch depends on what
another thread asks for meanwhile."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_calls_of_different_widths_from_several_threads():
    from paper_2607_10611_gb300 import _native as N
    N.lib()
    device = torch.cuda.current_device()
    failed = []

    class Calls:
        """Forward and backward of one width on a stream of its own."""

        def __init__(self, cols, rows=700):
            normal = lambda *s: torch.randn(*s, device="cuda")
            self.stream = torch.cuda.Stream()
            self.x, self.dy, self.w, self.b = normal(rows, cols), normal(rows, cols), normal(cols), normal(cols)
            self.out = [torch.empty(s, device="cuda") for s in ((rows, cols), (rows, cols), (cols,), (cols,), (rows,), (rows,))]
            bytes_of = N.mpadam_layer_norm_workspace(rows, cols)
            self.work = torch.empty(bytes_of, dtype=torch.uint8, device="cuda")
            y, dx, dw, db, mean, rstd = (t.data_ptr() for t in self.out)
            x, dy, w, b = (t.data_ptr() for t in (self.x, self.dy, self.w, self.b))
            self.forward = N.mpadam_layer_norm(x, cols, w, b, y, cols, mean, rstd, rows, cols, N.MPADAM_F32, N.MPADAM_F32, 1e-5, 0)
            self.backward = N.mpadam_layer_norm_grad(x, cols, dy, cols, w, mean, rstd, dx, cols, dw, db, self.work.data_ptr(), bytes_of,
                                                     rows, cols, N.MPADAM_F32, N.MPADAM_F32)

        def __call__(self):
            N.mpadam_layer_norm_forward(self.forward, self.stream.cuda_stream)
            N.mpadam_layer_norm_backward(self.backward, self.stream.cuda_stream)

        def many(self, times, start):
            torch.cuda.set_device(device)
            start.wait()
            try:
                for _ in range(times):
                    self()
            except N.MPAdamError as e:
                failed.append((self.x.shape, str(e)))

    calls = [Calls(cols) for cols in (8192, 4096, 6144, 2100)]
    torch.cuda.synchronize()
    alone = []
    for c in calls:
        c()
        c.stream.synchronize()
        alone.append([t.clone() for t in c.out])
    torch.cuda.synchronize()
    start = threading.Event()
    threads = [threading.Thread(target=c.many, args=(1500, start)) for c in calls]
    for t in threads:
        t.start()
    start.set()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed, failed
    for c, want in zip(calls, alone):
        assert all(torch.equal(a, b) for a, b in zip(c.out, want))
