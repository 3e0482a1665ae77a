"""The operators' C ABI from several threads at once, each with its own stream and workspace, in a process of its own: the first
launches of every kernel happen side by side, with different sizes of shared memory.  Every call succeeds, also the largest one
afterwards, and leaves the bits that it leaves alone."""
import ctypes as C
import os
import subprocess
import sys
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
WIDTHS = (4600, 520, 1000, 2000, 544, 3000, 4000, 1544)  # one kernel instance for each pair of types, 8 to 184 KB of stages
F32, BF16 = 0, 1
TYPE = {F32: torch.float32, BF16: torch.bfloat16}


class Caller:
    """Arguments of a gradient call, kept alive, with results of its own; parts are left out by turns."""

    def __init__(self, ops, d, xt, yt, whole, n=3):
        self.ops, self.stream = ops, torch.cuda.Stream()
        self.workspace = torch.empty(ops.residual_norm_grad_workspace(n, d), dtype=torch.uint8, device="cuda")
        make = lambda t: torch.randn(n, d, device="cuda").to(TYPE[t])  # noqa: E731
        x, y, dx, dh, gate = make(xt), make(yt), make(xt), make(yt), make(yt)
        w = torch.randn(d, device="cuda")
        self.out = [torch.zeros(n, d, device="cuda", dtype=TYPE[t]) for t in (xt, yt, yt)] + [torch.zeros(d, device="cuda")]
        self.kept = (x, y, dx, dh, gate, w)
        p = lambda t: t.data_ptr()  # noqa: E731
        a = ops.ResidualNormGradArgs(x_new=p(x), dh=p(dh), w_pre=p(w), dx=p(self.out[0]), dw_pre=p(self.out[3]), workspace=p(self.workspace),
                                     workspace_bytes=self.workspace.numel(), n_rows=n, dim=d, ld_x_new=d, ld_dh=d, ld_dx=d, x_dtype=xt,
                                     y_dtype=yt, pre=1, res_scale=1.0, eps=1e-6)
        if whole:
            a.y, a.dx_new, a.dy, a.gate, a.dgate, a.gate_kind = p(y), p(dx), p(self.out[1]), p(gate), p(self.out[2]), 2
            a.ld_y = a.ld_dx_new = a.ld_dy = a.ld_gate = a.ld_dgate = d
        self.args = a

    def call(self):
        return self.ops.lib.adascale_residual_norm_grad(C.byref(self.args), self.stream.cuda_stream)


def child():
    sys.path.insert(0, ROOT)
    from paper_2007_05105_b200 import ops
    torch.manual_seed(5)
    for xt, yt in ((F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)):
        callers = [Caller(ops, d, xt, yt, whole=i % 3 != 1) for i, d in enumerate(WIDTHS)]
        torch.cuda.synchronize()
        start, status = threading.Barrier(len(callers)), [None] * len(callers)

        def go(i):
            start.wait()
            status[i] = callers[i].call()
        threads = [threading.Thread(target=go, args=(i,)) for i in range(len(callers))]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        assert status == [0] * len(callers), status
        torch.cuda.synchronize()
        first = [[t.clone() for t in c.out] for c in callers]
        torch.cuda.synchronize()
        assert [c.call() for c in callers] == [0] * len(callers)  # one after another: the widest is still possible
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for got, c in zip(first, callers) for a, b in zip(got, c.out))


def test_first_calls_from_several_threads():
    done = subprocess.run([sys.executable, os.path.abspath(__file__)], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]


if __name__ == "__main__":
    child()
