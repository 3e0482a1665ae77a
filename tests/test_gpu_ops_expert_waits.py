"""What the experts' products do when a wait inside them runs out: the same source with waits that end at their first poll.

Nothing in it can fault or hang: the waits only end earlier, and those for copies and matrix instructions in flight keep their own bound.
"""
import ctypes as C
import os
import shutil
import subprocess

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

from paper_2007_05105_b200 import build, ops  # noqa: E402
from test_gpu_ops import BF16, DEV, F32, gen, normal  # noqa: E402
from test_gpu_ops_expert import offsets_of  # noqa: E402


@pytest.fixture(scope="module")
def hasty(tmp_path_factory):
    """The calls with waits of one poll, each of which may last 20 us: shorter than the sums below."""
    if shutil.which(build._nvcc()) is None:
        pytest.skip("needs nvcc")
    out = str(tmp_path_factory.mktemp("hasty") / "hasty.so")
    source = os.path.join(os.path.dirname(build.OPS_SOURCE), "ops_expert.cu")
    subprocess.check_call([build._nvcc()] + build.NVCC_FLAGS + ["-DADASCALE_EXPERT_POLLS=0u", "-o", out, source])
    lib = C.CDLL(out)
    for name, args in (("adascale_expert_matmul", ops.ExpertMatmulArgs), ("adascale_expert_matmul_grad", ops.ExpertMatmulGradArgs)):
        getattr(lib, name).argtypes = [C.POINTER(args), C.c_void_p]
    return lib


def call(function, args):
    assert function(C.byref(args), torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()


def code(dtype):
    return 0 if dtype == F32 else 1


def lost_or_right(got, want, what):
    lost = torch.isnan(got)
    assert bool(lost.any()), what + ": no wait ran out"
    assert torch.equal(torch.where(lost, 0.0, got), torch.where(lost, 0.0, want)), what


# three tiles a block and more; blocks in pairs, alone (fewer than 129 lanes; few rows an expert)
FORMS = [(4096, 4096, 4096, [2000, 0, 2029]), (120000, 128, 8192, [59000, 60000]), (160, 4096 * 5, 8192, [20] * 8)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,m,k,counts", FORMS, ids=str)
def test_products_whose_waits_run_out(hasty, n, m, k, counts, dtype):
    """Each result is NaN or right, rows of nobody are left alone, and the calls behind it are as ever."""
    g = gen(n)
    x, w, offsets = normal(g, n, k, dtype=BF16), normal(g, len(counts), m, k, dtype=BF16), offsets_of(counts)
    want = ops.expert_matmul(x, w, offsets, out=torch.full((n, m), 5.0, dtype=dtype, device=DEV))
    y = torch.full((n, m), 5.0, dtype=dtype, device=DEV)
    call(hasty.adascale_expert_matmul,
         ops.ExpertMatmulArgs(x=x.data_ptr(), w=w.data_ptr(), y=y.data_ptr(), offsets=offsets.data_ptr(), n_rows=n, n_experts=len(counts), in_dim=k,
                              out_dim=m, ld_x=k, ld_w=k, stride_w=m * k, ld_y=m, offset_type=0, y_dtype=code(dtype)))
    lost_or_right(y, want, "products")
    assert bool((y[sum(counts):] == 5.0).all())
    assert torch.equal(ops.expert_matmul(x, w, offsets, out_dtype=dtype)[:sum(counts)], want[:sum(counts)])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,m,k,counts", [(20000, 4096, 4096, [9984, 3, 9970]), (20000, 128, 4096 * 10, [9985, 9000])], ids=str)
def test_gradients_whose_waits_run_out(hasty, n, m, k, counts, dtype):
    g = gen(n)
    x, w, dy = normal(g, n, k, dtype=BF16), normal(g, len(counts), m, k, dtype=BF16), normal(g, n, m, dtype=BF16)
    offsets = offsets_of(counts, ids=torch.int64)
    want = ops.expert_matmul_grad(dy, offsets, x=x, w=w, dx=torch.full((n, k), 5.0, dtype=dtype, device=DEV), wgrad_dtype=dtype)
    dx, dw = torch.full((n, k), 5.0, dtype=dtype, device=DEV), torch.empty(len(counts), m, k, dtype=dtype, device=DEV)
    call(hasty.adascale_expert_matmul_grad,
         ops.ExpertMatmulGradArgs(dy=dy.data_ptr(), x=x.data_ptr(), w=w.data_ptr(), dx=dx.data_ptr(), dw=dw.data_ptr(), offsets=offsets.data_ptr(),
                                  n_rows=n, n_experts=len(counts), in_dim=k, out_dim=m, ld_dy=m, ld_x=k, ld_w=k, stride_w=m * k, ld_dx=k, ld_dw=k,
                                  stride_dw=m * k, offset_type=1, dx_dtype=code(dtype), dw_dtype=code(dtype)))
    lost_or_right(dw, want.dw, "dw")
    lost = torch.isnan(dx)
    assert torch.equal(torch.where(lost, 0.0, dx), torch.where(lost, 0.0, want.dx))
    assert bool((dx[sum(counts):] == 5.0).all())
    again = ops.expert_matmul_grad(dy, offsets, x=x, w=w, dx_dtype=dtype, wgrad_dtype=dtype)
    assert torch.equal(again.dx[:sum(counts)], want.dx[:sum(counts)]) and torch.equal(again.dw, want.dw)
