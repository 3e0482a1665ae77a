"""Embedding gradients directly before AdaScale steps that read their rows ahead of the kernel before them.

ADASCALE_FLAG_GRADS_READY wants the last kernel on the stream not to trigger programmatic dependent launches before its last
gradient store.  A few tokens need no kernel that joins pieces, none at all only the one that writes zeros.  The rows
change from step to step, and the parameters are bitwise those of the same steps with a synchronisation before each."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

from paper_2007_05105_b200 import binding as B  # noqa: E402
from paper_2007_05105_b200 import ops  # noqa: E402

DEV = torch.device("cuda:0")
VOCAB, WIDTH, S, STEPS = 7, 1 << 19, 2, 12


def _steps(tokens, dout, accumulate, synchronise):
    """Parameters after STEPS steps of which step k's rows come from tokens[k], dout[k]."""
    n = VOCAB * WIDTH
    rows = [torch.full((VOCAB, WIDTH), 0.01 * (i + 1), device=DEV) for i in range(S)]
    w, v = torch.linspace(-1.0, 1.0, n, device=DEV), torch.zeros(n, device=DEV)
    ada = B.AdaScale([n], S, "f32", momentum=0.9, flags=B.FLAG_GRADS_READY)
    sched = B.make_schedule("const", eta0=0.05)
    g, p, m = B.pointer_array([[r] for r in rows]), B.pointer_array([w]), B.pointer_array([v])
    room = torch.empty(ops.embed_grad_workspace(8, WIDTH), dtype=torch.uint8, device=DEV)
    for k in range(STEPS):
        for i, row in enumerate(rows):
            ops.embed_grad(tokens[k][i], dout[k][:len(tokens[k][i])], row, scale=1.0 + i, accumulate=accumulate, workspace=room)
        if synchronise:
            torch.cuda.synchronize()
        ada.step(g, p, m, sched)
    st = ada.get_gain_tau(True)
    torch.cuda.synchronize()
    ada.close()
    return w, v, st


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("n", [8, 3, 0])
def test_steps_behind_an_embedding_gradient_without_a_join(n, accumulate):
    g = torch.Generator(device=DEV)
    g.manual_seed(n)
    dout = [torch.empty(8, WIDTH, device=DEV).normal_(0.0, 1.0, generator=g) for _ in range(STEPS)]
    # without tokens every other step, so that zeros and sums follow each other
    tokens = [[torch.randint(0, VOCAB, (n if n or k % 2 else 8,), device=DEV, generator=g) for _ in range(S)] for k in range(STEPS)]
    a, b = _steps(tokens, dout, accumulate, False), _steps(tokens, dout, accumulate, True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert a[2].r == b[2].r and a[2].tau == b[2].tau and a[2].t == STEPS
