"""The example that trains with all operators: its gradients against those of the same model differentiated as a whole, and its loss."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("distill_decoder", os.path.join(ROOT, "examples", "distill_decoder.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def whole_model(model, text, teacher):
    """Loss and gradients of the same model in 64 bits, by automatic differentiation alone."""
    p = {n: w.double().detach().requires_grad_() for n, w in model.by.items()}
    rms = lambda v, w: v / torch.sqrt(v.pow(2).mean(-1, keepdim=True) + model.EPS) * w  # noqa: E731
    tok, label = text[:, :-1], text[:, 1:]
    x = torch.nn.functional.embedding(tok, p["table"]) * model.scale
    h = rms(x, p["first"])
    for i in range(model.layers):
        y = model.block(i, h, *(p["%s%d" % (n, i)] for n in ("qkv", "mix", "up", "down")))
        x = x + model.res_scale * p["gate%d" % i] * rms(y, p["post%d" % i])
        h = rms(x, p["pre%d" % i])
    z = (h @ p["table"].t()).reshape(-1, model.vocab)
    prev, T = tok.reshape(-1), model.T
    log_q = torch.log_softmax(teacher.logits[prev].double() / T, dim=1)
    log_p = torch.log_softmax(z / T, dim=1).gather(1, teacher.ids[prev].long())
    loss = model.ALPHA * T * T * (log_q.exp() * (log_q - log_p)).sum(1) + \
        model.BETA * torch.nn.functional.cross_entropy(z, label.reshape(-1), reduction="none")
    loss = loss.mean()
    return loss, torch.autograd.grad(loss, list(p.values()))


def test_gradients_of_a_microbatch(example):
    """Norm of the difference below 1e-4 of the gradient's: the matrix products are torch's in 32 bits (2^-24 a product, sums of up to
    1024 terms over a few layers: some 1e-6), the operators' own error is below that."""
    torch.backends.cuda.matmul.allow_tf32 = False
    teacher = example.Teacher(512, 8, "cuda", 3)
    model = example.Decoder(vocab=512, d=96, layers=3, heads=3, seed=4)
    text = teacher.text(4, 17)
    slots, = example.gradient_rows(model.params, 1, torch.float32)
    with torch.no_grad():
        loss = model.microbatch(text, teacher, slots)
    want, grads = whole_model(model, text, teacher)
    assert abs(float(loss) - float(want)) <= 1e-5 * abs(float(want))
    for name, got, g in zip(model.names, slots, grads):
        assert float((got.double() - g).norm()) <= 1e-4 * float(g.norm()), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_training_lowers_the_loss(example, dtype):
    losses, st = example.train(steps=80, S=3, batch=4, length=16, grad_dtype=dtype, vocab=256, every=79, log=None)
    assert math.isfinite(losses[-1]) and losses[-1] < 0.7 * losses[0]
    assert st.t == 80 and st.skipped == 0 and 1.0 <= st.r <= 3.0
