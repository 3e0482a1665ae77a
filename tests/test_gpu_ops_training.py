"""The clipping, position-bias and expert operators together: the example that trains with them, and calls from several streams and threads."""
import importlib.util
import math
import os
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

from paper_2007_05105_b200 import ops  # noqa: E402
from test_gpu_ops import BF16, DEV, gen, normal  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("experts_decoder", os.path.join(ROOT, "examples", "experts_decoder.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def whole_model(example, model, text, teacher):
    """Loss and gradients of the same model in 64 bits, by automatic differentiation alone."""

    class Plain(example.ExpertsDecoder):
        def __init__(self):
            self.__dict__.update(model.__dict__)

        def attention_weights(self, scores, bias, scale):
            n = scores.shape[-1]
            back = (torch.arange(n, device=DEV)[:, None] - torch.arange(n, device=DEV)).clamp(min=0)
            m, exact = bias.shape[0], bias.shape[0] // 2
            far = exact + torch.floor(torch.log(back.clamp(min=1).double() / exact) / math.log(self.max_distance / exact) * (m - exact) + 1e-9)
            z = scores * scale + bias[torch.where(back < exact, back, far.long().clamp(max=m - 1))].permute(2, 0, 1)
            return torch.softmax(z.masked_fill(torch.ones(n, n, dtype=torch.bool, device=DEV).triu(1), -math.inf), dim=-1)

        def products(self, x, w, offsets):
            o = offsets.tolist()
            return torch.cat([x[lo:hi] @ w[e].t() for e, (lo, hi) in enumerate(zip(o, o[1:]))])

    plain = Plain()
    p = {n: w.double().detach().requires_grad_() for n, w in model.by.items()}
    rms = lambda v, w: v / torch.sqrt(v.pow(2).mean(-1, keepdim=True) + model.EPS) * w  # noqa: E731
    tok, label = text[:, :-1], text[:, 1:]
    x = torch.nn.functional.embedding(tok, p["table"]) * model.scale
    h = rms(x, p["first"])
    for i in range(model.layers):
        y = plain.block(i, h, p["bias"], *(p["%s%d" % (n, i)] for n in model.BLOCK))
        x = x + model.res_scale * p["gate%d" % i] * rms(y, p["post%d" % i])
        h = rms(x, p["pre%d" % i])
    z = (h @ p["table"].t()).reshape(-1, model.vocab)
    prev, T = tok.reshape(-1), model.T
    log_q = torch.log_softmax(teacher.logits[prev].double() / T, dim=1)
    log_p = torch.log_softmax(z / T, dim=1).gather(1, teacher.ids[prev].long())
    loss = model.ALPHA * T * T * (log_q.exp() * (log_q - log_p)).sum(1) + \
        model.BETA * torch.nn.functional.cross_entropy(z, label.reshape(-1), reduction="none")
    loss = loss.mean()
    return loss, dict(zip(p, torch.autograd.grad(loss, list(p.values()))))


@pytest.mark.parametrize("share", [0.25, 4.0])
def test_gradients_of_a_microbatch(example, share):
    """All gradients together, clipped to a share of their norm and not.  The experts' products take bf16 operands: each operand is off by
    2^-9 of itself at most (half of 2^-8), two products forward and two backward have eight of them in a row and as many blocks as there
    are hand that on, so that 2 x 8 x 2^-9 = 0.03 of a gradient's norm covers it; the rest is in 32 bits.  A gradient that is
    small beside the others is off by that share of what it is a difference of, so the whole is compared, and each one roughly."""
    torch.backends.cuda.matmul.allow_tf32 = False
    teacher = example.Teacher(512, 8, "cuda", 3)
    model = example.ExpertsDecoder(vocab=512, d=96, layers=2, heads=3, experts=5, seed=4)
    text = teacher.text(4, 40)
    want, grads = whole_model(example, model, text, teacher)
    whole = math.sqrt(sum(float(g.square().sum()) for g in grads.values()))
    slots, = example.gradient_rows(model.params, 1, torch.float32)
    with torch.no_grad():
        loss, norm = model.microbatch(text, teacher, slots, share * whole)
    assert abs(float(loss) - float(want)) <= 0.01 * abs(float(want))
    assert abs(float(norm) - whole) <= 0.03 * whole
    c = min(1.0, share)
    off = math.sqrt(sum(float((got.double() - c * grads[name]).square().sum()) for name, got in zip(model.names, slots)))
    assert off <= (0.03 + 0.03) * c * whole  # the norm's error is in the factor
    for name, got in zip(model.names, slots):
        assert float((got.double() - c * grads[name]).norm()) <= 0.2 * c * float(grads[name].norm()), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_training_runs(example, dtype):
    losses, norms, st = example.train(steps=30, S=3, batch=4, length=16, grad_dtype=dtype, vocab=256, every=29, log=None)
    assert all(math.isfinite(v) for v in losses + norms)
    assert st.t == 30 and st.skipped == 0 and 1.0 <= st.r <= 3.0


def work(seed):
    """One of each call, on tensors of its own; what they returned."""
    g = gen(seed)
    x, w, dy = normal(g, 700, 128, dtype=BF16), normal(g, 5, 264, 128, dtype=BF16), normal(g, 700, 264, dtype=BF16)
    offsets = torch.tensor([0, 100, 100, 420, 650, 700], device=DEV)
    scores, table = normal(g, 2, 4, 50, 96, dtype=BF16), normal(g, 32, 4)
    grads = [normal(g, 3001 + k) for k in range(20)]

    def calls():
        y = ops.expert_matmul(x, w, offsets)
        e = ops.expert_matmul_grad(dy, offsets, x=x, w=w)
        probs = ops.position_softmax(scores, table, causal=True)
        s = ops.position_softmax_grad(probs, scores, 32, causal=True)
        out = [torch.empty_like(t) for t in grads]
        norm = ops.clip_grads(grads, 3.0, out=out)
        return [y, e.dx, e.dw, probs, s.dscores, s.dtable, norm] + out
    return calls


def test_several_streams_and_threads_at_once():
    """Calls that are in flight together, from threads of their own, give the bits that each gives alone."""
    jobs = [work(k) for k in range(4)]
    want = [job() for job in jobs]
    torch.cuda.synchronize()
    got, errors = [None] * 4, []

    def run(k):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    got[k] = jobs[k]()
                torch.cuda.current_stream().synchronize()
        except Exception as e:  # noqa: BLE001
            errors.append(e)
    threads = [threading.Thread(target=run, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors
    for a, b in zip(got, want):
        assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_two_graphs_replayed_together():
    """Captured calls have workspaces of their own: two graphs at once, and a third call between them."""
    jobs = [work(10), work(11)]
    want = [job() for job in jobs]
    graphs, got = [], []
    for job in jobs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got.append(job())
        graphs.append(graph)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(10):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        jobs[0]()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_on_a_stream_behind_others():
    """Each call on a side stream right behind what makes its inputs, and what reads its results right behind it."""
    stream = torch.cuda.Stream()
    job = work(20)
    want = job()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        for _ in range(10):
            got = [t.clone() for t in job()]
    stream.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(got, want))


def test_no_attachment_to_autograd():
    x = normal(gen(1), 40, 64, dtype=BF16).requires_grad_()
    w = normal(gen(2), 1, 32, 64, dtype=BF16).requires_grad_()
    y = ops.expert_matmul(x, w, torch.tensor([0, 40], device=DEV))
    s = normal(gen(3), 1, 2, 4, 8).requires_grad_()
    p = ops.position_softmax(s, normal(gen(4), 32, 2).requires_grad_())
    assert not y.requires_grad and not p.requires_grad and not ops.grad_norm([s]).requires_grad
