"""The norm over many gradients and clipping by it, against 64-bit sums.

Tolerances, with u = 2^-24: a thread adds at most 32 squares in 32 bits before it goes on in 64, so the sum of squares is off by at most
33 u of itself (all terms are positive), its root by half of that, and the norm's own rounding is u.  The factor c is off by as
much and one rounding, its product with an element by another u, the stored result by u or 2^-8 (bfloat16).
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

from paper_2007_05105_b200 import binding as B  # noqa: E402
from paper_2007_05105_b200 import ops  # noqa: E402
from test_gpu_ops import BF16, DEV, F32, U, check, gen, normal, rounding  # noqa: E402

NORM = 18 * U


def norm_of(grads):
    return math.sqrt(math.fsum(float(g.double().square().sum()) for g in grads))


def check_all(grads, out, norm, max_norm, eps=1e-6):
    want = norm_of(grads)
    assert norm.dtype == F32 and norm.dim() == 0
    assert abs(float(norm) - want) <= NORM * want
    c = min(1.0, max_norm / (want + eps)) if want + eps else 1.0
    for g, o in zip(grads, out):
        expect = c * g.double()
        check(o, expect, expect.abs() * (NORM + 2 * U + rounding(o.dtype) * 1.01) + 2.0 ** -149 + (2.0 ** -134 if o.dtype == BF16 else 0), "clipped")


SIZES = [[1], [0, 5, 0], [7, 4096, 4097, 1], [100000], [33] * 70, [1000, 3] * 300, [2_000_003, 17, 1_000_000], [64] * 2500]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "%dx%d" % (len(s), s[0]))
@pytest.mark.parametrize("g_t,o_t", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
def test_norm_and_clipping(sizes, g_t, o_t):
    g = gen(len(sizes))
    grads = [normal(g, n, dtype=g_t, std=3.0) for n in sizes]
    norm = ops.grad_norm(grads)
    want = norm_of(grads)
    assert abs(float(norm) - want) <= NORM * want
    for share in (0.3, 1.5):  # clipped, and not
        out = [torch.full((n,), 9.0, dtype=o_t, device=DEV) for n in sizes]
        got = ops.clip_grads(grads, share * want, out=out)
        assert torch.equal(got, norm)
        check_all(grads, out, got, float(torch.tensor(share * want, dtype=F32)))
        if g_t == o_t:
            place = [t.clone() for t in grads]
            assert torch.equal(ops.clip_grads(place, share * want), norm)
            assert all(torch.equal(a, b) for a, b in zip(place, out))


def test_mixed_types_alignments_and_orders():
    """Slots anywhere in a row, gradients of either type, channels last, slices; what lies between the slots is left alone."""
    g = gen(1)
    whole = normal(g, 40000)
    grads = [whole[3:5003].view(50, 100), whole[6001:9002], normal(g, 8, 16, 5, 5).to(memory_format=torch.channels_last), normal(g, 333, dtype=BF16)[1:],
             normal(g, 10, dtype=BF16), normal(g, 1, 70).t(), normal(g, 3, 4).t()]
    for o_t in (F32, BF16):
        row = torch.full((30000,), 5.0, dtype=o_t, device=DEV)
        used = torch.zeros(30000, dtype=torch.bool, device=DEV)
        out, at = [], 1
        for t in grads:
            flat = row[at:at + t.numel()]
            used[at:at + t.numel()] = True
            out.append(flat.as_strided(t.shape, t.stride(), flat.storage_offset()))
            at += t.numel() + 13
        norm = ops.clip_grads(grads, 2.0, out=out)
        check_all(grads, out, norm, 2.0)
        assert bool((row[~used] == 5.0).all())


def test_in_place_is_left_alone_where_nothing_is_clipped():
    t = normal(gen(2), 5000)
    before, version = t.clone(), t._version
    norm = ops.clip_grads([t], 1e6)
    assert torch.equal(t, before) and t._version > version and float(norm) > 60


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [1e-42, 3e-30, 1e-20, 1e18, 1e25, 1e37])
def test_squares_outside_the_range(size, dtype):
    """Elements whose squares leave 32 bits at either end, beside ordinary sizes of lists."""
    base = torch.linspace(0.5, 1.0, 70001, device=DEV, dtype=torch.float64)
    grads = [(size * base).to(dtype), (size * base[:9]).to(dtype)]
    if not any(bool(t.any()) for t in grads):
        pytest.skip("all round to zero")
    want = norm_of(grads)
    got = float(ops.grad_norm(grads))
    if want > torch.finfo(F32).max:  # 1e37 * 0.76 * sqrt(70010) = 2e39: infinite as a 32-bit number, and a quarter of it no max_norm
        assert got == math.inf
        with pytest.raises(B.AdaScaleError):
            ops.clip_grads(grads, want / 4, eps=0.0)
        return
    assert abs(got - want) <= NORM * want + 2.0 ** -149
    out = [torch.empty_like(t) for t in grads]
    norm = ops.clip_grads(grads, want / 4, out=out, eps=0.0)
    check_all(grads, out, norm, float(torch.tensor(want / 4, dtype=F32)), eps=0.0)


def test_norm_beyond_the_range():
    t = torch.full((1000,), 3e38, device=DEV)
    out = torch.empty_like(t)
    norm = ops.clip_grads([t], 10.0, out=[out])  # the norm itself does not fit, the factor is right all the same
    assert float(norm) == math.inf
    want = torch.full((1000,), 10.0 / math.sqrt(1000), dtype=torch.float64, device=DEV)
    check(out, want, want * (NORM + 3 * U), "clipped")


def test_zeros_nan_and_infinities():
    zero = torch.zeros(5000, device=DEV)
    out = torch.ones(5000, device=DEV)
    assert float(ops.clip_grads([zero], 1.0, out=[out])) == 0.0 and not out.any()
    assert float(ops.clip_grads([zero], 0.0, out=[out], eps=0.0)) == 0.0 and not out.any()
    grads = [normal(gen(3), 4000), normal(gen(4), 70, dtype=BF16)]
    out = [torch.ones_like(t) for t in grads]
    grads[0][1234] = float("nan")
    assert math.isnan(float(ops.clip_grads(grads, 1.0, out=out))) and all(bool(torch.isnan(o).all()) for o in out)
    grads[0][1234] = -math.inf
    assert float(ops.clip_grads(grads, 1.0, out=out)) == math.inf
    assert bool(torch.isnan(out[0][1234])) and not out[1].any() and not torch.cat([out[0][:1234], out[0][1235:]]).any()
    assert float(ops.grad_norm([torch.zeros(0, device=DEV)])) == 0.0


def test_long_tensors():
    """More than 2^31 elements, and the same bits from run to run."""
    t = torch.zeros((1 << 31) + 4099, dtype=BF16, device=DEV)
    t[-1], t[0], t[1 << 31] = 3.0, 4.0, 12.0
    assert float(ops.grad_norm([t])) == 13.0
    ops.clip_grads([t], 6.5, eps=0.0)
    assert (float(t[-1]), float(t[0]), float(t[1 << 31]), float(t[5])) == (1.5, 2.0, 6.0, 0.0)
    del t
    grads = [normal(gen(k), 300007) for k in range(5)]
    assert len({float(ops.grad_norm(grads)) for _ in range(5)}) == 1


def test_captured_and_on_a_stream():
    grads = [normal(gen(k), 3000 + k) for k in range(80)]
    out = [torch.empty(t.shape, dtype=BF16, device=DEV) for t in grads]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    other = ops.grad_norm(grads, stream=stream)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = ops.clip_grads(grads, 5.0, out=out)
    graph.replay()
    assert torch.equal(norm, other)
    for t in grads:
        t.mul_(0.5)
    graph.replay()
    check_all(grads, out, norm, 5.0)


def test_steps_directly_behind():
    """Rows that are clipped right before steps that read ahead: the same parameters as with a synchronisation before each."""
    sizes, S, steps = [1 << 19, 4099, 1 << 20], 2, 8

    def train(synchronise):
        g = gen(7)
        leaves = [[normal(g, n) for n in sizes] for _ in range(S * steps)]
        rows = [[torch.zeros(n, device=DEV) for n in sizes] for _ in range(S)]
        w, v = [torch.ones(n, device=DEV) for n in sizes], [torch.zeros(n, device=DEV) for n in sizes]
        ada = B.AdaScale(sizes, S, "f32", momentum=0.9, flags=B.FLAG_GRADS_READY)
        g_p, w_p, v_p, sched = B.pointer_array(rows), B.pointer_array(w), B.pointer_array(v), B.make_schedule("const", eta0=0.05)
        for k in range(steps):
            for i in range(S):
                ops.clip_grads(leaves[k * S + i], 1.0 + i, out=rows[i])
            if synchronise:
                torch.cuda.synchronize()
            ada.step(g_p, w_p, v_p, sched)
        st = ada.get_gain_tau(True)
        ada.close()
        return w, st

    (a, s), (b, t) = train(False), train(True)
    assert all(torch.equal(x, y) for x, y in zip(a, b)) and s.r == t.r and s.tau == t.tau


def test_refusals():
    t = torch.ones(10, device=DEV)
    for bad in [lambda: ops.grad_norm([]), lambda: ops.grad_norm([t.half()]), lambda: ops.grad_norm([t.cpu()]), lambda: ops.grad_norm([t, t.cpu()]),
                lambda: ops.grad_norm([t[::2]]), lambda: ops.grad_norm([t[:1].expand(5)]), lambda: ops.clip_grads([t], 1.0, out=[]),
                lambda: ops.clip_grads([t], 1.0, out=[t[:5]]), lambda: ops.clip_grads([t], 1.0, out=[t.half()]),
                lambda: ops.clip_grads([t.view(2, 5)], 1.0, out=[t.view(5, 2).t()]), lambda: ops.clip_grads([t], 1.0, out=[t.cpu()])]:
        with pytest.raises(ValueError):
            bad()
    for bad in [lambda: ops.grad_norm([None]), lambda: ops.grad_norm(5), lambda: ops.clip_grads([t], None), lambda: ops.clip_grads([t], "x")]:
        with pytest.raises(TypeError):
            bad()
    for bad in [lambda: ops.clip_grads([t], math.nan), lambda: ops.clip_grads([t], -1.0), lambda: ops.clip_grads([t], 1.0, eps=math.inf),
                lambda: ops.clip_grads([t, t], 1.0), lambda: ops.clip_grads([t, t[5:]], 1.0, out=[torch.ones_like(t), t[:5]]),
                lambda: ops.clip_grads([t[:9]], 1.0, out=[t[1:]]),
                lambda: ops.grad_norm([t], workspace=torch.zeros(16, dtype=torch.uint8, device=DEV))]:
        with pytest.raises(B.AdaScaleError):
            bad()


def test_any_iterable_of_gradients():
    grads = [normal(gen(k), 700 + k) for k in range(5)]
    want, stream = ops.grad_norm(grads), torch.cuda.Stream()
    torch.cuda.synchronize()
    for how in (None, stream):
        assert torch.equal(ops.grad_norm(tuple(grads), stream=how), want) and torch.equal(ops.grad_norm((t for t in grads), stream=how), want)
        by_name = {str(k): t.clone() for k, t in enumerate(grads)}
        out = {k: torch.empty_like(t) for k, t in by_name.items()}
        assert torch.equal(ops.clip_grads(by_name.values(), 3.0, out=out.values(), stream=how), want)
        torch.cuda.synchronize()
        check_all(grads, list(out.values()), want, 3.0)


def test_as_many_tensors_as_there_may_be():
    t = torch.full((3,), 2.0, device=DEV)
    want = math.sqrt(12 * 65536)
    assert abs(float(ops.grad_norm([t] * 65536)) - want) <= NORM * want
    with pytest.raises(B.AdaScaleError, match="maximum"):
        ops.grad_norm([t] * 65537)
