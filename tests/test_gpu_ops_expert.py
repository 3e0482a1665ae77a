"""Products with experts' weights over ragged groups of rows, and their gradients, against 64-bit products.

Tolerances: operands are bf16, so every product of two is exact in 32 bits.  The tensor cores add in 32 bits, each addition off
by at most one unit in the last place (2u = 2^-23, as they may cut instead of round) of what is being added up, m summands by
2 m u at most of the sum of the terms' magnitudes; errors of that many additions of either sign stay far below, so that bound is
never near.  Storing adds u (float32) or 2^-8 (bfloat16) of the value, adding to what a gradient holds another u.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

from paper_2007_05105_b200 import ops  # noqa: E402
from paper_2007_05105_b200.binding import AdaScaleError  # noqa: E402
from test_gpu_ops import BF16, DEV, F32, U, check, gen, normal, rounding, strided  # noqa: E402


def offsets_of(counts, first=0, ids=torch.int32):
    return torch.tensor([first] + counts, device=DEV).cumsum(0).to(ids)


def padded(t, pad):
    """The same values with rows 8 * pad elements further apart."""
    if not pad:
        return t
    wide = torch.full((*t.shape[:-1], (t.shape[-1] + 7) // 8 * 8 + 8 * pad), float("nan"), dtype=t.dtype, device=DEV)
    wide[..., :t.shape[-1]] = t
    return wide[..., :t.shape[-1]]


def aligned(t):
    """The same values in rows that start on 16-byte boundaries."""
    return t if t.shape[-1] % 8 == 0 else padded(t, 1)


def groups(offsets):
    o = offsets.tolist()
    return [(e, o[e], o[e + 1]) for e in range(len(o) - 1)]


def forward_check(x, w, offsets, y, before, what):
    want, mag = before.double(), torch.zeros(y.shape, dtype=torch.float64, device=DEV)
    for e, lo, hi in groups(offsets):
        want[lo:hi] = x[lo:hi].double() @ w[e].double().t()
        mag[lo:hi] = x[lo:hi].double().abs() @ w[e].double().abs().t()
    check(y, want, 2 * x.shape[1] * U * mag + rounding(y.dtype) * want.abs() * 1.01, what)


SHAPES = [  # rows of each expert, rows before the first and behind the last, in, out
    ([1], 0, 0, 8, 8),
    ([5], 0, 0, 64, 128),
    ([3, 0, 17, 1], 2, 5, 72, 40),
    ([0, 0, 33, 0], 0, 0, 264, 136),
    ([130, 7, 0, 255, 64], 0, 31, 136, 200),
    ([257, 512, 1, 300], 9, 0, 512, 264),
    ([700, 900], 0, 77, 1032, 520),
    ([1] * 70 + [0] * 9 + [2] * 50, 0, 0, 128, 64),
    ([40, 41], 0, 0, 13, 9),
    ([600, 100], 0, 3, 77, 301),
]


@pytest.mark.parametrize("out_t", [BF16, F32])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_products(shape, out_t):
    counts, first, tail, k, m = shape
    n = first + sum(counts) + tail
    g = gen(n + k)
    x, w = aligned(normal(g, n, k, dtype=BF16)), aligned(normal(g, len(counts), m, k, dtype=BF16))
    offsets = offsets_of(counts, first)
    before = normal(g, n, m, dtype=out_t)
    y, intact = strided(before, 3, 1)
    assert ops.expert_matmul(x, w, offsets, out=y) is y
    forward_check(x, w, offsets, y, before, "products")
    intact()


@pytest.mark.parametrize("dx_t,dw_t,accumulate", [(BF16, F32, False), (F32, BF16, False), (BF16, F32, True), (F32, BF16, True)])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_gradients(shape, dx_t, dw_t, accumulate):
    counts, first, tail, k, m = shape
    n = first + sum(counts) + tail
    g = gen(n + k + 1)
    x, w = aligned(normal(g, n, k, dtype=BF16)), aligned(normal(g, len(counts), m, k, dtype=BF16))
    dy = aligned(normal(g, n, m, dtype=BF16))
    x[:first], dy[:first] = float("nan"), float("inf")  # what no expert has is not used
    x[n - tail:], dy[n - tail:] = float("nan"), float("nan")
    offsets = offsets_of(counts, first, torch.int64)
    dx0, dw0 = normal(g, n, k, dtype=dx_t), normal(g, len(counts), m, k, dtype=dw_t)
    dx, dx_intact = strided(dx0, 1, 3)
    flat, dw_intact = strided(dw0.view(1, -1), 0, 64)
    dw = flat.view(len(counts), m, k)
    got = ops.expert_matmul_grad(dy, offsets, x=x, w=w, dx=dx, dw=dw, accumulate=accumulate)
    assert got.dx is dx and got.dw is dw
    want, mag = dx0.double(), torch.zeros(n, k, dtype=torch.float64, device=DEV)
    for e, lo, hi in groups(offsets):
        want[lo:hi] = dy[lo:hi].double() @ w[e].double()
        mag[lo:hi] = dy[lo:hi].double().abs() @ w[e].double().abs()
        part = dy[lo:hi].double().t() @ x[lo:hi].double()
        terms = dy[lo:hi].double().abs().t() @ x[lo:hi].double().abs()
        whole = part + dw0[e].double() if accumulate else part
        check(dw[e], whole, 2 * max(hi - lo, 1) * U * terms + U * whole.abs() + rounding(dw_t) * whole.abs() * 1.01, "dw of %d" % e)
    check(dx, want, 2 * m * U * mag + rounding(dx_t) * want.abs() * 1.01, "dx")
    dx_intact()
    dw_intact()


def test_against_differences():
    """The gradients of a weighted sum of results against that sum's own differences: exact steps, so that only the sum's
    rounding is between them."""
    counts, k, m = [3, 0, 20], 24, 16
    g = gen(5)
    n = sum(counts)
    whole = lambda *s: torch.randint(-4, 5, s, device=DEV, generator=g).to(BF16)  # noqa: E731
    x, w, dy, offsets = whole(n, k), whole(3, m, k), whole(n, m), offsets_of(counts)
    loss = lambda x, w: float((ops.expert_matmul(x, w, offsets, out_dtype=F32).double() * dy.double()).sum())  # noqa: E731
    got = ops.expert_matmul_grad(dy, offsets, x=x, w=w, dx_dtype=F32)
    for at in [(0, 0), (2, 23), (3, 7), (22, 11)]:  # whole numbers below 2^24: no rounding at all
        x2 = x.clone()
        x2[at] += 1
        assert loss(x2, w) - loss(x, w) == float(got.dx[at])
    for at in [(0, 0, 0), (1, 3, 3), (2, 15, 23)]:
        w2 = w.clone()
        w2[at] += 1
        assert loss(x, w2) - loss(x, w) == float(got.dw[at])


@pytest.mark.parametrize("rows", [1, 2, 16, 31, 32, 33, 64, 127, 128, 129, 255, 256, 257, 400])
def test_every_width_of_a_tile(rows):
    g = gen(rows)
    x, w, dy = normal(g, rows + 3, 192, dtype=BF16), normal(g, 2, 130, 192, dtype=BF16), normal(g, rows + 3, 130, dtype=BF16)
    dy = aligned(dy)
    offsets = offsets_of([rows, 2])
    before = torch.full((rows + 3, 130), 7.0, device=DEV)
    y = ops.expert_matmul(x, w, offsets, out=before.clone())
    forward_check(x, w, offsets, y, before, "width")
    got = ops.expert_matmul_grad(dy, offsets, x=x, w=w)
    for e, lo, hi in groups(offsets):
        part = dy[lo:hi].double().t() @ x[lo:hi].double()
        check(got.dw[e], part, 2 * rows * U * (dy[lo:hi].double().abs().t() @ x[lo:hi].double().abs()) + U * part.abs(), "dw")


def test_nan_stays_in_its_expert():
    """A NaN of one expert's rows is in nobody else's results, also where both are in one tile."""
    g = gen(2)
    x, w, dy = normal(g, 100, 64, dtype=BF16), normal(g, 3, 64, 64, dtype=BF16), normal(g, 100, 64, dtype=BF16)
    offsets = offsets_of([30, 37, 33])
    x[40], dy[50], w[1, 3, 3] = float("nan"), float("inf"), float("nan")
    y = ops.expert_matmul(x, w, offsets)
    got = ops.expert_matmul_grad(dy, offsets, x=x, w=w)
    for e, lo, hi in groups(offsets):
        bad = e == 1
        assert bool(torch.isnan(y[lo:hi]).any()) == bad and bool(torch.isnan(got.dx[lo:hi]).any()) == bad
        assert bool(torch.isnan(got.dw[e]).any()) == bad
    assert not torch.isnan(y[30:67, :3]).any(dim=1)[:10].any()  # in its expert: only the row, and the output it meets


def test_offsets_out_of_order_or_range():
    """Clamped to the rows, and never below an earlier one."""
    g = gen(3)
    x, w = normal(g, 50, 32, dtype=BF16), normal(g, 5, 24, 32, dtype=BF16)
    for ids in (torch.int32, torch.int64):
        given = torch.tensor([-7, 20, 10, 30, 1 << 30, 45], dtype=ids, device=DEV)
        meant = torch.tensor([0, 20, 20, 30, 50, 50], device=DEV)
        before = normal(g, 50, 24)
        y = ops.expert_matmul(x, w, given, out=before.clone())
        forward_check(x, w, meant, y, before, "offsets")
    wide = torch.tensor([0, 1 << 40, -(1 << 40), 3, 4, 5], device=DEV)
    y = ops.expert_matmul(x, w, wide, out_dtype=F32)
    forward_check(x, w, torch.tensor([0, 50, 50, 50, 50, 50], device=DEV), y, y * 0, "offsets")


def test_no_rows():
    w = normal(gen(0), 3, 16, 8, dtype=BF16)
    x, offsets = torch.empty(0, 8, dtype=BF16, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV)
    assert ops.expert_matmul(x, w, offsets).shape == (0, 16)
    dw = torch.full((3, 16, 8), 5.0, device=DEV)
    got = ops.expert_matmul_grad(x.new_empty(0, 16), offsets, x=x, w=w, dw=dw, accumulate=True)
    assert got.dx.shape == (0, 8) and bool((dw == 5.0).all())
    ops.expert_matmul_grad(x.new_empty(0, 16), offsets, x=x, dw=dw)
    assert not dw.any()
    x = normal(gen(0), 9, 8, dtype=BF16)  # rows, but nobody's
    dw.fill_(5.0)
    ops.expert_matmul_grad(normal(gen(0), 9, 16, dtype=BF16), offsets, x=x, dw=dw)
    assert not dw.any()


def test_strides_and_parts():
    """Rows and experts with room between them, slices of wider matrices, and either gradient alone; the same bits."""
    g = gen(11)
    x, w, dy = normal(g, 333, 136, dtype=BF16), normal(g, 4, 72, 136, dtype=BF16), normal(g, 333, 72, dtype=BF16)
    offsets = offsets_of([100, 200, 0, 33])
    y = ops.expert_matmul(x, w, offsets)
    assert torch.equal(ops.expert_matmul(padded(x, 2), padded(w, 3), offsets), y)
    room = torch.zeros(4, 100, 136, dtype=BF16, device=DEV)
    room[:, :72] = w
    assert torch.equal(ops.expert_matmul(x, room[:, :72], offsets), y)
    assert torch.equal(ops.expert_matmul(x, w, offsets, out_dtype=F32).to(BF16), y)
    both = ops.expert_matmul_grad(dy, offsets, x=x, w=w)
    only_dx, only_dw = ops.expert_matmul_grad(padded(dy, 1), offsets, w=padded(w, 1)), ops.expert_matmul_grad(dy, offsets, x=padded(x, 1))
    assert only_dx.dw is None and only_dw.dx is None
    assert torch.equal(only_dx.dx, both.dx) and torch.equal(only_dw.dw, both.dw)
    assert both.dx.dtype == BF16 and both.dw.dtype == F32
    slot = torch.zeros(1 + 4 * 72 * 136, dtype=BF16, device=DEV)
    ops.expert_matmul_grad(dy, offsets, x=x, dw=slot[1:].view(4, 72, 136))
    assert torch.equal(slot[1:].view(4, 72, 136), both.dw.to(BF16)) and float(slot[0]) == 0.0
    again = ops.expert_matmul_grad(dy, offsets, x=x, w=w)
    assert torch.equal(again.dx, both.dx) and torch.equal(again.dw, both.dw)


def test_results_far_behind_the_first():
    """More than 2^31 elements of results."""
    n, m = 70000, 32768
    x, w = torch.ones(n, 8, dtype=BF16, device=DEV), torch.ones(1, m, 8, dtype=BF16, device=DEV)
    x[-1] = 2.0
    y = ops.expert_matmul(x, w, offsets_of([n]))
    assert bool((y[-1] == 16.0).all()) and bool((y[-2] == 8.0).all()) and bool((y[0] == 8.0).all())
    assert bool((y[:, -1] == y[:, 0]).all())


def test_captured_and_on_a_stream():
    g = gen(8)
    x, w, dy = normal(g, 300, 256, dtype=BF16), normal(g, 4, 128, 256, dtype=BF16), normal(g, 300, 128, dtype=BF16)
    offsets = offsets_of([100, 0, 150, 50])
    want, wgrad = ops.expert_matmul(x, w, offsets), ops.expert_matmul_grad(dy, offsets, x=x, w=w)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    y = ops.expert_matmul(x, w, offsets, stream=stream)
    stream.synchronize()
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = ops.expert_matmul(x, w, offsets)
        got = ops.expert_matmul_grad(dy, offsets, x=x, w=w)
    for counts in ([100, 0, 150, 50], [7, 100, 20, 173]):  # the rows may be divided anew between replays
        offsets.copy_(offsets_of(counts))
        graph.replay()
        assert torch.equal(y, ops.expert_matmul(x, w, offsets))
        again = ops.expert_matmul_grad(dy, offsets, x=x, w=w)
        assert torch.equal(got.dx, again.dx) and torch.equal(got.dw, again.dw)


def test_refusals():
    x, w, dy = (torch.zeros(*s, dtype=BF16, device=DEV) for s in ((10, 16), (2, 24, 16), (10, 24)))
    offsets = offsets_of([5, 5])
    for bad in [lambda: ops.expert_matmul(x.float(), w, offsets), lambda: ops.expert_matmul(x, w.float(), offsets),
                lambda: ops.expert_matmul(x, w[:, :, :8], offsets), lambda: ops.expert_matmul(x, w, offsets[:2]),
                lambda: ops.expert_matmul(x, w, offsets.float()), lambda: ops.expert_matmul(x, w, offsets.cpu()),
                lambda: ops.expert_matmul(x.cpu(), w, offsets), lambda: ops.expert_matmul(x, w.transpose(1, 2), offsets),
                lambda: ops.expert_matmul(x, w, offsets, out=torch.zeros(10, 23, device=DEV)),
                lambda: ops.expert_matmul(x, w, offsets, out_dtype=torch.float16), lambda: ops.expert_matmul(x[0], w, offsets),
                lambda: ops.expert_matmul(x.t(), w, offsets), lambda: ops.expert_matmul_grad(dy, offsets),
                lambda: ops.expert_matmul_grad(dy, offsets, x=x[:9]), lambda: ops.expert_matmul_grad(dy, offsets, x=x, accumulate=True),
                lambda: ops.expert_matmul_grad(dy, offsets, w=w, dx=torch.zeros(10, 8, device=DEV)),
                lambda: ops.expert_matmul_grad(dy, offsets, x=x, w=w[:, :, :8])]:
        with pytest.raises(ValueError):
            bad()
    off = torch.zeros(10, 20, dtype=BF16, device=DEV)[:, 1:17]  # rows off their boundaries
    for bad in [lambda: ops.expert_matmul(off, w, offsets), lambda: ops.expert_matmul(x[:, :13].contiguous(), w[:, :, :13], offsets),
                lambda: ops.expert_matmul_grad(dy, offsets, x=off)]:
        with pytest.raises(AdaScaleError):
            bad()
    with pytest.raises(AdaScaleError):
        ops.expert_matmul(x, w[:1].expand(1025, 24, 16), offsets_of([0] * 1025))


@pytest.mark.parametrize("out_t", [BF16, F32])
@pytest.mark.parametrize("rows", [1, 15, 17, 31, 32, 33, 63, 64, 65, 100, 160, 255, 256, 257, 300, 449])
def test_every_width_of_a_tile_of_two_blocks(rows, out_t):
    """Enough summands for pairs of blocks, beside a large expert; NaN before the first row and behind the last."""
    k, m, counts = 576, 530, [rows, 1100]
    g = gen(rows)
    n = sum(counts) + 9
    x, w, dy = normal(g, n, k, dtype=BF16), normal(g, 2, m, k, dtype=BF16), aligned(normal(g, n, m, dtype=BF16))
    for t in (x, dy):
        t[:4], t[-5:] = float("nan"), float("nan")
    offsets = offsets_of(counts, 4)
    before = torch.full((n, m), 7.0, device=DEV, dtype=out_t)
    y = ops.expert_matmul(x, w, offsets, out=before.clone())
    forward_check(x, w, offsets, y, before, "product")
    before = torch.full((n, k), 7.0, device=DEV, dtype=out_t)
    dw0 = normal(g, 2, m, k, dtype=out_t)
    got = ops.expert_matmul_grad(dy, offsets, x=x, w=w, dx=before.clone(), dw=dw0.clone(), accumulate=True)
    want, mag = before.double(), torch.zeros(n, k, dtype=torch.float64, device=DEV)
    for e, lo, hi in groups(offsets):
        want[lo:hi], mag[lo:hi] = dy[lo:hi].double() @ w[e].double(), dy[lo:hi].double().abs() @ w[e].double().abs()
        whole = dw0[e].double() + dy[lo:hi].double().t() @ x[lo:hi].double()
        terms = dy[lo:hi].double().abs().t() @ x[lo:hi].double().abs()
        check(got.dw[e], whole, 2 * (hi - lo) * U * terms + U * whole.abs() + rounding(out_t) * whole.abs() * 1.01, "dw")
    check(got.dx, want, 2 * m * U * mag + rounding(out_t) * want.abs() * 1.01, "dx")


def test_long_sums_in_32_bits():
    """Sums of 20000 terms of one sign, which instructions that cut lose 2e-5 of: a float32 result is formed in parts of 768 terms, each cut 48
    times (16 terms an instruction) by less than 2^-23 of what it holds, and 27 rounded additions of parts by 2^-24 each."""
    g = gen(9)
    n = 20000
    x, dy = normal(g, n, 64, dtype=BF16).abs(), normal(g, n, 320, dtype=BF16).abs()
    got = ops.expert_matmul_grad(dy, offsets_of([n]), x=x)
    want = dy.double().t() @ x.double()
    check(got.dw[0], want, (48 * 2.0 ** -23 + 27 * U) * want, "dw")
    w = normal(g, 1, 200, 12000, dtype=BF16).abs()
    x = normal(g, 300, 12000, dtype=BF16).abs()
    y = ops.expert_matmul(x, w, offsets_of([300]), out_dtype=F32)
    want = x.double() @ w[0].double().t()
    check(y, want, (48 * 2.0 ** -23 + 16 * U) * want, "y")


def test_many_experts():
    """As many as there may be, most of them with a few rows or none; weights' gradients whole, zeros among them."""
    g = gen(21)
    counts = torch.randint(0, 5, (1024,), generator=torch.Generator().manual_seed(4)).tolist()
    counts[17], counts[500:520] = 300, [0] * 20
    n, k, m = sum(counts), 72, 40
    x, w, dy = normal(g, n, k, dtype=BF16), normal(g, 1024, m, k, dtype=BF16), normal(g, n, m, dtype=BF16)
    offsets = offsets_of(counts)
    owner = torch.repeat_interleave(torch.arange(1024, device=DEV), torch.tensor(counts, device=DEV))
    own = w[owner].double()
    y = ops.expert_matmul(x, w, offsets, out_dtype=F32)
    want = torch.einsum("rmk,rk->rm", own, x.double())
    check(y, want, 2 * k * U * torch.einsum("rmk,rk->rm", own.abs(), x.double().abs()) + U * want.abs(), "y")
    got = ops.expert_matmul_grad(dy, offsets, x=x, w=w, dx_dtype=F32)
    want = torch.einsum("rmk,rm->rk", own, dy.double())
    check(got.dx, want, 2 * m * U * torch.einsum("rmk,rm->rk", own.abs(), dy.double().abs()) + U * want.abs(), "dx")
    outer = dy.double()[:, :, None] * x.double()[:, None, :]
    want = torch.zeros(1024, m, k, dtype=torch.float64, device=DEV).index_add_(0, owner, outer)
    mag = torch.zeros_like(want).index_add_(0, owner, outer.abs())
    check(got.dw, want, 2 * 300 * U * mag + U * want.abs(), "dw")


@pytest.mark.parametrize("k,m", [(1, 1), (1, 9), (9, 1), (3, 130), (129, 2)])
def test_narrow_widths(k, m):
    g = gen(k + m)
    counts = [5, 0, 140, 1]
    n = sum(counts)
    x, w, dy = padded(normal(g, n, k, dtype=BF16), 1), padded(normal(g, 4, m, k, dtype=BF16), 1), padded(normal(g, n, m, dtype=BF16), 1)
    offsets = offsets_of(counts)
    for t in (BF16, F32):
        y = ops.expert_matmul(x, w, offsets, out_dtype=t)
        forward_check(x, w, offsets, y, torch.zeros_like(y), "narrow")
        got = ops.expert_matmul_grad(dy, offsets, x=x, w=w, dx_dtype=t, wgrad_dtype=t)
        for e, lo, hi in groups(offsets):
            want = dy[lo:hi].double() @ w[e].double()
            check(got.dx[lo:hi], want, 2 * m * U * (dy[lo:hi].double().abs() @ w[e].double().abs()) + rounding(t) * want.abs() * 1.01, "dx")
            want = dy[lo:hi].double().t() @ x[lo:hi].double()
            check(got.dw[e], want, 2 * 140 * U * (dy[lo:hi].double().abs().t() @ x[lo:hi].double().abs()) + rounding(t) * want.abs() * 1.01, "dw")


def test_gradients_one_behind_the_other():
    """Microbatches added into one gradient, each call's rows made by the kernel before it and its results read by the one behind it."""
    g = gen(31)
    x, w, dy = normal(g, 900, 640, dtype=BF16), normal(g, 3, 600, 640, dtype=BF16), normal(g, 900, 600, dtype=BF16)
    cuts = [offsets_of([300, 300, 300]), offsets_of([0, 899, 1]), offsets_of([13, 600, 200])]
    offsets = torch.zeros(4, dtype=torch.int32, device=DEV)
    for t in (F32, BF16):
        dw, alone = torch.zeros(3, 600, 640, dtype=t, device=DEV), torch.zeros(3, 600, 640, dtype=t, device=DEV)
        dx = torch.zeros(900, 640, dtype=BF16, device=DEV)
        seen, want = [], []
        for k in range(9):
            offsets.copy_(cuts[k % 3])
            ops.expert_matmul_grad(dy, offsets, x=x, w=w, dx=dx, dw=dw, accumulate=True)
            seen.append((dx.clone(), dw.clone()))
        for k in range(9):
            torch.cuda.synchronize()
            ops.expert_matmul_grad(dy, cuts[k % 3], w=w, dx=dx)
            torch.cuda.synchronize()
            ops.expert_matmul_grad(dy, cuts[k % 3], x=x, dw=alone, accumulate=True)
            torch.cuda.synchronize()
            want.append((None, alone.clone()))
        assert all(torch.equal(a[1], b[1]) for a, b in zip(seen, want))
        for k in range(9):
            o = cuts[k % 3].tolist()
            alone_dx = ops.expert_matmul_grad(dy, cuts[k % 3], w=w).dx
            assert torch.equal(seen[k][0][o[0]:o[3]], alone_dx[o[0]:o[3]])


@pytest.mark.parametrize("n,first", [((1 << 31) - 513, (1 << 31) - 1025), ((1 << 29) + 33, 1 << 29)])
def test_sums_that_last(n, first):
    """Up to as many rows as there may be, in one sum that takes seconds (3 and 13) on its block, which has a tile of another expert behind it; the end of the
    sum, or only of the one behind it, is no multiple of 64 rows.  Sums of ones and twos: all but the last are multiples of 768 below 2^32,
    which 32 bits hold, so that nothing is rounded but the result."""
    if torch.cuda.mem_get_info()[0] < n * 40:
        pytest.skip("wants %d GB" % (n * 40 >> 30))
    experts = torch.cuda.get_device_properties(0).multi_processor_count + 1
    x, dy = (torch.ones(n, 8, dtype=BF16, device=DEV) for _ in range(2))
    x[:, 5] = 2.0
    offsets = torch.full((experts + 1,), first, device=DEV)
    offsets[0], offsets[-1] = 0, n
    got = ops.expert_matmul_grad(dy, offsets, x=x)
    ones = torch.zeros(experts, dtype=torch.float64, device=DEV)
    ones[0], ones[-1] = first, n - first
    want = ones[:, None, None].expand(experts, 8, 8).clone()
    want[:, :, 5] *= 2.0
    check(got.dw, want, U * want, "dw")


@pytest.mark.parametrize("counts", [[768, 700], [5, 769, 768], [100] * 20 + [1537], [768, 0, 764]], ids=str)
def test_sums_around_a_part(counts):
    """Groups up to and beyond 768 rows, the length at which a float32 sum is cut, beside others; tolerances of short and of long sums."""
    g = gen(sum(counts))
    x, dy = normal(g, sum(counts), 320, dtype=BF16).abs(), normal(g, sum(counts), 264, dtype=BF16).abs()
    offsets = offsets_of(counts)
    dw0 = normal(g, len(counts), 264, 320)
    got, more = ops.expert_matmul_grad(dy, offsets, x=x).dw, dw0.clone()
    ops.expert_matmul_grad(dy, offsets, x=x, dw=more, accumulate=True)
    for e, lo, hi in groups(offsets):
        want = dy[lo:hi].double().t() @ x[lo:hi].double()
        off = (48 * 2.0 ** -23 + 2 * U) * want
        check(got[e], want, off, "dw")
        whole = dw0[e].double() + want
        check(more[e], whole, off + U * whole.abs(), "dw added")


def check_rounded_once(got, want, off):
    """bf16 results: half a step of the value, and `off` of it."""
    half = torch.exp2(torch.floor(torch.log2(want.abs())) - 8)
    check(got, want, half * (1 + 2.0 ** -20) + off * want.abs(), "rounded once")


# A part of 16384 terms of one sign is cut 1024 times (16 terms an instruction), each time by two units in the last place of what it holds, which is
# half of its end on average and whose unit is 2^-23 of it at most; each part's addition is rounded by 2^-24.
LONG = 1024 * 2.0 ** -23


@pytest.mark.parametrize("m", [64, 200])
def test_long_sums_in_bf16(m):
    """Sums so long that instructions that cut would lose more of them than the results' rounding: 2^23 rows of one expert (1e-2 of itself), beside
    another's, and 2^20 summands of a product (1e-3, half of a step's half), on blocks alone and in pairs."""
    g = gen(m)
    counts = [(1 << 23) + 40, 77, 65536]
    x, dy = (torch.empty(sum(counts), c, dtype=BF16, device=DEV).uniform_(0.5, 1.5, generator=g) for c in (32, m))
    offsets = offsets_of(counts, ids=torch.int64)
    got = ops.expert_matmul_grad(dy, offsets, x=x, wgrad_dtype=BF16).dw
    for e, lo, hi in groups(offsets):
        want = sum(dy[k:min(k + (1 << 20), hi)].double().t() @ x[k:min(k + (1 << 20), hi)].double() for k in range(lo, hi, 1 << 20))
        check_rounded_once(got[e], want, LONG + 520 * U)
    del x, dy
    k = 1 << 20
    x, w = (torch.empty(s, k, dtype=BF16, device=DEV).uniform_(0.5, 1.5, generator=g) for s in (70, m))
    want = sum(x[:, c:c + (1 << 16)].double() @ w[:, c:c + (1 << 16)].double().t() for c in range(0, k, 1 << 16))
    check_rounded_once(ops.expert_matmul(x, w.view(1, m, k), offsets_of([70])), want, LONG + 70 * U)
    wide = torch.empty(1, k, m, dtype=BF16, device=DEV).uniform_(0.5, 1.5, generator=g)
    want = sum(x[:, c:c + (1 << 16)].double() @ wide[0, c:c + (1 << 16)].double() for c in range(0, k, 1 << 16))
    check_rounded_once(ops.expert_matmul_grad(x, offsets_of([70]), w=wide).dx, want, LONG + 70 * U)


@pytest.mark.parametrize("counts", [[16384, 16000], [5, 16385, 16384], [32768, 32000], [5, 32769, 32768], [65537]], ids=str)
def test_bf16_sums_around_a_part(counts):
    """Whole numbers, so that every sum is exact but for the result's rounding."""
    g = gen(sum(counts))
    x, dy = (torch.randint(-2, 3, (sum(counts), c), device=DEV, generator=g).to(BF16) for c in (72, 136))
    dw0 = torch.randint(-9, 9, (len(counts), 136, 72), device=DEV, generator=g).to(BF16)
    offsets, more = offsets_of(counts), dw0.clone()
    got = ops.expert_matmul_grad(dy, offsets, x=x, wgrad_dtype=BF16).dw
    ops.expert_matmul_grad(dy, offsets, x=x, dw=more, accumulate=True)
    for e, lo, hi in groups(offsets):
        want = dy[lo:hi].double().t() @ x[lo:hi].double()
        assert torch.equal(got[e], want.to(BF16)) and torch.equal(more[e], (want + dw0[e].double()).to(BF16))


def test_as_many_rows_as_there_may_be_in_bf16():
    n = (1 << 31) - 513
    if torch.cuda.mem_get_info()[0] < n * 40:
        pytest.skip("wants %d GB" % (n * 40 >> 30))
    x, dy = (torch.ones(n, 8, dtype=BF16, device=DEV) for _ in range(2))
    x[:, 5] = 2.0
    got = ops.expert_matmul_grad(dy, torch.tensor([0, n], device=DEV), x=x, wgrad_dtype=BF16).dw
    want = torch.full((1, 8, 8), float(n), dtype=torch.float64, device=DEV)
    want[:, :, 5] *= 2.0
    check_rounded_once(got, want, 2 * U)


def test_gradients_that_would_not_be_written_are_refused():
    """A slot of a gradient row that is given without what its gradient is made of would stay as it was."""
    x, w, dy = (torch.zeros(*s, dtype=BF16, device=DEV) for s in ((10, 16), (2, 24, 16), (10, 24)))
    offsets, dx, dw = offsets_of([5, 5]), torch.zeros(10, 16, device=DEV), torch.zeros(2, 24, 16, device=DEV)
    for bad in [lambda: ops.expert_matmul_grad(dy, offsets, w=w, dw=dw), lambda: ops.expert_matmul_grad(dy, offsets, x=x, dx=dx),
                lambda: ops.expert_matmul_grad(dy, offsets, w=w, dx=dx, dw=dw, accumulate=True), lambda: ops.expert_matmul_grad(dy, offsets, x=x, dx=dx, dw=dw)]:
        with pytest.raises(ValueError):
            bad()
    got = ops.expert_matmul_grad(dy, offsets, w=w, accumulate=True)  # which is about dw alone
    assert got.dw is None and got.dx.shape == (10, 16)


def inside(shape, dtype, rows_around=3):
    """A matrix (or one of each expert) inside a wide buffer, its rows on 16-byte boundaries, with NaN on all sides; and whether those are left."""
    *e, n, d = shape
    whole = torch.full((*e, n + 2 * rows_around, 512), float("nan"), dtype=dtype, device=DEV)
    view = whole[..., rows_around:n + rows_around, 64:64 + d]

    def intact():
        around = torch.isnan(whole)
        around[..., rows_around:n + rows_around, 64:64 + d] = True
        assert bool(around.all()), "written beside the matrix"
    return view, intact


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width", [1, 7, 9, 12, 20, 33, 36, 39, 100, 130, 257])
def test_rows_that_end_inside_16_bytes(width, dtype):
    """Slices of wider matrices, on 16-byte boundaries: what is beside them, in the same 16 bytes, is someone else's."""
    g = gen(width)
    for counts in ([20], [32, 3], [70, 0, 64], [300, 520]):
        n, E = sum(counts), len(counts)
        offsets = offsets_of(counts)
        x, narrow, dy = normal(g, n, 40, dtype=BF16), padded(normal(g, n, width, dtype=BF16), 1), normal(g, n, 40, dtype=BF16)
        to, back = padded(normal(g, E, width, 40, dtype=BF16), 1), padded(normal(g, E, 40, width, dtype=BF16), 1)
        y, y_intact = inside((n, width), dtype)
        ops.expert_matmul(x, to, offsets, out=y)
        forward_check(x, to, offsets, y, torch.zeros_like(y), "y")
        y_intact()
        for accumulate in (False, True):
            dx, dx_intact = inside((n, width), dtype)
            dw, dw_intact = inside((E, 40, width), dtype)
            before = normal(g, E, 40, width, dtype=dtype)
            dw.copy_(before)
            ops.expert_matmul_grad(dy, offsets, x=narrow, w=back, dx=dx, dw=dw, accumulate=accumulate)
            for e, lo, hi in groups(offsets):
                want, mag = dy[lo:hi].double() @ back[e].double(), dy[lo:hi].double().abs() @ back[e].double().abs()
                check(dx[lo:hi], want, 80 * U * mag + rounding(dtype) * want.abs() * 1.01, "dx")
                part, mag = dy[lo:hi].double().t() @ narrow[lo:hi].double(), dy[lo:hi].double().abs().t() @ narrow[lo:hi].double().abs()
                whole = part + before[e].double() if accumulate else part
                check(dw[e], whole, 2 * max(hi - lo, 1) * U * mag + U * whole.abs() + rounding(dtype) * whole.abs() * 1.01, "dw")
            dx_intact()
            dw_intact()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_one_row_of_weights_between_other_slots(dtype):
    """A single output: its gradient's row is a slot of any width, with others' right behind it."""
    g = gen(6)
    for width in (3, 13, 37, 250):
        x, dy, offsets = padded(normal(g, 90, width, dtype=BF16), 1), padded(normal(g, 90, 1, dtype=BF16), 1), offsets_of([90])
        row = torch.full((width + 40,), float("nan"), dtype=dtype, device=DEV)
        ops.expert_matmul_grad(dy, offsets, x=x, dw=row[16:16 + width].view(1, 1, width))
        want = dy.double().t() @ x.double()
        check(row[16:16 + width].view(1, width), want, 180 * U * (dy.double().abs().t() @ x.double().abs()) + rounding(dtype) * want.abs() * 1.01, "dw")
        assert bool(torch.isnan(row[:16]).all()) and bool(torch.isnan(row[16 + width:]).all())
