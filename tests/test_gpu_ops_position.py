"""Attention weights with a relative position bias, and their gradient, against the formula in 64 bits.

Tolerances, with u = 2^-24.  A logit z = scale s + bias is off by u |z|, its distance from the row's largest by as much for either
and u |z - top| for the subtraction, two more such for the factor log2 e: with Z the row's largest |z| the exponent is off by
at most 2 u Z + 3 u 2 Z = 8 u Z, and the sum in the denominator relatively by as much; the exponential's own error is
2^-22 = 4 u twice, the sum of n terms, of which no thread adds more than c in a row, (c + 45) u, the quotient 2 u.  Results are rounded by u or 2^-8 of
the value (bfloat16), and weights below 2^-126 may be 0.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

from paper_2007_05105_b200 import ops  # noqa: E402
from paper_2007_05105_b200.binding import AdaScaleError  # noqa: E402
from test_gpu_ops import BF16, DEV, F32, LOWEST, U, check, gen, normal, rounding  # noqa: E402

TINY = 2.0 ** -126


def bucket(d, buckets, max_distance, both):
    """In whole numbers: the border of far bucket k is the smallest n with n^far >= exact^(far - k) max_distance^k."""
    m = buckets // 2 if both else buckets
    n = abs(d) if both else max(0, -d)
    exact, far = m // 2, m - m // 2
    if n >= max_distance:
        at = m - 1
    elif n >= exact:
        at = exact + sum(n ** far >= exact ** (far - k) * max_distance ** k for k in range(1, far))
    else:
        at = n
    return at + (m if both and d > 0 else 0)


def buckets_of(case, b, lq, lk):
    start = int(case["starts"][b]) if case["starts"] is not None else 0
    dist = torch.arange(lk)[None, :] - (start + torch.arange(lq))[:, None]
    dist = dist.clamp(-case["distance"], case["distance"])
    known = torch.tensor([bucket(d, case["buckets"], case["distance"], case["both"]) for d in range(-case["distance"], case["distance"] + 1)])
    return known[dist + case["distance"]].to(DEV)


def live_of(case, b, lq, lk):
    start = int(case["starts"][b]) if case["starts"] is not None else 0
    length = max(0, min(lk, int(case["lengths"][b]))) if case["lengths"] is not None else lk
    key = torch.arange(lk, device=DEV)[None, :]
    live = (key < length).expand(lq, lk)
    return live & (key <= start + torch.arange(lq, device=DEV)[:, None]) if case["causal"] else live


def how(case):
    return dict(max_distance=case["distance"], bidirectional=case["both"], scale=case["scale"], causal=case["causal"], lengths=case["lengths"],
                starts=case["starts"])


def longest_run(lk):
    return max(32, lk // 256)


def check_forward(probs, scores, table, case, what):
    for b in range(scores.shape[0]):
        lq, lk = scores.shape[2:]
        live = live_of(case, b, lq, lk)
        z = scores[b].double() * case["scale"] + table.double().t()[:, buckets_of(case, b, lq, lk)]
        z = z.masked_fill(~live, -math.inf)
        nothing = (z == -math.inf).all(dim=-1, keepdim=True)
        want = torch.where(nothing, 0.0, torch.softmax(z, dim=-1))
        want = torch.where(live, want, 0.0)
        size = z.masked_fill(torch.isinf(z), 0.0).abs().amax(dim=-1, keepdim=True)
        rel = U * (2 * 8 * size + 8 + longest_run(lk) + 45 + 2)
        check(probs[b], want, torch.nan_to_num(want * (rel + rounding(probs.dtype) * 1.01)) + TINY, what)


def check_gradient(got, probs, dprobs, case, before, what):
    B, H, lq, lk = probs.shape
    dtable = torch.zeros(case["buckets"], H, dtype=torch.float64, device=DEV)
    mag, err = torch.zeros_like(dtable), torch.zeros_like(dtable)
    for b in range(B):
        live = live_of(case, b, lq, lk)
        p, dp = (torch.where(live, t[b].double(), 0.0) for t in (probs, dprobs))
        dot, size = (p * dp).sum(-1, keepdim=True), (p * dp).abs().sum(-1, keepdim=True)
        g = p * (dp - dot)
        # the products' sum, the difference, the product
        off = p.abs() * (U * (dp - dot).abs() + (longest_run(lk) + 45) * U * size) + U * g.abs()
        if got.dscores is not None:
            want = case["scale"] * g
            check(got.dscores[b], want, abs(case["scale"]) * off + U * want.abs() + rounding(probs.dtype) * want.abs() * 1.01 + TINY, what + " dscores")
        at = buckets_of(case, b, lq, lk).reshape(-1)
        for total, term in ((dtable, g), (mag, g.abs()), (err, off)):
            total.index_add_(0, at, term.reshape(H, -1).t())
    if got.dtable is not None:
        terms = B * lq * longest_run(lk)  # of one lane, at most
        want = dtable if before is None else dtable + before.double()
        check(got.dtable, want, err + (terms + 45) * U * mag + (U + rounding(got.dtable.dtype) * 1.01) * want.abs() + TINY, what + " dtable")


def make(shape, dtype, seed, both, causal, ragged, starts, buckets=32, distance=128, shift=0, scale=0.125):
    """Scores with NaN where nothing is live, in rows that begin `shift` elements off their boundaries."""
    B, H, lq, lk = shape
    g = gen(seed)
    case = dict(buckets=buckets, distance=distance, both=both, causal=causal, scale=scale, lengths=None, starts=None)
    if ragged:
        case["lengths"] = torch.randint(0, lk + 1, (B,), device=DEV, generator=g, dtype=torch.int32)
        case["lengths"][0] = lk
    if starts:
        case["starts"] = torch.randint(-2, lk + 3, (B,), device=DEV, generator=g)
        case["starts"][0] = lk - lq
    live = torch.stack([live_of(case, b, lq, lk) for b in range(B)])[:, None]

    def tensor(std):
        t = torch.empty(B, H, lq, lk + shift, dtype=dtype, device=DEV)[..., shift:] if shift else torch.empty(shape, dtype=dtype, device=DEV)
        t.copy_(normal(g, *shape, std=std))
        return t.masked_fill_(~live, float("nan"))
    return case, tensor, normal(g, buckets, H)


MODES = [  # both sides, causal, ragged, starts
    (True, False, False, False), (False, True, False, False), (True, False, True, True), (False, True, True, True), (True, True, True, False),
]
SHAPES = [(1, 1, 1, 1), (2, 3, 1, 7), (3, 2, 5, 64), (2, 2, 33, 66), (1, 3, 17, 129), (2, 4, 40, 256), (1, 2, 9, 300), (2, 2, 70, 517),
          (1, 2, 6, 1024), (2, 1, 5, 1300), (1, 2, 3, 3000), (1, 1, 2, 8000), (2, 1, 2, 9001), (1, 1, 2, 33000)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("mode", MODES, ids=str)
def test_weights_and_gradient(shape, dtype, mode):
    for shift in (0, 1, 5):
        case, tensor, table = make(shape, dtype, sum(shape) + shift, *mode, shift=shift)
        scores = tensor(8.0)
        probs = ops.position_softmax(scores, table, **how(case))
        assert probs.dtype == dtype and probs.shape == scores.shape
        check_forward(probs, scores, table, case, "weights")
        dprobs = tensor(1.0)
        got = ops.position_softmax_grad(probs, dprobs, case["buckets"], **how(case))
        check_gradient(got, probs, dprobs, case, None, "gradient")
        assert torch.equal(ops.position_softmax(scores, table, **how(case)), probs)
        again = ops.position_softmax_grad(probs, dprobs, case["buckets"], **how(case))
        assert torch.equal(again.dscores, got.dscores) and torch.equal(again.dtable, got.dtable)


@pytest.mark.parametrize("buckets,distance,both", [(2, 2, False), (4, 2, True), (8, 3, True), (7, 20, False), (16, 16384, True), (32, 128, True), (64, 65, False),
                                                   (128, 33, True), (128, 65, False), (128, 1000, True), (32, 32768 // 2, False)])
def test_every_bucket(buckets, distance, both):
    """A table whose entries tell the buckets apart: log of the weight's ratio to that of the query's own position."""
    span = distance + 20
    case = dict(buckets=buckets, distance=distance, both=both, causal=False, scale=1.0, lengths=None,
                starts=torch.tensor([span], device=DEV))
    table = (torch.arange(buckets, device=DEV, dtype=F32)[:, None] / 8.0)
    scores = torch.zeros(1, 1, 1, 2 * span + 1, device=DEV)
    probs = ops.position_softmax(scores, table, **how(case))
    got = torch.round(8.0 * torch.log(probs[0, 0, 0].double() / probs[0, 0, 0, span].double())).long()
    want = torch.tensor([bucket(d, buckets, distance, both) for d in range(-span, span + 1)], device=DEV)
    assert torch.equal(got, want - want[span])
    g = ops.position_softmax_grad(torch.ones_like(scores), torch.zeros_like(scores), buckets, **how(case))
    assert not g.dtable.any()


@pytest.mark.parametrize("buckets", [2, 30, 64, 128])
@pytest.mark.parametrize("grad_t,accumulate", [(F32, False), (BF16, True), (F32, True)])
def test_table_gradient(buckets, grad_t, accumulate):
    case, tensor, table = make((3, 5, 50, 200), BF16, buckets, False, False, True, True, buckets=buckets, distance=100)
    probs, dprobs = torch.nan_to_num(torch.softmax(tensor(1.0).float(), -1)).to(BF16), tensor(1.0)
    wide = torch.full((buckets, 9), 3.0, dtype=grad_t, device=DEV)
    before = wide[:, 2:7].clone()
    got = ops.position_softmax_grad(probs, dprobs, buckets, **how(case), dtable=wide[:, 2:7], accumulate=accumulate, want_dscores=False)
    assert got.dscores is None
    check_gradient(got, probs, dprobs, case, before if accumulate else None, "table")
    assert bool((wide[:, :2] == 3.0).all()) and bool((wide[:, 7:] == 3.0).all())
    only = ops.position_softmax_grad(probs, dprobs, buckets, **how(case), want_dtable=False)
    assert only.dtable is None
    check_gradient(only, probs, dprobs, case, None, "scores")


def test_against_differences():
    """Of a weighted sum of weights, in 64-bit arithmetic on 32-bit results: a central difference of step h is off by h^2 / 6 times the third
    derivative, which for a softmax is below 6 max|c|, and by the results' errors over h."""
    case, tensor, table = make((2, 2, 6, 40), F32, 3, True, False, True, False, distance=20)
    scores, c = torch.nan_to_num(tensor(4.0)), normal(gen(4), 2, 2, 6, 40)
    probs = ops.position_softmax(scores, table, **how(case))
    got = ops.position_softmax_grad(probs, c, 32, **how(case))
    h = 2.0 ** -6
    loss = lambda s, t: float((ops.position_softmax(s, t, **how(case)).double() * c.double()).sum())  # noqa: E731
    size = float(c.abs().max())
    # logits below 8: a row's weights are off by 300 u of themselves, the rows' sums (24) by that of max|c| each
    noise = 24 * 300 * U * size / h
    for at in [(0, 0, 0, 0), (1, 1, 5, 3), (0, 1, 2, 17)]:
        up, down = scores.clone(), scores.clone()
        up[at] += h / case["scale"]
        down[at] -= h / case["scale"]
        slope = (loss(up, table) - loss(down, table)) / (2 * h)
        assert abs(slope - float(got.dscores[at]) / case["scale"]) <= h * h * size + noise
    for at in [(0, 0), (3, 1), (17, 0), (30, 1)]:
        up, down = table.clone(), table.clone()
        up[at] += h
        down[at] -= h
        slope = (loss(scores, up) - loss(scores, down)) / (2 * h)
        assert abs(slope - float(got.dtable[at])) <= 24 * h * h * size + noise


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lk", [20, 200, 1500, 9500])
def test_rows_of_infinities_and_lowest_values(dtype, lk):
    case, tensor, table = make((1, 2, 12, lk), dtype, lk, True, False, False, False)
    table = table.clone()
    scores = tensor(8.0)
    scores[0, :, 0] = -math.inf
    scores[0, :, 1, 1:] = -math.inf
    scores[0, :, 2, ::2] = -math.inf
    scores[0, :, 3, 5] = math.inf
    scores[0, :, 4, lk - 1] = float("nan")
    scores[0, :, 5, :] = -math.inf
    scores[0, :, 5, 7] = float("nan")
    scores[0, :, 6, 3:] = LOWEST[dtype]  # a mask added to the scores
    scores[0, :, 7] = 0.0
    probs = ops.position_softmax(scores, table, **how(case))
    assert not probs[0, :, 0].any() and bool((probs[0, :, 1, 0] == 1.0).all()) and not probs[0, :, 1, 1:].any()
    assert not probs[0, :, 2, ::2].any() and not probs[0, :, 6, 3:].any()
    assert bool(torch.isnan(probs[0, :, 3:6]).all()) and not torch.isnan(probs[0, :, :3]).any() and not torch.isnan(probs[0, :, 6:]).any()
    fine = [0, 1, 2, 6, 7, 8, 9, 10, 11]
    for i in fine:  # row by row: the check takes queries from position 0 on
        one = dict(case, starts=torch.tensor([i], device=DEV))
        check_forward(probs[:, :, i:i + 1], scores[:, :, i:i + 1], table, one, "row %d" % i)
    whole = torch.full((1, 2, 3, lk), LOWEST[dtype], dtype=dtype, device=DEV)  # nothing but the lowest value: the bias is swallowed, all are alike
    even = ops.position_softmax(whole, table, **dict(how(case), scale=1.0))
    check(even, torch.full(even.shape, 1.0 / lk, dtype=torch.float64, device=DEV), (U * (longest_run(lk) + 60) + rounding(dtype) * 1.01) / lk, "even")


def test_lengths_and_starts_outside():
    for ids in (torch.int32, torch.int64):
        lengths, starts = torch.tensor([-5, 0, 3, 900], dtype=ids, device=DEV), torch.tensor([-9, 4, 2 ** 31 - 1, 0], dtype=ids, device=DEV)
        case = dict(buckets=16, distance=50, both=False, causal=True, scale=1.0, lengths=lengths, starts=starts)
        scores, table = normal(gen(1), 4, 2, 10, 33), normal(gen(2), 16, 2)
        probs = ops.position_softmax(scores, table, **how(case))
        assert not probs[:2].any() and bool((probs[2].sum(-1) - 1).abs().max() < 1e-5) and not probs[2, :, :, 3:].any()
        check_forward(probs, scores, table, dict(case, starts=starts.long().clamp(max=1 << 20)), "outside")
        got = ops.position_softmax_grad(probs, scores, 16, **how(case))
        check_gradient(got, probs, scores, dict(case, starts=starts.long().clamp(max=1 << 20)), None, "outside")


def test_in_place_strides_and_broadcast():
    case, tensor, table = make((2, 4, 30, 136), BF16, 9, True, False, True, False)
    scores, dprobs = tensor(8.0), tensor(1.0)
    probs = ops.position_softmax(scores, table, **how(case))
    place = scores.clone()
    assert ops.position_softmax(place, table, **how(case), out=place) is place and torch.equal(place, probs)
    got = ops.position_softmax_grad(probs, dprobs, 32, **how(case))
    for alias in (0, 1):
        args = [probs.clone(), dprobs.clone()]
        again = ops.position_softmax_grad(*args, 32, **how(case), dscores=args[alias])
        assert torch.equal(args[alias], got.dscores) and torch.equal(again.dtable, got.dtable)
    # heads behind queries in memory, rows with room between them, another alignment for each matrix
    turned = torch.empty(2, 30, 4, 140, dtype=BF16, device=DEV).transpose(1, 2)[..., 3:139]
    turned.copy_(scores)
    out = torch.full((2, 4, 30, 150), 7.0, dtype=BF16, device=DEV)
    assert torch.equal(ops.position_softmax(turned, table, **how(case), out=out[..., 6:142]), probs)
    assert bool((out[..., :6] == 7.0).all()) and bool((out[..., 142:] == 7.0).all())
    again = ops.position_softmax_grad(out[..., 6:142], turned.copy_(dprobs), 32, **how(case))
    # other columns share a thread, so sums go in another order
    check_gradient(again, probs, dprobs, case, None, "turned")
    same = scores[:1, :1].nan_to_num()
    wide = ops.position_softmax(same.expand(2, 4, 30, 136), table, **how(case))
    assert torch.equal(wide, ops.position_softmax(same.expand(2, 4, 30, 136).contiguous(), table, **how(case)))
    # a gradient that arrives the same for all keys
    flat = torch.ones(1, 1, 1, 1, dtype=BF16, device=DEV).expand(2, 4, 30, 136)
    with pytest.raises(ValueError):  # keys are adjacent
        ops.position_softmax_grad(probs, flat, 32, **how(case))
    assert scores.data_ptr() != probs.data_ptr()


def test_nothing_to_do():
    table = normal(gen(0), 8, 2)
    for shape in [(0, 2, 3, 4), (1, 2, 0, 4), (1, 2, 3, 0)]:
        t = torch.empty(shape, device=DEV)
        assert ops.position_softmax(t, table).shape == shape
        d = torch.full((8, 2), 5.0, device=DEV)
        ops.position_softmax_grad(t, t, 8, dtable=d, accumulate=True)
        assert bool((d == 5.0).all())
        assert not ops.position_softmax_grad(t, t, 8, dtable=d).dtable.any()


def test_many_rows_far_behind_the_first():
    """More than 2^31 elements; each head's rows in several blocks."""
    B, H, lq, lk = 2, 4, 4100, 70000
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("wants 12 GB")
    scores = torch.zeros(B, H, lq, lk, dtype=BF16, device=DEV)
    scores[1, 3, -1, 5] = 80.0
    table = torch.zeros(8, H, device=DEV)
    probs = ops.position_softmax(scores, table, causal=True, bidirectional=False, out=scores)
    assert float(probs[1, 3, -1, 5]) == 1.0
    rest = math.exp(-80.0)  # beside 1 + 4099 e^-80, which is 1; its exponent is off by 8 u 80
    assert abs(float(probs[1, 3, -1, 6]) - rest) <= rest * (2.0 ** -8 * 1.01 + 700 * U)
    want = 1.0 / torch.arange(1, lq, device=DEV, dtype=torch.float64)
    check(probs[1, 2, :-1, 0], want, want * (2.0 ** -8 * 1.01 + 400 * U), "first key")
    assert not probs[:, :, :, lq:].any()


def test_captured_and_on_a_stream():
    case, tensor, table = make((2, 3, 20, 90), F32, 9, False, True, True, True)
    scores, dprobs = tensor(8.0), tensor(1.0)
    probs, got = None, None
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    other = ops.position_softmax(scores, table, **how(case), stream=stream)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        probs = ops.position_softmax(scores, table, **how(case))
        got = ops.position_softmax_grad(probs, dprobs, 32, **how(case))
    graph.replay()
    assert torch.equal(probs, other)
    scores.copy_(torch.nan_to_num(scores).flip(0))
    graph.replay()
    want = ops.position_softmax(scores, table, **how(case))
    again = ops.position_softmax_grad(want, dprobs, 32, **how(case))
    assert torch.equal(probs, want) and torch.equal(got.dscores, again.dscores) and torch.equal(got.dtable, again.dtable)


def test_refusals():
    s, table = torch.zeros(2, 3, 4, 5, device=DEV), torch.zeros(32, 3, device=DEV)
    n = torch.zeros(2, dtype=torch.int32, device=DEV)
    for bad in [lambda: ops.position_softmax(s[0], table), lambda: ops.position_softmax(s, table[:, :2]), lambda: ops.position_softmax(s, table.to(BF16)),
                lambda: ops.position_softmax(s.half(), table), lambda: ops.position_softmax(s.cpu(), table), lambda: ops.position_softmax(s, table.cpu()),
                lambda: ops.position_softmax(s, table, lengths=n[:1]), lambda: ops.position_softmax(s, table, starts=n.float()),
                lambda: ops.position_softmax(s, table, out=s.to(BF16)), lambda: ops.position_softmax(s.transpose(2, 3), table),
                lambda: ops.position_softmax(s, table, out=s[:, :, :, :4]), lambda: ops.position_softmax_grad(s, s[:, :, :3], 32),
                lambda: ops.position_softmax_grad(s, s, 32, dtable=table[:31]), lambda: ops.position_softmax_grad(s, s, 32, accumulate=True),
                lambda: ops.position_softmax_grad(s, s, 1 << 30), lambda: ops.position_softmax_grad(s, s.to(BF16), 32)]:
        with pytest.raises(ValueError):
            bad()
    for bad in [lambda: ops.position_softmax(s, table, max_distance=8), lambda: ops.position_softmax(s, table[:31]),
                lambda: ops.position_softmax(s, table, max_distance=1 << 20), lambda: ops.position_softmax(s, table, scale=math.inf),
                lambda: ops.position_softmax(s, torch.zeros(130, 3, device=DEV), max_distance=1000),
                lambda: ops.position_softmax(s, table, out=torch.zeros(1, 3, 4, 5, device=DEV).expand(2, 3, 4, 5)),
                lambda: ops.position_softmax_grad(s, s, 32, want_dscores=False, want_dtable=False),
                lambda: ops.position_softmax_grad(s, s, 32, workspace=torch.zeros(16, dtype=torch.uint8, device=DEV))]:
        with pytest.raises(AdaScaleError):
            bad()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape,distance", [((1, 2, 40, 1500), 1000), ((2, 1, 30, 5000), 3000), ((1, 1, 3, 20000), 16384), ((1, 2, 30, 700), 1025)])
def test_far_distances(shape, distance, dtype):
    """Maximum distances on either side of what is kept by distance, with buckets that change within a thread's keys."""
    for mode in [(True, False, False, True), (False, True, True, True)]:
        case, tensor, table = make(shape, dtype, distance, *mode, buckets=128, distance=distance)
        scores, dprobs = tensor(8.0), tensor(1.0)
        probs = ops.position_softmax(scores, table, **how(case))
        check_forward(probs, scores, table, case, "weights")
        got = ops.position_softmax_grad(probs, dprobs, 128, **how(case))
        check_gradient(got, probs, dprobs, case, None, "gradient")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_of_every_length(dtype):
    """One and the same row cut at every length, so that each part of an access is once the last live one; whole rows, and lengths."""
    g = gen(12)
    scores, dprobs, table = normal(g, 1, 2, 3, 140, dtype=dtype, std=8.0), normal(g, 1, 2, 3, 140, dtype=dtype), normal(g, 16, 2)
    for n in list(range(1, 40)) + [63, 64, 65, 71, 100, 127, 128, 129, 139, 140]:
        case = dict(buckets=16, distance=50, both=True, causal=False, scale=0.125, lengths=None, starts=torch.tensor([60], device=DEV))
        s, d = scores[..., :n].contiguous(), dprobs[..., :n].contiguous()
        probs = ops.position_softmax(s, table, **how(case))
        check_forward(probs, s, table, case, "cut at %d" % n)
        check_gradient(ops.position_softmax_grad(probs, d, 16, **how(case)), probs, d, case, None, "cut at %d" % n)
        case["lengths"] = torch.tensor([n], device=DEV)
        whole = ops.position_softmax(scores, table, **how(case))
        check_forward(whole, scores, table, case, "length %d" % n)
        check_gradient(ops.position_softmax_grad(whole, dprobs, 16, **how(case)), whole, dprobs, case, None, "length %d" % n)


def test_many_batches_and_heads():
    for shape in [(70000, 2, 1, 3), (2, 5000, 2, 9), (1, 1, 70000, 5)]:
        case, tensor, table = make(shape, BF16, 3, True, False, False, False, buckets=8, distance=6)
        scores, dprobs = tensor(8.0), tensor(1.0)
        probs = ops.position_softmax(scores, table, **how(case))
        z = scores.double() * case["scale"] + table.double().t()[None, :, buckets_of(case, 0, *shape[2:])].view(1, shape[1], *shape[2:])
        want = torch.softmax(z, dim=-1)
        size = z.abs().amax(dim=-1, keepdim=True)
        check(probs, want, want * (U * (16 * size + 90) + 2.0 ** -8 * 1.01) + TINY, "weights")
        got = ops.position_softmax_grad(probs, dprobs, 8, **how(case))
        p, dp = probs.double(), dprobs.double()
        g = p * (dp - (p * dp).sum(-1, keepdim=True))
        off = p * U * ((dp - (p * dp).sum(-1, keepdim=True)).abs() + 80 * (p * dp).abs().sum(-1, keepdim=True)) + U * g.abs()
        check(got.dscores, 0.125 * g, 0.125 * off + (U + 2.0 ** -8 * 1.01) * 0.125 * g.abs() + TINY, "dscores")
        at = buckets_of(case, 0, *shape[2:]).reshape(-1)
        flat = lambda t: torch.zeros(8, shape[1], dtype=torch.float64, device=DEV).index_add_(0, at, t.sum(0).reshape(shape[1], -1).t())  # noqa: E731
        terms = shape[0] * shape[2] * 32
        check(got.dtable, flat(g), flat(off) + (terms + 45) * U * flat(g.abs()) + 2 * U * flat(g).abs(), "dtable")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(2, 3, 200, 13), (2, 3, 150, 201), (2, 4, 120, 301), (1, 8, 300, 999), (1, 2, 40, 2051)])
def test_in_place_where_rows_share_accesses(shape, dtype):
    """Rows whose ends lie in 16 bytes with their neighbours', which other threads write at the same time: the same bits as elsewhere,
    in place and between poison on either side."""
    case, tensor, table = make(shape, dtype, 7, True, False, True, False)
    scores, dprobs = tensor(8.0), tensor(1.0)
    probs = ops.position_softmax(scores, table, **how(case))
    got = ops.position_softmax_grad(probs, dprobs, 32, **how(case))
    for _ in range(3):
        place = scores.clone()
        assert torch.equal(ops.position_softmax(place, table, **how(case), out=place), probs)
        for alias in (0, 1):
            args = [probs.clone(), dprobs.clone()]
            ops.position_softmax_grad(*args, 32, **how(case), dscores=args[alias])
            assert torch.equal(args[alias], got.dscores)
    for before in (1, 3, 8):  # whatever lies around the tensors is not used and stays
        whole = [torch.full((before + scores.numel() + 9,), float("nan"), dtype=dtype, device=DEV) for _ in range(4)]
        s, d, p, o = (w[before:before + scores.numel()].view(shape) for w in whole)
        s.copy_(scores)
        d.copy_(dprobs)
        ops.position_softmax(s, table, **how(case), out=p)
        again = ops.position_softmax_grad(p, d, 32, **how(case), dscores=o)
        check_forward(p, scores, table, case, "between poison")
        check_gradient(again, p, dprobs, case, None, "between poison")
        for w in whole:
            assert bool(torch.isnan(w[:before]).all()) and bool(torch.isnan(w[before + scores.numel():]).all())


def check_table_exactly(shape, dtype, case, shift, seed, what):
    """The table's gradient of weights 1/4 and whole numbers: products, rows' sums, differences and sums by bucket are multiples of 1/16
    which 32 bits hold, so that nothing is rounded, in whatever order it is added up."""
    g = gen(seed)
    B, H, lq, lk = shape
    live = torch.stack([live_of(case, b, lq, lk) for b in range(B)])[:, None]
    whole = torch.randint(-3, 4, shape, device=DEV, generator=g).double()
    # in whole rows of even length: as many of either sign, so that g is a small number
    pairs = whole[..., :lk // 2]
    whole = torch.cat([pairs, -pairs, whole[..., 2 * (lk // 2):]], dim=-1).gather(-1, torch.rand(shape, device=DEV, generator=g).argsort(dim=-1))

    def tensor(values):
        t = torch.empty(B, H, lq, lk + shift, dtype=dtype, device=DEV)[..., shift:] if shift else torch.empty(shape, dtype=dtype, device=DEV)
        return t.copy_(values).masked_fill_(~live, float("nan"))
    probs, dprobs = tensor(torch.full(shape, 0.25, device=DEV)), tensor(whole)
    kept = torch.where(live, whole, 0.0)
    terms = torch.where(live, 0.25 * (kept - 0.25 * kept.sum(-1, keepdim=True)), 0.0)
    want, size = (torch.zeros(case["buckets"], H, dtype=torch.float64, device=DEV) for _ in range(2))
    for b in range(B):
        at = buckets_of(case, b, lq, lk).reshape(-1)
        want.index_add_(0, at, terms[b].reshape(H, -1).t())
        size.index_add_(0, at, terms[b].abs().reshape(H, -1).t())
    assert float(size.max()) * 16 < 2 ** 24 and bool(want.any() or lk == 1)
    got = ops.position_softmax_grad(probs, dprobs, case["buckets"], **how(case))
    assert torch.equal(got.dtable.double(), want), what
    assert torch.equal(ops.position_softmax_grad(probs, dprobs, case["buckets"], **how(case), want_dscores=False).dtable, got.dtable)


BUCKETS = [(2, 2, False), (4, 2, True), (8, 3, True), (7, 20, False), (16, 16384, True), (32, 128, True), (64, 65, False), (128, 33, True),
           (128, 65, False), (128, 1000, True), (32, 16384, False), (30, 90, True), (64, 150, False)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("buckets,distance,both", BUCKETS)
def test_every_bucket_of_the_gradient(buckets, distance, both, dtype):
    """Keys on either side of queries before, among and behind them: near ones, which are summed by distance, and far ones; rows on
    16-byte boundaries and off them, of every kind of group."""
    for lk in (1, 50, 110, 160, 301, 700, 1500, 2 * distance + 41):
        for shift in (0, 3):
            starts = torch.tensor([0, lk // 2, lk + distance // 2, -(distance // 3), lk - 1], device=DEV)
            case = dict(buckets=buckets, distance=distance, both=both, causal=False, scale=0.125, lengths=None, starts=starts)
            check_table_exactly((5, 2, 3 if lk < 5000 else 1, lk), dtype, case, shift, lk, "%d keys, shift %d" % (lk, shift))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("buckets,distance", [(7, 20), (32, 128), (64, 65), (64, 150), (128, 1000)])
def test_every_bucket_of_the_gradient_with_masks(buckets, distance, dtype):
    for lk in (7, 66, 128, 250, 301, 700, 1500):
        for shift in (0, 1):
            lengths = torch.tensor([lk, 0, lk // 2 + 1, lk - 1], device=DEV)
            for causal, starts in ((True, torch.tensor([0, 3, lk // 3, lk - 4], device=DEV)), (False, None)):
                case = dict(buckets=buckets, distance=distance, both=False, causal=causal, scale=0.125, lengths=lengths, starts=starts)
                check_table_exactly((4, 3, 40, lk), dtype, case, shift, lk, "%d keys, shift %d" % (lk, shift))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(70000, 2, 1, 3), (2, 5000, 2, 9), (1, 1, 70000, 5), (9, 1, 3000, 20), (300, 4, 64, 64)])
def test_table_gradient_of_many_rows(shape, dtype):
    case = dict(buckets=8, distance=6, both=True, causal=False, scale=0.125, lengths=None, starts=None)
    if shape[0] > 1000:  # the formula a batch at a time would take minutes: all of them are alike
        g = gen(1)
        dprobs = torch.randint(-3, 4, shape, device=DEV, generator=g).double()
        terms = 0.25 * (dprobs - 0.25 * dprobs.sum(-1, keepdim=True))
        at = buckets_of(case, 0, *shape[2:]).reshape(-1)
        want, size = (torch.zeros(8, shape[1], dtype=torch.float64, device=DEV).index_add_(0, at, t.sum(0).reshape(shape[1], -1).t()) for t in (terms, terms.abs()))
        assert float(size.max()) * 16 < 2 ** 24 and bool(want.any())
        got = ops.position_softmax_grad(torch.full(shape, 0.25, dtype=dtype, device=DEV), dprobs.to(dtype), 8, **how(case))
        assert torch.equal(got.dtable.double(), want)
    else:
        check_table_exactly(shape, dtype, case, 0, 2, "many rows")
