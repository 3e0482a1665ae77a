"""The language-model operators against their formulas in 64 bits.

Tolerances follow from the arithmetic and are written beside each comparison.  Throughout, u = 2^-24 is
half a unit in the last place of a 32-bit float; a bf16 result (8 significant bits) carries a
further rounding of 2^-8 of its value; a sum of m terms of which no thread adds more than c in a row is off by at most
(c + 45) u times the sum of the terms' magnitudes (45: the joins over lanes, warps and pieces).
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

from paper_2007_05105_b200 import ops  # noqa: E402
from paper_2007_05105_b200.binding import AdaScaleError  # noqa: E402

DEV = torch.device("cuda:0")
U = 2.0 ** -24
BF = 2.0 ** -8
F32, BF16 = torch.float32, torch.bfloat16
LOWEST = {F32: torch.finfo(F32).min, BF16: torch.finfo(BF16).min}


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(g, *shape, dtype=F32, std=1.0, mean=0.0):
    return torch.empty(*shape, device=DEV).normal_(mean, std, generator=g).to(dtype)


def rounding(dtype):
    return BF + U if dtype == BF16 else U


def check(got, want, tol, what=""):
    """Element by element; NaN and infinities in the same places."""
    got, want = got.double(), want.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what + ": NaN elsewhere"
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]) and not torch.isinf(got[~inf]).any(), what + ": infinities elsewhere"
    fine = ~inf & ~torch.isnan(want)
    err, tol = (got - want).abs()[fine], torch.as_tensor(tol, device=DEV, dtype=torch.float64).expand(want.shape)[fine]
    bad = err > tol
    assert not bad.any(), "%s: %d elements off, worst %.3g of tolerance" % (what, int(bad.sum()), float((err / tol.clamp(min=1e-300)).max()))


def strided(t, pad, shift=0):
    """The matrix with `pad` elements between its rows and its first element `shift` elements off a 512-byte
    boundary, surrounded by a poison value; returns (matrix, check that the poison is intact)."""
    n, d = t.shape
    whole = torch.full((shift + n * (d + pad) + 64,), 77.0, dtype=t.dtype, device=DEV)
    view = whole[shift:shift + n * (d + pad)].view(n, d + pad)[:, :d]
    view.copy_(t)
    keep = torch.ones_like(whole, dtype=torch.bool)
    keep[shift:shift + n * (d + pad)].view(n, d + pad)[:, :d] = False

    def intact():
        assert bool((whole[keep] == 77.0).all()), "written outside the matrix"
    return view, intact


def empty_strided_out(n, d, dtype, pad, shift):
    return strided(torch.full((n, d), float("nan"), dtype=dtype, device=DEV), pad, shift)


# --------------------------------------------------------------------------
# token table
# --------------------------------------------------------------------------


def tokens_of(kind, n, vocab, g):
    if kind == "same":
        return torch.full((n,), vocab // 2, device=DEV)
    if kind == "zipf":
        return (vocab * torch.rand(n, device=DEV, generator=g, dtype=torch.float64) ** 4).long().clamp(max=vocab - 1)
    if kind == "blocks":  # runs of every length around the window's 64, in order and not
        t = torch.arange(n, device=DEV)
        return ((t // 63) * 7 + (t % 5 == 0) * 3) % vocab
    if kind == "sorted":
        return torch.randint(0, vocab, (n,), device=DEV, generator=g).sort().values
    if kind == "outside":
        t = torch.randint(-3, vocab + 3, (n,), device=DEV, generator=g)
        t[::7] = -1 - t[::7].abs()
        return t
    return torch.randint(0, vocab, (n,), device=DEV, generator=g)


@pytest.mark.parametrize("table_t,out_t", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("n,vocab,d,pad,shift", [(1, 1, 1, 0, 0), (1, 300, 512, 0, 0), (3, 2, 7, 1, 1), (257, 300, 513, 0, 0),
                                                 (257, 300, 1024, 8, 8), (33, 70000, 64, 3, 5), (1000, 50, 2056, 0, 0), (5, 9, 8, 0, 1)])
def test_embed(n, vocab, d, pad, shift, table_t, out_t):
    g = gen(n + d)
    table, _ = strided(normal(g, vocab, d, dtype=table_t), pad, shift)
    for ids in (torch.int64, torch.int32):
        tok = tokens_of("outside" if vocab > 10 else "any", n, vocab, g).to(ids)
        out, intact = empty_strided_out(n, d, out_t, pad, shift)
        assert ops.embed(tok, table, scale=math.sqrt(d), out=out) is out
        known = (tok >= 0) & (tok < vocab)
        want = table.double()[tok.long().clamp(0, vocab - 1)] * float(torch.tensor(math.sqrt(d), dtype=F32)) * known[:, None]
        check(out, want, want.abs() * rounding(out_t) * 1.01, "embed")  # one product, one rounding to the result's type
        intact()


def test_embed_keeps_the_shape_of_the_tokens_and_takes_none():
    table = normal(gen(0), 10, 16)
    tok = torch.randint(0, 10, (2, 3, 4), device=DEV)
    assert torch.equal(ops.embed(tok, table), table[tok])
    assert ops.embed(tok, table, out_dtype=BF16).dtype == BF16
    assert ops.embed(tok[:0], table).shape == (0, 3, 4, 16)


def embed_grad_check(tok, dout, grad, base, scale, padding, accumulate, what):
    vocab = grad.shape[0]
    keep = (tok >= 0) & (tok < vocab) & (tok != padding)
    terms, at = dout.double()[keep] * float(torch.tensor(scale, dtype=F32)), tok.long()[keep]
    want = torch.zeros(grad.shape, dtype=torch.float64, device=DEV).index_add_(0, at, terms)
    mag = torch.zeros_like(want).index_add_(0, at, terms.abs())
    if accumulate:
        want = want + base.double()
    # 128 terms in a row at most (a window and what its last run goes on into the next), then the pieces: a warp adds every
    # fourth; scale and base one rounding each
    count = torch.bincount(at, minlength=vocab).double()[:, None]
    in_a_row = count.clamp(max=128) + count / 256
    tol = mag * (in_a_row + 45) * U + want.abs() * (2 * U + (BF if grad.dtype == BF16 else 0.0))
    if accumulate:
        tol = tol * (count > 0)  # rows that no token names are as they were
    check(grad, want, tol, what)


@pytest.mark.parametrize("dout_t,grad_t", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("kind,n,vocab,d", [
    ("any", 1, 1, 1), ("any", 1, 1000, 8), ("any", 5, 3, 7), ("same", 63, 4, 16), ("same", 64, 4, 16), ("same", 65, 4, 16),
    ("same", 128, 4, 24), ("same", 129, 4, 24), ("same", 192, 1, 8), ("same", 193, 3, 8), ("same", 5000, 70001, 40),
    ("blocks", 1000, 50, 64), ("blocks", 4096, 9, 520), ("sorted", 777, 65535, 33), ("any", 3000, 65536, 16),
    ("zipf", 9001, 50257, 256), ("zipf", 20000, 300, 8), ("outside", 3000, 37, 100), ("any", 70000, 17, 8), ("zipf", 300, 20_000_000, 1)])
def test_embed_grad(kind, n, vocab, d, dout_t, grad_t):
    g = gen(n * 31 + d)
    tok = tokens_of(kind, n, vocab, g)
    dout = normal(g, n, d, dtype=dout_t)
    padding = int(tok[0]) if kind in ("zipf", "blocks") else -1
    for ids, accumulate in ((torch.int64, False), (torch.int32, True)):
        base = normal(g, vocab, d, dtype=grad_t) if accumulate else torch.full((vocab, d), float("nan"), dtype=grad_t, device=DEV)
        grad = base.clone()
        assert ops.embed_grad(tok.to(ids), dout, grad, scale=3.7, padding_idx=padding, accumulate=accumulate) is grad
        embed_grad_check(tok, dout, grad, base, 3.7, padding, accumulate, "embed_grad %s" % kind)
        again = base.clone()  # the same bits every time
        ops.embed_grad(tok.to(ids), dout, again, scale=3.7, padding_idx=padding, accumulate=accumulate)
        assert torch.equal(grad, again)


@pytest.mark.parametrize("pad,shift", [(8, 8), (1, 0), (0, 1), (3, 2)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_embed_grad_strides_and_workspace(pad, shift, accumulate):
    g = gen(5)
    n, vocab, d = 500, 90, 72
    tok = tokens_of("zipf", n, vocab, g)
    for dtype in (F32, BF16):
        dout, _ = strided(normal(g, n, d, dtype=dtype), pad, shift)
        base = normal(g, vocab, d, dtype=dtype)
        grad, intact = strided(base, pad, shift)
        need = ops.embed_grad_workspace(n, d)
        room = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device=DEV)
        ops.embed_grad(tok, dout, grad, scale=0.5, accumulate=accumulate, workspace=room[:need])
        embed_grad_check(tok, dout, grad, base, 0.5, -1, accumulate, "strided")
        intact()
        assert bool((room[need:] == 0xA5).all())


def test_embed_grad_without_tokens_writes_zeros():
    grad = torch.full((70, 24), float("nan"), device=DEV)
    ops.embed_grad(torch.empty(0, dtype=torch.int64, device=DEV), torch.empty(0, 24, device=DEV), grad)
    assert bool((grad == 0).all())
    grad.fill_(3.0)
    ops.embed_grad(torch.full((9,), 7, device=DEV), torch.ones(9, 24, device=DEV), grad, padding_idx=7)
    assert bool((grad == 0).all())


def test_embed_gradient_is_that_of_the_lookup_by_differences():
    """<dout, embed(W + h D) - embed(W - h D)> / 2h = <grad, D>: the lookup is linear, h = 1."""
    g = gen(11)
    tok, W, D, dout = tokens_of("zipf", 400, 100, g), normal(g, 100, 48), normal(g, 100, 48), normal(g, 400, 48)
    grad = ops.embed_grad(tok, dout, torch.empty_like(W), scale=1.5)
    up, down = (ops.embed(tok, W + s * D, scale=1.5).double() for s in (1, -1))
    left, right = (dout.double() * (up - down)).sum() / 2, (grad.double() * D.double()).sum()
    # roundings of W +- D and of the two lookups against terms of size |dout| (|W| + |D|), and those of the sums in grad
    tol = 4 * U * float((dout.double().abs() * (up.abs() + down.abs())).sum()) + 150 * U * float((dout.abs().sum(0) * D.abs().max()).sum()) * 1.5
    assert abs(float(left - right)) <= tol


# --------------------------------------------------------------------------
# distillation
# --------------------------------------------------------------------------


def distill_reference(z, t, ids, labels, T, alpha, beta, weight):
    """Loss per row and gradient in 64 bits from the formulas, and the magnitudes that the tolerances need."""
    n, vocab = z.shape
    z = z.double()
    some = ~torch.isneginf(z).all(dim=1)  # rows that have logits
    z = torch.where(some[:, None], z, torch.zeros_like(z))
    d = z - z.max(dim=1, keepdim=True).values
    row = torch.zeros(n, dtype=torch.float64, device=DEV)
    row_mag, grad, grad_mag = row.clone(), torch.zeros_like(z), torch.zeros_like(z)
    w = torch.ones_like(row) if weight is None else weight.double()
    T32 = float(torch.tensor(T, dtype=F32))
    a32, b32 = (float(torch.tensor(v, dtype=F32)) for v in (alpha, beta))
    reach = d.abs().clamp(max=120.0 * max(1.0, T32))  # beyond this the exponential is 0 or below every sum's last place
    # p's relative error: exponential and its argument (4 times that where it is a fourth power), and the sum of the row
    eps = 2.0 ** -20 + 2.0 ** -22 * reach * max(1.0, 1.0 / T32) + (vocab / 512 + 45) * U
    if alpha and t is not None and t.shape[1]:
        valid = (ids >= 0) & (ids < vocab) & ~torch.isneginf(t.double())
        has = valid.any(dim=1) & some
        td = t.double().masked_fill(~valid, float("-inf")) / T32
        q = torch.softmax(td, dim=1).masked_fill(~has[:, None] | ~valid, 0.0)
        at = ids.long().clamp(0, vocab - 1)
        lse = torch.logsumexp(d / T32, dim=1)
        dk = (d.gather(1, at) / T32).masked_fill(q == 0, 0.0)  # -inf where a wanted entry is masked: an infinite loss
        log_q = torch.where(q > 0, q, 1.0).log()
        row += torch.where(has, a32 * T32 ** 2 * (q * (log_q - dk)).sum(1) + a32 * T32 ** 2 * lse, 0.0)
        spread = (td.masked_fill(~valid, 0.0).abs().max(dim=1).values * 2 + 1)
        row_mag += has * a32 * T32 ** 2 * (((q * (log_q.abs() + dk.abs())).sum(1) + 1) * (spread * 2 ** -22 + 2 ** -21)
                                           + lse.abs() * 2 ** -21 + eps.min(dim=1).values + 2 ** -20)
        p = torch.softmax(d / T32, dim=1)
        coef = (a32 * T32 * has)[:, None]
        qs = torch.zeros_like(z).scatter_add_(1, at, q)
        grad += coef * (p - qs)
        grad_mag += coef * (p * eps + qs * (spread[:, None] * 2 ** -22 + 2 ** -21))
    if beta and labels is not None:
        has = (labels >= 0) & (labels < vocab) & some
        y = labels.long().clamp(0, vocab - 1)
        lse = torch.logsumexp(d, dim=1)
        dy = d.gather(1, y[:, None])[:, 0]
        row += torch.where(has, b32 * (lse - dy), 0.0)
        row_mag += has * b32 * ((lse.abs() + dy.abs()) * 2 ** -21 + eps.min(dim=1).values + 2 ** -20)
        p = torch.softmax(d, dim=1)
        hot = torch.zeros_like(z).scatter_(1, y[:, None], 1.0)
        grad += (b32 * has)[:, None] * (p - hot)
        grad_mag += (b32 * has)[:, None] * (p * eps + hot * 2 ** -22)
    return row * w, row_mag * w.abs(), grad * w[:, None], grad_mag * w.abs()[:, None]


def check_distill(got, z, t, ids, labels, T, alpha, beta, weight, what=""):
    row, row_tol, grad, grad_tol = distill_reference(z, t, ids, labels, T, alpha, beta, weight)
    check(got.row_loss, row, row_tol + 1e-37, what + " row_loss")
    check(got.loss, row.sum(), row_tol.sum() + row.abs().sum() * 2 * U + 1e-37, what + " loss")
    if got.dlogits is not None:
        # 2^-22: the products that make the coefficients; 1e-37: results below the normal range are flushed
        check(got.dlogits, grad, grad_tol + grad.abs() * (2 ** -22 + (BF if z.dtype == BF16 else 0)) + 1e-37, what + " dlogits")


def distill_inputs(n, vocab, k, dtype, seed, t_dtype=F32, id_dtype=torch.int32):
    g = gen(seed)
    z = normal(g, n, vocab, std=2.0)
    ids = torch.randint(0, vocab, (n, k), device=DEV, generator=g)  # repetitions happen
    t = 6.0 - 2.0 * torch.log1p(torch.arange(k, device=DEV, dtype=F32)) + normal(g, n, k, std=0.4)
    if k:
        z.scatter_(1, ids, 0.7 * t + normal(g, n, k, std=0.5))
        ids[:, k // 2 + 1:] = torch.where(torch.rand(n, k - k // 2 - 1, device=DEV, generator=g) < 0.3, -1, ids[:, k // 2 + 1:])
        ids[0, 0] = vocab if n > 1 else ids[0, 0]
    labels = torch.randint(0, vocab, (n,), device=DEV, generator=g)
    if k:
        labels[1::3] = ids[1::3, -1]
    labels[2::5] = -100
    weight = torch.rand(n, device=DEV, generator=g)
    weight[3::4] = 0.0
    return z.to(dtype), t.to(t_dtype), ids.to(id_dtype), labels, weight


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,alpha,beta", [(1.0, 1.0, 0.0), (1.0, 0.3, 0.7), (2.0, 0.5, 0.5), (4.0, 0.9, 0.1), (1.5, 0.5, 0.5), (3.0, 0.5, 0.5), (1.3, 0.5, 0.5),
                                          (0.5, 0.6, 0.4), (3.0, 1.0, 0.0), (2.0, 0.0, 1.0)])
@pytest.mark.parametrize("n,vocab,k", [(1, 1, 1), (1, 5, 0), (3, 17, 4), (7, 1000, 64), (40, 4099, 33), (2, 50257, 64), (170, 12345, 9),
                                       (9, 33000, 1024)])
def test_distill(n, vocab, k, T, alpha, beta, dtype):
    z, t, ids, labels, weight = distill_inputs(n, vocab, k, dtype, n + vocab)
    got = ops.distill(z, t, ids, labels=labels, T=T, alpha=alpha, beta=beta, row_weight=weight)
    check_distill(got, z, t, ids, labels, T, alpha, beta, weight)
    alone = ops.distill(z, t, ids, labels=labels, T=T, alpha=alpha, beta=beta, row_weight=weight, want_grad=False)
    assert alone.dlogits is None and torch.equal(alone.row_loss, got.row_loss) and torch.equal(alone.loss, got.loss)
    again = ops.distill(z, t, ids, labels=labels, T=T, alpha=alpha, beta=beta, row_weight=weight)
    assert torch.equal(again.loss, got.loss) and torch.equal(again.dlogits, got.dlogits)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_distill_types_strides_and_places(dtype):
    n, vocab, k = 6, 5003, 12
    for t_dtype, id_dtype in [(F32, torch.int64), (BF16, torch.int32)]:
        z0, t, ids, labels, weight = distill_inputs(n, vocab, k, dtype, 3, t_dtype, id_dtype)
        for pad, shift, out_pad, out_shift in [(0, 0, 0, 0), (5, 3, 5, 3), (5, 3, 0, 0), (3, 0, 1, 1), (8, 8, 8, 0)]:
            z, _ = strided(z0, pad, shift)
            out, intact = empty_strided_out(n, vocab, dtype, out_pad, out_shift)
            got = ops.distill(z, t, ids, labels=labels.to(id_dtype), T=2.0, alpha=0.5, beta=0.5, row_weight=weight, dlogits=out)
            check_distill(got, z, t, ids, labels, 2.0, 0.5, 0.5, weight, "strides")
            intact()
            place, intact = strided(z0, pad, shift)  # the gradient over the logits
            same = ops.distill(place, t, ids, labels=labels, T=2.0, alpha=0.5, beta=0.5, row_weight=weight, dlogits=place)
            assert torch.equal(same.loss, got.loss) and torch.equal(place, got.dlogits)
            intact()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T", [0.25, 1.0, 1.5, 2.0])
@pytest.mark.parametrize("vocab", [50, 20001])
def test_distill_masked_vocabulary_and_rows_with_nothing(vocab, T, dtype):
    n, k = 8, 6
    z, t, ids, labels, _ = distill_inputs(n, vocab, k, dtype, 21)
    keep = torch.zeros_like(z, dtype=torch.bool)
    keep.scatter_(1, ids.long().clamp(0, vocab - 1), True).scatter_(1, labels.clamp(min=0)[:, None], True)
    mask = torch.rand(n, vocab, device=DEV, generator=gen(1)) < 0.5
    z = torch.where(mask & ~keep, torch.full_like(z, float("-inf")), z)
    z[1] = torch.where(keep[1], z[1], torch.full_like(z[1], float("-inf")))
    z[2] = torch.where(keep[2], z[2], torch.full_like(z[2], LOWEST[dtype]))
    z[3] = LOWEST[dtype]            # every entry alike: the uniform distribution
    ids[4], labels[4] = -1, -100    # nothing to learn from
    labels[3], labels[5] = 4, -1
    t[5] = float("-inf")            # an empty list by its logits, and no label
    t[6, 1:] = float("-inf")
    weight = torch.full((n,), 0.3, device=DEV)
    weight[7] = 0.0
    got = ops.distill(z, t, ids, labels=labels, T=T, alpha=0.5, beta=0.5, row_weight=weight)
    check_distill(got, z, t, ids, labels, T, 0.5, 0.5, weight, "masks")
    assert float(got.row_loss[4]) == 0 and float(got.row_loss[5]) == 0 and not got.dlogits[4].any() and not got.dlogits[5].any()

    # rows that do not count may hold anything
    z[4], z[5], z[7] = float("nan"), float("inf"), float("nan")
    z[6] = float("-inf")
    got = ops.distill(z, t, ids, labels=labels, T=T, alpha=0.5, beta=0.5, row_weight=weight)
    for r in (4, 5, 6, 7):
        assert float(got.row_loss[r]) == 0 and not got.dlogits[r].any(), r
    assert math.isfinite(float(got.loss))

    # a NaN or +inf in a live row is that row's, and the loss's, alone
    for bad in (float("nan"), float("inf")):
        z[0, vocab // 3] = bad
        got = ops.distill(z, t, ids, labels=labels, T=T, alpha=0.5, beta=0.5, row_weight=weight)
        assert math.isnan(float(got.row_loss[0])) and bool(torch.isnan(got.dlogits[0]).all()) and math.isnan(float(got.loss))
        assert not torch.isnan(got.row_loss[1:]).any() and not torch.isnan(got.dlogits[1:]).any()


def test_distill_a_wanted_entry_that_is_masked_costs_infinitely_much():
    z = torch.zeros(2, 40, device=DEV)
    z[0, 3] = float("-inf")
    got = ops.distill(z, labels=torch.tensor([3, 3], device=DEV), alpha=0.0, beta=1.0)
    assert float(got.row_loss[0]) == math.inf and abs(float(got.row_loss[1]) - math.log(40)) < 4e-7 * math.log(40)
    assert float(got.dlogits[0, 3]) == -1.0


def test_distill_same_id_many_times():
    """A list that names one entry five times counts as one that names it once with the sum of its weights."""
    z = normal(gen(2), 1, 300)
    t = torch.tensor([[1.0, 2.0, 0.5, 1.5, 3.0, 0.0]], device=DEV)
    ids = torch.tensor([[7, 7, 7, 9, 7, 7]], device=DEV, dtype=torch.int32)
    got = ops.distill(z, t, ids)
    q = torch.softmax(t.double(), 1)[0]
    p = torch.softmax(z.double(), 1)[0]
    want = p.clone()
    want[7] -= q[[0, 1, 2, 4, 5]].sum()
    want[9] -= q[3]
    check(got.dlogits[0], want, 1e-6 * want.abs() + 2e-7 * p + 3e-7, "repeated ids")


def test_distill_without_rows_or_teacher():
    z = normal(gen(2), 0, 300)
    got = ops.distill(z, want_grad=True)
    assert float(got.loss) == 0 and got.row_loss.shape == (0,) and got.dlogits.shape == (0, 300)
    z = normal(gen(2), 4, 300)
    labels = torch.tensor([1, 2, -100, 299], device=DEV)
    got = ops.distill(z, labels=labels, alpha=0.0, beta=1.0)
    check_distill(got, z, None, None, labels, 1.0, 0.0, 1.0, None, "cross entropy")


@pytest.mark.parametrize("T", [1.0, 2.0, 1.5])
def test_distill_gradient_by_differences(T):
    """(loss(z + h D) - loss(z - h D)) / 2h against <dlogits, D>."""
    n, vocab, k = 5, 700, 8
    z, t, ids, labels, weight = distill_inputs(n, vocab, k, F32, 8)
    D, h = normal(gen(9), n, vocab), 2.0 ** -7
    at = dict(labels=labels, T=T, alpha=0.5, beta=0.5, row_weight=weight)
    up, down = (ops.distill(z + s * h * D, t, ids, want_grad=False, **at).row_loss.double() for s in (1, -1))
    slope = (ops.distill(z, t, ids, **at).dlogits.double() * D.double()).sum(1)
    # third derivative of a logsumexp along D: below 2 max|D|^3 (weights, 1/T and T^2 included: T <= 2);  a loss is off by 2^-18 of its size
    tol = h * h / 6 * 4 * float(D.abs().max()) ** 3 + 2.0 ** -18 * float((up.abs() + down.abs() + 20).max()) / (2 * h)
    assert float(((up - down) / (2 * h) - slope).abs().max()) <= tol


# --------------------------------------------------------------------------
# block boundary
# --------------------------------------------------------------------------


def norm64(v, kind, w, b, eps):
    """(n * w + b, n, 1 / deviation, |mean|)"""
    if kind in (None, "none"):
        return v, None, None, 0.0
    mean = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    r = 1.0 / torch.sqrt(((v - mean) ** 2).mean(1, keepdim=True) + eps)
    n = (v - mean) * r
    out = n * w
    return out + b if b is not None else out, n, r, mean.abs()


def boundary_inputs(n, d, x_t, y_t, pre, post, gate, seed):
    g = gen(seed)
    s = dict(x=normal(g, n, d, dtype=x_t, std=1.5), y=normal(g, n, d, dtype=y_t, std=0.7, mean=0.2))
    s["w_pre"], s["w_post"] = normal(g, d, std=0.3, mean=1.0), normal(g, d, std=0.3, mean=1.0) if post else None
    s["b_pre"] = normal(g, d) if pre == "layer" else None
    s["b_post"] = normal(g, d) if post == "layer" else None
    s["gate"] = {"none": None, "channel": normal(g, d), "element": normal(g, n, d, dtype=y_t, std=2.0)}[gate]
    s["dx"], s["dh"] = normal(g, n, d, dtype=x_t), normal(g, n, d, dtype=y_t)
    return s


def wide(v):
    return None if v is None else v.double()


KINDS = [("rms", None, "none"), ("layer", None, "channel"), ("rms", "rms", "none"), ("layer", "layer", "channel"),
         ("rms", "layer", "element"), ("layer", "rms", "element")]
SIZES = [(1, 1), (1, 1024), (3, 7), (5, 64), (33, 509), (130, 512), (7, 2048), (4, 4100), (2, 8192), (3, 16384), (2, 16381), (700, 256)]
SCALE, EPS = 0.625, 1e-5


def sums_in_a_row(n):
    """Steps of a sum over rows: a group adds every 148th row at most, then partial sums are joined."""
    return min(n, n / 148 + 150)


@pytest.mark.parametrize("x_t,y_t", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("n,d", SIZES)
@pytest.mark.parametrize("pre,post,gate", KINDS)
def test_boundary_and_its_gradient(pre, post, gate, n, d, x_t, y_t):
    s = boundary_inputs(n, d, x_t, y_t, pre, post, gate, n + d)
    kw = dict(pre=pre, post=post, w_pre=s["w_pre"], w_post=s["w_post"], gate=s["gate"], res_scale=SCALE, eps=EPS)
    x_new, h = ops.residual_norm(s["x"], s["y"], b_pre=s["b_pre"], b_post=s["b_post"], **kw)
    assert x_new.dtype == x_t and h.dtype == y_t
    x, y, G = wide(s["x"]), wide(s["y"]), wide(s["gate"])
    G = torch.ones(1, 1, dtype=torch.float64, device=DEV) if G is None else torch.sigmoid(G) if G.dim() == 2 else G[None]
    wp, bp, wq, bq = wide(s["w_post"]), wide(s["b_post"]), wide(s["w_pre"]), wide(s["b_pre"])
    zero = torch.zeros((), dtype=torch.float64, device=DEV)
    # every value is a product or sum of a few roundings and of sums over the row (8 or 16 terms per thread, 45 joins):
    # C u of the magnitudes that go into it; K is how much larger a row's elements are than its deviation
    C = 80 * U
    u, ny, ry, my = norm64(y, post, wp, bp, EPS)
    K_y = 1 + (((y.abs() + my) * ry).max(1, keepdim=True).values if post else 0)
    u_mag = (u.abs() + (bp.abs() if bp is not None else zero) + (((y.abs() + my) * ry * wp.abs()) if post else zero)) * K_y
    want_x = x + SCALE * G * u
    x_tol = C * (x.abs() + SCALE * G.abs() * u_mag)
    check(x_new, want_x, x_tol + want_x.abs() * rounding(x_t), "x_new")
    want_h, nx, rx, mx = norm64(want_x, pre, wq, bq, EPS)
    off = (x_tol + x_tol.mean(1, keepdim=True)) * rx * wq.abs()  # of x_new before it is rounded
    K_x = 1 + ((want_x.abs() + mx) * rx).max(1, keepdim=True).values
    h_tol = off * K_x + C * K_x * ((want_x.abs() + mx) * rx * wq.abs() + (bq.abs() if bq is not None else zero))
    check(h, want_h, h_tol + want_h.abs() * rounding(y_t), "h")

    # the gradient, with x as the stream after the block
    for wgrad in (F32, BF16):
        got = ops.residual_norm_grad(s["x"], s["y"], s["dx"], s["dh"], b_post=s["b_post"], wgrad_dtype=wgrad, **kw)
        _, nx, rx, mx = norm64(x, pre, wq, bq, EPS)
        K_x = 1 + ((x.abs() + mx) * rx).max(1, keepdim=True).values
        dh, c = wide(s["dh"]), rounding(wgrad)
        dn = dh * wq

        def back(dn, mag, n_, r_, kind):
            """Gradient of the norm's input and the magnitudes in it."""
            mean = dn.mean(1, keepdim=True) if kind == "layer" else 0.0
            dv = r_ * (dn - n_ * (dn * n_).mean(1, keepdim=True) - mean)
            return dv, r_ * (mag + n_.abs() * (mag * n_.abs()).mean(1, keepdim=True) + mag.mean(1, keepdim=True))
        dv, dv_mag = back(dn, dn.abs(), nx, rx, pre)
        dx = wide(s["dx"]) + dv
        dx_mag = (wide(s["dx"]).abs() + dv_mag) * K_x
        check(got.dx, dx, C * dx_mag + dx.abs() * rounding(x_t), "dx")
        rows = sums_in_a_row(n) * U
        def column(got_v, terms, mags, what):
            check(got_v, terms.sum(0), (C + rows) * mags.sum(0) + terms.sum(0).abs() * c, what)
        column(got.dw_pre, dh * nx, dh.abs() * (nx.abs() + (x.abs() + mx) * rx) * K_x, "dw_pre")
        if pre == "layer":
            column(got.db_pre, dh, dh.abs(), "db_pre")
        else:
            assert got.db_pre is None
        ds, ds_mag = SCALE * dx, SCALE * dx_mag
        if gate == "channel":
            column(got.dgate, ds * u, ds_mag * u_mag, "dgate")
        elif gate == "element":
            want = ds * u * G * (1 - G)
            # 1 - G is off by an ulp of 1
            check(got.dgate, want, C * ds_mag * u_mag * G + want.abs() * rounding(y_t), "dgate")
        else:
            assert got.dgate is None
        du, du_mag = ds * G, ds_mag * G.abs()
        if post:
            column(got.dw_post, du * ny, du_mag * (ny.abs() + (y.abs() + my) * ry) * K_y, "dw_post")
            if post == "layer":
                column(got.db_post, du, du_mag, "db_post")
            dy, dy_mag = back(du * wp, du_mag * wp.abs(), ny, ry, post)
            check(got.dy, dy, C * dy_mag * K_y + dy.abs() * rounding(y_t), "dy")
        else:
            assert got.dw_post is None and got.db_post is None
            check(got.dy, du, C * du_mag + du.abs() * rounding(y_t), "dy")


@pytest.mark.parametrize("x_t,y_t", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("n,d", [(5000, 72), (3000, 384), (2500, 640), (1500, 768), (1100, 1280), (700, 1536), (700, 2144), (330, 4352),
                                 (160, 4800), (160, 6144), (1700, 333), (1500, 771), (900, 1279), (450, 2049), (170, 4099),
                                 (160, 8191), (4, 9000), (4, 9001), (3, 12000)])
@pytest.mark.parametrize("pre,post,gate", [("rms", "rms", "none"), ("layer", "layer", "channel"), ("rms", "layer", "element")])
def test_boundary_of_other_widths(pre, post, gate, n, d, x_t, y_t):
    test_boundary_and_its_gradient(pre, post, gate, n, d, x_t, y_t)


@pytest.mark.parametrize("pad,shift", [(8, 8), (1, 3)])
@pytest.mark.parametrize("d", [64, 1000, 2600])
def test_boundary_strides_places_and_slots(d, pad, shift):
    n = 37
    for x_t, y_t in [(F32, BF16), (BF16, F32)]:
        s = boundary_inputs(n, d, x_t, y_t, "layer", "layer", "element", 4)
        kw = dict(pre="layer", post="layer", w_pre=s["w_pre"], w_post=s["w_post"], b_post=s["b_post"], res_scale=SCALE, eps=EPS)
        want = ops.residual_norm(s["x"], s["y"], b_pre=s["b_pre"], gate=s["gate"], **kw)
        x, ix = strided(s["x"], pad, shift)
        y, iy = strided(s["y"], pad, shift)
        gate, ig = strided(s["gate"], pad, shift)
        got = ops.residual_norm(x, y, b_pre=s["b_pre"], gate=gate, x_new=x, h=y, **kw)  # in place
        assert got[0] is x and got[1] is y
        ulp = lambda t: 2 * rounding(t.dtype) * t.double().abs() + 64 * U * (1 + t.double().abs())  # noqa: E731
        check(x, want[0], ulp(want[0]), "x in place")  # the two paths add in other orders
        check(y, want[1], ulp(want[1]), "h in place")
        for i in (ix, iy, ig):
            i()
        want = ops.residual_norm_grad(s["x"], s["y"], s["dx"], s["dh"], gate=s["gate"], **kw)
        x, y = strided(s["x"], pad, shift)[0], strided(s["y"], pad, shift)[0]
        dx, idx = strided(s["dx"], pad, shift)
        dh, idh = strided(s["dh"], pad, shift)
        dgate, idg = strided(torch.zeros_like(s["gate"]), pad, shift)
        row = torch.full((4 * (d + 3) + 5,), 77.0, device=DEV)  # slots of a gradient row, one after another
        slot = [row[5 + k * (d + 3):5 + k * (d + 3) + d] for k in range(4)]
        need = ops.residual_norm_grad_workspace(n, d)
        room = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device=DEV)
        got = ops.residual_norm_grad(x, y, dx, dh, gate=gate, dx=dx, dy=dh, dgate=dgate, dw_post=slot[0], db_post=slot[1],
                                     dw_pre=slot[2], db_pre=slot[3], workspace=room[:need], **kw)
        for name in got._fields:
            a, b = getattr(got, name), getattr(want, name)
            check(a, b, ulp(b) * 4 + 2e-5 * n ** 0.5, name + " in place")
        for i in (idx, idh, idg):
            i()
        assert bool((room[need:] == 0xA5).all())
        used = torch.zeros_like(row, dtype=torch.bool)
        for k in range(4):
            used[5 + k * (d + 3):5 + k * (d + 3) + d] = True
        assert bool((row[~used] == 77.0).all())


def test_boundary_without_a_block_and_without_an_arriving_gradient():
    s = boundary_inputs(9, 320, F32, F32, "layer", None, "none", 6)
    x_new, h = ops.residual_norm(s["x"], None, s["w_pre"], s["b_pre"], pre="layer", eps=EPS)
    assert x_new is s["x"]
    want = norm64(wide(s["x"]), "layer", wide(s["w_pre"]), wide(s["b_pre"]), EPS)[0]
    check(h, want, 80 * U * 8 * (1 + want.abs()), "plain norm")
    h16 = ops.residual_norm(s["x"], None, s["w_pre"], s["b_pre"], pre="layer", eps=EPS, h=torch.empty(9, 320, dtype=BF16, device=DEV))[1]
    check(h16, want, 80 * U * 8 * (1 + want.abs()) + BF * want.abs(), "plain norm, bf16")
    got = ops.residual_norm_grad(s["x"], None, None, s["dh"], s["w_pre"], pre="layer", eps=EPS)
    assert got.dy is None and got.dgate is None and got.dw_post is None
    x = wide(s["x"]).requires_grad_()
    out = torch.nn.functional.layer_norm(x, (320,), wide(s["w_pre"]), wide(s["b_pre"]), EPS)
    dx, = torch.autograd.grad(out, x, wide(s["dh"]))
    check(got.dx, dx, 80 * U * 40 * (1 + dx.abs()), "dx of a plain norm")
    none = ops.residual_norm(s["x"][:0], s["y"][:0], s["w_pre"])
    assert none[0].shape == (0, 320) and none[1].shape == (0, 320)
    got = ops.residual_norm_grad(s["x"][:0], s["y"][:0], s["dx"][:0], s["dh"][:0], s["w_pre"])
    assert bool((got.dw_pre == 0).all()) and got.dx.shape == (0, 320)


@pytest.mark.parametrize("pre,post,gate", [("rms", "rms", "element"), ("layer", "layer", "channel")])
def test_boundary_gradient_by_differences(pre, post, gate):
    """f = <dx', x_new> + <dh, h> along a direction of x and of y; the stream handed to the gradient is x_new itself."""
    n, d = 6, 96
    s = boundary_inputs(n, d, F32, F32, pre, post, gate, 12)
    kw = dict(pre=pre, post=post, w_pre=s["w_pre"], w_post=s["w_post"], b_post=s["b_post"], gate=s["gate"], res_scale=SCALE, eps=EPS)
    x_new, _ = ops.residual_norm(s["x"], s["y"], b_pre=s["b_pre"], **kw)
    got = ops.residual_norm_grad(x_new, s["y"], s["dx"], s["dh"], **kw)
    h = 2.0 ** -8
    for name, grad in (("x", got.dx), ("y", got.dy)):
        D = normal(gen(13), n, d)
        f = []
        for sign in (1, -1):
            moved = dict(x=s["x"], y=s["y"])
            moved[name] = moved[name] + sign * h * D
            a, b = ops.residual_norm(moved["x"], moved["y"], b_pre=s["b_pre"], **kw)
            f.append((s["dx"].double() * a.double() + s["dh"].double() * b.double()).sum(1))
        slope = (grad.double() * D.double()).sum(1)
        # f is off by 100 u of its terms; the third derivative of a norm of d values near deviation 1 along D is below 60 |D|_3^3
        size = (s["dx"].abs() * x_new.abs()).sum(1).double() + (s["dh"].abs() * 4).sum(1).double()
        tol = 100 * U * size / h + h * h / 6 * 60 * (D.abs() ** 3).sum(1).double()
        assert bool((((f[0] - f[1]) / (2 * h) - slope).abs() <= tol).all()), name


def test_boundary_a_nan_stays_in_its_row():
    s = boundary_inputs(40, 256, F32, F32, "rms", "rms", "none", 3)
    s["y"][7, 11] = float("nan")
    s["x"][9, 0] = float("inf")
    x_new, h = ops.residual_norm(s["x"], s["y"], s["w_pre"], w_post=s["w_post"], pre="rms", post="rms")
    assert bool(torch.isnan(h[7]).all()) and bool(torch.isnan(h[9, 0]))
    rest = [i for i in range(40) if i not in (7, 9)]
    assert bool(torch.isfinite(h[rest]).all()) and bool(torch.isfinite(x_new[rest]).all())


# --------------------------------------------------------------------------
# how they are called
# --------------------------------------------------------------------------


def _everything(seed):
    """One call of each operator; returns all results."""
    g = gen(seed)
    tok, table = tokens_of("zipf", 600, 3000, g), normal(g, 3000, 128)
    z, t, ids, labels, weight = distill_inputs(30, 3000, 10, BF16, seed)
    s = boundary_inputs(50, 128, F32, BF16, "layer", "rms", "channel", seed)

    def go(stream=None):
        kw = dict(pre="layer", post="rms", w_pre=s["w_pre"], w_post=s["w_post"], gate=s["gate"], stream=stream)
        out = [ops.embed(tok, table, scale=2.0, stream=stream)]
        out.append(ops.embed_grad(tok, out[0], torch.empty_like(table), stream=stream))
        out += ops.distill(z, t, ids, labels=labels, T=2.0, alpha=0.5, beta=0.5, row_weight=weight, stream=stream)
        out += ops.residual_norm(s["x"], s["y"], b_pre=s["b_pre"], **kw)
        out += [v for v in ops.residual_norm_grad(s["x"], s["y"], s["dx"], s["dh"], **kw) if v is not None]
        return out
    return go


def test_other_streams():
    go = _everything(1)
    want = go()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    busy = torch.zeros(1 << 26, device=DEV)
    with torch.cuda.stream(side):
        for _ in range(20):
            busy += 1.0
        first = go()
    by_object, by_address = go(side), go(side.cuda_stream)
    side.synchronize()
    for got in (first, by_object, by_address):
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_graph_capture():
    go = _everything(2)
    want = go()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = go()
    for t in got:
        t.fill_(-1.0)
    graph.replay()
    torch.cuda.synchronize()
    # the captured gradient call reads the captured lookup's result
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_wrong_shapes_and_types_are_refused():
    table, tok = torch.zeros(10, 16, device=DEV), torch.zeros(4, dtype=torch.int64, device=DEV)
    half = torch.zeros(10, 16, dtype=torch.float16, device=DEV)
    vec = torch.ones(16, device=DEV)
    refused = [
        lambda: ops.embed(tok, half), lambda: ops.embed(tok.float(), table), lambda: ops.embed(tok, table.t()),
        lambda: ops.embed(tok, table, out=torch.zeros(3, 16, device=DEV)), lambda: ops.embed(tok.cpu(), table),
        lambda: ops.embed(tok, table, out=torch.zeros(4, 16, device=DEV), out_dtype=BF16),
        lambda: ops.embed_grad(tok, table, torch.zeros(10, 16, device=DEV)),
        lambda: ops.embed_grad(tok, torch.zeros(4, 16, device=DEV), torch.zeros(1, 16, device=DEV).expand(10, 16)),
        lambda: ops.distill(half), lambda: ops.distill(table, table[:, :3], None),
        lambda: ops.distill(table, table[:, :3], torch.zeros(10, 4, dtype=torch.int32, device=DEV)),
        lambda: ops.distill(table, labels=tok), lambda: ops.distill(table, dlogits=table.bfloat16()),
        lambda: ops.distill(table, row_weight=torch.ones(10, dtype=torch.float64, device=DEV)),
        lambda: ops.residual_norm(table, table[:5], vec), lambda: ops.residual_norm(table, table, vec[:8]),
        lambda: ops.residual_norm(table, table, vec, pre="group"), lambda: ops.residual_norm(table, table, vec, pre=None),
        lambda: ops.residual_norm(table, table, vec, gate=table.bfloat16()), lambda: ops.residual_norm(table, table, vec.bfloat16()),
        lambda: ops.residual_norm_grad(table, table, table, table.bfloat16(), vec),
        lambda: ops.residual_norm_grad(table, table, table, table, vec, wgrad_dtype=torch.float16),
    ]
    for k, call in enumerate(refused):
        with pytest.raises(ValueError):
            call()
            pytest.fail("call %d was accepted" % k)
    small = torch.empty(8, dtype=torch.uint8, device=DEV)
    for call in (lambda: ops.embed_grad(tok, torch.zeros(4, 16, device=DEV), table, workspace=small),
                 lambda: ops.residual_norm_grad(table, table, table, table, vec, workspace=small),
                 lambda: ops.residual_norm(table, table, vec, post="rms"),  # no w_post
                 lambda: ops.distill(table, T=0.0)):
        with pytest.raises(AdaScaleError) as e:
            call()
        assert e.value.status == 1


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,alpha,beta", [(1.0, 0.3, 0.7), (2.0, 0.5, 0.5), (4.0, 0.9, 0.1), (1.5, 0.5, 0.5), (3.0, 0.5, 0.5), (1.3, 0.5, 0.5),
                                          (3.0, 1.0, 0.0), (2.0, 0.0, 1.0)])
@pytest.mark.parametrize("n,vocab,k", [(900, 20001, 17), (911, 50257, 64), (890, 90003, 128), (80, 300007, 5)])
def test_distill_many_long_rows(n, vocab, k, T, alpha, beta, dtype):
    """Enough of them that rows stay in shared memory between the two walks; over several blocks where one cannot hold them."""
    z, t, ids, labels, weight = distill_inputs(n, vocab, k, dtype, n + vocab)
    z[5] = float("-inf")
    z[9, 1::2] = float("-inf")
    z[11] = LOWEST[dtype]
    ids[13], labels[13] = -1, -100
    weight[[5, 9, 11, 13]] = 1.0
    ids[17] = ids[17, 0].clone()  # one id all over
    labels[18] = ids[18, 0]
    labels[[19, 20]] = torch.tensor([0, vocab - 1], device=DEV)
    got = ops.distill(z, t, ids, labels=labels, T=T, alpha=alpha, beta=beta, row_weight=weight)
    rows = torch.arange(n, device=DEV).split(100)
    for part in rows:  # the reference's temporaries are large
        check_distill(ops.Distilled(got.row_loss[part].sum(), got.row_loss[part], got.dlogits[part]), z[part], t[part], ids[part],
                      labels[part], T, alpha, beta, weight[part], "long rows")
    assert float(got.loss) == math.inf if bool(torch.isinf(got.row_loss).any()) else \
        abs(float(got.loss.double() - got.row_loss.double().sum())) <= 2 * U * float(got.row_loss.double().abs().sum())
    again = ops.distill(z, t, ids, labels=labels, T=T, alpha=alpha, beta=beta, row_weight=weight)
    assert torch.equal(again.loss, got.loss) and torch.equal(again.dlogits, got.dlogits)
    place = z.clone()
    ops.distill(place, t, ids, labels=labels, T=T, alpha=alpha, beta=beta, row_weight=weight, dlogits=place)
    assert torch.equal(place, got.dlogits)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,alpha,beta", [(1.0, 0.3, 0.7), (2.0, 0.5, 0.5), (1.5, 0.9, 0.1), (1.3, 0.5, 0.5), (4.0, 1.0, 0.0)])
@pytest.mark.parametrize("n,vocab,k", [(3000, 140, 5), (2600, 1000, 128), (2500, 5421, 50), (1300, 9001, 1), (900, 18433, 20)])
def test_distill_many_short_rows(n, vocab, k, T, alpha, beta, dtype):
    test_distill_many_long_rows(n, vocab, k, T, alpha, beta, dtype)


@pytest.mark.parametrize("dtype,vocab", [(BF16, 33001), (F32, 30001), (F32, 40001), (BF16, 3001), (F32, 1001)])
def test_distill_many_long_rows_most_of_them_masked(dtype, vocab):
    """Rows that are skipped between rows that are not; NaN in what is skipped."""
    n, k = 900, 9
    z, t, ids, labels, weight = distill_inputs(n, vocab, k, dtype, 77)
    weight[:] = 0.5
    weight[(torch.arange(n, device=DEV) * 7) % 11 < 8] = 0.0
    z[weight == 0] = float("nan")
    got = ops.distill(z, t, ids, labels=labels, T=2.0, alpha=0.5, beta=0.5, row_weight=weight)
    live = weight != 0
    assert not got.row_loss[~live].any() and not got.dlogits[~live].any()
    check_distill(ops.Distilled(got.row_loss[live].sum(), got.row_loss[live], got.dlogits[live]), z[live], t[live], ids[live], labels[live],
                  2.0, 0.5, 0.5, weight[live], "masked")
    z[3], weight[3] = float("nan"), 1.0
    got = ops.distill(z, t, ids, labels=labels, T=2.0, alpha=0.5, beta=0.5, row_weight=weight)
    assert math.isnan(float(got.row_loss[3])) and bool(torch.isnan(got.dlogits[3]).all()) and not torch.isnan(got.dlogits[4:]).any()
