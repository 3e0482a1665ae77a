"""The language-model operators at the edges of what their kernels take: alignments at which one kernel hands over to another,
batches that are mostly padding, arguments that are refused.  Tolerances and helpers are those of test_gpu_ops.py."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

import test_gpu_ops as T  # noqa: E402
from paper_2007_05105_b200 import ops  # noqa: E402

DEV, F32, BF16, U = T.DEV, T.F32, T.BF16, T.U


# --------------------------------------------------------------------------
# block boundary, bf16 on both sides: rows on 16 bytes go through bulk copies, others may not
# --------------------------------------------------------------------------


@pytest.mark.parametrize("pre,post,gate", [("rms", None, "none"), ("layer", "layer", "channel"), ("rms", "layer", "element")])
@pytest.mark.parametrize("n,d", [(6, 1020), (6, 1024), (6, 1028), (6, 1032), (6, 1100), (6, 1276), (6, 1280), (6, 1284), (7200, 1028), (7200, 1280)])
def test_boundary_widths_around_the_widest_row_of_a_warp(pre, post, gate, n, d):
    """n = 7200: blocks that fill an SM and keep the vectors in shared memory."""
    T.test_boundary_and_its_gradient(pre, post, gate, n, d, BF16, BF16)


@pytest.mark.parametrize("pad,shift", [(0, 4), (4, 0), (4, 4), (8, 4), (8, 8), (1, 3)])
@pytest.mark.parametrize("d", [72, 512, 1024, 1028, 1032, 1100, 1276, 1280, 1536])
def test_boundary_bf16_strides_shifts_and_places(d, pad, shift):
    n = 21
    for pre, post, kind in (("layer", "layer", "element"), ("rms", None, "none")):
        s = T.boundary_inputs(n, d, BF16, BF16, pre, post, kind, 14)
        kw = dict(pre=pre, post=post, w_pre=s["w_pre"], b_pre=s["b_pre"], w_post=s["w_post"], b_post=s["b_post"], res_scale=T.SCALE, eps=T.EPS)
        want = ops.residual_norm(s["x"], s["y"], gate=s["gate"], **kw)
        x, ix = T.strided(s["x"], pad, shift)
        y, iy = T.strided(s["y"], pad, shift)
        gate, ig = T.strided(s["gate"], pad, shift) if s["gate"] is not None else (None, lambda: None)
        got = ops.residual_norm(x, y, gate=gate, x_new=x, h=y, **kw)
        assert got[0] is x and got[1] is y
        # kernels that add in another order: results one rounding apart
        near = lambda t: 2 * T.rounding(BF16) * t.double().abs() + 64 * U * (1 + t.double().abs())  # noqa: E731
        T.check(x, want[0], near(want[0]), "x in place")
        T.check(y, want[1], near(want[1]), "h in place")
        for intact in (ix, iy, ig):
            intact()
    # the norm alone
    x, ix = T.strided(s["x"], pad, shift)
    h, ih = T.empty_strided_out(n, d, BF16, pad, shift)
    ops.residual_norm(x, None, s["w_pre"], pre="rms", eps=T.EPS, h=h)
    want = T.norm64(T.wide(s["x"]), "rms", T.wide(s["w_pre"]), None, T.EPS)[0]
    T.check(h, want, 80 * U * 8 * (1 + want.abs()) + T.BF * want.abs(), "norm alone")
    ix(), ih()


# --------------------------------------------------------------------------
# embedding gradient: batches of which most tokens have no part in it
# --------------------------------------------------------------------------


@pytest.mark.parametrize("dout_t,grad_t", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("n,kept,vocab,d", [(4099, 99, 32768, 512), (1200, 60, 5, 8), (1200, 3, 5, 7), (2000, 1000, 300, 1), (33000, 17, 900, 24),
                                            (33000, 33, 2, 16), (9001, 9000, 50257, 64), (40, 9, 3, 1024), (5000, 0, 70, 40)])
def test_embed_grad_of_a_batch_that_is_mostly_padding(n, kept, vocab, d, dout_t, grad_t):
    """Padding that fills windows, blocks and whole walks behind the tokens' last run; half of it by ids outside the table.  The same
    list without a token that counts goes first, on the same multiprocessors."""
    g = T.gen(n + kept)
    tok = torch.full((n,), vocab - 1, device=DEV)  # the padding token
    tok[1::2] = torch.randint(vocab, 2 * vocab, (n // 2,), device=DEV, generator=g)
    nothing = tok.clone()
    at = torch.randperm(n, device=DEV, generator=g)[:kept]
    tok[at] = torch.randint(0, vocab, (kept,), device=DEV, generator=g)
    dout = T.normal(g, n, d, dtype=dout_t)
    for ids, accumulate in ((torch.int64, False), (torch.int32, True)):
        base = T.normal(g, vocab, d, dtype=grad_t) if accumulate else torch.zeros(vocab, d, dtype=grad_t, device=DEV)
        grad = base.clone()
        ops.embed_grad(nothing.to(ids), dout, grad, scale=1.7, padding_idx=vocab - 1, accumulate=accumulate)
        assert torch.equal(grad, base)
        ops.embed_grad(tok.to(ids), dout, grad, scale=1.7, padding_idx=vocab - 1, accumulate=accumulate)
        T.embed_grad_check(tok, dout, grad, base, 1.7, vocab - 1, accumulate, "mostly padding")


# --------------------------------------------------------------------------
# arguments
# --------------------------------------------------------------------------


def test_a_workspace_that_cannot_be_one_is_refused():
    """On the host, of another type, with gaps: refused before anything is enqueued, results untouched."""
    n, vocab, d = 40, 30, 16
    tok, dout = torch.zeros(n, dtype=torch.int64, device=DEV), torch.ones(n, d, device=DEV)
    x, vec = torch.ones(n, d, device=DEV), torch.ones(d, device=DEV)
    need = max(ops.embed_grad_workspace(n, d), ops.residual_norm_grad_workspace(n, d))
    good = torch.empty(need, dtype=torch.uint8, device=DEV)
    for bad in (torch.empty(need, dtype=torch.uint8), torch.empty(need, dtype=torch.float32, device=DEV),
                torch.empty(2 * need, dtype=torch.uint8, device=DEV)[::2], torch.empty(2, need, dtype=torch.uint8, device=DEV)[:, :need // 2 + 8]):
        grad, dw = torch.full((vocab, d), 5.0, device=DEV), torch.full((d,), 5.0, device=DEV)
        with pytest.raises(ValueError):
            ops.embed_grad(tok, dout, grad, workspace=bad)
        with pytest.raises(ValueError):
            ops.residual_norm_grad(x, None, None, x, vec, dw_pre=dw, workspace=bad)
        assert bool((grad == 5.0).all()) and bool((dw == 5.0).all())
    with pytest.raises(TypeError):
        ops.embed_grad(tok, dout, grad, workspace=need)
    ops.embed_grad(tok, dout, grad, workspace=good)
    assert bool((grad[0] == n).all()) and not grad[1:].any()
    ops.residual_norm_grad(x, None, None, x, vec, dw_pre=dw, workspace=good.view(2, -1))


# --------------------------------------------------------------------------
# distillation: a teacher's list that is not finite
# --------------------------------------------------------------------------


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,vocab,k", [(3, 5003, 6), (900, 5003, 6), (900, 20001, 40), (900, 50257, 6), (3, 5003, 200)])
def test_distill_a_teacher_that_is_not_finite(n, vocab, k, dtype, bad):
    """Rows read twice and rows kept in shared memory: the loss, and the gradient where the list names an entry, are NaN; the rest is
    as if the list had been finite; other rows do not notice."""
    z, t, ids, labels, _ = T.distill_inputs(n, vocab, k, dtype, 31)
    ids[:] = torch.arange(k, device=DEV, dtype=ids.dtype) * 7 + 3
    ids[:, -1] = ids[:, 0]    # named twice
    ids[:, 2] = -1            # not an entry: its logit is not looked at
    t[:, 2] = bad
    labels[:] = 11            # no 7 m + 3
    labels[0] = 3             # in the list
    at = dict(labels=labels, T=2.0, alpha=0.5, beta=0.5)
    want = ops.distill(z, t, ids, **at)
    assert not torch.isnan(want.row_loss).any() and not torch.isnan(want.dlogits).any()
    t[:2, 1] = bad
    got = ops.distill(z, t, ids, **at)
    named = torch.zeros(n, vocab, dtype=torch.bool, device=DEV)
    named[:2, ids[0, ids[0] >= 0].long()] = True
    assert torch.equal(torch.isnan(got.dlogits), named)
    assert bool(torch.isnan(got.row_loss[:2]).all()) and bool(torch.isnan(got.loss))
    assert torch.equal(got.row_loss[2:], want.row_loss[2:]) and torch.equal(got.dlogits[~named], want.dlogits[~named])


def test_tensors_that_are_written_to_say_so():
    """torch's version counters: up by each call that writes to a given tensor, not by one that only reads it or is refused."""
    n, d = 8, 16
    tok = torch.arange(n, device=DEV)
    m = lambda: torch.ones(n, d, device=DEV)  # noqa: E731
    v = lambda: torch.ones(d, device=DEV)  # noqa: E731
    x, y, dx, dh, w, out, grad, z, gate = m(), m(), m(), m(), v(), m(), m(), m(), v()
    gx, gy, ge, gw = m(), m(), m(), [v() for _ in range(5)]
    calls = [
        (lambda: ops.embed(tok, x, out=out), [out], [x, tok]),
        (lambda: ops.embed_grad(tok, dx, grad), [grad], [dx]),
        (lambda: ops.distill(z, labels=tok, alpha=0.0, beta=1.0, dlogits=z), [z], [tok]),
        (lambda: ops.distill(z, labels=tok, alpha=0.0, beta=1.0), [], [z]),
        (lambda: ops.residual_norm(x, y, w, gate=gate, x_new=x, h=y), [x, y], [w, gate]),
        (lambda: ops.residual_norm(x, None, w, h=out), [out], [x, w]),
        (lambda: ops.residual_norm_grad(x, y, dx, dh, w, w, w, pre="layer", post="layer", gate=gate, dx=dx, dy=dh, dgate=gw[0], dw_post=gw[1],
                                        db_post=gw[2], dw_pre=gw[3], db_pre=gw[4]), [dx, dh] + gw, [x, y, w, gate]),
        (lambda: ops.residual_norm_grad(x, y, dx, dh, w, gate=y, dx=gx, dy=gy, dgate=ge, dw_pre=gw[0]), [gx, gy, ge, gw[0]], [x, y, dx, dh, gw[1]]),
    ]
    for k, (call, writes, reads) in enumerate(calls):
        before = [t._version for t in writes + reads]
        call()
        assert [t._version - b for t, b in zip(writes + reads, before)] == [1] * len(writes) + [0] * len(reads), k
    row = torch.zeros(4 * d, device=DEV)  # a slot is part of its row
    ops.residual_norm_grad(x, None, None, dh, w, dw_pre=row[d:2 * d])
    assert row._version == 1
    with pytest.raises(ValueError):
        ops.embed(tok, x, out=out[:3])
    with pytest.raises(ops.AdaScaleError):
        ops.distill(z, T=0.0, dlogits=z)
    assert out._version == 2 and z._version == 1
    # what torch's own check makes of it
    leaf = m().requires_grad_()
    kept = leaf * 2.0
    loss = (kept * kept).sum()
    ops.embed(tok, x, out=kept.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    with torch.inference_mode():
        ops.embed(tok, x, out=m())


def test_flags_without_a_truth_value_are_refused():
    class Neither:
        def __bool__(self):
            raise KeyError("neither")

    tok, z = torch.zeros(3, dtype=torch.int64, device=DEV), torch.zeros(3, 8, device=DEV)
    grad = torch.full((4, 8), 5.0, device=DEV)
    for flag, error in ((Neither(), KeyError), (torch.zeros(2), RuntimeError)):
        with pytest.raises(error):
            ops.embed_grad(tok, z, grad, accumulate=flag)
        with pytest.raises(error):
            ops.distill(z, labels=tok, alpha=0.0, beta=1.0, want_grad=flag)
    assert bool((grad == 5.0).all())


def test_leading_dimensions_that_are_not_one():
    """Rows at a common stride are taken, whatever the dimensions before the last; others are refused as a wrong shape."""
    tok = torch.randint(0, 9, (2, 5), device=DEV)
    table, w = T.normal(T.gen(3), 9, 16), torch.ones(16, device=DEV)
    wider, longer = torch.zeros(2, 5, 24, device=DEV)[..., :16], torch.zeros(2, 8, 16, device=DEV)[:, :5]
    assert torch.equal(ops.embed(tok, table, out=wider), table[tok])
    assert torch.equal(ops.residual_norm(wider, None, w)[1], ops.residual_norm(wider.contiguous(), None, w)[1])
    for call in (lambda: ops.embed(tok, table, out=longer), lambda: ops.embed_grad(tok, longer, torch.zeros(9, 16, device=DEV)),
                 lambda: ops.distill(longer), lambda: ops.distill(wider, dlogits=longer), lambda: ops.residual_norm(longer, longer, w),
                 lambda: ops.residual_norm_grad(longer, None, None, wider, w), lambda: ops.residual_norm_grad(wider, None, longer, wider, w)):
        with pytest.raises(ValueError, match="common stride"):
            call()


def test_a_stream_of_another_device_is_refused():
    """It would leave the tensors' device on its own current stream."""
    class Elsewhere:
        device = torch.device("cuda", DEV.index + 1)

    side = torch.cuda.Stream()
    with pytest.raises(ValueError, match="the stream is on cuda:0"):
        ops._on(side, Elsewhere())
    with pytest.raises(ValueError):
        ops.embed(torch.zeros(3, dtype=torch.int64), torch.zeros(4, 8), stream=side)  # tensors on the host
    with ops._on(side, torch.zeros(1, device=DEV)):
        assert torch.cuda.current_stream() == side


# --------------------------------------------------------------------------
# embedding gradient: what is added to is below the normal range
# --------------------------------------------------------------------------


@pytest.mark.parametrize("grad_t", [F32, BF16])
@pytest.mark.parametrize("d", [7, 64])
@pytest.mark.parametrize("n", [5, 4000])
def test_embed_grad_added_to_subnormal_values(n, d, grad_t):
    """Off by less than the least normal number where a token points, the same bits elsewhere; normal results unaffected."""
    g = T.gen(n + d)
    vocab, least = 40, 2.0 ** -126
    base = (T.normal(g, vocab, d) * 2.0 ** -130).to(grad_t)
    assert bool(((base != 0) & (base.double().abs() < least)).any())
    tok = torch.randint(0, vocab // 2, (n,), device=DEV, generator=g)
    dout = T.normal(g, n, d)
    dout[:, 0] = 0.0
    dout[:, 1] *= 2.0 ** -128
    grad = base.clone()
    ops.embed_grad(tok, dout, grad, accumulate=True)
    sums = torch.zeros(vocab, d, dtype=torch.float64, device=DEV).index_add_(0, tok, dout.double())
    mag = torch.zeros_like(sums).index_add_(0, tok, dout.double().abs())
    want = base.double() + sums
    # 128 terms in a row and the joins as in embed_grad_check; operand, result and their sum may each lose a subnormal part
    T.check(grad, want, mag * (128 + n / 256 + 45) * U + want.abs() * T.rounding(grad_t) + 2 * least, "subnormal")
    assert torch.equal(grad[vocab // 2:], base[vocab // 2:])
