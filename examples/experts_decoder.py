"""Trains a small decoder with experts and a shared relative position bias against a teacher, with clipped gradients and AdaScale SGD.

    python examples/experts_decoder.py [--steps 200] [--rows 4] [--grad-dtype bf16] [--max-norm 1.0]

As ``distill_decoder.py``, whose teacher, token table, block boundaries and loss it uses.  Between the boundaries a block has
attention whose weights come from ``position_softmax`` - one table of biases by relative position for all blocks - and, side by side
with it, a feed-forward net of experts: a router picks one for each token, the tokens are sorted by expert, and ``expert_matmul``
makes the two products.  torch differentiates what is around the operators, their own gradients are calls inside
``torch.autograd.Function``.  Before AdaScale reads a microbatch's row, ``clip_grads`` clips all of its gradients by
their common norm: those that torch made on the way into their slots, the others in place.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

from distill_decoder import Decoder, Teacher, gradient_rows  # noqa: E402
from paper_2007_05105_b200 import binding as B  # noqa: E402
from paper_2007_05105_b200 import ops  # noqa: E402


class PositionSoftmax(torch.autograd.Function):
    """Causal attention weights with a bias by buckets of the distance back."""

    @staticmethod
    def forward(ctx, scores, table, scale, max_distance):
        how = dict(max_distance=max_distance, bidirectional=False, scale=scale, causal=True)
        probs = ops.position_softmax(scores, table, **how)
        ctx.save_for_backward(probs)
        ctx.how, ctx.buckets = how, table.shape[0]
        return probs

    @staticmethod
    def backward(ctx, dprobs):
        g = ops.position_softmax_grad(*ctx.saved_tensors, dprobs.contiguous(), ctx.buckets, **ctx.how)
        return g.dscores, g.dtable, None, None


class ExpertMatmul(torch.autograd.Function):
    """Rows sorted by expert times their experts' weights, which are kept in 32 bits and multiplied in bf16."""

    @staticmethod
    def forward(ctx, x, w, offsets):
        x, w = x.bfloat16(), w.bfloat16()
        ctx.save_for_backward(x, w, offsets)
        return ops.expert_matmul(x, w, offsets, out_dtype=torch.float32)

    @staticmethod
    def backward(ctx, dy):
        x, w, offsets = ctx.saved_tensors
        g = ops.expert_matmul_grad(dy.bfloat16(), offsets, x=x, w=w, dx_dtype=torch.float32)
        return g.dx, g.dw, None


class ExpertsDecoder(Decoder):
    """Shapes, parameters and one microbatch's passes."""

    BLOCK = ("qkv", "mix", "router", "up", "down")

    def __init__(self, vocab=1024, d=128, layers=2, heads=4, experts=4, buckets=16, max_distance=64, device="cuda", seed=1):
        super().__init__(vocab, d, layers, heads, device, seed)
        self.experts, self.max_distance = experts, max_distance
        self.names, self.params = self.names[:2], self.params[:2]  # token table and first norm; the blocks are others
        shapes = [("bias", (buckets, heads))]
        for i in range(layers):
            shapes += [("qkv%d" % i, (3 * d, d)), ("mix%d" % i, (d, d)), ("router%d" % i, (experts, d)), ("up%d" % i, (experts, 2 * d, d)),
                       ("down%d" % i, (experts, d, 2 * d)), ("post%d" % i, (d,)), ("gate%d" % i, (d,)), ("pre%d" % i, (d,))]
        g = torch.Generator(device=device)
        g.manual_seed(seed + 1)
        for name, shape in shapes:
            if len(shape) > 1:
                p = torch.empty(shape, device=device).normal_(0.0, 0.1 if name == "bias" else shape[-1] ** -0.5, generator=g)
            else:
                p = torch.full(shape, 0.2 if name.startswith("gate") else 1.0, device=device)
            self.names.append(name)
            self.params.append(p)
        self.by = dict(zip(self.names, self.params))

    def block(self, i, h, bias, qkv, mix, router, up, down):
        """Attention and experts side by side; h: [batch, length, d]."""
        b, n, d = h.shape
        q, k, v = (h @ qkv.t()).view(b, n, 3, self.heads, d // self.heads).permute(2, 0, 3, 1, 4)
        weights = self.attention_weights(q @ k.transpose(-1, -2), bias, 1.0 / math.sqrt(d // self.heads))
        attended = (weights @ v).transpose(1, 2).reshape(b, n, d) @ mix.t()
        rows = h.reshape(-1, d)
        share, chosen = torch.softmax(rows @ router.t(), dim=1).max(dim=1)
        order = torch.argsort(chosen, stable=True)
        counts = torch.bincount(chosen, minlength=self.experts)
        offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
        y = self.products(rows[order], up, offsets)
        y = self.products(torch.nn.functional.gelu(y), down, offsets) * share[order, None]
        return attended + torch.zeros_like(rows).index_copy(0, order, y).view(b, n, d)

    def attention_weights(self, scores, bias, scale):
        return PositionSoftmax.apply(scores, bias, scale, self.max_distance)

    def products(self, x, w, offsets):
        return ExpertMatmul.apply(x, w, offsets)

    def _weights(self, i):
        return [self.by["bias"]] + [self.by["%s%d" % (n, i)] for n in self.BLOCK]

    def microbatch(self, text, teacher, slots, max_norm):
        """Loss and gradient norm of the microbatch, as device scalars; its clipped gradients go to ``slots`` (one view per parameter)."""
        slot = dict(zip(self.names, slots))
        by, tok, label = self.by, text[:, :-1].contiguous(), text[:, 1:].contiguous()
        shape = (*tok.shape, self.d)
        wgrad = slots[0].dtype
        # forward
        x = ops.embed(tok, by["table"], scale=self.scale)
        x0, h = ops.residual_norm(x, None, by["first"], pre="rms", eps=self.EPS)
        kept = []
        for i in range(self.layers):
            leaf = h.view(shape).requires_grad_()
            weights = [w.detach().requires_grad_() for w in self._weights(i)]
            with torch.enable_grad():
                y = self.block(i, leaf, *weights)
            x, h = ops.residual_norm(x, y.detach(), **self._boundary(i))
            kept.append((leaf, weights, y, x))
        flat = h.reshape(-1, self.d)
        logits = flat @ by["table"].t()
        n, prev = logits.shape[0], tok.reshape(-1)
        weight = torch.full((n,), 1.0 / n, device=logits.device)
        loss, _, dlogits = ops.distill(logits, teacher.logits[prev], teacher.ids[prev], labels=label.reshape(-1), T=self.T,
                                       alpha=self.ALPHA, beta=self.BETA, row_weight=weight, dlogits=logits)
        # backward: gradients that are not in their slots yet
        loose = {"table": dlogits.t() @ flat}  # the output projection's part of the tied table
        dh, dx = (dlogits @ by["table"]).view(shape), None
        for i in reversed(range(self.layers)):
            leaf, weights, y, x = kept[i]
            g = ops.residual_norm_grad(x, y.detach(), dx, dh, wgrad_dtype=wgrad, dgate=slot["gate%d" % i], dw_post=slot["post%d" % i],
                                       dw_pre=slot["pre%d" % i], **self._boundary(i))
            dx = g.dx
            dh, dbias, *dw = torch.autograd.grad(y, [leaf] + weights, g.dy)
            loose["bias"] = dbias if i == self.layers - 1 else loose["bias"].add_(dbias)
            loose.update(("%s%d" % (name, i), grad) for name, grad in zip(self.BLOCK, dw))
        dx = ops.residual_norm_grad(x0, None, dx, dh, by["first"], pre="rms", eps=self.EPS, wgrad_dtype=wgrad, dw_pre=slot["first"]).dx
        ops.embed_grad(tok, dx, loose["table"], scale=self.scale, accumulate=True)
        norm = ops.clip_grads([loose.get(name, slot[name]) for name in self.names], max_norm, out=slots)
        return loss, norm


def train(steps=200, S=4, batch=8, length=32, grad_dtype="f32", vocab=1024, k=16, lr=0.2, max_norm=1.0, seed=1, every=20, log=print):
    """Returns the losses and gradient norms (means over the S microbatches) and the last AdaScale statistics."""
    teacher = Teacher(vocab, k, "cuda", seed)
    model = ExpertsDecoder(vocab=vocab, seed=seed)
    momentum = [torch.zeros_like(p) for p in model.params]
    rows = gradient_rows(model.params, S, {"f32": torch.float32, "bf16": torch.bfloat16}[grad_dtype])
    ada = B.AdaScale([p.numel() for p in model.params], S, grad_dtype, momentum=0.9)
    sched = B.make_schedule("const", eta0=lr)
    grads_p, params_p, mom_p = B.pointer_array(rows), B.pointer_array(model.params), B.pointer_array(momentum)
    losses, norms = [], []
    with torch.no_grad():
        for step in range(steps):
            loss, norm = (torch.stack(v).mean() for v in zip(*(model.microbatch(teacher.text(batch, length), teacher, row, max_norm) for row in rows)))
            ada.step(grads_p, params_p, mom_p, sched)
            if step % every == 0 or step == steps - 1:
                st = ada.get_gain_tau(True)
                losses.append(float(loss))
                norms.append(float(norm))
                if log:
                    log("step %4d  loss %.4f  gradient norm %.3f  gain %.3f  scale-invariant iterations %.1f" % (step, losses[-1], norms[-1], st.r, st.tau))
    st = ada.get_gain_tau(True)
    ada.close()
    return losses, norms, st


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--rows", type=int, default=4, help="microbatches per iteration (the scale S)")
    ap.add_argument("--grad-dtype", choices=("f32", "bf16"), default="f32")
    ap.add_argument("--lr", type=float, default=0.2)
    ap.add_argument("--max-norm", type=float, default=1.0, help="norm to which a microbatch's gradient is clipped")
    a = ap.parse_args()
    train(a.steps, a.rows, grad_dtype=a.grad_dtype, lr=a.lr, max_norm=a.max_norm)


if __name__ == "__main__":
    main()
