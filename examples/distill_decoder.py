"""Trains a small decoder against a teacher's top logits with AdaScale SGD on one GPU.

    python examples/distill_decoder.py [--steps 200] [--rows 4] [--grad-dtype bf16]

Every iteration runs S microbatches.  Each leaves its gradients in a row of its own - one flat buffer with
a slot per parameter tensor - and ``adascale_step`` makes the step from the S rows.  The operators of
``paper_2007_05105_b200.ops`` do what is neither a matrix product nor attention: the scaled token
lookup, the boundaries between blocks and the distillation loss going forward, and their gradients
coming back, written into the slots.  torch does the blocks (attention and feed-forward in one residual
branch) and differentiates them.

The teacher is a fixed random Markov chain over the vocabulary: for every token it gives the logits of
its most likely successors, which is also what the text is drawn from.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2007_05105_b200 import binding as B  # noqa: E402
from paper_2007_05105_b200 import ops  # noqa: E402


class Teacher:
    """Top-K logits of the next token, one list per token, and text that follows them."""

    def __init__(self, vocab, k, device, seed):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.ids = torch.rand(vocab, vocab, device=device, generator=g).topk(k).indices.int()
        self.logits = torch.empty(vocab, k, device=device).normal_(0.0, 2.0, generator=g).sort(dim=1, descending=True).values
        self.vocab, self.g = vocab, g

    def text(self, batch, length):
        tok = torch.randint(0, self.vocab, (batch, 1), device=self.ids.device, generator=self.g)
        for _ in range(length):
            pick = torch.multinomial(torch.softmax(self.logits[tok[:, -1]], dim=1), 1, generator=self.g)
            tok = torch.cat([tok, self.ids[tok[:, -1]].gather(1, pick).long()], dim=1)
        return tok


class Decoder:
    """Pre- and post-normed decoder with tied token table: shapes, parameters and one microbatch's passes."""

    T, ALPHA, BETA = 2.0, 0.7, 0.3
    EPS = 1e-6

    def __init__(self, vocab=1024, d=128, layers=2, heads=4, device="cuda", seed=1):
        self.vocab, self.d, self.layers, self.heads = vocab, d, layers, heads
        self.scale, self.res_scale = math.sqrt(d), 1.0 / math.sqrt(layers)
        shapes = [("table", (vocab, d)), ("first", (d,))]
        for i in range(layers):
            shapes += [("qkv%d" % i, (3 * d, d)), ("mix%d" % i, (d, d)), ("up%d" % i, (4 * d, d)), ("down%d" % i, (d, 4 * d)),
                       ("post%d" % i, (d,)), ("gate%d" % i, (d,)), ("pre%d" % i, (d,))]
        self.names = [n for n, _ in shapes]
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.params = []
        for name, shape in shapes:
            if len(shape) == 2:
                p = torch.empty(shape, device=device).normal_(0.0, shape[1] ** -0.5, generator=g)
            else:  # norms at 1, layer gates small: blocks come in gradually
                p = torch.full(shape, 0.2 if name.startswith("gate") else 1.0, device=device)
            self.params.append(p)
        self.by = dict(zip(self.names, self.params))

    def block(self, i, h, qkv, mix, up, down):
        """Causal attention and a feed-forward net side by side; h: [batch, length, d]."""
        b, n, d = h.shape
        q, k, v = (h @ qkv.t()).view(b, n, 3, self.heads, d // self.heads).permute(2, 0, 3, 1, 4)
        s = q @ k.transpose(-1, -2) / math.sqrt(d // self.heads)
        s = s.masked_fill(torch.ones(n, n, dtype=torch.bool, device=h.device).triu(1), float("-inf"))
        a = (torch.softmax(s, dim=-1) @ v).transpose(1, 2).reshape(b, n, d)
        return a @ mix.t() + torch.nn.functional.gelu(h @ up.t()) @ down.t()

    def _weights(self, i):
        return [self.by["%s%d" % (n, i)] for n in ("qkv", "mix", "up", "down")]

    def _boundary(self, i):
        return dict(w_pre=self.by["pre%d" % i], w_post=self.by["post%d" % i], gate=self.by["gate%d" % i], pre="rms",
                    post="rms", res_scale=self.res_scale, eps=self.EPS)

    def microbatch(self, text, teacher, slots):
        """Loss of the microbatch, as a device scalar; its gradients go to ``slots`` (one view per parameter)."""
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
        n = logits.shape[0]
        weight = torch.full((n,), 1.0 / n, device=logits.device)
        prev = tok.reshape(-1)
        loss, _, dlogits = ops.distill(logits, teacher.logits[prev], teacher.ids[prev], labels=label.reshape(-1), T=self.T,
                                       alpha=self.ALPHA, beta=self.BETA, row_weight=weight, dlogits=logits)
        # backward
        slot["table"].copy_(dlogits.t() @ flat)   # the output projection's part of the tied table
        dh, dx = (dlogits @ by["table"]).view(shape), None
        for i in reversed(range(self.layers)):
            leaf, weights, y, x = kept[i]
            g = ops.residual_norm_grad(x, y.detach(), dx, dh, wgrad_dtype=wgrad, dgate=slot["gate%d" % i], dw_post=slot["post%d" % i],
                                       dw_pre=slot["pre%d" % i], **self._boundary(i))
            dx = g.dx
            dh, *dw = torch.autograd.grad(y, [leaf] + weights, g.dy)
            for name, grad in zip(("qkv", "mix", "up", "down"), dw):
                slot["%s%d" % (name, i)].copy_(grad)
        dx = ops.residual_norm_grad(x0, None, dx, dh, by["first"], pre="rms", eps=self.EPS, wgrad_dtype=wgrad, dw_pre=slot["first"]).dx
        ops.embed_grad(tok, dx, slot["table"], scale=self.scale, accumulate=True)
        return loss


def gradient_rows(params, S, dtype, align=64):
    """S flat buffers and, in each, a view per parameter at offsets rounded up to ``align`` elements."""
    offsets, end = [], 0
    for p in params:
        offsets.append(end)
        end += -(-p.numel() // align) * align
    flat = [torch.zeros(end, dtype=dtype, device=params[0].device) for _ in range(S)]
    return [[f[o:o + p.numel()].view(p.shape) for o, p in zip(offsets, params)] for f in flat]


def train(steps=200, S=4, batch=8, length=32, grad_dtype="f32", vocab=1024, k=16, lr=0.2, seed=1, every=20, log=print):
    """Returns the losses (mean over the S microbatches) and the last AdaScale statistics."""
    teacher = Teacher(vocab, k, "cuda", seed)
    model = Decoder(vocab=vocab, seed=seed)
    momentum = [torch.zeros_like(p) for p in model.params]
    rows = gradient_rows(model.params, S, {"f32": torch.float32, "bf16": torch.bfloat16}[grad_dtype])
    ada = B.AdaScale([p.numel() for p in model.params], S, grad_dtype, momentum=0.9)
    sched = B.make_schedule("const", eta0=lr)
    grads_p, params_p, mom_p = B.pointer_array(rows), B.pointer_array(model.params), B.pointer_array(momentum)
    losses = []
    with torch.no_grad():
        for step in range(steps):
            loss = torch.stack([model.microbatch(teacher.text(batch, length), teacher, row) for row in rows]).mean()
            ada.step(grads_p, params_p, mom_p, sched)
            if step % every == 0 or step == steps - 1:
                st = ada.get_gain_tau(True)
                losses.append(float(loss))
                if log:
                    log("step %4d  loss %.4f  gain %.3f  scale-invariant iterations %.1f" % (step, losses[-1], st.r, st.tau))
    st = ada.get_gain_tau(True)
    ada.close()
    return losses, st


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--rows", type=int, default=4, help="microbatches per iteration (the scale S)")
    ap.add_argument("--grad-dtype", choices=("f32", "bf16"), default="f32")
    ap.add_argument("--lr", type=float, default=0.2)
    a = ap.parse_args()
    train(a.steps, a.rows, grad_dtype=a.grad_dtype, lr=a.lr)


if __name__ == "__main__":
    main()
