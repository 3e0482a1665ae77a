"""Cases for timing and checking the language-model operators of ``paper_2007_05105_b200.ops``.

Three operators at the ends and along the residual path of a Transformer whose gradients the
AdaScale step consumes: the scaled embedding lookup with its gradient by sorted tokens, the
distillation loss against a teacher's top logits with its gradient, and the block boundary (norm
of a block's output, gate, residual scale, norm of the stream for the next block) with its
gradient.  Each has a plain form here, in elementary torch operations in 32 bits, and a 64-bit
form in ``exact``.  Sizes are those of the Transformer-base and decoder tensor lists in
``synthetic.py`` (width 512 and 1024, vocabularies 32768, 50257 and 16384, 1024 positions) or generic.
"""
import math

import torch

own = False

F32, BF16 = "f32", "bf16"
_DTYPE = {F32: torch.float32, BF16: torch.bfloat16}
_BYTES = {F32: 4, BF16: 2}


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------


def listed():
    return [
        # one sequence of the decoder enters the network: master weights in, activations out
        dict(name="embed_sequence", op="embed", N=1024, V=50257, d=1024, table=F32, out=BF16, ids="i64"),
        # a microbatch of 128 sequences of 512 tokens at Transformer-base width, all in 32 bits
        dict(name="embed_batch", op="embed", N=65536, V=32768, d=512, table=F32, out=F32, ids="i64"),
        # the token table's slot of one bf16 gradient row, for 32 sequences of 1024 tokens
        dict(name="embed_grad_batch", op="embed_grad", N=32768, V=50257, d=1024, dout=BF16, grad=BF16, ids="i64",
             pad=False, accumulate=False),
        # tied table: the lookup's part is added to what the output projection already left in the
        # row; a ragged batch with padding tokens
        dict(name="embed_grad_tied", op="embed_grad", N=4099, V=32768, d=512, dout=F32, grad=F32, ids="i32",
             pad=True, accumulate=True),
        # a few rows: the last microbatch of an epoch, or one short prompt with its answer
        dict(name="distill_few_rows", op="distill", N=16, V=50257, K=8, T=2.0, alpha=0.5, beta=0.5, z=BF16,
             masked=0.0, grad=True),
        # evaluation of the loss alone at a high temperature, no labels
        dict(name="distill_eval", op="distill", N=1000, V=16384, K=20, T=4.0, alpha=1.0, beta=0.0, z=F32,
             masked=0.0, grad=False),
        # Transformer-base training, 32-bit logits, padded target positions weigh nothing
        dict(name="distill_transformer", op="distill", N=2048, V=32768, K=32, T=1.0, alpha=0.7, beta=0.3, z=F32,
             masked=0.1, grad=True),
        # decoder training, 8 sequences of 1024 tokens, odd vocabulary
        dict(name="distill_decoder", op="distill", N=8192, V=50257, K=64, T=2.0, alpha=0.5, beta=0.5, z=BF16,
             masked=0.0, grad=True),
        # one token of a generation
        dict(name="boundary_token", op="boundary", N=1, d=1024, x=BF16, y=BF16, pre="rms", post="rms", gate="none"),
        # a training microbatch of the decoder, layer norms, one gate per channel
        dict(name="boundary_batch", op="boundary", N=16384, d=1024, x=F32, y=BF16, pre="layer", post="layer",
             gate="channel"),
        # its gradient
        dict(name="boundary_grad_batch", op="boundary_grad", N=16384, d=1024, x=F32, y=BF16, pre="layer",
             post="layer", gate="channel", wgrad=BF16),
        # a ragged number of rows of an odd width, gates from a projection
        dict(name="boundary_grad_odd", op="boundary_grad", N=1777, d=509, x=F32, y=F32, pre="rms", post="rms",
             gate="element", wgrad=F32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A model width: mostly a multiple of 8, now and then any number."""
    d = _log_int(rng, lo, hi)
    return d if rng.random() < 0.25 else max(8, d // 8 * 8)


def _rows(rng, hi, most):
    """A number of rows, of at most `most`."""
    return max(1, min(_log_int(rng, 1, hi), int(most)))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "distill", "boundary", "boundary_grad"])
    any_type = lambda: rng.choice([F32, BF16])  # noqa: E731
    if op in ("embed", "embed_grad"):
        d = _width(rng, 64, 2048)
        V = _log_int(rng, 1000, min(131072, 100_000_000 // d))
        N = _rows(rng, 65536, 67_000_000 / d)
        c = dict(op=op, N=N, V=V, d=d, ids=rng.choice(["i64", "i32"]))
        if op == "embed":
            return dict(c, table=any_type(), out=any_type())
        return dict(c, dout=any_type(), grad=any_type(), pad=rng.random() < 0.5, accumulate=rng.random() < 0.5)
    if op == "distill":
        z = any_type()
        V = _log_int(rng, 1000, 131072)
        N = _rows(rng, 8192, 1.6e9 / (2 * V * _BYTES[z]))
        alpha = rng.choice([0.0, 0.5, 0.9, 1.0])
        return dict(op=op, N=N, V=V, K=_log_int(rng, 1, 128), T=rng.choice([1.0, 1.5, 2.0, 3.0, 4.0]), alpha=alpha,
                    beta=1.0 - alpha, z=z, masked=rng.choice([0.0, 0.25]), grad=rng.random() < 0.75)
    d = _width(rng, 64, 8192)
    c = dict(op=op, N=_rows(rng, 65536, 33_000_000 / d), d=d, x=any_type(), y=any_type(),
             pre=rng.choice(["rms", "layer"]), post=rng.choice(["none", "rms", "layer"]),
             gate=rng.choice(["none", "channel", "element"]))
    return dict(c, wgrad=any_type()) if op == "boundary_grad" else c


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

_PAD = 1  # the padding token of a batch that has one


def _token_probs(V):
    """Token frequencies fall off like 1 / (rank + 2.7), as in running text."""
    p = 1.0 / (torch.arange(V, dtype=torch.float64) + 2.7)
    return p / p.sum()


def _tokens(case, gen):
    """Token ids of a batch: frequency ranks spread over the table; a padded batch ends in padding."""
    N, V = case["N"], case["V"]
    cdf = _token_probs(V).cuda().cumsum(0)
    rank = torch.searchsorted(cdf, torch.rand(N, dtype=torch.float64, device="cuda", generator=gen)).clamp_(max=V - 1)
    ids = torch.randperm(V, device="cuda", generator=gen)[rank]
    if case.get("pad"):
        ids[N - N // 8:] = _PAD
    return ids.to(torch.int64 if case["ids"] == "i64" else torch.int32)


def _normal(gen, *shape, dtype=torch.float32, std=1.0, mean=0.0):
    t = torch.empty(*shape, dtype=torch.float32, device="cuda")
    return t.normal_(mean, std, generator=gen).to(dtype)


def _prepare_embed(case, gen):
    s = dict(tokens=_tokens(case, gen), scale=math.sqrt(case["d"]))
    if case["op"] == "embed":
        s["table"] = _normal(gen, case["V"], case["d"], dtype=_DTYPE[case["table"]], std=case["d"] ** -0.5)
        s["out_dtype"] = _DTYPE[case["out"]]
        return s
    s["dout"] = _normal(gen, case["N"], case["d"], dtype=_DTYPE[case["dout"]], std=1e-3)
    s["pad"] = _PAD if case["pad"] else -1
    s["accumulate"] = case["accumulate"]
    # the table's slot of the gradient row; with a tied table it holds the output projection's part
    if case["accumulate"]:
        s["grad"] = _normal(gen, case["V"], case["d"], dtype=_DTYPE[case["grad"]], std=1e-3)
    else:
        s["grad"] = torch.empty(case["V"], case["d"], dtype=_DTYPE[case["grad"]], device="cuda")
    return s


def _prepare_distill(case, gen):
    N, V, K = case["N"], case["V"], case["K"]
    z = _normal(gen, N, V, std=2.0)
    # the teacher's list: ids without repetition (one from each of K equal parts of the vocabulary,
    # in shuffled order), logits falling off from the first; the student has learned some of it
    part = V // K
    shuffle = torch.rand(N, K, device="cuda", generator=gen).argsort(dim=1)
    ids = shuffle * part + torch.randint(0, part, (N, K), device="cuda", generator=gen)
    t = 14.0 - 2.0 * torch.log1p(torch.arange(K, device="cuda", dtype=torch.float32)) + _normal(gen, N, K, std=0.3)
    z.scatter_(1, ids, 0.8 * t + _normal(gen, N, K, std=0.5))
    # labels: mostly among the teacher's first, some elsewhere, a few positions without one
    pick = torch.rand(N, device="cuda", generator=gen)
    labels = torch.where(pick < 0.7, ids[:, 0], torch.randint(0, V, (N,), device="cuda", generator=gen))
    labels = torch.where(pick > 0.97, torch.full_like(labels, -100), labels)
    # lists of different lengths, filled up with -1
    length = torch.randint(max(1, K // 2), K + 1, (N, 1), device="cuda", generator=gen)
    ids = torch.where(torch.arange(K, device="cuda") < length, ids, torch.full_like(ids, -1))
    weight = torch.ones(N, device="cuda")
    masked = int(case["masked"] * N)
    if masked:
        weight[torch.randperm(N, device="cuda", generator=gen)[:masked]] = 0.0
    weight /= N - masked
    return dict(logits=z.to(_DTYPE[case["z"]]), t=t, ids=ids.to(torch.int32), labels=labels if case["beta"] else None,
                weight=weight, T=case["T"], alpha=case["alpha"], beta=case["beta"], grad=case["grad"])


def _prepare_boundary(case, gen):
    N, d = case["N"], case["d"]
    xt, yt = _DTYPE[case["x"]], _DTYPE[case["y"]]
    layer = {"none": False, "rms": False, "layer": True}
    s = dict(pre=case["pre"], post=case["post"], res_scale=0.7, eps=1e-5)
    s["x"] = _normal(gen, N, d, dtype=xt, std=2.0)      # the stream before the block, after it for the gradient
    s["y"] = _normal(gen, N, d, dtype=yt, std=0.5, mean=0.05)
    s["w_pre"] = _normal(gen, d, std=0.1, mean=1.0)
    s["b_pre"] = _normal(gen, d, std=0.1) if layer[case["pre"]] else None
    s["w_post"] = None if case["post"] == "none" else _normal(gen, d, std=0.1, mean=1.0)
    s["b_post"] = _normal(gen, d, std=0.1) if layer[case["post"]] else None
    s["gate"] = {"none": lambda: None, "channel": lambda: _normal(gen, d, std=0.2, mean=0.5),
                 "element": lambda: _normal(gen, N, d, dtype=yt)}[case["gate"]]()
    if case["op"] == "boundary_grad":
        s["dx"] = _normal(gen, N, d, dtype=xt, std=1e-2)
        s["dh"] = _normal(gen, N, d, dtype=yt, std=1e-2)
        s["wgrad"] = case["wgrad"]
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 1000003 + 17)
    maker = {"e": _prepare_embed, "d": _prepare_distill, "b": _prepare_boundary}[case["op"][0]]
    return dict(maker(case, gen), op=case["op"])


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------


def _plain_embed(s):
    return {"out": (s["table"][s["tokens"]].float() * s["scale"]).to(s["out_dtype"])}


def _plain_embed_grad(s):
    tok, grad = s["tokens"], s["grad"]
    dy = s["dout"].float() * (s["scale"] * (tok != s["pad"]))[:, None]
    if s["accumulate"] and grad.dtype == torch.float32:
        return {"grad": grad.index_add_(0, tok, dy)}
    total = grad.float() if s["accumulate"] else torch.zeros(grad.shape, device="cuda")
    total.index_add_(0, tok, dy)
    return {"grad": grad.copy_(total) if s["accumulate"] else total.to(grad.dtype)}


def _plain_distill(s):
    z, T, alpha, beta, w = s["logits"].float(), s["T"], s["alpha"], s["beta"], s["weight"]
    N = z.shape[0]
    loss, dz = torch.zeros(N, device="cuda"), None
    top = z.max(dim=1, keepdim=True).values
    rows = torch.arange(N, device="cuda")
    if alpha:
        valid = s["ids"] >= 0
        ids = s["ids"].long().clamp(min=0)
        t = torch.where(valid, s["t"], float("-inf"))
        q = torch.exp((t - t.max(dim=1, keepdim=True).values) / T)
        q = q / q.sum(dim=1, keepdim=True)
        e = torch.exp((z - top) / T)
        total = e.sum(dim=1, keepdim=True)
        log_p = (z.gather(1, ids) - top) / T - torch.log(total)
        log_q = torch.log(torch.where(q > 0, q, 1.0))
        loss += alpha * T * T * (q * (log_q - log_p)).sum(dim=1)
        if s["grad"]:
            dz = e.mul_(alpha * T / total).scatter_add_(1, ids, -alpha * T * q)
    if beta:
        has = (s["labels"] >= 0).float()
        label = s["labels"].clamp(min=0)
        e = torch.exp(z - top)
        total = e.sum(dim=1, keepdim=True)
        loss += beta * has * (torch.log(total) - (z[rows, label][:, None] - top))[:, 0]
        if s["grad"]:
            e.mul_(beta * has[:, None] / total)
            e[rows, label] -= beta * has
            dz = e if dz is None else dz.add_(e)
    loss = loss * w
    return dict(loss=loss.sum(), row_loss=loss, **({"dlogits": dz.mul_(w[:, None]).to(s["logits"].dtype)} if s["grad"] else {}))


def _plain_stats(v, kind, eps):
    """(v - mean) / deviation and 1 / deviation of each row."""
    if kind == "layer":
        v = v - v.mean(dim=1, keepdim=True)
    r = torch.rsqrt((v * v).mean(dim=1, keepdim=True) + eps)
    return v * r, r


def _plain_scaled(n, w, b):
    n = n if w is None else n * w
    return n if b is None else n + b


def _plain_gate(s):
    g = s["gate"]
    return 1.0 if g is None else g if g.dim() == 1 else 1.0 / (1.0 + torch.exp(-g.float()))


def _plain_boundary(s):
    u = s["y"].float()
    if s["post"] != "none":
        u = _plain_scaled(_plain_stats(u, s["post"], s["eps"])[0], s["w_post"], s["b_post"])
    x = s["x"].float() + s["res_scale"] * _plain_gate(s) * u
    h = _plain_scaled(_plain_stats(x, s["pre"], s["eps"])[0], s["w_pre"], s["b_pre"])
    return {"x": x.to(s["x"].dtype), "h": h.to(s["y"].dtype)}


def _plain_norm_grad(dn, n, r, kind):
    """Gradient of v from that of n = (v - mean) / deviation."""
    g = dn - n * (dn * n).mean(dim=1, keepdim=True)
    return r * (g - dn.mean(dim=1, keepdim=True) if kind == "layer" else g)


def _plain_boundary_grad(s):
    wt = _DTYPE[s["wgrad"]]
    y, dh, gate = s["y"].float(), s["dh"].float(), _plain_gate(s)
    n, r = _plain_stats(s["x"].float(), s["pre"], s["eps"])
    dx = s["dx"].float() + _plain_norm_grad(dh * s["w_pre"], n, r, s["pre"])
    out = {"dx": dx.to(s["x"].dtype), "dw_pre": (dh * n).sum(dim=0).to(wt)}
    if s["pre"] == "layer":
        out["db_pre"] = dh.sum(dim=0).to(wt)
    u = y
    if s["post"] != "none":
        n, r = _plain_stats(y, s["post"], s["eps"])
        u = _plain_scaled(n, s["w_post"], s["b_post"])
    ds = s["res_scale"] * dx
    if s["gate"] is not None:
        dg = ds * u
        out["dgate"] = dg.sum(dim=0).to(wt) if s["gate"].dim() == 1 else (dg * gate * (1.0 - gate)).to(s["gate"].dtype)
    du = ds * gate
    if s["post"] != "none":
        out["dw_post"] = (du * n).sum(dim=0).to(wt)
        if s["post"] == "layer":
            out["db_post"] = du.sum(dim=0).to(wt)
        du = _plain_norm_grad(du * s["w_post"], n, r, s["post"])
    out["dy"] = du.to(s["y"].dtype)
    return out


def _own(s):
    from paper_2007_05105_b200 import ops

    if s["op"] == "embed":
        return {"out": ops.embed(s["tokens"], s["table"], scale=s["scale"], out_dtype=s["out_dtype"])}
    if s["op"] == "embed_grad":
        return {"grad": ops.embed_grad(s["tokens"], s["dout"], s["grad"], scale=s["scale"], padding_idx=s["pad"],
                                       accumulate=s["accumulate"])}
    if s["op"] == "distill":
        r = ops.distill(s["logits"], s["t"], s["ids"], labels=s["labels"], T=s["T"], alpha=s["alpha"], beta=s["beta"],
                        row_weight=s["weight"], want_grad=s["grad"])
        return dict(loss=r.loss, row_loss=r.row_loss, **({"dlogits": r.dlogits} if s["grad"] else {}))
    norm = dict(pre=s["pre"], post=s["post"], w_pre=s["w_pre"], w_post=s["w_post"], gate=s["gate"],
                res_scale=s["res_scale"], eps=s["eps"])
    if s["op"] == "boundary":
        x, h = ops.residual_norm(s["x"], s["y"], b_pre=s["b_pre"], b_post=s["b_post"], **norm)
        return {"x": x, "h": h}
    g = ops.residual_norm_grad(s["x"], s["y"], s["dx"], s["dh"], b_post=s["b_post"], wgrad_dtype=_DTYPE[s["wgrad"]], **norm)
    return {k: v for k, v in g._asdict().items() if v is not None}


def run(state):
    if own:
        return _own(state)
    return {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "distill": _plain_distill,
            "boundary": _plain_boundary, "boundary_grad": _plain_boundary_grad}[state["op"]](state)


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------


def _distinct(case):
    """Expected number of different tokens in the batch."""
    n = case["N"] - (case["N"] // 8 if case.get("pad") else 0)
    return float((1.0 - (1.0 - _token_probs(case["V"])) ** n).sum())


def work(case):
    op, N = case["op"], case["N"]
    if op in ("embed", "embed_grad"):
        V, d = case["V"], case["d"]
        ids = N * (8 if case["ids"] == "i64" else 4)
        if op == "embed":
            return {"bytes": ids + _distinct(case) * d * _BYTES[case["table"]] + N * d * _BYTES[case["out"]], "flops": N * d}
        read = N - (N // 8 if case["pad"] else 0)  # rows of padding tokens need not be read
        rows = 2 * _distinct(case) if case["accumulate"] else V
        return {"bytes": ids + read * d * _BYTES[case["dout"]] + rows * d * _BYTES[case["grad"]], "flops": 2 * read * d}
    if op == "distill":
        V, K, b = case["V"], case["K"], _BYTES[case["z"]]
        live = N - int(case["masked"] * N)
        small = live * K * 8 + N * (8 + (8 if case["beta"] else 0))
        exps = (1 if case["alpha"] else 0) + (1 if case["beta"] else 0)
        exps = 1 if case["T"] == 1.0 else exps
        return {"bytes": live * V * b + (N * V * b if case["grad"] else 0) + small,
                "flops": live * V * (1 + 4 * exps + (2 * exps if case["grad"] else 0))}
    d, x, y = case["d"], _BYTES[case["x"]], _BYTES[case["y"]]
    vectors = 1 + (case["post"] != "none") + (case["pre"] == "layer") + (case["post"] == "layer") + (case["gate"] == "channel")
    if op == "boundary":
        gate = y if case["gate"] == "element" else 0
        return {"bytes": N * d * (2 * x + 2 * y + gate) + 4 * d * vectors, "flops": 16 * N * d}
    gate = 2 * y if case["gate"] == "element" else 0
    return {"bytes": N * d * (3 * x + 3 * y + gate) + d * vectors * (4 + _BYTES[case["wgrad"]]), "flops": 40 * N * d}


# --------------------------------------------------------------------------
# the operators in 64 bits
# --------------------------------------------------------------------------


def _exact_embed_grad(s):
    order = torch.argsort(s["tokens"], stable=True)
    tok = s["tokens"][order].long()
    running = torch.cumsum(s["dout"][order].double(), dim=0)
    last = torch.ones_like(tok, dtype=torch.bool)
    last[:-1] = tok[1:] != tok[:-1]
    ends = running[last]
    ends[1:] -= running[last][:-1]
    present = tok[last]
    keep = present != s["pad"]
    grad = s["grad"].double() if s["accumulate"] else torch.zeros(s["grad"].shape, dtype=torch.float64, device="cuda")
    grad[present[keep]] += s["scale"] * ends[keep]
    return {"grad": grad}


def _exact_distill(s):
    T, out = s["T"], {"row_loss": [], "dlogits": []}
    for rows in torch.arange(s["logits"].shape[0], device="cuda").split(256):
        z = s["logits"][rows].double().requires_grad_()
        loss = torch.zeros(len(rows), dtype=torch.float64, device="cuda")
        if s["alpha"]:
            t = s["t"][rows].double().masked_fill(s["ids"][rows] < 0, float("-inf")) / T
            log_q = torch.log_softmax(t, dim=1).masked_fill(s["ids"][rows] < 0, 0.0)
            q = torch.softmax(t, dim=1)
            log_p = torch.log_softmax(z / T, dim=1).gather(1, s["ids"][rows].long().clamp(min=0))
            loss = loss + s["alpha"] * T ** 2 * (q * (log_q - log_p)).sum(dim=1)
        if s["beta"]:
            loss = loss + s["beta"] * torch.nn.functional.cross_entropy(z, s["labels"][rows], ignore_index=-100, reduction="none")
        loss = loss * s["weight"][rows].double()
        out["row_loss"].append(loss.detach())
        if s["grad"]:
            out["dlogits"].append(torch.autograd.grad(loss.sum(), z)[0])
    out = {k: torch.cat(v) for k, v in out.items() if v}
    return dict(out, loss=out["row_loss"].sum())


def _exact_norm(v, kind, w, b, eps):
    if kind == "none":
        return v
    if kind == "layer":
        return torch.nn.functional.layer_norm(v, v.shape[1:], w, b, eps)
    return v / torch.sqrt(v.pow(2).mean(dim=1, keepdim=True) + eps) * w


def _exact_boundary(s):
    f = {k: s[k].double() for k in ("x", "y", "w_pre", "b_pre", "w_post", "b_post", "gate") if s[k] is not None}
    gate = f.get("gate", 1.0)
    gate = torch.sigmoid(gate) if s["gate"] is not None and s["gate"].dim() == 2 else gate
    x = f["x"] + s["res_scale"] * gate * _exact_norm(f["y"], s["post"], f.get("w_post"), f.get("b_post"), s["eps"])
    return {"x": x, "h": _exact_norm(x, s["pre"], f["w_pre"], f.get("b_pre"), s["eps"])}


def _exact_boundary_grad(s):
    """By differentiation: h of the given stream, then the block's part with the stream's whole gradient."""
    f = {k: s[k].double().requires_grad_() for k in ("x", "y", "w_pre", "b_pre", "w_post", "b_post", "gate") if s[k] is not None}
    h = _exact_norm(f["x"], s["pre"], f["w_pre"], f.get("b_pre"), s["eps"])
    asked = [k for k in ("w_pre", "b_pre") if k in f]
    got = dict(zip(["x"] + asked, torch.autograd.grad(h, [f["x"]] + [f[k] for k in asked], s["dh"].double())))
    dx = s["dx"].double() + got["x"]
    gate = f.get("gate", 1.0)
    gate = torch.sigmoid(gate) if s["gate"] is not None and s["gate"].dim() == 2 else gate
    part = s["res_scale"] * gate * _exact_norm(f["y"], s["post"], f.get("w_post"), f.get("b_post"), s["eps"])
    asked = [k for k in ("y", "w_post", "b_post", "gate") if k in f]
    got.update(zip(asked, torch.autograd.grad(part, [f[k] for k in asked], dx)))
    name = {k: "d" + k for k in got}
    return dict({name[k]: v for k, v in got.items()}, dx=dx)


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "embed":
        return {"out": torch.nn.functional.embedding(s["tokens"].long(), s["table"].double()) * s["scale"]}
    return {"embed_grad": _exact_embed_grad, "distill": _exact_distill, "boundary": _exact_boundary,
            "boundary_grad": _exact_boundary_grad}[s["op"]](s)
