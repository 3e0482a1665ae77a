"""Cases for timing and checking three more language-model operators of ``paper_2007_05105_b200.ops``.

They stand between a decoder's layers and the gradient rows that the AdaScale step consumes: the gradient
norm over all of a model's tensors with clipping on the way into a row's slots, the attention
weights with a learned relative position bias (softmax over scores, bias by buckets, masks) with their gradient, and the
products with experts' weights over ragged groups of rows with their gradients.  Each has a
plain form here, in elementary torch operations in 32 bits, and a 64-bit form in ``exact``.  Sizes are
those of the Transformer-base and decoder tensor lists in ``synthetic.py`` (width 512 and 1024, feed-forward 2048 and
4096, 8 and 16 heads, 1024 positions) or generic.
"""
import functools
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
        # the gradients of one block of Transformer-base are clipped into their slots
        dict(name="clip_block", op="clip", d=512, ffn=2048, layers=1, vocab=0, g=F32, out=F32, clipped=True),
        # the norm alone, for a log, of all gradients of a model of Transformer-base's size
        dict(name="norm_transformer", op="norm", d=512, ffn=2048, layers=14, vocab=32768, g=F32),
        # the same gradients from 32-bit leaves into a bf16 row
        dict(name="clip_transformer", op="clip", d=512, ffn=2048, layers=14, vocab=32768, g=F32, out=BF16, clipped=True),
        # the 24-layer decoder, bf16 throughout
        dict(name="clip_decoder", op="clip", d=1024, ffn=4096, layers=24, vocab=50257, g=BF16, out=BF16, clipped=True),
        # one token of each of 8 sequences attends to what came before, in a padded cache of 1024 positions
        dict(name="weights_token", op="weights", B=8, H=16, Lq=1, Lk=1024, s=BF16, buckets=32, distance=128, both=False,
             causal=True, ragged=True, starts=True),
        # an encoder's microbatch at Transformer-base width, padded sequences, all in 32 bits
        dict(name="weights_batch", op="weights", B=32, H=8, Lq=512, Lk=512, s=F32, buckets=32, distance=128, both=True,
             causal=False, ragged=True, starts=False),
        # the gradient for the decoder's microbatch of 8 full sequences
        dict(name="weights_grad_batch", op="weights_grad", B=8, H=16, Lq=1024, Lk=1024, s=BF16, buckets=32, distance=128,
             both=False, causal=True, ragged=False, grad=BF16, accumulate=False),
        # odd lengths of queries and keys; the table is shared by the layers, this one's part is added
        dict(name="weights_grad_odd", op="weights_grad", B=3, H=8, Lq=333, Lk=517, s=F32, buckets=64, distance=300, both=True,
             causal=False, ragged=True, grad=F32, accumulate=True),
        # 8 tokens are generated at once, two experts each
        dict(name="experts_token", op="experts", N=16, E=8, K=1024, M=4096, out=BF16, tail=0, ids="i32"),
        # a training microbatch of 8 sequences of 1024 tokens, two of 16 experts each
        dict(name="experts_batch", op="experts", N=16384, E=16, K=1024, M=4096, out=BF16, tail=0, ids="i32"),
        # the gradients of the experts' second product
        dict(name="experts_grad_batch", op="experts_grad", N=8192, E=8, K=4096, M=1024, out=BF16, grad=BF16, accumulate=False,
             tail=0, ids="i32"),
        # an odd number of rows in a buffer with room behind them; weight gradients added up in 32 bits
        dict(name="experts_grad_odd", op="experts_grad", N=1777, E=12, K=512, M=1032, out=BF16, grad=F32, accumulate=True,
             tail=271, ids="i64"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi, step=8):
    return max(step, _log_int(rng, lo, hi) // step * step)


def draw(rng):
    op = rng.choice(["norm", "clip", "weights", "weights", "weights_grad", "experts", "experts", "experts_grad"])
    any_type = lambda: rng.choice([F32, BF16])  # noqa: E731
    if op in ("norm", "clip"):
        d = _width(rng, 64, 1280, rng.choice([1, 8]))
        layers = _log_int(rng, 1, 24)
        vocab = rng.choice([0, _log_int(rng, 1000, 50257)])
        c = dict(op=op, d=d, ffn=4 * d, layers=layers, vocab=vocab, g=any_type())
        while _numel(c) > 170_000_000:
            c["layers"] = max(1, c["layers"] // 2)
            c["vocab"] //= 2
        return dict(c, out=any_type(), clipped=rng.random() < 0.75) if op == "clip" else c
    if op in ("weights", "weights_grad"):
        H = rng.choice([4, 8, 12, 16])
        single = op == "weights" and rng.random() < 0.3
        Lk = _log_int(rng, 1, 16384 if single else 2048)
        Lq = 1 if single else Lk if rng.random() < 0.6 else _log_int(rng, 1, 2048)
        s = any_type()
        B = max(1, min(_log_int(rng, 1, 64), int(2.2e8 / (H * Lq * Lk * _BYTES[s]))))
        both = rng.random() < 0.5
        c = dict(op=op, B=B, H=H, Lq=Lq, Lk=Lk, s=s, buckets=rng.choice([16, 32, 64]), distance=rng.choice([64, 128, 300, 1000]),
                 both=both, causal=not both and rng.random() < 0.7, ragged=rng.random() < 0.5)
        if op == "weights":
            return dict(c, starts=single)
        return dict(c, grad=any_type(), accumulate=rng.random() < 0.5)
    E = _log_int(rng, 1, 64)
    K, M = _width(rng, 64, 4096), _width(rng, 64, 4096)
    while E * K * M > 68_000_000:
        E = max(1, E // 2)
        if E == 1:
            break
    N = max(1, min(_log_int(rng, 1, 16384), int(6.8e10 / (K * M))))
    if op == "experts_grad":
        N = max(1, min(N, int(3.4e10 / (K * M))))
    c = dict(op=op, N=N, E=E, K=K, M=M, out=any_type(), tail=rng.choice([0, _log_int(rng, 1, 500)]), ids=rng.choice(["i32", "i64"]))
    return dict(c, grad=any_type(), accumulate=rng.random() < 0.5) if op == "experts_grad" else c


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------


def _shapes(case):
    """Weights and biases of a decoder: token table, then blocks of fused attention projections, feed-forward and norms."""
    d, f = case["d"], case["ffn"]
    block = [(d,), (d,), (3 * d, d), (3 * d,), (d, d), (d,), (d,), (d,), (f, d), (f,), (d, f), (d,)]
    return ([(case["vocab"], d)] if case["vocab"] else []) + block * case["layers"]


def _numel(case):
    return sum(math.prod(s) for s in _shapes(case))


def _normal(gen, *shape, dtype=torch.float32, std=1.0, mean=0.0):
    t = torch.empty(*shape, dtype=torch.float32, device="cuda")
    return t.normal_(mean, std, generator=gen).to(dtype)


def _prepare_clip(case, gen):
    shapes = _shapes(case)
    sizes = [math.prod(s) for s in shapes]
    flat = _normal(gen, sum(sizes), dtype=_DTYPE[case["g"]], std=1e-3)
    # leaves' gradients as a backward pass leaves them: tensors of their own
    s = dict(grads=[t.clone().view(shape) for t, shape in zip(flat.split(sizes), shapes)], sizes=sizes)
    if case["op"] == "clip":
        # the slots of one gradient row, each at a multiple of 64 elements
        starts, end = [], 0
        for n in sizes:
            starts.append(end)
            end += -(-n // 64) * 64
        s["row"] = torch.zeros(end, dtype=_DTYPE[case["out"]], device="cuda")
        s["slots"] = [s["row"][o:o + n].view(shape) for o, n, shape in zip(starts, sizes, shapes)]
        s["max_norm"] = 1e-3 * math.sqrt(sum(sizes)) * (0.4 if case["clipped"] else 2.5)
    return s


def _kept(s):
    """Which keys a query may see: [B, 1, Lq, Lk] (or one for every batch), True to keep; None where all are."""
    keep = None
    key = torch.arange(s["Lk"], device="cuda")
    if s["lengths"] is not None:
        keep = (key < s["lengths"].view(-1, 1, 1, 1))
    if s["causal"]:
        seen = key <= _queries(s)[..., None]
        seen = seen.view(-1, 1, s["Lq"], s["Lk"])
        keep = seen if keep is None else keep & seen
    return keep


def _queries(s):
    """Positions of the queries: [Lq], or [B, Lq] where each sequence starts elsewhere."""
    q = torch.arange(s["Lq"], device="cuda")
    return q if s["starts"] is None else s["starts"].view(-1, 1) + q


def _prepare_weights(case, gen):
    B, H, Lq, Lk, t = case["B"], case["H"], case["Lq"], case["Lk"], _DTYPE[case["s"]]
    s = dict(Lq=Lq, Lk=Lk, buckets=case["buckets"], distance=case["distance"], both=case["both"], causal=case["causal"],
             scale=0.125, lengths=None, starts=None)
    if case["ragged"]:
        s["lengths"] = torch.randint(max(1, Lk // 2), Lk + 1, (B,), device="cuda", generator=gen, dtype=torch.int32)
    if case.get("starts"):  # the queries are the last of their sequences
        s["starts"] = (torch.full((B,), Lk, device="cuda", dtype=torch.int32) if s["lengths"] is None else s["lengths"]) - Lq
    if case["op"] == "weights":
        s["scores"] = _normal(gen, B, H, Lq, Lk, dtype=t, std=8.0)
        s["table"] = _normal(gen, case["buckets"], H, std=1.0)
        return s
    z = _normal(gen, B, H, Lq, Lk, std=1.0)
    keep = _kept(s)
    if keep is not None:
        z.masked_fill_(~keep, float("-inf"))
    s["probs"] = torch.nan_to_num(torch.softmax(z, dim=-1)).to(t)
    del z
    s["dprobs"] = _normal(gen, B, H, Lq, Lk, dtype=t, std=1e-2)
    s["grad"], s["accumulate"] = _DTYPE[case["grad"]], case["accumulate"]
    s["dtable"] = _normal(gen, case["buckets"], H, dtype=s["grad"], std=1e-2) if case["accumulate"] else None
    return s


def _prepare_experts(case, gen):
    N, E, K, M, tail = case["N"], case["E"], case["K"], case["M"], case["tail"]
    # some experts are chosen more often than others, some not at all
    share = torch.softmax(_normal(gen, E, std=0.5), dim=0)
    chosen = torch.multinomial(share, N, replacement=True, generator=gen)
    counts = torch.bincount(chosen, minlength=E)
    ends = counts.cumsum(0)
    s = dict(offsets=torch.cat([ends.new_zeros(1), ends]).to(torch.int64 if case["ids"] == "i64" else torch.int32),
             groups=[(e, int(end) - int(n), int(end)) for e, (end, n) in enumerate(zip(ends.tolist(), counts.tolist())) if n])
    s["x"] = _normal(gen, N + tail, K, dtype=torch.bfloat16)
    s["w"] = _normal(gen, E, M, K, dtype=torch.bfloat16, std=K ** -0.5)
    out = _DTYPE[case["out"]]
    if case["op"] == "experts":
        s["y"] = torch.zeros(N + tail, M, dtype=out, device="cuda")
        return s
    s["dy"] = _normal(gen, N + tail, M, dtype=torch.bfloat16, std=1e-2)
    s["dx"] = torch.zeros(N + tail, K, dtype=out, device="cuda")
    s["accumulate"] = case["accumulate"]
    s["dw"] = _normal(gen, E, M, K, dtype=_DTYPE[case["grad"]], std=1e-2)  # the experts' slot of a gradient row
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 1000003 + 29)
    maker = {"n": _prepare_clip, "c": _prepare_clip, "w": _prepare_weights, "e": _prepare_experts}[case["op"][0]]
    return dict(maker(case, gen), op=case["op"])


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------


def _plain_norm(s):
    flat = torch.cat([g.reshape(-1) for g in s["grads"]]).float()
    norm = torch.sqrt((flat * flat).sum())
    if s["op"] == "norm":
        return {"norm": norm}
    flat *= torch.clamp(s["max_norm"] / (norm + 1e-6), max=1.0)
    torch._foreach_copy_([t.view(-1) for t in s["slots"]], list(flat.split(s["sizes"])))
    return {"norm": norm, "row": s["row"]}


def _plain_buckets(s):
    """Bucket of every query and key, [Lq, Lk] or [B, Lq, Lk]."""
    d = torch.arange(s["Lk"], device="cuda") - _queries(s)[..., None]
    m = s["buckets"]
    side = torch.zeros_like(d)
    if s["both"]:
        m //= 2
        side = m * (d > 0)
        n = d.abs()
    else:
        n = (-d).clamp(min=0)
    exact = m // 2
    # in 64 bits, and a hair up: distances on a border belong to the bucket above it
    far = torch.log(n.clamp(min=1).double() / exact) / math.log(s["distance"] / exact) * (m - exact)
    far = (exact + torch.floor(far + 1e-9)).long().clamp(max=m - 1)
    return side + torch.where(n < exact, n, far)


def _plain_weights(s):
    bias = s["table"][_plain_buckets(s)].movedim(-1, -3)
    z = s["scores"].float() * s["scale"] + bias
    keep = _kept(s)
    if keep is not None:
        z = torch.where(keep, z, float("-inf"))
    top = z.max(dim=-1, keepdim=True).values
    e = torch.exp(z - torch.where(top == float("-inf"), 0.0, top))
    total = e.sum(dim=-1, keepdim=True)
    return {"probs": (e / torch.where(total == 0.0, 1.0, total)).to(s["scores"].dtype)}


def _plain_weights_grad(s):
    p, dp = s["probs"].float(), s["dprobs"].float()
    dz = p * (dp - (p * dp).sum(dim=-1, keepdim=True))
    which = _plain_buckets(s).reshape(-1, 1) == torch.arange(s["buckets"], device="cuda")
    total = which.float().t() @ dz.sum(dim=0).reshape(dz.shape[1], -1).t()
    if s["accumulate"]:
        total = s["dtable"].copy_(total + s["dtable"])
    return {"dscores": (dz * s["scale"]).to(s["probs"].dtype), "dtable": total.to(s["grad"])}


def _plain_experts(s):
    for e, lo, hi in s["groups"]:
        s["y"][lo:hi] = s["x"][lo:hi].float() @ s["w"][e].float().t()
    return {"y": s["y"]}


def _plain_experts_grad(s):
    if not s["accumulate"]:
        s["dw"].zero_()
    for e, lo, hi in s["groups"]:
        dy = s["dy"][lo:hi].float()
        s["dx"][lo:hi] = dy @ s["w"][e].float()
        s["dw"][e] = s["dw"][e] + dy.t() @ s["x"][lo:hi].float()
    return {"dx": s["dx"], "dw": s["dw"]}


def _own(s):
    from paper_2007_05105_b200 import ops

    if s["op"] == "norm":
        return {"norm": ops.grad_norm(s["grads"])}
    if s["op"] == "clip":
        return {"norm": ops.clip_grads(s["grads"], s["max_norm"], out=s["slots"]), "row": s["row"]}
    if s["op"] in ("weights", "weights_grad"):
        how = dict(max_distance=s["distance"], bidirectional=s["both"], scale=s["scale"], causal=s["causal"],
                   lengths=s["lengths"], starts=s["starts"])
        if s["op"] == "weights":
            return {"probs": ops.position_softmax(s["scores"], s["table"], **how)}
        g = ops.position_softmax_grad(s["probs"], s["dprobs"], s["buckets"], wgrad_dtype=s["grad"], dtable=s["dtable"],
                                      accumulate=s["accumulate"], **how)
        return {"dscores": g.dscores, "dtable": g.dtable}
    if s["op"] == "experts":
        return {"y": ops.expert_matmul(s["x"], s["w"], s["offsets"], out=s["y"])}
    g = ops.expert_matmul_grad(s["dy"], s["offsets"], x=s["x"], w=s["w"], dx=s["dx"], dw=s["dw"], accumulate=s["accumulate"])
    return {"dx": g.dx, "dw": g.dw}


def run(state):
    if own:
        return _own(state)
    return {"norm": _plain_norm, "clip": _plain_norm, "weights": _plain_weights, "weights_grad": _plain_weights_grad,
            "experts": _plain_experts, "experts_grad": _plain_experts_grad}[state["op"]](state)


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------


def work(case):
    op = case["op"]
    if op in ("norm", "clip"):
        n = _numel(case)
        return {"bytes": n * (_BYTES[case["g"]] + (_BYTES[case["out"]] if op == "clip" else 0)), "flops": n * (3 if op == "clip" else 2)}
    if op in ("weights", "weights_grad"):
        B, H, Lq, Lk, b = case["B"], case["H"], case["Lq"], case["Lk"], _BYTES[case["s"]]
        share = 0.75 if case["ragged"] else 1.0  # of the keys that are there, on average
        if case["causal"] and not case.get("starts"):  # of those, the ones that a query may see
            share *= sum(min(i + 1, Lk) for i in range(Lq)) / (Lq * Lk)
        seen, whole = B * H * Lq * Lk * share, B * H * Lq * Lk
        table = case["buckets"] * H
        if op == "weights":
            return {"bytes": (seen + whole) * b + 4 * table, "flops": 8 * seen}
        return {"bytes": (2 * seen + whole) * b + table * _BYTES[case["grad"]] * (2 if case["accumulate"] else 1), "flops": 7 * seen}
    N, E, K, M = case["N"], case["E"], case["K"], case["M"]
    out = _BYTES[case["out"]]
    active = E * (1.0 - (1.0 - 1.0 / E) ** N)  # experts with rows, if all are as likely
    if op == "experts":
        return {"bytes": 2 * N * K + out * N * M + 2 * active * K * M, "flops": 2 * N * K * M}
    grad = _BYTES[case["grad"]] * (2 * active if case["accumulate"] else E)
    return {"bytes": 2 * N * (K + M) + out * N * K + (2 * active + grad) * K * M, "flops": 4 * N * K * M}


# --------------------------------------------------------------------------
# the operators in 64 bits
# --------------------------------------------------------------------------


def _exact_clip(s):
    total = math.sqrt(math.fsum(float(torch.dot(g.double().view(-1), g.double().view(-1))) for g in s["grads"]))
    norm = torch.tensor(total, dtype=torch.float64)
    if s["op"] == "norm":
        return {"norm": norm}
    row = torch.zeros(s["row"].shape, dtype=torch.float64, device="cuda")
    for g, slot in zip(s["grads"], s["slots"]):
        at = slot.storage_offset()
        row[at:at + g.numel()] = g.double().view(-1) * min(1.0, s["max_norm"] / (total + 1e-6))
    return {"norm": norm, "row": row}


@functools.lru_cache(maxsize=None)
def _bucket(d, buckets, distance, both):
    """Bucket of one distance, in whole numbers: the k-th far bucket begins at exact * (distance / exact) ** (k / far)."""
    m = buckets // 2 if both else buckets
    n = abs(d) if both else max(-d, 0)
    exact = m // 2
    if n >= distance:
        n = m - 1
    elif n >= exact:
        far, k = m - exact, 0
        while k < far - 1 and n ** far >= exact ** (far - k - 1) * distance ** (k + 1):
            k += 1
        n = exact + k
    return n + (m if both and d > 0 else 0)


def _exact_buckets(s, b):
    """Of sequence b, [Lq, Lk]: every distance looked up once."""
    start = 0 if s["starts"] is None else int(s["starts"][b])
    span = range(-(start + s["Lq"] - 1), s["Lk"] - start)
    at_most = s["distance"]  # beyond it nothing changes
    by = [_bucket(max(-at_most, min(at_most, d)), s["buckets"], s["distance"], s["both"]) for d in span]
    by = torch.tensor(by, device="cuda")
    at = torch.arange(s["Lk"], device="cuda")[None, :] + torch.arange(s["Lq"] - 1, -1, -1, device="cuda")[:, None]
    return by[at]


def _hidden(s, b):
    """Which keys sequence b's queries may not see, [Lq, Lk]."""
    start = 0 if s["starts"] is None else int(s["starts"][b])
    length = s["Lk"] if s["lengths"] is None else int(s["lengths"][b])
    hide = torch.ones(s["Lq"], s["Lk"], dtype=torch.bool, device="cuda")
    hide[:, :length] = False
    return hide | hide.new_ones(hide.shape).triu(start + 1) if s["causal"] else hide


def _exact_weights(s):
    out, by = [], None
    for b in range(s["scores"].shape[0]):
        by = _exact_buckets(s, b) if by is None or s["starts"] is not None else by
        z = s["scores"][b].double() * s["scale"] + s["table"].double().t()[:, by]
        out.append(torch.softmax(z.masked_fill(_hidden(s, b), float("-inf")), dim=-1).nan_to_num(0.0))
    return {"probs": torch.stack(out)}


def _exact_weights_grad(s):
    table = s["dtable"].double() if s["accumulate"] else torch.zeros(s["buckets"], s["probs"].shape[1], dtype=torch.float64, device="cuda")
    out, which = [], torch.nn.functional.one_hot(_exact_buckets(s, 0), s["buckets"]).double()
    for b in range(s["probs"].shape[0]):
        p, dp = s["probs"][b].double(), s["dprobs"][b].double()
        dz = p * dp - p * torch.einsum("hij,hij->hi", p, dp)[..., None]
        out.append(s["scale"] * dz)
        table = table + torch.einsum("hij,ijk->kh", dz, which)
    return {"dscores": torch.stack(out), "dtable": table}


def _exact_experts(s):
    if s["op"] == "experts":
        y = torch.zeros(s["y"].shape, dtype=torch.float64, device="cuda")
        for e, lo, hi in s["groups"]:
            y[lo:hi] = torch.nn.functional.linear(s["x"][lo:hi].double(), s["w"][e].double())
        return {"y": y}
    dx = torch.zeros(s["dx"].shape, dtype=torch.float64, device="cuda")
    dw = s["dw"].double() if s["accumulate"] else torch.zeros(s["dw"].shape, dtype=torch.float64, device="cuda")
    for e, lo, hi in s["groups"]:
        x, w = s["x"][lo:hi].double().requires_grad_(), s["w"][e].double().requires_grad_()
        dx[lo:hi], part = torch.autograd.grad(torch.nn.functional.linear(x, w), (x, w), s["dy"][lo:hi].double())
        dw[e] += part
    return {"dx": dx, "dw": dw}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("norm", "clip"):
        return _exact_clip(s)
    return {"weights": _exact_weights, "weights_grad": _exact_weights_grad, "experts": _exact_experts, "experts_grad": _exact_experts}[case["op"]](s)
