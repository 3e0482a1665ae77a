"""Language-model operators beside the AdaScale step: thin wrappers of ``include/adascale_ops.h``.

The AdaScale step consumes the S gradient rows of a model.  These calls make the parts of such a row,
and of the training step around it, that a library's matrix products and attention do not:

``embed``, ``embed_grad``
    the token table: scaled lookup, and its gradient by sorted tokens
``distill``
    the loss against a teacher's top logits, mixed with cross entropy, and its gradient
``residual_norm``, ``residual_norm_grad``
    a block's boundary: norm of its output, gate, residual scale, norm of the stream
``position_softmax``, ``position_softmax_grad``
    attention weights from scores, with a learned bias by buckets of relative positions, lengths and causality
``expert_matmul``, ``expert_matmul_grad``
    products with experts' weights over ragged groups of rows
``grad_norm``, ``clip_grads``
    the norm over all of a model's gradients, and clipping by it on the way into a row's slots

Tensors live on one CUDA device; a call enqueues its kernels on ``stream`` (None: the current stream
of that device; an address or a ``torch.cuda.Stream`` otherwise) and returns.  Results go to the tensors
given for them - a slot of a gradient row, say - or to new ones; workspaces come from torch's
caching allocator.  With another stream than the current one, new tensors belong to that stream, and
ordering it against the producers of the inputs is the caller's, as everywhere in torch.  The last dimension of every
matrix is contiguous; rows may have any stride.  There is no fallback and no autograd: gradients
are calls of their own, and results do not require one.  Wrong shapes or types raise ``ValueError``; what the library refuses
raises ``AdaScaleError``.
"""
from __future__ import annotations

import ctypes as C
from collections import namedtuple

import torch

from .binding import AdaScaleError, lib  # noqa: F401

try:
    from . import _ops_binding as _c
except ImportError as e:
    raise ImportError("the operators' binding is missing: build it with `python -m paper_2007_05105_b200.build` (%s)" % e) from e

EXPORTS = ("adascale_embed", "adascale_embed_grad", "adascale_embed_grad_workspace", "adascale_distill",
           "adascale_residual_norm", "adascale_residual_norm_grad", "adascale_residual_norm_grad_workspace",
           "adascale_position_softmax", "adascale_position_softmax_grad", "adascale_position_softmax_grad_workspace",
           "adascale_expert_matmul", "adascale_expert_matmul_grad", "adascale_clip_grads", "adascale_clip_grads_workspace")

I32, I64 = 0, 1
NORM_NONE, NORM_RMS, NORM_LAYER = 0, 1, 2
GATE_NONE, GATE_CHANNEL, GATE_SIGMOID = 0, 1, 2
EMBED_MAX_DIM = 1 << 30
DISTILL_MAX_K = 1024
NORM_MAX_DIM = 16384
POSITION_MAX_BUCKETS = 128
POSITION_MAX_DISTANCE = 16384
EXPERT_MAX_EXPERTS = 1024
EXPERT_MAX_DIM = 1 << 20
CLIP_MAX_TENSORS = 65536

# The C ABI's structs, for callers that hold addresses instead of tensors.
_p, _i32, _i64, _f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float


def _struct(name, spec):
    """A ctypes structure from lines of "type: names"."""
    kinds = {"ptr": _p, "i32": _i32, "i64": _i64, "f32": _f32}
    fields = [(n, kinds[kind]) for kind, names in spec for n in names.split()]
    return type(name, (C.Structure,), {"_fields_": fields})


EmbedArgs = _struct("EmbedArgs", [
    ("ptr", "tokens table out"), ("i64", "n_tokens vocab dim ld_table ld_out"),
    ("i32", "token_type table_dtype out_dtype"), ("f32", "scale")])
EmbedGradArgs = _struct("EmbedGradArgs", [
    ("ptr", "tokens dout grad workspace"), ("i64", "workspace_bytes n_tokens vocab dim ld_dout ld_grad padding_idx"),
    ("i32", "token_type dout_dtype grad_dtype accumulate"), ("f32", "scale")])
DistillArgs = _struct("DistillArgs", [
    ("ptr", "logits dlogits teacher_logits teacher_ids labels weight row_loss loss"),
    ("i64", "n_rows vocab n_top ld_logits ld_dlogits ld_teacher ld_ids"),
    ("i32", "dtype teacher_dtype id_type label_type"), ("f32", "temperature alpha beta")])
ResidualNormArgs = _struct("ResidualNormArgs", [
    ("ptr", "x y x_new h gate w_post b_post w_pre b_pre"), ("i64", "n_rows dim ld_x ld_y ld_x_new ld_h ld_gate"),
    ("i32", "x_dtype y_dtype post pre gate_kind"), ("f32", "res_scale eps")])
ResidualNormGradArgs = _struct("ResidualNormGradArgs", [
    ("ptr", "x_new y dx_new dh gate w_post b_post w_pre dx dy dgate dw_post db_post dw_pre db_pre workspace"),
    ("i64", "workspace_bytes n_rows dim ld_x_new ld_y ld_dx_new ld_dh ld_gate ld_dx ld_dy ld_dgate"),
    ("i32", "x_dtype y_dtype wgrad_dtype post pre gate_kind"), ("f32", "res_scale eps")])
PositionSoftmaxArgs = _struct("PositionSoftmaxArgs", [
    ("ptr", "scores probs table lengths starts"),
    ("i64", "batch heads n_queries n_keys scores_stride_b scores_stride_h scores_stride_q probs_stride_b probs_stride_h probs_stride_q "
            "ld_table"),
    ("i32", "dtype length_type start_type n_buckets max_distance bidirectional causal"), ("f32", "scale")])
PositionSoftmaxGradArgs = _struct("PositionSoftmaxGradArgs", [
    ("ptr", "probs dprobs dscores dtable lengths starts workspace"),
    ("i64", "workspace_bytes batch heads n_queries n_keys probs_stride_b probs_stride_h probs_stride_q dprobs_stride_b dprobs_stride_h "
            "dprobs_stride_q dscores_stride_b dscores_stride_h dscores_stride_q ld_dtable"),
    ("i32", "dtype wgrad_dtype length_type start_type n_buckets max_distance bidirectional causal accumulate"), ("f32", "scale")])
ExpertMatmulArgs = _struct("ExpertMatmulArgs", [
    ("ptr", "x w y offsets"), ("i64", "n_rows n_experts in_dim out_dim ld_x ld_w stride_w ld_y"), ("i32", "offset_type y_dtype")])
ExpertMatmulGradArgs = _struct("ExpertMatmulGradArgs", [
    ("ptr", "dy x w dx dw offsets"),
    ("i64", "n_rows n_experts in_dim out_dim ld_dy ld_x ld_w stride_w ld_dx ld_dw stride_dw"),
    ("i32", "offset_type dx_dtype dw_dtype accumulate")])
ClipGradsArgs = _struct("ClipGradsArgs", [
    ("ptr", "grads out numels grad_dtypes out_dtypes norm workspace"), ("i64", "workspace_bytes n_tensors"), ("f32", "max_norm eps")])

for _name, _args in [("adascale_embed", EmbedArgs), ("adascale_embed_grad", EmbedGradArgs),
                     ("adascale_distill", DistillArgs), ("adascale_residual_norm", ResidualNormArgs),
                     ("adascale_residual_norm_grad", ResidualNormGradArgs), ("adascale_position_softmax", PositionSoftmaxArgs),
                     ("adascale_position_softmax_grad", PositionSoftmaxGradArgs), ("adascale_expert_matmul", ExpertMatmulArgs),
                     ("adascale_expert_matmul_grad", ExpertMatmulGradArgs), ("adascale_clip_grads", ClipGradsArgs)]:
    getattr(lib, _name).argtypes = [C.POINTER(_args), _p]
    getattr(lib, _name).restype = C.c_int
for _name in ("adascale_embed_grad_workspace", "adascale_residual_norm_grad_workspace", "adascale_position_softmax_grad_workspace"):
    getattr(lib, _name).argtypes = [_i64, _i64]
    getattr(lib, _name).restype = _i64
lib.adascale_clip_grads_workspace.argtypes, lib.adascale_clip_grads_workspace.restype = [_i64], _i64

Distilled = namedtuple("Distilled", "loss row_loss dlogits")
PositionGrads = namedtuple("PositionGrads", "dscores dtable")
ExpertGrads = namedtuple("ExpertGrads", "dx dw")
BoundaryGrads = namedtuple("BoundaryGrads", "dx dy dgate dw_post db_post dw_pre db_pre")

_NORM = {None: NORM_NONE, "none": NORM_NONE, "rms": NORM_RMS, "layer": NORM_LAYER}


def _kind(name, none_too):
    kind = _NORM.get(name, -1)
    if kind < 0 or kind == NORM_NONE and not none_too:
        raise ValueError("a norm is 'rms' or 'layer'%s: got %r" % (" or None" if none_too else "", name))
    return kind


def _on(stream, t):
    """Makes another stream (an address or a torch.cuda.Stream) the current one of t's device."""
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream), device=t.device)
    elif stream.device != t.device:
        raise ValueError("the stream is on %s, the tensors are on %s" % (stream.device, t.device))
    return torch.cuda.stream(stream)


# --------------------------------------------------------------------------
# token table
# --------------------------------------------------------------------------


def embed(tokens, table, scale=1.0, out=None, out_dtype=None, stream=None):
    """``out[n] = scale * table[tokens[n]]``: rows of zeros for tokens outside the table.

    tokens: int32 or int64, any shape, contiguous.  table: [vocab, dim], float32 or bfloat16.  ``out``: [*tokens.shape,
    dim], made here in ``out_dtype`` (the table's) when not given.
    """
    if stream is not None:
        with _on(stream, table):
            return embed(tokens, table, scale, out, out_dtype)
    return _c.embed(tokens, table, scale, out, out_dtype)


def embed_grad(tokens, dout, grad, scale=1.0, padding_idx=-1, accumulate=False, workspace=None, stream=None):
    """``grad[v] (+)= scale * sum of dout[n] over tokens[n] == v``, in the order of n.

    ``grad`` is [vocab, dim], float32 or bfloat16: the table's slot of a gradient row.  Without ``accumulate`` all of it is
    written; with it the sums are added to what it holds and rows of absent tokens are not touched.
    Tokens equal to ``padding_idx`` (-1: none) or outside the table have no part.  ``workspace``: a uint8
    tensor of at least ``embed_grad_workspace(n, dim)`` bytes, made here when not given.
    """
    if stream is not None:
        with _on(stream, grad):
            return embed_grad(tokens, dout, grad, scale, padding_idx, accumulate, workspace)
    return _c.embed_grad(tokens, dout, grad, scale, padding_idx, accumulate, workspace)


def embed_grad_workspace(n_tokens, dim) -> int:
    return lib.adascale_embed_grad_workspace(n_tokens, dim)


# --------------------------------------------------------------------------
# distillation
# --------------------------------------------------------------------------


def distill(logits, teacher_logits=None, teacher_ids=None, labels=None, T=1.0, alpha=1.0, beta=0.0, row_weight=None,
            want_grad=True, dlogits=None, stream=None):
    """Loss of ``logits`` against a teacher's top logits, and its gradient.

    For row n: ``weight * (alpha T^2 KL(q || p_T) + beta CE(labels))`` with q the softmax of the teacher's list
    (``teacher_logits`` [n, k] at ``teacher_ids`` [n, k]; ids outside the vocabulary, -1 say, fill up short lists) and
    p_T that of ``logits`` over the whole vocabulary, both at temperature T.  Returns ``(loss, row_loss, dlogits)``:
    ``loss`` is the sum of ``row_loss``, ``dlogits`` its gradient in the type of ``logits`` (None without ``want_grad``).
    (``loss`` and ``row_loss`` are parts of one allocation: a loss that is kept keeps both.)
    ``row_weight`` (float32) holds masks, means and upstream factors; rows of weight 0 are not read.
    ``dlogits`` may be given, also as ``logits`` itself.
    """
    if stream is not None:
        with _on(stream, logits):
            return distill(logits, teacher_logits, teacher_ids, labels, T, alpha, beta, row_weight, want_grad, dlogits)
    return Distilled(*_c.distill(logits, teacher_logits, teacher_ids, labels, T, alpha, beta, row_weight, want_grad, dlogits))


# --------------------------------------------------------------------------
# block boundary
# --------------------------------------------------------------------------


def residual_norm(x, y, w_pre, b_pre=None, w_post=None, b_post=None, pre="rms", post=None, gate=None, res_scale=1.0,
                  eps=1e-6, x_new=None, h=None, stream=None):
    """``x_new = x + res_scale * G * post(y)``, ``h = pre(x_new)``: one pass over a block's boundary.

    x: the residual stream, [n, dim]; y: the block's output, same shape (None: ``h = pre(x)``, the norm before the first
    block, in x's type unless ``h`` is given).  ``pre``, ``post``: "rms" or "layer" (post: None for no norm); weights and biases float32 [dim].
    G: 1, a float32 [dim] vector, or sigmoid of a [n, dim] matrix of y's type.  Returns ``(x_new, h)`` of the
    types of x and y; ``x_new`` may be given as x, ``h`` as y.
    """
    if stream is not None:
        with _on(stream, x):
            return residual_norm(x, y, w_pre, b_pre, w_post, b_post, pre, post, gate, res_scale, eps, x_new, h)
    return _c.residual_norm(x, y, w_pre, b_pre, w_post, b_post, _kind(pre, False), _kind(post, True), gate, res_scale, eps, x_new, h)


def residual_norm_grad(x_new, y, dx_new, dh, w_pre, w_post=None, b_post=None, pre="rms", post=None, gate=None,
                       res_scale=1.0, eps=1e-6, wgrad_dtype=torch.float32, dx=None, dy=None, dgate=None, dw_post=None,
                       db_post=None, dw_pre=None, db_pre=None, workspace=None, stream=None):
    """Gradients of ``residual_norm`` from the stream after the block and the block's output.

    dx_new: the gradient that arrives at x_new (None: none does); dh: the one at h.  Returns ``(dx, dy, dgate, dw_post,
    db_post, dw_pre, db_pre)``, None where there is no such input.  Gradients of vectors are written in
    ``wgrad_dtype``, the type of the gradient row; pass slots of that row for them (and ``dx_new`` as dx, ``dh`` as dy, where
    they are not needed any more).  ``workspace``: a uint8 tensor of at least
    ``residual_norm_grad_workspace(n, dim)`` bytes, made here when not given.
    """
    if stream is not None:
        with _on(stream, x_new):
            return residual_norm_grad(x_new, y, dx_new, dh, w_pre, w_post, b_post, pre, post, gate, res_scale, eps, wgrad_dtype,
                                      dx, dy, dgate, dw_post, db_post, dw_pre, db_pre, workspace)
    return BoundaryGrads(*_c.residual_norm_grad(
        x_new, y, dx_new, dh, w_pre, w_post, b_post, _kind(pre, False), _kind(post, True), gate, res_scale, eps, wgrad_dtype,
        dx, dy, dgate, dw_post, db_post, dw_pre, db_pre, workspace))


def residual_norm_grad_workspace(n_rows, dim) -> int:
    return lib.adascale_residual_norm_grad_workspace(n_rows, dim)


# --------------------------------------------------------------------------
# attention weights with a relative position bias
# --------------------------------------------------------------------------


def position_softmax(scores, table, max_distance=128, bidirectional=True, scale=1.0, causal=False, lengths=None, starts=None,
                     out=None, stream=None):
    """``softmax(scale * scores[b, h, i, j] + table[bucket(j - (starts[b] + i)), h])`` over the keys j that are live.

    scores: [batch, heads, queries, keys], float32 or bfloat16, any strides but the last.  table: float32 [buckets, heads].
    Live are the keys below ``lengths[b]`` (int32 or int64; None: all) and, if ``causal``, up to the query's position; the others
    get 0 whatever their scores are, and a query without live keys gets zeros.  ``starts``: the position of each sequence's
    first query (None: 0) - of a single token's query, the number of those before it.  Buckets are single distances
    up to half of them (of each side's, if ``bidirectional``; otherwise keys ahead are all in bucket 0), then grow
    logarithmically; from ``max_distance`` on all are in the last.  ``out`` (the type of scores) may be ``scores``.
    """
    if stream is not None:
        with _on(stream, scores):
            return position_softmax(scores, table, max_distance, bidirectional, scale, causal, lengths, starts, out)
    return _c.position_softmax(scores, table, max_distance, bidirectional, scale, causal, lengths, starts, out)


def position_softmax_grad(probs, dprobs, num_buckets, max_distance=128, bidirectional=True, scale=1.0, causal=False, lengths=None,
                          starts=None, wgrad_dtype=torch.float32, accumulate=False, want_dscores=True, want_dtable=True, dscores=None,
                          dtable=None, workspace=None, stream=None):
    """Gradients of ``position_softmax`` from its result: ``(dscores, dtable)``.

    dprobs: the gradient that arrives at probs; ``dscores`` has their type and may be either of them.  ``dtable``, [num_buckets, heads] in
    ``wgrad_dtype`` or a given slot of a gradient row, is written, or added to with ``accumulate`` (a table that several layers share).
    Without ``want_dscores`` or ``want_dtable`` that one is None.  ``workspace``: a uint8 tensor of at least
    ``position_softmax_grad_workspace(heads, num_buckets)`` bytes, made here when not given.
    """
    if stream is not None:
        with _on(stream, probs):
            return position_softmax_grad(probs, dprobs, num_buckets, max_distance, bidirectional, scale, causal, lengths, starts, wgrad_dtype,
                                         accumulate, want_dscores, want_dtable, dscores, dtable, workspace)
    return PositionGrads(*_c.position_softmax_grad(probs, dprobs, num_buckets, max_distance, bidirectional, scale, causal, lengths, starts,
                                                   wgrad_dtype, accumulate, want_dscores, want_dtable, dscores, dtable, workspace))


def position_softmax_grad_workspace(heads, num_buckets) -> int:
    return lib.adascale_position_softmax_grad_workspace(heads, num_buckets)


# --------------------------------------------------------------------------
# experts
# --------------------------------------------------------------------------


def expert_matmul(x, w, offsets, out=None, out_dtype=None, stream=None):
    """``out[r] = w[e] @ x[r]`` for the rows r of expert e, ``offsets[e] <= r < offsets[e + 1]``.

    x: [rows, in], w: [experts, out, in], bfloat16, their rows on 16-byte boundaries.  offsets: int32 or int64 [experts + 1], ascending, on
    the device: nothing is copied to the host.  Sums are 32-bit; ``out`` is bfloat16 or float32 (``out_dtype``, bfloat16
    when not given).  Rows before the first offset and behind the last are neither used nor written: in a new ``out`` they hold anything.
    (Many of them cost a little: widths of tiles go by all rows.  Where the host knows better, give a slice.)
    """
    if stream is not None:
        with _on(stream, x):
            return expert_matmul(x, w, offsets, out, out_dtype)
    return _c.expert_matmul(x, w, offsets, out, out_dtype)


def expert_matmul_grad(dy, offsets, x=None, w=None, dx_dtype=None, wgrad_dtype=None, accumulate=False, dx=None, dw=None, stream=None):
    """Gradients of ``expert_matmul`` from ``dy`` [rows, out], bfloat16: ``(dx, dw)``.

    ``dx[r] = w[e]^T dy[r]`` where ``w`` is given (bfloat16 unless ``dx_dtype`` or ``dx`` say otherwise), ``dw[e] = sum of dy[r] x[r]^T`` where
    ``x`` is (float32 unless ``wgrad_dtype`` or ``dw``, a slot of a gradient row say, do); None otherwise.  With ``accumulate``
    the sums are added to what ``dw`` holds and experts without rows are not touched, without it theirs are zeros.  A ``dx`` without ``w``
    and a ``dw`` without ``x`` are refused.
    """
    if stream is not None:
        with _on(stream, dy):
            return expert_matmul_grad(dy, offsets, x, w, dx_dtype, wgrad_dtype, accumulate, dx, dw)
    return ExpertGrads(*_c.expert_matmul_grad(dy, offsets, x, w, dx_dtype, wgrad_dtype, accumulate, dx, dw))


# --------------------------------------------------------------------------
# gradient norm and clipping
# --------------------------------------------------------------------------


def _listed(grads):
    """As a list that has a first tensor, whose device the stream is to be on."""
    try:
        grads = list(grads)
    except TypeError:
        raise TypeError("grads is not a list of tensors") from None
    if not grads:
        raise ValueError("grads: the list is empty")
    if not isinstance(grads[0], torch.Tensor):
        raise TypeError("grads is not a tensor")
    return grads


def grad_norm(grads, workspace=None, stream=None):
    """2-norm over all elements of a list (or another iterable) of float32 and bfloat16 tensors, as a float32 scalar on the device."""
    if stream is not None:
        grads = _listed(grads)
        with _on(stream, grads[0]):
            return grad_norm(grads, workspace)
    return _c.clip_grads(grads, None, None, 0.0, workspace)


def clip_grads(grads, max_norm, out=None, eps=1e-6, workspace=None, stream=None):
    """``out[k] = min(1, max_norm / (norm + eps)) * grads[k]`` with the norm over all of ``grads``; returns the norm.

    ``out``: a tensor for each gradient, of its shape and order in memory - the slots of a gradient row, in that row's type - or
    None: in place.  Nothing waits for the device.  Elements of a tensor are adjacent; no two outputs overlap.  Rows that are clipped one by one
    have norms of their own: the step's gain is that of the clipped gradients.
    ``workspace``: a uint8 tensor of at least ``clip_grads_workspace(len(grads))`` bytes, made here when not given.
    """
    if stream is not None:
        grads = _listed(grads)
        with _on(stream, grads[0]):
            return clip_grads(grads, max_norm, out, eps, workspace)
    if max_norm is None:
        raise TypeError("max_norm is not a number")
    return _c.clip_grads(grads, max_norm, out, eps, workspace)


def clip_grads_workspace(n_tensors) -> int:
    return lib.adascale_clip_grads_workspace(n_tensors)
