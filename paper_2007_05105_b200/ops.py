"""Language-model operators beside the AdaScale step: thin wrappers of ``include/adascale_ops.h``.

The AdaScale step consumes the S gradient rows of a model.  These calls make the parts of such a row,
and of the training step around it, that are neither a matrix product nor attention:

``embed``, ``embed_grad``
    the token table: scaled lookup, and its gradient by sorted tokens
``distill``
    the loss against a teacher's top logits, mixed with cross entropy, and its gradient
``residual_norm``, ``residual_norm_grad``
    a block's boundary: norm of its output, gate, residual scale, norm of the stream

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
           "adascale_residual_norm", "adascale_residual_norm_grad", "adascale_residual_norm_grad_workspace")

I32, I64 = 0, 1
NORM_NONE, NORM_RMS, NORM_LAYER = 0, 1, 2
GATE_NONE, GATE_CHANNEL, GATE_SIGMOID = 0, 1, 2
EMBED_MAX_DIM = 1 << 30
DISTILL_MAX_K = 1024
NORM_MAX_DIM = 16384

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

for _name, _args in [("adascale_embed", EmbedArgs), ("adascale_embed_grad", EmbedGradArgs),
                     ("adascale_distill", DistillArgs), ("adascale_residual_norm", ResidualNormArgs),
                     ("adascale_residual_norm_grad", ResidualNormGradArgs)]:
    getattr(lib, _name).argtypes = [C.POINTER(_args), _p]
    getattr(lib, _name).restype = C.c_int
for _name in ("adascale_embed_grad_workspace", "adascale_residual_norm_grad_workspace"):
    getattr(lib, _name).argtypes = [_i64, _i64]
    getattr(lib, _name).restype = _i64

Distilled = namedtuple("Distilled", "loss row_loss dlogits")
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
