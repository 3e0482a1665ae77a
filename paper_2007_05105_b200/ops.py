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
are calls of their own.  Wrong shapes or types raise ``ValueError``; what the library refuses
raises ``AdaScaleError``.
"""
from __future__ import annotations

import ctypes as C
from collections import namedtuple

import torch

from .binding import BF16, F32, OK, AdaScaleError, lib, strerror

EXPORTS = ("adascale_embed", "adascale_embed_grad", "adascale_embed_grad_workspace", "adascale_distill",
           "adascale_residual_norm", "adascale_residual_norm_grad", "adascale_residual_norm_grad_workspace")

I32, I64 = 0, 1
NORM_NONE, NORM_RMS, NORM_LAYER = 0, 1, 2
GATE_NONE, GATE_CHANNEL, GATE_SIGMOID = 0, 1, 2
DISTILL_MAX_K = 1024
NORM_MAX_DIM = 16384

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

_DTYPE = {torch.float32: F32, torch.bfloat16: BF16}
_ITYPE = {torch.int32: I32, torch.int64: I64}
_NORM = {None: NORM_NONE, "none": NORM_NONE, "rms": NORM_RMS, "layer": NORM_LAYER}


# --------------------------------------------------------------------------
# plumbing
# --------------------------------------------------------------------------


def _call(fn, args, device, stream):
    if stream is None:
        stream = torch.cuda.current_stream(device).cuda_stream
    status = fn(args, stream)
    if status != OK:
        raise AdaScaleError(status, strerror(status))


def _place(t, stream):
    """Device of the call, and the context in which its new tensors are made (None: as things are)."""
    if not t.is_cuda:
        raise ValueError("the operators take CUDA tensors")
    device = t.device
    if stream is None and device.index == torch.cuda.current_device():
        return device, None
    return device, _On(device, stream)


class _On:
    """Makes a device and a stream current."""

    def __init__(self, device, stream):
        self.device = torch.cuda.device(device)
        if stream is not None and not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(int(stream), device=device)
        self.stream = torch.cuda.stream(stream)

    def __enter__(self):
        self.device.__enter__()
        self.stream.__enter__()

    def __exit__(self, *exc):
        self.stream.__exit__(*exc)
        self.device.__exit__(*exc)


def _code(codes, t, what):
    try:
        return codes[t.dtype]
    except KeyError:
        raise ValueError("%s: %s is not one of %s" % (what, t.dtype, ", ".join(str(k) for k in codes))) from None


def _matrix(t, n, d, device, what):
    """Address and row stride of a tensor of n rows of d elements (leading dimensions are one)."""
    if t.device != device:
        raise ValueError("%s is on %s, not on %s" % (what, t.device, device))
    if t.dim() != 2:
        if t.dim() == 0 or t.shape[-1] != d:
            raise ValueError("%s: shape %s, not %d rows of %d" % (what, tuple(t.shape), n, d))
        t = t.view(n, d) if t.numel() == n * d else t
    if t.shape[0] != n or t.shape[1] != d:
        raise ValueError("%s: shape %s, not %d rows of %d" % (what, tuple(t.shape), n, d))
    row, one = t.stride()
    if one != 1 and d > 1:
        raise ValueError("%s: the last dimension is not contiguous" % what)
    if n <= 1:
        row = d
    elif row < d:  # expanded or overlapping rows
        raise ValueError("%s: rows overlap (row stride %d, %d elements)" % (what, row, d))
    return t.data_ptr(), row


def _vector(t, n, dtypes, device, what):
    if t.device != device or t.numel() != n or not t.is_contiguous():
        raise ValueError("%s: want %d contiguous elements on %s" % (what, n, device))
    if t.dtype not in dtypes:
        raise ValueError("%s: %s is not one of %s" % (what, t.dtype, ", ".join(str(k) for k in dtypes)))
    return t.data_ptr()


_ONLY_F32 = (torch.float32,)


def _f32_vector(t, n, device, what):
    return None if t is None else _vector(t, n, _ONLY_F32, device, what)


def _rows_of(t, what):
    if t.dim() == 0:
        raise ValueError("%s: a scalar has no rows" % what)
    d = t.shape[-1]
    return (t.shape[0] if t.dim() == 2 else t.numel() // d if d else 0), d


# --------------------------------------------------------------------------
# token table
# --------------------------------------------------------------------------


def embed(tokens, table, scale=1.0, out=None, out_dtype=None, stream=None):
    """``out[n] = scale * table[tokens[n]]``: rows of zeros for tokens outside the table.

    tokens: int32 or int64, any shape, contiguous.  table: [vocab, dim], float32 or bfloat16.  ``out``: [*tokens.shape,
    dim], made here in ``out_dtype`` (the table's) when not given.
    """
    device, at = _place(table, stream)
    if at is not None:
        with at:
            return embed(tokens, table, scale, out, out_dtype)
    vocab, dim = table.shape
    n = tokens.numel()
    if out is None:
        out = torch.empty((*tokens.shape, dim), dtype=out_dtype or table.dtype, device=device)
    elif out_dtype is not None and out.dtype != out_dtype:
        raise ValueError("out is %s, not %s" % (out.dtype, out_dtype))
    table_at, ld_table = _matrix(table, vocab, dim, device, "table")
    out_at, ld_out = _matrix(out, n, dim, device, "out")
    _call(lib.adascale_embed, EmbedArgs(
        _vector(tokens, n, _ITYPE, device, "tokens"), table_at, out_at, n, vocab, dim, ld_table, ld_out,
        _ITYPE[tokens.dtype], _code(_DTYPE, table, "table"), _code(_DTYPE, out, "out"), scale), device, None)
    return out


def embed_grad(tokens, dout, grad, scale=1.0, padding_idx=-1, accumulate=False, workspace=None, stream=None):
    """``grad[v] (+)= scale * sum of dout[n] over tokens[n] == v``, in the order of n.

    ``grad`` is [vocab, dim], float32 or bfloat16: the table's slot of a gradient row.  Without ``accumulate`` all of it is
    written; with it the sums are added to what it holds and rows of absent tokens are not touched.
    Tokens equal to ``padding_idx`` (-1: none) or outside the table have no part.  ``workspace``: a uint8
    tensor of at least ``embed_grad_workspace(n, dim)`` bytes, made here when not given.
    """
    device, at = _place(grad, stream)
    if at is not None:
        with at:
            return embed_grad(tokens, dout, grad, scale, padding_idx, accumulate, workspace)
    if grad.dim() != 2:
        raise ValueError("grad: shape %s, not [vocab, dim]" % (tuple(grad.shape),))
    vocab, dim = grad.shape
    n = tokens.numel()
    need = lib.adascale_embed_grad_workspace(n, dim)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
    dout_at, ld_dout = _matrix(dout, n, dim, device, "dout")
    grad_at, ld_grad = _matrix(grad, vocab, dim, device, "grad")
    _call(lib.adascale_embed_grad, EmbedGradArgs(
        _vector(tokens, n, _ITYPE, device, "tokens"), dout_at, grad_at, workspace.data_ptr(), workspace.nbytes, n, vocab,
        dim, ld_dout, ld_grad, padding_idx, _ITYPE[tokens.dtype], _code(_DTYPE, dout, "dout"),
        _code(_DTYPE, grad, "grad"), 1 if accumulate else 0, scale), device, None)
    return grad


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
    ``row_weight`` (float32) holds masks, means and upstream factors; rows of weight 0 are not read.
    ``dlogits`` may be given, also as ``logits`` itself.
    """
    device, at = _place(logits, stream)
    if at is not None:
        with at:
            return distill(logits, teacher_logits, teacher_ids, labels, T, alpha, beta, row_weight, want_grad, dlogits)
    n, vocab = _rows_of(logits, "logits")
    z_at, ld_z = _matrix(logits, n, vocab, device, "logits")
    t_at = ids_at = None
    k = ld_t = ld_ids = t_code = id_code = 0
    if teacher_logits is not None or teacher_ids is not None:
        if teacher_logits is None or teacher_ids is None:
            raise ValueError("teacher_logits and teacher_ids come together")
        k = teacher_ids.shape[-1]
        t_at, ld_t = _matrix(teacher_logits, n, k, device, "teacher_logits")
        ids_at, ld_ids = _matrix(teacher_ids, n, k, device, "teacher_ids")
        t_code, id_code = _code(_DTYPE, teacher_logits, "teacher_logits"), _code(_ITYPE, teacher_ids, "teacher_ids")
    labels_at = label_code = 0
    if labels is not None:
        labels_at, label_code = _vector(labels, n, _ITYPE, device, "labels"), _ITYPE[labels.dtype]
    row_loss = torch.empty(n + 1, dtype=torch.float32, device=device)  # and the loss behind it
    d_at = ld_d = 0
    if dlogits is None and want_grad:
        dlogits = torch.empty(logits.shape, dtype=logits.dtype, device=device)
    if dlogits is not None:
        if dlogits.dtype != logits.dtype:
            raise ValueError("dlogits is %s, logits are %s" % (dlogits.dtype, logits.dtype))
        d_at, ld_d = _matrix(dlogits, n, vocab, device, "dlogits")
    at_rows = row_loss.data_ptr()
    _call(lib.adascale_distill, DistillArgs(
        z_at, d_at, t_at, ids_at, labels_at, _f32_vector(row_weight, n, device, "row_weight"), at_rows, at_rows + 4 * n,
        n, vocab, k, ld_z, ld_d, ld_t, ld_ids, _code(_DTYPE, logits, "logits"), t_code, id_code, label_code, T, alpha,
        beta), device, None)
    return Distilled(row_loss[n], row_loss[:n], dlogits)


# --------------------------------------------------------------------------
# block boundary
# --------------------------------------------------------------------------


def _kinds(pre, post):
    try:
        pre, post = _NORM[pre], _NORM[post]
    except KeyError:
        raise ValueError("norms are 'rms', 'layer' or (post only) None: got pre=%r, post=%r" % (pre, post)) from None
    if pre == NORM_NONE:
        raise ValueError("the norm before the next block is 'rms' or 'layer'")
    return pre, post


def _gate(gate, n, d, y, device):
    """Kind, address and row stride of a gate: a float32 [dim] vector or [n, dim] of y's type."""
    if gate is None:
        return GATE_NONE, None, 0
    if gate.dim() == 1:
        return GATE_CHANNEL, _f32_vector(gate, d, device, "gate"), 0
    if gate.dtype != y.dtype:
        raise ValueError("gate is %s, y is %s" % (gate.dtype, y.dtype))
    return (GATE_SIGMOID, *_matrix(gate, n, d, device, "gate"))


def residual_norm(x, y, w_pre, b_pre=None, w_post=None, b_post=None, pre="rms", post=None, gate=None, res_scale=1.0,
                  eps=1e-6, x_new=None, h=None, stream=None):
    """``x_new = x + res_scale * G * post(y)``, ``h = pre(x_new)``: one pass over a block's boundary.

    x: the residual stream, [n, dim]; y: the block's output, same shape (None: ``h = pre(x)``, the norm before the first
    block, in x's type unless ``h`` is given).  ``pre``, ``post``: "rms" or "layer" (post: None for no norm); weights and biases float32 [dim].
    G: 1, a float32 [dim] vector, or sigmoid of a [n, dim] matrix of y's type.  Returns ``(x_new, h)`` of the
    types of x and y; ``x_new`` may be given as x, ``h`` as y.
    """
    device, at = _place(x, stream)
    if at is not None:
        with at:
            return residual_norm(x, y, w_pre, b_pre, w_post, b_post, pre, post, gate, res_scale, eps, x_new, h)
    pre, post = _kinds(pre, post)
    n, d = _rows_of(x, "x")
    x_at, ld_x = _matrix(x, n, d, device, "x")
    y_at = new_at = gate_at = None
    ld_y = ld_new = ld_gate = 0
    kind = GATE_NONE
    if y is None:
        x_new = x
        if h is None:
            h = torch.empty(x.shape, dtype=x.dtype, device=device)
    else:
        if x_new is None:
            x_new = torch.empty(x.shape, dtype=x.dtype, device=device)
        elif x_new.dtype != x.dtype:
            raise ValueError("x_new is %s, x is %s" % (x_new.dtype, x.dtype))
        if h is None:
            h = torch.empty(x.shape, dtype=y.dtype, device=device)
        elif h.dtype != y.dtype:
            raise ValueError("h is %s, y is %s" % (h.dtype, y.dtype))
        y_at, ld_y = _matrix(y, n, d, device, "y")
        new_at, ld_new = _matrix(x_new, n, d, device, "x_new")
        kind, gate_at, ld_gate = _gate(gate, n, d, y, device)
    h_at, ld_h = _matrix(h, n, d, device, "h")
    _call(lib.adascale_residual_norm, ResidualNormArgs(
        x_at, y_at, new_at, h_at, gate_at, _f32_vector(w_post, d, device, "w_post"),
        _f32_vector(b_post, d, device, "b_post"), _f32_vector(w_pre, d, device, "w_pre"),
        _f32_vector(b_pre, d, device, "b_pre"), n, d, ld_x, ld_y, ld_new, ld_h, ld_gate, _code(_DTYPE, x, "x"),
        _code(_DTYPE, h, "h"), post, pre, kind, res_scale, eps), device, None)
    return x_new, h


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
    device, at = _place(x_new, stream)
    if at is not None:
        with at:
            return residual_norm_grad(x_new, y, dx_new, dh, w_pre, w_post, b_post, pre, post, gate, res_scale, eps,
                                      wgrad_dtype, dx, dy, dgate, dw_post, db_post, dw_pre, db_pre, workspace)
    pre, post = _kinds(pre, post)
    n, d = _rows_of(x_new, "x_new")
    if wgrad_dtype not in _DTYPE:
        raise ValueError("wgrad_dtype is float32 or bfloat16")
    if y is None:
        post, gate, dy, dgate = NORM_NONE, None, None, None

    def vector(t, wanted, what):
        """Slot of a vector's gradient and its address."""
        if not wanted:
            return None, None
        if t is None:
            t = torch.empty(d, dtype=wgrad_dtype, device=device)
            return t, t.data_ptr()
        return t, _vector(t, d, (wgrad_dtype,), device, what)

    def matrix(t, like, what):
        if t is None:
            t = torch.empty(x_new.shape, dtype=like.dtype, device=device)
        elif t.dtype != like.dtype:
            raise ValueError("%s is %s, not %s" % (what, t.dtype, like.dtype))
        return (t, *_matrix(t, n, d, device, what))

    x_at, ld_x = _matrix(x_new, n, d, device, "x_new")
    dh_at, ld_dh = _matrix(dh, n, d, device, "dh")
    dx, dx_at, ld_dx = matrix(dx, x_new, "dx")
    new_at = y_at = dy_at = gate_at = dgate_at = None
    ld_new = ld_y = ld_dy = ld_gate = ld_dgate = 0
    kind = GATE_NONE
    if dx_new is not None:
        if dx_new.dtype != x_new.dtype:
            raise ValueError("dx_new is %s, x_new is %s" % (dx_new.dtype, x_new.dtype))
        new_at, ld_new = _matrix(dx_new, n, d, device, "dx_new")
    if y is not None:
        if y.dtype != dh.dtype:
            raise ValueError("y is %s, dh is %s" % (y.dtype, dh.dtype))
        y_at, ld_y = _matrix(y, n, d, device, "y")
        dy, dy_at, ld_dy = matrix(dy, y, "dy")
        kind, gate_at, ld_gate = _gate(gate, n, d, y, device)
        if kind == GATE_SIGMOID:
            dgate, dgate_at, ld_dgate = matrix(dgate, y, "dgate")
        else:
            dgate, dgate_at = vector(dgate, kind == GATE_CHANNEL, "dgate")
    dw_post, dw_post_at = vector(dw_post, post != NORM_NONE, "dw_post")
    db_post, db_post_at = vector(db_post, post == NORM_LAYER, "db_post")
    dw_pre, dw_pre_at = vector(dw_pre, True, "dw_pre")
    db_pre, db_pre_at = vector(db_pre, pre == NORM_LAYER, "db_pre")
    if workspace is None:
        workspace = torch.empty(lib.adascale_residual_norm_grad_workspace(n, d), dtype=torch.uint8, device=device)
    _call(lib.adascale_residual_norm_grad, ResidualNormGradArgs(
        x_at, y_at, new_at, dh_at, gate_at, _f32_vector(w_post, d, device, "w_post"),
        _f32_vector(b_post, d, device, "b_post"), _f32_vector(w_pre, d, device, "w_pre"), dx_at, dy_at, dgate_at,
        dw_post_at, db_post_at, dw_pre_at, db_pre_at, workspace.data_ptr(), workspace.nbytes, n, d, ld_x, ld_y, ld_new,
        ld_dh, ld_gate, ld_dx, ld_dy, ld_dgate, _code(_DTYPE, x_new, "x_new"), _code(_DTYPE, dh, "dh"),
        _DTYPE[wgrad_dtype], post, pre, kind, res_scale, eps), device, None)
    return BoundaryGrads(dx, dy, dgate, dw_post, db_post, dw_pre, db_pre)


def residual_norm_grad_workspace(n_rows, dim) -> int:
    return lib.adascale_residual_norm_grad_workspace(n_rows, dim)
