"""Host-only checks of the language-model operators' C ABI: exports, struct layouts, refusals before any CUDA call."""
import ctypes as C
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ops():
    from paper_2007_05105_b200 import build
    build.build()
    from paper_2007_05105_b200 import ops
    return ops


def _header():
    text = open(os.path.join(ROOT, "include", "adascale_ops.h")).read()
    return re.sub(r"/\*.*?\*/", "", text, flags=re.S)


def test_library_exports_every_declared_symbol(ops):
    declared = set(re.findall(r"\b(adascale_[a-z_]+)\s*\(", _header()))
    assert declared == set(ops.EXPORTS)
    for name in declared:
        assert hasattr(ops.lib, name), name


STRUCTS = {"adascale_embed_args": "EmbedArgs", "adascale_embed_grad_args": "EmbedGradArgs",
           "adascale_distill_args": "DistillArgs", "adascale_residual_norm_args": "ResidualNormArgs",
           "adascale_residual_norm_grad_args": "ResidualNormGradArgs"}


def test_struct_layouts_match_the_header(ops, tmp_path):
    """Size of every struct and offset of every field, as a C compiler sees them."""
    lines = []
    for c_name, py_name in STRUCTS.items():
        lines.append('printf("%s %%zu\\n", sizeof(%s));' % (py_name, c_name))
        for field, _ in getattr(ops, py_name)._fields_:
            lines.append('printf("%s.%s %%zu\\n", offsetof(%s, %s));' % (py_name, field, c_name, field))
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "%s"\nint main(void) { %s return 0; }\n'
                   % (os.path.join(ROOT, "include", "adascale_ops.h"), "\n".join(lines)))
    subprocess.check_call(["gcc", "-o", str(tmp_path / "layout"), str(src)])
    for line in subprocess.check_output([str(tmp_path / "layout")], text=True).splitlines():
        name, value = line.split()
        cls, _, field = name.partition(".")
        cls = getattr(ops, cls)
        assert (getattr(cls, field).offset if field else C.sizeof(cls)) == int(value), name


# valid arguments of every call, as far as the host can tell; the addresses are never followed
A = 1 << 20
VALID = {
    "embed": dict(tokens=A, table=A, out=A, n_tokens=4, vocab=10, dim=8, ld_table=8, ld_out=8, scale=1.0),
    "embed_grad": dict(tokens=A, dout=A, grad=A, workspace=A, workspace_bytes=1 << 20, n_tokens=4, vocab=10, dim=8,
                       ld_dout=8, ld_grad=8, padding_idx=-1, scale=1.0),
    "distill": dict(logits=A, dlogits=A, teacher_logits=A, teacher_ids=A, row_loss=A, loss=A, n_rows=2, vocab=16, n_top=4,
                    ld_logits=16, ld_dlogits=16, ld_teacher=4, ld_ids=4, temperature=1.0, alpha=1.0, beta=0.0),
    "residual_norm": dict(x=A, y=A, x_new=A, h=2 * A, w_post=A, w_pre=A, n_rows=2, dim=8, ld_x=8, ld_y=8, ld_x_new=8,
                          ld_h=8, post=1, pre=1, res_scale=1.0, eps=1e-6),
    "residual_norm_grad": dict(x_new=A, y=A, dx_new=A, dh=A, w_post=A, w_pre=A, dx=2 * A, dy=2 * A, workspace=A,
                               workspace_bytes=1 << 20, n_rows=2, dim=8, ld_x_new=8, ld_y=8, ld_dx_new=8, ld_dh=8,
                               ld_dx=8, ld_dy=8, post=1, pre=1, res_scale=1.0, eps=1e-6),
}
CLASS = {"embed": "EmbedArgs", "embed_grad": "EmbedGradArgs", "distill": "DistillArgs",
         "residual_norm": "ResidualNormArgs", "residual_norm_grad": "ResidualNormGradArgs"}


def _status(ops, call, **over):
    args = getattr(ops, CLASS[call])(**{**VALID[call], **over})
    return getattr(ops.lib, "adascale_" + call)(C.byref(args), None)


NAN, INF = float("nan"), float("inf")
REFUSED = [
    ("embed", 1, [dict(tokens=None), dict(table=None), dict(out=None), dict(n_tokens=-1), dict(vocab=0), dict(dim=0),
                  dict(ld_table=7), dict(ld_out=7), dict(token_type=2), dict(table_dtype=5), dict(out_dtype=-1),
                  dict(scale=NAN), dict(scale=INF)]),
    ("embed", 2, [dict(tokens=A + 2), dict(tokens=A + 4, token_type=1), dict(table=A + 2), dict(out=A + 1, out_dtype=1)]),
    ("embed", 5, [dict(n_tokens=1 << 31), dict(vocab=1 << 31)]),
    ("embed_grad", 1, [dict(tokens=None), dict(dout=None), dict(grad=None), dict(workspace=None), dict(workspace_bytes=64),
                       dict(n_tokens=-1), dict(vocab=0), dict(dim=0), dict(ld_dout=7), dict(ld_grad=7),
                       dict(token_type=2), dict(dout_dtype=2), dict(grad_dtype=2), dict(scale=NAN)]),
    ("embed_grad", 2, [dict(tokens=A + 1), dict(dout=A + 2), dict(grad=A + 2), dict(workspace=A + 8)]),
    ("embed_grad", 5, [dict(n_tokens=1 << 31), dict(vocab=1 << 31)]),
    ("distill", 1, [dict(logits=None), dict(row_loss=None), dict(loss=None), dict(teacher_logits=None),
                    dict(teacher_ids=None), dict(n_rows=-1), dict(vocab=0), dict(n_top=-1), dict(ld_logits=15),
                    dict(ld_dlogits=15), dict(ld_teacher=3), dict(ld_ids=3), dict(dtype=2), dict(teacher_dtype=2),
                    dict(id_type=2), dict(label_type=2), dict(temperature=0.0), dict(temperature=NAN),
                    dict(temperature=1e4), dict(alpha=-1.0), dict(alpha=NAN), dict(beta=INF),
                    dict(dlogits=A, logits=A, ld_dlogits=32)]),
    ("distill", 2, [dict(logits=A + 2), dict(dlogits=A + 2), dict(row_loss=A + 2), dict(loss=A + 2), dict(weight=A + 2),
                    dict(teacher_logits=A + 2), dict(teacher_ids=A + 4, id_type=1), dict(labels=A + 2)]),
    ("distill", 5, [dict(n_top=1025, ld_teacher=1025, ld_ids=1025), dict(vocab=1 << 31, ld_logits=1 << 31)]),
    ("residual_norm", 1, [dict(x=None), dict(h=None), dict(w_pre=None), dict(w_post=None), dict(x_new=None),
                          dict(n_rows=-1), dict(dim=0), dict(ld_x=7), dict(ld_y=7), dict(ld_x_new=7), dict(ld_h=7),
                          dict(pre=0), dict(pre=3), dict(post=3), dict(gate_kind=3), dict(gate_kind=1),
                          dict(gate_kind=2, gate=A, ld_gate=7), dict(x_dtype=2), dict(y_dtype=2), dict(eps=-1.0),
                          dict(eps=NAN), dict(res_scale=INF), dict(x=A, x_new=A, ld_x_new=16), dict(h=A, y=A, ld_h=16)]),
    ("residual_norm", 2, [dict(x=A + 2), dict(y=A + 1, y_dtype=1), dict(h=A + 2), dict(x_new=A + 2), dict(w_pre=A + 2),
                          dict(w_post=A + 1), dict(gate_kind=1, gate=A + 2)]),
    ("residual_norm", 5, [dict(dim=16385, ld_x=16385, ld_y=16385, ld_x_new=16385, ld_h=16385)]),
    ("residual_norm_grad", 1, [dict(x_new=None), dict(dh=None), dict(dx=None), dict(w_pre=None), dict(w_post=None),
                               dict(workspace=None), dict(workspace_bytes=16), dict(n_rows=-1), dict(dim=0),
                               dict(ld_x_new=7), dict(ld_y=7), dict(ld_dx_new=7), dict(ld_dh=7), dict(ld_dx=7),
                               dict(ld_dy=7), dict(pre=0), dict(post=3), dict(gate_kind=1), dict(wgrad_dtype=2),
                               dict(gate_kind=2, gate=A, ld_gate=8, dgate=A, ld_dgate=7), dict(eps=NAN),
                               dict(dx=A, dx_new=A, ld_dx=16), dict(dy=A, dh=A, ld_dy=16)]),
    ("residual_norm_grad", 2, [dict(x_new=A + 2), dict(dh=A + 2), dict(dx=A + 2), dict(dy=A + 2), dict(workspace=A + 4),
                               dict(dw_pre=A + 2), dict(db_post=A + 1, wgrad_dtype=1), dict(gate_kind=1, gate=A, dgate=A + 2)]),
    ("residual_norm_grad", 5, [dict(dim=16385)]),
]


@pytest.mark.parametrize("call,status,over", [(c, s, o) for c, s, group in REFUSED for o in group])
def test_refusals(ops, call, status, over):
    assert _status(ops, call, **over) == status


def test_null_arguments_are_refused(ops):
    for call in VALID:
        assert getattr(ops.lib, "adascale_" + call)(None, None) == 1


def test_nothing_to_do_is_no_error(ops):
    assert _status(ops, "embed", n_tokens=0, tokens=None, table=None, out=None) == 0
    assert _status(ops, "embed_grad", n_tokens=0, accumulate=1, tokens=None, dout=None) == 0
    assert _status(ops, "residual_norm", n_rows=0, x=None) == 0


def test_without_a_device_the_calls_fail_cleanly(ops):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a device is present")
    for call in VALID:
        assert _status(ops, call) == 3


def test_workspace_sizes(ops):
    assert ops.embed_grad_workspace(0, 8) == 0
    assert ops.embed_grad_workspace(-1, 8) == 0 and ops.embed_grad_workspace(4, 0) == 0
    assert ops.embed_grad_workspace(1 << 31, 8) == 0
    small, large = ops.embed_grad_workspace(100, 64), ops.embed_grad_workspace(100000, 64)
    assert 0 < small < large
    assert ops.residual_norm_grad_workspace(1, 16385) == 0
    assert 0 < ops.residual_norm_grad_workspace(1, 9) <= ops.residual_norm_grad_workspace(1 << 30, 9)


def test_tensors_on_the_host_are_refused(ops):
    import torch
    t = torch.zeros(2, 8)
    ids = torch.zeros(2, dtype=torch.int64)
    with pytest.raises(ValueError):
        ops.embed(ids, t)
    with pytest.raises(ValueError):
        ops.embed_grad(ids, t, t)
    with pytest.raises(ValueError):
        ops.distill(t)
    with pytest.raises(ValueError):
        ops.residual_norm(t, t, t[0])
    with pytest.raises(ValueError):
        ops.residual_norm_grad(t, t, t, t, t[0])
