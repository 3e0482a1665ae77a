"""Host-only checks of the C ABI of the position-bias, expert and clipping operators: struct layouts, limits, refusals before any CUDA call."""
import ctypes as C
import re
import subprocess

import pytest

import test_ops_abi as A
from test_ops_abi import ops  # noqa: F401  (the fixture)

STRUCTS = {"adascale_position_softmax_args": "PositionSoftmaxArgs", "adascale_position_softmax_grad_args": "PositionSoftmaxGradArgs",
           "adascale_expert_matmul_args": "ExpertMatmulArgs", "adascale_expert_matmul_grad_args": "ExpertMatmulGradArgs",
           "adascale_clip_grads_args": "ClipGradsArgs"}


def test_struct_layouts_match_the_header(ops, tmp_path, monkeypatch):  # noqa: F811
    monkeypatch.setattr(A, "STRUCTS", STRUCTS)
    A.test_struct_layouts_match_the_header(ops, tmp_path)


def test_limits_are_those_of_the_header(ops):  # noqa: F811
    header = A._header()
    for name in ("POSITION_MAX_BUCKETS", "POSITION_MAX_DISTANCE", "EXPERT_MAX_EXPERTS", "EXPERT_MAX_DIM", "CLIP_MAX_TENSORS"):
        assert int(re.search(r"#define ADASCALE_%s (\d+)" % name, header).group(1)) == getattr(ops, name)


P = 1 << 20  # an address that is never followed
ROWS = dict(batch=2, heads=3, n_queries=4, n_keys=8)


def strides(name):
    return {"%s_stride_b" % name: 96, "%s_stride_h" % name: 32, "%s_stride_q" % name: 8}


VALID = {
    "position_softmax": dict(scores=P, probs=2 * P, table=P, ld_table=3, n_buckets=8, max_distance=16, scale=1.0, **ROWS, **strides("scores"),
                             **strides("probs")),
    "position_softmax_grad": dict(probs=P, dprobs=P, dscores=2 * P, dtable=P, workspace=P, workspace_bytes=1 << 20, ld_dtable=3, n_buckets=8,
                                  max_distance=16, scale=1.0, **ROWS, **strides("probs"), **strides("dprobs"), **strides("dscores")),
    "expert_matmul": dict(x=P, w=P, y=2 * P, offsets=P, n_rows=10, n_experts=2, in_dim=16, out_dim=24, ld_x=16, ld_w=16, stride_w=384, ld_y=24),
    "expert_matmul_grad": dict(dy=P, x=P, w=P, dx=2 * P, dw=3 * P, offsets=P, n_rows=10, n_experts=2, in_dim=16, out_dim=24, ld_dy=24, ld_x=16,
                               ld_w=16, stride_w=384, ld_dx=16, ld_dw=16, stride_dw=384),
}
CLASS = {"position_softmax": "PositionSoftmaxArgs", "position_softmax_grad": "PositionSoftmaxGradArgs", "expert_matmul": "ExpertMatmulArgs",
         "expert_matmul_grad": "ExpertMatmulGradArgs"}
NAN, INF, BIG = float("nan"), float("inf"), 1 << 31


def status(ops, call, **over):  # noqa: F811
    args = getattr(ops, CLASS[call])(**{**VALID[call], **over})
    return getattr(ops.lib, "adascale_" + call)(C.byref(args), None)


COMMON = [dict(batch=-1), dict(heads=-1), dict(n_queries=-1), dict(n_keys=-1), dict(dtype=2), dict(scale=NAN), dict(scale=INF),
          dict(lengths=P, length_type=2), dict(starts=P, start_type=-1), dict(n_buckets=1), dict(n_buckets=7, bidirectional=1), dict(n_buckets=2, bidirectional=1),
          dict(max_distance=4), dict(max_distance=2, bidirectional=1), dict(max_distance=0)]
REFUSED = [
    ("position_softmax", 1, COMMON + [dict(scores=None), dict(probs=None), dict(table=None), dict(ld_table=2), dict(scores_stride_b=-1),
                                      dict(probs_stride_q=7), dict(probs_stride_h=31), dict(probs_stride_b=0), dict(probs=P, scores=P, probs_stride_h=40, probs_stride_b=200)]),
    ("position_softmax", 2, [dict(scores=P + 2), dict(probs=P + 1, dtype=1), dict(table=P + 2), dict(lengths=P + 4, length_type=1), dict(starts=P + 2)]),
    ("position_softmax", 5, [dict(n_buckets=129, max_distance=1000), dict(max_distance=16385), dict(n_keys=(1 << 29) + 1), dict(n_queries=(1 << 29) + 1),
                             dict(batch=BIG), dict(heads=65536), dict(batch=1 << 20, n_queries=1 << 20)]),
    ("position_softmax_grad", 1, COMMON + [dict(probs=None), dict(dprobs=None), dict(dscores=None, dtable=None), dict(workspace=None), dict(workspace_bytes=64),
                                           dict(wgrad_dtype=2), dict(ld_dtable=2), dict(dscores_stride_q=0), dict(dprobs_stride_h=-1),
                                           dict(dscores=P, dscores_stride_b=128), dict(dscores=P, probs=3 * P, dprobs_stride_b=128)]),
    ("position_softmax_grad", 2, [dict(probs=P + 2), dict(dprobs=P + 1, dtype=1), dict(dscores=P + 2), dict(dtable=P + 2), dict(workspace=P + 8)]),
    ("position_softmax_grad", 5, [dict(n_buckets=130, max_distance=1000), dict(n_keys=(1 << 29) + 1)]),
    ("expert_matmul", 1, [dict(x=None), dict(w=None), dict(y=None), dict(offsets=None), dict(n_rows=-1), dict(n_experts=0), dict(in_dim=0), dict(out_dim=0),
                          dict(ld_x=8), dict(ld_w=8), dict(stride_w=376), dict(ld_y=23), dict(offset_type=2), dict(y_dtype=2)]),
    ("expert_matmul", 2, [dict(x=P + 8), dict(w=P + 2), dict(y=P + 2), dict(y=P + 1, y_dtype=1), dict(offsets=P + 4, offset_type=1), dict(ld_x=17),
                          dict(ld_w=20, stride_w=480), dict(stride_w=388)]),
    ("expert_matmul", 5, [dict(n_rows=BIG), dict(n_experts=1025), dict(in_dim=(1 << 20) + 8), dict(out_dim=(1 << 20) + 8),
                          dict(n_rows=BIG - 1024, out_dim=1 << 20)]),
    ("expert_matmul_grad", 1, [dict(dy=None), dict(x=None, w=None, dw=None), dict(dx=None), dict(dw=None), dict(offsets=None), dict(n_rows=-1), dict(dx_dtype=2),
                               dict(dw_dtype=2), dict(ld_dy=23), dict(ld_x=8), dict(ld_dx=15), dict(ld_dw=15), dict(stride_dw=383), dict(stride_w=376)]),
    ("expert_matmul_grad", 2, [dict(dy=P + 2), dict(x=P + 8), dict(w=P + 8), dict(dx=P + 2), dict(dw=P + 2), dict(ld_dy=25), dict(ld_x=20), dict(stride_w=388)]),
    ("expert_matmul_grad", 5, [dict(n_experts=1025), dict(n_rows=BIG)]),
]


@pytest.mark.parametrize("call,code,over", [(c, s, o) for c, s, group in REFUSED for o in group])
def test_refusals(ops, call, code, over):  # noqa: F811
    assert status(ops, call, **over) == code


def clip(ops, n=3, null=(), **over):  # noqa: F811
    """Status of a call with three gradients of 100 elements."""
    lists = dict(grads=[P, 2 * P, 3 * P], out=[4 * P, 5 * P, 6 * P], numels=[100, 0, 100], grad_dtypes=[0, 0, 1], out_dtypes=[1, 1, 1])
    kinds = dict(grads=C.c_void_p, out=C.c_void_p, numels=C.c_int64, grad_dtypes=C.c_int32, out_dtypes=C.c_int32)
    plain = dict(norm=P, workspace=P, workspace_bytes=1 << 20, n_tensors=n, max_norm=1.0, eps=1e-6)
    for name, value in over.items():
        if name in lists:
            lists[name] = value
        else:
            plain[name] = value
    held = {k: (kinds[k] * 3)(*v) for k, v in lists.items()}
    args = ops.ClipGradsArgs(**plain, **{k: None if k in null else C.addressof(v) for k, v in held.items()})
    return ops.lib.adascale_clip_grads(C.byref(args), None)


@pytest.mark.parametrize("code,over", [(1, o) for o in [
    dict(n=-1), dict(null=("grads",)), dict(null=("numels",)), dict(null=("grad_dtypes",)), dict(null=("out_dtypes",)), dict(norm=None), dict(workspace=None),
    dict(workspace_bytes=64), dict(max_norm=NAN), dict(max_norm=-1.0), dict(eps=INF), dict(eps=-1.0), dict(numels=[100, -1, 100]), dict(grad_dtypes=[0, 0, 2]),
    dict(out_dtypes=[0, 3, 0]), dict(grads=[None, P, P]), dict(out=[None, P, P]), dict(out=[4 * P, P, 4 * P]), dict(out=[4 * P, P, 4 * P + 198]), dict(out=[P, 2 * P, P]),
    dict(out=[3 * P + 100, 2 * P, 6 * P]), dict(out=[P, 2 * P, 6 * P])]] + [(2, o) for o in [
        dict(grads=[P + 2, P, P]), dict(grads=[P, P, 3 * P + 1]), dict(out=[4 * P + 1, P, 6 * P]), dict(norm=P + 2), dict(workspace=P + 8)]] + [(5, o) for o in [
            dict(n=65537), dict(numels=[1 << 41, 0, 1])]])
def test_clip_refusals(ops, code, over):  # noqa: F811
    assert clip(ops, **over) == code


def test_null_arguments_are_refused(ops):  # noqa: F811
    for call in (*VALID, "clip_grads"):
        assert getattr(ops.lib, "adascale_" + call)(None, None) == 1


def test_nothing_to_do_is_no_error(ops):  # noqa: F811
    for name in ("batch", "heads", "n_queries", "n_keys"):
        assert status(ops, "position_softmax", **{name: 0}, scores=None, probs=None, table=None) == 0
        assert status(ops, "position_softmax_grad", **{name: 0}, probs=None, dprobs=None, accumulate=1) == 0
    assert status(ops, "expert_matmul", n_rows=0, x=None, y=None) == 0
    assert status(ops, "expert_matmul_grad", n_rows=0, x=None, dy=None, dx=None, accumulate=1) == 0


def test_without_a_device_the_calls_fail_cleanly(ops):  # noqa: F811
    import torch
    if torch.cuda.is_available():
        pytest.skip("a device is present")
    for call in VALID:
        assert status(ops, call) == 3
    assert clip(ops) == 3


def test_workspace_sizes(ops):  # noqa: F811
    assert ops.clip_grads_workspace(-1) == 0 and ops.clip_grads_workspace(65537) == 0
    assert 0 < ops.clip_grads_workspace(0) <= ops.clip_grads_workspace(5000)
    assert ops.position_softmax_grad_workspace(-1, 8) == 0 and ops.position_softmax_grad_workspace(4, 129) == 0
    assert 0 < ops.position_softmax_grad_workspace(4, 8) <= ops.position_softmax_grad_workspace(65535, 128)


def test_tensors_on_the_host_are_refused(ops):  # noqa: F811
    import torch
    t, s = torch.zeros(2, 8), torch.zeros(1, 2, 3, 4)
    ids = torch.zeros(2, dtype=torch.int64)
    for bad in [lambda: ops.position_softmax(s, t), lambda: ops.position_softmax_grad(s, s, 8), lambda: ops.expert_matmul(t, t[None], ids),
                lambda: ops.expert_matmul_grad(t, ids, x=t), lambda: ops.grad_norm([t]), lambda: ops.clip_grads([t], 1.0)]:
        with pytest.raises(ValueError):
            bad()


def test_slots_without_what_they_are_made_of_are_refused(ops):  # noqa: F811
    """Before the tensors' device is looked at."""
    import torch
    x, w, dy, ids = torch.zeros(10, 16), torch.zeros(2, 24, 16), torch.zeros(10, 24), torch.zeros(3, dtype=torch.int64)
    for given in (dict(w=w, dw=torch.zeros(2, 24, 16)), dict(x=x, dx=torch.zeros(10, 16))):
        with pytest.raises(ValueError, match="needed for it"):
            ops.expert_matmul_grad(dy, ids, **given)


@pytest.mark.parametrize("stream", [None, 0])
def test_what_is_no_list_of_gradients(ops, stream):  # noqa: F811
    """Refused in the same way with a stream and without."""
    for call in (lambda g: ops.grad_norm(g, stream=stream), lambda g: ops.clip_grads(g, 1.0, stream=stream)):
        for empty in ([], (), iter(())):
            with pytest.raises(ValueError, match="empty"):
                call(empty)
        for bad in (5, [None], (3,), None):
            with pytest.raises(TypeError):
                call(bad)


def test_a_list_too_long_is_too_large(ops):  # noqa: F811
    """Also with the workspace that its size asks for, which is none."""
    assert clip(ops, n=65537, workspace=None, workspace_bytes=ops.clip_grads_workspace(65537)) == 5
