"""Host-only: the largest sizes of the language-model operators, refused one beyond, before any CUDA call."""
import re

import pytest

import test_ops_abi as A
from test_ops_abi import ops  # noqa: F401  (the fixture)


def test_limits_are_those_of_the_header(ops):  # noqa: F811
    header = A._header()
    for name in ("EMBED_MAX_DIM", "DISTILL_MAX_K", "NORM_MAX_DIM"):
        assert int(re.search(r"#define ADASCALE_%s (\d+)" % name, header).group(1)) == getattr(ops, name)


@pytest.mark.parametrize("call,lds", [("embed", ("ld_table", "ld_out")), ("embed_grad", ("ld_dout", "ld_grad"))])
def test_widest_token_table(ops, call, lds):  # noqa: F811
    """Columns are 32-bit numbers in the kernels."""
    for dim in (ops.EMBED_MAX_DIM + 1, (1 << 31) - 1, 1 << 31, 1 << 40):
        assert A._status(ops, call, dim=dim, **{k: dim for k in lds}) == 5
    assert ops.embed_grad_workspace(4, ops.EMBED_MAX_DIM) > 0 and ops.embed_grad_workspace(4, ops.EMBED_MAX_DIM + 1) == 0
