"""Projections in 8 bits: the largest strides and sizes that the C entries take."""
import pytest

import paper_2602_12957_amd.binding as B
from test_linear8_host import FAKE, call, rows, weight


@pytest.mark.parametrize("name,where", [("rows", "out"), ("norm_rows", "out"), ("read_rows", "rows"), ("linear", "rows"), ("gated", "rows"), ("gated", "out")])
def test_rows_too_far_apart(name, where):
    assert call(name, n_rows=4, **{where: rows(code_stride=(1 << 23) + 16)}) == B.HSD_ERANGE


@pytest.mark.parametrize("name,kw", [("weights", dict(n_out=4)), ("linear", dict(n_rows=4)), ("gated", dict(n_rows=4))])
def test_weight_rows_too_far_apart(name, kw):
    assert call(name, **kw, **{"out" if name == "weights" else "w": weight(code_stride=(1 << 23) + 16)}) == B.HSD_ERANGE


def test_too_many_weight_rows_to_be_made():
    assert call("weights", n_out=65535 * 128 + 1, w=FAKE, out=weight()) == B.HSD_ERANGE
