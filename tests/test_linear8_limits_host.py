"""Projections in 8 bits: the largest strides and sizes that the C entries take, and whether the count of other codes that the GPU tests go by sees what it is for."""
import pytest
import torch

import paper_2602_12957_amd.binding as B
from linear8_testlib import U, moved_codes, nearest_codes_values
from test_linear8_host import FAKE, call, rows, weight


@pytest.mark.parametrize("name,where", [("rows", "out"), ("norm_rows", "out"), ("read_rows", "rows"), ("linear", "rows"), ("gated", "rows"), ("gated", "out")])
def test_rows_too_far_apart(name, where):
    assert call(name, n_rows=4, **{where: rows(code_stride=(1 << 23) + 16)}) == B.HSD_ERANGE


@pytest.mark.parametrize("name,kw", [("weights", dict(n_out=4)), ("linear", dict(n_rows=4)), ("gated", dict(n_rows=4))])
def test_weight_rows_too_far_apart(name, kw):
    assert call(name, **kw, **{"out" if name == "weights" else "w": weight(code_stride=(1 << 23) + 16)}) == B.HSD_ERANGE


def test_too_many_weight_rows_to_be_made():
    assert call("weights", n_out=65535 * 128 + 1, w=FAKE, out=weight()) == B.HSD_ERANGE


def gates(dim, seed):
    """Sums of 2 * 256 columns of 512 rows as products of normal operands have them, their rms errors in fp32, and silu(gate) * up."""
    g = torch.Generator().manual_seed(seed)
    s = torch.randn((512, 512), generator=g, dtype=torch.float64)
    return s, U * (dim / 6.0) ** 0.5 * torch.ones_like(s)


def swiglu(s):
    g, u = s.split(256, 1)
    return g * torch.sigmoid(g) * u


def rms_of(s, r):
    g, u = s.split(256, 1)
    rg, ru = r.split(256, 1)
    sig = torch.sigmoid(g)
    return ((sig * (1 + g * (1 - sig)) * u * rg).square() + (g * sig * ru).square()).sqrt()


@pytest.mark.parametrize("dim", [1024, 4096])
@pytest.mark.parametrize("seed", [1, 2, 3])
def test_the_count_of_other_codes(dim, seed):
    """Codes of sums with the errors that fp32 leaves pass; of sums with errors of 1.5e-5, as 8-bit products leave them, they do not."""
    s, r = gates(dim, seed)
    y, rms = swiglu(s), rms_of(s, r)
    g = torch.Generator().manual_seed(seed + 100)
    noise = torch.randn(s.shape, generator=g, dtype=torch.float64)
    moved, most = moved_codes(nearest_codes_values(swiglu(s + r * noise))[0], y, rms)
    assert 0 < moved <= most
    moved, most = moved_codes(nearest_codes_values(swiglu(s + 1.5e-5 * noise))[0], y, rms)
    assert moved > most
