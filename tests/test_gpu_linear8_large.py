"""Projections in 8 bits of as many rows as the calls take."""
import pytest
import torch

from linear8_testlib import check_product, check_rows, gate_and_up, random_rows, random_rows8, random_weight8

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32 = torch.float32
MOST = (1 << 24) - 1


def lib():
    from paper_2602_12957_amd import linear8
    return linear8


def room(gb):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gb << 30:
        pytest.skip(f"needs {gb} GB")


# ------------------------------------------------------------------------------------------------------------ as many as there may be
def sparse_rows8(rows, dim, at, seed):
    """Rows of zeros but for those at `at`, and these by themselves."""
    L = lib()
    r, few = L.Rows8.empty(rows, dim, DEV), random_rows8(len(at), dim, seed)
    r.codes.zero_(), r.scale.fill_(127)
    r.codes[at], r.scale[at] = few.codes, few.scale
    return r, few


def places(*near):
    return torch.cat([torch.arange(3)] + [torch.arange(n - 3, n + 3) for n in near] + [torch.arange(MOST - 3, MOST)]).to(DEV)


@pytest.mark.parametrize("scale", [torch.uint8, F32])
def test_gated_of_the_most_rows(scale):
    """2^24 - 1 rows of 128 to 8192: more tiles than a launch has, results behind 2^37 bytes."""
    room(150)
    L = lib()
    at = places(1 << 23, 65535 * 256)
    a, few = sparse_rows8(MOST, 128, at, 1)
    w = L.Weight8.quantize(random_rows(2 * 8192, 128, 2, F32, spread=0.3) / 128, scale)
    got = L.gated(a, w)
    want, worst, _ = gate_and_up(few, w)
    check_rows(type("R", (), dict(codes=got.codes[at], scale=got.scale[at], dim=8192, rows=len(at))), want, worst)
    others = torch.arange(3, MOST, 99991, device=DEV)
    others = others[~torch.isin(others, at)]
    assert not bool((got.codes[others] & 127).any()) and bool((got.scale[others, :64] == 127).all())


def test_linear_of_the_most_rows():
    """2^24 - 1 rows of 128 to 2048 in fp32, float scales: more tiles than a launch has."""
    room(150)
    L = lib()
    at = places(1 << 23, (4194303 // 16) * 64)
    a, few = sparse_rows8(MOST, 128, at, 1)
    w = random_weight8(2048, 128, 2, F32)
    got = L.linear(a, w, F32)
    check_product(got[at], few, w)
    others = torch.arange(3, MOST, 99991, device=DEV)
    others = others[~torch.isin(others, at)]
    assert not bool(got[others].any())
