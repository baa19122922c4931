"""Projections in 8 bits at their largest: few rows to many columns, long sums, and as many rows as the calls take."""
import pytest
import torch

from linear8_testlib import BLOCK, check_product, check_rows, gate_and_up, random_rows, random_rows8, random_weight8, row_values

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
MOST = (1 << 24) - 1


def lib():
    from paper_2602_12957_amd import linear8
    return linear8


def room(gb):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gb << 30:
        pytest.skip(f"needs {gb} GB")


# ------------------------------------------------------------------------------------------------------------ wide and long ones
@pytest.mark.parametrize("rows,n_out,dim", [(1, 70001, 300), (1, 131073, 130), (17, 70000, 256), (64, 70000, 256), (64, 33000, 1000), (3, 40, 1 << 20), (20, 100, 70000), (300, 256, 65664),
                                            (2100, 520, 16500)])
@pytest.mark.parametrize("scale", [torch.uint8, F32])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_linear_wide_and_long(rows, n_out, dim, scale, dtype):
    a, w = random_rows8(rows, dim, rows + dim), random_weight8(n_out, dim, n_out, scale)
    check_product(lib().linear(a, w, dtype), a, w)


@pytest.mark.parametrize("rows,d_ffn,dim", [(1, 33024, 128), (5, 33024, 300), (70, 33024, 130), (3, 128, 65664), (300, 256, 16500)])
@pytest.mark.parametrize("scale", [torch.uint8, F32])
def test_gated_wide_and_long(rows, d_ffn, dim, scale):
    L = lib()
    a = L.quantize_rows(random_rows(rows, dim, rows + dim, spread=0.5))
    w = L.Weight8.quantize(random_rows(2 * d_ffn, dim, d_ffn, F32, spread=0.3) / dim ** 0.5, scale)
    want, worst, _ = gate_and_up(a, w)
    check_rows(L.gated(a, w), want, worst)


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


def test_reading_the_most_rows():
    room(70)
    at = places(1 << 23)
    a, few = sparse_rows8(MOST, 1100, at, 1)
    got = a.read(BF)
    assert torch.equal(got[at].double(), row_values(few.codes, few.scale, 1100))
    others = torch.arange(3, MOST, 99991, device=DEV)
    others = others[~torch.isin(others, at)]
    assert not bool(got[others].any())


@pytest.mark.parametrize("scale", [torch.uint8, F32])
def test_making_the_most_weight_rows(scale):
    room(20)
    L = lib()
    n = 65535 * BLOCK
    w = torch.zeros((n, 100), dtype=BF, device=DEV)
    w[:3 * BLOCK], w[-3 * BLOCK:] = random_rows(3 * BLOCK, 100, 1), random_rows(3 * BLOCK, 100, 2)
    all8, first, last = (L.Weight8.quantize(x, scale) for x in (w, w[:3 * BLOCK], w[-3 * BLOCK:]))
    assert torch.equal(all8.codes[:3 * BLOCK], first.codes) and torch.equal(all8.scale[:3], first.scale)
    assert torch.equal(all8.codes[-3 * BLOCK:], last.codes) and torch.equal(all8.scale[-3:], last.scale)
    assert not bool(all8.codes[3 * BLOCK:-3 * BLOCK].any()) and bool((all8.scale[3:-3] == (127 if scale == torch.uint8 else 1)).all())


@pytest.mark.parametrize("rows", [1, 70])
@pytest.mark.parametrize("scale", [torch.uint8, F32])
def test_linear_to_the_most_columns(rows, scale):
    room(30)
    L = lib()
    g = torch.Generator(device=DEV).manual_seed(1)
    a, small = random_rows8(rows, 100, 1), random_weight8(1, 100, 2, scale)
    codes = torch.randint(0, 127, (MOST, 128), generator=g, device=DEV, dtype=torch.uint8)
    codes[:, 100:] = 0
    w = L.Weight8(codes, small.scale.expand(1 << 17, 1).contiguous(), 100)
    w.scale[-7:] = w.scale[-7:] * 2 if scale == F32 else w.scale[-7:] + 1
    for dtype in (BF, F32):
        got = L.linear(a, w, dtype)
        for first in (0, 1 << 23, (1 << 24) - 4096):
            check_product(got[:, first:first + 4096], a, L.Weight8(codes[first:first + 4096], w.scale[first // BLOCK:first // BLOCK + 32], 100))
