"""Products in 8 bits by value: codes of gate and up that are the definition's, float scales of every kind, scales that are no numbers, sums that cancel,
weights of small magnitudes."""
import math

import pytest
import torch

from linear8_testlib import (BLOCK, HALF, U, check_product, check_rows, exponent, gate_and_up, moved_codes, product, random_rows, random_rows8,
                             random_weight8, weight_values)

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
FORMS = [300, 700, 1500, 4000]      # rows that 4096 weight rows' gate and up take in tiles of 32, 64, 128 and 256


def lib():
    from paper_2602_12957_amd import linear8
    return linear8


@pytest.mark.parametrize("rows", FORMS)
@pytest.mark.parametrize("dim", [1024, 4096])
@pytest.mark.parametrize("scale", [torch.uint8, F32])
def test_gated_codes_are_the_definition_s(rows, dim, scale):
    """Other codes than those of the sums in 64 bits are as few as fp32's roundings make them: the 8-bit products' cut (1.5e-5 of a sum) would make many more."""
    L = lib()
    a = L.quantize_rows(random_rows(rows, dim, rows + dim, spread=0.5))
    w = L.Weight8.quantize(random_rows(4096, dim, 7, F32, spread=0.3) / dim ** 0.5, scale)
    want, worst, rms = gate_and_up(a, w)
    got = L.gated(a, w)
    check_rows(got, want, worst)
    moved, most = moved_codes(got.read(F32).double(), want, rms)
    assert moved <= most, (moved, most)


def small_codes(n, dim, seed, size):
    """e4m3 codes of normal values times `size`, padded to whole blocks with zeros."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.nn.functional.pad(torch.randn((n, dim), generator=g, device=DEV) * size, (0, -dim % BLOCK))
    return x.to(torch.float8_e4m3fn).view(torch.uint8)


def float_scaled(rows, dim, t, cg, cu, size=1.0, f=2048):
    """Rows whose block b has the power 2^t[b], and gate and up weights whose scales take it back but for 2^cg and 2^cu: +-[1, 2) * 2^(c - t[b])."""
    L = lib()
    a = L.Rows8(small_codes(rows, dim, rows, size), torch.tensor(([127 + e for e in t] + [127])[:4], dtype=torch.uint8, device=DEV).expand(rows, 4).contiguous(), dim)
    g = torch.Generator().manual_seed(5)
    s = 1 + torch.rand((2 * f // BLOCK, len(t)), generator=g, dtype=torch.float64)
    s = torch.where(torch.rand(s.shape, generator=g) < 0.5, -s, s)
    s[:f // BLOCK] *= torch.exp2(torch.tensor([float(cg - e) for e in t], dtype=torch.float64))
    s[f // BLOCK:] *= torch.exp2(torch.tensor([float(cu - e) for e in t], dtype=torch.float64))
    s = s.float()
    assert bool(torch.isfinite(s).all())
    return a, L.Weight8(small_codes(2 * f, dim, 3, size), s.to(DEV), dim)


SCALES = {   # powers of the rows' four blocks, of the gate's and of the up projection's scales beside them, size of the codes
    "signs": ([0, 3, -2, 1], -4, 0, 1.0),
    "up_subnormal": ([100, 119, 90, 110], -4, -25, 1.0),
    "gate_subnormal": ([119, 118, 117, 119], -9, 40, 1.0),
    "both_subnormal": ([119, 119, 118, 119], -12, -20, 1.0),
    "up_large": ([-100, -90, -95, -100], -4, 26, 1.0),
    "gate_large": ([-100, -99, -100, -98], 24, 2, 2.0 ** -5),
    "from_block_to_block": ([-100, 119, 0, -60], -4, 5, 1.0),
}


@pytest.mark.parametrize("rows", FORMS)
@pytest.mark.parametrize("kind", list(SCALES))
@pytest.mark.parametrize("dim", [512, 460])
def test_gated_with_float_scales(rows, kind, dim):
    """Scales of both signs, subnormal, below 2^-118 and above 2^118 ones, gate and up far apart: every value that is not lost to its block's scale."""
    L = lib()
    a, w = float_scaled(rows, dim, *SCALES[kind])
    want, worst, _ = gate_and_up(a, w)
    got = L.gated(a, w)
    check_rows(got, want, worst)
    v = got.read(F32).double()
    assert float((v - want).norm() / want.norm()) < 0.04        # (2.65 % is what codes round)
    assert float((v == 0).double().mean()) < (0.7 if kind == "gate_large" else 0.05)   # (there, gates far below 0 have a silu of 0)
    assert torch.equal(L.gated(a, w).codes, got.codes)


@pytest.mark.parametrize("rows", FORMS)
def test_gated_with_float_scales_that_are_zero_in_some_blocks(rows):
    L = lib()
    a, w = float_scaled(rows, 512, [0, 20, -3, 1], -4, 3)
    w.scale[:16, 1], w.scale[16:, 2] = 0, 0                     # of the gate, of the up projection
    w.scale[5], w.scale[16 + 9] = 0, 0                          # columns of nothing
    want, worst, _ = gate_and_up(a, w)
    got = L.gated(a, w)
    check_rows(got, want, worst)
    zero = (want == 0).reshape(rows, 16, BLOCK).all(-1)
    assert torch.equal(zero, torch.tensor([i in (5, 9) for i in range(16)], device=DEV).expand(rows, 16))


@pytest.mark.parametrize("rows", FORMS)
def test_gated_with_the_smallest_codes_at_the_smallest_scales(rows):
    """Codes of 2^-9 times scales of 2^-118, 2^-126 and less: no product of theirs is lost to the operands' type."""
    L = lib()
    for power in (-118, -119, -126, -140):
        a = L.Rows8(torch.full((rows, 128), 1, dtype=torch.uint8, device=DEV), torch.full((rows, 4), 246, dtype=torch.uint8, device=DEV), 128)
        codes = torch.full((4096, 128), 1, dtype=torch.uint8, device=DEV)
        codes[:, 64:] = 0
        codes[:2048, 3] = 9                                     # (a normal code: 2^-9 * 9)
        s = torch.tensor([[1.5 * 2.0 ** power]] * 16 + [[2.0 ** power]] * 16, dtype=torch.float64).float().to(DEV)
        w = L.Weight8(codes, s, 128)
        want, worst, _ = gate_and_up(a, w)
        got = L.gated(a, w)
        check_rows(got, want, worst)
        assert bool((got.read(F32) > 0).all())


@pytest.mark.parametrize("rows", FORMS)
@pytest.mark.parametrize("power", [118, 119, 123, 127])
def test_gated_of_the_largest_values_times_nothing(rows, power):
    """A block whose rows are as large as they can be and whose weights are codes of 0 with a large scale adds nothing, before and behind one that counts."""
    L = lib()
    a, w = float_scaled(rows, 384, [119, 0, 119], -4, 0)
    for b in (0, 2):
        w.codes[:, b * BLOCK:(b + 1) * BLOCK] = 0
        w.scale[:, b] = torch.where(torch.arange(32, device=DEV) % 3 == 0, -1.9, 1.9) * 2.0 ** power
    a.codes[:, :BLOCK], a.codes[:, 2 * BLOCK:] = 126, 254       # +-448
    want, worst, _ = gate_and_up(a, w)
    got = L.gated(a, w)
    check_rows(got, want, worst)
    assert bool((got.read(F32) != 0).double().mean() > 0.95)
    for dtype in (BF, F32):
        check_product(L.linear(a, w, dtype), a, w)


@pytest.mark.parametrize("rows", [6, 70, 300, 700, 1500, 4000])
def test_gated_of_large_values_zeros_and_nan(rows):
    """Gates far out on either side, a row of zeros, NaN in one row and in one column, within what exact products leave."""
    L = lib()
    f = 256 if rows < 512 else 2048
    x = random_rows(rows, 256, 3, F32, spread=0.0)
    x[0] *= 1e4
    x[1] = 0
    a, w = L.quantize_rows(x), L.Weight8.quantize(random_rows(2 * f, 256, 4, F32, spread=0.0))
    a.codes[2, 17], w.codes[f + 100, 5] = 127, 127
    want, worst, _ = gate_and_up(a, w)
    assert bool(torch.isnan(want[2]).all()) and bool(torch.isnan(want[:, 100]).all()) and int(torch.isnan(want).sum()) == f + rows - 1
    check_rows(L.gated(a, w), want, worst)


# ------------------------------------------------------------------------------------------------------------ scales that are no numbers
@pytest.mark.parametrize("rows", FORMS)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_gated_with_a_scale_that_is_no_number(rows, bad):
    """It shows in every value of its 128 columns, in any block of the sum and in the gate or the up projection, and nowhere else."""
    L = lib()
    a, w = float_scaled(rows, 512, [0, 3, -2, 1], -4, 0)
    at = {1: 0, 4: 2, 7: 3}                                     # columns' block: block of the sum
    for c, b in at.items():
        w.scale[c + 16 * (c == 4), b] = bad
    got = L.gated(a, w).read(F32)
    nan = torch.isnan(got).reshape(rows, 16, BLOCK)
    want = torch.tensor([c in at for c in range(16)], device=DEV)[None, :, None].expand_as(nan)
    assert torch.equal(nan, want)


@pytest.mark.parametrize("rows,n_out", [(8, 512), (100, 512), (300, 512), (2100, 512), (1500, 1600), (5000, 4096)])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_linear_with_a_scale_that_is_no_number(rows, n_out, bad, dtype):
    L = lib()
    a, w = random_rows8(rows, 512, rows), random_weight8(n_out, 512, 3, F32)
    fine = L.linear(a, w, dtype)
    check_product(fine, a, w)
    w.scale[1, 0], w.scale[3, 3] = bad, bad
    got = L.linear(a, w, dtype)
    odd = torch.zeros(n_out, dtype=torch.bool, device=DEV)
    odd[128:256], odd[384:512] = True, True
    assert not bool(torch.isfinite(got[:, odd]).any()) and torch.equal(got[:, ~odd], fine[:, ~odd])


# ------------------------------------------------------------------------------------------------------------ sums that cancel
@pytest.mark.parametrize("rows,n_out", [(5, 40), (60, 200), (300, 300), (1500, 1600), (2100, 2100)])
@pytest.mark.parametrize("scale", [torch.uint8, F32])
def test_sums_that_cancel(rows, n_out, scale):
    """Two products of 448 * 448 that cancel beside one of 20, in one group of eight columns and in different ones, and in random places: fp32 results are
    the sums, bf16 ones within 7 * 2^-13 of the magnitudes."""
    L = lib()
    a, w = random_rows8(rows, 256, 1), random_weight8(n_out, 256, 2, scale)
    values = torch.zeros((2, 256), device=DEV)
    values[:, 0], values[0, 1], values[1, 1], values[0, 2], values[1, 2] = 448.0, 448.0, -448.0, 20.0, 1.0
    spread = torch.zeros((2, 256), device=DEV)
    spread[:, 0], spread[0, 131], spread[1, 131], spread[0, 70], spread[1, 70] = 448.0, 448.0, -448.0, 20.0, 1.0
    for v in (values, spread):
        c = v.to(torch.float8_e4m3fn).view(torch.uint8)
        a.codes.copy_(c[:1].expand(rows, 256)), w.codes.copy_(c[1:].expand(n_out, 256))
        a.scale.fill_(127)
        w.scale.fill_(1 if scale == F32 else 127)
        assert bool((L.linear(a, w, F32) == 20.0).all())
        got = L.linear(a, w, BF).double()
        y, mag, err = product(a, w)
        assert bool(((got - y).abs() <= err[BF] * (1 + HALF[BF]) + HALF[BF] * y.abs()).all())
    # every row's other half is its first with the other sign, but for one product of each
    g = torch.Generator(device=DEV).manual_seed(9)
    c = torch.randint(1, 127, (rows, 128), generator=g, device=DEV).to(torch.uint8)
    a.codes.copy_(torch.cat([c, c], 1))
    c = torch.randint(1, 127, (n_out, 128), generator=g, device=DEV).to(torch.uint8)
    w.codes.copy_(torch.cat([c, c | 128], 1))
    w.codes[:, 200] = 0
    for dtype in (BF, F32):
        got = L.linear(a, w, dtype).double()
        y, mag, err = product(a, w)
        assert bool(((got - y).abs() <= err[dtype] * (1 + HALF[dtype]) + HALF[dtype] * y.abs()).all())


# ------------------------------------------------------------------------------------------------------------ weights of small magnitudes
@pytest.mark.parametrize("power", [-60, -98, -101, -112, -117, -120, -126, -127, -130, -140, -149])
@pytest.mark.parametrize("scale", [torch.uint8, F32])
def test_weights_of_small_magnitudes(power, scale):
    """A block's scale is its largest magnitude / 448, but no smaller than 2^-126, or the least power of two from 2^-100 on; codes are the nearest of the values over it."""
    g = torch.Generator().manual_seed(power + 200)
    w = torch.rand((256, 200), generator=g, dtype=torch.float64) * 2 - 1
    w[3, 5], w[200, 199] = 1.0, -1.75
    w = (w * 2.0 ** power).float()
    w8 = lib().Weight8.quantize(w.to(DEV), scale)
    w = w.double()
    top = torch.nn.functional.pad(w.abs(), (0, 56)).reshape(2, BLOCK, 2, BLOCK).amax((1, 3))
    got = w8.scale.cpu().double() if scale == F32 else torch.exp2(w8.scale.cpu().double() - 127)
    if scale == F32:
        want = torch.where(top > 0, (top / 448).clamp(min=2.0 ** -126), torch.ones_like(top))
        assert bool(((got - want).abs() <= 2 * U * want).all())   # (one division)
    else:
        assert torch.equal(got, torch.exp2(exponent(top)))
    v = weight_values(w8.codes.cpu(), w8.scale.cpu(), 200)
    each = got.repeat_interleave(BLOCK, 0).repeat_interleave(BLOCK, 1)[:, :200]
    step = torch.exp2(torch.floor(torch.log2((w.abs() / each).clamp(min=2.0 ** -6))) - 3) * each
    assert bool(((v - w).abs() <= step / 2 * (1 + 4 * U) + 2 * U * w.abs()).all())


# ------------------------------------------------------------------------------------------------------------ one tensor for all
@pytest.mark.parametrize("rows,dim", [(3, 200), (700, 1000), (2000, 1024), (40, 4096), (600, 8192), (2, 20000)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_norm_rows_of_a_tensor_added_to_itself(rows, dim, dtype):
    """x, the residual and the place of their sum are the same tensor."""
    x = random_rows(rows, dim, rows + dim, dtype)
    h = 2 * x.double()
    eps = 2.0 ** -16
    r, total = lib().norm_rows(x, None, eps, residual=x, out=x)
    assert total is x and torch.equal(x.double(), h)   # (twice a value is exact)
    y = h / torch.sqrt(h.square().mean(-1, keepdim=True) + eps)
    check_rows(r, y, (dim + 60) * 2.0 ** -53 * y.abs() + 2.0 ** -149)
