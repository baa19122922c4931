"""Projections in 8 bits on the GPU: rows and weights made, normalised, multiplied, against their definitions in 64 bits."""
import pytest
import torch

from linear8_testlib import (BLOCK, HALF, U, block_tops, check_product, check_rows, e4m3_values, exponent, product, random_rows, random_rows8,
                             random_weight8, row_values, weight_values)

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def lib():
    from paper_2602_12957_amd import linear8
    return linear8


# ------------------------------------------------------------------------------------------------------------ rows
def test_every_bf16_value():
    """Each of the 65536 bf16 patterns in a block that nothing larger than it is in: with itself alone, and beside a value 2^6 larger."""
    x = torch.arange(65536, device=DEV).to(torch.int32).to(torch.int16).view(BF)
    alone = torch.zeros((65536, 3), dtype=BF, device=DEV)
    alone[:, 1] = x
    r = lib().quantize_rows(alone)
    check_rows(r, alone.double(), 0.0)
    for dtype in (BF, F32):
        got = r.read(dtype)
        want = row_values(r.codes, r.scale, 3)
        assert torch.equal(torch.nan_to_num(got.double(), nan=7.0), torch.nan_to_num(want, nan=7.0))
    beside = alone.clone()
    beside[:, 2] = torch.where(torch.isfinite(x.float() * 64), x.float() * 64, torch.zeros_like(x.float())).to(BF)
    check_rows(lib().quantize_rows(beside), beside.double(), 0.0)


def test_scales_at_their_borders():
    """Blocks whose largest value is 448 * 2^e exactly, one step below and one above."""
    v = []
    for e in range(-140, 120):
        for m in (448.0, 448.0 - 2.0 ** -15, 448.0 + 2.0 ** -15):
            v.append(m * 2.0 ** e)
    x = torch.tensor(v, dtype=torch.float64).clamp(max=3e38).float().to(DEV)[:, None] * torch.ones((1, 130), device=DEV)
    r = lib().quantize_rows(x)
    assert torch.equal(r.scale[:, :2].double() - 127, exponent(block_tops(x.double())))
    check_rows(r, x.double(), 0.0)


@pytest.mark.parametrize("rows,dim", [(0, 64), (1, 1), (1, 1024), (2, 7), (3, 127), (5, 128), (4, 129), (70, 1000), (33, 2047), (9, 2049), (3, 8192), (2, 16389), (1, 70001),
                                      (1856, 1024), (4097, 200)])
@pytest.mark.parametrize("xt,rt,gain", [(BF, F32, True), (BF, BF, True), (F32, F32, True), (F32, BF, False), (BF, None, True), (F32, None, False)])
def test_norm_rows(rows, dim, xt, rt, gain):
    x = random_rows(rows, dim, 3 + rows + dim, xt)
    res = None if rt is None else random_rows(rows, dim, 5 + rows + dim, rt, spread=2.0)
    g = 1 + 0.3 * random_rows(1, dim, 9, F32, spread=0.0)[0] if gain else None
    r, total = lib().norm_rows(x, g, 1e-5, residual=res)
    h = x.double() + (0 if res is None else res.double())
    if rt is None:
        assert total is x
    else:
        assert total.dtype == rt and bool(((total.double() - h).abs() <= (HALF[rt] * (1 + U) + U) * h.abs()).all())
    # everything in 64 bits but the value that is rounded to a code (one rounding) and eps, which is a float (half a rounding, of which the
    # root halves the share that it has in the mean)
    y = h / torch.sqrt(h.square().mean(-1, keepdim=True) + 1e-5) * (1 if g is None else g.double())
    check_rows(r, y, 2 * U * y.abs() + 2.0 ** -149)
    assert r.read().shape == (rows, dim)


def test_norm_rows_next_to_a_border():
    """Four million values, some of them within 2^-25 of the border between two codes: each gets the code of its value in 64 bits."""
    x, g = random_rows(4096, 1024, 31, F32), 1 + 0.3 * random_rows(1, 1024, 32, F32, spread=0.0)[0]
    eps = 2.0 ** -16                                # (a float)
    r, _ = lib().norm_rows(x, g, eps)
    h = x.double()
    y = h / torch.sqrt(h.square().mean(-1, keepdim=True) + eps) * g.double()
    # sums of squares of 1024 terms in any order: 1024 * 2^-53 relative at most, here and there, half of it after the root; a few more roundings
    check_rows(r, y, 1100 * 2.0 ** -53 * y.abs() + 2.0 ** -149)


def test_norm_rows_of_more_threads_than_a_launch():
    """Rows of 16 waves each, more of them than a launch of 2^31 threads holds."""
    rows, dim = (1 << 21) + 5, 16400
    if torch.cuda.mem_get_info()[0] < 120 << 30:
        pytest.skip("needs 120 GB")
    L = lib()
    x = torch.ones((rows, dim), dtype=BF, device=DEV)
    at = torch.cat([torch.arange(0, 3), torch.arange((1 << 21) - 3, rows)]).to(DEV)
    x[at] = random_rows(len(at), dim, 33, BF)
    r, small = L.quantize_rows(x), L.quantize_rows(x[at])
    assert torch.equal(r.codes[at], small.codes) and torch.equal(r.scale[at, :129], small.scale[:, :129])
    assert bool((r.scale[3:(1 << 21) - 3, :129] == r.scale[3, 0]).all())


def test_norm_rows_of_unusual_values():
    x = random_rows(12, 300, 1, F32)
    x[1] = 0
    x[2, 128:256] = 0
    x[3] *= 1e-30
    x[4] *= 1e16
    x[5] *= 1e-42
    x[6, 3], x[7, 299], x[8, 130] = float("nan"), float("inf"), float("-inf")
    x[9] *= 1e30                       # squares beyond fp32's range
    x[10, 5] = 1e5 * x[10].abs().max()
    r, _ = lib().norm_rows(x, None, 1e-6)
    v = row_values(r.codes, r.scale, 300)
    assert bool(torch.isnan(v[6]).all())
    for i, at in ((7, 299), (8, 130)):   # inf / inf there, and 0 elsewhere
        assert torch.equal(torch.isnan(v[i]), torch.arange(300, device=DEV) == at) and not bool(torch.nan_to_num(v[i]).any())
    keep = [0, 1, 2, 3, 4, 5, 9, 10, 11]
    h = x[keep].double()
    y = h / torch.sqrt(h.square().mean(-1, keepdim=True) + 1e-6)
    sub = type("R", (), dict(codes=r.codes[keep], scale=r.scale[keep], dim=300, rows=len(keep)))
    check_rows(sub, y, 2 * U * y.abs() + 2.0 ** -149)   # (its value in 32 bits, and eps as a float)
    # a row of zeros without eps is 0 / 0
    r, _ = lib().norm_rows(x[1:2], None, 0.0)
    assert bool(torch.isnan(row_values(r.codes, r.scale, 300)).all())


def test_rows_that_lie_apart():
    """Rows with a stride, from an address that only their elements are aligned to; the sum in place of the residual, which lies apart too."""
    for xt in (BF, F32):
        for rt in (BF, F32):
            big, rbig = random_rows(40, 700, 4, xt), random_rows(40, 901, 6, rt)
            x, res = big[::2, 3:3 + 517], rbig[::2, 1:1 + 517]
            want, total = lib().norm_rows(x.contiguous(), None, 1e-6, residual=res.contiguous())
            before = rbig.clone()
            got, out = lib().norm_rows(x, None, 1e-6, residual=res, out=res)
            assert out is res and torch.equal(got.codes, want.codes) and torch.equal(got.scale[:, :5], want.scale[:, :5])
            before[::2, 1:1 + 517] = total
            assert torch.equal(rbig, before)
            q = lib().quantize_rows(x)
            w = lib().quantize_rows(x.contiguous())
            assert torch.equal(q.codes, w.codes) and torch.equal(q.scale[:, :5], w.scale[:, :5])


# ------------------------------------------------------------------------------------------------------------ weights
@pytest.mark.parametrize("n_out,dim", [(1, 1), (128, 128), (129, 257), (300, 1000), (64, 100), (1000, 384)])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("scale", [torch.uint8, F32])
def test_weights(n_out, dim, dtype, scale):
    w = random_rows(n_out, dim, n_out + dim, dtype) * 0.02
    if n_out > 200:
        w[:128, :128] = 0
    w8 = lib().Weight8.quantize(w, scale)
    top = torch.nn.functional.pad(w.double().abs(), (0, -dim % BLOCK, 0, -n_out % BLOCK)).reshape(-(-n_out // BLOCK), BLOCK, -1, BLOCK).amax((1, 3))
    s = torch.exp2(exponent(top)) if scale == torch.uint8 else torch.where(top > 0, (top / 448).float().double(), torch.ones_like(top))
    got = torch.exp2(w8.scale.double() - 127) if scale == torch.uint8 else w8.scale.double()
    assert bool(((got - s).abs() <= (0 if scale == torch.uint8 else 2 * U) * s).all())
    v = weight_values(w8.codes, w8.scale, dim)
    each = got.repeat_interleave(BLOCK, 0)[:n_out].repeat_interleave(BLOCK, 1)[:, :dim]
    step = torch.exp2(torch.floor(torch.log2((w.double().abs() / each).clamp(min=2.0 ** -6))) - 3) * each
    assert bool(((v - w.double()).abs() <= step / 2 * (1 + 4 * U) + 2 * U * w.double().abs()).all())
    assert not bool((w8.codes[:, dim:] & 127).any())


def test_weights_that_are_no_numbers():
    w = random_rows(130, 140, 1, F32)
    w[3, 5], w[129, 139], w[7, 130] = float("nan"), float("inf"), float("-inf")
    for scale in (torch.uint8, F32):
        w8 = lib().Weight8.quantize(w, scale)
        assert torch.equal(torch.isnan(weight_values(w8.codes, w8.scale, 140)), ~torch.isfinite(w))


# ------------------------------------------------------------------------------------------------------------ products
SIZES = [(1, 1, 1), (1, 16, 128), (1, 1536, 1024), (2, 17, 129), (3, 128, 384), (15, 130, 512), (16, 64, 640), (17, 257, 1000), (31, 100, 100), (32, 32, 2048), (33, 1000, 896),
         (48, 129, 4096), (63, 96, 256), (64, 1024, 4096), (65, 255, 1024), (96, 513, 300), (127, 127, 127), (128, 128, 128), (129, 129, 129), (130, 1, 513),
         (200, 384, 1152), (255, 640, 2176), (256, 256, 256), (257, 257, 257), (300, 1537, 777), (511, 100, 128), (512, 1024, 1024), (777, 1537, 1000), (1000, 900, 4096),
         (1025, 1030, 640), (1856, 1024, 512), (2050, 520, 1920), (4100, 300, 256), (70000, 5, 130),
         (1500, 1600, 512), (2050, 2050, 300), (2500, 4200, 130), (4097, 2600, 257), (8196, 2048, 128), (16390, 1030, 384), (64, 4097, 300), (16, 8192, 257), (17, 8200, 129), (5, 9000, 640)]


@pytest.mark.parametrize("rows,n_out,dim", SIZES)
@pytest.mark.parametrize("scale", [torch.uint8, F32])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_linear(rows, n_out, dim, scale, dtype):
    a, w = random_rows8(rows, dim, rows + dim), random_weight8(n_out, dim, n_out, scale)
    check_product(lib().linear(a, w, dtype), a, w)


@pytest.mark.parametrize("rows,n_out", [(5, 100), (70, 300), (600, 700)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_linear_into_a_larger_tensor(rows, n_out, dtype):
    """Rows of the result lie apart and start at odd elements: nothing beside them changes."""
    a, w = random_rows8(rows, 700, 1), random_weight8(n_out, 700, 2)
    room = torch.full((rows + 3, n_out + 37), 7.0, dtype=dtype, device=DEV)
    out = room[1:1 + rows, 5:5 + n_out]
    assert lib().linear(a, w, out=out) is out
    check_product(out, a, w)
    room[1:1 + rows, 5:5 + n_out] = 7.0
    assert bool((room == 7.0).all())
    assert torch.equal(lib().linear(a, w, dtype), lib().linear(a, w, dtype))


def test_rows_and_weights_that_lie_apart():
    """Codes and scales as parts of larger tensors, whose other places hold NaN codes and the largest bytes."""
    L = lib()
    for rows, n_out, dim in ((7, 200, 300), (90, 333, 640), (700, 300, 1000)):
        a, w = random_rows8(rows, dim, 5), random_weight8(n_out, dim, 6)
        wide = a.codes.shape[1]
        ac = torch.full((rows + 2, wide + 48), 127, dtype=torch.uint8, device=DEV)
        asc = torch.full((rows + 2, a.scale.shape[1] + 8), 255, dtype=torch.uint8, device=DEV)
        wc = torch.full((n_out + 200, wide + 16), 127, dtype=torch.uint8, device=DEV)
        wsc = torch.full((w.scale.shape[0] + 2, w.scale.shape[1] + 3), 255, dtype=torch.uint8, device=DEV)
        ac[1:-1, 16:16 + wide], asc[1:-1, 4:4 + a.scale.shape[1]] = a.codes, a.scale
        asc[1:-1, 4 + wide // BLOCK:] = 255
        wc[:n_out, :wide], wsc[1:-1, 1:1 + w.scale.shape[1]] = w.codes, w.scale
        a2 = L.Rows8(ac[1:-1, 16:16 + wide], asc[1:-1, 4:4 + a.scale.shape[1]], dim)
        w2 = L.Weight8(wc[:n_out, :wide], wsc[1:-1, 1:1 + w.scale.shape[1]], dim)
        for dtype in (BF, F32):
            assert torch.equal(L.linear(a2, w2, dtype), L.linear(a, w, dtype))


@pytest.mark.parametrize("rows,n_out,dim", [(3, 40, 300), (64, 512, 1024), (130, 257, 640), (520, 300, 512)])
def test_nan_stays_in_its_row_and_column(rows, n_out, dim):
    a, w = random_rows8(rows, dim, 5), random_weight8(n_out, dim, 6)
    a.codes[1, 200], w.codes[n_out - 2, dim - 1] = 127, 255
    for dtype in (BF, F32):
        got = torch.isnan(lib().linear(a, w, dtype))
        want = torch.zeros_like(got)
        want[1], want[:, n_out - 2] = True, True
        assert torch.equal(got, want)


@pytest.mark.parametrize("rows", [8, 100, 300, 2100, 5000])
def test_float_scales_that_are_small_or_zero(rows):
    """Scales of 0, subnormal and just normal ones, and large ones, beside each other, with rows' scales that bring their blocks' products together."""
    L = lib()
    a, w = random_rows8(rows, 1024, rows), random_weight8(512, 1024, 3, F32)
    s = torch.tensor([1.0, 0.0, 2.0 ** -149, -3e-42, 1.7e-38, 0.0, 1e25, -1.9], device=DEV)
    w.scale.copy_(torch.stack([s.roll(k) for k in range(4)]))
    a.scale.copy_(torch.randint(112, 125, (1, 8), generator=torch.Generator(device=DEV).manual_seed(5), device=DEV).expand(rows, 8))
    for dtype in (BF, F32):
        check_product(L.linear(a, w, dtype), a, w)
    small = torch.where(s.abs() < 1e-37, s, torch.zeros_like(s))   # only those, against large scales of the rows
    w.scale.copy_(torch.stack([small.roll(k) for k in range(4)]))
    a.scale.fill_(215)
    for dtype in (BF, F32):
        check_product(L.linear(a, w, dtype), a, w)
    w.scale[:2] = 0                                                # gates of 0
    assert not bool((L.gated(a, w).codes & 127).any())


def test_scales_from_end_to_end():
    """Blocks whose powers of two are the smallest and the largest that rows and weights hold: results beyond fp32 are infinite, those
    below vanish, those between are right."""
    L = lib()
    for rows in (4, 80, 300):
        for ea, ew in ((27, 27), (27, 246), (40, 200), (127, 127), (246, 27), (246, 246), (60, 60), (130, 30)):
            a, w = random_rows8(rows, 256, 1), random_weight8(70, 256, 2)
            a.scale.fill_(ea), w.scale.fill_(ew)
            y, mag, err = product(a, w)
            for dtype in (BF, F32):
                got = L.linear(a, w, dtype).double()
                most = (err[dtype] + HALF[dtype] * y.abs()) * 1.01 + 2.0 ** -126 * 256   # (sums below 2^-126 may be held as 0)
                over = y.abs() + most > 3.38e38
                right = bool((((got - y).abs() <= most) | over).all()) and bool((torch.isinf(got) | torch.isnan(got) | ~(y.abs() - most > 3.41e38)).all())
                assert right, (rows, ea, ew, dtype)


# ------------------------------------------------------------------------------------------------------------ gate and up
@pytest.mark.parametrize("rows,d_ffn,dim", [(1, 128, 1), (1, 256, 1024), (5, 128, 128), (16, 384, 1000), (17, 128, 300), (33, 256, 640), (64, 512, 512), (65, 128, 1024), (100, 256, 129),
                                            (128, 128, 256), (129, 384, 384), (200, 128, 4096), (256, 256, 256), (257, 640, 896), (600, 1024, 512), (1856, 256, 1024), (70000, 128, 100), (1100, 2048, 129),
                                            (2100, 2048, 300), (8196, 1024, 128), (4097, 1152, 257)])
@pytest.mark.parametrize("scale", [torch.uint8, F32])
def test_gated(rows, d_ffn, dim, scale):
    L = lib()
    a = L.quantize_rows(random_rows(rows, dim, rows + dim, spread=0.5))
    w = L.Weight8.quantize(random_rows(2 * d_ffn, dim, d_ffn, F32, spread=0.3) / dim ** 0.5, scale)
    got = L.gated(a, w)
    y, _, err = product(a, w)
    e = err[F32]                                  # (products of the codes are exact, whatever the rows are)
    g, u, eg, eu = y[:, :d_ffn], y[:, d_ffn:], e[:, :d_ffn], e[:, d_ffn:]
    want = g * torch.sigmoid(g) * u
    # |silu'| <= 1.1; silu itself and the product round eight times at most, its exponential's argument to |g| 2 roundings
    near = (g * torch.sigmoid(g)).abs()
    most = (1.1 * eg * (u.abs() + eu) + near * eu) * 1.01 + (8 + 2 * g.abs()) * U * want.abs() + 2.0 ** -126
    check_rows(got, want, most)


def test_gated_of_unusual_values():
    """Gates far out on either side, rows of zeros, NaN in one row and in one column (which takes the 128 columns' other values along only as NaN of its own)."""
    L = lib()
    for rows in (6, 70, 300):
        x = random_rows(rows, 256, 3, F32, spread=0.0)
        x[0] *= 1e4
        x[1] = 0
        a = L.quantize_rows(x)
        w = L.Weight8.quantize(random_rows(512, 256, 4, F32, spread=0.0))
        a.codes[2, 17] = 127
        w.codes[256 + 100, 5] = 127
        r = L.gated(a, w)
        v = r.read(F32)
        nan = torch.zeros_like(v, dtype=torch.bool)
        nan[2], nan[:, 100] = True, True
        assert torch.equal(torch.isnan(v), nan)
        y, _, err = product(a, w)
        y, e = torch.nan_to_num(y), torch.nan_to_num(err[BF])
        g, u = y[:, :256], y[:, 256:]
        want = g * torch.sigmoid(g) * u
        most = (1.1 * e[:, :256] * (u.abs() + e[:, 256:]) + (g * torch.sigmoid(g)).abs() * e[:, 256:]) * 1.01 + (8 + 2 * g.abs()) * U * want.abs() + 2.0 ** -126
        check_rows(r, torch.where(nan, torch.full_like(want, float("nan")), want), most)


# ------------------------------------------------------------------------------------------------------------ together
def _layer(L, x, res, gain, gate_up, down):
    a, h = L.norm_rows(x, gain, 1e-6, residual=res)
    u = L.gated(a, gate_up)
    return a, h, u, L.linear(u, down), L.linear(a, gate_up, F32)


@pytest.mark.parametrize("rows", [1, 16, 100, 1000])
def test_feed_forward_block(rows):
    """The residual's addition, norm, gate and up, down: each call on what the one before it gave."""
    L = lib()
    d, f = 384, 512
    x, res = random_rows(rows, d, 1), random_rows(rows, d, 2, F32)
    gain = 1 + 0.1 * random_rows(1, d, 3, F32, spread=0.0)[0]
    gu, dn = L.Weight8.quantize(random_rows(2 * f, d, 4, spread=0.2) / d ** 0.5), L.Weight8.quantize(random_rows(d, f, 5, spread=0.2) / f ** 0.5)
    a, h, u, out, _ = _layer(L, x, res, gain, gu, dn)
    check_product(out, u, dn)
    # the whole against weights and values that nothing rounds: three roundings to 8 bits (2^-4 at most, 2.65 % of the norm each) meet
    hd = x.double() + res.double()
    n = hd / torch.sqrt(hd.square().mean(-1, keepdim=True) + 1e-6) * gain.double()
    wgu, wdn = random_rows(2 * f, d, 4, spread=0.2).double() / d ** 0.5, random_rows(d, f, 5, spread=0.2).double() / f ** 0.5
    g, up = (n @ wgu.T).split(f, 1)
    want = (g * torch.sigmoid(g) * up) @ wdn.T
    assert float((out.double() - want).norm() / want.norm()) < 5 * 2.0 ** -4   # a's and gate_up's in gate and in up, u's, down's: 6 of 2.65 % in quadrature, far below


def test_another_stream_and_replays():
    """The calls on a stream of their own, then captured into a graph and replayed on new inputs, with other work between."""
    L = lib()
    d, f, rows = 256, 256, 70
    gu, dn = L.Weight8.quantize(random_rows(2 * f, d, 4) / 16), L.Weight8.quantize(random_rows(d, f, 5) / 16)
    x, res, gain = random_rows(rows, d, 1), random_rows(rows, d, 2, F32), torch.ones(d, device=DEV)
    want = _layer(L, x, res, gain, gu, dn)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = _layer(L, x, res, gain, gu, dn)
    side.synchronize()
    same = lambda p, q: torch.equal(p.read(F32), q.read(F32)) if isinstance(p, L.Rows8) else torch.equal(p, q)   # noqa: E731
    assert all(same(p, q) for p, q in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = _layer(L, x, res, gain, gu, dn)
    for seed in range(4):
        x.copy_(random_rows(rows, d, 100 + seed)), res.copy_(random_rows(rows, d, 200 + seed, F32))
        graph.replay()
        torch.cuda.synchronize()
        now = _layer(L, x, res, gain, gu, dn)
        torch.cuda.synchronize()
        assert all(same(p, q) for p, q in zip(kept, now))


@pytest.mark.parametrize("rows", [8, 64, 200, 700])
def test_the_same_call_gives_the_same_bits(rows):
    L = lib()
    a, w = random_rows8(rows, 512, rows), random_weight8(640, 512, 3)
    u = L.gated(a, random_weight8(512, 512, 4))
    for _ in range(3):
        assert torch.equal(L.linear(a, w), L.linear(a, w)) and torch.equal(L.linear(a, w, F32), L.linear(a, w, F32))
        assert torch.equal(L.gated(a, random_weight8(512, 512, 4)).codes, u.codes)


def test_two_streams_at_once():
    """The same calls on two streams without a wait between them, each into tensors of its own."""
    L = lib()
    d, f = 256, 512
    gu, dn = L.Weight8.quantize(random_rows(2 * f, d, 4) / 16), L.Weight8.quantize(random_rows(d, f, 5) / 16)
    gain, sides = torch.ones(d, device=DEV), [torch.cuda.Stream(), torch.cuda.Stream()]
    inputs = [(random_rows(rows, d, rows), random_rows(rows, d, 2, F32)) for rows in (16, 300)]
    want = [_layer(L, x, res, gain, gu, dn) for x, res in inputs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(4):
        for k, side in enumerate(sides):
            with torch.cuda.stream(side):
                got[k].append(_layer(L, *inputs[k], gain, gu, dn))
    torch.cuda.synchronize()
    for k in range(2):
        for g in got[k]:
            assert all(torch.equal(p.read(F32), q.read(F32)) if isinstance(p, L.Rows8) else torch.equal(p, q) for p, q in zip(want[k], g))


def test_codes_of_torchs_own_types():
    L = lib()
    a, w = random_rows8(9, 300, 1), random_weight8(200, 300, 2)
    a8 = L.Rows8(a.codes.view(torch.float8_e4m3fn), a.scale.view(torch.float8_e8m0fnu), 300)
    w8 = L.Weight8(w.codes.view(torch.float8_e4m3fn), w.scale.view(torch.float8_e8m0fnu), 300)
    assert torch.equal(L.linear(a8, w8), L.linear(a, w)) and torch.equal(a8.read(F32), a.read(F32))


def test_no_rows():
    L = lib()
    a, w = L.Rows8.empty(0, 300, DEV), random_weight8(256, 300, 1)
    assert L.linear(a, w).shape == (0, 256) and L.gated(a, w).rows == 0 and a.read().shape == (0, 300)
    r, total = L.norm_rows(torch.empty((0, 300), device=DEV), residual=torch.empty((0, 300), device=DEV))
    assert r.rows == 0 and total.shape == (0, 300)
    assert e4m3_values()[126] == 448


# ------------------------------------------------------------------------------------------------------------ refusals
def test_refused_tensors():
    L = lib()
    x, w = random_rows(4, 256, 1), L.Weight8.quantize(random_rows(256, 256, 2))
    a = L.quantize_rows(x)
    for call in (lambda: L.quantize_rows(x.cpu()), lambda: L.quantize_rows(x.half()), lambda: L.quantize_rows(x[0]), lambda: L.quantize_rows(x.t()[:, :2].t().t()),
                 lambda: L.quantize_rows(torch.empty((4, 0), device=DEV)), lambda: L.norm_rows(x, torch.ones(255, device=DEV)), lambda: L.norm_rows(x, torch.ones(256)),
                 lambda: L.norm_rows(x, torch.ones(256, device=DEV, dtype=BF)), lambda: L.norm_rows(x, residual=x[:3]), lambda: L.norm_rows(x, out=x),
                 lambda: L.norm_rows(x, residual=x, out=x.float()), lambda: L.norm_rows(x, residual=x.half()), lambda: L.linear(x, w), lambda: L.linear(a, x),
                 lambda: L.linear(L.quantize_rows(x[:, :128]), w), lambda: L.linear(a, w, torch.float16), lambda: L.linear(a, w, out=torch.empty((4, 255), device=DEV)),
                 lambda: L.linear(a, w, out=torch.empty((256, 4), device=DEV).t()), lambda: L.gated(a, L.Weight8.quantize(random_rows(254, 256, 2))),
                 lambda: L.gated(a, L.Weight8.quantize(random_rows(255, 256, 2))), lambda: L.Weight8.quantize(x, BF), lambda: L.Weight8.quantize(x[:0]),
                 lambda: L.Rows8(a.codes[:, :128], a.scale, 256), lambda: L.Rows8(a.codes, a.scale[:, :3], 256), lambda: L.Rows8(a.codes[:, 1:], a.scale, 128),
                 lambda: L.Rows8(a.codes, a.scale[:3], 256), lambda: L.Rows8(a.codes.float(), a.scale, 256), lambda: L.Rows8(a.codes.cpu(), a.scale, 256),
                 lambda: L.Rows8(a.codes, a.scale, 0), lambda: L.Rows8(a.codes, a.scale.cpu(), 256), lambda: L.Weight8(w.codes, w.scale[:1], 256),
                 lambda: L.Weight8(w.codes, w.scale.to(BF), 256), lambda: L.Weight8(w.codes[:, :100], w.scale, 256), lambda: a.read(torch.float16),
                 lambda: L.Rows8.empty(4, 256, "cpu"), lambda: L.Rows8.empty(4, 0, DEV), lambda: L.Rows8.empty(-1, 4, DEV)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(RuntimeError):
        L.norm_rows(x, eps=float("nan"))
    with pytest.raises(RuntimeError):
        L.norm_rows(x, eps=-1.0)
