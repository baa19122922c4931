"""Projections in 8 bits: what the C entries refuse before they touch a device, and the definitions that the GPU tests go by."""
import ctypes as C

import pytest
import torch

import paper_2602_12957_amd.binding as B
from linear8_testlib import block_tops, e4m3_values, exponent

FAKE = 0x1000   # never dereferenced: every call here is refused, or has no rows


def rows(**kw):
    base = dict(codes=FAKE, scale=FAKE, code_stride=1024, scale_stride=8)
    base.update(kw)
    return B.hsd_rows_quant(*[base[n] for n, _ in B.hsd_rows_quant._fields_])


def weight(**kw):
    base = dict(codes=FAKE, scale=FAKE, code_stride=1024, scale_stride=8, scale_type=B.HSD_SCALE_POW2)
    base.update(kw)
    return B.hsd_weight_quant(*[base[n] for n, _ in B.hsd_weight_quant._fields_])


def call(name, **kw):
    args = {
        "rows": dict(stream=None, n_rows=0, dim=1000, dtype=B.HSD_BF16, x=FAKE, x_stride=1000, out=rows()),
        "norm_rows": dict(stream=None, n_rows=0, dim=1000, dtype=B.HSD_BF16, x=FAKE, x_stride=1000, res_dtype=B.HSD_FP32, residual=FAKE, res_stride=1000, sum=FAKE,
                          sum_stride=1000, gain=FAKE, eps=1e-6, out=rows()),
        "read_rows": dict(stream=None, n_rows=0, dim=1000, rows=rows(), dtype=B.HSD_BF16, out=FAKE, out_stride=1000),
        "weights": dict(stream=None, n_out=0, dim=1000, dtype=B.HSD_BF16, w=FAKE, w_stride=1000, out=weight()),
        "linear": dict(stream=None, n_rows=0, n_out=300, dim=1000, rows=rows(), w=weight(), dtype=B.HSD_BF16, out=FAKE, out_stride=300),
        "gated": dict(stream=None, n_rows=0, d_ffn=256, dim=1000, rows=rows(), w=weight(), out=rows(code_stride=256, scale_stride=4)),
    }[name]
    assert set(kw) <= set(args), kw
    args.update(kw)
    return getattr(B.lib, "hsd_quant_" + name)(*args.values())


def test_no_rows_is_no_work():
    for name in ("rows", "norm_rows", "read_rows", "linear", "gated"):
        assert call(name) == B.HSD_OK


ROWS = [(dict(codes=0), -1), (dict(scale=0), -1), (dict(codes=FAKE + 8), -1), (dict(scale=FAKE + 2), -1), (dict(code_stride=1008), -1), (dict(code_stride=1032), -1),
        (dict(scale_stride=4), -1), (dict(scale_stride=10), -1)]


@pytest.mark.parametrize("kw,code", ROWS)
def test_bad_rows(kw, code):
    bad = rows(**kw)
    assert call("rows", n_rows=4, out=bad) == code
    assert call("norm_rows", n_rows=4, out=bad) == code
    assert call("read_rows", n_rows=4, rows=bad) == code
    assert call("linear", n_rows=4, rows=bad) == code
    assert call("gated", n_rows=4, rows=bad) == code


@pytest.mark.parametrize("kw", [dict(codes=0), dict(scale=0), dict(codes=FAKE + 4), dict(code_stride=1008), dict(code_stride=1025), dict(scale_stride=7), dict(scale_type=2),
                                dict(scale_type=-1), dict(scale_type=B.HSD_SCALE_FP32, scale=FAKE + 1)])
def test_bad_weights(kw):
    bad = weight(**kw)
    assert call("linear", n_rows=4, w=bad) == B.HSD_EINVAL
    assert call("gated", n_rows=4, w=bad) == B.HSD_EINVAL
    assert call("weights", n_out=4, out=bad) == B.HSD_EINVAL


@pytest.mark.parametrize("name,kw,code", [
    ("rows", dict(n_rows=-1), -1), ("rows", dict(dim=0), -1), ("rows", dict(n_rows=1 << 24), -3), ("rows", dict(dim=(1 << 20) + 1), -3), ("rows", dict(n_rows=4, dtype=2), -1),
    ("rows", dict(n_rows=4, x=None), -1), ("rows", dict(n_rows=4, x_stride=999), -1), ("rows", dict(n_rows=4, out=None), -1),
    ("norm_rows", dict(n_rows=4, dtype=-1), -1), ("norm_rows", dict(n_rows=4, res_dtype=2), -1), ("norm_rows", dict(n_rows=4, eps=-1e-9), -1),
    ("norm_rows", dict(n_rows=4, eps=float("nan")), -1), ("norm_rows", dict(n_rows=4, eps=float("inf")), -1), ("norm_rows", dict(n_rows=4, x=None), -1),
    ("norm_rows", dict(n_rows=4, residual=None), -1), ("norm_rows", dict(n_rows=4, res_stride=999), -1), ("norm_rows", dict(n_rows=4, sum_stride=999), -1),
    ("norm_rows", dict(n_rows=4, x_stride=0), -1),
    ("read_rows", dict(n_rows=4, dtype=3), -1), ("read_rows", dict(n_rows=4, out=None), -1), ("read_rows", dict(n_rows=4, out_stride=999), -1),
    ("weights", dict(n_out=0), -1), ("weights", dict(n_out=4, w=None), -1), ("weights", dict(n_out=4, w_stride=999), -1), ("weights", dict(n_out=4, dtype=9), -1),
    ("weights", dict(n_out=1 << 24), -3), ("weights", dict(n_out=4, out=None), -1),
    ("linear", dict(n_rows=4, n_out=0), -1), ("linear", dict(n_rows=4, out=None), -1), ("linear", dict(n_rows=4, out_stride=299), -1), ("linear", dict(n_rows=4, dtype=5), -1),
    ("linear", dict(n_rows=1 << 24), -3), ("linear", dict(n_out=1 << 24), -3), ("linear", dict(n_rows=-4), -1), ("linear", dict(n_rows=4, w=None), -1), ("linear", dict(n_rows=4, rows=None), -1),
    ("gated", dict(d_ffn=0), -1), ("gated", dict(d_ffn=200), -1), ("gated", dict(d_ffn=1 << 21), -3), ("gated", dict(n_rows=4, out=None), -1), ("gated", dict(n_rows=4, w=None), -1),
    ("gated", dict(n_rows=4, out=rows(code_stride=128, scale_stride=4)), -1), ("gated", dict(n_rows=4, rows=None), -1),
])
def test_bad_arguments(name, kw, code):
    assert call(name, **kw) == code


def test_structs_are_the_header_s():
    assert C.sizeof(B.hsd_rows_quant) == 32 and C.sizeof(B.hsd_weight_quant) == 40


def test_tensors_on_the_host_are_refused():
    from paper_2602_12957_amd import linear8 as L
    x = torch.zeros((4, 256))
    for f in (lambda: L.quantize_rows(x), lambda: L.norm_rows(x), lambda: L.Weight8.quantize(x), lambda: L.Rows8(x.byte(), x.byte(), 256), lambda: L.Weight8(x.byte(), x.byte(), 256)):
        with pytest.raises(ValueError):
            f()


def test_the_definition_is_torch_s_e4m3():
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double()
    got = e4m3_values()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


def test_exponents():
    top = torch.tensor([0.0, 448.0, 448.1, 224.0, 1.75, 1.7501, 2.0 ** -140, 3e38], dtype=torch.float64)
    assert exponent(top).tolist() == [0, 0, 1, -1, -8, -7, -100, 119]
    x = torch.tensor([[1.0, -3.0, float("inf"), float("nan")]], dtype=torch.float64)
    assert block_tops(x).tolist() == [[3.0]]
