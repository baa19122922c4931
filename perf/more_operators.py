"""A decoder's projections in 8 bits, as calls that can be timed and compared.

A layer on them adds the last projection to the residual stream, normalises and rounds the sum to 8 bits (`norm_rows`), and
multiplies such rows with weights that are held in 8 bits as well (`linear`; in a feed-forward block `gated`, the gate and up
projections with the SwiGLU between them, whose rows are rounded to 8 bits again, and `linear` for down).  Codes are e4m3.  Rows have a power of two
for each 128 columns, the smallest 2^e with 448 * 2^e >= the largest magnitude of the block; weights have one scale for each
block of 128 by 128, a power of two as well or any number of 32 bits.  Rows of codes are padded with zeros to whole blocks.

With `own` false the operators run in plain torch, 32 bits, rounded once at the end.  Rows in 8 bits that a call returns are read
back as the values that they stand for, which bf16 holds exactly.
"""
import math
from types import SimpleNamespace

import torch

own = False
DEV = "cuda:0"
BLOCK, TOP, EPS = 128, 448.0, 1e-6
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # the norm in front of a projection while one sequence decodes: the smallest call
        dict(name="norm_step_1", op="norm", rows=1, dim=1024, x="bf16", res="fp32"),
        # one round of 16 regions: the residual stream in 32 bits
        dict(name="norm_region_1856", op="norm", rows=1856, dim=1024, x="bf16", res="fp32"),
        # four pages of 8193 rows, a residual stream in 16 bits
        dict(name="norm_page_32772", op="norm", rows=32772, dim=1024, x="bf16", res="bf16"),
        # the QKV projection while one sequence decodes
        dict(name="linear_step_1", op="linear", rows=1, dim=1024, n_out=1536, scale="pow2", out="bf16"),
        # the down projection while 64 sequences decode
        dict(name="linear_step_64", op="linear", rows=64, dim=4096, n_out=1024, scale="pow2", out="bf16"),
        # the LM head over 64 rows, logits in 32 bits: weights read once
        dict(name="linear_head_64", op="linear", rows=64, dim=1024, n_out=32768, scale="pow2", out="fp32"),
        # the down projection of one round of 16 regions
        dict(name="linear_region_1856", op="linear", rows=1856, dim=4096, n_out=1024, scale="pow2", out="bf16"),
        # odd sizes everywhere, weights that came with scales of their own
        dict(name="linear_odd_777", op="linear", rows=777, dim=1000, n_out=1537, scale="fp32", out="fp32"),
        # a large square product: the largest call
        dict(name="linear_square_8192", op="linear", rows=8192, dim=8192, n_out=8192, scale="pow2", out="bf16"),
        # a feed-forward block while 16 sequences decode
        dict(name="ffn_step_16", op="ffn", rows=16, dim=1024, d_ffn=4096, scale="pow2", out="bf16"),
        # the same for one round of 16 regions
        dict(name="ffn_region_1856", op="ffn", rows=1856, dim=1024, d_ffn=4096, scale="pow2", out="bf16"),
        # and for four pages of 8193 rows, weights that came with scales of their own
        dict(name="ffn_page_32772", op="ffn", rows=32772, dim=1024, d_ffn=4096, scale="fp32", out="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "linear", "linear", "linear", "linear", "ffn", "ffn"])
    if op == "norm":
        dim = _log(rng, 16, 16384)
        return dict(op="norm", rows=_log(rng, 1, min(32768, (1 << 25) // dim)), dim=dim, x=rng.choice(["bf16", "bf16", "fp32"]),
                    res=rng.choice(["fp32", "fp32", "bf16"]))
    dim, scale = _log(rng, 32, 8192), rng.choice(["pow2", "pow2", "fp32"])
    if op == "linear":
        n_out = _log(rng, 8, 32768)
        most = min(32768, (1 << 27) // n_out, (1 << 37) // (n_out * dim))
        return dict(op="linear", rows=_log(rng, 1, max(2, most)), dim=dim, n_out=n_out, scale=scale, out=rng.choice(["bf16", "bf16", "fp32"]))
    d_ffn = BLOCK * _log(rng, 1, 96)
    most = min(32768, (1 << 27) // d_ffn, (1 << 36) // (d_ffn * dim))
    return dict(op="ffn", rows=_log(rng, 1, max(2, most)), dim=dim, d_ffn=d_ffn, scale=scale, out="bf16")


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def work(case):
    rows, dim = case["rows"], case["dim"]
    size = {"bf16": 2, "fp32": 4}
    held = lambda n: rows * (n + _blocks(n))   # noqa: E731  codes and scales
    if case["op"] == "norm":   # x and the sum's old part in, the sum, the codes and scales and the values read back out
        return {"bytes": rows * dim * (size[case["x"]] + 2 * size[case["res"]] + 2) + held(dim) + 4 * dim, "flops": 8 * rows * dim}
    byte = 1 if case["scale"] == "pow2" else 4
    if case["op"] == "linear":
        held_w, products = [(case["n_out"], dim)], rows * dim * case["n_out"]
    else:   # (the rows between the products need not leave the chip)
        held_w, products = [(2 * case["d_ffn"], dim), (dim, case["d_ffn"])], 3 * rows * dim * case["d_ffn"]
    read = held(dim) + sum(n * k + _blocks(n) * _blocks(k) * byte for n, k in held_w)
    return {"bytes": read + rows * held_w[-1][0] * size[case["out"]], "flops": 2 * products}


# ---------------------------------------------------------------------------------------------------- plain operators
def _two_to(e):
    """2^e in 32 bits for whole e in -126 .. 127, by its bits."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _round_rows(y):
    """e4m3 codes of rows (padded to whole blocks) and the exponents of their blocks, -100 .. 119 plus 127 as bytes."""
    n, dim = y.shape
    y = torch.nn.functional.pad(y, (0, -dim % BLOCK)).reshape(n, -1, BLOCK)
    top = y.abs().amax(-1)
    m, x = torch.frexp(top)                      # top = m * 2^x, m in [0.5, 1); 448 = 0.875 * 2^9
    e = torch.where(m <= 0.875, x - 9, x - 8).clamp(-100, 119)
    e = torch.where(top > 0, e, torch.zeros_like(e))
    codes = (y * _two_to(-e)[..., None]).to(torch.float8_e4m3fn)
    scale = torch.nn.functional.pad(e + 127, (0, -e.shape[1] % 4)).to(torch.uint8)
    return codes.reshape(n, -1).view(torch.uint8), scale


def _row_values(codes, scale, dim):
    """What rows of codes stand for, in 32 bits."""
    n = codes.shape[0]
    y = codes.view(torch.float8_e4m3fn).float().reshape(n, -1, BLOCK)
    s = _two_to(scale[:, :y.shape[1]].int() - 127)
    return (y * s[..., None]).reshape(n, -1)[:, :dim]


def _weight_values(codes, scale, dim):
    n = codes.shape[0]
    s = _two_to(scale.int() - 127) if scale.dtype == torch.uint8 else scale
    s = s.repeat_interleave(BLOCK, 0)[:n].repeat_interleave(BLOCK, 1)
    return (codes.view(torch.float8_e4m3fn).float() * s)[:, :dim]


def _plain(s):
    if s.op == "norm":
        h = s.x.float() + s.res.float()
        y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * s.gain
        return {"values": _row_values(*_round_rows(y), s.dim).to(torch.bfloat16), "sum": h.to(s.res.dtype)}
    a, w = _row_values(*s.a, s.dim), _weight_values(*s.w, s.dim)
    if s.op == "linear":
        return torch.matmul(a, w.T).to(s.out)
    g, u = torch.matmul(a, w[:s.d_ffn].T), torch.matmul(a, w[s.d_ffn:].T)
    y = _row_values(*_round_rows(g / (1.0 + torch.exp(-g)) * u), s.d_ffn)
    return torch.matmul(y, _weight_values(*s.down, s.d_ffn).T).to(s.out)


# ---------------------------------------------------------------------------------------------------- inputs
def _activations(g, rows, dim):
    """Rows whose channels differ in size, a few of them much larger than the others, as those of trained decoders are."""
    gain = torch.exp(0.5 * torch.randn((dim,), generator=g, device=DEV))
    gain[torch.randint(dim, (1 + dim // 256,), generator=g, device=DEV)] *= 12.0
    return torch.randn((rows, dim), generator=g, device=DEV) * gain


def _norm_inputs(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rows, dim = case["rows"], case["dim"]
    x = (0.3 * torch.randn((rows, dim), generator=g, device=DEV)).to(DTYPES[case["x"]])
    res = _activations(g, rows, dim).to(DTYPES[case["res"]])
    return x, res, 1.0 + 0.1 * torch.randn((dim,), generator=g, device=DEV)


def _weights(g, n_out, dim, kind):
    """Codes and scales of a weight matrix whose rows differ in size."""
    w = torch.randn((n_out, dim), generator=g, device=DEV) * (torch.exp(0.3 * torch.randn((n_out, 1), generator=g, device=DEV)) / math.sqrt(dim))
    w = torch.nn.functional.pad(w, (0, -dim % BLOCK, 0, -n_out % BLOCK)).reshape(_blocks(n_out), BLOCK, _blocks(dim), BLOCK)
    top = w.abs().amax((1, 3))
    if kind == "pow2":
        m, x = torch.frexp(top)
        e = torch.where(m <= 0.875, x - 9, x - 8).clamp(-100, 119)
        scale, s = (e + 127).to(torch.uint8), _two_to(e)
    else:
        scale = s = top / TOP
    codes = (w / s[:, None, :, None]).clamp(-TOP, TOP).to(torch.float8_e4m3fn)
    return codes.reshape(_blocks(n_out) * BLOCK, -1)[:n_out].view(torch.uint8), scale


def _product_inputs(case, seed):
    """Codes and scales of the rows and of the weights (a feed-forward block's: gate and up, then down)."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    dim = case["dim"]
    x = _activations(g, case["rows"], dim)
    a = _round_rows(x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS))
    if case["op"] == "linear":
        return a, _weights(g, case["n_out"], dim, case["scale"]), None
    return a, _weights(g, 2 * case["d_ffn"], dim, case["scale"]), _weights(g, dim, case["d_ffn"], case["scale"])


def prepare(case, seed):
    s = SimpleNamespace(op=case["op"], dim=case["dim"])
    if s.op == "norm":
        s.x, s.res, s.gain = _norm_inputs(case, seed)
    else:
        s.a, s.w, s.down = _product_inputs(case, seed)
        s.d_ffn, s.out = case.get("d_ffn"), DTYPES[case["out"]]
    if own:
        from paper_2602_12957_amd import linear8
        s.lib = linear8
        if s.op != "norm":
            s.rows8, s.weight8 = linear8.Rows8(*s.a, s.dim), linear8.Weight8(*s.w, s.dim)
        if s.op == "ffn":
            s.down8 = linear8.Weight8(*s.down, s.d_ffn)
    return s


def run(s):
    if not own:
        return _plain(s)
    if s.op == "norm":
        rows8, total = s.lib.norm_rows(s.x, s.gain, EPS, residual=s.res)
        return {"values": rows8.read(), "sum": total}
    if s.op == "linear":
        return s.lib.linear(s.rows8, s.weight8, s.out)
    return s.lib.linear(s.lib.gated(s.rows8, s.weight8), s.down8, s.out)


# ---------------------------------------------------------------------------------------------------- in 64 bits
def _nearest(y):
    """The values that rows in 8 bits hold of y (64 bits): nearest multiples of the step that e4m3 has at their place."""
    out = torch.empty_like(y)
    for a in range(0, y.shape[1], BLOCK):
        part = y[:, a:a + BLOCK]
        top = part.abs().amax(1, keepdim=True)
        e = torch.ceil(torch.log2(top / TOP))
        e = torch.where(TOP * torch.exp2(e) < top, e + 1, torch.where(TOP * torch.exp2(e - 1) >= top, e - 1, e))
        s = torch.exp2(torch.where(top > 0, e.clamp(-100, 119), torch.zeros_like(e)))
        v = part / s
        step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
        out[:, a:a + BLOCK] = torch.round(v / step) * step * s
    return out


def _held_weights(codes, scale, dim):
    s = torch.exp2(scale.double() - 127) if scale.dtype == torch.uint8 else scale.double()
    of = torch.arange(codes.shape[0], device=DEV) // BLOCK
    return codes.view(torch.float8_e4m3fn)[:, :dim].double() * s[of][:, torch.arange(dim, device=DEV) // BLOCK]


def exact(case, seed):
    if case["op"] == "norm":
        x, res, gain = _norm_inputs(case, seed)
        h = x.double() + res.double()
        return {"values": _nearest(h / torch.sqrt(h.square().mean(-1, keepdim=True) + EPS) * gain.double()), "sum": h}
    a, w, down = _product_inputs(case, seed)
    w, dim = _held_weights(*w, case["dim"]), case["dim"]
    parts = []
    for r in range(0, case["rows"], 4096):
        y = (a[0][r:r + 4096].view(torch.float8_e4m3fn).double() * torch.exp2(a[1][r:r + 4096].double() - 127).repeat_interleave(BLOCK, 1)[:, :a[0].shape[1]])[:, :dim] @ w.T
        if case["op"] == "ffn":
            gate, up = y.split(case["d_ffn"], 1)
            y = _nearest(gate * torch.sigmoid(gate) * up) @ _held_weights(*down, case["d_ffn"]).T
        parts.append(y)
    return torch.cat(parts)
