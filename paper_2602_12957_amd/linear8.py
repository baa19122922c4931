"""Projections in 8 bits: rows and weights held as e4m3 codes with a scale for each block of 128, and the calls on them
(include/hsd.h: hsd_quant_rows, hsd_quant_norm_rows, hsd_quant_weights, hsd_quant_linear, hsd_quant_gated).

Every call enqueues on torch's current stream of its tensors' device and returns; nothing waits; there is no gradient.  A decoder
layer's feed-forward block on them, `res` being the residual stream and `delta` the attention's projection:

    gate_up, down = Weight8.quantize(w_gate_up), Weight8.quantize(w_down)      # once, [2 * d_ffn, d] (gate, then up) and [d, d_ffn]
    a, res = norm_rows(delta, ffn_norm, eps, residual=res, out=res)            # res + delta, in place, and its norm in 8 bits
    delta = linear(gated(a, gate_up), down)
"""
from __future__ import annotations

from typing import Optional, Tuple

import torch

from . import binding as B

_TYPES = {torch.bfloat16: B.HSD_BF16, torch.float32: B.HSD_FP32}
_BLOCK = B.HSD_QUANT_BLOCK
_CODES, _BYTES = (torch.uint8, torch.float8_e4m3fn), (torch.uint8, torch.float8_e8m0fnu)


def _matrix(name: str, t: torch.Tensor, index: int = -1, shape=None) -> int:
    """A [rows, columns] tensor on a GPU whose rows may lie apart; returns the distance of its rows in elements."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or (index >= 0 and t.get_device() != index):
        raise ValueError(f"{name} must be a tensor on {'a GPU' if index < 0 else f'cuda:{index}'}; there is no CPU fallback")
    if t.dtype not in _TYPES:
        raise ValueError(f"{name}: bfloat16 or float32, got {t.dtype}")
    if t.dim() != 2 or t.shape[1] < 1 or (shape is not None and t.shape != shape):
        raise ValueError(f"{name} must be {'[rows, columns]' if shape is None else list(shape)}, got {tuple(t.shape)}")
    n, m = t.shape
    if t.is_contiguous():
        return m
    s = t.stride()
    if (m > 1 and s[1] != 1) or (n > 1 and s[0] < m):
        raise ValueError(f"{name}: a row's values must lie one after the other and rows must not overlap")
    return s[0] if n > 1 else m


def _held(name: str, t: torch.Tensor, rows: int, least: int, step: int, index: int, types) -> int:
    """A tensor of codes or scales, [rows, at least `least`]; returns the distance of its rows."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype not in types or (index >= 0 and t.get_device() != index):
        raise ValueError(f"{name} must be a {' or '.join(str(x) for x in types)} tensor on {'a GPU' if index < 0 else f'cuda:{index}'}")
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] < least:
        raise ValueError(f"{name} must be [{rows}, {least} or more], got {tuple(t.shape)}")
    s = t.stride() if rows > 1 else (-(-t.shape[1] // step) * step, t.stride(1))
    if (t.shape[1] > 1 and s[1] != 1) or s[0] < t.shape[1] or s[0] % step:
        raise ValueError(f"{name}: rows must lie one after the other, without overlap, a multiple of {step} apart")
    return s[0]


class Rows8:
    """Rows of `dim` values in 8 bits.  codes: uint8 (or float8_e4m3fn) [rows, 128 * ceil(dim / 128)], zeros behind dim; scale: uint8 (or
    float8_e8m0fnu) [rows, ceil(dim / 128) rounded up to a multiple of 4]; value = code * 2^(scale - 127), bytes 27 .. 246 (others have no meaning)."""
    __slots__ = ("_codes", "_scale", "_room", "dim", "rows", "index", "device", "c")

    def __init__(self, codes: torch.Tensor, scale: torch.Tensor, dim: int):
        if dim < 1 or not isinstance(codes, torch.Tensor) or codes.dim() != 2:
            raise ValueError("rows in 8 bits: dim must be positive and codes [rows, 128 * ceil(dim / 128)]")
        n, blocks = codes.shape[0], -(-dim // _BLOCK)
        cs = _held("codes", codes, n, blocks * _BLOCK, 16, -1, _CODES)
        self.index = codes.get_device()
        ss = _held("scale", scale, n, -(-blocks // 4) * 4, 4, self.index, _BYTES)
        if codes.data_ptr() % 16 or scale.data_ptr() % 4:
            raise ValueError("codes must be aligned to 16 bytes and scale to 4")
        self._codes, self._scale, self._room, self.dim, self.rows, self.device = codes, scale, None, dim, n, codes.device
        self.c = B.hsd_rows_quant(codes.data_ptr(), scale.data_ptr(), cs, ss)

    @classmethod
    def empty(cls, rows: int, dim: int, device) -> "Rows8":
        """Room for rows that a call writes: one tensor, the codes and the bytes behind them."""
        if rows < 0 or dim < 1:
            raise ValueError(f"rows must not be negative and dim must be positive, got {rows} and {dim}")
        blocks = (dim + _BLOCK - 1) // _BLOCK
        width, bytes_ = blocks * _BLOCK, (blocks + 3) // 4 * 4
        r = cls.__new__(cls)
        r._codes = r._scale = None
        r._room = room = torch.empty(rows * (width + bytes_), dtype=torch.uint8, device=device)
        r.dim, r.rows, r.index, r.device = dim, rows, room.get_device(), room.device
        if r.index < 0:
            raise ValueError("rows in 8 bits are held on a GPU; there is no CPU fallback")
        p = room.data_ptr()
        r.c = B.hsd_rows_quant(p, p + rows * width, width, bytes_)
        return r

    @property
    def codes(self) -> torch.Tensor:
        if self._codes is None:
            self._codes = self._room[:self.rows * self.c.code_stride].view(self.rows, self.c.code_stride)
        return self._codes

    @property
    def scale(self) -> torch.Tensor:
        if self._scale is None:
            self._scale = self._room[self.rows * self.c.code_stride:].view(self.rows, self.c.scale_stride)
        return self._scale

    def read(self, dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
        """The values, [rows, dim], exact in both types."""
        if dtype not in _TYPES:
            raise ValueError(f"bfloat16 or float32, got {dtype}")
        out = torch.empty((self.rows, self.dim), dtype=dtype, device=self.device)
        with B.on_device(self.index):
            B.hsd_quant_read_rows(B.current_stream(self.index), self.rows, self.dim, self.c, _TYPES[dtype], out.data_ptr(), self.dim)
        return out


class Weight8:
    """A weight matrix [n_out, dim] in 8 bits, blocks of 128 rows by 128 columns.  codes: uint8 (or float8_e4m3fn) [n_out, 128 * ceil(dim / 128)],
    zeros behind dim; scale: [ceil(n_out / 128), ceil(dim / 128)], uint8 or float8_e8m0fnu (value = code * 2^(scale - 127); bytes 27 .. 246, others have no
    meaning) or float32 (value = code * scale; any finite number, others leave no finite result in their columns)."""
    __slots__ = ("codes", "scale", "dim", "n_out", "index", "c")

    def __init__(self, codes: torch.Tensor, scale: torch.Tensor, dim: int):
        if dim < 1 or not isinstance(codes, torch.Tensor) or codes.dim() != 2 or codes.shape[0] < 1:
            raise ValueError("weights in 8 bits: dim must be positive and codes [n_out, 128 * ceil(dim / 128)]")
        n, blocks = codes.shape[0], -(-dim // _BLOCK)
        cs = _held("codes", codes, n, blocks * _BLOCK, 16, -1, _CODES)
        self.index = codes.get_device()
        ss = _held("scale", scale, -(-n // _BLOCK), blocks, 1, self.index, _BYTES + (torch.float32,))
        if codes.data_ptr() % 16:
            raise ValueError("codes must be aligned to 16 bytes")
        self.codes, self.scale, self.dim, self.n_out = codes, scale, dim, n
        self.c = B.hsd_weight_quant(codes.data_ptr(), scale.data_ptr(), cs, ss, B.HSD_SCALE_FP32 if scale.dtype == torch.float32 else B.HSD_SCALE_POW2)

    @classmethod
    def quantize(cls, w: torch.Tensor, scale: torch.dtype = torch.uint8) -> "Weight8":
        """w [n_out, dim], bfloat16 or float32, to 8 bits.  scale: uint8 for powers of two (the faster ones), float32 for the largest magnitude / 448 (2^-126 at least)."""
        stride = _matrix("w", w)
        if w.shape[0] < 1 or scale not in (torch.uint8, torch.float32):
            raise ValueError(f"w must have rows, and scale be uint8 or float32; got {tuple(w.shape)} and {scale}")
        n, dim = w.shape
        blocks = -(-dim // _BLOCK)
        r = cls(torch.empty((n, blocks * _BLOCK), dtype=torch.uint8, device=w.device), torch.empty((-(-n // _BLOCK), blocks), dtype=scale, device=w.device), dim)
        with B.on_device(r.index):
            B.hsd_quant_weights(B.current_stream(r.index), n, dim, _TYPES[w.dtype], w.data_ptr(), stride, r.c)
        return r


def quantize_rows(x: torch.Tensor) -> Rows8:
    """x [rows, dim], bfloat16 or float32, to 8 bits: for each 128 columns of a row the smallest power of two that covers them, values to the
    nearest code.  NaN and infinities become NaN."""
    stride = _matrix("x", x)
    n, dim = x.shape
    out = Rows8.empty(n, dim, x.device)
    with B.on_device(out.index):
        B.hsd_quant_rows(B.current_stream(out.index), n, dim, _TYPES[x.dtype], x.data_ptr(), stride, out.c)
    return out


def norm_rows(x: torch.Tensor, gain: Optional[torch.Tensor] = None, eps: float = 1e-6, residual: Optional[torch.Tensor] = None,
              out: Optional[torch.Tensor] = None) -> Tuple[Rows8, torch.Tensor]:
    """h = x + residual, and h * gain / sqrt(mean(h^2) + eps) in 8 bits.  Returns (rows, h): h in the residual's type, in `out` if given (which may be
    residual itself) or a new tensor; x itself without a residual.  x and residual: [rows, dim], bfloat16 or float32 each; gain:
    float32 [dim].  The norm is of the unrounded h, in 64 bits."""
    xs = _matrix("x", x)
    n, dim = x.shape
    index = x.get_device()
    if gain is not None and (not isinstance(gain, torch.Tensor) or gain.get_device() != index or gain.dtype != torch.float32 or gain.shape != (dim,) or not gain.is_contiguous()):
        raise ValueError(f"gain must be a contiguous float32 tensor [{dim}] on x's device")
    rs = os = 0
    if residual is not None:
        rs = _matrix("residual", residual, index, x.shape)
        if out is None:
            out, os = torch.empty((n, dim), dtype=residual.dtype, device=x.device), dim
        else:
            os = _matrix("out", out, index, x.shape)
            if out.dtype != residual.dtype:
                raise ValueError(f"out must have the residual's type, got {out.dtype}")
    elif out is not None:
        raise ValueError("out takes the sum of x and the residual: there is no residual")
    rows = Rows8.empty(n, dim, x.device)
    with B.on_device(index):
        B.hsd_quant_norm_rows(B.current_stream(index), n, dim, _TYPES[x.dtype], x.data_ptr(), xs, _TYPES[x.dtype if residual is None else residual.dtype],
                              None if residual is None else residual.data_ptr(), rs, None if residual is None else out.data_ptr(), os,
                              None if gain is None else gain.data_ptr(), eps, rows.c)
    return rows, x if residual is None else out


def _pair(rows: Rows8, w: Weight8):
    if not isinstance(rows, Rows8) or not isinstance(w, Weight8):
        raise ValueError("a product in 8 bits takes Rows8 and Weight8 (quantize_rows, norm_rows; Weight8.quantize)")
    if rows.dim != w.dim or rows.index != w.index:
        raise ValueError(f"rows of {rows.dim} values on cuda:{rows.index} and weights of {w.dim} on cuda:{w.index}")


def linear(rows: Rows8, w: Weight8, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """rows * w^T, [rows, n_out] in bfloat16 or float32 (that of `out` if given), sums in 32 bits.  For bfloat16 each eight neighbouring products lose what lies
    13 bits below the largest of them (7 * 2^-13 of the products' magnitudes at most); where large products cancel, take float32."""
    _pair(rows, w)
    if out is None:
        if dtype not in _TYPES:
            raise ValueError(f"bfloat16 or float32, got {dtype}")
        out, stride = torch.empty((rows.rows, w.n_out), dtype=dtype, device=rows.device), w.n_out
    else:
        stride = _matrix("out", out, rows.index, (rows.rows, w.n_out))
    with B.on_device(rows.index):
        B.hsd_quant_linear(B.current_stream(rows.index), rows.rows, w.n_out, rows.dim, rows.c, w.c, _TYPES[out.dtype], out.data_ptr(), stride)
    return out


def gated(rows: Rows8, w: Weight8) -> Rows8:
    """silu(rows * gate^T) * (rows * up^T) in 8 bits, w holding the gate's rows and then the up projection's: [rows, n_out / 2], a multiple of 128."""
    _pair(rows, w)
    d_ffn = w.n_out // 2
    if w.n_out != 2 * d_ffn or d_ffn % _BLOCK:
        raise ValueError(f"gate and up must have a multiple of {_BLOCK} rows each, got {w.n_out} together")
    out = Rows8.empty(rows.rows, d_ffn, rows.device)
    with B.on_device(rows.index):
        B.hsd_quant_gated(B.current_stream(rows.index), rows.rows, d_ffn, rows.dim, rows.c, w.c, out.c)
    return out
