"""Channel mixing in 8-bit floating point (the fno_fp8_* calls): rounding to
codes with a scale for each block of 128, products of such codes, and a linear
map over channels, forward and backward, built of both.

PyTorch supplies memory and streams only; every step runs in the HIP kernels
behind the entry points.  Codes are torch.float8_e4m3fn or torch.float8_e5m2,
rows of `cols` codes rounded up to 16 (zeros behind them); scales are
torch.float8_e8m0fnu (powers of two) or float32, one for each block of 128
consecutive codes of a row [ceil(cols / 128), rows], or for each 128 x 128 tile
[ceil(cols / 128), ceil(rows / 128)].
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from . import binding as B
from .layer import DTYPE_CODES, _addr, _stream_of, _Workspace

FORMATS = {B.FNO_FP8_E4M3: torch.float8_e4m3fn, B.FNO_FP8_E5M2: torch.float8_e5m2}


class Fp8Codes(NamedTuple):
    """A matrix in codes."""
    codes: torch.Tensor
    scale: torch.Tensor


class Fp8Weights(NamedTuple):
    """Weights [c_out, c_in] in codes by tiles, and their transpose (for the
    backward; None where only the forward runs)."""
    codes: torch.Tensor
    scale: torch.Tensor
    codes_t: Optional[torch.Tensor]
    scale_t: Optional[torch.Tensor]


def _blocks(n: int) -> int:
    return -(-n // B.FNO_FP8_BLOCK)


class _Shape:
    """Shapes and types of a matrix [rows, cols] in codes."""

    def __init__(self, rows: int, cols: int, fmt: int, pow2: bool, tile: bool):
        if fmt not in FORMATS:
            raise ValueError(f"format {fmt}, expected FNO_FP8_E4M3 or FNO_FP8_E5M2")
        self.codes = (rows, B.fno_fp8_pitch(cols))
        self.scale = (_blocks(cols), _blocks(rows) if tile else rows)
        self.type = FORMATS[fmt]
        self.scale_type = torch.float8_e8m0fnu if pow2 else torch.float32
        self.scale_bytes = self.scale[0] * self.scale[1] * (1 if pow2 else 4)

    def check(self, m, name, device):
        """Addresses of a matrix's codes and scales."""
        if len(m) != 2 or m[0] is None or m[1] is None:
            raise ValueError(f"{name}: codes and scale are required")
        return (_addr(m[0], self.codes, self.type, f"{name}.codes", device),
                _addr(m[1], self.scale, self.scale_type, f"{name}.scale", device))

    def new(self, device) -> Fp8Codes:
        return Fp8Codes(torch.empty(self.codes, dtype=self.type, device=device),
                        torch.empty(self.scale, dtype=self.scale_type, device=device))

    def bytes(self):
        """(codes, scales), each rounded up to 256."""
        return ((self.codes[0] * self.codes[1] + 255) // 256 * 256,
                (self.scale_bytes + 255) // 256 * 256)


def _dtype_code(dtype) -> int:
    if dtype not in DTYPE_CODES:
        raise ValueError(f"dtype {dtype}, expected float32, float16 or bfloat16")
    return DTYPE_CODES[dtype]


def _rows_addr(t, name, rows, cols, dtype, device):
    """Address of a tensor [..., cols] of `rows` rows (0 for None)."""
    if t is None:
        return 0
    a = _addr(t, None, dtype, name, device)
    if t.dim() < 1 or t.shape[-1] != cols or t.numel() != rows * cols:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected [..., {cols}] with {rows} rows")
    return a


def _given(stream, name):
    if stream is not None:
        raise ValueError(f"{name} is required where a stream is given")


class Fp8Quantize:
    """Rounds act(x), x [..., cols] with `rows` rows of `dtype`, to codes.

    A block's scale is the least power of two (`pow2_scales`) that brings its
    largest size within the format's, or that size times the fp32 reciprocal of the
    format's.  Blocks are 128 columns of a row, and 128 rows of a column for the transpose;
    with `tile`, 128 x 128 for both.

    An object keeps one workspace, memory of the first call's stream, so its
    calls belong on one stream (or on streams that wait for each other), and it
    outlives the graphs that hold its calls.  Where `stream` is given, outputs are
    the caller's too.
    """

    def __init__(self, rows: int, cols: int, dtype: torch.dtype = torch.float16,
                 format: int = B.FNO_FP8_E4M3, pow2_scales: bool = True, tile: bool = False,
                 activation: int = B.FNO_NORM_ACT_NONE, device: str = "cuda"):
        self.rows, self.cols, self.dtype = int(rows), int(cols), dtype
        self.device = torch.device(device)
        self.desc = B.make_fp8_quantize_desc(self.rows, self.cols, _dtype_code(dtype), format,
                                             B.FNO_SCALE_POW2 if pow2_scales else B.FNO_SCALE_F32,
                                             B.FNO_BLOCKS_TILE if tile else B.FNO_BLOCKS_ROW,
                                             activation)
        self.ws_bytes = B.fno_fp8_quantize_workspace_size(self.desc)  # checks the descriptor
        self.shape = _Shape(self.rows, self.cols, format, pow2_scales, tile)
        self.shape_t = _Shape(self.cols, self.rows, format, pow2_scales, tile)
        self._ws = _Workspace()

    def run(self, x, codes: bool = True, transpose: bool = False, col_sums: bool = False,
            out: Optional[Fp8Codes] = None, out_t: Optional[Fp8Codes] = None, out_sums=None,
            stream: Optional[int] = None):
        """(codes of act(x), codes of its transpose, sums of act(x) over rows
        [cols] float32), None for those not asked for."""
        if x is None:
            raise ValueError("x is required")
        codes, transpose = codes or out is not None, transpose or out_t is not None
        col_sums = col_sums or out_sums is not None
        if not codes and not transpose:
            raise ValueError("neither codes nor those of the transpose are asked for")
        ax, dev = _rows_addr(x, "x", self.rows, self.cols, self.dtype, self.device), x.device
        ac = self.shape.check(out, "out", dev) if out is not None else (0, 0)
        at = self.shape_t.check(out_t, "out_t", dev) if out_t is not None else (0, 0)
        asum = _addr(out_sums, (self.cols,), torch.float32, "out_sums", dev)
        s = _stream_of(dev, stream)
        if codes and out is None:
            _given(stream, "out")
            out = self.shape.new(dev)
            ac = (out[0].data_ptr(), out[1].data_ptr())
        if transpose and out_t is None:
            _given(stream, "out_t")
            out_t = self.shape_t.new(dev)
            at = (out_t[0].data_ptr(), out_t[1].data_ptr())
        if col_sums and out_sums is None:
            _given(stream, "out_sums")
            out_sums = torch.empty(self.cols, dtype=torch.float32, device=dev)
            asum = out_sums.data_ptr()
        ws = self._ws.get(self.ws_bytes, dev, s) if col_sums else (0, 0)
        B.fno_fp8_quantize(self.desc, ax, *ac, *at, asum, *ws, s)
        return out, out_t, out_sums


class Fp8Matmul:
    """out = (A B^T) act'(z) + bias of matrices in codes: A [rows, inner], B [cols,
    inner], out and z [rows, cols] of `dtype`, bias float32 [cols].  tile_a and
    tile_b: scales by tiles.  Workspace and streams as Fp8Quantize."""

    def __init__(self, rows: int, cols: int, inner: int, dtype: torch.dtype = torch.float16,
                 format_a: int = B.FNO_FP8_E4M3, format_b: int = B.FNO_FP8_E4M3,
                 pow2_scales: bool = True, tile_a: bool = False, tile_b: bool = False,
                 activation: int = B.FNO_NORM_ACT_NONE, device: str = "cuda"):
        self.rows, self.cols, self.inner, self.dtype = int(rows), int(cols), int(inner), dtype
        self.activation, self.device = activation, torch.device(device)
        kind = lambda t: B.FNO_BLOCKS_TILE if t else B.FNO_BLOCKS_ROW  # noqa: E731
        self.desc = B.make_fp8_matmul_desc(self.rows, self.cols, self.inner, _dtype_code(dtype),
                                           format_a, format_b,
                                           B.FNO_SCALE_POW2 if pow2_scales else B.FNO_SCALE_F32,
                                           kind(tile_a), kind(tile_b), activation)
        self.ws_bytes = B.fno_fp8_matmul_workspace_size(self.desc)  # checks the descriptor
        self.shape_a = _Shape(self.rows, self.inner, format_a, pow2_scales, tile_a)
        self.shape_b = _Shape(self.cols, self.inner, format_b, pow2_scales, tile_b)
        self._ws = _Workspace()

    def run(self, a: Fp8Codes, b: Fp8Codes, z=None, bias=None, out=None,
            stream: Optional[int] = None):
        """out [rows, cols] (or of the given tensor's shape)."""
        if a is None or b is None:
            raise ValueError("a and b are required")
        if (z is not None) != (self.activation != B.FNO_NORM_ACT_NONE):
            raise ValueError("z belongs to an activation, and an activation needs z")
        aa, dev = self.shape_a.check(a, "a", self.device), a[0].device
        ab = self.shape_b.check(b, "b", dev)
        az = _rows_addr(z, "z", self.rows, self.cols, self.dtype, dev)
        abias = _addr(bias, (self.cols,), torch.float32, "bias", dev)
        ao = _rows_addr(out, "out", self.rows, self.cols, self.dtype, dev)
        s = _stream_of(dev, stream)
        if out is None:
            _given(stream, "out")
            out = torch.empty((self.rows, self.cols), dtype=self.dtype, device=dev)
            ao = out.data_ptr()
        B.fno_fp8_matmul(self.desc, *aa, *ab, az, abias, ao, *self._ws.get(self.ws_bytes, dev, s), s)
        return out


class Fp8Linear:
    """A linear map over channels in 8-bit floating point,

        y = Q(act(x)) Q(W)^T + bias,

    x [..., c_in] with `rows` rows and y [..., c_out] of `dtype` (float32, float16
    or bfloat16), W [c_out, c_in] in codes of e4m3 by 128 x 128 tiles (`pack`),
    bias float32 [c_out].  Q rounds x and, in the backward, the output's gradient
    (to e5m2, or `grad_format`) to codes with one scale for each 128 consecutive
    values along the axis that is summed:

        gx = (Q(g) Q(W)) act'(x),   gW = Q(g^T) Q(act(x)^T)^T,   gb = sum of g over rows.

    For the backward the forward keeps the codes of act(x)^T, and with an
    activation x itself is needed again.  Workspace and streams as Fp8Quantize.
    """

    def __init__(self, rows: int, c_in: int, c_out: int, dtype: torch.dtype = torch.float16,
                 activation: int = B.FNO_NORM_ACT_NONE, pow2_scales: bool = True,
                 grad_format: int = B.FNO_FP8_E5M2, device: str = "cuda"):
        self.rows, self.c_in, self.c_out = int(rows), int(c_in), int(c_out)
        self.dtype, self.activation, self.device = dtype, activation, torch.device(device)
        kw = dict(pow2_scales=pow2_scales, device=device)
        E4M3 = B.FNO_FP8_E4M3
        self.q_w = Fp8Quantize(self.c_out, self.c_in, dtype, E4M3, tile=True, **kw)
        self.q_x = Fp8Quantize(self.rows, self.c_in, dtype, E4M3, activation=activation, **kw)
        self.q_g = Fp8Quantize(self.rows, self.c_out, dtype, grad_format, **kw)
        self.mm_y = Fp8Matmul(self.rows, self.c_out, self.c_in, dtype, tile_b=True, **kw)
        self.mm_x = Fp8Matmul(self.rows, self.c_in, self.c_out, dtype, grad_format, E4M3,
                              tile_b=True, activation=activation, **kw)
        self.mm_w = Fp8Matmul(self.c_out, self.c_in, self.rows, torch.float32, grad_format, E4M3,
                              **kw)
        part = lambda q, t: q.bytes() + (t.bytes() if t else ())  # noqa: E731
        self._fwd_parts = part(self.q_x.shape, None) + (self.mm_y.ws_bytes,)
        self._bwd_parts = part(self.q_g.shape, self.q_g.shape_t) + (
            max(self.q_g.ws_bytes, self.mm_x.ws_bytes, self.mm_w.ws_bytes),)
        self._ws = _Workspace()

    def _places(self, parts, dev, s):
        """Addresses of the parts of the workspace."""
        at, _ = self._ws.get(max(sum(self._fwd_parts), sum(self._bwd_parts)), dev, s)
        places = []
        for n in parts:
            places.append(at)
            at += n
        return places

    def pack(self, w, out: Optional[Fp8Weights] = None, stream: Optional[int] = None) -> Fp8Weights:
        """The weights' codes, both ways, from w [c_out, c_in] of `dtype`.  (fp32 weights
        beside 16-bit rows need not be rounded to those first: Fp8Quantize(c_out, c_in,
        torch.float32, tile=True) forms the same codes from them.)"""
        if out is not None and (out.codes_t is None or out.scale_t is None):
            raise ValueError("out: codes_t and scale_t are written too")
        q, t, _ = self.q_w.run(w, transpose=True, out=None if out is None else Fp8Codes(*out[:2]),
                               out_t=None if out is None else Fp8Codes(*out[2:]), stream=stream)
        return Fp8Weights(*q, *t)

    def fwd(self, x, weights: Fp8Weights, bias=None, y=None, keep: bool = True,
            kept: Optional[Fp8Codes] = None, stream: Optional[int] = None):
        """(y, kept); kept, the codes of act(x)^T for the backward's gW, is None
        unless kept."""
        if x is None or weights is None:
            raise ValueError("x and weights are required")
        ax, dev = _rows_addr(x, "x", self.rows, self.c_in, self.dtype, self.device), x.device
        aw = self.mm_y.shape_b.check(weights[:2], "weights", dev)
        abias = _addr(bias, (self.c_out,), torch.float32, "bias", dev)
        ay = _rows_addr(y, "y", self.rows, self.c_out, self.dtype, dev)
        keep = keep or kept is not None
        ak = self.q_x.shape_t.check(kept, "kept", dev) if kept is not None else (0, 0)
        s = _stream_of(dev, stream)
        if y is None:
            _given(stream, "y")
            y = torch.empty(x.shape[:-1] + (self.c_out,), dtype=self.dtype, device=dev)
            ay = y.data_ptr()
        if keep and kept is None:
            _given(stream, "kept")
            kept = self.q_x.shape_t.new(dev)
            ak = (kept[0].data_ptr(), kept[1].data_ptr())
        q, qs, ws = self._places(self._fwd_parts, dev, s)
        B.fno_fp8_quantize(self.q_x.desc, ax, q, qs, *ak, 0, 0, 0, s)
        B.fno_fp8_matmul(self.mm_y.desc, q, qs, *aw, 0, abias, ay, ws, self.mm_y.ws_bytes, s)
        return y, kept

    def bwd(self, g, weights: Fp8Weights, kept: Optional[Fp8Codes] = None, x=None,
            bias: bool = True, gx=None, gw=None, gb=None, need_x: bool = True,
            stream: Optional[int] = None):
        """(gx, gw, gb), float32 gw [c_out, c_in] and gb [c_out]; gx is None with
        need_x=False, gw without kept, gb with bias=False.  x is the forward's,
        needed for gx with an activation."""
        if g is None:
            raise ValueError("g is required")
        if need_x and weights is None or not need_x and gx is not None:
            raise ValueError("weights belong to gx, which need_x asks for")
        if need_x and weights.codes_t is None:
            raise ValueError("weights: codes_t and scale_t are required for gx")
        if gw is not None and kept is None:
            raise ValueError("kept is required for gw")
        act = self.activation != B.FNO_NORM_ACT_NONE
        if need_x and act and x is None:
            raise ValueError("x is required for gx with an activation")
        if not need_x and kept is None:
            raise ValueError("neither gx nor gw is asked for")
        ag, dev = _rows_addr(g, "g", self.rows, self.c_out, self.dtype, self.device), g.device
        aw = self.mm_x.shape_b.check(weights[2:], "weights", dev) if need_x else (0, 0)
        ak = self.mm_w.shape_b.check(kept, "kept", dev) if kept is not None else (0, 0)
        ax = _rows_addr(x, "x", self.rows, self.c_in, self.dtype, dev) if act else 0
        agx = _rows_addr(gx, "gx", self.rows, self.c_in, self.dtype, dev)
        agw = _addr(gw, (self.c_out, self.c_in), torch.float32, "gw", dev)
        bias = bias or gb is not None
        agb = _addr(gb, (self.c_out,), torch.float32, "gb", dev)
        given = [a for a in (agx, agw, agb) if a]
        if len(set(given)) < len(given):
            raise ValueError("gx, gw and gb: one buffer is given twice")
        s = _stream_of(dev, stream)
        if need_x and gx is None:
            _given(stream, "gx")
            gx = torch.empty(g.shape[:-1] + (self.c_in,), dtype=self.dtype, device=dev)
            agx = gx.data_ptr()
        if kept is not None and gw is None:
            _given(stream, "gw")
            gw = torch.empty((self.c_out, self.c_in), dtype=torch.float32, device=dev)
            agw = gw.data_ptr()
        if bias and gb is None:
            _given(stream, "gb")
            gb = torch.empty(self.c_out, dtype=torch.float32, device=dev)
            agb = gb.data_ptr()
        q, qs, t, ts, ws = self._places(self._bwd_parts, dev, s)
        if not need_x:
            q = qs = 0
        if kept is None:
            t = ts = 0
        n = self._bwd_parts[-1]
        B.fno_fp8_quantize(self.q_g.desc, ag, q, qs, t, ts, agb, ws, n, s)
        if need_x:
            B.fno_fp8_matmul(self.mm_x.desc, q, qs, *aw, ax, 0, agx, ws, n, s)
        if kept is not None:
            B.fno_fp8_matmul(self.mm_w.desc, t, ts, *ak, 0, 0, agw, ws, n, s)
        return gx, gw, gb
