"""Matrices in microscaled 4-bit floating point: ctypes binding of the conversion to and from blocks of 32 codes with a scale, and of the products
grouped by expert (same names as the C entry points, argument marshalling only).

`stream` (None: torch's current stream) is where a call runs.  What it allocates is that stream's memory; as with any work on several streams, the
caller makes `stream` wait for the arguments, keeps them until it has read them, and waits for it before using the results elsewhere."""
import collections
import ctypes
import math

import torch

from .binding import ACT, _check, _new, _stream_ptr, lib
from .experts import _dense, _device, _matrix, _no_graph, _type

_i, _p, _l = ctypes.c_int, ctypes.c_void_p, ctypes.c_int64
for _name, _args in {
        "polydl_mx4_quantise": [_l, _i, _p, _l, _i, _p, _p, _p],
        "polydl_mx4_dequantise": [_l, _i, _p, _p, _p, _l, _i, _p],
        "polydl_mx4_gemm": [_i] * 4 + [_p, _p, _i] + [_p] * 5 + [_l, _i, _i, _p]}.items():
    getattr(lib, _name).argtypes = _args
    getattr(lib, _name).restype = _i

Mx4 = collections.namedtuple("Mx4", "q scales")


def mx4_shapes(*shape):
    """Shapes of the codes (uint8, two a byte) and scales (uint8) of a tensor [...][K]."""
    blocks = -(-shape[-1] // 128) * 4
    return (*shape[:-1], blocks * 16), (*shape[:-1], blocks)


def mx4_quantise(x, out=None, stream=None):
    """polydl_mx4_quantise: Mx4(q, scales) of x [rows][K] (any row stride) or [...][K] (contiguous), float32 or bfloat16."""
    if x.requires_grad:
        _no_graph()
    dev, K = _device(), x.shape[-1]
    codes, scales = mx4_shapes(*x.shape)
    if x.dim() == 2:
        rows, (xp, ldx) = x.shape[0], _matrix(x, "x", x.dtype, x.shape, dev)
    else:
        rows, xp, ldx = math.prod(x.shape[:-1]), _dense(x, "x", x.dtype, x.shape, dev), K
    if out is None:
        out = Mx4(_new(codes, torch.uint8, x, stream), _new(scales, torch.uint8, x, stream))
        qp, sp = out.q.data_ptr(), out.scales.data_ptr()
    else:
        out = Mx4(*out)
        qp, sp = _dense(out.q, "q", torch.uint8, codes, dev), _dense(out.scales, "scales", torch.uint8, scales, dev)
    _check(lib.polydl_mx4_quantise(rows, K, xp, ldx, _type(x.dtype), qp, sp, _stream_ptr(stream)), "polydl_mx4_quantise")
    return out


def mx4_dequantise(x, K, out=None, out_dtype=torch.bfloat16, stream=None):
    """polydl_mx4_dequantise: the values [...][K] of Mx4(q, scales)."""
    q, scales = x
    dev, lead = _device(), tuple(q.shape[:-1])
    codes, per_block = mx4_shapes(*lead, K)
    if out is None:
        out = _new((*lead, K), out_dtype, q, stream)
    if len(lead) == 1:
        rows, (yp, ldy) = lead[0], _matrix(out, "out", out.dtype, (*lead, K), dev)
    else:
        rows, yp, ldy = math.prod(lead), _dense(out, "out", out.dtype, (*lead, K), dev), K
    _check(lib.polydl_mx4_dequantise(rows, K, _dense(q, "q", torch.uint8, codes, dev), _dense(scales, "scales", torch.uint8, per_block, dev), yp, ldy,
                                     _type(out.dtype), _stream_ptr(stream)), "polydl_mx4_dequantise")
    return out


def mx4_gemm(x, w, offsets=None, rows=None, act=None, out=None, out_dtype=torch.bfloat16, stream=None):
    """polydl_mx4_gemm: act(x[rows] @ w[e].T) for the rows of each group e, x an Mx4 of [x_rows][K] and w one of [E][N][K] or [N][K]; without
    offsets all rows are one group.  Rows are filled up to 128 inputs, as mx4_shapes says."""
    (xq, xs), (wq, ws), dev = x, w, _device()
    E, N, width = wq.shape if wq.dim() == 3 else (1, *wq.shape)
    # (the C call takes K and fills rows up to whole 128 inputs: shorter ones would be read with the stride of longer ones)
    if width % 64:
        raise ValueError("w.q must have rows of whole 64 bytes (mx4_shapes: filled up to 128 inputs), not of %d" % width)
    x_rows, blocks = xq.shape[0], width // 16
    if offsets is None and E > 1:
        raise ValueError("more than one matrix needs offsets")
    M = x_rows if rows is None else rows.shape[0]
    if out is None:
        out = _new((M, N), out_dtype, xq, stream)
    yp, ldy = _matrix(out, "out", out.dtype, (M, N), dev)
    _check(lib.polydl_mx4_gemm(E, M, N, blocks * 32, _dense(offsets, "offsets", torch.int32, (E + 1,), dev), _dense(rows, "rows", torch.int32, (M,), dev),
                               x_rows, _dense(xq, "x.q", torch.uint8, (x_rows, blocks * 16), dev),
                               _dense(xs, "x.scales", torch.uint8, (x_rows, blocks), dev),
                               _dense(wq, "w.q", torch.uint8, (*wq.shape[:-1], blocks * 16), dev),
                               _dense(ws, "w.scales", torch.uint8, (*wq.shape[:-1], blocks), dev), yp, ldy, _type(out.dtype), ACT[act],
                               _stream_ptr(stream)), "polydl_mx4_gemm")
    return out
