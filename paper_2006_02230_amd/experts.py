"""The layer of experts: ctypes binding of the router, the products grouped by expert, the weighted sum and the products
with 4-bit weights (same names as the C entry points, argument marshalling only), and a layer that runs them together.

Rows sorted by expert, their offsets, `tokens` and `slots` are tensors on the device (`route` makes them); nothing here waits for the
device.  Matrices may have any row stride; their columns are contiguous.

The gradients are calls of their own (route_bwd, combine_bwd_bf16, grouped_gemm_dx_bf16, grouped_gemm_dw_bf16): results carry no graph, so while torch records one,
the calls that have a gradient refuse arguments that require theirs.

`stream` (None: torch's current stream) is where a call runs.  What it allocates is that stream's memory; as with any work on several streams, the
caller makes `stream` wait for the arguments, keeps them until it has read them, and waits for it before using the results elsewhere."""
import collections
import ctypes

import torch

from .binding import ACT, _check, _current_device, _new, _stream_ptr, lib

_i, _p, _l, _z = ctypes.c_int, ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t
for _name, _args in {
        "polydl_route": [_i] * 3 + [_p, _i] + [_p] * 5 + [_p, _z, _p],
        "polydl_route_bwd": [_i] * 3 + [_p] * 4 + [_i, _p, _p],
        "polydl_combine_bf16": [_i] * 4 + [_p] * 4 + [_i, _p],
        "polydl_combine_bwd_bf16": [_i] * 4 + [_p] * 7,
        "polydl_grouped_gemm_bf16": [_i] * 4 + [_p, _p, _i, _p, _l, _p, _p, _l, _i, _i, _p],
        "polydl_grouped_gemm_dx_bf16": [_i] * 4 + [_p, _p, _l, _p, _p, _l, _i, _p, _l, _i, _p],
        "polydl_grouped_gemm_dw_bf16": [_i] * 4 + [_p, _p, _l, _p, _i, _p, _l, _p, _i, _i, _p],
        "polydl_w4_pack_bf16": [_i] * 4 + [_p] * 5,
        "polydl_w4_gemm_bf16": [_i] * 5 + [_p, _p, _i, _p, _l, _p, _p, _p, _p, _l, _i, _i, _p]}.items():
    getattr(lib, _name).argtypes = _args
    getattr(lib, _name).restype = _i
lib.polydl_route_workspace_bytes.argtypes = [_i, _i]
lib.polydl_route_workspace_bytes.restype = _z

_TYPES = {torch.float32: 0, torch.bfloat16: 1}

Route = collections.namedtuple("Route", "ids weights offsets tokens slots")
W4 = collections.namedtuple("W4", "q scales zeros")


# A call's checks are one comparison a tensor where all is well: with a message's worth of them a small product's host side took
# 11 us, more than its kernel.
def _device():
    try:
        return _current_device() if _current_device is not None else torch.cuda.current_device()
    except (RuntimeError, AssertionError):         # no device: no tensor is on it
        return None


def _no_graph():
    if torch.is_grad_enabled():
        raise RuntimeError("an argument requires its gradient, which would be lost: results carry no graph.  Call under torch.no_grad() or in an "
                           "autograd.Function, whose backward calls the operator's gradient")


def _refuse(t, name, dtype, shape, dev):
    if not isinstance(t, torch.Tensor) or t.dtype != dtype:
        raise TypeError("%s must be a %s tensor" % (name, dtype))
    if not t.is_cuda or t.get_device() != dev:
        raise TypeError("%s must be in the current device's memory" % name)
    if shape is not None and t.shape != shape:
        raise ValueError("%s must have the shape %s, not %s" % (name, tuple(shape), tuple(t.shape)))
    raise TypeError("%s must be contiguous" % name)


def _dense(t, name, dtype, shape, dev):
    """Device pointer of a contiguous tensor of one type and shape (None passes NULL)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != dev or t.shape != shape or not t.is_contiguous():
        _refuse(t, name, dtype, shape, dev)
    return t.data_ptr()


def _matrix(t, name, dtype, shape, dev):
    """Device pointer and row stride of a matrix with contiguous columns."""
    if t.dtype is not dtype or t.get_device() != dev or t.shape != shape:
        _refuse(t, name, dtype, shape, dev)
    row, col = t.stride()
    if col != 1 and shape[1] > 1:
        raise TypeError("%s must have contiguous columns" % name)
    return t.data_ptr(), row if shape[0] > 1 else shape[1]


def _type(dtype):
    if dtype not in _TYPES:
        raise TypeError("results are float32 or bfloat16")
    return _TYPES[dtype]


def route(logits, k, renorm=True, stream=None):
    """polydl_route on float32 logits [T][E]: Route(ids [T][k], weights [T][k], offsets [E+1], tokens [T*k], slots [T][k])."""
    if logits.requires_grad:
        _no_graph()
    T, E = logits.shape
    src = _dense(logits, "logits", torch.float32, (T, E), _device())
    ids, slots, weights = _new((3, T, k), torch.int32, logits, stream).unbind(0)          # allocations take longer than views
    weights = weights.view(torch.float32)
    tokens, offsets = _new((T * k + E + 1,), torch.int32, logits, stream).split_with_sizes((T * k, E + 1))
    need = lib.polydl_route_workspace_bytes(T, E) if T > 64 else 0
    space = _new((need,), torch.uint8, logits, stream) if need else None
    _check(lib.polydl_route(T, E, k, src, bool(renorm), ids.data_ptr(), weights.data_ptr(), offsets.data_ptr(), tokens.data_ptr(),
                            slots.data_ptr(), space.data_ptr() if need else None, need, _stream_ptr(stream)), "polydl_route")
    return Route(ids, weights, offsets, tokens, slots)


def route_bwd(logits, ids, weights, dweights, renorm=True, out=None, stream=None):
    """polydl_route_bwd: the gradient of the logits [T][E] from that of the weights."""
    (T, E), k, dev = logits.shape, ids.shape[1], _device()
    if out is None:
        out = _new((T, E), torch.float32, logits, stream)
    _check(lib.polydl_route_bwd(T, E, k, _dense(logits, "logits", torch.float32, (T, E), dev), _dense(ids, "ids", torch.int32, (T, k), dev),
                                _dense(weights, "weights", torch.float32, (T, k), dev), _dense(dweights, "dweights", torch.float32, (T, k), dev),
                                bool(renorm), _dense(out, "out", torch.float32, (T, E), dev), _stream_ptr(stream)), "polydl_route_bwd")
    return out


def combine_bf16(y, slots, weights=None, out=None, out_dtype=torch.bfloat16, stream=None):
    """polydl_combine_bf16: [T][D] from y [M][D] (bfloat16), slots [T][k] and weights [T][k] (None: ones)."""
    if y.requires_grad or weights is not None and weights.requires_grad:
        _no_graph()
    (M, D), (T, k), dev = y.shape, slots.shape, _device()
    if out is None:
        out = _new((T, D), out_dtype, y, stream)
    _check(lib.polydl_combine_bf16(T, k, M, D, _dense(y, "y", torch.bfloat16, (M, D), dev), _dense(slots, "slots", torch.int32, (T, k), dev),
                                   _dense(weights, "weights", torch.float32, (T, k), dev), _dense(out, "out", out.dtype, (T, D), dev),
                                   _type(out.dtype), _stream_ptr(stream)), "polydl_combine_bf16")
    return out


def combine_bwd_bf16(dout, y, slots, weights=None, dy=None, stream=None):
    """polydl_combine_bwd_bf16: (dy [M][D] bfloat16, dweights [T][k] float32).  Rows of dy that are no token's slot keep what they hold."""
    (M, D), (T, k), dev = y.shape, slots.shape, _device()
    if dy is None:
        dy = _new((M, D), torch.bfloat16, y, stream)
    dweights = _new((T, k), torch.float32, y, stream)
    _check(lib.polydl_combine_bwd_bf16(T, k, M, D, _dense(dout, "dout", torch.bfloat16, (T, D), dev), _dense(y, "y", torch.bfloat16, (M, D), dev),
                                       _dense(slots, "slots", torch.int32, (T, k), dev), _dense(weights, "weights", torch.float32, (T, k), dev),
                                       _dense(dy, "dy", torch.bfloat16, (M, D), dev), dweights.data_ptr(), _stream_ptr(stream)),
           "polydl_combine_bwd_bf16")
    return dy, dweights


def grouped_gemm_bf16(x, w, offsets, rows=None, act=None, out=None, out_dtype=torch.bfloat16, stream=None):
    """polydl_grouped_gemm_bf16: act(x[rows] @ w[e].T) for the rows of each group e; w [E][N][K], offsets [E+1], rows [M] or None."""
    if x.requires_grad or w.requires_grad:
        _no_graph()
    (E, N, K), x_rows, dev = w.shape, x.shape[0], _device()
    M = x_rows if rows is None else rows.shape[0]
    if out is None:
        out = _new((M, N), out_dtype, x, stream)
    xp, ldx = _matrix(x, "x", torch.bfloat16, (x_rows, K), dev)
    yp, ldy = _matrix(out, "out", out.dtype, (M, N), dev)
    _check(lib.polydl_grouped_gemm_bf16(E, M, N, K, _dense(offsets, "offsets", torch.int32, (E + 1,), dev), _dense(rows, "rows", torch.int32, (M,), dev),
                                        x_rows, xp, ldx, _dense(w, "w", torch.bfloat16, (E, N, K), dev), yp, ldy, _type(out.dtype), ACT[act],
                                        _stream_ptr(stream)), "polydl_grouped_gemm_bf16")
    return out


def grouped_gemm_dx_bf16(dy, w, offsets, h=None, act=None, out=None, out_dtype=torch.bfloat16, stream=None):
    """polydl_grouped_gemm_dx_bf16: dy @ w[e] for the rows of each group, where act is given through its derivative at h, what it gave."""
    (E, N, K), M, dev = w.shape, dy.shape[0], _device()
    if ACT[act] and h is None:
        raise ValueError("the gradient through an activation needs h, what it gave")
    if out is None:
        out = _new((M, K), out_dtype, dy, stream)
    dp, ldd = _matrix(dy, "dy", torch.bfloat16, (M, N), dev)
    hp, ldh = _matrix(h, "h", torch.bfloat16, (M, K), dev) if ACT[act] else (None, 0)
    op, ldo = _matrix(out, "out", out.dtype, (M, K), dev)
    _check(lib.polydl_grouped_gemm_dx_bf16(E, M, N, K, _dense(offsets, "offsets", torch.int32, (E + 1,), dev), dp, ldd,
                                           _dense(w, "w", torch.bfloat16, (E, N, K), dev), hp, ldh, ACT[act], op, ldo, _type(out.dtype),
                                           _stream_ptr(stream)), "polydl_grouped_gemm_dx_bf16")
    return out


def grouped_gemm_dw_bf16(dy, x, offsets, rows=None, out=None, out_dtype=torch.float32, accumulate=False, stream=None):
    """polydl_grouped_gemm_dw_bf16: dy[group].T @ x[rows of the group] for each group: [E][N][K]; accumulate adds to out (float32)."""
    E, (M, N), (x_rows, K), dev = offsets.shape[0] - 1, dy.shape, x.shape, _device()
    if rows is None and x_rows != M:
        raise ValueError("x must have dy's rows, or rows be given")
    if accumulate and out is None:
        raise ValueError("accumulate needs out")
    if out is None:
        out = _new((E, N, K), out_dtype, dy, stream)
    dp, ldd = _matrix(dy, "dy", torch.bfloat16, (M, N), dev)
    xp, ldx = _matrix(x, "x", torch.bfloat16, (x_rows, K), dev)
    _check(lib.polydl_grouped_gemm_dw_bf16(E, M, N, K, _dense(offsets, "offsets", torch.int32, (E + 1,), dev), dp, ldd,
                                           _dense(rows, "rows", torch.int32, (M,), dev), x_rows, xp, ldx,
                                           _dense(out, "out", out.dtype, (E, N, K), dev), _type(out.dtype), bool(accumulate),
                                           _stream_ptr(stream)), "polydl_grouped_gemm_dw_bf16")
    return out


def w4_shapes(E, N, K, group):
    """Shapes of the packed codes and of the scales (and zero points) of E matrices [N][K]."""
    if group not in (32, 64, 128):
        raise ValueError("group must be 32, 64 or 128")
    tiles, steps = -(-N // 16), -(-K // 128)
    return (E, tiles, steps, 64, 16), (E, tiles, steps * (128 // group), 16)


def w4_pack_bf16(w, group=128, asymmetric=False, stream=None):
    """polydl_w4_pack_bf16: W4(q, scales, zeros) of w [E][N][K] or [N][K] (bfloat16); zeros is None unless asymmetric."""
    E, N, K = w.shape if w.dim() == 3 else (1, *w.shape)
    codes, scales = w4_shapes(E, N, K, group)
    src = _dense(w, "w", torch.bfloat16, w.shape, _device())
    r = W4(_new(codes, torch.uint8, w, stream), _new(scales, torch.bfloat16, w, stream),
           _new(scales, torch.uint8, w, stream) if asymmetric else None)
    _check(lib.polydl_w4_pack_bf16(E, N, K, group, src, r.q.data_ptr(), r.scales.data_ptr(), r.zeros.data_ptr() if asymmetric else None,
                                   _stream_ptr(stream)), "polydl_w4_pack_bf16")
    return r


def w4_gemm_bf16(x, q, scales, N, group, zeros=None, offsets=None, rows=None, act=None, out=None, out_dtype=torch.bfloat16, stream=None):
    """polydl_w4_gemm_bf16: act(x[rows] @ w[e].T) with the packed 4-bit weights of w4_pack_bf16, [N][x.shape[1]] each."""
    if x.requires_grad or scales.requires_grad:
        _no_graph()
    E, (x_rows, K), dev = q.shape[0], x.shape, _device()
    M = x_rows if rows is None else rows.shape[0]
    codes, per_group = w4_shapes(E, N, K, group)
    if out is None:
        out = _new((M, N), out_dtype, x, stream)
    xp, ldx = _matrix(x, "x", torch.bfloat16, (x_rows, K), dev)
    yp, ldy = _matrix(out, "out", out.dtype, (M, N), dev)
    _check(lib.polydl_w4_gemm_bf16(E, M, N, K, group, _dense(offsets, "offsets", torch.int32, (E + 1,), dev), _dense(rows, "rows", torch.int32, (M,), dev),
                                   x_rows, xp, ldx, _dense(q, "q", torch.uint8, codes, dev), _dense(scales, "scales", torch.bfloat16, per_group, dev),
                                   _dense(zeros, "zeros", torch.uint8, per_group, dev), yp, ldy, _type(out.dtype), ACT[act],
                                   _stream_ptr(stream)), "polydl_w4_gemm_bf16")
    return out
