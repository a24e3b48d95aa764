"""What a training step needs around a layer of experts: ctypes binding of the layer norm, the router's balance loss, the norm of all gradients
and their clipping (same names as the C entry points, argument marshalling only).

As in the layer of experts, gradients are calls of their own, results carry no graph, and nothing here waits for the device.  While torch records
a graph, every call refuses arguments that require a gradient, the gradients' calls among them: second derivatives would be lost.  Matrices may
have any row stride; their columns are contiguous.

`stream` (None: torch's current stream) is where a call runs.  What it allocates is that stream's memory; as with any work on several streams, the
caller makes `stream` wait for the arguments, keeps them until it has read them, and waits for it before using the results elsewhere."""
import array
import collections
import ctypes

import torch

from .binding import _check, _new, _stream_ptr, lib
from .experts import _dense, _device, _matrix, _no_graph, _type

_i, _p, _l, _z, _f, _d = ctypes.c_int, ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float, ctypes.c_double
for _name, _args in {
        "polydl_layernorm_fwd": [_i, _i, _p, _l, _i, _p, _p, _f, _p, _l, _i, _p, _p, _p],
        "polydl_layernorm_bwd": [_i, _i, _p, _l, _i, _p, _l, _i, _p, _p, _p, _p, _l, _p, _p, _i, _p, _z, _p],
        "polydl_balance": [_i] * 3 + [_p] * 7 + [_z, _p],
        "polydl_balance_bwd": [_i, _i, _p, _p, _p, _f, _p, _p, _i, _p],
        "polydl_grad_norm": [_i, _p, _p, _p, _p, _p, _z, _p],
        "polydl_clip_grads": [_i, _p, _p, _p, _d, _p, _p, _p, _z, _p]}.items():
    getattr(lib, _name).argtypes = _args
    getattr(lib, _name).restype = _i
for _name, _args in {"polydl_layernorm_bwd_workspace_bytes": [_i, _i], "polydl_balance_workspace_bytes": [_i, _i],
                     "polydl_clip_workspace_bytes": [_i, _p]}.items():
    getattr(lib, _name).argtypes = _args
    getattr(lib, _name).restype = _z

Norm = collections.namedtuple("Norm", "y mean rstd")
NormGradients = collections.namedtuple("NormGradients", "dx dgamma dbeta")
Balance = collections.namedtuple("Balance", "loss counts shares rows")


def _lost(*tensors):
    """Refuses arguments whose gradient would be lost."""
    if torch.is_grad_enabled() and any(isinstance(t, torch.Tensor) and t.requires_grad for t in tensors):
        _no_graph()


def layernorm_fwd(x, gamma=None, beta=None, eps=1e-5, out=None, out_dtype=None, stream=None):
    """polydl_layernorm_fwd on the rows of x [T][D] (float32 or bfloat16): Norm(y [T][D] of out_dtype (None: x's), mean [T], rstd [T])."""
    _lost(x, gamma, beta)
    (T, D), dev = x.shape, _device()
    xp, ldx = _matrix(x, "x", x.dtype, (T, D), dev)
    if out is None:
        out = _new((T, D), x.dtype if out_dtype is None else out_dtype, x, stream)
        yp, ldy = out.data_ptr(), D
    else:
        yp, ldy = _matrix(out, "out", out.dtype, (T, D), dev)
    mean, rstd = _new((2, T), torch.float32, x, stream).unbind(0)
    _check(lib.polydl_layernorm_fwd(T, D, xp, ldx, _type(x.dtype), _dense(gamma, "gamma", torch.float32, (D,), dev),
                                    _dense(beta, "beta", torch.float32, (D,), dev), eps, yp, ldy, _type(out.dtype), mean.data_ptr(), rstd.data_ptr(),
                                    _stream_ptr(stream)), "polydl_layernorm_fwd")
    return Norm(out, mean, rstd)


def layernorm_bwd(dy, x, mean, rstd, gamma=None, dx=None, dgamma=None, dbeta=None, accumulate=False, weights=True, stream=None):
    """polydl_layernorm_bwd: NormGradients(dx [T][D] of x's type, dgamma [D], dbeta [D] float32).  accumulate adds to the dgamma and dbeta that
    are given; weights=False leaves them out (None)."""
    if dy.requires_grad or x.requires_grad or mean.requires_grad or rstd.requires_grad or gamma is not None and gamma.requires_grad:
        _no_graph()
    (T, D), dev = x.shape, _device()
    if not weights and (accumulate or dgamma is not None or dbeta is not None):
        raise ValueError("weights=False forms neither dgamma nor dbeta")
    if accumulate and (dgamma is None or dbeta is None):
        raise ValueError("accumulate needs dgamma and dbeta")
    dp, lddy = _matrix(dy, "dy", dy.dtype, (T, D), dev)
    xp, ldx = _matrix(x, "x", x.dtype, (T, D), dev)
    if dx is None:
        dx = _new((T, D), x.dtype, x, stream)
        op, lddx = dx.data_ptr(), D
    else:
        op, lddx = _matrix(dx, "dx", x.dtype, (T, D), dev)
    if weights and dgamma is None and dbeta is None:
        dgamma, dbeta = _new((2, D), torch.float32, x, stream).unbind(0)          # an allocation takes longer than a view
    elif weights:
        dgamma, dbeta = (_new((D,), torch.float32, x, stream) if t is None else t for t in (dgamma, dbeta))
    need = lib.polydl_layernorm_bwd_workspace_bytes(T, D) if weights else 0
    space = _new((need,), torch.uint8, x, stream) if need else None
    _check(lib.polydl_layernorm_bwd(T, D, dp, lddy, _type(dy.dtype), xp, ldx, _type(x.dtype), _dense(mean, "mean", torch.float32, (T,), dev),
                                    _dense(rstd, "rstd", torch.float32, (T,), dev), _dense(gamma, "gamma", torch.float32, (D,), dev), op, lddx,
                                    _dense(dgamma, "dgamma", torch.float32, (D,), dev), _dense(dbeta, "dbeta", torch.float32, (D,), dev),
                                    bool(accumulate), space.data_ptr() if need else None, need, _stream_ptr(stream)), "polydl_layernorm_bwd")
    return NormGradients(dx, dgamma, dbeta)


def balance(logits, ids, stream=None):
    """polydl_balance on a router's logits [T][E] and choices [T][k]: Balance(loss [], counts [E] int32, shares [E], rows [] int32)."""
    _lost(logits)
    (T, E), k, dev = logits.shape, ids.shape[1], _device()
    src = _dense(logits, "logits", torch.float32, (T, E), dev)
    loss, shares, counts, rows = _new((2 * E + 2,), torch.int32, logits, stream).split_with_sizes((1, E, E, 1))     # one allocation
    need = lib.polydl_balance_workspace_bytes(T, E)
    space = _new((need,), torch.uint8, logits, stream) if need else None
    _check(lib.polydl_balance(T, E, k, src, _dense(ids, "ids", torch.int32, (T, k), dev), loss.data_ptr(), counts.data_ptr(), shares.data_ptr(),
                              rows.data_ptr(), space.data_ptr() if need else None, need, _stream_ptr(stream)), "polydl_balance")
    return Balance(loss.view(torch.float32)[0], counts, shares.view(torch.float32), rows[0])


def balance_bwd(logits, counts, rows, dloss=1.0, out=None, accumulate=False, stream=None):
    """polydl_balance_bwd: the gradient of the logits [T][E] from that of the loss, a number or a float32 tensor of one value; accumulate adds it
    to out."""
    given = isinstance(dloss, torch.Tensor)
    if logits.requires_grad or given and dloss.requires_grad:
        _no_graph()
    (T, E), dev = logits.shape, _device()
    if accumulate and out is None:
        raise ValueError("accumulate needs out")
    if out is None:
        out = _new((T, E), torch.float32, logits, stream)
    for t, name in ((rows, "rows"),) + (((dloss, "dloss"),) if given else ()):
        if t.numel() != 1:
            raise ValueError("%s must hold one value" % name)
    _check(lib.polydl_balance_bwd(T, E, _dense(logits, "logits", torch.float32, (T, E), dev), _dense(counts, "counts", torch.int32, (E,), dev),
                                  _dense(rows, "rows", torch.int32, rows.shape, dev), 1.0 if given else dloss,
                                  _dense(dloss, "dloss", torch.float32, dloss.shape, dev) if given else None,
                                  _dense(out, "out", torch.float32, (T, E), dev), bool(accumulate), _stream_ptr(stream)), "polydl_balance_bwd")
    return out


def _filled(t):
    """Whether a tensor's values lie without gaps or overlaps, in whatever order of its axes."""
    if t.is_contiguous():
        return True
    step = 1
    for stride, size in sorted((st, n) for st, n in zip(t.stride(), t.shape) if n != 1):
        if stride != step:
            return False
        step *= size
    return True


_Tensor = torch.Tensor


# A check is one pass over the list: tensor by tensor, with calls for each, 300 tensors took 145 us.
def _listed(tensors, name, dev):
    """The types, lengths and layouts (None: all contiguous) of a list of dense tensors, checked."""
    types = [getattr(t, "dtype", None) for t in tensors]
    if not set(types) <= {torch.float32, torch.bfloat16}:
        raise TypeError("%s must be float32 or bfloat16 tensors" % name)
    if set(map(_Tensor.get_device, tensors)) - {dev} or dev is None:
        raise TypeError("%s must be in the current device's memory" % name)
    layouts = None
    if not all(map(_Tensor.is_contiguous, tensors)):
        if not all(map(_filled, tensors)):
            raise TypeError("%s must be dense" % name)
        layouts = [None if t.is_contiguous() else (t.shape, t.stride()) for t in tensors]
    return types, list(map(_Tensor.numel, tensors)), layouts


# (a ctypes array from a list takes four times as long as one of `array`)
def _addresses(tensors):
    return array.array("q", list(map(_Tensor.data_ptr, tensors)))


def _at(values):
    return values.buffer_info()[0]


def _gradients(grads):
    """The list, its types, lengths and layouts, and the host arrays of addresses, lengths and types that a call takes."""
    grads = list(grads)
    if not grads:
        raise ValueError("there are no gradients")
    types, counts, layouts = _listed(grads, "grads", _device())
    if torch.is_grad_enabled() and any([t.requires_grad for t in grads]):
        _no_graph()
    half = torch.bfloat16
    return grads, types, counts, layouts, _addresses(grads), array.array("q", counts), array.array("i", [t is half for t in types])


def _norm_space(like, n, counts, stream):
    need = lib.polydl_clip_workspace_bytes(n, _at(counts))
    return _new((), torch.float32, like, stream), _new((need,), torch.uint8, like, stream), need


def grad_norm(grads, stream=None):
    """polydl_grad_norm: the norm [] (float32) of a list of tensors (float32 or bfloat16, dense) taken as one vector."""
    grads, _, _, _, at, counts, types = _gradients(grads)
    norm, space, need = _norm_space(grads[0], len(grads), counts, stream)
    _check(lib.polydl_grad_norm(len(grads), _at(at), _at(counts), _at(types), norm.data_ptr(), space.data_ptr(), need, _stream_ptr(stream)), "polydl_grad_norm")
    return norm


def clip_grads(grads, max_norm, out=None, stream=None):
    """polydl_clip_grads: scales a list of tensors to a norm of at most max_norm, in place or into the tensors of `out` (of the same types and
    lengths, and where they are not contiguous of the same shapes and strides); returns the norm [] (float32) before.  Where an infinity or NaN is
    among the values, nothing is scaled."""
    grads, kinds, lengths, layouts, at, counts, types = _gradients(grads)
    to = None
    if out is not None:
        out = list(out)
        if _listed(out, "out", _device()) != (kinds, lengths, layouts):
            raise ValueError("out must be tensors of the gradients' types, lengths and layouts")
        to = _addresses(out)
    norm, space, need = _norm_space(grads[0], len(grads), counts, stream)
    _check(lib.polydl_clip_grads(len(grads), _at(at), _at(counts), _at(types), float(max_norm), None if to is None else _at(to), norm.data_ptr(),
                                 space.data_ptr(), need, _stream_ptr(stream)), "polydl_clip_grads")
    return norm
