"""Refusals of what stands around a layer of experts, on a machine without a GPU: every argument error is reported before the device is
looked at; and the binding's own checks."""
import ctypes

import pytest

import paper_2006_02230_amd as P

OK, NULL, DIM, UNSUPPORTED, NO_DEVICE = 0, -1, -2, -3, -5
Z = None
AT = 4096          # an address that is aligned and never looked at
BIG = (1 << 31) - 1


def st(name, *args):
    return getattr(P.lib, name)(*args, None)


def refuses(f, status, *cases):
    for kw in cases:
        assert f(**kw) == status, kw


def test_layernorm_refusals():
    def f(T=4, D=8, x=AT, ldx=8, x_type=0, gamma=AT, beta=AT, eps=1e-5, y=AT, ldy=8, y_type=1, mean=AT, rstd=AT):
        return st("polydl_layernorm_fwd", T, D, x, ldx, x_type, gamma, beta, eps, y, ldy, y_type, mean, rstd)
    refuses(f, DIM, {"T": -1}, {"D": 0}, {"D": -3}, {"ldx": 7}, {"ldy": 7})
    refuses(f, NULL, {"x": Z}, {"y": Z})
    refuses(f, UNSUPPORTED, {"x_type": 2}, {"y_type": -1}, {"D": (1 << 24) + 1, "ldx": 1 << 25, "ldy": 1 << 25}, {"ldx": (1 << 40) + 1}, {"eps": -1e-5},
            {"eps": float("nan")}, {"eps": float("inf")}, {"x": AT + 2}, {"x": AT + 1, "x_type": 1}, {"y": AT + 1}, {"gamma": AT + 2}, {"beta": AT + 2},
            {"mean": AT + 2}, {"rstd": AT + 2})


def test_layernorm_gradient_refusals():
    def f(T=4, D=8, dy=AT, lddy=8, dy_type=1, x=AT, ldx=8, x_type=0, mean=AT, rstd=AT, gamma=AT, dx=AT, lddx=8, dgamma=AT, dbeta=AT, acc=0, space=AT,
          size=1 << 30):
        return st("polydl_layernorm_bwd", T, D, dy, lddy, dy_type, x, ldx, x_type, mean, rstd, gamma, dx, lddx, dgamma, dbeta, acc, space, size)
    refuses(f, DIM, {"T": -1}, {"D": 0}, {"lddy": 7}, {"ldx": 7}, {"lddx": 7}, {"size": P.lib.polydl_layernorm_bwd_workspace_bytes(4, 8) - 1})
    refuses(f, NULL, {"dy": Z}, {"x": Z}, {"mean": Z}, {"rstd": Z}, {"space": Z})
    refuses(f, UNSUPPORTED, {"dy_type": 2}, {"x_type": 2}, {"D": (1 << 24) + 1, "ldx": 1 << 25, "lddy": 1 << 25, "lddx": 1 << 25}, {"dx": AT + 2},
            {"dgamma": AT + 2}, {"dbeta": AT + 1}, {"space": AT + 2}, {"gamma": AT + 2}, {"lddx": (1 << 40) + 1})
    f = P.lib.polydl_layernorm_bwd_workspace_bytes
    assert f(0, 8) == 0 and f(4, 0) == 0 and f(4, (1 << 24) + 1) == 0 and f(1, 8) >= 64 and f(BIG, 1 << 24) >= 1 << 27


def test_balance_refusals():
    def f(T=4, E=8, k=2, logits=AT, ids=AT, loss=AT, counts=AT, shares=AT, rows=AT, space=AT, size=1 << 24):
        return st("polydl_balance", T, E, k, logits, ids, loss, counts, shares, rows, space, size)
    refuses(f, DIM, {"T": -1}, {"E": 0}, {"k": 0}, {"T": 5000, "size": P.lib.polydl_balance_workspace_bytes(5000, 8) - 1})
    refuses(f, NULL, *({name: Z} for name in ("logits", "ids", "loss", "counts", "shares", "rows")), {"T": 5000, "space": Z}, {"T": 0, "loss": Z})
    refuses(f, UNSUPPORTED, {"E": 1025}, {"k": 33}, {"T": BIG}, {"T": 5000, "space": AT + 2},
            *({name: AT + 2} for name in ("logits", "ids", "loss", "counts", "shares", "rows")))

    def g(T=4, E=8, logits=AT, counts=AT, rows=AT, c=1.0, dloss=AT, dlogits=AT, acc=0):
        return st("polydl_balance_bwd", T, E, logits, counts, rows, c, dloss, dlogits, acc)
    refuses(g, DIM, {"T": -1}, {"E": 0})
    refuses(g, NULL, *({name: Z} for name in ("logits", "counts", "rows", "dlogits")))
    refuses(g, UNSUPPORTED, {"E": 1025}, *({name: AT + 2} for name in ("logits", "counts", "rows", "dloss", "dlogits")))
    f = P.lib.polydl_balance_workspace_bytes
    assert f(0, 8) == 0 and f(8, 0) == 0 and f(8, 1025) == 0 and f(BIG, 1024) >= 8 * 1024


def table(grads, counts, types, out=None):
    n = len(counts)
    make = lambda kind, v: (kind * max(n, 1))(*v)                     # noqa: E731
    return (n, make(ctypes.c_void_p, grads), make(ctypes.c_int64, counts), make(ctypes.c_int, types), None if out is None else make(ctypes.c_void_p, out))


def test_clip_refusals():
    def f(grads=(AT, 2 * AT), counts=(10, 20), types=(0, 1), out=None, max_norm=1.0, norm=AT, space=AT, size=1 << 20):
        n, g, c, t, o = table(grads, counts, types, out)
        status = st("polydl_clip_grads", n, g, c, t, max_norm, o, norm, space, size)
        if out is None and max_norm == 1.0 and not any(a == b for a in grads for b in grads if a is not b):
            assert st("polydl_grad_norm", n, g, c, t, norm, space, size) in (status, NO_DEVICE)
        return status
    refuses(f, DIM, {"counts": (10, -1)}, {"size": 8})
    refuses(f, NULL, {"grads": (AT, Z)}, {"norm": Z}, {"space": Z}, {"out": (AT, Z)})
    refuses(f, UNSUPPORTED, {"types": (0, 2)}, {"types": (-1, 1)}, {"counts": (10, (1 << 42) + 1)}, {"grads": (AT + 2, 2 * AT)}, {"grads": (AT, 2 * AT + 1)},
            {"norm": AT + 2}, {"space": AT + 4}, {"max_norm": -1.0}, {"max_norm": float("nan")}, {"out": (AT + 2, 2 * AT)}, {"out": (AT, 2 * AT + 1)},
            # what is written overlaps another tensor
            {"grads": (AT, AT)}, {"grads": (AT, AT + 36)}, {"grads": (AT + 38, AT), "types": (1, 0)}, {"out": (3 * AT, 3 * AT)}, {"out": (2 * AT, AT)},
            {"out": (2 * AT + 36, 3 * AT)}, {"out": (AT + 4, 3 * AT)})
    assert st("polydl_clip_grads", -1, None, None, None, 1.0, None, AT, AT, 64) == DIM
    for args in ((None, table([AT], [1], [0])[2], table([AT], [1], [0])[3]), (table([AT], [1], [0])[1], None, table([AT], [1], [0])[3]),
                 (table([AT], [1], [0])[1], table([AT], [1], [0])[2], None)):
        assert st("polydl_clip_grads", 1, *args, 1.0, None, AT, AT, 64) == NULL


def test_clip_accepts_what_does_not_overlap():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a call that is accepted would run")
    for grads, counts, types, out in (((AT, AT + 40), (10, 20), (0, 1), None), ((AT, AT), (10, 10), (0, 0), (2 * AT, 3 * AT)), ((AT, Z), (3, 0), (0, 1), None),
                                      ((), (), (), None), ((AT, AT + 40), (10, 10), (0, 0), (AT, 2 * AT)), ((AT + 20, AT), (4, 5), (0, 0), None)):
        n, g, c, t, o = table(grads, counts, types, out)
        assert st("polydl_clip_grads", n, g, c, t, 1.0, o, AT, AT, 1 << 20) == NO_DEVICE


def test_clip_workspace():
    def f(*counts):
        return P.lib.polydl_clip_workspace_bytes(len(counts), table(counts, counts, counts)[2])
    assert f() == 8 and f(0, 0) == 8 and f(5) == 16 and f(1 << 42) <= 1 << 15 and f(*[5] * 1000) <= 16 * 1024
    assert P.lib.polydl_clip_workspace_bytes(-1, None) == 0 and P.lib.polydl_clip_workspace_bytes(3, None) == 0


def test_mx4_refusals():
    def q(rows=4, K=40, x=AT, ldx=40, kind=1, q=AT, scales=AT, name="polydl_mx4_quantise"):
        if name == "polydl_mx4_quantise":
            return st(name, rows, K, x, ldx, kind, q, scales)
        return st(name, rows, K, q, scales, x, ldx, kind)
    for name in ("polydl_mx4_quantise", "polydl_mx4_dequantise"):
        def f(**kw):
            return q(name=name, **kw)
        refuses(f, DIM, {"rows": -1}, {"K": 0}, {"ldx": 39})
        refuses(f, NULL, {"x": Z}, {"q": Z}, {"scales": Z})
        refuses(f, UNSUPPORTED, {"kind": 2}, {"K": BIG, "ldx": BIG}, {"rows": 1 << 60}, {"ldx": (1 << 40) + 1}, {"q": AT + 8}, {"scales": AT + 2}, {"x": AT + 1},
                {"x": AT + 2, "kind": 0})

    def f(E=2, M=8, N=16, K=24, offsets=AT, rows=Z, x_rows=8, xq=AT, xs=AT, wq=AT, ws=AT, y=AT, ldy=16, kind=1, act=0):
        return st("polydl_mx4_gemm", E, M, N, K, offsets, rows, x_rows, xq, xs, wq, ws, y, ldy, kind, act)
    refuses(f, DIM, {"E": 0}, {"M": -1, "x_rows": -1}, {"N": 0}, {"K": 0}, {"ldy": 15}, {"x_rows": 7}, {"x_rows": -1, "rows": AT})
    refuses(f, NULL, *({name: Z} for name in ("offsets", "xq", "xs", "wq", "ws", "y")))
    refuses(f, UNSUPPORTED, {"act": 3}, {"kind": 2}, {"ldy": (1 << 40) + 1}, {"E": BIG}, {"K": BIG}, {"N": BIG, "ldy": BIG}, {"M": BIG, "x_rows": BIG},
            {"E": 1 << 30, "N": 1 << 20, "ldy": 1 << 20, "K": 1 << 20}, {"offsets": AT + 2}, {"rows": AT + 2}, {"xq": AT + 8}, {"xs": AT + 2}, {"wq": AT + 8},
            {"ws": AT + 2}, {"y": AT + 1}, {"y": AT + 2, "kind": 0})


def test_shapes():
    assert P.mx4_shapes(7, 1) == ((7, 64), (7, 4)) and P.mx4_shapes(2, 7, 128) == ((2, 7, 64), (2, 7, 4)) and P.mx4_shapes(1, 129) == ((1, 128), (1, 8))


def test_binding_refusals():
    import torch
    x, w = torch.ones(4, 8), torch.ones(8)
    ids = torch.zeros(4, 1, dtype=torch.int32)
    one = torch.ones(4)
    calls = [lambda: P.layernorm_fwd(x, w, w), lambda: P.layernorm_bwd(x, x, one, one), lambda: P.balance(x, ids),
             lambda: P.balance_bwd(x, torch.zeros(8, dtype=torch.int32), torch.zeros((), dtype=torch.int32)), lambda: P.grad_norm([x]),
             lambda: P.clip_grads([x], 1.0), lambda: P.mx4_quantise(x), lambda: P.mx4_dequantise(P.Mx4(*(torch.zeros(s, dtype=torch.uint8) for s in P.mx4_shapes(4, 8))), 8)]
    for call in calls:
        with pytest.raises(TypeError, match="memory"):                    # not in device memory
            call()
    for call in (lambda: P.layernorm_bwd(x, x, one, one, weights=False, dgamma=w), lambda: P.layernorm_bwd(x, x, one, one, accumulate=True),
                 lambda: P.layernorm_bwd(x, x, one, one, weights=False, accumulate=True), lambda: P.balance_bwd(x, ids, ids, accumulate=True),
                 lambda: P.balance_bwd(x, ids, ids), lambda: P.balance_bwd(x, ids, torch.zeros(()), torch.ones(2)), lambda: P.grad_norm([]),
                 lambda: P.mx4_gemm(P.Mx4(*(torch.zeros(s, dtype=torch.uint8) for s in P.mx4_shapes(4, 8))),
                                    P.Mx4(*(torch.zeros(s, dtype=torch.uint8) for s in P.mx4_shapes(2, 4, 8)))),
                 lambda: P.layernorm_fwd(torch.ones(3))):
        with pytest.raises(ValueError):
            call()
    for bad in (x.double(), x.half(), x.int(), [1.0]):
        with pytest.raises((TypeError, AttributeError)):
            P.clip_grads([bad], 1.0)
    for t, filled in ((torch.empty(3, 4, 5).permute(2, 0, 1), True), (torch.empty(3, 4)[:, :2], False), (torch.empty(1, 4).expand(3, 4), False),
                      (torch.empty(5, 1, 3)[:, :, :1], False), (torch.empty(4, 3).t(), True)):
        assert P.training._filled(t) == filled


def test_clip_workspace_of_refused_lengths():
    import numpy as np
    for bad in (-1, (1 << 42) + 1, (1 << 63) - 1):
        counts = np.array([5, bad], dtype=np.int64)
        assert P.lib.polydl_clip_workspace_bytes(2, counts.ctypes.data) == 0


def test_clip_refuses_what_is_no_tensor():
    import numpy as np
    for bad in (None, 1.0, np.zeros(3, dtype=np.float32)):
        for call in (lambda: P.grad_norm([bad]), lambda: P.clip_grads([bad], 1.0)):
            with pytest.raises(TypeError):
                call()


def test_mx4_product_refuses_rows_that_are_not_filled_up():
    # rows of 1, 2, 3, 5, 6, 7 blocks, or of no whole block, of x and w alike: the library's rows are whole fours of blocks, and it would read the next ones'
    import torch
    zeros = lambda *s: torch.zeros(s, dtype=torch.uint8)                  # noqa: E731
    for width in (1, 16, 32, 48, 63, 65, 80, 96, 112, 1040):
        x, w = P.Mx4(zeros(4, width), zeros(4, width // 16)), P.Mx4(zeros(6, width), zeros(6, width // 16))
        for call in (lambda: P.mx4_gemm(x, w), lambda: P.mx4_gemm(x, P.Mx4(w.q[None], w.scales[None]), offsets=torch.zeros(2, dtype=torch.int32))):
            with pytest.raises(ValueError, match="128"):
                call()


def test_second_derivatives_that_would_be_lost_are_refused():
    # the gradients' own arguments, before anything else is looked at
    import torch
    x, w, one = torch.ones(4, 8), torch.ones(8), torch.ones(4)
    counts, rows = torch.zeros(8, dtype=torch.int32), torch.zeros((), dtype=torch.int32)
    norm = lambda dy=x, x=x, mean=one, rstd=one, gamma=w: P.layernorm_bwd(dy, x, mean, rstd, gamma)      # noqa: E731
    balance = lambda logits=x, dloss=torch.ones(1): P.balance_bwd(logits, counts, rows, dloss)           # noqa: E731
    for f, name, t in [(norm, n, x) for n in ("dy", "x")] + [(norm, n, one) for n in ("mean", "rstd")] + [(norm, "gamma", w), (balance, "logits", x),
                                                                                                          (balance, "dloss", torch.ones(1))]:
        leaf = t.clone().requires_grad_()
        with pytest.raises(RuntimeError, match="requires its gradient"):
            f(**{name: leaf})
        with torch.no_grad(), pytest.raises(TypeError, match="memory"):                                  # (the next check, on any machine)
            f(**{name: leaf})
