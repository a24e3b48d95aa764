"""Refusals of the entry points of the layer of experts, on a machine without a GPU: every argument error is reported before the
device is looked at; and the binding's own checks."""
import ctypes

import pytest

import paper_2006_02230_amd as P

OK, NULL, DIM, UNSUPPORTED, NO_DEVICE = 0, -1, -2, -3, -5
Z = None
AT = 4096          # an address that is aligned and never looked at
BIG = (1 << 31) - 1


def st(name, *args):
    return getattr(P.lib, name)(*args, None)


def route(T=4, E=8, k=2, logits=AT, renorm=1, ids=AT, weights=AT, offsets=AT, tokens=AT, slots=AT, space=AT, size=1 << 20):
    return st("polydl_route", T, E, k, logits, renorm, ids, weights, offsets, tokens, slots, space, size)


def test_route_refusals():
    for kw in ({"T": -1}, {"E": 0}, {"k": 0}, {"k": 9}, {"T": 65, "size": 8 * 4 - 1}):
        assert route(**kw) == DIM, kw
    for name in ("logits", "ids", "weights", "offsets", "tokens", "slots"):
        assert route(**{name: Z}) == NULL, name
        assert route(**{name: AT + 2}) == UNSUPPORTED, name
    assert route(T=65, space=Z) == NULL
    assert route(T=65, space=AT + 1) == UNSUPPORTED
    assert route(E=1025) == UNSUPPORTED and route(E=64, k=33) == UNSUPPORTED and route(T=BIG, k=2) == UNSUPPORTED
    assert route(T=0, offsets=Z) == NULL


def test_route_workspace():
    f = P.lib.polydl_route_workspace_bytes
    assert f(64, 8) == 0 and f(0, 8) == 0 and f(65, 0) == 0 and f(65, 1025) == 0
    # counts (a byte an expert and 64 tokens, rows of whole words), sums before each 64 and in all (a word each)
    assert f(65, 8) == 256 + (8 * 2 + 8) * 4
    assert f(64 * 1000 + 1, 256) == 256 * 1004 + (256 * 1001 + 256) * 4
    assert f(BIG, 1024) > 1 << 32


def test_route_bwd_refusals():
    def f(T=4, E=8, k=2, logits=AT, ids=AT, weights=AT, dweights=AT, renorm=1, dlogits=AT):
        return st("polydl_route_bwd", T, E, k, logits, ids, weights, dweights, renorm, dlogits)
    for kw in ({"T": -1}, {"E": 0}, {"k": 0}, {"k": 9}):
        assert f(**kw) == DIM, kw
    for kw in ({"ids": Z}, {"dweights": Z}, {"dlogits": Z}, {"weights": Z}, {"logits": Z, "renorm": 0}):
        assert f(**kw) == NULL, kw
    assert f(E=1025) == UNSUPPORTED and f(E=64, k=33) == UNSUPPORTED and f(dlogits=AT + 2) == UNSUPPORTED


def test_combine_refusals():
    def f(T=4, k=2, M=8, D=16, y=AT, slots=AT, weights=AT, out=AT, kind=1):
        return st("polydl_combine_bf16", T, k, M, D, y, slots, weights, out, kind)
    for kw in ({"T": -1}, {"k": 0}, {"M": -1}, {"D": 0}):
        assert f(**kw) == DIM, kw
    for kw in ({"y": Z}, {"slots": Z}, {"out": Z}):
        assert f(**kw) == NULL, kw
    for kw in ({"kind": 2}, {"kind": -1}, {"D": (1 << 24) + 1}, {"T": BIG}, {"y": AT + 1}, {"slots": AT + 2}, {"weights": AT + 2},
               {"out": AT + 1}, {"out": AT + 2, "kind": 0}):
        assert f(**kw) == UNSUPPORTED, kw

    def g(T=4, k=2, M=8, D=16, dout=AT, y=AT, slots=AT, weights=AT, dy=AT, dweights=AT):
        return st("polydl_combine_bwd_bf16", T, k, M, D, dout, y, slots, weights, dy, dweights)
    for kw in ({"T": -1}, {"k": 0}, {"M": -1}, {"D": 0}):
        assert g(**kw) == DIM, kw
    for kw in ({"dout": Z}, {"y": Z}, {"slots": Z}, {"dy": Z}):
        assert g(**kw) == NULL, kw
    for kw in ({"D": (1 << 24) + 1}, {"T": BIG}, {"dy": AT + 1}, {"dweights": AT + 2}):
        assert g(**kw) == UNSUPPORTED, kw


def fwd(E=2, M=8, N=16, K=24, offsets=AT, rows=Z, x_rows=8, x=AT, ldx=24, w=AT, y=AT, ldy=16, kind=1, act=0):
    return st("polydl_grouped_gemm_bf16", E, M, N, K, offsets, rows, x_rows, x, ldx, w, y, ldy, kind, act)


def dx(E=2, M=8, N=16, K=24, offsets=AT, dy=AT, lddy=16, w=AT, h=AT, ldh=24, act=1, out=AT, ldo=24, kind=1):
    return st("polydl_grouped_gemm_dx_bf16", E, M, N, K, offsets, dy, lddy, w, h, ldh, act, out, ldo, kind)


def dw(E=2, M=8, N=16, K=24, offsets=AT, dy=AT, lddy=16, rows=Z, x_rows=8, x=AT, ldx=24, out=AT, kind=0, acc=0):
    return st("polydl_grouped_gemm_dw_bf16", E, M, N, K, offsets, dy, lddy, rows, x_rows, x, ldx, out, kind, acc)


def w4(E=2, M=8, N=16, K=24, group=32, offsets=AT, rows=Z, x_rows=8, x=AT, ldx=24, q=AT, scales=AT, zeros=AT, y=AT, ldy=16, kind=1, act=0):
    return st("polydl_w4_gemm_bf16", E, M, N, K, group, offsets, rows, x_rows, x, ldx, q, scales, zeros, y, ldy, kind, act)


def test_product_refusals():
    for f in (fwd, dx, dw, w4):
        for kw in ({"E": 0}, {"M": -1}, {"N": 0}, {"K": 0}):
            assert f(**kw) == DIM, (f.__name__, kw)
        assert f(offsets=Z) == NULL and f(offsets=AT + 2) == UNSUPPORTED and f(kind=2) == UNSUPPORTED
    for f in (fwd, w4):
        for kw in ({"ldx": 23}, {"ldy": 15}, {"x_rows": 7}, {"x_rows": -1, "rows": AT}):
            assert f(**kw) == DIM, (f.__name__, kw)
        assert f(x=Z) == NULL and f(y=Z) == NULL
        for kw in ({"act": 3}, {"act": -1}, {"x": AT + 1}, {"rows": AT + 1}, {"y": AT + 2, "kind": 0}, {"ldx": 1 << 41}):
            assert f(**kw) == UNSUPPORTED, (f.__name__, kw)
    assert fwd(w=Z) == NULL and fwd(w=AT + 1) == UNSUPPORTED and fwd(E=BIG, N=BIG, K=BIG, ldx=BIG, ldy=BIG) == UNSUPPORTED
    for kw in ({"lddy": 15}, {"ldo": 23}, {"ldh": 23}):
        assert dx(**kw) == DIM, kw
    for kw in ({"dy": Z}, {"w": Z}, {"h": Z}, {"out": Z}):
        assert dx(**kw) == NULL, kw
    assert dx(act=3) == UNSUPPORTED and dx(h=AT + 1) == UNSUPPORTED
    for kw in ({"lddy": 15}, {"ldx": 23}, {"x_rows": 9}):
        assert dw(**kw) == DIM, kw
    for kw in ({"dy": Z}, {"x": Z}, {"out": Z}):
        assert dw(**kw) == NULL, kw
    assert dw(kind=1, acc=1) == UNSUPPORTED and dw(out=AT + 2) == UNSUPPORTED
    for kw in ({"q": Z}, {"scales": Z}):
        assert w4(**kw) == NULL, kw
    for kw in ({"group": 16}, {"group": 256}, {"q": AT + 8}, {"scales": AT + 4}, {"K": 0x7fffff01, "ldx": BIG}):
        assert w4(**kw) == UNSUPPORTED, kw


def test_pack_refusals():
    def f(E=1, N=16, K=24, group=32, w=AT, q=AT, scales=AT, zeros=AT):
        return st("polydl_w4_pack_bf16", E, N, K, group, w, q, scales, zeros)
    for kw in ({"E": 0}, {"N": 0}, {"K": 0}):
        assert f(**kw) == DIM, kw
    for kw in ({"w": Z}, {"q": Z}, {"scales": Z}):
        assert f(**kw) == NULL, kw
    for kw in ({"group": 48}, {"w": AT + 1}, {"q": AT + 8}, {"scales": AT + 4}):
        assert f(**kw) == UNSUPPORTED, kw


def test_valid_arguments_need_a_device():
    import torch
    if torch.cuda.is_available():
        pytest.skip("there is one")
    assert route() == NO_DEVICE and fwd() == NO_DEVICE and dx() == NO_DEVICE and dw() == NO_DEVICE and w4() == NO_DEVICE
    assert w4(E=1, offsets=Z, zeros=Z) == NO_DEVICE and dx(act=0, h=Z) == NO_DEVICE and dw(acc=1) == NO_DEVICE
    assert fwd(M=0, x_rows=0, x=Z, y=Z) == NO_DEVICE and route(T=0, logits=Z, ids=Z, weights=Z, tokens=Z, slots=Z, space=Z) == NO_DEVICE


def test_binding_refuses_host_tensors_and_types():
    import torch
    x, w, o = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(2, 16, 8, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(TypeError):
        P.grouped_gemm_bf16(x, w, o)
    with pytest.raises(TypeError):
        P.route(torch.zeros(4, 8), 2)
    with pytest.raises(TypeError):
        P.route(torch.zeros(4, 8, dtype=torch.float64), 2)
    with pytest.raises(ValueError):
        P.w4_gemm_bf16(x, torch.zeros(1, 1, 1, 64, 16, dtype=torch.uint8), torch.zeros(1, 1, 1, 16, dtype=torch.bfloat16), 16, 48)
    with pytest.raises(ValueError):
        P.grouped_gemm_dx_bf16(torch.zeros(4, 16, dtype=torch.bfloat16), w, o, act="relu")
    with pytest.raises(ValueError):
        P.grouped_gemm_dw_bf16(torch.zeros(5, 16, dtype=torch.bfloat16), x, o)
    assert P.w4_shapes(3, 17, 129, 32) == ((3, 2, 2, 64, 16), (3, 2, 8, 16))
