"""The oracle of what stands around a layer of experts: gradients against differences, values worked out by hand."""
import numpy as np

from oracle import block as ob


def differences(f, x, step=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        a, b = x.copy(), x.copy()
        a[i] += step
        b[i] -= step
        g[i] = (f(a) - f(b)) / (2 * step)
    return g


def test_layernorm_by_hand():
    y, mean, rstd = ob.layernorm(np.array([[1.0, 3.0]]), np.array([2.0, 2.0]), np.array([0.0, 1.0]), 0.0)
    assert mean[0] == 2 and rstd[0] == 1 and (y == [[-2.0, 3.0]]).all()


def test_layernorm_gradients_against_differences():
    r = np.random.default_rng(0)
    x, gamma, beta, dy = r.normal(size=(3, 7)), r.normal(size=7), r.normal(size=7), r.normal(size=(3, 7))
    _, mean, rstd = ob.layernorm(x, gamma, beta)
    dx, dg, db = ob.layernorm_bwd(dy, x, mean, rstd, gamma)
    assert np.allclose(dx, differences(lambda v: (ob.layernorm(v, gamma, beta)[0] * dy).sum(), x), atol=1e-7)
    assert np.allclose(dg, differences(lambda v: (ob.layernorm(x, v, beta)[0] * dy).sum(), gamma), atol=1e-7)
    assert np.allclose(db, differences(lambda v: (ob.layernorm(x, gamma, v)[0] * dy).sum(), beta), atol=1e-7)


def test_balance_by_hand():
    loss, counts, shares, rows = ob.balance(np.log([[0.5, 0.25, 0.25], [0.25, 0.5, 0.25]]), np.array([[0], [1]]))
    assert counts.tolist() == [1, 1, 0] and rows == 2 and np.allclose(shares, [0.375, 0.375, 0.25])
    assert np.isclose(loss, 3 * 0.375)
    # as even as can be: 1
    assert np.isclose(ob.balance(np.zeros((4, 4)), np.arange(4)[:, None])[0], 1)
    assert ob.balance(np.full((2, 3), -np.inf), np.full((2, 1), -1))[0] == 0


def test_balance_gradient_against_differences():
    r = np.random.default_rng(1)
    x, ids = r.normal(size=(5, 4)), r.integers(0, 4, (5, 2))
    x[3] = -np.inf
    _, counts, _, rows = ob.balance(x, ids)
    open_ = np.isfinite(x)

    def f(v):
        return ob.balance(np.where(open_, v, -np.inf), ids)[0]
    want = differences(f, np.where(open_, x, 0.0))
    assert np.allclose(ob.balance_bwd(x, counts, rows), want, atol=1e-8)


def test_clipping_by_hand():
    norm, (a, b) = ob.clipped([np.array([3.0]), np.array([[4.0]])], 1.0)
    assert norm == 5 and np.allclose(a, 0.6) and np.allclose(b, 0.8)
    assert (ob.clipped([np.array([3.0, np.inf])], 1.0)[1][0] == [3, np.inf]).all()


def test_mx4_by_hand():
    x = np.zeros((1, 40))
    x[0, :9] = [6, -5, 2.5, 0.25, 0.75, 1.25, 1.75, 3.5, -0.1]       # largest 6: scale 1, ties to the even code
    x[0, 32:34] = [7.9, 2.0 ** -10]                                   # saturates at 6, scale 1
    codes, scales = ob.mx4_codes(x)
    assert scales.tolist() == [[127, 127, 0, 0]]
    v = ob.mx4_values(ob.mx4_pack(codes), scales, 40)
    assert v[0, :9].tolist() == [6, -4, 2, 0, 1, 1, 2, 4, 0] and v[0, 32:34].tolist() == [6, 0]
    codes, scales = ob.mx4_codes(np.array([[2.0 ** -130, 2.0 ** -126]]))
    assert scales[0, 0] == 0 and codes[0, :2].tolist() == [0, 4]
    assert ob.mx4_codes(np.array([[1.0, np.nan]]))[1][0, 0] == 255
    assert np.isnan(ob.mx4_values(np.zeros((1, 64), np.uint8), np.array([[255, 0, 0, 0]], np.uint8))[0, :32]).all()
