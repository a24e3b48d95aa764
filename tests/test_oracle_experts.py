"""Pins of the 64-bit definitions of the layer of experts: worked by hand, and gradients against differences."""
import numpy as np

from oracle import experts as ox


def test_route_by_hand():
    inf = np.inf
    x = np.array([[0.0, np.log(3.0), 0.0], [-inf, 2.0, -inf], [-inf, -inf, -inf], [1.0, 1.0, 1.0]])
    ids, w, offsets, tokens, slots = ox.route(x, 2, False)
    assert ids.tolist() == [[1, 0], [1, -1], [-1, -1], [0, 1]]
    assert np.allclose(w, [[0.6, 0.2], [1, 0], [0, 0], [1 / 3, 1 / 3]])
    assert offsets.tolist() == [0, 2, 5, 5] and tokens.tolist() == [0, 3, 0, 1, 3, -1, -1, -1]
    assert slots.tolist() == [[2, 0], [3, -1], [-1, -1], [1, 4]]
    assert np.allclose(ox.route(x, 2, True)[1], [[0.75, 0.25], [1, 0], [0, 0], [0.5, 0.5]])
    ids, w = ox.route(np.array([[inf, np.nan, 3.0]]), 2, True)[:2]
    assert ids.tolist() == [[1, 0]] and np.isnan(w).all()


def test_route_gradient_against_differences():
    r = np.random.RandomState(3)
    x, g = r.randn(5, 9), r.randn(5, 3)
    for renorm in (False, True):
        ids, w = ox.route(x, 3, renorm)[:2]
        d = ox.route_bwd(x, ids, w, g, renorm)
        for e in range(9):
            h = np.zeros_like(x)
            h[:, e] = 1e-6
            diff = ((ox.route(x + h, 3, renorm)[1] - ox.route(x - h, 3, renorm)[1]) * g).sum(1) / 2e-6
            assert np.abs(diff - d[:, e]).max() < 1e-8


def test_layout_by_hand():
    # one tile of 16 rows and 128 inputs: the code of row 3, input 77 = 64 + 13: word 2, block 1, value 5: nibble 2 + 4
    q = np.full((1, 1, 1, 64, 16), 0x88, np.uint8)
    q[0, 0, 0, 16 + 3, 2 * 4 + 3] = 0x8f
    s = np.ones((1, 1, 4, 16))
    s[0, 0, 2, 3] = 0.5
    w = ox.w4_weights(q, s, None, 16, 128, 32)
    assert w[0, 3, 77] == 3.5 and np.count_nonzero(w) == 1
