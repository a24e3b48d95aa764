"""The layer of experts on the GPU where it is easily wrong: equal logits of either sign, weights that no code can hold, results for
another stream, launches of more threads than one axis of a grid holds."""
import numpy as np
import pytest

from oracle import experts as ox

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2006_02230_amd as p
    return p


def gen(seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape):
    import torch
    return torch.randn(*shape, generator=g, device="cuda")


# ---- router ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("T,E,k", [(1, 5, 3), (130, 70, 8), (66, 600, 10)])
@pytest.mark.parametrize("renorm", [False, True])
def test_zeros_of_either_sign_are_equal_logits(P, T, E, k, renorm):
    import torch
    g = gen(E)
    x = torch.randint(-1, 2, (T, E), generator=g, device="cuda").float()
    x = torch.where(torch.rand(T, E, generator=g, device="cuda") < 0.5, -x, x)         # zeros of both signs
    x[0] = torch.where(torch.arange(E, device="cuda") % 2 == 0, -0.0, 0.0)
    assert bool((torch.signbit(x) & (x == 0)).any()) and bool((~torch.signbit(x) & (x == 0)).any())
    r = P.route(x, k, renorm=renorm)
    ids, w, offsets, tokens, slots = ox.route(x.cpu().numpy(), k, renorm)
    assert r.ids[0].tolist() == list(range(k))
    for got, want in zip((r.ids, r.offsets, r.tokens, r.slots), (ids, offsets, tokens, slots)):
        assert np.array_equal(got.cpu().numpy(), want)
    # a difference of logits of at most 2, exponentials, a sum, a quotient
    assert (np.abs(r.weights.cpu().numpy() - w) <= w * (2 * 2 + 8 + 16 + E / 64) * 2.0 ** -23).all()
