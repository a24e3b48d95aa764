"""Layer norm, balance loss, gradient norm and clipping on the GPU against their definitions in 64 bits.

Tolerances: u = 2^-24 is half a step of float32 relative to the value, and a sum of n values in any order is off by at most (adds that a value
passes through) * u * the sum of magnitudes; each formula's own roundings are counted beside its test."""
import numpy as np
import pytest

from oracle import block as ob

pytestmark = pytest.mark.gpu
u = 2.0 ** -24


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


def kind(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def host(t):
    return t.double().cpu().numpy()


def half_step(name):
    """of the type a result is rounded to; float32's own roundings are counted in the formula"""
    return 2.0 ** -8 if name == "bf16" else 0.0


def strided(t, pad=5, first=0):
    """The same matrix with longer rows, the first value `first` elements into its memory."""
    import torch
    T, D = t.shape
    flat = torch.full((first + T * (D + pad),), 7.0, dtype=t.dtype, device=t.device)
    v = flat[first:].view(T, D + pad)[:, :D]
    v.copy_(t)
    return v


# ---- layer norm --------------------------------------------------------------------------------------------------

SHAPES = [(1, 1), (1, 7), (3, 8), (5, 63), (17, 128), (33, 129), (9, 512), (4, 513), (6, 1000), (2, 1024), (5, 1025), (3, 2048), (2, 2049), (5, 3000),
          (2, 4096), (3, 4097), (2, 8192), (3, 8193), (2, 16384), (2, 16385), (2, 40001), (700, 96), (300, 520)]


def adds(D):
    """A value of a row passes through at most: 4 units of 8 in a lane (more in rows past 16384), 6 adds of a wave, 16 of its workgroup."""
    return 64 + D // 128


def norm_bounds(x, gamma, beta, eps, want, y_name):
    """Bounds of y, mean, rstd.  The mean: adds(D) u mean|x|, and its quotient.  A centred value: the mean's error and its own rounding.  The
    variance: the mean's error enters squared (the centred values sum to zero), every square with three roundings.  rstd: half of it, sum, root,
    quotient.  y: three products and a sum."""
    D = x.shape[1]
    y, mean, rstd = want
    dm = (adds(D) + 2) * u * np.abs(x).mean(1)
    c = np.abs(x - mean[:, None])
    var = (c * c).mean(1)
    dv = (adds(D) + 8) * u * var + 2 * dm ** 2 + 4 * u * (c.mean(1) * dm)
    rel = 0.5 * dv / (var + eps) + 4 * u
    g = np.abs(gamma)
    dy = g * rstd[:, None] * (dm[:, None] + c * (rel[:, None] + 5 * u)) + 2 * u * (np.abs(beta) + np.abs(y))
    return dy + half_step(y_name) * (np.abs(y) + dy), dm, rstd * rel


@pytest.mark.parametrize("T,D", SHAPES)
@pytest.mark.parametrize("x_name,y_name", [("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32"), ("f32", "f32")])
def test_layernorm(P, T, D, x_name, y_name):
    g = gen(T * 1000 + D)
    x = (randn(g, T, D) * 2 + randn(g, T, 1) * 4).to(kind(x_name))
    gamma, beta = 1 + 0.2 * randn(g, D), 0.3 * randn(g, D)
    got = P.layernorm_fwd(x, gamma, beta, out_dtype=kind(y_name))
    assert got.y.dtype == kind(y_name) and got.mean.shape == got.rstd.shape == (T,)
    hx, hg, hb = host(x), host(gamma), host(beta)
    want = ob.layernorm(hx, hg, hb)
    for a, b, tol in zip(got, want, norm_bounds(hx, hg, hb, 1e-5, want, y_name)):
        assert (np.abs(host(a) - b) <= tol).all(), (np.abs(host(a) - b) / tol).max()


@pytest.mark.parametrize("T,D,first", [(4, 77, 1), (3, 700, 3), (3, 1500, 1), (2, 3001, 7), (2, 7001, 1), (2, 12001, 5), (2, 20001, 3)])
@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_layernorm_strides_and_missing_weights(P, T, D, first, name):
    import torch
    g = gen(D)
    x = randn(g, T, D).to(kind(name))
    xs = strided(x, 5, first)
    out = torch.full((T, D + 3), 9.0, dtype=kind(name), device="cuda")
    got = P.layernorm_fwd(xs, out=out[:, :D], eps=0.1)
    assert torch.equal(out[:, D:], torch.full_like(out[:, D:], 9.0))
    want = ob.layernorm(host(x), eps=0.1)
    for a, b, tol in zip(got, want, norm_bounds(host(x), 1.0, 0.0, 0.1, want, name)):
        assert (np.abs(host(a) - b) <= tol).all()
    assert torch.equal(P.layernorm_fwd(x, eps=0.1).y, out[:, :D])
    only = P.layernorm_fwd(x, gamma=torch.full((D,), 2.0, device="cuda"), eps=0.1, out_dtype=torch.float32).y
    both = P.layernorm_fwd(x, gamma=torch.full((D,), 2.0, device="cuda"), beta=torch.zeros(D, device="cuda"), eps=0.1, out_dtype=torch.float32).y
    assert torch.equal(only, both)


@pytest.mark.parametrize("D", [100, 1000, 3000, 9000, 20000])
def test_layernorm_of_a_large_mean_keeps_the_variance(P, D):
    # 4096 and a variance near 1: a difference of mean squares would lose it all
    g = gen(D)
    x = randn(g, 3, D) + 4096
    want = ob.layernorm(host(x))
    got = P.layernorm_fwd(x)
    for a, b, tol in zip(got, want, norm_bounds(host(x), 1.0, 0.0, 1e-5, want, "f32")):
        assert (np.abs(host(a) - b) <= tol).all()


def centred_bounds(x, gamma, beta, eps, want, y_name):
    """Bounds where the mean's own rounding must not reach y.  Whatever a first mean is off by, e <= (adds(D) + 2) u mean|x|, is among the values that it
    leaves, and so in their mean, which is formed of |c| + e and taken out: a centred value is off by (adds(D) + 3) u (mean|c| + e) for all alike and by two
    roundings of its own.  The variance, rstd and y follow as in norm_bounds; the mean is rounded once."""
    D = x.shape[1]
    y, mean, rstd = want
    e = (adds(D) + 2) * u * np.abs(x).mean(1)
    c = np.abs(x - mean[:, None])
    var = (c * c).mean(1)
    dc = (adds(D) + 3) * u * (c.mean(1) + e)
    rel = 0.5 * ((adds(D) + 10) * u * var + 2 * dc ** 2) / (var + eps) + 4 * u
    g = np.abs(gamma)
    dy = g * rstd[:, None] * (dc[:, None] + c * (rel[:, None] + 7 * u)) + 2 * u * (np.abs(beta) + np.abs(y))
    return dy + half_step(y_name) * (np.abs(y) + dy), u * np.abs(mean) + dc, rstd * rel


@pytest.mark.parametrize("D", [100, 128, 500, 1000, 2000, 3000, 7000, 12288, 16384, 20001, 70001])
@pytest.mark.parametrize("mean", [0.3, 4096.0, -50000.3, 1e6])
def test_layernorm_of_a_large_mean(P, D, mean):
    # a mean of up to a million times the spread; and rows whose first value, or one in the middle, is far larger than the others
    g = gen(D)
    x = randn(g, 5, D) + mean
    x[3, 0], x[4, D // 2] = 3e4, -3e4
    gamma, beta = 1 + 0.2 * randn(g, D), 0.3 * randn(g, D)
    want = ob.layernorm(host(x), host(gamma), host(beta))
    got = P.layernorm_fwd(x, gamma, beta)
    for a, b, tol in zip(got, want, centred_bounds(host(x), host(gamma), host(beta), 1e-5, want, "f32")):
        assert (np.abs(host(a) - b) <= tol).all(), (np.abs(host(a) - b) / tol).max()


@pytest.mark.parametrize("D", [1, 3, 100, 300, 1000, 1999, 3000, 4097, 12288, 16383, 20001, 300001])
@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_layernorm_of_equal_values_whose_sums_round(P, D, name):
    import torch
    x = torch.tensor([[0.1], [1000.7], [-4097.3], [50000.3], [1e-30], [3e30]], device="cuda").to(kind(name)).expand(6, D).contiguous()
    beta = randn(gen(D), D)
    f = P.layernorm_fwd(x, beta=beta, out_dtype=torch.float32)
    assert torch.equal(f.mean, x[:, 0].float()) and torch.equal(f.y, beta.expand(6, D))
    assert (np.abs(host(f.rstd) * 1e-5 ** 0.5 - 1) <= 4 * u).all()                # eps, rounded, its root and quotient
    none = P.layernorm_fwd(x, eps=0.0)
    assert bool(torch.isinf(none.rstd).all()) and bool(torch.isnan(none.y).all()) and torch.equal(none.mean, f.mean)


@pytest.mark.parametrize("D", [50, 600, 2500, 17000])
def test_broken_rows_stay_alone(P, D):
    import torch
    g = gen(D)
    x, dy = randn(g, 9, D), randn(g, 9, D)
    y = P.layernorm_fwd(x)
    dx = P.layernorm_bwd(dy, x, y.mean, y.rstd).dx
    bad = x.clone()
    bad[2, D // 2], bad[5, 0], bad[7, D - 1] = float("nan"), float("inf"), -float("inf")
    z = P.layernorm_fwd(bad)
    dz = P.layernorm_bwd(dy, bad, z.mean, z.rstd).dx
    broken = torch.zeros(9, dtype=torch.bool, device="cuda")
    broken[[2, 5, 7]] = True
    for got, was in ((z.y, y.y), (dz, dx)):
        assert bool(torch.isnan(got[broken]).any(1).all()) and torch.equal(got[~broken], was[~broken])


def grad_bounds(dy, x, mean, rstd, gamma, T, D, x_name):
    """h has two roundings and g one; the two means adds(D) and their products' roundings; dx five more.  The weights' sums: a value passes
    through at most T/64 + 64 adds, a term has four roundings."""
    h, g = np.abs((x - mean[:, None]) * rstd[:, None]), np.abs(dy * gamma)
    n = adds(D) + 12
    dx = rstd[:, None] * n * u * (g + g.mean(1, keepdims=True) + h * (g * h).mean(1, keepdims=True))
    m = (T / 64 + 64 + 5) * u
    return dx, m * (np.abs(dy) * h).sum(0), m * np.abs(dy).sum(0)


def check_gradients(P, dy, x, gamma, got, f, x_name, before=(0.0, 0.0)):
    want = ob.layernorm_bwd(host(dy), host(x), host(f.mean), host(f.rstd), 1.0 if gamma is None else host(gamma))
    T, D = x.shape
    tol = grad_bounds(host(dy), host(x), host(f.mean), host(f.rstd), 1.0 if gamma is None else host(gamma), T, D, x_name)
    dx_tol = tol[0] + half_step(x_name) * (np.abs(want[0]) + tol[0]) + u * np.abs(want[0])
    assert (np.abs(host(got.dx) - want[0]) <= dx_tol).all(), (np.abs(host(got.dx) - want[0]) / dx_tol).max()
    for a, b, t, was in zip(got[1:], want[1:], tol[1:], before):
        assert (np.abs(host(a) - (b + was)) <= t + u * np.abs(b + was)).all(), (np.abs(host(a) - (b + was)) / (t + 1e-30)).max()


@pytest.mark.parametrize("T,D", SHAPES + [(4100, 72), (1030, 600), (2100, 33), (900, 2050)])
@pytest.mark.parametrize("dy_name,x_name", [("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32"), ("f32", "f32")])
def test_layernorm_gradient(P, T, D, dy_name, x_name):
    g = gen(T * 1000 + D + 1)
    x, dy = (randn(g, T, D) * 2 + 1).to(kind(x_name)), randn(g, T, D).to(kind(dy_name))
    gamma = 1 + 0.2 * randn(g, D)
    f = P.layernorm_fwd(x, gamma)
    check_gradients(P, dy, x, gamma, P.layernorm_bwd(dy, x, f.mean, f.rstd, gamma), f, x_name)


@pytest.mark.parametrize("T,D,first", [(9, 77, 1), (130, 700, 3), (70, 3001, 7), (5, 20001, 3)])
@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_layernorm_gradient_strides_and_sums(P, T, D, first, name):
    import torch
    g = gen(D + 2)
    x, dy = randn(g, T, D).to(kind(name)), randn(g, T, D).to(kind(name))
    f = P.layernorm_fwd(x)
    out = torch.full((T, D + 3), 9.0, dtype=kind(name), device="cuda")
    dgamma, dbeta = randn(g, D), randn(g, D)
    before = host(dgamma), host(dbeta)
    got = P.layernorm_bwd(strided(dy, 3, first), strided(x, 5, first), f.mean, f.rstd, dx=out[:, :D], dgamma=dgamma, dbeta=dbeta, accumulate=True)
    assert got.dgamma is dgamma and torch.equal(out[:, D:], torch.full_like(out[:, D:], 9.0))
    check_gradients(P, dy, x, None, got, f, name, before)
    only = P.layernorm_bwd(dy, x, f.mean, f.rstd, weights=False)
    assert only.dgamma is None and only.dbeta is None and torch.equal(only.dx, out[:, :D])


def test_layernorm_without_rows(P):
    import torch
    x = torch.empty(0, 40, device="cuda")
    f = P.layernorm_fwd(x)
    assert f.y.shape == (0, 40) and f.mean.shape == (0,)
    got = P.layernorm_bwd(x, x, f.mean, f.rstd)
    assert got.dx.shape == (0, 40) and not got.dgamma.any() and not got.dbeta.any()
    kept = torch.ones(40, device="cuda"), torch.ones(40, device="cuda")
    P.layernorm_bwd(x, x, f.mean, f.rstd, dgamma=kept[0], dbeta=kept[1], accumulate=True)
    assert bool((kept[0] == 1).all()) and bool((kept[1] == 1).all())


def test_layernorm_of_equal_values(P):
    import torch
    x = torch.full((2, 300), 3.0, device="cuda")
    f = P.layernorm_fwd(x, beta=torch.arange(300.0, device="cuda"))
    assert bool((f.mean == 3).all()) and torch.equal(f.y, torch.arange(300.0, device="cuda").expand(2, 300))
    assert bool(torch.isinf(P.layernorm_fwd(x, eps=0.0).rstd).all())


def test_layernorm_against_differences(P):
    # the gradient of sum(y * dy), along a direction: the forward pass at both sides in float32, whose rounding (bound of y above, summed) is
    # divided by the step; the third derivative's term is below it at this step
    g = gen(9)
    T, D, step = 6, 257, 2.0 ** -7
    x, dy, v, gamma = randn(g, T, D), randn(g, T, D), randn(g, T, D), randn(g, D)
    f = P.layernorm_fwd(x, gamma)
    got = P.layernorm_bwd(dy, x, f.mean, f.rstd, gamma)
    a, b = (host(P.layernorm_fwd(x + s * step * v, gamma).y) for s in (1, -1))
    slope = ((a - b) * host(dy)).sum() / (2 * step)
    want = (host(got.dx) * host(v)).sum()
    hx = host(x)
    tol = 2 * (norm_bounds(hx, host(gamma), 0.0, 1e-5, ob.layernorm(hx, host(gamma)), "f32")[0] * np.abs(host(dy))).sum() / (2 * step)
    # third derivative: the oracle's own differences, in 64 bits, say how far they are from the gradient at this step
    c, d = (ob.layernorm(hx + s * step * host(v), host(gamma))[0] for s in (1, -1))
    exact = (ob.layernorm_bwd(host(dy), hx, host(f.mean), host(f.rstd), host(gamma))[0] * host(v)).sum()
    curve = abs(((c - d) * host(dy)).sum() / (2 * step) - exact)
    # x + step v is rounded to float32, too: u |x| / step of slope a value
    moved = (np.abs(host(got.dx)) * u * (np.abs(hx) + 1)).sum() / step
    assert abs(slope - want) <= tol + 1.01 * curve + moved + 1e-5 * abs(want)


# ---- balance loss ------------------------------------------------------------------------------------------------

BALANCE = [(1, 1, 1), (1, 5, 2), (3, 64, 4), (128, 16, 2), (129, 17, 3), (300, 70, 8), (700, 256, 8), (300, 257, 6), (200, 600, 10), (500, 1024, 32),
           (9000, 33, 2), (17000, 128, 1)]


def router(g, T, E, k, masked=True):
    """Logits with rows that are all masked, entries that are, and choices as the router makes them."""
    import torch
    x = 2 * randn(g, T, E)
    if masked:
        x = torch.where(torch.rand(T, E, generator=g, device="cuda") < 0.2, -torch.inf, x)
        x = torch.where(torch.rand(T, 1, generator=g, device="cuda") < 0.1, -torch.inf, x)
    top = x.topk(k, 1)
    return x.contiguous(), torch.where(top.values == -torch.inf, -1, top.indices).int()


def rel_p(x, E):
    """A probability: its distance from the largest logit, rounded (that times u), the exponential, a sum of E and a quotient."""
    with np.errstate(invalid="ignore"):
        far = np.where(np.isfinite(x), x, np.nan)
        reach = np.nan_to_num(np.nanmax(far, initial=-np.inf, where=np.isfinite(far)) - np.nanmin(far, initial=np.inf, where=np.isfinite(far)), posinf=0, neginf=0)
    return (2 * abs(reach) + 16 + 6 + E / 16) * 2 * u


@pytest.mark.parametrize("T,E,k", BALANCE)
@pytest.mark.parametrize("masked", [False, True])
def test_balance(P, T, E, k, masked):
    x, ids = router(gen(T + E), T, E, k, masked)
    got = P.balance(x, ids)
    loss, counts, shares, rows = ob.balance(host(x), ids.cpu().numpy())
    assert got.loss.shape == got.rows.shape == ()
    assert int(got.rows) == rows and np.array_equal(got.counts.cpu().numpy(), counts)
    rel = rel_p(host(x), E) + (T / 64 + 100) * u           # sums over rows: a lane's, 4 of a wave, the waves', the workgroups'
    assert (np.abs(host(got.shares) - shares) <= rel * shares + 1e-37).all()
    assert abs(float(got.loss) - loss) <= (rel + 4 * u) * loss


@pytest.mark.parametrize("T,E,k", BALANCE)
def test_balance_gradient(P, T, E, k):
    import torch
    g = gen(T + E + 1)
    x, ids = router(g, T, E, k)
    b = P.balance(x, ids)
    dloss = torch.rand(1, generator=g, device="cuda")
    want = ob.balance_bwd(host(x), b.counts.cpu().numpy(), int(b.rows), float(dloss))
    p, _ = ob.probabilities(host(x))
    f = host(b.counts) / max(1.0, host(b.counts).sum())
    # p's own error, the sums of counts and of p f, five products
    tol = (rel_p(host(x), E) * 2 + (E / 16 + 32) * u) * float(dloss) * E / max(1, int(b.rows)) * p * (f + (p @ f)[:, None]) + 1e-37
    got = P.balance_bwd(x, b.counts, b.rows, dloss)
    assert (np.abs(host(got) - want) <= tol).all()
    assert torch.equal(got, P.balance_bwd(x, b.counts, b.rows, dloss[0]))
    before = randn(g, T, E)
    total = P.balance_bwd(x, b.counts, b.rows, dloss, out=before.clone(), accumulate=True)
    assert torch.equal(total, before + got)
    half = P.balance_bwd(x, b.counts, b.rows, 0.5)
    assert (np.abs(host(half) * 2 * float(dloss) - want) <= tol + 4 * u * np.abs(want)).all()


@pytest.mark.parametrize("T,E,scale", [(5, 8, 1), (300, 6, 1), (70, 300, 1 << 20)])
def test_balance_gradient_of_even_use(P, T, E, scale):
    # evenly used experts: no gradient, not what roundings leave of one; and with one choice more each for a few, all of its digits
    import torch
    x = randn(gen(E), T, E)
    rows = torch.tensor(T, dtype=torch.int32, device="cuda")
    counts = torch.full((E,), 40 * scale, dtype=torch.int32, device="cuda")
    assert not P.balance_bwd(x, counts, rows).any()
    counts[::3] += 1
    got, p = host(P.balance_bwd(x, counts, rows)), ob.probabilities(host(x))[0]
    f = host(counts) / host(counts).sum() - 1 / E
    # p's own error, a sum of E, five products
    tol = (rel_p(host(x), E) * 2 + (E / 16 + 32) * u) * E / T * p * (np.abs(f) + (p @ np.abs(f))[:, None])
    assert (np.abs(got - ob.balance_bwd(host(x), counts.cpu().numpy(), T)) <= tol + 1e-15 * p * E / T).all()


def test_balance_without_rows_or_choices(P):
    import torch
    empty = P.balance(torch.empty(0, 6, device="cuda"), torch.empty(0, 2, dtype=torch.int32, device="cuda"))
    assert float(empty.loss) == 0 and int(empty.rows) == 0 and not empty.counts.any() and not empty.shares.any()
    assert P.balance_bwd(torch.empty(0, 6, device="cuda"), empty.counts, empty.rows).shape == (0, 6)
    for T in (5, 300):
        x = torch.full((T, 6), -torch.inf, device="cuda")
        b = P.balance(x, torch.full((T, 2), -1, dtype=torch.int32, device="cuda"))
        assert float(b.loss) == 0 and int(b.rows) == 0 and not b.counts.any() and not b.shares.any()
        assert not P.balance_bwd(x, b.counts, b.rows).any()


def test_balance_ids_that_are_none(P):
    import torch
    x = torch.zeros(400, 5, device="cuda")
    ids = torch.tensor([[0, -1], [5, 1], [1, 1 << 30], [-(1 << 31), 4]], dtype=torch.int32, device="cuda").repeat(100, 1)
    b = P.balance(x, ids)
    assert b.counts.tolist() == [100, 200, 0, 0, 100] and abs(float(b.loss) - 1) <= 400 * u


@pytest.mark.parametrize("T", [7, 600])
def test_balance_broken_logits(P, T):
    import torch
    x, ids = router(gen(T), T, 20, 2, False)
    good = P.balance_bwd(x, *P.balance(x, ids)[1::2])
    for bad in (float("nan"), float("inf")):
        y = x.clone()
        y[3, 4] = bad
        b = P.balance(y, ids)
        assert bool(torch.isnan(b.loss)) and bool(torch.isnan(b.shares).all()) and int(b.rows) == T
        d = P.balance_bwd(y, b.counts, b.rows)
        assert bool(torch.isnan(d[3]).all()) and torch.equal(d[4:], good[4:]) and torch.equal(d[:3], good[:3])


# ---- gradient norm and clipping ----------------------------------------------------------------------------------

def tensors(g, sizes, mixed=True):
    import torch
    return [(randn(g, n) * 10.0 ** (i % 4 - 2)).to(torch.bfloat16 if mixed and i % 3 == 1 else torch.float32) for i, n in enumerate(sizes)]


SIZES = [[1], [7, 0, 9], [8192], [8193, 1, 8191], [100000, 3, 77777, 0, 12], [i * 37 % 501 for i in range(250)], [5] * 120, [5] * 121, [1 << 22, 5],
         [40000 + i for i in range(241)]]


def name_of(t):
    import torch
    return "f32" if t.dtype == torch.float32 else "bf16"


@pytest.mark.parametrize("case", range(len(SIZES)))
@pytest.mark.parametrize("ratio", [0.25, 1.5])
@pytest.mark.parametrize("in_place", [False, True])
def test_clipping(P, case, ratio, in_place):
    import torch
    grads = tensors(gen(case), SIZES[case])
    before = [host(t) for t in grads]
    norm = ob.total_norm(before)
    max_norm = ratio * norm
    _, want = ob.clipped(before, max_norm)
    assert abs(float(P.grad_norm(grads)) - norm) <= 1.01 * u * norm          # summed in 64 bits, rounded once
    out = None if in_place else [torch.full_like(t, 9.0) for t in grads]
    got = P.clip_grads(grads, max_norm, out=out)
    assert got.shape == () and abs(float(got) - norm) <= 1.01 * u * norm
    for t, w, b, o in zip(grads, want, before, grads if in_place else out):
        # rounded to float32, then to the tensor's type
        assert (np.abs(host(o) - w) <= np.abs(w) * (1.01 * u + 1.01 * half_step(name_of(t))) + 1e-44).all()
        if not in_place:
            assert np.array_equal(host(t), b)
        if ratio > 1:
            assert np.array_equal(host(o), b)


def nearest_bf16(w):
    """64-bit values to the nearest bfloat16 ones, ties to even."""
    step = np.exp2(np.maximum(np.frexp(w)[1] - 1, -126) - 7.0)
    return np.round(w / step) * step


@pytest.mark.parametrize("n", [3, 8192, 20000])
@pytest.mark.parametrize("scale", [0, -100, -126, -130])
def test_clipping_rounds_once(P, n, scale):
    # products just beside the middle of two bfloat16 values, nearer to it than a float32 value is: one that is rounded to float32 on its way falls on the
    # middle, and then on the even side of it.  Down to values below the normal ones, whose steps are equal.
    import torch
    wrong = 0
    for i in range(12):
        x = (1.5 + (2 * i + 1) / 128) * 2.0 ** scale
        x = float(nearest_bf16(np.array([x]))[0])
        low = nearest_bf16(np.array([x * (0.55 + 0.03 * i)]))[0]
        step = 2.0 ** (max(np.frexp(low)[1] - 1, -126) - 7)
        even = round(low / step) % 2 == 0                    # then the middle above goes down, and what is just above it must not
        t = (low + step / 2) * (1 + (1 if even else -1) * 2.0 ** -27)
        grad = torch.full((n,), x, dtype=torch.float64, device="cuda").bfloat16()
        grad[1::2] *= -1
        assert float(grad[0]) == x
        before = host(grad)
        f = t / x
        assert f < 1
        out = torch.zeros_like(grad)
        P.clip_grads([grad], f * ob.total_norm([before]), out=[out])
        want = before * f
        assert np.array_equal(nearest_bf16(want), np.sign(before) * (low + step * even))
        assert np.array_equal(host(out), nearest_bf16(want)), (x, f)
        wrong += int((host(torch.from_numpy(want).float().bfloat16()) != host(out)).any())
    assert wrong == 12                                       # (the cases are such)


def test_clipping_any_alignment_and_order(P):
    import torch
    g = gen(3)
    flat = [randn(g, 60001), randn(g, 60001).bfloat16()]
    grads = [f[a:a + n] for f in flat for a, n in ((1, 9001), (9003, 17), (9025, 40000))] + [randn(g, 300, 50).t(), randn(g, 6, 5, 4).permute(1, 2, 0)]
    kept = [f.clone() for f in flat]
    before = [host(t) for t in grads]
    norm, want = ob.clipped(before, 3.0)
    assert abs(float(P.clip_grads(grads, 3.0)) - norm) <= 1.01 * u * norm
    for t, w in zip(grads, want):
        assert (np.abs(host(t) - w) <= np.abs(w) * (1.01 * u + 1.01 * half_step(name_of(t)))).all()
    for f, k in zip(flat, kept):
        for a, b in ((0, 1), (9002, 9003), (9020, 9025), (49025, 60001)):
            assert torch.equal(f[a:b], k[a:b])


def test_clipping_values_whose_squares_do_not_fit(P):
    import torch
    for scale in (1e38, 1e-30):
        grads = [torch.full((1000,), scale, device="cuda"), torch.full((24,), -scale, device="cuda")]
        norm = float(P.clip_grads(grads, scale))
        want = 32.0 * float(torch.tensor(scale))
        assert abs(norm - want) <= 4 * u * want if want < 3e38 else norm == float("inf")
        assert bool(((grads[0] * 32 / scale - 1).abs() < 1e-6).all()) and bool(((grads[1] * 32 / scale + 1).abs() < 1e-6).all())


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_clipping_leaves_broken_gradients(P, bad):
    import torch
    grads = tensors(gen(5), [500, 9000, 30])
    grads[1][8999] = bad
    before = [t.clone() for t in grads]
    out = [torch.zeros_like(t) for t in grads]
    norm = P.clip_grads(grads, 1.0)
    assert not bool(torch.isfinite(norm)) and not bool(torch.isfinite(P.clip_grads(grads, 1.0, out=out)))
    for t, b, o in zip(grads, before, out):
        assert torch.equal(t.view(-1).view(torch.uint8), b.view(torch.uint8)) and torch.equal(o.view(torch.uint8), b.view(torch.uint8))


def test_clipping_to_zero_and_of_zeros(P):
    import torch
    grads = [torch.ones(100, device="cuda"), torch.zeros(7, device="cuda")]
    assert float(P.clip_grads(grads, 0.0)) == 10 and not grads[0].any()
    assert float(P.clip_grads(grads, 1.0)) == 0 and float(P.grad_norm([torch.empty(0, device="cuda")])) == 0


def test_clipping_refuses_tensors_that_overlap(P):
    import torch
    t = torch.ones(100, device="cuda")
    other = torch.ones(100, device="cuda")
    for grads, out in (([t, t], None), ([t[:60], t[50:]], None), ([t[:50], other[:50]], [t[10:60], other[50:]]), ([t, other], [other, t]),
                       ([t[:50], t[50:]], [t[50:], t[:50]]), ([t, other], [t, t])):
        with pytest.raises(P.PolydlError, match="polydl_clip_grads"):
            P.clip_grads(grads, 1.0, out=out)
    assert bool((t == 1).all()) and bool((other == 1).all())
    assert abs(float(P.grad_norm([t, t])) - 200 ** 0.5) < 1e-5
    halves = torch.empty(200, device="cuda")
    P.clip_grads([t, t], 200 ** 0.5 / 2, out=[halves[:100], halves[100:]])
    assert bool(((halves - 0.5).abs() < 1e-6).all())


# ---- all of them: graphs, streams, binding -----------------------------------------------------------------------

def test_captured_and_replayed(P):
    import torch
    g = gen(11)
    T, D, E = 700, 1100, 40
    x, dy, gamma = randn(g, T, D).bfloat16(), randn(g, T, D).bfloat16(), randn(g, D)
    logits, ids = router(g, T, E, 3)
    grads = tensors(g, [70000, 500, 9000])
    source = [t.clone() for t in grads]

    def run():
        f = P.layernorm_fwd(x, gamma)
        b = P.balance(logits, ids)
        return (*f, *P.layernorm_bwd(dy, x, f.mean, f.rstd, gamma), *b, P.balance_bwd(logits, b.counts, b.rows, b.loss), P.grad_norm(grads),
                P.clip_grads(grads, 1.0), P.grad_norm(grads))
    run()
    torch.cuda.synchronize()
    for t, s in zip(grads, source):
        t.copy_(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run()
    for seed in range(4):
        x.copy_(randn(gen(seed), T, D))
        logits.copy_(router(gen(seed), T, E, 3)[0])
        for t, s in zip(grads, source):
            t.copy_(s * (seed + 1))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        clipped = [t.clone() for t in grads]
        for t, s in zip(grads, source):
            t.copy_(s * (seed + 1))
        for a, b in zip(got, run()):
            assert torch.equal(a, b)
        for a, b in zip(clipped, grads):
            assert torch.equal(a, b)


def test_another_stream(P):
    import torch
    g = gen(12)
    T, D, E = 300, 520, 24
    x, dy, gamma = randn(g, T, D), randn(g, T, D).bfloat16(), randn(g, D)
    logits, ids = router(g, T, E, 2)
    grads = tensors(g, [70000, 500])
    side = torch.cuda.Stream()

    def run(stream):
        f = P.layernorm_fwd(x, gamma, stream=stream)
        b = P.balance(logits, ids, stream=stream)
        mine = [t.clone() for t in grads]
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        n = P.clip_grads(mine, 1.0, stream=stream)
        return [*f, *P.layernorm_bwd(dy, x, f.mean, f.rstd, gamma, stream=stream), *b, P.balance_bwd(logits, b.counts, b.rows, stream=stream), n,
                P.grad_norm(grads, stream=stream), *mine]
    want = run(None)
    torch.cuda.synchronize()
    got = run(side)
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_results_do_not_depend_on_the_run(P):
    import torch
    g = gen(13)
    x, dy = randn(g, 5000, 700), randn(g, 5000, 700)
    logits, ids = router(g, 9000, 50, 4)
    f = P.layernorm_fwd(x)
    first = None
    for _ in range(5):
        now = [*P.layernorm_bwd(dy, x, f.mean, f.rstd), *P.balance(logits, ids), P.grad_norm([x, dy])]
        first = first or [t.clone() for t in now]
        assert all(torch.equal(a, b) for a, b in zip(now, first))


def test_gradients_that_would_be_lost_are_refused(P):
    import torch
    x = torch.randn(4, 8, device="cuda", requires_grad=True)
    y = torch.randn(4, 8, device="cuda")
    w = torch.ones(8, device="cuda", requires_grad=True)
    ids = torch.zeros(4, 1, dtype=torch.int32, device="cuda")
    for call in (lambda: P.layernorm_fwd(x), lambda: P.layernorm_fwd(y, gamma=w), lambda: P.layernorm_fwd(y, beta=w), lambda: P.balance(x, ids),
                 lambda: P.grad_norm([y, x]), lambda: P.clip_grads([x], 1.0)):
        with pytest.raises(RuntimeError, match="requires its gradient"):
            call()
        with torch.no_grad():
            call()
