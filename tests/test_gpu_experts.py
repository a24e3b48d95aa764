"""The layer of experts on the GPU against its definitions in 64 bits: the router and its plan, the products grouped by expert in
three directions, the weighted sum, the products with 4-bit weights.

Tolerances count roundings.  A float32 sum on the matrix cores of R products passes R/32 + 1 instructions that add 32 products
each: at most R/32 + 33 roundings of 2^-23 of the sum of the terms' magnitudes; a bfloat16 result is off by 2^-8 of itself more."""
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


def ints(v):
    import torch
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def close(got, want, mag, reduction, what=""):
    """got within the roundings of a sum of `reduction` terms whose magnitudes sum to mag, and of its own type."""
    import torch
    tol = mag * ((reduction / 32 + 33) * 2.0 ** -23)
    if got.dtype == torch.bfloat16:
        tol = tol * (1 + 2.0 ** -8) + want.abs() * 2.0 ** -8
    else:
        tol = tol + want.abs() * 2.0 ** -24
    off = (got.double() - want).abs()
    assert got.shape == want.shape
    assert not torch.isnan(got).any(), what
    bad = off > tol
    assert not bad.any(), (what, int(bad.sum()), float((off - tol).max()), bad.nonzero()[:4].tolist())


# ---- router ------------------------------------------------------------------------------------------------------

def check_route(P, x, k, renorm):
    import torch
    r = P.route(x, k, renorm=renorm)
    ids, w, offsets, tokens, slots = ox.route(x.cpu().numpy(), k, renorm)
    assert np.array_equal(r.ids.cpu().numpy(), ids)
    assert np.array_equal(r.offsets.cpu().numpy(), offsets)
    assert np.array_equal(r.tokens.cpu().numpy(), tokens)
    assert np.array_equal(r.slots.cpu().numpy(), slots)
    got = r.weights.cpu().numpy().astype(np.float64)
    # a difference of logits, two exponentials (2 roundings each and one of the difference, times up to its size), a sum, a quotient
    size = np.nanmax(np.where(np.isinf(x.cpu().numpy()), np.nan, np.abs(x.cpu().numpy())), initial=1.0)
    E = x.shape[1]
    assert np.array_equal(np.isnan(got), np.isnan(w))
    assert np.nanmax(np.abs(got - w) / np.maximum(w, 1e-30), initial=0.0) <= (2 * size + 8 + 16 + E / 64) * 2.0 ** -23
    return r


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 64, 4), (63, 7, 7), (64, 65, 8), (65, 8, 2), (128, 128, 6), (200, 130, 32), (333, 257, 3),
                                   (70, 600, 10), (64, 1024, 32), (1027, 1000, 5), (4097, 16, 2)])
@pytest.mark.parametrize("renorm", [False, True])
def test_route(P, T, E, k, renorm):
    check_route(P, randn(gen(T + E), T, E) * 2, k, renorm)


def test_route_long_batches(P):
    # many workgroups: the counts added up by every one of them, and by a launch of its own (more than 32 MB to read again)
    import torch
    for T, E, k in ((16000, 64, 2), (16400, 1024, 2), (70000, 33, 1)):
        x = randn(gen(T), T, E)
        r = P.route(x, k)
        ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k]
        assert torch.equal(r.ids, ids.int())
        offsets, tokens, slots = ox.plan(ids.cpu().numpy(), E)
        assert np.array_equal(r.offsets.cpu().numpy(), offsets) and np.array_equal(r.tokens.cpu().numpy(), tokens)
        assert np.array_equal(r.slots.cpu().numpy(), slots)


@pytest.mark.parametrize("T,E,k", [(1, 3, 2), (130, 70, 8), (300, 9, 9)])
def test_route_ties_masks_and_nan(P, T, E, k):
    import torch
    g = gen(5)
    ties = torch.randint(-2, 3, (T, E), generator=g, device="cuda").float()
    check_route(P, ties, k, True)
    masked = torch.where(torch.rand(T, E, generator=g, device="cuda") < 0.7, -float("inf"), ties)
    masked[T // 2] = -float("inf")                                     # a row without an open expert
    for renorm in (False, True):
        check_route(P, masked, k, renorm)
    check_route(P, torch.full((T, E), -float("inf"), device="cuda"), k, False)
    lowest = torch.full((T, E), torch.finfo(torch.float32).min, device="cuda")   # not masked: equal logits
    r = P.route(lowest, k)
    assert torch.equal(r.ids, torch.arange(k, device="cuda").int().expand(T, k)) and torch.allclose(r.weights, torch.full_like(r.weights, 1 / k))
    odd = ties.clone()
    odd[0, E // 2] = float("nan")
    odd[T - 1, E - 1] = float("inf")
    r = P.route(odd, k)
    ids, w = ox.route(odd.cpu().numpy(), k, True)[:2]
    assert np.array_equal(r.ids.cpu().numpy(), ids) and np.array_equal(np.isnan(r.weights.cpu().numpy()), np.isnan(w))


def test_route_nothing(P):
    import torch
    r = P.route(torch.empty(0, 5, device="cuda"), 2)
    assert r.offsets.tolist() == [0] * 6 and r.ids.shape == (0, 2) and r.tokens.numel() == 0


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (5, 8, 3), (67, 64, 8), (131, 100, 4), (40, 300, 16), (33, 700, 2), (9, 1024, 32)])
@pytest.mark.parametrize("renorm", [False, True])
def test_route_gradient(P, T, E, k, renorm):
    import torch
    g = gen(E)
    x, d = randn(g, T, E) * 2, randn(g, T, k)
    x = torch.where(torch.rand(T, E, generator=g, device="cuda") < 0.3, -float("inf"), x)
    x[T // 2] = -float("inf")
    r = P.route(x, k, renorm=renorm)
    got = P.route_bwd(x, r.ids, r.weights, d, renorm=renorm).cpu().numpy().astype(np.float64)
    want = ox.route_bwd(x.cpu().numpy(), r.ids.cpu().numpy(), r.weights.cpu().numpy().astype(np.float64), d.cpu().numpy().astype(np.float64), renorm)
    # p is off by the roundings of test_route's weights, the bracket by those of a sum of k products
    scale = np.abs(d.cpu().numpy()).max() * (2 * 10 + 24 + E / 64 + 2 * k) * 2.0 ** -23
    assert np.abs(got - want).max() <= 2 * scale
    assert not np.isnan(got).any()


def test_route_gradient_against_differences(P):
    import torch
    g = gen(11)
    x, d = randn(g, 6, 10), randn(g, 6, 3)
    for renorm in (False, True):
        r = P.route(x, 3, renorm=renorm)
        got = P.route_bwd(x, r.ids, r.weights, d, renorm=renorm).cpu().numpy()
        for e in range(10):
            h = np.zeros((6, 10))
            h[:, e] = 1e-6
            xs = x.cpu().numpy().astype(np.float64)
            diff = ((ox.route(xs + h, 3, renorm)[1] - ox.route(xs - h, 3, renorm)[1]) * d.cpu().numpy()).sum(1) / 2e-6
            assert np.abs(diff - got[:, e]).max() < 1e-5


# ---- weighted sum ------------------------------------------------------------------------------------------------

def some_plan(T, E, k, seed, drop=0.0):
    """ids, offsets, tokens, slots, with a share of the choices dropped."""
    r = np.random.RandomState(seed)
    ids = np.argsort(r.rand(T, E), axis=1)[:, :k]
    ids = np.where(r.rand(T, k) < drop, -1, ids)
    return (ids,) + ox.plan(ids, E)


@pytest.mark.parametrize("T,E,k,D", [(1, 1, 1, 1), (1, 8, 8, 4096), (5, 6, 3, 7), (130, 9, 2, 64), (33, 16, 9, 1001), (257, 4, 4, 2056), (3, 40, 32, 2500)])
@pytest.mark.parametrize("weighted", [True, False])
def test_combine(P, T, E, k, D, weighted):
    import torch
    g = gen(D)
    _, offsets, tokens, slots = some_plan(T, E, k, T, drop=0.2)
    M = T * k
    y = randn(g, M, D).bfloat16()
    y[offsets[E]:] = float("nan")                                      # slots of no token are not read
    w = randn(g, T, k) if weighted else None
    s = torch.tensor(slots, device="cuda")
    rows = torch.where(s[:, :, None] >= 0, y.double()[s.clamp(min=0)], 0.0)
    terms = rows * (w.double().unsqueeze(2) if weighted else 1.0)
    for dtype in (torch.bfloat16, torch.float32):
        close(P.combine_bf16(y, ints(slots), w, out_dtype=dtype), terms.sum(1), terms.abs().sum(1), k, dtype)


@pytest.mark.parametrize("T,E,k,D", [(1, 1, 1, 1), (1, 8, 8, 4096), (5, 6, 3, 7), (130, 9, 2, 64), (33, 16, 9, 1001), (3, 40, 32, 2500)])
def test_combine_gradient(P, T, E, k, D):
    import torch
    g = gen(D + 1)
    _, offsets, tokens, slots = some_plan(T, E, k, T, drop=0.2)
    M = T * k
    y, d, w = randn(g, M, D).bfloat16(), randn(g, T, D).bfloat16(), randn(g, T, k)
    y[offsets[E]:] = float("nan")
    s = torch.tensor(slots, device="cuda")
    there = s >= 0
    before = torch.full((M, D), 7.0, dtype=torch.bfloat16, device="cuda")
    dy, dwt = P.combine_bwd_bf16(d, y, ints(slots), w, dy=before.clone())
    want = before.double().clone()
    want[s[there]] = (d.double().unsqueeze(1) * w.double().unsqueeze(2))[there]
    off = (dy.double() - want).abs()                                   # a product, rounded to 32 bits and to 16
    assert not (off > want.abs() * (2.0 ** -8 + 2.0 ** -23)).any()
    terms = torch.where(there[:, :, None], y.double()[s.clamp(min=0)], 0.0) * d.double().unsqueeze(1)
    tol = terms.abs().sum(2) * ((D / 128 + 16) * 2.0 ** -24 * 2)       # per lane two sums of D/512 times 4 products, then a tree
    assert not ((dwt.double() - terms.sum(2)).abs() > tol + 1e-30).any()
    # differences: the weights enter linearly, so a step of 1 is exact up to the roundings
    step = (P.combine_bf16(y, ints(slots), w + 1, out_dtype=torch.float32) - P.combine_bf16(y, ints(slots), w, out_dtype=torch.float32)).double()
    total = (step * d.double()).sum()
    scale = (torch.where(there[:, :, None], y.double()[s.clamp(min=0)].abs(), 0.0) * (2 * w.double().abs() + 1).unsqueeze(2)).sum(1)
    assert abs(total - dwt.double().sum()) <= ((scale * d.double().abs()).sum() * (k + 2) + tol.sum() * 2 ** 24) * 2.0 ** -23


# ---- products grouped by expert ------------------------------------------------------------------------------------

# rows of each group, slots behind the last one, N, K
SHAPES = [
    ((1,), 0, 1, 1), ((1,), 0, 8, 8), ((0, 1, 0), 0, 16, 64), ((5, 0, 17, 3), 2, 40, 72), ((64, 1, 63), 0, 128, 64), ((200, 130, 0, 7), 9, 264, 136),
    ((3, 2), 1, 77, 53), ((150, 0, 41), 5, 129, 67), ((300, 513), 0, 512, 320), ((257, 700, 1), 40, 300, 520), ((0, 0, 0), 6, 32, 32),
    (tuple(i % 5 for i in range(150)), 3, 48, 136), ((1000,), 0, 256, 1032), ((31, 33, 32, 16, 15, 17), 0, 200, 1000),
]


def ragged(counts, tail):
    offsets = np.concatenate([[0], np.cumsum(counts)])
    return offsets, int(offsets[-1]) + tail


def rows_for(M, src, offsets, seed):
    """Rows of a source for each slot, some of them none, all of it none behind the last group."""
    r = np.random.RandomState(seed)
    rows = r.randint(0, src, M)
    rows[r.rand(M) < 0.1] = -1
    if M > 2:
        rows[M // 2] = src + 3
    rows[offsets[-1]:] = -1
    return rows


def reference_rows(x, rows):
    import torch
    if rows is None:
        return x.double()
    idx = torch.tensor(rows, device="cuda")
    ok = (idx >= 0) & (idx < x.shape[0])
    return torch.where(ok[:, None], x.double()[torch.where(ok, idx, 0)], 0.0)


def strided(t, extra, shift=0):
    """The same matrix with a longer row, NaN between the rows, `shift` elements into its memory."""
    import torch
    r, c = t.shape
    flat = torch.full((r * (c + extra) + shift + 8,), float("nan"), dtype=t.dtype, device=t.device)
    v = flat[shift:shift + r * (c + extra)].view(r, c + extra)[:, :c]
    v.copy_(t)
    return v


def views(t, how):
    return t if how == "dense" else strided(t, 8 if t.shape[1] % 8 == 0 else 3) if how == "strided" else strided(t, 5, 1)


@pytest.mark.parametrize("how", ["dense", "strided", "odd"])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("counts,tail,N,K", SHAPES, ids=[str(i) for i in range(len(SHAPES))])
def test_grouped_forward(P, counts, tail, N, K, gather, how):
    import torch
    E = len(counts)
    offsets, M = ragged(counts, tail)
    g = gen(M + N)
    src = max(1, M // 2) if gather else M
    x = randn(g, src, K).bfloat16()
    w = (randn(g, E, N, K) * K ** -0.5).bfloat16()
    rows = rows_for(M, src, offsets, 1) if gather else None
    xs = reference_rows(x, rows)
    for e in range(E):
        if counts[e] == 0:
            w[e] = float("nan")                                        # experts without rows are not read into a result
    if not gather and tail:
        x[offsets[-1]:] = float("nan")
    want, mag = torch.zeros(M, N, dtype=torch.float64, device="cuda"), torch.zeros(M, N, dtype=torch.float64, device="cuda")
    for e in range(E):
        a, b = offsets[e], offsets[e + 1]
        if b > a:
            want[a:b] = xs[a:b] @ w[e].double().T
            mag[a:b] = xs[a:b].abs() @ w[e].double().abs().T
    act, dtype = ((None, torch.float32), ("relu", torch.bfloat16), ("relu6", torch.float32))[(M + N) % 3]
    ref = want if act is None else want.clamp(min=0) if act == "relu" else (want * 1).clamp(0, 6)
    out = torch.full((M, N + 4), -3.0, dtype=dtype, device="cuda")
    view = out[:, :N] if how != "dense" else None
    got = P.grouped_gemm_bf16(views(x, how), w, ints(offsets), rows=None if rows is None else ints(rows), act=act, out=view, out_dtype=dtype)
    close(got, ref, mag, K, (act, dtype))
    if view is not None:
        assert bool((out[:, N:] == -3.0).all())
    again = P.grouped_gemm_bf16(views(x, how), w, ints(offsets), rows=None if rows is None else ints(rows), act=act, out_dtype=dtype)
    assert torch.equal(again, got)


@pytest.mark.parametrize("how", ["dense", "strided", "odd"])
@pytest.mark.parametrize("act", [None, "relu", "relu6"])
@pytest.mark.parametrize("counts,tail,N,K", SHAPES, ids=[str(i) for i in range(len(SHAPES))])
def test_grouped_gradient_of_rows(P, counts, tail, N, K, act, how):
    import torch
    E = len(counts)
    offsets, M = ragged(counts, tail)
    g = gen(M + K)
    dy, w = randn(g, M, N).bfloat16(), (randn(g, E, N, K) * N ** -0.5).bfloat16()
    h = (randn(g, M, K) * 4).clamp(min=0)
    h = (h.clamp(max=6) if act == "relu6" else h).bfloat16()
    if tail:
        dy[offsets[-1]:] = float("nan")
    for e in range(E):
        if counts[e] == 0:
            w[e] = float("nan")
    want, mag = torch.zeros(M, K, dtype=torch.float64, device="cuda"), torch.zeros(M, K, dtype=torch.float64, device="cuda")
    for e in range(E):
        a, b = offsets[e], offsets[e + 1]
        if b > a:
            want[a:b] = dy[a:b].double() @ w[e].double()
            mag[a:b] = dy[a:b].double().abs() @ w[e].double().abs()
    open_ = torch.ones_like(want, dtype=torch.bool) if act is None else (h > 0) if act == "relu" else (h > 0) & (h < 6)
    want = torch.where(open_, want, 0.0)
    dtype = torch.float32 if (M + K) % 2 else torch.bfloat16
    got = P.grouped_gemm_dx_bf16(views(dy, how), w, ints(offsets), h=views(h, how), act=act, out_dtype=dtype)
    close(got, want, mag, N, (act, dtype))


@pytest.mark.parametrize("how", ["dense", "strided", "odd"])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("counts,tail,N,K", SHAPES, ids=[str(i) for i in range(len(SHAPES))])
def test_grouped_gradient_of_weights(P, counts, tail, N, K, gather, how):
    import torch
    E = len(counts)
    offsets, M = ragged(counts, tail)
    g = gen(M + N + K)
    src = max(1, M // 2) if gather else M
    dy, x = randn(g, M, N).bfloat16(), randn(g, src, K).bfloat16()
    rows = rows_for(M, src, offsets, 2) if gather else None
    xs = reference_rows(x, rows)
    if tail:
        dy[offsets[-1]:] = float("nan")
        if not gather:
            x[offsets[-1]:] = float("nan")
    want = torch.zeros(E, N, K, dtype=torch.float64, device="cuda")
    mag = torch.zeros_like(want)
    for e in range(E):
        a, b = offsets[e], offsets[e + 1]
        if b > a:
            want[e] = dy[a:b].double().T @ xs[a:b]
            mag[e] = dy[a:b].double().abs().T @ xs[a:b].abs()
    args = (views(dy, how), views(x, how), ints(offsets))
    r = None if rows is None else ints(rows)
    got = P.grouped_gemm_dw_bf16(*args, rows=r)
    close(got, want, mag, max(counts), "f32")
    close(P.grouped_gemm_dw_bf16(*args, rows=r, out_dtype=torch.bfloat16), want, mag, max(counts), "bf16")
    base = randn(g, E, N, K)
    acc = P.grouped_gemm_dw_bf16(*args, rows=r, out=base.clone(), accumulate=True)
    assert torch.equal(acc, base + got)                                # one more sum, rounded once
    assert torch.equal(P.grouped_gemm_dw_bf16(*args, rows=r), got)


def test_grouped_gradients_against_differences(P):
    # the product is linear in either operand: a step in one direction changes it by the gradient's inner product with the step
    import torch
    offsets, M = ragged((40, 0, 25, 70), 0)
    E, N, K = 4, 96, 72
    g = gen(8)
    small = lambda *s: torch.randint(-3, 4, s, generator=g, device="cuda").bfloat16()   # noqa: E731  exact in every sum
    x, w, dy, sx, sw = small(M, K), small(E, N, K), small(M, N), small(M, K), small(E, N, K)
    o = ints(offsets)
    f = lambda a, b: (P.grouped_gemm_bf16(a, b, o, out_dtype=torch.float32).double() * dy.double()).sum()   # noqa: E731
    dx = P.grouped_gemm_dx_bf16(dy, w, o, out_dtype=torch.float32)
    dw = P.grouped_gemm_dw_bf16(dy, x, o)
    assert f(x + sx, w) - f(x, w) == (dx.double() * sx.double()).sum()
    assert f(x, w + sw) - f(x, w) == (dw.double() * sw.double()).sum()


@pytest.mark.parametrize("N,K,how", [(72, 64, "dense"), (75, 61, "dense"), (136, 520, "strided"), (4096, 4096, "dense")])
def test_gradient_of_weights_over_long_groups(P, N, K, how):
    # more rows by index than are held at a time (4096), in every kind of tile
    import torch
    counts = (4096, 9001, 3) if N < 4096 else (9001,)
    offsets, M = ragged(counts, 2)
    g = gen(N)
    dy, x = randn(g, M, N).bfloat16(), randn(g, 5000, K).bfloat16()
    rows = rows_for(M, 5000, offsets, 4)
    got = P.grouped_gemm_dw_bf16(views(dy, how), views(x, how), ints(offsets), rows=ints(rows))
    xs = reference_rows(x, rows)
    for e in range(len(counts)):
        a, b = offsets[e], offsets[e + 1]
        close(got[e], dy[a:b].double().T @ xs[a:b], dy[a:b].double().abs().T @ xs[a:b].abs(), counts[e], e)


# groups of tiles of 256: whole and partial ones, groups that end in few rows, empty ones, rows behind the last; results too large for any cache
LARGE = [((1500, 77, 0, 2300, 300), 40, 2056, 136), ((30000, 19000, 159), 0, 2056, 64)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("act", [None, "relu", "relu6"])
@pytest.mark.parametrize("counts,tail,N,K", LARGE, ids=["partial", "past"])
def test_grouped_forward_in_large_tiles(P, counts, tail, N, K, act, dtype):
    import torch
    E = len(counts)
    offsets, M = ragged(counts, tail)
    g = gen(31)
    x, w = randn(g, M, K).bfloat16(), (randn(g, E, N, K) * 3 * K ** -0.5).bfloat16()
    broken = [5, offsets[1] - 1, offsets[-1] - 1]                     # in a whole tile, in partial ones
    x[broken] = float("nan")
    got = P.grouped_gemm_bf16(x, w, ints(offsets), act=act, out_dtype=getattr(torch, dtype))
    assert bool(torch.isnan(got[broken]).all())
    got[broken] = 0.0
    x[broken] = 0.0
    assert bool((got[offsets[-1]:] == 0).all())
    for e in range(E):
        a, b = offsets[e], offsets[e + 1]
        want, mag = x[a:b].double() @ w[e].double().T, x[a:b].double().abs() @ w[e].double().abs().T
        want = want if act is None else want.clamp(min=0) if act == "relu" else want.clamp(0, 6)
        close(got[a:b], want, mag, K, (e, act, dtype))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("act", [None, "relu", "relu6"])
@pytest.mark.parametrize("counts,tail,K,N", LARGE, ids=["partial", "past"])
def test_grouped_gradient_of_rows_in_large_tiles(P, counts, tail, K, N, act, dtype):
    import torch
    E = len(counts)
    offsets, M = ragged(counts, tail)
    g = gen(32)
    dy, w = randn(g, M, N).bfloat16(), (randn(g, E, N, K) * N ** -0.5).bfloat16()
    h = (randn(g, M, K) * 4).bfloat16()                               # negative ones, infinities and NaN among them: closed, open (ReLU), closed
    h[7, 3::50], h[offsets[1] - 1, 1::50] = float("inf"), float("nan")
    got = P.grouped_gemm_dx_bf16(dy, w, ints(offsets), h=h, act=act, out_dtype=getattr(torch, dtype))
    assert bool((got[offsets[-1]:] == 0).all())
    for e in range(E):
        a, b = offsets[e], offsets[e + 1]
        want, mag = dy[a:b].double() @ w[e].double(), dy[a:b].double().abs() @ w[e].double().abs()
        if act is not None:
            want = torch.where((h[a:b] > 0) & ((h[a:b] < 6) if act == "relu6" else True), want, 0.0)
        close(got[a:b], want, mag, N, (e, act, dtype))


def test_grouped_infinities_stay_in_their_rows(P):
    import torch
    offsets, M = ragged((70, 60), 0)
    g = gen(21)
    x, w = randn(g, M, 128).bfloat16(), randn(g, 2, 136, 128).bfloat16()
    clean = P.grouped_gemm_bf16(x, w, ints(offsets))
    x[3, 5], x[100, 127] = float("inf"), float("nan")
    got = P.grouped_gemm_bf16(x, w, ints(offsets))
    keep = torch.ones(M, dtype=torch.bool, device="cuda")
    keep[3] = keep[100] = False
    assert torch.equal(got[keep], clean[keep])
    assert torch.isinf(got[3]).all() and torch.isnan(got[100]).all()
    assert torch.isnan(P.grouped_gemm_bf16(x, w, ints(offsets), act="relu")[100]).all()


def test_grouped_nothing(P):
    import torch
    o = ints([0, 0, 0])
    w = torch.zeros(2, 16, 24, dtype=torch.bfloat16, device="cuda")
    x, d = torch.empty(0, 24, dtype=torch.bfloat16, device="cuda"), torch.empty(0, 16, dtype=torch.bfloat16, device="cuda")
    assert P.grouped_gemm_bf16(x, w, o).shape == (0, 16) and P.grouped_gemm_dx_bf16(d, w, o).shape == (0, 24)
    assert bool((P.grouped_gemm_dw_bf16(d, x, o) == 0).all())
    base = torch.ones(2, 16, 24, device="cuda")
    assert bool((P.grouped_gemm_dw_bf16(d, x, o, out=base, accumulate=True) == 1).all())


def test_offsets_that_are_no_plan_stay_inside(P):
    import torch
    M, N, K, E = 40, 72, 64, 3
    g = gen(2)
    x, w, dy = randn(g, M, K).bfloat16(), randn(g, E, N, K).bfloat16(), randn(g, M, N).bfloat16()
    for bad in ([0, 50, 20, 90], [-5, -1, 10, 41], [7, 3, 60, 2], [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1, 0]):
        o = ints(bad)
        out = torch.full((M + 2, N), 5.0, dtype=torch.bfloat16, device="cuda")
        P.grouped_gemm_bf16(x, w, o, out=out[1:M + 1])
        assert bool((out[0] == 5).all()) and bool((out[M + 1] == 5).all())
        P.grouped_gemm_dx_bf16(dy, w, o)
        P.grouped_gemm_dw_bf16(dy, x, o)
        torch.cuda.synchronize()


def test_grouped_offsets_past_32_bits(P):
    # weights of 2.7 GB and results of 5.4 GB, and a source of 4.9 GB read by row: the last places are right
    import torch
    g = gen(4)
    E, N, K, M = 40, 4096, 8192, 80
    w = torch.zeros(E, N, K, dtype=torch.bfloat16, device="cuda")
    w[E - 1] = randn(g, N, K).bfloat16()
    offsets = ints([2 * e for e in range(E + 1)])
    x = randn(g, M, K).bfloat16()
    got = P.grouped_gemm_bf16(x, w, offsets, out_dtype=torch.float32)
    xs, ws = x[M - 2:].double(), w[E - 1].double()
    close(got[M - 2:], xs @ ws.T, xs.abs() @ ws.abs().T, K)
    assert bool((got[:M - 2] == 0).all())
    dy = randn(g, M, N).bfloat16()
    close(P.grouped_gemm_dx_bf16(dy, w, offsets, out_dtype=torch.float32)[M - 2:], dy[M - 2:].double() @ ws, dy[M - 2:].double().abs() @ ws.abs(), N)
    del w
    dw = P.grouped_gemm_dw_bf16(dy, x, offsets)
    for e in (0, 17, E - 1):
        a, b = dy[2 * e:2 * e + 2].double(), x[2 * e:2 * e + 2].double()
        close(dw[e], a.T @ b, a.abs().T @ b.abs(), 2, e)
    del dw
    src = torch.zeros(600000, 4096, dtype=torch.bfloat16, device="cuda")
    rows = np.array([599999 - 7 * i for i in range(M)])
    src[ints(rows).long()] = randn(g, M, 4096).bfloat16()
    w = (randn(g, E, 64, 4096)).bfloat16()
    xs = src[ints(rows).long()].double()
    got = P.grouped_gemm_bf16(src, w, offsets, rows=ints(rows), out_dtype=torch.float32)
    dw = P.grouped_gemm_dw_bf16(dy[:, :64].contiguous(), src, offsets, rows=ints(rows))
    for e in (0, E - 1):
        s = slice(2 * e, 2 * e + 2)
        close(got[s], xs[s] @ w[e].double().T, xs[s].abs() @ w[e].double().abs().T, 4096, e)
        a = dy[s, :64].double()
        close(dw[e], a.T @ xs[s], a.abs().T @ xs[s].abs(), 2, e)


# ---- 4-bit weights ---------------------------------------------------------------------------------------------------

W4_SHAPES = [((1,), 0, 16, 128), ((1,), 0, 1, 1), ((3,), 0, 33, 200), ((16,), 0, 64, 1024), ((17,), 0, 48, 260), ((40,), 0, 100, 129), ((70,), 0, 256, 512),
             ((0, 2, 0, 1, 5), 2, 80, 384), ((20, 0, 33, 64, 130), 3, 37, 333), ((1,) * 30 + (0,) * 40, 0, 64, 640), ((200, 90), 0, 272, 136)]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("asymmetric", [False, True])
@pytest.mark.parametrize("N,K", [(16, 128), (1, 1), (33, 200), (100, 1000)])
def test_w4_pack(P, N, K, group, asymmetric):
    import torch
    w = randn(gen(N + K), 2, N, K).bfloat16()
    w[0, 0, :K // 2 + 1] = 0                                           # groups of zeros too
    if asymmetric:
        w[1] = w[1].abs()
    p = P.w4_pack_bf16(w, group, asymmetric)
    back = ox.w4_weights(p.q.cpu().numpy(), p.scales.float().cpu().numpy(), p.zeros.cpu().numpy() if asymmetric else None, N, K, group)
    v = w.double().cpu().numpy()
    pad = np.zeros((2, N, -K % group))
    v = np.concatenate([v, pad], 2).reshape(2, N, -1, group)
    hi, lo = np.maximum(v.max(3), 0), np.minimum(v.min(3), 0)
    scale = (hi - lo) / 15 if asymmetric else np.maximum(hi, -lo) / 7
    # half a step; the scale is rounded to bfloat16 (2^-8), the ends lie up to 15 steps out; a zero point is off by half a step
    # more, which the ends of the range may lose
    bound = (scale * (1 + 2.0 ** -7) * (0.5 + 15 * 2.0 ** -8 + (0.5 if asymmetric else 0)))[..., None]
    got = np.concatenate([back, pad], 2).reshape(v.shape)
    assert (np.abs(got - v) <= bound + 1e-30).all()
    assert np.isfinite(p.scales.float().cpu().numpy()).all()


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("counts,tail,N,K", W4_SHAPES, ids=[str(i) for i in range(len(W4_SHAPES))])
def test_w4_product(P, counts, tail, N, K, gather, group):
    import torch
    E = len(counts)
    offsets, M = ragged(counts, tail)
    g = gen(M + N + K)
    asymmetric = (N + K + group) % 64 >= 32
    p = P.w4_pack_bf16((randn(g, E, N, K) * K ** -0.5).bfloat16(), group, asymmetric)
    w = torch.tensor(ox.w4_weights(p.q.cpu().numpy(), p.scales.float().cpu().numpy(), p.zeros.cpu().numpy() if asymmetric else None, N, K, group),
                     device="cuda")
    big = torch.tensor(ox.w4_weights(np.zeros_like(p.q.cpu().numpy()), np.abs(p.scales.float().cpu().numpy()), None, N, K, group), device="cuda").abs()
    src = max(1, M // 2) if gather else M
    x = randn(g, src, K).bfloat16()
    rows = rows_for(M, src, offsets, 3) if gather else None
    xs = reference_rows(x, rows)
    if tail and not gather:
        x[offsets[-1]:] = float("nan")
    want, mag = torch.zeros(M, N, dtype=torch.float64, device="cuda"), torch.zeros(M, N, dtype=torch.float64, device="cuda")
    for e in range(E):
        a, b = offsets[e], offsets[e + 1]
        if b > a:
            want[a:b] = xs[a:b] @ w[e].T
            # the sums are of (16 + q) x and (16 + zero) x, at most 31 scale |x| each; `big` is 8 scale
            mag[a:b] = xs[a:b].abs() @ (big[e].T * (62 / 8))
    how = ("dense", "strided", "odd")[(N + group) % 3]
    for act, dtype in ((None, torch.float32), ("relu", torch.bfloat16), ("relu6", torch.float32)):
        ref = want if act is None else want.clamp(min=0) if act == "relu" else want.clamp(0, 6)
        got = P.w4_gemm_bf16(views(x, how), p.q, p.scales, N, group, zeros=p.zeros, offsets=None if E == 1 and not tail else ints(offsets),
                             rows=None if rows is None else ints(rows), act=act, out_dtype=dtype)
        close(got, ref, mag, K, (act, dtype))
        again = P.w4_gemm_bf16(views(x, how), p.q, p.scales, N, group, zeros=p.zeros, offsets=None if E == 1 and not tail else ints(offsets),
                               rows=None if rows is None else ints(rows), act=act, out_dtype=dtype)
        assert torch.equal(again, got)


def test_w4_strided_result_and_offsets_past_32_bits(P):
    # codes of 2.4 GB: the last expert's are found
    import torch
    g = gen(9)
    E, N, K = 36, 8192, 16384
    codes, per_group = P.w4_shapes(E, N, K, 128)
    q = torch.full(codes, 0x88, dtype=torch.uint8, device="cuda")
    scales = torch.ones(per_group, dtype=torch.bfloat16, device="cuda")
    one = P.w4_pack_bf16((randn(g, N, K)).bfloat16(), 128)
    q[E - 1], scales[E - 1] = one.q[0], one.scales[0]
    x = randn(g, 2, K).bfloat16()
    out = torch.full((2, N + 3), -1.0, dtype=torch.bfloat16, device="cuda")
    offsets = ints([0] * (E - 1) + [1, 2])
    P.w4_gemm_bf16(x, q, scales, N, 128, offsets=offsets, out=out[:, :N])
    alone = P.w4_gemm_bf16(x[1:], one.q, one.scales, N, 128)
    assert torch.equal(out[1:, :N], alone) and bool((out[:, N:] == -1).all()) and bool((out[0, :N] == 0).all())


# ---- the layer --------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("T,D,F,E,k", [(1, 64, 128, 4, 2), (100, 72, 88, 6, 3), (700, 256, 512, 8, 2)])
def test_layer_against_64_bits(P, T, D, F, E, k):
    import torch
    from paper_2006_02230_amd.expert_layer import ExpertLayer
    g = gen(T)
    router = randn(g, D, E) * D ** -0.5
    w1, w2 = (randn(g, E, F, D) * D ** -0.5).bfloat16(), (randn(g, E, D, F) * F ** -0.5).bfloat16()
    x, dout = randn(g, T, D).bfloat16(), randn(g, T, D).bfloat16()
    layer = ExpertLayer(router, w1, w2, k)
    out = layer.forward(x)
    grads = layer.backward(dout)
    ids = layer.kept[3].ids.long()
    X, R, W1, W2 = (v.double().requires_grad_() for v in (x, router, w1, w2))
    p = torch.gather(X @ R, 1, ids).softmax(1)
    want = torch.zeros(T, D, dtype=torch.float64, device="cuda")
    for e in range(E):
        there = (ids == e)
        t = there.any(1).nonzero()[:, 0]
        want = want.index_add(0, t, (p * there).sum(1)[t, None] * (torch.relu(X[t] @ W1[e].T) @ W2[e].T))
    want.backward(dout.double())
    # three roundings to bfloat16 on the way of every term forward and four backward, each of 2^-8 of it, independent: 2^-8 sqrt(n) of the norm
    # and a half more for the terms' unequal sizes
    for got, ref, n in ((out, want, 3), (grads.x, X.grad, 4), (grads.router, R.grad, 4), (grads.w1, W1.grad, 4), (grads.w2, W2.grad, 4)):
        off = (got.double() - ref).norm() / ref.norm()
        assert off <= 1.5 * n ** 0.5 * 2.0 ** -8, (float(off), n)


def test_layer_trains_and_answers_in_4_bits(P):
    from paper_2006_02230_amd.expert_layer import main
    first, last, coded = main()
    assert last < 0.5 * first and coded < first, (first, last, coded)


# ---- streams and graphs ------------------------------------------------------------------------------------------------

def layer(P, x, logits, w1, w2, k):
    """Forward and backward of a layer on given logits; every result."""
    r = P.route(logits, k)
    h = P.grouped_gemm_bf16(x, w1, r.offsets, rows=r.tokens, act="relu")
    y = P.grouped_gemm_bf16(h, w2, r.offsets)
    out = P.combine_bf16(y, r.slots, r.weights)
    dy, dwt = P.combine_bwd_bf16(out, y, r.slots, r.weights)
    dh = P.grouped_gemm_dx_bf16(dy, w2, r.offsets, h=h, act="relu")
    return [*r, h, y, out, dy, dwt, dh, P.grouped_gemm_dw_bf16(dy, h, r.offsets), P.grouped_gemm_dw_bf16(dh, x, r.offsets, rows=r.tokens),
            P.combine_bf16(P.grouped_gemm_dx_bf16(dh, w1, r.offsets), r.slots), P.route_bwd(logits, r.ids, r.weights, dwt)]


@pytest.mark.parametrize("T", [5, 300])
def test_captured_layer_replays_to_the_eager_result(P, T):
    import torch
    g = gen(T)
    D, F, E, k = 128, 256, 8, 2
    make = lambda: (randn(g, T, D).bfloat16(), randn(g, T, E))   # noqa: E731
    w1, w2 = (randn(g, E, F, D) * D ** -0.5).bfloat16(), (randn(g, E, D, F) * F ** -0.5).bfloat16()
    x, logits = make()
    layer(P, x, logits, w1, w2, k)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = layer(P, x, logits, w1, w2, k)
    for _ in range(4):
        nx, nl = make()
        x.copy_(nx)
        logits.copy_(nl)
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, layer(P, x, logits, w1, w2, k)):
            assert torch.equal(a, b)
        torch.cuda.synchronize()


def test_another_stream(P):
    import torch
    g = gen(77)
    x, logits = randn(g, 500, 128).bfloat16(), randn(g, 500, 16)
    w1, w2 = randn(g, 16, 192, 128).bfloat16(), randn(g, 16, 128, 192).bfloat16()
    want = layer(P, x, logits, w1, w2, 4)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    r = P.route(logits, 4, stream=side)
    h = P.grouped_gemm_bf16(x, w1, r.offsets, rows=r.tokens, act="relu", stream=side)
    y = P.grouped_gemm_bf16(h, w2, r.offsets, stream=side)
    out = P.combine_bf16(y, r.slots, r.weights, stream=side)
    side.synchronize()
    assert torch.equal(h, want[5]) and torch.equal(out, want[7])
