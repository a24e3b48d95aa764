"""The products grouped by expert in every kind of tile: each case names the tile that the library's rule takes for it, by a copy of that rule,
so that no kernel goes untested.  Groups are uneven: empty ones, of one row, ending inside tiles, with slots behind the last."""
import numpy as np
import pytest

from oracle import experts as ox

pytestmark = pytest.mark.gpu

CUS = 256          # compute units of an MI355X


@pytest.fixture(scope="module")
def P():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    assert torch.cuda.get_device_properties(0).multi_processor_count == CUS
    import paper_2006_02230_amd as p
    return p


def up(a, b):
    return -(-a // b)


def tile(form, E, M, N, K, whole):
    """Side of the tiles that the library takes; "few": its kernel of few rows.  whole: 16-byte rows, and sources that 32-bit offsets reach."""
    if form == "fwd" and M <= 16 * E:
        return "few"
    cols = N if form == "fwd" else K

    def rounds(side, at_a_time):
        down = up(N, side) * E if form == "dw" else up(M, side) if E == 1 else (M + E * (side // 2) + side - 1) // side
        return up(up(cols, side) * down, at_a_time)
    of128 = rounds(128, 2 * CUS)
    if not whole:
        return 64 if 0.5 * rounds(64, 3 * CUS) <= of128 else 128
    empty = up(N, 256) * up(K, 256) < 8 if form == "dw" else M <= 128 * E
    if not empty and rounds(256, CUS) <= 0.65 * of128:
        return 256
    return 64 if 0.55 * rounds(64, 2 * CUS) <= of128 else 128


def gen(seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape):
    import torch
    return torch.randn(*shape, generator=g, device="cuda")


def ints(v):
    import torch
    return torch.tensor([int(i) for i in v], dtype=torch.int32, device="cuda")


def ragged(counts, tail):
    offsets = [0]
    for c in counts:
        offsets.append(offsets[-1] + c)
    return offsets, offsets[-1] + tail


def close(got, want, mag, reduction, what):
    """A float32 sum on the matrix cores of R products passes R/32 + 1 instructions that add 32 products each: at most R/32 + 33 roundings of 2^-23
    of the sum of the terms' magnitudes; a bfloat16 result is off by 2^-8 of itself more."""
    import torch
    tol = mag * ((reduction / 32 + 33) * 2.0 ** -23)
    tol = tol * (1 + 2.0 ** -8) + want.abs() * 2.0 ** -8 if got.dtype == torch.bfloat16 else tol + want.abs() * 2.0 ** -24
    assert got.shape == want.shape and not bool(torch.isnan(got).any()), what
    bad = (got.double() - want).abs() > tol
    assert not bool(bad.any()), (what, int(bad.sum()), bad.nonzero()[:4].tolist())


def row_indices(M, src, end, seed):
    """A source row for each slot, a tenth of them none, and all of those behind the last group."""
    import torch
    g = gen(seed)
    rows = torch.randint(0, src, (M,), generator=g, device="cuda")
    rows = torch.where(torch.rand(M, generator=g, device="cuda") < 0.1, torch.where(rows % 2 == 0, -1, src + 3), rows)
    rows[end:] = -1
    return rows.int()


def gathered(x, rows):
    import torch
    there = (rows >= 0) & (rows < x.shape[0])
    return torch.where(there[:, None], x.double()[torch.where(there, rows, 0).long()], 0.0)


def guarded(shape, dtype, gap=0):
    """A result between rows that nobody may write, its own rows `gap` longer than it needs; and how to see that they are whole."""
    import torch
    mark = -3.0
    if len(shape) == 3:
        buf = torch.full((shape[0] + 2, *shape[1:]), mark, dtype=dtype, device="cuda")
        view = buf[1:-1]
    else:
        buf = torch.full((shape[0] + 2, shape[1] + gap), mark, dtype=dtype, device="cuda")
        view = buf[1:-1, :shape[1]]

    def whole():
        assert bool((buf[0] == mark).all()) and bool((buf[-1] == mark).all())
        assert len(shape) == 3 or bool((buf[:, shape[1]:] == mark).all())
    return view, whole


def odd(t, is_odd):
    """The matrix, or a copy of it that begins at an odd element and has odd rows, NaN between them."""
    import torch
    if not is_odd:
        return t
    r, c = t.shape
    flat = torch.full((r * (c + 5) + 9,), float("nan"), dtype=t.dtype, device=t.device)
    v = flat[1:1 + r * (c + 5)].view(r, c + 5)[:, :c]
    v.copy_(t)
    return v


SIXTEEN = (300, 0, 1, 511, 256, 255, 257, 700, 64, 63, 129, 400, 2, 333, 600, 350)      # 4221 rows
EIGHT = (2500, 0, 1900, 1, 2049, 3000, 2300, 2050)                                      # 13800
# tile, rows of each group, slots behind the last one, N, K
FORWARD = [
    (256, SIXTEEN, 33, 2056, 264), (256, (3000, 1, 0, 5500), 7, 4104, 72), (128, SIXTEEN, 33, 1032, 136), (64, (65, 0, 100, 31), 5, 200, 136),
    ("reg 128", EIGHT, 9, 2047, 131), ("reg 64", (65, 0, 100, 31), 5, 203, 133), (256, tuple(150 + 13 * i for i in range(70)), 11, 2048, 72),
    (64, tuple(i % 41 for i in range(150)), 11, 136, 72), (256, (30000, 19000, 159), 0, 2056, 64), ("few", (20, 0, 3, 40, 1, 0, 0, 5), 3, 200, 136),
]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("side,counts,tail,N,K", FORWARD, ids=["%s-%d" % (c[0], i) for i, c in enumerate(FORWARD)])
def test_forward(P, side, counts, tail, N, K, gather, dtype):
    import torch
    E, dtype, reg = len(counts), getattr(torch, dtype), str(side).startswith("reg")
    offsets, M = ragged(counts, tail)
    assert tile("fwd", E, M, N, K, not reg) == (int(side[4:]) if reg else side)
    g = gen(M + N)
    x, w = randn(g, max(1, M // 2) if gather else M, K).bfloat16(), (randn(g, E, N, K) * 3 * K ** -0.5).bfloat16()
    for e in range(E):
        if counts[e] == 0:
            w[e] = float("nan")                                       # of experts without rows nothing is seen
    rows = row_indices(M, x.shape[0], offsets[-1], 1) if gather else None
    if not gather:
        x[offsets[-1]:] = float("nan")
    xs = gathered(x, rows) if gather else x.double()
    for act in (None, "relu6"):
        out, whole = guarded((M, N), dtype, 8)
        P.grouped_gemm_bf16(odd(x, reg), w, ints(offsets), rows=rows, act=act, out=out)
        whole()
        assert not bool(out[offsets[-1]:].any())
        for e in range(E):
            a, b = offsets[e], offsets[e + 1]
            want = xs[a:b] @ w[e].double().T
            close(out[a:b], want if act is None else want.clamp(0, 6), xs[a:b].abs() @ w[e].double().abs().T, K, (e, act))


# tile, rows of each group, slots behind the last one, N, K
ROWS = [
    (256, SIXTEEN, 33, 264, 2056), (256, (3000, 1, 0, 5500), 7, 72, 4104), (128, SIXTEEN, 33, 136, 1032), (64, (65, 0, 100, 31), 5, 136, 200),
    ("reg 128", EIGHT, 9, 131, 2047), ("reg 64", (65, 0, 100, 31), 5, 133, 203), (256, tuple(150 + 13 * i for i in range(70)), 11, 72, 2048),
]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("act", [None, "relu", "relu6"])
@pytest.mark.parametrize("side,counts,tail,N,K", ROWS, ids=["%s-%d" % (c[0], i) for i, c in enumerate(ROWS)])
def test_gradient_of_rows(P, side, counts, tail, N, K, act, dtype):
    import torch
    E, dtype, reg = len(counts), getattr(torch, dtype), str(side).startswith("reg")
    offsets, M = ragged(counts, tail)
    assert tile("dx", E, M, N, K, not reg) == (int(side[4:]) if reg else side)
    g = gen(M + K)
    dy, w, h = randn(g, M, N).bfloat16(), (randn(g, E, N, K) * N ** -0.5).bfloat16(), (randn(g, M, K) * 4).bfloat16()
    h[::7, ::5] = 6.0
    for e in range(E):
        if counts[e] == 0:
            w[e] = float("nan")
    dy[offsets[-1]:] = float("nan")
    out, whole = guarded((M, K), dtype, 8)
    P.grouped_gemm_dx_bf16(odd(dy, reg), w, ints(offsets), h=odd(h, reg), act=act, out=out)
    whole()
    assert not bool(out[offsets[-1]:].any())
    for e in range(E):
        a, b = offsets[e], offsets[e + 1]
        want = dy[a:b].double() @ w[e].double()
        if act is not None:
            want = torch.where((h[a:b] > 0) & ((h[a:b] < 6) if act == "relu6" else True), want, 0.0)
        close(out[a:b], want, dy[a:b].double().abs() @ w[e].double().abs(), N, (e, act))


# tile, rows of each group, slots behind the last one, N, K
WEIGHTS = [
    (256, (300, 0, 1, 511, 700, 64, 129, 65), 21, 1032, 1032), (256, (700, 0, 1, 1300), 5, 4104, 2056), (128, (300, 0, 1, 511, 700, 64, 129, 65), 21, 1016, 1000),
    (64, (300, 0, 1, 511), 21, 136, 200), ("reg 128", (300, 0, 1, 511, 700, 64, 129, 65), 21, 2047, 2047), ("reg 64", (300, 0, 1, 511), 21, 133, 203),
    # more rows by index than are in LDS at a time (4096)
    (256, (4097, 9001, 3, 0, 4096), 21, 2056, 1032), (128, (4097, 9001, 3, 0, 4096, 70, 1, 8500), 21, 1016, 1000),
    ("reg 128", (4097, 9001, 3, 0, 4096, 70, 1, 8500), 21, 2047, 2047),
    # more groups than are put in the order of their lengths
    (256, tuple(40 * (i % 5) for i in range(40)), 21, 1032, 1032),
]


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("side,counts,tail,N,K", WEIGHTS, ids=["%s-%d" % (c[0], i) for i, c in enumerate(WEIGHTS)])
def test_gradient_of_weights(P, side, counts, tail, N, K, gather):
    import torch
    E, reg = len(counts), str(side).startswith("reg")
    offsets, M = ragged(counts, tail)
    assert tile("dw", E, M, N, K, not reg) == (int(side[4:]) if reg else side)
    g = gen(M + N + K)
    dy, x = randn(g, M, N).bfloat16(), randn(g, max(1, M // 2) if gather else M, K).bfloat16()
    rows = row_indices(M, x.shape[0], offsets[-1], 2) if gather else None
    dy[offsets[-1]:] = float("nan")
    if not gather:
        x[offsets[-1]:] = float("nan")
    args = (odd(dy, reg), odd(x, reg), ints(offsets))
    f32, whole = guarded((E, N, K), torch.float32)
    P.grouped_gemm_dw_bf16(*args, rows=rows, out=f32)
    whole()
    b16, whole = guarded((E, N, K), torch.bfloat16)
    P.grouped_gemm_dw_bf16(*args, rows=rows, out=b16)
    whole()
    base = randn(g, E, N, K)
    total = P.grouped_gemm_dw_bf16(*args, rows=rows, out=base.clone(), accumulate=True)
    assert torch.equal(total, base + f32)                             # one more sum, rounded once
    del total, base
    xs = gathered(x, rows) if gather else x.double()
    for e in range(E):
        a, b = offsets[e], offsets[e + 1]
        d = dy[a:b].double()
        want, mag = d.T @ xs[a:b], d.abs().T @ xs[a:b].abs()
        close(f32[e], want, mag, counts[e], (e, "float32"))
        close(b16[e], want, mag, counts[e], (e, "bfloat16"))


@pytest.mark.parametrize("E,each,N,side", [(2, 60, 72, 64), (8, 2000, 2048, 128)])
def test_sources_past_32_bits(P, E, each, N, side):
    # 4.9 GB read by row: whole units, but at offsets that 32 bits do not hold
    import torch
    K = 4096
    g = gen(6)
    M, S = E * each, 600000
    offsets = [e * each for e in range(E + 1)]
    assert tile("fwd", E, M, N, K, False) == side
    src = torch.zeros(S, K, dtype=torch.bfloat16, device="cuda")
    rows = (S - 1 - 37 * torch.arange(M, device="cuda")).int()
    src[rows.long()] = randn(g, M, K).bfloat16()
    w, dy = (randn(g, E, N, K) * K ** -0.5).bfloat16(), randn(g, M, N).bfloat16()
    got = P.grouped_gemm_bf16(src, w, ints(offsets), rows=rows)
    dw = P.grouped_gemm_dw_bf16(dy, src, ints(offsets), rows=rows)
    for e in range(E):
        s = slice(offsets[e], offsets[e + 1])
        x, d = src[rows[s].long()].double(), dy[s].double()
        close(got[s], x @ w[e].double().T, x.abs() @ w[e].double().abs().T, K, e)
        close(dw[e], d.T @ x, d.abs().T @ x.abs(), each, e)


@pytest.mark.parametrize("M,N,K,reg,sides", [(40, 72, 64, False, ("few", 64, 64)), (4000, 1032, 1024, False, (128, 128, 128)), (300, 71, 63, True, (64, 64, 64)),
                                             (9000, 2056, 2048, False, (128, 128, 256)), (9000, 1048, 1056, False, (256, 256, 128))])
def test_offsets_that_are_no_plan(P, M, N, K, reg, sides):
    # nothing beside a result is written, and offsets outside [0, M] are the nearest bound
    import torch
    E = 3
    assert tuple(tile(f, E, M, N, K, not reg) for f in ("fwd", "dx", "dw")) == sides
    g = gen(2)
    x, w, dy = randn(g, M, K).bfloat16(), (randn(g, E, N, K) * K ** -0.5).bfloat16(), randn(g, M, N).bfloat16()
    q = P.w4_pack_bf16(w, 32, True)
    largest = 2 ** 31 - 1
    for bad in ([0, M + 10, M // 2, 2 * M], [-5, -1, M // 4, M + 1], [7, 3, M + 20, 2], [largest, -largest - 1, largest, 0]):
        o = ints(bad)
        for dtype in (torch.bfloat16, torch.float32):
            y, y_whole = guarded((M, N), dtype, 8)
            z, z_whole = guarded((M, N), dtype, 8)
            dx, dx_whole = guarded((M, K), dtype, 8)
            dw, dw_whole = guarded((E, N, K), dtype)
            P.grouped_gemm_bf16(x, w, o, out=y)
            P.w4_gemm_bf16(x, q.q, q.scales, N, 32, zeros=q.zeros, offsets=o, out=z)
            P.grouped_gemm_dx_bf16(dy, w, o, out=dx)
            P.grouped_gemm_dw_bf16(dy, x, o, out=dw)
            for whole in (y_whole, z_whole, dx_whole, dw_whole):
                whole()
            if bad[0] != -5:
                continue                                              # groups overlap: any of them may write a row
            cut = M // 4                                              # 0 rows, a quarter, the rest
            good = ints([0, 0, cut, M])
            assert torch.equal(y, P.grouped_gemm_bf16(x, w, good, out_dtype=dtype))
            assert torch.equal(z, P.w4_gemm_bf16(x, q.q, q.scales, N, 32, zeros=q.zeros, offsets=good, out_dtype=dtype))
            assert torch.equal(dx, P.grouped_gemm_dx_bf16(dy, w, good, out_dtype=dtype))
            assert torch.equal(dw, P.grouped_gemm_dw_bf16(dy, x, good, out_dtype=dtype))


# ---- few rows ----------------------------------------------------------------------------------------------------------

def few_tile(E, M, N):
    """Sixteens of outputs and of rows that a workgroup of the few-rows kernel takes, and its waves."""
    rows, tiles = up(M, E), min(M, E) * up(N, 32)
    if rows <= 16:
        return (1, 1, 8) if tiles < CUS else (2, 1, 8) if tiles < 4 * CUS else (2, 1, 4)
    return (2, 2, 8) if rows <= 32 else (2, 4, 8)


# what few_tile says, rows of each group, slots behind the last one, N, K
FEW = [
    ((1, 1, 8), (3, 0, 17, 1), 2, 200, 300), ((2, 1, 8), (0, 1, 16, 17, 33, 2, 0, 5), 3, 1110, 300), ((2, 1, 4), (1, 0, 40, 16, 5, 17, 2, 3) * 2, 5, 2090, 260),
    ((2, 2, 8), (70, 0, 16, 17, 1), 9, 130, 333), ((2, 4, 8), (200, 64, 0, 65, 1), 9, 130, 333),
]


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("case,kind", [(c, kind) for c in FEW for kind in ("bfloat16", "32", "64", "128", "32 zeros", "64 zeros", "128 zeros")
                                       if c[0][1] == 1 or kind != "bfloat16"],           # bfloat16 weights of more rows are the tiles'
                         ids=lambda v: v if isinstance(v, str) else "%dx%dx%d" % v[0])
def test_few_rows(P, case, kind, gather):
    import torch
    shape, counts, tail, N, K = case
    E = len(counts)
    offsets, M = ragged(counts, tail)
    assert few_tile(E, M, N) == shape and (kind != "bfloat16" or tile("fwd", E, M, N, K, True) == "few")
    g = gen(M + N)
    x, w = randn(g, max(1, M // 2) if gather else M, K).bfloat16(), (randn(g, E, N, K) * K ** -0.5).bfloat16()
    rows = row_indices(M, x.shape[0], offsets[-1], 3) if gather else None
    if not gather:
        x[offsets[-1]:] = float("nan")
    xs = gathered(x, rows) if gather else x.double()
    if kind == "bfloat16":
        weights, big = w.double(), w.double().abs()

        def product(act, out):
            P.grouped_gemm_bf16(x, w, ints(offsets), rows=rows, act=act, out=out)
    else:
        group = int(kind.split()[0])
        q = P.w4_pack_bf16(w, group, "zeros" in kind)
        codes, scales, zeros = q.q.cpu().numpy(), q.scales.float().cpu().numpy(), None if q.zeros is None else q.zeros.cpu().numpy()
        weights = torch.tensor(ox.w4_weights(codes, scales, zeros, N, K, group), device="cuda")
        # the sums are of (16 + q) x and (16 + zero) x, at most 31 scale |x| each
        big = torch.tensor(ox.w4_weights(np.zeros_like(codes), scales, None, N, K, group), device="cuda").abs() * (62 / 8)

        def product(act, out):
            P.w4_gemm_bf16(x, q.q, q.scales, N, group, zeros=q.zeros, offsets=ints(offsets), rows=rows, act=act, out=out)
    for act, dtype in ((None, torch.float32), ("relu", torch.bfloat16)):
        out, whole = guarded((M, N), dtype, 3 if gather else 4)
        product(act, out)
        whole()
        assert not bool(out[offsets[-1]:].any())
        for e in range(E):
            a, b = offsets[e], offsets[e + 1]
            want = xs[a:b] @ weights[e].T
            close(out[a:b], want if act is None else want.clamp(min=0), xs[a:b].abs() @ big[e].T, K, (e, act))


# ---- router ------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("E", [16, 17, 32, 33, 64, 65, 128, 129, 256, 257, 512, 513, 1024])
@pytest.mark.parametrize("T", [3, 64, 65, 500])
def test_router_of_every_width(P, T, E):
    # a kernel for every number of logits a lane holds, alone and with a plan of its own
    import torch
    g = gen(T + E)
    k = min(E, 17)                                                     # more choices than lanes take a token at once
    x, d = randn(g, T, E), randn(g, T, k)
    x[T // 2, ::2] = -float("inf")
    for renorm in (False, True):
        r = P.route(x, k, renorm=renorm)
        ids, w, offsets, tokens, slots = ox.route(x.cpu().numpy(), k, renorm)
        for got, want in zip((r.ids, r.offsets, r.tokens, r.slots), (ids, offsets, tokens, slots)):
            assert np.array_equal(got.cpu().numpy(), want)
        # logits of at most 6: a difference, exponentials, a sum and a quotient
        assert np.abs(r.weights.cpu().numpy() - w).max() <= (2 * 12 + 24 + E / 64) * 2.0 ** -23
        got = P.route_bwd(x, r.ids, r.weights, d, renorm=renorm).cpu().numpy().astype(np.float64)
        want = ox.route_bwd(x.cpu().numpy(), ids, r.weights.cpu().numpy().astype(np.float64), d.cpu().numpy().astype(np.float64), renorm)
        assert np.abs(got - want).max() <= 2 * np.abs(d.cpu().numpy()).max() * (2 * 12 + 24 + E / 64 + 2 * k) * 2.0 ** -23
