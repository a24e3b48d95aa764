"""Microscaled 4-bit floating point on the GPU: codes and scales bit for bit, values, and the products against 64 bits."""
import numpy as np
import pytest

from oracle import block as ob
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


def kind(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def same(got, x):
    codes, scales = ob.mx4_codes(x)
    return np.array_equal(got.q.cpu().numpy(), ob.mx4_pack(codes)) and np.array_equal(got.scales.cpu().numpy(), scales)


# ---- conversion --------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("rows,K", [(1, 1), (1, 31), (3, 32), (2, 33), (5, 127), (7, 128), (4, 129), (3, 777), (300, 1000), (2, 4096)])
@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_quantise(P, rows, K, name):
    import torch
    g = gen(rows + K)
    x = (randn(g, rows, K) * torch.exp2(torch.randint(-20, 20, (rows, K), generator=g, device="cuda").float() * (torch.rand(rows, 1, generator=g, device="cuda") < 0.5)))
    x = x.to(kind(name))
    q = P.mx4_quantise(x)
    assert (tuple(q.q.shape), tuple(q.scales.shape)) == P.mx4_shapes(rows, K)
    assert same(q, x.double().cpu().numpy())
    for out in ("bf16", "f32"):
        want = torch.from_numpy(ob.mx4_values(q.q.cpu().numpy(), q.scales.cpu().numpy(), K)).to(kind(out))
        got = P.mx4_dequantise(q, K, out_dtype=kind(out)).cpu()
        assert torch.equal(got, want) and torch.equal(torch.signbit(got), torch.signbit(want))


def test_quantise_borders(P):
    # every border between two codes, just below and above, of either sign, at every scale that a float can have
    import torch
    base = np.array([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7, 7.75], np.float32)
    near = np.concatenate([base, np.nextafter(base, np.float32(100)), np.nextafter(base, np.float32(-1))])
    near = np.concatenate([near[near >= 0], -near[near >= 0]])
    rows = []
    for e in list(range(-127, 126, 7)) + [-126, -125, 125]:
        for start in range(0, len(near), 31):
            v = np.zeros(32, np.float32)
            part = near[start:start + 31]
            v[:len(part)] = part
            v[31] = 4                                           # so that the scale is 2^e
            rows.append(np.ldexp(v.astype(np.float64), e).astype(np.float32))
    x = np.stack(rows)
    assert same(P.mx4_quantise(torch.from_numpy(x).cuda()), x)


def test_quantise_special_blocks(P):
    import torch
    x = torch.zeros(12, 128)
    x[1, 5] = 2.0 ** -149                    # below every scale
    x[2, 0] = 3.4e38
    x[3, 40] = float("nan")
    x[4, 127] = -float("inf")
    x[5] = -0.0
    x[6, 64:96] = 2.0 ** -126
    x[7] = 1e-39
    x[8, 0], x[8, 1] = 1e30, 1e-30
    x[9] = float("nan")
    q = P.mx4_quantise(x.cuda())
    assert same(q, x.double().numpy())
    assert q.scales[3].tolist()[1] == 255 and q.scales[4].tolist()[3] == 255 and q.scales[0].tolist() == [0] * 4
    v = P.mx4_dequantise(q, 128, out_dtype=torch.float32)
    assert bool(torch.isnan(v[3, 32:64]).all()) and not bool(torch.isnan(v[3, :32]).any()) and bool((v[0] == 0).all())


def test_dequantise_every_byte(P):
    import torch
    q = torch.arange(256, dtype=torch.int64).to(torch.uint8).reshape(4, 64).repeat(64, 1).cuda()           # codes of every kind at every scale
    s = torch.arange(256, dtype=torch.int64).to(torch.uint8)[:, None].repeat(1, 4).cuda()
    for name in ("f32", "bf16"):
        with np.errstate(over="ignore"):
            want = torch.from_numpy(ob.mx4_values(q.cpu().numpy(), s.cpu().numpy())).to(kind(name))
        got = P.mx4_dequantise(P.Mx4(q, s), 128, out_dtype=kind(name)).cpu()
        assert torch.equal(torch.nan_to_num(got, nan=77.0), torch.nan_to_num(want, nan=77.0))


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_conversion_strides(P, name):
    import torch
    g = gen(4)
    flat = randn(g, 1 + 9 * 140).to(kind(name))
    x = flat[1:].view(9, 140)[:, :131]
    q = P.mx4_quantise(x)
    assert same(q, x.double().cpu().numpy())
    out = torch.full((9, 140), 9.0, device="cuda", dtype=kind(name))
    P.mx4_dequantise(q, 131, out=out[:, :131])
    assert bool((out[:, 131:] == 9).all()) and torch.equal(out[:, :131], P.mx4_dequantise(q, 131, out_dtype=kind(name)))
    three = P.mx4_quantise(x.reshape(3, 3, 131).contiguous())
    assert torch.equal(three.q.reshape(9, -1), q.q) and torch.equal(three.scales.reshape(9, -1), q.scales)
    assert torch.equal(P.mx4_dequantise(three, 131).reshape(9, 131), P.mx4_dequantise(q, 131))
    four = P.mx4_quantise(x.reshape(3, 1, 3, 131).contiguous())
    assert torch.equal(four.q.reshape(9, -1), q.q) and torch.equal(P.mx4_dequantise(four, 131).reshape(9, 131), P.mx4_dequantise(q, 131))
    one = P.mx4_quantise(x[4].contiguous())
    assert torch.equal(one.q, q.q[4]) and torch.equal(one.scales, q.scales[4]) and torch.equal(P.mx4_dequantise(one, 131), P.mx4_dequantise(q, 131)[4])
    for shape in ((0, 131), (2, 0, 131)):
        none = P.mx4_quantise(torch.empty(shape, device="cuda"))
        assert P.mx4_dequantise(none, 131).shape == shape
    given = P.Mx4(torch.zeros_like(q.q), torch.zeros_like(q.scales))
    assert P.mx4_quantise(x, out=given).q is given.q and torch.equal(given.q, q.q)


# ---- products ----------------------------------------------------------------------------------------------------

def offsets_of(g, E, M, behind=0):
    """Uneven groups, some empty, `behind` slots after the last."""
    import torch
    cuts = torch.randint(0, M - behind + 1, (E - 1,), generator=g, device="cuda").sort().values if E > 1 else torch.zeros(0, dtype=torch.int64, device="cuda")
    return torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), cuts, torch.full((1,), M - behind, device="cuda")]).int()


def product(x, w, offsets, rows, act, N):
    """The result and the sum of magnitudes, in 64 bits."""
    xv = ox.gathered(x, rows)
    M = len(xv)
    o = [0, M] if offsets is None else [int(v) for v in offsets]
    y, m = np.zeros((M, N)), np.zeros((M, N))
    for e in range(len(o) - 1):
        a, b = o[e], o[e + 1]
        y[a:b], m[a:b] = xv[a:b] @ w[e].T, np.abs(xv[a:b]) @ np.abs(w[e]).T
    return ox.act(y, act), m


def check(got, want, m, K, name):
    # products of the codes are exact; sums are float32: a value passes through at most K/64 instructions and the waves' 16 adds, and inside
    # one it is added with at most 64 others and scaled; twice the half step, since the matrix cores may cut off instead of rounding
    tol = (K / 64 + 16 + 8) * 2.0 ** -23 * m
    tol = tol + (2.0 ** -8 * (np.abs(want) + tol) if name == "bf16" else 0)
    err = np.abs(got.double().cpu().numpy() - want)
    assert (err <= tol + 1e-38).all(), (err / (tol + 1e-38)).max()


def values(P, q, K):
    return ob.mx4_values(q.q.cpu().numpy(), q.scales.cpu().numpy(), K)


GEMMS = [(1, 1, 1, 1), (1, 1, 33, 40), (1, 3, 5, 129), (1, 17, 64, 256), (1, 40, 100, 300), (1, 300, 257, 520), (1, 257, 300, 128), (4, 50, 96, 200), (3, 700, 333, 260),
         (8, 20, 130, 1000), (5, 3, 48, 64), (70, 300, 40, 96), (2, 1500, 512, 384), (64, 256, 256, 512), (1, 1000, 1001, 777), (16, 1, 512, 4096)]


@pytest.mark.parametrize("E,M,N,K", GEMMS)
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_product(P, E, M, N, K, gather, out):
    import torch
    g = gen(E + M + N + K)
    x_rows = M + 3 if gather else M
    x, w = P.mx4_quantise(randn(g, x_rows, K).bfloat16()), P.mx4_quantise(randn(g, E, N, K) * K ** -0.5)
    offsets = offsets_of(g, E, M, min(2, M - 1)) if E > 1 or gather else None
    rows = torch.randint(-1, x_rows + 1, (M,), generator=g, device="cuda").int() if gather else None
    act = ("relu", "relu6", None)[(M + N) % 3]
    got = P.mx4_gemm(x, w, offsets=offsets, rows=rows, act=act, out_dtype=kind(out))
    want, m = product(values(P, x, K), values(P, w, K), None if offsets is None else offsets.cpu().numpy(), None if rows is None else rows.cpu().numpy(),
                      act, N)
    check(got, want, m, K, out)


# what the rule gives tiles of 64, 128 and 256, each with whole tiles, edges, groups of no rows, one to five stages and rows of less than 16 scales; several tiles a
# workgroup
TILES = [(1, 70, 130, k) for k in (30, 100, 256, 300, 400, 513, 1000, 1300)] + [(4, 9000, 1000, 130), (3, 12000, 700, 500)] + \
    [(1, 2100, 2300, k) for k in (100, 400, 600)] + [(5, 1900, 2100, 300)] + [(1, 4096, 4100, k) for k in (96, 384, 777)] + [(6, 9001, 3001, 257), (3, 20000, 2050, 128)]


@pytest.mark.parametrize("E,M,N,K", TILES)
def test_tiles(P, E, M, N, K):
    import torch
    g = gen(M + K)
    # the reference on the GPU in 64 bits: the values are exact there, and so is their product up to its own sums' 2^-53
    x, w = P.mx4_quantise(randn(g, M, K).bfloat16()), P.mx4_quantise(randn(g, E, N, K) * K ** -0.5)
    offsets = offsets_of(g, E, M, 3)
    xv, wv = P.mx4_dequantise(x, K, out_dtype=torch.float32).double(), P.mx4_dequantise(w, K, out_dtype=torch.float32).double()
    rows = torch.randint(0, M, (M,), generator=g, device="cuda").int() if K % 2 else None
    if rows is not None:
        xv = xv[rows.long()]
    name, act = ("bf16", "relu") if K % 3 else ("f32", None)
    got = P.mx4_gemm(x, w, offsets=offsets, rows=rows, act=act, out_dtype=kind(name))
    o = offsets.tolist()
    for e in range(E):
        a, b = o[e], o[e + 1]
        y, m = xv[a:b] @ wv[e].T, xv[a:b].abs() @ wv[e].abs().T
        check(got[a:b], (y.clamp(min=0) if act else y).cpu().numpy(), m.cpu().numpy(), K, name)
    assert not got[o[E]:].any()


@pytest.mark.parametrize("E,M,N,K", [(1, 2, 40, 200), (3, 90, 100, 130), (2, 600, 300, 256)])
def test_product_into_rows_of_a_longer_tensor(P, E, M, N, K):
    import torch
    g = gen(M)
    x, w = P.mx4_quantise(randn(g, M, K)), P.mx4_quantise(randn(g, E, N, K))
    o = offsets_of(g, E, M)
    for name in ("bf16", "f32"):
        for first, pad in ((0, 8), (1, 3)):
            flat = torch.full((first + M * (N + pad),), 9.0, device="cuda", dtype=kind(name))
            out = flat[first:].view(M, N + pad)
            P.mx4_gemm(x, w, offsets=o, out=out[:, :N])
            assert torch.equal(out[:, :N], P.mx4_gemm(x, w, offsets=o, out_dtype=kind(name))) and bool((out[:, N:] == 9).all()) and bool((flat[:first] == 9).all())


def test_product_of_one_matrix(P):
    import torch
    g = gen(8)
    x, w = P.mx4_quantise(randn(g, 30, 100)), P.mx4_quantise(randn(g, 50, 100))
    assert torch.equal(P.mx4_gemm(x, w), P.mx4_gemm(x, P.Mx4(w.q[None], w.scales[None]), offsets=torch.tensor([0, 30], dtype=torch.int32, device="cuda")))
    assert P.mx4_gemm(P.Mx4(x.q[:0], x.scales[:0]), w).shape == (0, 50)


def test_product_refuses_rows_that_are_not_filled_up(P):
    # refused before a kernel that would read past them; the same codes filled up are taken
    import torch
    g = gen(9)
    for M, N, K in ((1, 40, 32), (20, 70, 96), (300, 300, 160)):
        x, w = P.mx4_quantise(randn(g, M, K)), P.mx4_quantise(randn(g, N, K))
        short = [P.Mx4(t.q[:, :K // 2].contiguous(), t.scales[:, :K // 32].contiguous()) for t in (x, w)]
        with pytest.raises(ValueError, match="128"):
            P.mx4_gemm(*short)
        for a, b in ((x, short[1]), (short[0], w)):
            with pytest.raises(ValueError):
                P.mx4_gemm(a, b)
        want, m = product(values(P, x, K), values(P, w, K)[None], None, None, None, N)
        check(P.mx4_gemm(x, w, out_dtype=torch.float32), want, m, K, "f32")


@pytest.mark.parametrize("E,M", [(3, 40), (2, 700), (4, 5)])
def test_product_plans_that_are_none(P, E, M):
    # offsets past the end, that go backwards or are negative: the nearest plan; no row is read or written elsewhere
    import torch
    g = gen(M)
    N, K = 70, 256
    x, w = P.mx4_quantise(randn(g, M, K)), P.mx4_quantise(randn(g, E, N, K))
    for o in ([-5] + [M * 2] * E, [0] + [M // 2] * (E - 1) + [3], [M] * (E + 1), [0] * (E + 1)):
        offsets = torch.tensor(o, dtype=torch.int32, device="cuda")
        out = torch.full((M + 2, N), 9.0, device="cuda")
        P.mx4_gemm(x, w, offsets=offsets, out=out[1:M + 1])
        assert bool((out[0] == 9).all()) and bool((out[M + 1] == 9).all())
        near = [min(max(o[0], 0), M)]
        for v in o[1:]:
            near.append(max(near[-1], min(max(v, 0), M)))
        if o[0] <= 0 and all(b >= a for a, b in zip(o, o[1:])):
            want, m = product(values(P, x, K), values(P, w, K), near, None, None, N)
            check(out[1:M + 1], want, m, K, "f32")


@pytest.mark.parametrize("M", [1, 20, 300, 900])
def test_broken_blocks_reach_their_row_or_column_alone(P, M):
    import torch
    g = gen(M)
    N, K = 300, 640
    a, b = randn(g, M, K), randn(g, N, K)
    x, w = P.mx4_quantise(a), P.mx4_quantise(b)
    good = P.mx4_gemm(x, w, out_dtype=torch.float32)
    a[M // 2, 639], b[17, 0], b[299, 330] = float("nan"), float("inf"), -float("inf")
    got = P.mx4_gemm(P.mx4_quantise(a), P.mx4_quantise(b), out_dtype=torch.float32)
    broken = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    broken[M // 2], broken[:, 17], broken[:, 299] = True, True, True
    assert bool(torch.isnan(got[broken]).all()) and torch.equal(got[~broken], good[~broken])
    for act in ("relu", "relu6"):
        assert bool(torch.isnan(P.mx4_gemm(P.mx4_quantise(a), P.mx4_quantise(b), act=act)[broken]).all())


def test_rows_by_index_past_4_gib(P):
    # rows on both sides of 2^32 bytes, which no 32-bit offset reaches; the others are never read
    import torch
    g = gen(77)
    K, M, N = 8192, 40, 70
    x_rows = (1 << 20) + 50
    q, s = torch.empty((x_rows, K // 2), dtype=torch.uint8, device="cuda"), torch.empty((x_rows, K // 32), dtype=torch.uint8, device="cuda")
    rows = torch.cat([torch.arange(20, device="cuda"), torch.arange(x_rows - 20, x_rows, device="cuda")])
    x, w = P.mx4_quantise(randn(g, M, K)), P.mx4_quantise(randn(g, N, K))
    q[rows], s[rows] = x.q, x.scales
    got = P.mx4_gemm(P.Mx4(q, s), w, rows=rows.int(), out_dtype=torch.float32)
    want, m = product(values(P, x, K), values(P, w, K)[None], None, None, None, N)
    check(got, want, m, K, "f32")


def test_results_do_not_depend_on_the_run_or_the_other_rows(P):
    import torch
    g = gen(21)
    x, w = P.mx4_quantise(randn(g, 700, 900)), P.mx4_quantise(randn(g, 2, 500, 900))
    o = torch.tensor([0, 333, 700], dtype=torch.int32, device="cuda")
    first = P.mx4_gemm(x, w, offsets=o, out_dtype=torch.float32)
    for _ in range(4):
        assert torch.equal(P.mx4_gemm(x, w, offsets=o, out_dtype=torch.float32), first)


# by the rule: few rows of one matrix and of several, tiles of 64, of 128 and of 256
@pytest.mark.parametrize("E,M,N,K", [(1, 16, 70, 900), (3, 20, 300, 520), (2, 700, 500, 900), (1, 2500, 2300, 400), (2, 9000, 3000, 300)])
@pytest.mark.parametrize("gather", [False, True])
def test_rows_do_not_depend_on_the_other_rows(P, E, M, N, K, gather):
    # every third row kept, what is around it in its tile and in the other groups changed: other values, far larger ones, blocks of NaN, zeros, rows that are
    # none; the kept rows' results are the same bits, and so are the columns' whose neighbours change
    import torch
    g = gen(M + N)
    a, b = randn(g, M, K), randn(g, E, N, K)
    o = offsets_of(g, E, M)
    rows = torch.randperm(M, generator=g, device="cuda").int() if gather else None
    kept = torch.arange(M, device="cuda") % 3 == 1
    want = P.mx4_gemm(P.mx4_quantise(a), P.mx4_quantise(b), offsets=o, rows=rows, out_dtype=torch.float32)
    at = kept if rows is None else kept[rows.long()]
    w = P.mx4_quantise(b)
    for fill in (None, 1e30, float("nan"), 0.0):
        other = torch.where(kept[:, None], a, randn(g, M, K) if fill is None else torch.full((), fill, device="cuda"))
        got = P.mx4_gemm(P.mx4_quantise(other), w, offsets=o, rows=rows, out_dtype=torch.float32)
        assert torch.equal(got[at], want[at]) and not torch.equal(got, want)
    if rows is not None:
        got = P.mx4_gemm(P.mx4_quantise(a), w, offsets=o, rows=torch.where(at, rows, -1).int(), out_dtype=torch.float32)
        assert torch.equal(got[at], want[at]) and not got[~at].any()
    column = torch.arange(N, device="cuda") % 5 == 2
    c = torch.where(column[None, :, None], b, torch.full((), float("nan"), device="cuda"))
    got = P.mx4_gemm(P.mx4_quantise(a), P.mx4_quantise(c), offsets=o, rows=rows, out_dtype=torch.float32)
    assert torch.equal(got[:, column], want[:, column]) and bool(torch.isnan(got[:, ~column]).all())


def test_captured_and_replayed_and_on_another_stream(P):
    import torch
    g = gen(31)
    a = randn(g, 400, 500).bfloat16()
    w = P.mx4_quantise(randn(g, 4, 300, 500))
    o = torch.tensor([0, 100, 100, 390, 400], dtype=torch.int32, device="cuda")

    def run(stream=None):
        x = P.mx4_quantise(a, stream=stream)
        return P.mx4_gemm(x, w, offsets=o, act="relu", stream=stream), P.mx4_dequantise(x, 500, stream=stream), \
            P.mx4_gemm(P.Mx4(x.q[:5], x.scales[:5]), P.Mx4(w.q[0], w.scales[0]), stream=stream)
    want = run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = run(side)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run()
    for seed in range(3):
        a.copy_(randn(gen(seed), 400, 500))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip([t.clone() for t in held], run()))


def test_gradients_that_would_be_lost_are_refused(P):
    import torch
    x = torch.randn(4, 8, device="cuda", requires_grad=True)
    with pytest.raises(RuntimeError, match="requires its gradient"):
        P.mx4_quantise(x)
    with torch.no_grad():
        P.mx4_quantise(x)
