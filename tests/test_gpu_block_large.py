"""What stands around a layer of experts past 32 bits: tensors of more than 2^31 values and 2^32 bytes, and calls on two streams at once.

The rows looked at lie on both sides of the borders; what they have to be is what a small call gives, bit for bit, since a row's result does not depend on the
others."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2006_02230_amd as p
    yield p
    torch.cuda.empty_cache()


def gen(seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape):
    import torch
    return torch.randn(*shape, generator=g, device="cuda")


@pytest.mark.parametrize("D", [1000, 9000])
def test_layernorm_past_2_31_values(P, D):
    import torch
    g = gen(D)
    T = ((1 << 31) + (1 << 27)) // D
    rows = torch.cat([torch.arange(3, device="cuda"), (1 << 31) // D + torch.arange(-2, 3, device="cuda"), T - 3 + torch.arange(3, device="cuda")])
    x, dy = torch.zeros(T, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, D, dtype=torch.bfloat16, device="cuda")
    x[rows], dy[rows] = randn(g, len(rows), D).bfloat16(), randn(g, len(rows), D).bfloat16()
    gamma, beta = randn(g, D), randn(g, D)
    f, small = P.layernorm_fwd(x, gamma, beta), P.layernorm_fwd(x[rows], gamma, beta)
    for a, b in zip(f, small):
        assert torch.equal(a[rows], b)
    assert torch.equal(f.y[12345], beta.bfloat16())
    got, want = P.layernorm_bwd(dy, x, f.mean, f.rstd, gamma), P.layernorm_bwd(dy[rows], x[rows], small.mean, small.rstd, gamma)
    assert torch.equal(got.dx[rows], want.dx) and not bool(got.dx[12345].any())
    # the other rows add zeros; eleven terms in another order: ten adds and four roundings of terms
    h = (x[rows].double() - small.mean.double()[:, None]) * small.rstd.double()[:, None]
    assert bool(((got.dgamma - want.dgamma).abs() <= 28 * 2.0 ** -24 * (dy[rows].double() * h).abs().sum(0)).all())
    assert bool(((got.dbeta - want.dbeta).abs() <= 20 * 2.0 ** -24 * dy[rows].double().abs().sum(0)).all())


def test_clipping_a_tensor_past_2_31_values(P):
    import torch
    n = (1 << 31) + 12345
    big, other = torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.full((7,), 4.0, device="cuda")
    at = torch.tensor([0, (1 << 31) - 1, 1 << 31, n - 1], device="cuda")
    big[at] = 3.0
    want = (7 * 16 + 4 * 9) ** 0.5
    assert abs(float(P.clip_grads([other, big], want / 2)) - want) <= 1e-5
    assert bool((big[at] == 1.5).all()) and bool((other == 2).all()) and int((big != 0).sum()) == 4


def test_conversion_past_2_32_words(P):
    # rows that are not whole, so that a word's row is a quotient: the 64-bit one
    import torch
    g = gen(1)
    K, rows = 100, (1 << 28) + 40
    x = torch.zeros(rows, K, dtype=torch.bfloat16, device="cuda")
    at = torch.cat([torch.arange(5, device="cuda"), (1 << 27) + torch.arange(-2, 3, device="cuda"), rows - 45 + torch.arange(45, device="cuda")])
    x[at] = randn(g, len(at), K).bfloat16()
    small = P.mx4_quantise(x[at])
    q = P.mx4_quantise(x)
    assert torch.equal(q.q[at], small.q) and torch.equal(q.scales[at], small.scales) and not bool(q.q[12345].any())
    P.mx4_dequantise(q, K, out=x)
    assert torch.equal(x[at], P.mx4_dequantise(small, K))


@pytest.mark.parametrize("M", [30, 900])
def test_products_with_weights_past_2_32_bytes(P, M):
    import torch
    g = gen(M)
    E, N, K = 36, 8192, 32768
    codes, per_block = P.mx4_shapes(E, N, K)
    w = P.Mx4(torch.zeros(codes, dtype=torch.uint8, device="cuda"), torch.zeros(per_block, dtype=torch.uint8, device="cuda"))
    one = P.mx4_quantise(randn(g, N, K).bfloat16())
    w.q[E - 1], w.scales[E - 1] = one.q, one.scales
    x = P.mx4_quantise(randn(g, M, K).bfloat16())
    offsets = torch.tensor([0] * (E - 1) + [M // 3, M], dtype=torch.int32, device="cuda")
    got = P.mx4_gemm(x, w, offsets=offsets)
    part = torch.tensor([0] * E + [M - M // 3], dtype=torch.int32, device="cuda")
    alone = P.mx4_gemm(P.Mx4(x.q[M // 3:], x.scales[M // 3:]), w, offsets=part)
    assert torch.equal(got[M // 3:], alone) and not bool(got[:M // 3].any()) and bool(alone.any())
    # and what they are: one matrix's own product, whose sums are float32 in another order
    want = P.mx4_gemm(P.Mx4(x.q[M // 3:], x.scales[M // 3:]), one)
    assert float((alone.double() - want.double()).norm() / want.double().norm()) <= 2.0 ** -8


def test_results_past_2_32_bytes(P):
    import torch
    g = gen(4)
    M, N, K = 270000, 4100, 128
    x, w = P.mx4_quantise(randn(g, M, K).bfloat16()), P.mx4_quantise(randn(g, N, K))
    y = P.mx4_gemm(x, w, out_dtype=torch.float32)
    for a in (0, (1 << 30) // N - 200, M - 400):
        assert torch.equal(y[a:a + 400], P.mx4_gemm(P.Mx4(x.q[a:a + 400], x.scales[a:a + 400]), w, out_dtype=torch.float32))


def test_two_streams_at_once(P):
    import torch
    g = gen(9)
    work = []
    for i in range(2):
        T, E = 3000 + 700 * i, 64
        logits = randn(g, T, E)
        work.append((randn(g, T, 1000), randn(g, T, 1000).bfloat16(), logits, logits.topk(4, 1).indices.int(), [randn(g, 300000), randn(g, 77).bfloat16()],
                     P.mx4_quantise(randn(g, 2, 600, 1000)), torch.tensor([0, T // 3, T], dtype=torch.int32, device="cuda")))

    def run(i, stream):
        x, dy, logits, ids, grads, w, offsets = work[i]
        f = P.layernorm_fwd(x, stream=stream)
        b = P.balance(logits, ids, stream=stream)
        out = [torch.empty_like(t) for t in grads]
        return [*f, *P.layernorm_bwd(dy, x, f.mean, f.rstd, stream=stream), *b, P.balance_bwd(logits, b.counts, b.rows, stream=stream),
                P.clip_grads(grads, 1.0, out=out, stream=stream), *out, P.mx4_gemm(P.mx4_quantise(x, stream=stream), w, offsets=offsets, stream=stream)]
    want = [run(i, None) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = [run(i, streams[i]) for i in range(2)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(p, q) for p, q in zip(a, b))
