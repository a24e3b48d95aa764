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


# ---- another stream ----------------------------------------------------------------------------------------------

def test_calls_on_another_stream_leave_the_current_streams_memory_alone(P):
    # blocks that the current stream has freed, of every result's size, while its work may still use them: no result lies in one
    import torch
    g = gen(3)
    T, E, k, D, F = 500, 16, 4, 128, 192
    x, logits, w1 = randn(g, T, D).bfloat16(), randn(g, T, E), randn(g, E, F, D).bfloat16()
    side = torch.cuda.Stream()
    calls = {}

    def run(stream):
        r = calls["route"] = P.route(logits, k, stream=stream)
        h = calls["forward"] = P.grouped_gemm_bf16(x, w1, r.offsets, rows=r.tokens, stream=stream)
        calls["combine"] = P.combine_bf16(h, r.slots, r.weights, stream=stream)
        calls["combine_bwd"] = P.combine_bwd_bf16(calls["combine"], h, r.slots, r.weights, stream=stream)
        calls["dx"] = P.grouped_gemm_dx_bf16(h, w1, r.offsets, stream=stream)
        calls["dw"] = P.grouped_gemm_dw_bf16(h, x, r.offsets, rows=r.tokens, stream=stream)
        calls["route_bwd"] = P.route_bwd(logits, r.ids, r.weights, r.weights, stream=stream)
        q = calls["pack"] = P.w4_pack_bf16(w1, 128, True, stream=stream)
        calls["w4"] = P.w4_gemm_bf16(x, q.q, q.scales, F, 128, zeros=q.zeros, offsets=r.offsets, rows=r.tokens, stream=stream)
        return {(name, i): t for name, v in calls.items() for i, t in enumerate((v,) if isinstance(v, torch.Tensor) else v)}

    want = run(None)
    torch.cuda.synchronize()
    freed = [(t.untyped_storage().data_ptr(), t.untyped_storage().nbytes()) for t in want.values()]
    values = {name: t.clone() for name, t in want.items()}
    calls.clear()
    del want
    got = run(side)
    side.synchronize()
    for name, t in got.items():
        at = t.untyped_storage().data_ptr()
        assert not any(a < at + t.untyped_storage().nbytes() and at < a + n for a, n in freed), name
        assert torch.equal(t.reshape(-1).view(torch.uint8), values[name].reshape(-1).view(torch.uint8)), name


def test_convolutions_on_another_stream_leave_the_current_streams_memory_alone(P):
    import torch
    g = gen(5)
    x, w = randn(g, 2, 64, 14, 14), randn(g, 64, 64, 3, 3)
    xh, wh = x.bfloat16(), w.bfloat16()
    side = torch.cuda.Stream()

    def run(stream):
        return [P.conv2d_fwd(x, w, pad=1, stream=stream), P.conv2d_fwd_bf16(xh, wh, pad=1, stream=stream), P.filter_tap_copy(w, stream=stream),
                P.nchw_to_nchwc(x, 8, stream=stream)]
    want = run(None)
    torch.cuda.synchronize()
    values = [t.clone() for t in want]
    freed = [(t.untyped_storage().data_ptr(), t.untyped_storage().nbytes()) for t in want]
    del want
    got = run(side)
    side.synchronize()
    for t, v in zip(got, values):
        at = t.untyped_storage().data_ptr()
        assert not any(a < at + t.untyped_storage().nbytes() and at < a + n for a, n in freed)
        assert torch.equal(t, v)


# ---- 4-bit weights ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("asymmetric", [False, True])
@pytest.mark.parametrize("value", ["nan", "inf", "-inf"])
def test_weights_that_no_code_holds_show(P, value, asymmetric, group):
    import torch
    E, N, K = 2, 37, 300
    g = gen(group)
    clean = randn(g, E, N, K).bfloat16()
    w, x = clean.clone(), randn(g, 6, K).bfloat16()
    broken = [(0, 0, 0), (0, 17, 131), (1, 36, K - 1), (1, 20, 64), (1, 20, 200)]
    for at in broken:
        w[at] = float(value)
    a, b = P.w4_pack_bf16(clean, group, asymmetric), P.w4_pack_bf16(w, group, asymmetric)
    scales = torch.zeros(b.scales.shape, dtype=torch.bool, device="cuda")
    for e, n, k in broken:
        scales[e, n // 16, k // group, n % 16] = True
    assert torch.equal(torch.isnan(b.scales), scales) and torch.equal(b.scales[~scales], a.scales[~scales])
    offsets = torch.tensor([0, 2, 6], dtype=torch.int32, device="cuda")
    ya, yb = (P.w4_gemm_bf16(x, p.q, p.scales, N, group, zeros=p.zeros, offsets=offsets) for p in (a, b))
    gone = torch.zeros(6, N, dtype=torch.bool, device="cuda")
    for e, n, k in broken:
        gone[[0, 1] if e == 0 else [2, 3, 4, 5], n] = True
    assert torch.equal(torch.isnan(yb), gone) and torch.equal(yb[~gone], ya[~gone])


@pytest.mark.parametrize("group", [32, 64, 128])
def test_weights_whose_range_passes_the_largest_float(P, group):
    import torch
    K = 256
    w = randn(gen(group), 1, 16, K).bfloat16() * 1e37
    w[0, :, 3], w[0, :, group - 1] = torch.finfo(torch.bfloat16).max, torch.finfo(torch.bfloat16).min
    w[0, 1, group - 1] = 1.0
    p = P.w4_pack_bf16(w, group, True)
    scales = p.scales.double().cpu().numpy()
    assert np.isfinite(scales).all()
    back = ox.w4_weights(p.q.cpu().numpy(), p.scales.float().cpu().numpy(), p.zeros.cpu().numpy(), 16, K, group)
    v = w.double().cpu().numpy()
    parts = v.reshape(1, 16, -1, group)
    scale = (np.maximum(parts.max(3), 0) - np.minimum(parts.min(3), 0)) / 15
    # half a step, half a step more for the zero point, and the scale's rounding over 15 steps
    bound = (scale * (1 + 2.0 ** -7) * (0.5 + 0.5 + 15 * 2.0 ** -8))[..., None]
    assert (np.abs(back.reshape(parts.shape) - parts) <= bound).all()


def test_scales_are_what_they_were(P):
    # the range over 15 in 32 bits, rounded to bfloat16, small and large weights and the smallest ones there are
    import torch
    g = gen(1)
    w = randn(g, 1, 64, 512) * torch.exp2(torch.randint(-140, 120, (1, 64, 1), generator=g, device="cuda").float())
    w = w.bfloat16()
    w[0, 0] = torch.randint(-2, 3, (512,), generator=g, device="cuda", dtype=torch.int16).abs().view(torch.bfloat16)
    p = P.w4_pack_bf16(w, 128, True)
    parts = w.float().reshape(64, 4, 128)
    want = ((parts.amax(2).clamp(min=0) - parts.amin(2).clamp(max=0)) / 15).bfloat16()
    got = p.scales.reshape(4, 4, 16).transpose(1, 2).reshape(64, 4)
    assert torch.equal(got, want)


# ---- more threads than one axis of a grid holds (2^32) ------------------------------------------------------------------

@pytest.fixture
def room(P):
    """Memory that earlier tests' tensors leave unused goes back before and after tests of large ones."""
    import torch
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def test_router_of_2_28_tokens(P, room):
    # 1024 threads for 64 tokens in the choice and the plan
    import torch
    T = (1 << 28) + 70
    x = randn(gen(1), T, 2)
    x[-3] = -float("inf")
    r = P.route(x, 1)
    first = (x[:, 0] >= x[:, 1]) & (x[:, 0] != -float("inf"))
    want = torch.where(first, 0, 1).int()
    want[-3] = -1
    assert torch.equal(r.ids[:, 0], want)
    n0 = int(first.sum())
    assert r.offsets.tolist() == [0, n0, T - 1]
    at = torch.where(first, torch.cumsum(first, 0) - 1, n0 + torch.cumsum(want == 1, 0) - 1)    # by the tokens up to this one
    at[-3] = -1
    assert torch.equal(r.slots[:, 0], at.int())
    tokens = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    there = want >= 0
    tokens[at[there]] = there.nonzero()[:, 0].int()
    assert torch.equal(r.tokens, tokens)
    assert bool((r.weights[there] == 1).all()) and float(r.weights[-3]) == 0


def test_router_gradient_of_2_28_tokens(P, room):
    # 16 lanes a token
    import torch
    T = (1 << 28) + 9
    x = randn(gen(2), T, 2)
    ids = torch.zeros(T, 1, dtype=torch.int32, device="cuda")
    d = torch.ones(T, 1, device="cuda")
    got = torch.full((T, 2), 7.0, device="cuda")
    P.route_bwd(x, ids, d, d, renorm=False, out=got)
    assert not bool((got == 7).any())
    for at in (0, 1 << 24, T - 5000):
        p = torch.softmax(x[at:at + 5000].double(), 1)
        want = p * (torch.tensor([1.0, 0.0], device="cuda") - p[:, :1])
        # probabilities off by the roundings of a difference of up to 12, an exponential, a sum and a quotient, twice
        assert float((got[at:at + 5000].double() - want).abs().max()) <= 2 * (2 * 12 + 8) * 2.0 ** -23


def test_weighted_sum_of_2_24_long_rows(P, room):
    # a workgroup of 256 for every token
    import torch
    T, D = (1 << 24) + 5, 1032
    y = randn(gen(3), 3, D).bfloat16()
    slots = (torch.arange(T, device="cuda") % 4 - 1).int().reshape(T, 1)                # -1, 0, 1, 2
    out = P.combine_bf16(y, slots)
    rows = torch.cat([torch.zeros_like(y[:1]), y])
    for a in range(0, T, 1 << 20):
        assert torch.equal(out[a:a + (1 << 20)], rows[slots[a:a + (1 << 20), 0].long() + 1]), a


def test_gradient_of_the_weighted_sum_of_2_26_slots(P, room):
    # a wave a slot
    import torch
    T, k, M, D = (1 << 21) + 1, 32, 40, 3
    g = gen(4)
    y, d, w = randn(g, M, D).bfloat16(), randn(g, T, D).bfloat16(), torch.ones(T, k, device="cuda")
    slots = torch.full((T, k), -1, dtype=torch.int32, device="cuda")
    places = [(0, 0, 5), (1 << 20, 31, 7), (T - 2, 3, 0), (T - 1, 0, 1), (T - 1, 31, 39)]
    for t, j, s in places:
        slots[t, j] = s
    before = torch.full((M, D), 7.0, dtype=torch.bfloat16, device="cuda")
    dy, dw = P.combine_bwd_bf16(d, y, slots, w, dy=before.clone())
    want = before
    for t, j, s in places:
        want[s] = d[t]
        assert abs(float(dw[t, j]) - float((d[t].double() * y[s].double()).sum())) <= 4 * 2.0 ** -23 * float((d[t].double() * y[s].double()).abs().sum())
        dw[t, j] = 0
    assert torch.equal(dy, want) and not bool(dw.any())


def test_products_of_few_rows_with_2_29_columns(P, room):
    # 256 threads for 32 columns
    import torch
    N = (1 << 29) + 40
    w = randn(gen(5), 1, N, 1).bfloat16()
    x = torch.full((1, 1), 0.7, device="cuda").bfloat16()
    got = P.grouped_gemm_bf16(x, w, torch.tensor([0, 1], dtype=torch.int32, device="cuda"))
    assert torch.equal(got[0], w[0, :, 0] * x[0])                     # one product, rounded once


def test_gradient_of_the_weights_of_2_21_experts(P, room):
    # eight workgroups of 256 for every expert
    import torch
    E = (1 << 21) + 3
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[E // 2:], offsets[E] = 2, 5
    dy, x = (randn(gen(s), 5, 1).bfloat16() for s in (6, 7))
    got = torch.full((E, 1, 1), 7.0, device="cuda")
    P.grouped_gemm_dw_bf16(dy, x, offsets, out=got)
    for e, rows in ((E // 2 - 1, slice(0, 2)), (E - 1, slice(2, 5))):
        terms = (dy[rows].double() * x[rows].double())
        assert abs(float(got[e]) - float(terms.sum())) <= 34 * 2.0 ** -23 * float(terms.abs().sum())
        got[e] = 0
    assert not bool(got.any())


def test_packing_of_2_26_tiles(P, room):
    # 64 threads a tile
    import torch
    N = (1 << 30) + 48
    w = randn(gen(8), N, 1).bfloat16()
    p = P.w4_pack_bf16(w, 128)
    for a in (0, 1 << 29, N - 64):
        part = P.w4_pack_bf16(w[a:a + 64], 128)
        assert torch.equal(p.q[:, a // 16:a // 16 + 4], part.q) and torch.equal(p.scales[:, a // 16:a // 16 + 4], part.scales)


# ---- the layer ----------------------------------------------------------------------------------------------------------

def test_layer_without_tokens(P):
    import torch
    from paper_2006_02230_amd.expert_layer import ExpertLayer
    g = gen(12)
    layer = ExpertLayer(randn(g, 64, 4), randn(g, 4, 128, 64).bfloat16(), randn(g, 4, 64, 128).bfloat16(), 2)
    x = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    assert layer.forward(x).shape == (0, 64) and layer.coded().forward(x).shape == (0, 64)
    grads = layer.backward(x)
    assert grads.x.shape == (0, 64) and grads.x.dtype == torch.bfloat16
    for got, like in ((grads.router, layer.router), (grads.w1, layer.w1), (grads.w2, layer.w2)):
        assert got.shape == like.shape and got.dtype == torch.float32 and not bool(got.any())


def test_another_stream_inside_a_captured_graph(P):
    import torch
    g = gen(13)
    x, w, logits = randn(g, 300, 128).bfloat16(), randn(g, 8, 192, 128).bfloat16(), randn(g, 300, 8)
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        r = P.route(logits, 2, stream=side)
        y = P.grouped_gemm_bf16(x, w, r.offsets, rows=r.tokens, stream=side)
        main.wait_stream(side)
        out = P.combine_bf16(y, r.slots, r.weights)
        del r, y
    for seed in range(3):
        logits.copy_(randn(gen(seed), 300, 8))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        r = P.route(logits, 2)
        assert torch.equal(out, P.combine_bf16(P.grouped_gemm_bf16(x, w, r.offsets, rows=r.tokens), r.slots, r.weights)), seed
        torch.cuda.synchronize()
