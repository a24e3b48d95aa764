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
