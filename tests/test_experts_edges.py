"""The layer of experts where it is easily wrong, on a machine without a GPU: sizes at the edge of 32 bits, memory for another
stream, gradients that nobody would get, forwards without their backward."""
import pytest

import paper_2006_02230_amd as P

OK, NULL, DIM, UNSUPPORTED, NO_DEVICE = 0, -1, -2, -3, -5
AT = 4096          # an address that is aligned and never looked at
MOST = (1 << 31) - (1 << 16)
BIG = (1 << 31) - 1


def st(name, *args):
    return getattr(P.lib, name)(*args, None)


def fwd(E=2, M=8, N=16, K=24):
    return st("polydl_grouped_gemm_bf16", E, M, N, K, AT, None, M, AT, K, AT, AT, N, 1, 0)


def dx(E=2, M=8, N=16, K=24):
    return st("polydl_grouped_gemm_dx_bf16", E, M, N, K, AT, AT, N, AT, AT, K, 1, AT, K, 1)


def dw(E=2, M=8, N=16, K=24):
    return st("polydl_grouped_gemm_dw_bf16", E, M, N, K, AT, AT, N, None, M, AT, K, AT, 0, 0)


def w4(E=2, M=8, N=16, K=24):
    return st("polydl_w4_gemm_bf16", E, M, N, K, 32, AT, None, M, AT, K, AT, AT, AT, AT, N, 1, 0)


def pack(E=2, N=16, K=24):
    return st("polydl_w4_pack_bf16", E, N, K, 32, AT, AT, AT, AT)


@pytest.mark.parametrize("f,names", [(fwd, "EMNK"), (dx, "EMNK"), (dw, "EMNK"), (w4, "EMNK"), (pack, "ENK")])
def test_lengths_past_the_kernels_arithmetic_are_refused(f, names):
    # a tile, a stage or a window of row indices that begins before the end may end past 2^31
    import torch
    for name in names:
        for n in (MOST + 1, BIG - 300, BIG):
            assert f(**{name: n}) == UNSUPPORTED, (f.__name__, name, n)
        if not torch.cuda.is_available():
            assert f(**{name: MOST}) == NO_DEVICE, (f.__name__, name)


class Recorder:
    """Stands in for a tensor, torch's streams and its allocator; writes down who allocates where."""

    def __init__(self, monkeypatch):
        import contextlib

        import torch
        self.at, self.log, self.is_cuda = "current", [], True

        @contextlib.contextmanager
        def on(stream):
            before, self.at = self.at, stream
            yield
            self.at = before
        monkeypatch.setattr(torch.cuda, "stream", on)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: self.at)

    def new_empty(self, shape, dtype=None):
        self.log.append(("empty", self.at))
        return self

    def record_stream(self, stream):
        self.log.append(("record", stream))


def test_memory_for_another_stream_is_that_streams(monkeypatch):
    # memory of the current stream may be under work queued there, which a call on another stream does not wait for
    import torch
    from paper_2006_02230_amd import experts
    like = Recorder(monkeypatch)
    experts._new((3,), torch.float32, like, "side")
    assert like.log == [("empty", "side"), ("record", "current")] and like.at == "current"
    like.log.clear()
    experts._new((3,), torch.float32, like, None)
    assert like.log == [("empty", "current")]


def test_every_call_allocates_for_its_stream(monkeypatch):
    import torch
    from paper_2006_02230_amd import binding

    class Allocated(Exception):
        pass

    def new(shape, dtype, like, stream):
        raise Allocated(stream)
    monkeypatch.setattr(binding, "_new", new)
    f, h = torch.zeros, torch.bfloat16
    calls = [lambda s: P.nchw_to_nchwc_bf16(f(1, 8, 4, 4, dtype=h), stream=s), lambda s: P.kcrs_to_kcrsck_bf16(f(8, 8, 1, 1, dtype=h), stream=s),
             lambda s: P.conv2d_fwd_bf16_blocked(f(1, 1, 4, 4, 8, dtype=h), f(8, 1, 1, 1, 8, 1, dtype=h), 8, stream=s),
             lambda s: P.conv2d_fwd_bf16(f(1, 8, 4, 4, dtype=h), f(8, 8, 1, 1, dtype=h), stream=s),
             lambda s: P.conv2d_fwd_bf16(f(1, 8, 4, 4, dtype=h), f(8, 8, 1, 1, dtype=h), workspace=f(1), stream=s),
             lambda s: P.conv2d_fwd(f(1, 8, 4, 4), f(8, 8, 1, 1), stream=s), lambda s: P.filter_tap_copy(f(8, 8, 1, 1), stream=s),
             lambda s: P.nchw_to_nchwc(f(1, 8, 4, 4), 8, stream=s), lambda s: P.nchwc_to_nchw(f(1, 1, 4, 4, 8), 8, stream=s),
             lambda s: P.kcrs_to_kcrsck(f(8, 8, 1, 1), 8, 1, stream=s),
             lambda s: P.bnorm_fwd(f(1, 8, 4, 4), f(8), f(8), f(8), f(8), stream=s)]
    for i, call in enumerate(calls):
        with pytest.raises(Allocated) as e:
            call("side")
        assert e.value.args == ("side",), i


@pytest.fixture
def layer(monkeypatch):
    """An ExpertLayer whose operators are their definitions in 64 bits on the CPU."""
    import numpy as np
    import torch

    from oracle import experts as ox
    from paper_2006_02230_amd import expert_layer as L
    t, n = torch.tensor, lambda v: v.double().numpy()   # noqa: E731

    def route(logits, k):
        ids, w, offsets, tokens, slots = ox.route(n(logits), k, True)
        return P.Route(t(ids), t(w), t(offsets), t(tokens), t(slots))

    def groups(offsets):
        return [slice(int(a), int(b)) for a, b in zip(offsets[:-1], offsets[1:])]

    def forward(x, w, offsets, rows=None, act=None):
        x = x if rows is None else x[rows]
        return ox.act(torch.cat([x[g].double() @ w[e].double().T for e, g in enumerate(groups(offsets))]).numpy(), act)

    def dx(dy, w, offsets, h=None, act=None, out_dtype=None):
        d = torch.cat([dy[g].double() @ w[e].double() for e, g in enumerate(groups(offsets))])
        return d if act is None else d * (h > 0)

    def dw(dy, x, offsets, rows=None):
        x = x if rows is None else x[rows]
        return torch.stack([dy[g].double().T @ x[g].double() for g in groups(offsets)])

    def combine(y, slots, weights=None, out_dtype=None):
        return (y[slots] * (1.0 if weights is None else weights.unsqueeze(2))).sum(1)

    def combine_bwd(dout, y, slots, weights):
        dy = torch.empty_like(y)
        dy[slots] = dout.double().unsqueeze(1) * weights.unsqueeze(2)
        return dy, (dout.double().unsqueeze(1) * y[slots]).sum(2)

    def sgemm(a, b, c, alpha=1.0, beta=1.0):
        return c.copy_(beta * c + alpha * (a.double() @ b.double()) if beta else alpha * (a.double() @ b.double()))
    for name, f in {"route": route, "grouped_gemm_bf16": lambda *a, **k: t(forward(*a, **k)), "grouped_gemm_dx_bf16": dx, "grouped_gemm_dw_bf16": dw,
                    "combine_bf16": combine, "combine_bwd_bf16": combine_bwd,
                    "route_bwd": lambda logits, ids, w, d: t(ox.route_bwd(n(logits), ids.numpy(), n(w), n(d), True)),
                    "w4_pack_bf16": lambda w, *a: P.W4(w[:, :1, :1].clone(), w[:, :1, :1].clone(), None)}.items():
        monkeypatch.setattr(L.X, name, f)
    monkeypatch.setattr(L.B, "sgemm", sgemm)
    r = np.random.RandomState(0)
    make = lambda *s: t(r.randn(*s))   # noqa: E731
    return L.ExpertLayer(make(6, 4), make(4, 5, 6), make(4, 6, 5), 2), make


def same(a, b):
    import torch
    return all(torch.equal(p, q) for p, q in zip(a, b))


def test_gradients_are_those_of_the_forward_they_belong_to(layer):
    layer, make = layer
    a, b, da, db = make(7, 6), make(7, 6), make(7, 6), make(7, 6)
    with pytest.raises(RuntimeError):
        layer.backward(da)
    layer.forward(a)
    want_a = layer.backward(da)
    layer.forward(b)
    want_b = layer.backward(db)
    assert not same(want_a, want_b) and same(want_b, layer.backward(db))         # the last one's again
    layer.forward(a)
    kept_a = layer.kept
    layer.forward(b)
    with pytest.raises(RuntimeError):                                             # whose?
        layer.backward(da)
    kept_b = layer.kept
    assert same(layer.backward(da, kept_a), want_a) and same(layer.backward(db, kept_b), want_b)
    layer.forward(a)
    layer.forward(b, keep=False)
    assert same(layer.backward(da), want_a)


def test_answers_keep_nothing(layer):
    layer, make = layer
    layer.forward(make(3, 6), keep=False)
    assert layer.kept is None


def test_weights_in_4_bits_take_the_others_place(layer):
    import gc

    import torch
    layer, make = layer
    coded, sizes = layer.coded(), {layer.w1.data_ptr(), layer.w2.data_ptr()}
    held = [v for o in (coded, *vars(coded).values()) for v in gc.get_referents(o) if isinstance(v, torch.Tensor)]
    held += [v for v in vars(coded).values() if isinstance(v, torch.Tensor)]
    assert held and not any(v.data_ptr() in sizes for v in held)
    assert not any(v is layer for v in vars(coded).values())


def test_arguments_whose_gradient_would_be_lost_are_refused():
    import torch
    z = lambda *s, d=torch.bfloat16: torch.zeros(*s, dtype=d)   # noqa: E731
    f32, i32 = torch.float32, torch.int32
    calls = [(P.route, (z(4, 8, d=f32),), (2,)), (P.combine_bf16, (z(4, 8), None), (z(2, 2, d=i32),)),
             (P.combine_bf16, (z(4, 8), z(2, 2, d=f32)), (z(2, 2, d=i32),)), (P.grouped_gemm_bf16, (z(4, 8), z(2, 16, 8)), (z(3, d=i32),)),
             (P.w4_gemm_bf16, (z(4, 8), z(1, 1, 4, 16)), (16, 32))]

    def call(f, wants, rest):
        if f is P.combine_bf16:
            return f(wants[0], rest[0], wants[1])
        if f is P.w4_gemm_bf16:
            return f(wants[0], torch.zeros(1, 1, 1, 64, 16, dtype=torch.uint8), wants[1], *rest)
        return f(*wants, *rest)
    for f, wants, rest in calls:
        for i, t in enumerate(wants):
            if t is None:
                continue
            asks = [v if j != i else t.clone().requires_grad_() for j, v in enumerate(wants)]
            with pytest.raises(RuntimeError, match="gradient"):
                call(f, asks, rest)
            with torch.no_grad(), pytest.raises(TypeError):            # host tensors
                call(f, asks, rest)


def test_assembly_leaves_no_register_that_the_compiler_does_not_know_of():
    # registers named in the text of an assembly statement, rather than given as its operands
    import glob
    import os
    import re
    for path in glob.glob(os.path.join(os.path.dirname(P.__file__), "csrc", "*.h*")):
        for text in re.findall(r"\basm\s*(?:volatile)?\s*\((\"[^;]*?);\n", open(path).read(), re.S):
            code = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', text.split(":")[0]))
            assert not re.search(r"\b(m0|vcc\w*|exec\w*|scc|[sva]\d+|[sva]\[\d+:\d+\])\b", code.replace("\\n", " ").replace("\\t", " ")), (path, code)


def test_barriers_order_memory_for_the_compiler_too():
    # the bare builtin of a barrier orders the waves, not what the compiler does with reads and writes around it
    import glob
    import os
    import re
    for path in glob.glob(os.path.join(os.path.dirname(P.__file__), "csrc", "*.h*")):
        text = open(path).read()
        bare = len(re.findall(r"__builtin_amdgcn_s_barrier\(\)", text))
        clobber = r'asm volatile\("" ::: "memory"\);\s*'
        assert bare == len(re.findall(clobber + r"(?:gg_wait<[^;]*;\s*)?__builtin_amdgcn_s_barrier\(\);\s*" + clobber, text)), path
