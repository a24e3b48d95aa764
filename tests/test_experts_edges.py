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
