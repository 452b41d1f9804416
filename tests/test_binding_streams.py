"""Whose memory a call's own outputs are.  An output that a call allocates is
written on the call's stream, so it comes from that stream's memory: memory of
the current stream may have been freed there with work on it still to run.  The
current stream, on which the caller goes on with it, is recorded.  Stand-ins of
tensors, streams and the library; no GPU is needed."""

import contextlib
import types

import pytest
import torch

from paper_2606_14782_gb300 import bacon
from test_cache_binding import BF16, CALLS, F32, MORE, Stream, Tensor, cache, lib  # noqa: F401

CURRENT, SIDE = Stream(), Stream()
CURRENT.cuda_stream = 0x11
PLAIN = types.SimpleNamespace(cuda_stream=0x99)  # a stream of somebody else's


class Output(Tensor):
    made = []

    def __init__(self, shape, dtype, stream):
        super().__init__(shape, dtype)
        self.stream, self.recorded = stream, []
        Output.made.append(self)

    def record_stream(self, stream):
        self.recorded.append(stream)

    def element_size(self):
        return 2


@pytest.fixture
def streams(monkeypatch, lib):  # noqa: F811
    at = [CURRENT]

    @contextlib.contextmanager
    def stream(s):
        at.append(s)
        yield
        at.pop()

    def empty(*shape, dtype=F32, device=None, **kw):
        shape = shape[0] if len(shape) == 1 and not isinstance(shape[0], int) else shape
        return Output(shape, dtype, at[-1])

    Output.made = []
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda address, device: PLAIN
                        if address == PLAIN.cuda_stream else None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: at[-1])
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: at[-1].cuda_stream,
                        raising=False)
    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch, "empty_like", lambda t: Output(t.shape, t.dtype, at[-1]))


def own(stream):
    assert Output.made
    for t in Output.made:
        assert t.stream is (stream or CURRENT)
        assert t.recorded == ([] if stream in (None, CURRENT) else [CURRENT])


OUTPUTS = {"plan": ("slots", "lengths_out", "state_out"), "locate": ("slots",),
           "load": ("k_out", "v_out"), "attend": ("out", "lse")}


@pytest.mark.parametrize("stream", [None, CURRENT, SIDE, PLAIN])
@pytest.mark.parametrize("name", OUTPUTS)
def test_outputs_of_the_cache(streams, name, stream):
    c = cache()
    args = {n: Tensor(s, t) for n, (s, t) in CALLS[name].items() if n not in OUTPUTS[name]}
    if name == "attend":
        args["lse"] = True
    getattr(c, name)(**args, **MORE.get(name, {}), stream=stream)
    assert len(Output.made) == len(OUTPUTS[name])
    own(stream)


R, L, HQ, H, W, N, D = 2, 3, 4, 2, 8, 40, 64


class Input(Tensor):
    def element_size(self):
        return 2


def rows(heads, n, dtype=BF16, *more):
    return Input((R, L, heads, n, *more), dtype)


QWIN, KV = rows(HQ, W, BF16, D), rows(H, N, BF16, D)
CONTEXT_CALLS = {
    "compress_all_layers": (QWIN, KV, KV, 16),
    "compress_layer_budgets": (QWIN, KV, KV, [16, 12, 20]),
    "compress_with_lse": (QWIN, KV, KV, rows(HQ, W, F32), 16),
    "compress_adaptive": (QWIN, KV, KV, 16),
    "sweep": (QWIN, KV, 16, [{}, {}]),
    "scores": ("S",),
    "compact": (Input((H, N, D), BF16), Input((H, N, D), BF16), Input((H, 16), torch.int32)),
}


@pytest.mark.parametrize("stream", [None, CURRENT, SIDE, PLAIN])
@pytest.mark.parametrize("name", CONTEXT_CALLS)
def test_outputs_of_a_context(streams, name, stream):
    ctx = bacon.Context.__new__(bacon.Context)
    ctx.handle, ctx.kv_heads, ctx.params = None, H, bacon.Params()
    ctx._last_units, ctx._last_N = R * L * H, N
    getattr(ctx, name)(*CONTEXT_CALLS[name], stream=stream)
    own(stream)


@pytest.mark.parametrize("stream", [None, CURRENT, SIDE, PLAIN])
def test_outputs_of_a_state(streams, stream):
    state = bacon.State.__new__(bacon.State)
    state.ctx = bacon.Context.__new__(bacon.Context)
    state.ctx.handle, state.ctx.kv_heads, state.handle = None, H, None
    state.score_layer(0, Input((HQ, W, D), BF16), Input((H, N, D), BF16), True, stream=stream)
    state.select(16, N, stream=stream)
    assert len(Output.made) == 2
    own(stream)
