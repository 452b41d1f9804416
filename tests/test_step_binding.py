"""Arguments of rotary rows, block norms, logits and rotated stores in the
binding: a call runs on the device of its tensors, and what lies elsewhere is
refused before the library is called.  Stand-ins of tensors, streams and the
library; no GPU is needed."""

import pytest
import torch

import test_cache_binding as stand_ins
from test_cache_binding import Stream, Tensor, lib  # noqa: F401  (a fixture)
from paper_2606_14782_gb300 import bacon

BF16, I32, F32 = torch.bfloat16, torch.int32, torch.float32
T, HQ, H, D, V, ROWS, W = 6, 4, 2, 64, 100, 3, 48


class Strided(Tensor):
    def stride(self, i=None):
        s = Tensor.stride(self)
        return s if i is None else s[i]


GIVEN = {
    "rotary": dict(q=((T, HQ, D), BF16), k=((T, H, D), BF16), positions=((T,), I32), q_weight=((D,), BF16),
                   k_weight=((D,), BF16), q_out=((T, HQ, D), BF16), k_out=((T, H, D), BF16)),
    "norm": dict(y=((T, W), BF16), x=((T, W), F32), gate=((T, W), BF16), sum_out=((T, W), F32),
                 norm_out=((T, W), BF16)),
    "logits": dict(logits=((ROWS, V), BF16), tokens=((ROWS, 9), I32), lengths=((ROWS,), I32), prompt=((ROWS,), I32),
                   request=((ROWS,), I32), repetition=((ROWS,), F32), frequency=((ROWS,), F32),
                   presence=((ROWS,), F32), temperature=((ROWS,), F32), bias_tokens=((ROWS, 2), I32),
                   bias_values=((ROWS, 2), F32), mask=((ROWS, 4), I32), out=((ROWS, V), F32)),
    "store": dict(q=((T, HQ, D), BF16), k=((T, H, D), BF16), v=((T, H, D), BF16), positions=((T,), I32),
                  slots=((T, H), I32), q_weight=((D,), BF16), k_weight=((D,), BF16), q_out=((T, HQ, D), BF16)),
}
NAMES = {"rotary": "bacon_rotary_apply", "norm": "bacon_block_norm", "logits": "bacon_logits_process",
         "store": "bacon_cache_store_rotated"}


@pytest.fixture
def calls(lib, monkeypatch):  # noqa: F811
    monkeypatch.setattr(bacon, "_device", lambda: lib.device)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 0x100 + i, raising=False)
    monkeypatch.setattr(bacon, "_empty", lambda shape, dtype, device, stream: Strided(shape, dtype, device.index))
    return lib


def call(which, index=0, other=None, stream=None, at=None):
    """One call with its tensors on device `index`, but `other` on device `at`."""
    given = {n: Strided(s, t, at if n == other else index) for n, (s, t) in GIVEN[which].items()}
    if which == "rotary":
        return bacon.Rotary(D).apply(**given, stream=stream)
    if which == "norm":
        return bacon.BlockNorm(W, post="rms")(**given, stream=stream)
    if which == "logits":
        h = bacon.Logits(V, device=torch.device("cuda", index))
        return h.process(**given, greedy=False, stream=stream)
    cache = bacon.Cache(1, H, HQ, D, 10, page=16, max_requests=3, max_blocks=4,
                        **{n: Strided(t.shape, t.dtype, index) for n, t in stand_ins.pools().items()})
    return cache.store_rotated(bacon.Rotary(D), **given, stream=stream)


@pytest.mark.parametrize("which", list(GIVEN))
@pytest.mark.parametrize("index", [0, 1])
def test_a_call_runs_on_its_tensors_device(calls, which, index):
    call(which, index)
    made = [d for n, d in calls.calls if n == NAMES[which]]
    # handles that belong to a device set it themselves; the others need it current
    assert made == [index if which in ("rotary", "norm") else 0] and calls.device == 0


@pytest.mark.parametrize("which,name", [(w, n) for w in GIVEN for n in GIVEN[w]])
@pytest.mark.parametrize("at", [-1, 1])
def test_a_tensor_apart_is_refused(calls, which, name, at):
    if (which, name) in (("rotary", "q"), ("norm", "y")) and at == 1:
        pytest.skip("the first tensor says where the call is")
    with pytest.raises(ValueError):
        call(which, 0, name, at=at)
    assert NAMES[which] not in [n for n, _ in calls.calls]


@pytest.mark.parametrize("which", list(GIVEN))
def test_another_devices_stream_is_refused(calls, which):
    with pytest.raises(ValueError):
        call(which, 0, stream=Stream(1))
    assert NAMES[which] not in [n for n, _ in calls.calls]
    call(which, 1, stream=Stream(1))
    assert NAMES[which] in [n for n, _ in calls.calls]


def test_weights_say_where_a_norm_is(calls):
    layer = bacon.BlockNorm(W, pre_weight=Strided((W,), BF16, 1))
    with pytest.raises(ValueError):
        layer(Strided((T, W), BF16, 0))
    layer(Strided((T, W), BF16, 1))
    with pytest.raises(ValueError):
        bacon.BlockNorm(W, pre_weight=Strided((W,), BF16, 1), pre_bias=Strided((W,), BF16, 0))(
            Strided((T, W), BF16, 1))
    with pytest.raises(ValueError):
        bacon.BlockNorm(W, pre_weight=Strided((W,), BF16, -1))


def test_logits_belong_to_the_device_that_is_named(calls):
    assert bacon.Logits(V).device.index == bacon.Logits(V, device="cuda").device.index == 0
    with torch.cuda.device(1):
        assert bacon.Logits(V).device.index == bacon.Logits(V, device="cuda").device.index == 1
        assert bacon.Logits(V, device="cuda:0").device.index == 0
    assert [d for n, d in calls.calls if n == "bacon_logits_create"] == [0, 0, 1, 1, 0]
