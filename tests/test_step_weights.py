"""A norm's weights are what their tensors hold when it is called: data that a parameter
was given since then, of another place or type.  Stand-ins; no GPU is needed but for the
last test."""

import pytest
import torch

from test_cache_binding import lib  # noqa: F401  (a fixture)
from test_step_binding import BF16, F32, T, W, Strided, calls  # noqa: F401
from paper_2606_14782_gb300 import bacon, build

NAMES = ("post_weight", "post_bias", "pre_weight", "pre_bias")


class Placed(Strided):
    place, whole = 1 << 20, True

    def data_ptr(self):
        return self.place

    def is_contiguous(self):
        return self.whole


@pytest.fixture
def block(calls, monkeypatch):  # noqa: F811
    """The descriptor of a call."""
    seen = []
    monkeypatch.setattr(calls, "bacon_block_norm", lambda desc, stream: seen.append(desc) or bacon.BACON_OK,
                        raising=False)

    def call(layer):
        seen.clear()
        layer(Strided((T, W), BF16))
        raw, = seen
        return bacon.Block.from_buffer_copy(raw.ljust(bacon.ctypes.sizeof(bacon.Block), b"\0"))
    return call


def test_places_are_read_at_each_call(block):
    w = {n: Placed((W,), BF16) for n in NAMES}
    layer = bacon.BlockNorm(W, pre="layer", post="layer", **w)
    for first in (1 << 20, 1 << 24):
        for i, n in enumerate(NAMES):
            w[n].place = first + 4096 * i
        d = block(layer)
        assert [getattr(d, n) for n in NAMES] == [first + 4096 * i for i in range(4)]


def test_types_are_read_at_each_call(block):
    w = Placed((W,), BF16)
    layer = bacon.BlockNorm(W, pre_weight=w)
    assert block(layer).weight_dtype == bacon.DTYPES[BF16]
    w.dtype = F32
    assert block(layer).weight_dtype == bacon.DTYPES[F32]
    w.dtype = BF16
    assert block(layer).weight_dtype == bacon.DTYPES[BF16]


@pytest.mark.parametrize("change", [dict(dtype=torch.float16), dict(shape=torch.Size((W - 1,))), dict(index=1),
                                    dict(index=-1), dict(whole=False)])
def test_weights_that_became_others_are_refused(block, change):
    w = Placed((W,), BF16)
    layer = bacon.BlockNorm(W, pre_weight=w)
    block(layer)
    for n, v in change.items():
        setattr(w, n, v)
    with pytest.raises(ValueError):
        block(layer)


def test_weights_without_memory_are_refused(block, calls):  # noqa: F811
    """A freed storage has no address, and without one there would be no weight."""
    w = Placed((W,), BF16)
    layer = bacon.BlockNorm(W, pre_weight=w)
    block(layer)
    w.place = 0
    with pytest.raises(ValueError):
        block(layer)
    d = Placed((64,), BF16)
    d.place = 0
    rotary, q, at = bacon.Rotary(64), Strided((T, 4, 64), BF16), Strided((T,), torch.int32)
    with pytest.raises(ValueError):
        rotary.apply(q, None, at, q_weight=d)
    assert "bacon_rotary_apply" not in [n for n, _ in calls.calls]


@pytest.mark.gpu
def test_a_parameter_with_other_data():
    build.build()
    gen = torch.Generator(device="cuda").manual_seed(1)

    def draw(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    width = 3584
    y = draw(7, width).bfloat16()
    w, b = (torch.nn.Parameter(draw(width).bfloat16()) for _ in range(2))
    layer = bacon.BlockNorm(width, pre="layer", pre_weight=w, pre_bias=b)
    layer(y)
    for kind in (torch.bfloat16, torch.float32):
        w.data, b.data = draw(width).to(kind), draw(width).to(kind)
        fresh = bacon.BlockNorm(width, pre="layer", pre_weight=w.detach().clone(), pre_bias=b.detach().clone())
        assert torch.equal(layer(y)[1], fresh(y)[1])
    with torch.no_grad():
        w.mul_(2)
    assert not torch.equal(layer(y)[1], fresh(y)[1])
