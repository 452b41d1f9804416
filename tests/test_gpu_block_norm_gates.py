"""Gates that are not finite: NaN stays NaN, and infinities have their limits."""

import pytest
import torch

from paper_2606_14782_gb300 import bacon, build

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    bacon.load()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("width", [96, 1111, 3584, 20000])
@pytest.mark.parametrize("kind", list(bacon.GATES))
@pytest.mark.parametrize("shape", ["channel", "token", "full"])
def test_gates_that_are_not_finite(kind, width, shape, dtype):
    T = 5
    gate = torch.ones({"channel": (width,), "token": (T, 1), "full": (T, width)}[shape], device="cuda")
    at = {"channel": [(3,), (40,), (77,)], "token": [(1, 0), (3, 0), (4, 0)], "full": [(1, 3), (3, 40), (4, 77)]}[shape]
    for i, v in zip(at, (NAN, -INF, INF)):
        gate[i] = v
    y = torch.full((T, width), 2.0, device="cuda").to(dtype)
    total, n = bacon.BlockNorm(width, gate=kind)(y, y, gate.to(dtype))
    g = gate.double().expand(T, width)
    want = {"linear": g, "sigmoid": torch.sigmoid(g), "tanh": torch.tanh(g),
            "silu": torch.where(g == -INF, 0.0, g * torch.sigmoid(g))}[kind] * 2 + 2
    assert torch.equal(total.isnan(), want.isnan())
    ok = want.isfinite()
    assert torch.equal(total.double()[~ok & ~want.isnan()], want[~ok & ~want.isnan()])
    # an activation to 2^-21, a product and a sum of 2^-23, and half a step of the type
    off = 2.0 ** -20 + torch.finfo(dtype).eps / 2
    assert bool(((total.double() - want)[ok].abs() <= off * 4).all())
    # a row with a NaN has no norm
    assert torch.equal(n.isnan().any(-1), ~ok.all(-1)) and bool(n[want.isnan().any(-1)].isnan().all())
