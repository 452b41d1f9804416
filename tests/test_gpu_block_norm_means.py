"""Layer norms of rows that lie far off 0 for their spread, up to rows of one value.

Why a row of one value c (64 sqrt(eps) or more) is 0 exactly: its mean is off by at
most 2^-17 c (under 100 roundings), so c less the mean is exact, and 256 units of c's
last place at most; 2^15 of them add up exactly, and their mean, which is one of
them, is found exactly.  Less that, the row is 0, and the output the bias."""

import pytest
import torch

import step_reference as ref
from paper_2606_14782_gb300 import bacon, build

pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
WIDTHS = [1, 2, 7, 8, 64, 250, 256, 520, 1024, 1111, 2048, 3584, 4100, 8200, 12288, 16384, 16391, 20000, 32767, 32768]


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    bacon.load()


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
def test_rows_of_one_value(width, dtype):
    most = torch.finfo(dtype).max
    values = torch.tensor([-most, most, 1.0, 3.14159, -1000.1, 65504.0, most / 3, most / 1000.1, 0.0],
                          dtype=FP32, device="cuda").to(dtype)
    y = values[:, None].repeat(3, width)  # (narrow rows share a warp)
    gen = torch.Generator(device="cuda").manual_seed(1)
    w, b = (torch.randn(width, generator=gen, device="cuda").to(dtype) for _ in range(2))
    _, n = bacon.BlockNorm(width, pre="layer")(y)
    assert bool((n == 0).all())
    _, n = bacon.BlockNorm(width, pre="layer", pre_weight=w, pre_bias=b)(y)
    assert bool((n == b).all())
    total, _ = bacon.BlockNorm(width, pre=None, post="layer", post_weight=w, post_bias=b)(y)
    assert bool((total == b).all())


@pytest.mark.parametrize("width", [64, 1024, 1111, 3584])
def test_a_residual_sum_of_one_value(width):
    """The sum in fp32 is x, since a is 0 exactly."""
    y = torch.zeros(5, width, dtype=BF16, device="cuda")
    x = torch.tensor([3e38, -2.0 ** 127, 1e15, 77.7, -1e30], device="cuda")[:, None].repeat(1, width)
    total, n = bacon.BlockNorm(width, pre="layer")(y, x)
    assert torch.equal(total, x) and bool((n == 0).all())


@pytest.mark.parametrize("width", [64, 250, 1024, 1111, 3584, 20000])
def test_rows_that_differ_in_last_places(width):
    """One channel a unit in the last place above the others.  With the mean off twice
    the values are whole units at most, and what is left of a common error is 2^-22 of
    one: 2^-22 sqrt(width) < 2^-14 of the spread.  Roots and products: 2^-18."""
    c = torch.tensor([1.0, 777.7, 1e15, 3e38, -1.7e38, 1e30], device="cuda")
    y = c[:, None].repeat(1, width)
    y[:, 5] = torch.nextafter(c, torch.full_like(c, float("inf")))
    eps = 1e-20
    _, n = bacon.BlockNorm(width, pre="layer", eps=eps)(y)
    want = ref.normed(y.double(), "layer", None, None, eps, 0.0)
    assert bool(((n.double() - want).abs() <= 2.0 ** -14 + 2.0 ** -18 * want.abs()).all())


@pytest.mark.parametrize("width", [8, 40, 64, 200])
def test_such_rows_do_not_change_those_beside_them(width):
    gen = torch.Generator(device="cuda").manual_seed(2)
    y = torch.randn(40, width, generator=gen, device="cuda")
    y[3] = -0.0
    y[5] = 3e38
    y[9] = 12345.6
    y[9, 2] = 12345.7
    y[11] += 1000
    layer = bacon.BlockNorm(width, pre="layer")
    _, n = layer(y)
    for r in range(40):
        assert torch.equal(layer(y[r:r + 1])[1][0].view(torch.int32), n[r].view(torch.int32))
