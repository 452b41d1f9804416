"""One row of a tensor gives the bits that it gives among the others, wherever the rows
start and however far they are apart."""

import pytest
import torch

from paper_2606_14782_gb300 import bacon, build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    bacon.load()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("width", [64, 200, 1024, 3584, 8192, 20000])
@pytest.mark.parametrize("apart", [0, 1, 6, 8])
@pytest.mark.parametrize("which", ["y", "x", "gate", "sum_out", "norm_out"])
def test_a_row_by_itself(width, apart, dtype, which):
    """`which` has its rows width + apart from one another, the others follow on."""
    T = 9
    gen = torch.Generator(device="cuda").manual_seed(width + apart)

    def rows(name):
        flat = torch.randn(T, width + (apart if name == which else 0), generator=gen, device="cuda").to(dtype)
        return flat[:, :width]

    layer = bacon.BlockNorm(width, pre="rms", post="layer", gate="sigmoid")
    t = {n: rows(n) for n in ("y", "x", "gate", "sum_out", "norm_out")}
    total, n = layer(t["y"], t["x"], t["gate"], sum_out=t["sum_out"], norm_out=t["norm_out"])
    total, n = total.clone(), n.clone()
    for r in range(T):
        t["sum_out"].zero_()
        t["norm_out"].zero_()
        one = {n: v[r:r + 1] for n, v in t.items()}
        a, b = layer(one["y"], one["x"], one["gate"], sum_out=one["sum_out"], norm_out=one["norm_out"])
        assert torch.equal(a, total[r:r + 1]) and torch.equal(b, n[r:r + 1])


def test_a_row_of_a_transposed_column():
    """One row whose distance to a next one is less than its width, and says nothing."""
    y = torch.randn(640, 1, device="cuda").bfloat16().t()
    assert y.shape == (1, 640) and y.stride() == (1, 1)
    layer = bacon.BlockNorm(640)
    want = layer(y.clone(memory_format=torch.contiguous_format))[1].double()
    # the same row added up in another order: sums to 2^-18, one rounding each
    assert bool(((layer(y)[1].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -17) * want.abs()).all())
    out = torch.empty(640, 1, dtype=torch.bfloat16, device="cuda").t()
    assert torch.equal(layer(y, norm_out=out)[1], layer(y)[1])
