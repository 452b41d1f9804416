"""Queries at the ends of bf16's range, against the 64-bit reference and within
the bounds of test_gpu_cache.py."""

import pytest
import torch

from paper_2606_14782_gb300 import bacon, build
from test_gpu_cache import check_attend, fill, poison

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    bacon.load()


@pytest.mark.parametrize("asked", [1, 70])  # either kernel
@pytest.mark.parametrize("format", ["e4m3", "int8"])
@pytest.mark.parametrize("largest,scale", [(3.38e38, 2e-38), (3.05e38, 2e-38), (2.9e38, 2e-38),
                                           (1e-38, 1e37)])
def test_largest_and_smallest_queries(asked, format, largest, scale):
    gen = torch.Generator(device="cuda").manual_seed(1)
    cache = bacon.Cache(1, 1, 4, 64, 12, page=16, format=format, max_requests=1, max_blocks=12)
    fill(cache, gen)
    table = torch.randperm(12, generator=torch.Generator().manual_seed(2)).int().cuda().view(1, 1, 1, 12)
    n = torch.tensor([[[11 * 16 + 5]]], dtype=torch.int32)
    poison(cache, table, n, 0)
    q = torch.rand(asked, 4, 64, generator=gen, device="cuda") * 2 - 1
    q[:, :, 7] = 1
    q = (q.double() * largest).to(torch.bfloat16)
    assert bool(torch.isfinite(q).all())
    out, lse = cache.attend(0, q, n.cuda(), table, lse=True, scale=scale)
    cache.sync()
    check_attend(cache, q, n, table, 0, [asked], True, scale, out, lse)
