"""Rotated stores of as many heads as a store takes: where a launch's grid has no room for
Q beside K the call is two launches, with the same results."""

import ctypes

import pytest
import torch

from paper_2606_14782_gb300 import bacon, build

A = 1 << 20  # an address that nobody follows


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    import fake_cuda
    return fake_cuda.library(str(tmp_path_factory.mktemp("fake")))


@pytest.mark.parametrize("heads,q_heads,tokens,launches", [
    (2, 4, 3, 1), (65535, 0, 1, 1), (65535, 1, 1, 2), (65535, 65535, 2, 2), (65534, 1, 1, 1), (1, 1 << 24, 1, 2)])
def test_every_number_of_heads_is_taken(lib, heads, q_heads, tokens, launches):
    from test_cache_host_order import create
    cache, rotary = create(lib), bacon.Rotary(64)
    q = bacon._pack_rows(A, A, 0, q_heads, 0, 64 * q_heads, 64, 0, 64 * q_heads, 64)
    k = bacon._pack_rows(A, 0, 0, heads, 0, 64 * heads, 64, 0, 0, 0)
    lib.fake_launches.restype = ctypes.c_int
    before = lib.fake_launches(0)
    assert lib.bacon_cache_store_rotated(cache, rotary.handle, tokens, q, k, A, 64 * heads, 64, 0, 1e-6, 0.0, A, A,
                                         None) == bacon.BACON_OK, lib.bacon_last_error()
    assert lib.fake_launches(0) - before == launches
    lib.bacon_cache_destroy(cache)


@pytest.mark.gpu
@pytest.mark.parametrize("heads,q_heads", [(65535, 3), (65530, 2000), (40, 3)])
def test_many_heads_are_the_two_calls(heads, q_heads):
    build.build()
    gen = torch.Generator(device="cuda").manual_seed(heads)

    def draw(n):
        return torch.randn(2, n, 64, generator=gen, device="cuda").bfloat16()

    q, k, v, w = draw(q_heads), draw(heads), draw(heads), draw(1)[0, 0].contiguous()
    at = torch.tensor([5, 6], dtype=torch.int32, device="cuda")
    first = 16 * torch.randperm(heads, generator=gen, device="cuda")
    slots = torch.stack((first, first + 1)).int()  # a page for each head
    one, two = (bacon.Cache(1, 1, 1, 64, heads, page=16, max_requests=1) for _ in range(2))
    r = bacon.Rotary(64)
    got = one.store_rotated(r, q, k, v, at, slots, q_weight=w, k_weight=w)
    turned, kr = r.apply(q, k, at, q_weight=w, k_weight=w)
    two.store(kr, v, slots)
    for cache in (one, two):
        cache.sync()
    assert torch.equal(got, turned)
    for a, b in zip(one.load(slots), two.load(slots)):
        assert torch.equal(a, b)
