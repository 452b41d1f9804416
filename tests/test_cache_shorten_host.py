"""Refusals of bacon_cache_shorten before anything is launched."""

import pytest

import fake_cuda
from paper_2606_14782_gb300 import bacon
from test_cache_host_order import create


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return fake_cuda.library(str(tmp_path_factory.mktemp("fake")))


def test_refusals(lib):
    args = [1 << 20, 1 << 21, 1 << 22, 1 << 23, 1 << 24]
    assert lib.bacon_cache_shorten(None, 1, *args, None) == bacon.BACON_EINVAL
    cache = create(lib, max_requests=3)
    before = lib.fake_launches(0)
    for requests in (0, -1, 4):
        assert lib.bacon_cache_shorten(cache, requests, *args, None) == bacon.BACON_EINVAL
        assert "requests" in lib.bacon_last_error().decode()
    for i in range(5):
        assert lib.bacon_cache_shorten(cache, 1, *args[:i], None, *args[i + 1:], None) \
            == bacon.BACON_EINVAL
    assert lib.fake_launches(0) == before
    assert lib.bacon_cache_shorten(cache, 3, *args, None) == bacon.BACON_OK
    assert lib.fake_launches(0) == before + 1
    lib.bacon_cache_destroy(cache)
