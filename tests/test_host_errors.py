"""An error that a call returns is the call's: the runtime's record of the last
error, which the caller's other libraries look at after their own launches, does
not keep it.  On a CUDA runtime of the host."""

import ctypes

import pytest

import fake_cuda
from paper_2606_14782_gb300 import bacon
from test_cache_host_devices import attend
from test_cache_host_order import create, desc


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return fake_cuda.library(str(tmp_path_factory.mktemp("fake")))


def test_creation_without_memory(lib):
    h = ctypes.c_void_p()
    lib.fake_fail_allocations(1)
    assert lib.bacon_cache_create(ctypes.byref(h), ctypes.byref(desc())) == bacon.BACON_ENOMEM
    assert not h.value and lib.cudaPeekAtLastError() == 0
    lib.bacon_cache_destroy(create(lib))


@pytest.mark.parametrize("tokens", [1, 100])
def test_a_launch_that_is_refused(lib, tokens):
    cache = create(lib)
    lib.fake_fail_attributes(1)
    assert attend(lib, cache, tokens) == bacon.BACON_ECUDA
    assert lib.cudaPeekAtLastError() == 0
    assert attend(lib, cache, tokens) == bacon.BACON_OK
    lib.bacon_cache_destroy(cache)
