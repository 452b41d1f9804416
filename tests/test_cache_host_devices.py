"""The 8-bit cache on two devices of one process, on a CUDA runtime of the host
whose functions have their attributes per device, as CUDA's do."""

import ctypes

import pytest

import fake_cuda
from paper_2606_14782_gb300 import bacon
from test_cache_host_order import create


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return fake_cuda.library(str(tmp_path_factory.mktemp("fake")))


def attend(lib, cache, tokens):
    return lib.bacon_cache_attend(cache, 1, 0, tokens, 1 << 20, 8 * 64, 64, None, 1 << 21, 1 << 22,
                                  1, 0.0, 1 << 23, None, None)


FORMS = [(q_heads, d, format, tokens) for q_heads in (2, 20, 40) for d in (64, 128)
         for format in (0, 1) for tokens in (1, 100)]  # every kernel of the attention


@pytest.mark.parametrize("q_heads,d,format,tokens", FORMS)
def test_every_device_can_attend(lib, q_heads, d, format, tokens):
    for device in (0, 1, 0):
        assert lib.cudaSetDevice(device) == 0
        cache = create(lib, q_heads=q_heads, head_dim=d, format=format)
        assert lib.cudaSetDevice(0) == 0
        before = lib.fake_launches(device)
        assert attend(lib, cache, tokens) == bacon.BACON_OK, lib.bacon_last_error().decode()
        assert lib.fake_launches(device) == before + 1
        current = ctypes.c_int(-1)
        assert lib.cudaGetDevice(ctypes.byref(current)) == 0 and current.value == 0
        lib.bacon_cache_destroy(cache)


@pytest.mark.parametrize("tokens", [1, 100])
def test_a_failure_is_that_calls_alone(tmp_path, tokens):
    lib = fake_cuda.library(str(tmp_path))  # no call has been made on it
    cache = create(lib)
    lib.fake_fail_attributes(1)
    assert attend(lib, cache, tokens) == bacon.BACON_ECUDA
    assert attend(lib, cache, tokens) == bacon.BACON_OK
    lib.bacon_cache_destroy(cache)
