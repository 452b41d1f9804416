"""What a context's host code leaves behind when a call returns, on a CUDA
runtime of the host that runs nothing before it is waited for: the error word
that the kernels of any stream write to is clear by then."""

import ctypes

import pytest

import fake_cuda
from paper_2606_14782_gb300 import bacon

SIDE, OTHER = 0x5100, 0x5200  # two streams


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return fake_cuda.library(str(tmp_path_factory.mktemp("fake")))


def context(lib):
    h = ctypes.c_void_p()
    p = bacon.Params()
    lib.bacon_default_params(ctypes.byref(p))
    p.max_seq_len, p.max_requests = 256, 1
    assert lib.bacon_init(ctypes.byref(h), 2, 2, 4, 64, 32, 7, 64, ctypes.byref(p)) == bacon.BACON_OK
    return h, ctypes.c_int.from_address(lib.fake_allocation_of(4))


def test_a_new_context_is_clear_when_it_is_handed_out(lib):
    seen = ctypes.c_int(0)
    for s in (None, SIDE):
        lib.fake_device_work(s, ctypes.addressof(seen), 1)
    ctx, word = context(lib)
    assert word.value == 0
    assert seen.value == 0 and lib.fake_pending() == 2  # which it does not wait for
    lib.bacon_destroy(ctx)


@pytest.mark.parametrize("code,status", [(1, bacon.BACON_EINVAL), (2, bacon.BACON_ECUDA),
                                         (3, bacon.BACON_ETIMEOUT)])
def test_a_reported_error_leaves_nothing_to_clear(lib, code, status):
    ctx, word = context(lib)
    lib.cudaDeviceSynchronize()
    lib.fake_device_work(SIDE, ctypes.addressof(word), code)
    seen = ctypes.c_int(0)
    for s in (None, OTHER):
        lib.fake_device_work(s, ctypes.addressof(seen), 1)
    assert lib.bacon_sync(ctx, SIDE) == status
    assert word.value == 0
    assert seen.value == 0 and lib.fake_pending() == 2
    assert lib.bacon_sync(ctx, SIDE) == bacon.BACON_OK
    lib.bacon_destroy(ctx)
