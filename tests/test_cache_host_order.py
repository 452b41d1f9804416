"""What the 8-bit cache's host code leaves behind when a call returns, on a
CUDA runtime of the host that runs nothing before it is waited for: counts and
error words that a kernel of any stream relies on are clear by then."""

import ctypes

import pytest

import fake_cuda
from paper_2606_14782_gb300 import bacon

SIDE, OTHER = 0x5100, 0x5200  # two streams


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return fake_cuda.library(str(tmp_path_factory.mktemp("fake")))


@pytest.fixture
def idle(lib):
    lib.cudaDeviceSynchronize()
    assert lib.cudaSetDevice(0) == 0
    yield
    lib.cudaDeviceSynchronize()
    assert lib.cudaSetDevice(0) == 0


def desc(**kw):
    d = dict(layers=2, kv_heads=2, q_heads=8, head_dim=64, page=16, pages=10, max_requests=3,
             max_blocks=4, format=0, dtype=0, k=1 << 20, v=2 << 20, k_scale=3 << 20,
             v_scale=4 << 20)
    d.update(kw)
    return bacon.CacheDesc(**d)


def create(lib, **kw):
    h = ctypes.c_void_p()
    assert lib.bacon_cache_create(ctypes.byref(h), ctypes.byref(desc(**kw))) == bacon.BACON_OK
    return h


def words(lib, count):
    """The last words of the last allocation: arrival counts, then the error."""
    size = ctypes.c_size_t()
    base = lib.fake_last_allocation(ctypes.byref(size))
    return (ctypes.c_int * count).from_address(base + size.value - 4 * count)


COUNTS = 152 * 3 + 152 * 2  # of both attention kernels


def test_a_new_cache_is_clear_when_it_is_handed_out(lib, idle):
    cache = create(lib)
    assert list(words(lib, COUNTS + 1)) == [0] * (COUNTS + 1)
    assert lib.fake_pending() == 0
    lib.bacon_cache_destroy(cache)


def test_creation_waits_for_no_other_stream(lib, idle):
    word = ctypes.c_int(0)
    for s in (None, SIDE):  # a prefill on its way, say
        lib.fake_device_work(s, ctypes.addressof(word), 1)
    cache = create(lib)
    assert list(words(lib, COUNTS + 1)) == [0] * (COUNTS + 1)
    assert word.value == 0 and lib.fake_pending() == 2
    lib.bacon_cache_destroy(cache)


@pytest.mark.parametrize("code,status", [(1, bacon.BACON_EINVAL), (2, bacon.BACON_ENOMEM),
                                         (3, bacon.BACON_ETIMEOUT)])
def test_a_reported_error_leaves_nothing_to_clear(lib, idle, code, status):
    cache = create(lib)
    lib.cudaDeviceSynchronize()
    state = words(lib, COUNTS + 1)
    # a kernel on the caller's stream leaves a count and the error
    address = ctypes.addressof(state)
    lib.fake_device_work(SIDE, address + 4 * 7, 5)
    lib.fake_device_work(SIDE, address + 4 * COUNTS, code)
    word = ctypes.c_int(0)
    for s in (None, OTHER):
        lib.fake_device_work(s, ctypes.addressof(word), 1)
    assert lib.bacon_cache_sync(cache, SIDE) == status
    assert list(state) == [0] * (COUNTS + 1)
    assert word.value == 0 and lib.fake_pending() == 2  # other streams' work is not waited for
    assert lib.bacon_cache_sync(cache, SIDE) == bacon.BACON_OK
    lib.bacon_cache_destroy(cache)
