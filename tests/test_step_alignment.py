"""Addresses of positions and slots that no int32 can have: a kernel would fault on them,
so they are refused on the host.  On a CUDA runtime of the host; no GPU is needed."""

import pytest

from paper_2606_14782_gb300 import bacon
from test_step_host import A, EINVAL, handle, rows  # noqa: F401  (a fixture)


@pytest.mark.parametrize("off", [1, 2, 3])
def test_positions_and_slots_that_are_not_aligned(handle, off):  # noqa: F811
    from test_cache_host_order import create
    lib, _ = handle
    rotary, word = bacon.Rotary(64), lib.bacon_last_error
    q = rows(in_token=256, in_head=64, out_token=256, out_head=64)
    args = [rotary.handle, 1, 3, q, None, 0, 0, 1e-6, 0.0, 0]
    assert lib.bacon_rotary_apply(*args, A + off, None) == EINVAL
    assert "positions must be aligned" in word().decode()
    cache = create(lib)
    k = rows(out=0, heads=2, in_token=128, in_head=64)
    for positions, slots, said in ((A + off, A, "positions"), (A, A + off, "slots")):
        assert lib.bacon_cache_store_rotated(cache, rotary.handle, 3, None, k, A, 128, 64, 0, 1e-6, 0.0, positions,
                                             slots, None) == EINVAL
        assert said + " must be aligned" in word().decode()
    lib.bacon_cache_destroy(cache)
