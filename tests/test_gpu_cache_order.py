"""The 8-bit cache on streams that nothing orders: a cache made while the
default stream is busy serves a stream of its own at once."""

import pytest
import torch

from paper_2606_14782_gb300 import bacon, build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    bacon.load()


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def served(asked):
    """A cache with some thousand tokens a unit, so that items are cut, and a
    layer's queries over it."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    R, H, G, d, page, held = 2, 2, 4, 64, 16, 3000
    blocks = -(-held // page)
    cache = bacon.Cache(1, H, H * G, d, R * H * blocks, page=page, max_requests=R, max_blocks=blocks)
    lengths, table, ring, state = cache.tables(R)
    n = R * H * held
    slots, lengths, _ = cache.plan(lengths, torch.full_like(lengths, held), table, ring, state, n)
    rows = [torch.randn(n, d, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2)]
    cache.store(*rows, slots)
    q = torch.randn(R * asked, H * G, d, generator=gen, device="cuda").to(torch.bfloat16)
    return cache, q, lengths, table


def over(cache):
    return bacon.Cache(1, cache.kv_heads, cache.q_heads, cache.head_dim, cache.pages,
                       page=cache.page, max_requests=cache.max_requests,
                       max_blocks=cache.max_blocks, k=cache.k, v=cache.v, k_scale=cache.k_scale,
                       v_scale=cache.v_scale)


@pytest.mark.parametrize("asked", [1, 90])  # either kernel
def test_a_new_cache_on_a_side_stream(asked):
    cache, q, lengths, table = served(asked)
    want, lse = cache.attend(0, q, lengths, table, lse=True)
    out, z = torch.empty_like(want), torch.empty_like(lse)
    side = torch.cuda.Stream()
    cache.sync()
    torch.cuda.synchronize()
    torch.cuda._sleep(300_000_000)  # about 0.15 s of the default stream
    fresh = over(cache)
    for _ in range(3):
        fresh.attend(0, q, lengths, table, out=out, lse=z, stream=side)
    fresh.sync(side)
    assert torch.equal(out, want) and torch.equal(z, lse)
    torch.cuda.synchronize()


def test_a_reported_error_is_gone_for_another_stream():
    cache, q, lengths, table = served(1)
    want = cache.attend(0, q, lengths, table)
    cache.sync()
    bad = table.clone()
    bad[0, 0, 0, 0] = cache.pages
    out = torch.empty_like(want)
    first, second = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(300_000_000)
    cache.attend(0, q, lengths, bad, out=out, stream=first)
    with pytest.raises(bacon.BaconError) as e:
        cache.sync(first)
    assert e.value.status == bacon.BACON_EINVAL
    cache.attend(0, q, lengths, table, out=out, stream=second)
    cache.sync(second)
    assert torch.equal(out, want)
    torch.cuda.synchronize()


def test_outputs_for_a_side_stream_are_not_the_current_ones_memory():
    """Freed memory of the current stream, with work on it still to run, is not
    what a call on another stream writes its outputs to."""
    cache, *_ = served(1)
    rows = 200_000  # 25 MB an output
    slots = torch.arange(rows, dtype=torch.int32, device="cuda") % (cache.pages * cache.page)
    want = cache.load(slots)
    side = torch.cuda.Stream()
    cache.sync()
    torch.cuda.synchronize()
    busy = [torch.empty_like(want[0]) for _ in range(2)]
    freed = {t.data_ptr() for t in busy}
    torch.cuda._sleep(300_000_000)
    for t in busy:
        t.fill_(7)
    del busy, t
    got = cache.load(slots, stream=side)
    assert not freed & {t.data_ptr() for t in got}
    side.synchronize()
    torch.cuda.synchronize()
    # (bit by bit: rows that nobody stored hold anything, NaN too)
    assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(got, want))


@pytest.mark.parametrize("requests,starts", [
    (4, [0, 90, 0, 90, 90]), (4, [0, 90, 40, 90, 90]), (3, [0, 60, 30, 90]), (2, [1, 40, 90]),
    (2, [0, 91, 90]), (2, [0, 40, 89]), (3, [-1, 0, 1, 90]), (2, [0, -2 ** 31, 90]),
    (24, [0 if r % 2 == 0 else 90 for r in range(24)] + [90])])
def test_ranges_that_do_not_follow_one_another(requests, starts):
    """Nothing is attended, and nothing of it is left for the next call, which
    comes before the error has been asked for."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    H, G, d, page, held, asked = 1, 7, 128, 32, 2500, 90
    blocks = -(-held // page)
    cache = bacon.Cache(1, H, H * G, d, requests * H * blocks, page=page, format="int8",
                        max_requests=requests, max_blocks=blocks)
    for codes, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        codes.copy_(torch.randint(0, 256, codes.shape, generator=gen, device="cuda"))
        scale.fill_(0.01)
    table = torch.randperm(requests * H * blocks, generator=gen, device="cuda").int()
    table = table.view(requests, 1, H, blocks)
    lengths = torch.full((requests, 1, H), held, dtype=torch.int32, device="cuda")
    q = torch.randn(asked, H * G, d, generator=gen, device="cuda").to(torch.bfloat16)
    fine = ints([round(asked * r / requests) for r in range(requests + 1)])
    want, lse = cache.attend(0, q, lengths, table, starts=fine, lse=True)
    cache.sync()
    out, z = torch.full_like(want, 7), torch.full_like(lse, 7)
    bad = ints(starts)
    for _ in range(3):
        cache.attend(0, q, lengths, table, starts=bad, out=out, lse=z)
    again, y = cache.attend(0, q, lengths, table, starts=fine, lse=True)
    with pytest.raises(bacon.BaconError) as e:
        cache.sync()
    assert e.value.status == bacon.BACON_EINVAL
    assert bool((out == 7).all()) and bool((z == 7).all())
    assert torch.equal(again, want) and torch.equal(y, lse)
