"""Rows of a page that do not follow one another in a call of store: what comes
after the first of them is left out and reported."""

import pytest
import torch

import cache_reference as ref
from paper_2606_14782_gb300 import bacon, build
from test_gpu_cache import ints

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    bacon.load()


# slots of a call (pages of 16), and those whose rows are stored
CASES = [
    ([16, 17, 19, 20], [16, 17]),              # a gap
    ([16, 18, 17], [16]),                      # out of order
    ([20, 20, 21], [20]),                      # the same slot twice
    ([17, 18, 16], [17, 18]),                  # the page's first row last
    ([-1, 5, 6, 4, 32, 33], [5, 6, 32, 33]),   # other pages are stored
    ([16, 17, 30, 31, 32], [16, 17, 32]),
]


@pytest.mark.parametrize("slots,kept", CASES)
@pytest.mark.parametrize("format", ["e4m3", "int8"])
@pytest.mark.parametrize("repeat", [1, 700])  # a window of one token, and of several
def test_rows_apart_are_left_out(slots, kept, format, repeat):
    gen = torch.Generator().manual_seed(1)
    cache = bacon.Cache(1, 1, 1, 64, 3 * repeat, page=16, format=format, max_requests=1, max_blocks=1)
    for t in (cache.k, cache.v):
        t.fill_(0x11)
    for t in (cache.k_scale, cache.v_scale):
        t.fill_(2.0 ** -20)
    every = [s + 48 * i if s >= 0 else s for i in range(repeat) for s in slots]
    stored = {s + 48 * i for i in range(repeat) for s in kept}
    k, v = (torch.randn(len(every), 64, generator=gen).to(torch.bfloat16) for _ in range(2))
    cache.store(k.cuda(), v.cuda(), ints(every))
    with pytest.raises(bacon.BaconError) as e:
        cache.sync()
    assert e.value.status == bacon.BACON_EINVAL
    untouched = torch.ones(cache.pages * 16, dtype=torch.bool)
    for rows, codes, scale in ((k, cache.k, cache.k_scale), (v, cache.v, cache.v_scale)):
        codes, scale = codes.cpu().view(-1, 64), scale.cpu()
        pages = ref.Pages(format, 16, 64)
        # (a page that is appended to has a scale already, of rows that it holds)
        at, done = 0, set()
        while at < len(every):
            n = 1
            while at + n < len(every) and every[at + n] == every[at] + n and every[at + n] % 16:
                n += 1
            s = every[at]
            if s in stored and s not in done:
                page, off = divmod(s, 16)
                if off:
                    old = ref.value(torch.full((16, 64), 0x11, dtype=torch.uint8), format)
                    pages.pages[page] = (2.0 ** -20, old)
                pages.store(rows[at:at + n], every[at:at + n])
                done |= set(every[at:at + n])
            at += n
        assert done == stored
        want = pages.load(sorted(stored))
        index = torch.tensor(sorted(stored))
        got = ref.value(codes[index], format) * scale[index // 16].double()[:, None]
        assert torch.equal(got, want)
        # rows that were left out, and pages without a run, are as they were
        held = {s // 16: s % 16 for s in stored}
        untouched[index] = False
        first = torch.tensor([s % 16 < held.get(s // 16, 0) for s in range(len(untouched))])
        assert bool((codes[untouched & ~first] == 0x11).all())
