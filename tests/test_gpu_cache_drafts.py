"""Drafted tokens that are not taken: the units get shorter, and the pages that
held nothing else go back to the ring.  (A length put back by hand leaves such
pages in the table, where the next plan writes others over them.)"""

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


def free_pages(ring, state):
    head, count = state.tolist()
    return [int(ring[(head + i) % len(ring)]) for i in range(count)]


def accounted(cache, lengths, table, ring, state):
    """Every page is free or some unit's, once, and a unit has what its length
    asks for."""
    lengths, table = lengths.cpu(), table.cpu()
    blocks = (lengths + cache.page - 1) // cache.page
    assert torch.equal((table >= 0).sum(-1), blocks)
    column = torch.arange(cache.max_blocks)
    assert torch.equal(table >= 0, column < blocks[..., None])
    free = free_pages(ring.cpu(), state)
    assert sorted(free + table[table >= 0].tolist()) == list(range(cache.pages))


@pytest.mark.parametrize("R,L,H,page", [(1, 1, 1, 16), (5, 3, 2, 16), (4, 28, 4, 64), (40, 1, 8, 32),
                                        (3, 32, 32, 16)])
def test_shorten(R, L, H, page):
    gen = torch.Generator().manual_seed(R)
    held = torch.randint(0, 90, (R, L, H), generator=gen, dtype=torch.int32)
    fewer = torch.tensor([int(torch.randint(0, int(held[r].min()) + 1, (1,), generator=gen))
                          for r in range(R)], dtype=torch.int32)
    if R > 2:
        held[1], fewer[1] = held[1].clamp(min=70), 70  # whole pages of every unit
        fewer[2] = 0
    blocks = -(-90 // page)
    need = int(((held + page - 1) // page).sum())
    cache = bacon.Cache(L, H, H, 64, need + 7, page=page, max_requests=R, max_blocks=blocks)
    _, table, _, _ = cache.tables(R)
    table = table.cpu()
    order = torch.randperm(cache.pages, generator=gen).int()
    used = 0
    for u, n in enumerate(held.view(-1).tolist()):
        b = -(-n // page)
        table.view(-1, blocks)[u, :b] = order[used:used + b]
        used += b
    head = cache.pages // 3
    ring = torch.cat([order[used:], order[:used]]).roll(head)
    state = torch.tensor([head, cache.pages - used], dtype=torch.int32)
    lengths, dev, r, st = held.cuda(), table.cuda(), ring.cuda(), state.cuda()
    accounted(cache, lengths, dev, r, st)
    cache.shorten(fewer.cuda(), lengths, dev, r, st)
    cache.sync()
    want, at = table.clone(), int(state.sum())
    want_ring = ring.clone()
    for q in range(R):
        for l in range(L):
            for h in range(H):
                n = int(held[q, l, h])
                for b in range(-(-(n - int(fewer[q])) // page), -(-n // page)):
                    want_ring[at % cache.pages] = want[q, l, h, b]
                    want[q, l, h, b] = -1
                    at += 1
    assert torch.equal(lengths.cpu(), held - fewer[:, None, None])
    assert torch.equal(dev.cpu(), want) and torch.equal(r.cpu(), want_ring)
    assert st.tolist() == [head, at - head]
    accounted(cache, lengths, dev, r, st)


@pytest.mark.parametrize("what", ["too many", "negative", "page", "length", "ring"])
def test_shorten_changes_nothing_when_it_cannot(what):
    cache = bacon.Cache(1, 2, 2, 64, 12, page=16, max_requests=2, max_blocks=3)
    held = torch.tensor([[[20, 33]], [[40, 48]]], dtype=torch.int32)
    table = torch.tensor([[[[0, 1, -1], [2, 3, 4]]], [[[5, 6, 7], [8, 9, 10]]]], dtype=torch.int32)
    ring, state = torch.arange(12, dtype=torch.int32).roll(-11), torch.tensor([0, 1], dtype=torch.int32)
    fewer = torch.tensor([18, 40], dtype=torch.int32)
    if what == "too many":
        fewer[1] = 41
    elif what == "negative":
        fewer[0] = -1
    elif what == "page":
        table[1, 0, 0, 1] = 12
    elif what == "length":
        held[0, 0, 1] = 49
    else:
        state[1] = 7
    args = [x.cuda() for x in (fewer, held, table, ring, state)]
    cache.shorten(*args)
    with pytest.raises(bacon.BaconError) as e:
        cache.sync()
    assert e.value.status == bacon.BACON_EINVAL
    for got, want in zip(args, (fewer, held, table, ring, state)):
        assert torch.equal(got.cpu(), want)


def test_drafting_loses_no_page():
    """Rounds of drafts of which some tokens are taken, over page edges: every
    page stays accounted for, what is kept is read as it was stored, and the
    next turn attends to it."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    choose = torch.Generator().manual_seed(7)
    R, L, H, G, d, page, drafted = 3, 2, 2, 3, 64, 16, 7
    cache = bacon.Cache(L, H, H * G, d, 80, page=page, max_requests=R, max_blocks=6)
    lengths, table, ring, state = cache.tables(R)
    first = ints([[[9, 15], [16, 17]], [[1, 31], [14, 2]], [[0, 3], [30, 16]]])
    n = int(first.sum())
    slots, lengths, state = cache.plan(lengths, first, table, ring, state, n)

    def rows(*shape):  # of one size, so that no page's scale grows
        return (torch.randint(0, 2, shape, generator=gen, device="cuda") * 2.0 - 1).to(torch.bfloat16)

    flat = rows(n, d)
    cache.store(flat, flat, slots)
    kept = [[[flat[int(first.view(-1)[:u].sum()):][:int(first.view(-1)[u])]
              for u in range((r * L + l) * H, (r * L + l + 1) * H)] for l in range(L)]
            for r in range(R)]
    for _ in range(12):
        slots, lengths, state = cache.plan(lengths, ints([drafted] * R), table, ring, state, R * drafted)
        new = [rows(R * drafted, H, d) for _ in range(L)]
        for l in range(L):
            cache.store(new[l], new[l], slots[l])
        taken = torch.randint(0, 4, (R,), generator=choose)
        cache.shorten(ints((drafted - taken).tolist()), lengths, table, ring, state)
        accounted(cache, lengths, table, ring, state)
        for r in range(R):
            mine = slice(r * drafted, r * drafted + int(taken[r]))
            for l in range(L):
                for h in range(H):
                    kept[r][l][h] = torch.cat([kept[r][l][h], new[l][mine, h]])
    every = cache.locate(lengths, table, int(lengths.sum()))
    k, v = cache.load(every)
    cache.sync()
    want = torch.cat([kept[r][l][h] for r in range(R) for l in range(L) for h in range(H)])
    assert torch.equal(k, want) and torch.equal(v, want)
    cache.release(ints([1] * R), lengths, table, ring, state)
    cache.sync()
    accounted(cache, lengths, table, ring, state)
    assert int(state[1]) == 80
