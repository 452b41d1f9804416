"""The 8-bit paged cache against a plain 64-bit reference.

Plans, slots, codes and scales are exact.  Attention is held to bounds stated
before its first run: with A = sum p |v| / sum p, an output may be off by its
own rounding (the unit roundoff of 8 significant bits, 2^-8 of it, for bf16, of
11 bits, 2^-11, for fp16, and half the smallest subnormal), by the rounding of the
softmax weights to 11 bits (2^-11 A) and by the logits' (fp32 sums of d
products of size S = scale sum |q k|: 2^-16 S in the exponent, so 2 * 2^-16 S A;
the exponential unit's 2^-22 is inside), and by what vanishes below fp16's least
step: a weight w = p v_scale is held as fp16 with the largest at 2^14, so it is
off by 2^-25 at least steps of 2^-24, which is 2^-39 of the largest, times a
code of at most 448 for each of the n tokens: 2^-30 n max(p v_scale) / sum p.
The log-sum-exp may be off by 2^-16 S + 2^-20 (1 + |lse|)."""

import math

import pytest
import torch

import cache_reference as ref
from paper_2606_14782_gb300 import bacon, build

pytestmark = pytest.mark.gpu

DTYPES = ref.DTYPES


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    bacon.load()


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# -------------------------------------------------------------------- plan

def shuffled(cache, requests, lengths, seed):
    """Tables of units that hold `lengths`, their pages anywhere in the pool,
    the ring turned."""
    gen = torch.Generator().manual_seed(seed)
    _, table, _, _ = cache.tables(requests)
    table = table.cpu()
    order = torch.randperm(cache.pages, generator=gen).int()
    used = 0
    flat = table.view(-1, cache.max_blocks)
    for u, n in enumerate(lengths.view(-1).tolist()):
        b = -(-n // cache.page)
        flat[u, :b] = order[used:used + b]
        used += b
    head = cache.pages // 3
    ring = torch.cat([order[used:], order[:used]]).roll(head)
    return table, ring, torch.tensor([head, cache.pages - used], dtype=torch.int32)


@pytest.mark.parametrize("R,L,H,page,mode,most_held,most_new", [
    (1, 1, 1, 16, "units", 0, 1), (1, 1, 1, 128, "tokens", 0, 1), (3, 2, 4, 16, "tokens", 40, 1),
    (3, 2, 4, 16, "tokens", 40, 50), (2, 3, 2, 64, "units", 100, 200), (5, 28, 4, 32, "units", 0, 60),
    (7, 3, 5, 16, "none", 33, 1), (40, 1, 8, 64, "tokens", 300, 9), (2, 32, 32, 16, "units", 20, 20),
])
def test_plan(R, L, H, page, mode, most_held, most_new):
    gen = torch.Generator().manual_seed(R + L)
    held = torch.randint(0, most_held + 1, (R, L, H), generator=gen, dtype=torch.int32)
    if mode == "units":
        added = torch.randint(0, most_new + 1, (R, L, H), generator=gen, dtype=torch.int32)
        each = added
    else:
        added = (torch.ones(R, dtype=torch.int32) if mode == "none" else
                 torch.randint(0, most_new + 1, (R,), generator=gen, dtype=torch.int32))
        each = added[:, None, None].expand(R, L, H).contiguous()
    blocks = -(-(most_held + most_new) // page) + 1
    pages = int(((held + each + page - 1) // page).sum()) + 3
    cache = bacon.Cache(L, H, H, 64, pages, page=page, max_requests=R, max_blocks=blocks)
    table, ring, state = shuffled(cache, R, held, 1)
    want_table, want_len, want_state, want = ref.plan(held, each, table, ring, state, page)
    rows = int(added.sum()) + 5
    dev = table.cuda()
    slots, lengths, st = cache.plan(held.cuda(), None if mode == "none" else added.cuda(), dev,
                                    ring.cuda(), state.cuda(), rows)
    cache.sync()
    assert torch.equal(dev.cpu(), want_table)
    assert torch.equal(lengths.cpu(), want_len)
    assert torch.equal(st.cpu(), want_state)
    if mode == "units":
        flat = [s for mine in want for s in mine]
        assert slots.tolist() == flat + [-1] * 5
        got = cache.locate(added.cuda(), dev, rows, first=held.cuda())
        assert torch.equal(got, slots)
        whole = cache.locate(lengths, dev, int(lengths.sum()))
        cache.sync()
        u = torch.repeat_interleave(torch.arange(R * L * H), want_len.view(-1))
        x = torch.cat([torch.arange(n) for n in want_len.view(-1).tolist()] or [torch.zeros(0)])
        expect = want_table.view(R * L * H, -1)[u, x.long() // page] * page + x % page
        assert torch.equal(whole.cpu(), expect.int())
    else:
        expect = torch.full((L, rows, H), -1, dtype=torch.int32)
        start = 0
        for r in range(R):
            for l in range(L):
                for h in range(H):
                    mine = want[(r * L + l) * H + h]
                    expect[l, start:start + len(mine), h] = torch.tensor(mine, dtype=torch.int32)
            start += int(added[r])
        assert torch.equal(slots.cpu(), expect)


@pytest.mark.parametrize("what,status", [
    ("pages", bacon.BACON_ENOMEM), ("rows", bacon.BACON_EINVAL), ("columns", bacon.BACON_EINVAL),
    ("negative length", bacon.BACON_EINVAL), ("negative number", bacon.BACON_EINVAL),
    ("ring", bacon.BACON_EINVAL)])
def test_plan_gives_nothing_when_it_cannot_give_all(what, status):
    cache = bacon.Cache(2, 3, 3, 64, 40, page=16, max_requests=4, max_blocks=3)
    held = torch.full((4, 2, 3), 15, dtype=torch.int32)
    table, ring, state = shuffled(cache, 4, held, 2)
    added = torch.full((4, 2, 3), 2, dtype=torch.int32)
    rows = int(added.sum())
    if what == "pages":
        state[1] -= 40 - 24 - 24 + 9   # one page fewer than the 24 that are asked for
        state[1] = 23 if state[1] >= 24 or state[1] < 0 else state[1]
    elif what == "rows":
        rows -= 1
    elif what == "columns":
        added[1, 0, 2] = 3 * 16 - 15 + 1
        rows += 64
    elif what == "negative length":
        held[3, 1, 2] = -1
    elif what == "negative number":
        added[0, 0, 0] = -1
    else:
        state[0] = 40
    dev = table.cuda()
    slots, lengths, st = cache.plan(held.cuda(), added.cuda(), dev, ring.cuda(), state.cuda(), rows)
    with pytest.raises(bacon.BaconError) as e:
        cache.sync()
    assert e.value.status == status
    assert torch.equal(dev.cpu(), table) and torch.equal(lengths.cpu(), held)
    assert torch.equal(st.cpu(), state) and bool((slots == -1).all())
    cache.sync()  # the latched error is gone


def test_release_gives_the_pages_back_in_order():
    cache = bacon.Cache(3, 2, 2, 64, 200, page=16, max_requests=5, max_blocks=6)
    gen = torch.Generator().manual_seed(9)
    held = torch.randint(0, 90, (5, 3, 2), generator=gen, dtype=torch.int32)
    table, ring, state = shuffled(cache, 5, held, 3)
    done = [0, 7, 0, 1, 1]
    lengths, dev, r, st = held.cuda(), table.cuda(), ring.cuda(), state.cuda()
    cache.release(ints(done), lengths, dev, r, st)
    cache.sync()
    want_ring, at = ring.clone(), int(state.sum())
    for q, d in enumerate(done):
        if d:
            for l in range(3):
                for h in range(2):
                    for b in range(-(-int(held[q, l, h]) // 16)):
                        want_ring[at % 200] = table[q, l, h, b]
                        table[q, l, h, b] = -1
                        at += 1
            held[q] = 0
    assert torch.equal(dev.cpu(), table) and torch.equal(lengths.cpu(), held)
    assert torch.equal(r.cpu(), want_ring)
    assert st.tolist() == [int(state[0]), at - int(state[0])]
    # every page is either free or some unit's
    free = [int(want_ring[(int(st[0]) + i) % 200]) for i in range(int(st[1]))]
    assert sorted(free + table[table >= 0].tolist()) == list(range(200))
    cache.release(ints(done), lengths, dev, r, st)  # nothing is left to give
    cache.sync()
    assert torch.equal(r.cpu(), want_ring)


def test_release_refuses_what_is_no_page():
    cache = bacon.Cache(1, 1, 1, 64, 8, page=16, max_requests=1, max_blocks=4)
    for table, length, state in (([0, 8, 1, 2], 40, [0, 5]), ([0, -1, 1, 2], 40, [0, 5]),
                                 ([0, 1, 2, 3], 65, [0, 4]), ([0, 1, 2, 3], 64, [0, 5])):
        t, n, ring, st = ints([[[table]]]), ints([[[length]]]), ints(list(range(8))), ints(state)
        cache.release(ints([1]), n, t, ring, st)
        with pytest.raises(bacon.BaconError) as e:
            cache.sync()
        assert e.value.status == bacon.BACON_EINVAL
        assert t.flatten().tolist() == table and n.item() == length and st.tolist() == state


# ------------------------------------------------------------- store, load

def check_pages(cache, pages, slots, rows_kv):
    """Every stored row as the reference holds it, exactly."""
    k, v = cache.load(slots)
    raw = []
    for codes, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        at = slots.long().clamp(min=0)
        x = ref.value(codes.view(-1, cache.head_dim)[at].cpu(), cache.format)
        raw.append(x * scale[at // cache.page].double().cpu()[:, None])
    cache.sync()
    live = (slots >= 0).cpu()
    for got, held, out in zip(raw, pages, (k, v)):
        want = held.load(slots.tolist())
        torch.testing.assert_close(got[live], want[live], rtol=0, atol=0, equal_nan=True)
        torch.testing.assert_close(out.cpu(), want.to(cache.dtype), rtol=0, atol=0,
                                   equal_nan=True)


def odd_rows(n, d, dtype, gen):
    """Rows of very different sizes, ties of the rounding among them, some with
    values that are not finite."""
    x = torch.randn(n, d, generator=gen) * torch.exp(2 * torch.randn(n, 1, generator=gen))
    x[n // 2] = torch.arange(d) * 0.25 - 3
    x[n // 3, 5], x[n // 3, 6], x[n // 3, 7] = float("inf"), float("nan"), -float("inf")
    return x.to(dtype)


@pytest.mark.parametrize("format", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_store_appends_and_grows_scales(format, dtype, d, page):
    gen = torch.Generator().manual_seed(page + d)
    H, dt = 3, DTYPES[dtype]
    cache = bacon.Cache(1, H, H, d, 40, page=page, format=format, dtype=dt, max_requests=2,
                        max_blocks=8)
    cache.k.fill_(0x7F), cache.v.fill_(0xFF)  # what nobody wrote is NaN or a large code
    pages = [ref.Pages(format, page, d) for _ in range(2)]
    lengths, table, ring, state = cache.tables(2)
    for step, added in enumerate(([5, 1], [1, 1], [page, 2 * page + 3], [0, 7], [1, 1], [2, page - 1])):
        T = sum(added)
        slots, lengths, state = cache.plan(lengths, ints(added), table, ring, state, T)
        fused = torch.empty(T, 2 + 2 * H + 1, d, dtype=dt, device="cuda")
        for i in range(2):
            x = odd_rows(T * H, d, dt, gen).view(T, H, d) * (4.0 ** step if step % 2 else 0.1)
            fused[:, 2 + i * H:2 + (i + 1) * H] = x.cuda()
        k, v = fused[:, 2:2 + H], fused[:, 2 + H:2 + 2 * H]
        cache.store(k, v, slots[0])
        for h in range(H):
            # a unit's rows of one call follow one another
            mine = slots[0, :, h].tolist()
            for held, x in zip(pages, (k, v)):
                held.store(x[:, h].cpu(), mine)
        every = cache.locate(lengths, table, int(lengths.sum()))
        check_pages(cache, pages, every, (k, v))


@pytest.mark.parametrize("format", ["e4m3", "int8"])
def test_store_of_flat_rows_and_of_nothing(format):
    gen = torch.Generator().manual_seed(4)
    cache = bacon.Cache(2, 2, 2, 128, 30, page=32, format=format, max_requests=3, max_blocks=4)
    lengths, table, ring, state = cache.tables(3)
    added = ints([[[0, 33], [1, 64]], [[100, 0], [31, 32]], [[2, 3], [65, 1]]])
    total = int(added.sum())
    slots, lengths, state = cache.plan(lengths, added, table, ring, state, total + 9)
    k, v = (odd_rows(total + 9, 128, torch.bfloat16, gen).cuda() for _ in range(2))
    k[3] = 0
    cache.store(k, v, slots)  # the last nine rows have no slot
    pages = [ref.Pages(format, 32, 128) for _ in range(2)]
    for held, x in zip(pages, (k, v)):
        held.store(x[:total].cpu(), slots[:total].tolist())
    check_pages(cache, pages, slots, (k, v))
    before = cache.k.clone()
    cache.store(k[:0], v[:0], slots[:0])
    cache.store(k[:9], v[:9], slots[total:])
    cache.sync()
    assert torch.equal(before, cache.k)
    out = cache.load(slots[:0])
    assert out[0].shape == (0, 128)


@pytest.mark.parametrize("format", ["e4m3", "int8"])
@pytest.mark.parametrize("x", [0.0, 1e-38, 2.0 ** -60, 448.0, 449.0, 127.0, 1e38, 3.3e38,
                               2.0 ** -53, 1.75, 1.76171875, float("nan"), float("inf")])
def test_store_at_the_scales_edges(format, x):
    cache = bacon.Cache(1, 1, 1, 64, 2, page=16, format=format, max_requests=1, max_blocks=1)
    rows = torch.full((16, 64), x).to(torch.bfloat16)
    rows[1:, ::2] *= -0.37
    rows = rows.cuda()
    slots = ints(list(range(16, 32)))
    cache.store(rows, rows, slots)
    pages = [ref.Pages(format, 16, 64) for _ in range(2)]
    for held in pages:
        held.store(rows.cpu(), slots.tolist())
    check_pages(cache, pages, slots, None)


@pytest.mark.parametrize("slot", [-2, 64, 2 ** 31 - 1, -2 ** 31])
def test_bad_slots_are_reported_and_skipped(slot):
    cache = bacon.Cache(1, 1, 1, 64, 4, page=16, max_requests=1, max_blocks=1)
    cache.k.zero_(), cache.v.zero_()
    rows = torch.ones(3, 64, dtype=torch.bfloat16, device="cuda")
    for call in (lambda: cache.store(rows, rows, ints([0, slot, 32])),
                 lambda: cache.load(ints([0, slot, 32]))):
        out = call()
        with pytest.raises(bacon.BaconError) as e:
            cache.sync()
        assert e.value.status == bacon.BACON_EINVAL
    assert out[0][:, 0].tolist() == [1, 0, 1]
    assert int((cache.k != 0).sum()) == 128


# ------------------------------------------------------------------ attend

def fill(cache, gen, poison=True):
    """Random codes; what lies beyond the units' tokens is poisoned later."""
    dev = "cuda"
    n = cache.pages
    for codes, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        x = torch.randn(n, cache.page, cache.head_dim, generator=gen, device=dev)
        x *= torch.exp(0.5 * torch.randn(n, cache.page, 1, generator=gen, device=dev))
        if cache.format == "e4m3":
            s = 2.0 ** torch.randint(-8, 0, (n,), generator=gen, device=dev).float()
            codes.copy_((x / s[:, None, None]).clamp(-448, 448).to(torch.float8_e4m3fn)
                        .view(torch.uint8))
        else:
            s = x.abs().amax((1, 2)) / 127
            codes.copy_((x / s[:, None, None]).round().to(torch.int8).view(torch.uint8))
        scale.copy_(s)


def poison(cache, table, lengths, layer):
    """NaN (or the lowest code) in every row that no unit of the layer holds,
    NaN in every other page's scale."""
    used = torch.zeros(cache.pages * cache.page, dtype=torch.bool, device="cuda")
    live = torch.zeros(cache.pages, dtype=torch.bool, device="cuda")
    for r in range(lengths.shape[0]):
        for h in range(lengths.shape[2]):
            n = int(lengths[r, layer, h])
            pos = torch.arange(n, device="cuda")
            page = table[r, layer, h].long()[pos // cache.page]
            used[page * cache.page + pos % cache.page] = True
            live[page] = True
    code = 0x7F if cache.format == "e4m3" else 0x80
    for codes, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        codes.view(-1, cache.head_dim)[~used] = code
        scale[~live] = float("nan")


def check_attend(cache, q, lengths, table, layer, asked, causal, scale, out, lse):
    R, H = lengths.shape[0], cache.kv_heads
    G, p, d = cache.q_heads // H, cache.page, cache.head_dim
    u = 2.0 ** -8 if cache.dtype is torch.bfloat16 else 2.0 ** -11
    tiny = 2.0 ** -25 if cache.dtype is torch.float16 else 0.0
    scale = 1 / math.sqrt(d) if scale is None else scale
    t = 0
    for r in range(R):
        a = asked[r]
        for h in range(H):
            n = int(lengths[r, layer, h])
            page = table[r, layer, h, :-(-n // p)].long()
            k, v = ((ref.value(c[page], cache.format) * s[page].double()[:, None, None])
                    .reshape(-1, d)[:n] for c, s in ((cache.k, cache.k_scale),
                                                     (cache.v, cache.v_scale)))
            size = cache.v_scale[page].double().repeat_interleave(p)[:n]
            j = torch.arange(a, device="cuda")
            seen = n - a + j + 1 if causal else torch.full_like(j, n)
            o, z, A, S, w = ref.attend(q[t:t + a, h * G:(h + 1) * G].double().transpose(0, 1), k,
                                       v, seen, scale, size)
            got = out[t:t + a, h * G:(h + 1) * G].double().transpose(0, 1)
            bound = (u * o.abs() + tiny + (2.0 ** -11 + 2.0 ** -15 * S[..., None]) * A
                     + 2.0 ** -30 * n * w[..., None])
            off = (got - o).abs()
            assert bool((off <= bound).all()), (r, h, n, a, float((off - bound).max()),
                                                float(off.max()))
            if lse is not None:
                got = lse[t:t + a, h * G:(h + 1) * G].double().T
                empty = z.isinf()
                assert torch.equal(got.isinf() & (got < 0), empty)
                off = torch.where(empty, 0, (got - z)).abs()
                assert bool((off <= 2.0 ** -16 * S + 2.0 ** -20 * (1 + torch.where(empty, 0, z)
                                                                   .abs())).all()), (r, h, n, a)
        t += a


def run_attend(R, Hq, H, d, page, format, dtype, lengths, asked, causal=True, L=1, layer=0,
               scale=None, lse=True, seed=0, pages=None):
    """lengths: list of [H] per request (the new tokens among them)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = torch.zeros(R, L, H, dtype=torch.int32)
    n[:, layer] = torch.tensor(lengths, dtype=torch.int32)
    blocks = max(1, -(-int(n.max()) // page))
    need = int(((n + page - 1) // page).sum())
    cache = bacon.Cache(L, H, Hq, d, pages or need + 2, page=page, format=format,
                        dtype=DTYPES[dtype], max_requests=R, max_blocks=blocks)
    fill(cache, gen)
    table = shuffled(cache, R, n, seed + 1)[0].cuda()
    poison(cache, table, n, layer)
    T = sum(asked)
    fused = torch.randn(T, Hq + 3, d, generator=gen, device="cuda").to(cache.dtype)
    q = fused[:, 2:2 + Hq]
    starts = None
    if len(set(asked)) > 1 or seed % 2:
        starts = ints([sum(asked[:i]) for i in range(R + 1)])
    got = cache.attend(layer, q, n.cuda(), table, starts=starts, causal=causal, scale=scale,
                       lse=lse or None)
    cache.sync()
    out, z = got if lse else (got, None)
    check_attend(cache, q, n, table, layer, asked, causal, scale, out, z)
    return cache, q, n, table, out, z


HEADS = [(4, 4), (28, 4), (32, 8), (2, 1), (16, 1), (12, 2), (33, 1)]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("format", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d,page", [(64, 16), (64, 64), (128, 16), (128, 32), (128, 64), (128, 128)])
def test_attend_one_token(heads, format, dtype, d, page):
    Hq, H = heads
    around = [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 200, 255, 256, 257, 300, 511, 700]
    R = 5
    lengths = [[around[(7 * r + 3 * h + d + page) % len(around)] for h in range(H)] for r in range(R)]
    run_attend(R, Hq, H, d, page, format, dtype, lengths, [1] * R, seed=page + Hq)


@pytest.mark.parametrize("asked", [[0, 1, 3], [2, 2, 2], [5, 17, 1], [40, 1, 9], [129, 64, 200],
                                   [1, 300, 0]])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,d,page,format,dtype", [
    ((28, 4), 128, 64, "e4m3", "bf16"), ((4, 4), 64, 16, "int8", "fp16"),
    ((12, 2), 64, 32, "e4m3", "fp16"), ((8, 1), 128, 16, "int8", "bf16"),
    ((32, 8), 128, 128, "e4m3", "bf16"), ((6, 2), 128, 32, "int8", "fp16")])
def test_attend_several_tokens(asked, causal, heads, d, page, format, dtype):
    Hq, H = heads
    gen = torch.Generator().manual_seed(sum(asked))
    lengths = [[asked[r] + int(torch.randint(0, 260, (1,), generator=gen)) for _ in range(H)]
               for r in range(3)]
    run_attend(3, Hq, H, d, page, format, dtype, lengths, asked, causal=causal, L=3, layer=1,
               seed=sum(asked))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("asked", [[1, 1, 1, 1], [4, 4, 4, 4], [70, 33, 129, 2]])
@pytest.mark.parametrize("d,format", [(64, "int8"), (128, "e4m3")])
def test_queries_that_see_nothing(causal, asked, d, format):
    """Units of no tokens at all, and causal queries before a unit's first."""
    lengths = [[0, 1, 3], [0, 0, 0], [2, 40, 17], [1, 0, 0]]
    *_, out, lse = run_attend(4, 6, 3, d, 16, format, "bf16", lengths, asked, causal=causal, seed=3)
    assert bool(torch.isfinite(out).all())


@pytest.mark.parametrize("scale", [1.0, 0.01, 3.7])
@pytest.mark.parametrize("asked", [1, 50])
def test_attend_takes_a_scale(scale, asked):
    run_attend(2, 8, 2, 64, 32, "int8", "bf16", [[77, 300]] * 2, [asked] * 2, scale=scale, lse=False)


@pytest.mark.parametrize("asked,lengths", [([1], [[40000, 39999]]), ([3], [[70001, 5]]),
                                           ([200], [[20011, 300]]), ([1] * 3, [[1, 50000]] * 3)])
@pytest.mark.parametrize("format", ["e4m3", "int8"])
def test_attend_long(asked, lengths, format):
    run_attend(len(asked), 14, 2, 128, 64, format, "bf16", lengths, asked, seed=11)


def test_attend_is_the_same_every_time():
    for asked, lengths in (([1] * 6, [[5000, 77, 1800]] * 6), ([90] * 2, [[3000, 100, 90]] * 2)):
        cache, q, n, table, out, lse = run_attend(len(asked), 21, 3, 128, 32, "e4m3", "bf16",
                                                  lengths, asked)
        for _ in range(5):
            again, z = cache.attend(0, q, n.cuda(), table, lse=True)
            assert torch.equal(again, out) and torch.equal(z, lse)
        cache.sync()


@pytest.mark.parametrize("asked", [1, 130])
def test_values_and_scales_of_extreme_size(asked):
    """Pages whose V scales differ by 2^60, rows of the largest logits, queries
    near the ends of fp16's range."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    cache = bacon.Cache(1, 1, 4, 64, 20, page=16, format="e4m3", dtype=torch.bfloat16,
                        max_requests=1, max_blocks=20)
    fill(cache, gen)
    cache.v_scale.copy_(2.0 ** torch.linspace(-50, 10, 20).round())
    cache.k_scale.copy_(2.0 ** torch.linspace(-12, 3, 20).round())
    table = torch.randperm(20, generator=torch.Generator().manual_seed(2)).int().cuda().view(1, 1, 1, 20)
    n = ints([[[19 * 16 + 5]]])
    poison(cache, table, n, 0)
    q = torch.randn(asked, 4, 64, generator=gen, device="cuda")
    q[:, 1] *= 1e-7
    q[:, 2] *= 1e4
    q[:, 3, 1:] *= 1e-9
    q = q.to(torch.bfloat16)
    out, lse = cache.attend(0, q, n, table, lse=True, scale=0.01)
    cache.sync()
    check_attend(cache, q, n.cpu(), table, 0, [asked], True, 0.01, out, lse)


@pytest.mark.parametrize("asked", [1, 40])
def test_nan_reaches_only_the_rows_that_see_it(asked):
    cache, q, n, table, out, lse = run_attend(2, 4, 2, 64, 16, "e4m3", "fp16", [[50, 60], [47, 90]],
                                              [asked] * 2, seed=5)
    t = int(table[0, 0, 1, (60 - 1) // 16]) * 16 + (60 - 1) % 16  # the last token of a unit
    q = q.clone()
    for codes in (cache.k, cache.v):
        kept = codes.clone()
        codes.view(-1, 64)[t, 9] = 0x7F
        again, z = cache.attend(0, q, n.cuda(), table, lse=True)
        hit = torch.zeros(2 * asked, 4, dtype=torch.bool, device="cuda")
        hit[asked - 1, 2:] = True
        assert torch.equal(again.isnan().any(-1), hit)
        assert torch.equal(again[~hit], out[~hit])
        codes.copy_(kept)
    q[0, 0, 3] = float("nan")
    again, z = cache.attend(0, q, n.cuda(), table, lse=True)
    hit = torch.zeros(2 * asked, 4, dtype=torch.bool, device="cuda")
    hit[0, 0] = True
    assert torch.equal(again.isnan().any(-1), hit) and torch.equal(z.isnan(), hit)
    cache.sync()


def test_pools_beyond_32_bits():
    """A pool of more than 2^32 bytes: pages at its end."""
    pages = (1 << 32) // (128 * 128) + 40
    cache = bacon.Cache(1, 1, 4, 128, pages, page=128, format="int8", max_requests=1, max_blocks=3)
    gen = torch.Generator(device="cuda").manual_seed(1)
    table = ints([[[[pages - 1, 1, pages - 33]]]])
    n = 300
    k, v = (torch.randn(n, 128, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    slots = cache.locate(ints([[[n]]]), table, n)
    cache.store(k, v, slots)
    held = [ref.Pages("int8", 128, 128) for _ in range(2)]
    for h, x in zip(held, (k, v)):
        h.store(x.cpu(), slots.tolist())
    check_pages(cache, held, slots, None)
    for asked in (1, 70):
        q = torch.randn(asked, 4, 128, generator=gen, device="cuda").to(torch.bfloat16)
        out, lse = cache.attend(0, q, ints([[[n]]]), table, lse=True)
        cache.sync()
        check_attend(cache, q, torch.tensor([[[n]]]), table, 0, [asked], True, None, out, lse)


@pytest.mark.parametrize("what", ["page", "negative page", "length", "negative length", "starts",
                                  "end of starts"])
@pytest.mark.parametrize("asked", [1, 60])
def test_bad_indexes_are_reported(what, asked):
    cache, q, n, table, out, lse = run_attend(2, 4, 2, 64, 16, "e4m3", "bf16", [[70, 80]] * 2,
                                              [asked] * 2)
    n, table, starts = n.cuda(), table.clone(), ints([0, asked, 2 * asked])
    if what == "page":
        table[1, 0, 0, 2] = cache.pages
    elif what == "negative page":
        table[0, 0, 1, 0] = -1
    elif what == "length":
        n[0, 0, 0] = cache.max_blocks * 16 + 1
    elif what == "negative length":
        n[0, 0, 0] = -5
    elif what == "starts":
        starts[1] = 5 * asked
    else:
        starts[2] = 2 * asked + 1
    cache.attend(0, q, n, table, starts=starts)
    with pytest.raises(bacon.BaconError) as e:
        cache.sync()
    assert e.value.status == bacon.BACON_EINVAL
    # the handle is usable afterwards
    again, z = cache.attend(0, q, ints([[[70, 80]]] * 2), table.copy_(_table_of(cache)), lse=True)
    cache.sync()


def _table_of(cache):
    n = torch.full((2, 1, 2), 70, dtype=torch.int32)
    n[:, :, 1] = 80
    return shuffled(cache, 2, n, 1)[0].cuda()


# ------------------------------------------------- streams, graphs, refusals

def test_another_stream_and_a_graph():
    """The calls of a step on a stream of their own, then captured and replayed
    on other inputs."""
    cache = bacon.Cache(2, 2, 8, 64, 64, page=16, max_requests=3, max_blocks=6)
    lengths, table, ring, state = cache.tables(3)
    gen = torch.Generator(device="cuda").manual_seed(8)
    first = ints([[[20, 33], [1, 40]]] * 3)
    total = int(first.sum())
    slots, lengths, state = cache.plan(lengths, first, table, ring, state, total)
    rows = [torch.randn(total, 64, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2)]
    cache.store(*rows, slots)
    cache.sync()
    x = torch.randn(3, 8 + 4, 64, generator=gen, device="cuda").to(torch.bfloat16)
    outs = dict(slots=torch.empty(2, 3, 2, dtype=torch.int32, device="cuda"),
                lengths_out=torch.empty_like(lengths), state_out=torch.empty_like(state))
    out = [torch.empty(3, 8, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]

    def step(stream=None):
        s, n, _ = cache.plan(lengths, None, table, ring, state, 3, stream=stream, **outs)
        for l in range(2):
            cache.store(x[:, 8:10], x[:, 10:], s[l], stream=stream)
            cache.attend(l, x[:, :8], n, table, out=out[l], stream=stream)

    step()
    torch.cuda.synchronize()
    want = [o.clone() for o in out]
    side = torch.cuda.Stream()
    for o in out:
        o.zero_()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    cache.sync(side)
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for o in out:
        o.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    x.mul_(0.5)
    graph.replay()
    torch.cuda.synchronize()
    got = [o.clone() for o in out]
    step()
    cache.sync()
    assert all(torch.equal(a, b) for a, b in zip(out, got))


def test_refusals():
    cache = bacon.Cache(2, 2, 8, 64, 16, page=16, max_requests=2, max_blocks=4)
    lengths, table, ring, state = cache.tables(2)
    q = torch.zeros(2, 8, 64, dtype=torch.bfloat16, device="cuda")
    kv = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    one = ints([1, 1])

    def refused(call, error=bacon.BaconError):
        with pytest.raises(error):
            call()

    refused(lambda: bacon.Cache(2, 2, 8, 64, 16, format="int4"), ValueError)
    refused(lambda: bacon.Cache(2, 2, 8, 64, 16, dtype=torch.float32), ValueError)
    refused(lambda: bacon.Cache(2, 2, 8, 64, 16, page=16, k=torch.empty(16, 16, 64, device="cuda")),
            ValueError)
    refused(lambda: bacon.Cache(2, 2, 7, 64, 16))
    refused(lambda: bacon.Cache(2, 2, 8, 80, 16))
    refused(lambda: cache.plan(lengths.long(), one, table, ring, state, 2), ValueError)
    refused(lambda: cache.plan(lengths, one, table[:1], ring, state, 2), ValueError)
    refused(lambda: cache.plan(lengths, one, table, ring[:5], state, 2), ValueError)
    refused(lambda: cache.plan(lengths, one, table, ring, state, 2, lengths_out=lengths))
    refused(lambda: cache.plan(lengths, one, table, ring, state, 2, state_out=state))
    refused(lambda: cache.plan(*bacon.Cache.tables(cache, 3)[:1], None, cache.tables(3)[1], ring,
                               state, 3))
    refused(lambda: cache.store(kv.float(), kv.float(), ints([0] * 4)), ValueError)
    refused(lambda: cache.store(kv, kv[:3], ints([0] * 4)), ValueError)
    refused(lambda: cache.store(kv.t().contiguous().t(), kv, ints([0] * 4)), ValueError)
    refused(lambda: cache.store(kv, kv, ints([0] * 3)), ValueError)
    odd = torch.zeros(4 * 65 + 8, dtype=torch.bfloat16, device="cuda")
    refused(lambda: cache.store(odd[:4 * 65].view(4, 65)[:, :64], kv, ints([0] * 4)))
    refused(lambda: cache.store(odd[4:260].view(4, 64), kv, ints([0] * 4)))
    refused(lambda: cache.load(ints([0, 1]), k_out=kv), ValueError)
    refused(lambda: cache.attend(2, q, lengths, table))
    refused(lambda: cache.attend(-1, q, lengths, table))
    refused(lambda: cache.attend(0, q[:1], lengths, table))
    refused(lambda: cache.attend(0, q[:, :4], lengths, table), ValueError)
    refused(lambda: cache.attend(0, q.float(), lengths, table), ValueError)
    refused(lambda: cache.attend(0, q, lengths, table, scale=float("nan")))
    refused(lambda: cache.attend(0, q, lengths, table, scale=-1.0))
    refused(lambda: cache.attend(0, q, lengths, table, starts=ints([0, 1])), ValueError)
    refused(lambda: cache.attend(0, q, lengths, table, lse=torch.empty(2, 8, device="cuda",
                                                                       dtype=torch.float64)), ValueError)
    out = cache.attend(0, q[:0], lengths, table)
    assert out.shape == (0, 8, 64)
    cache.sync()
    cache.close()
    refused(lambda: cache.sync())


@pytest.mark.parametrize("format,most", [("e4m3", 0.05), ("int8", 0.02)])
def test_the_example_serves_kept_rows(format, most):
    """Codes are off by a sixteenth (e4m3: 2^-4 of the value) or a 127th of the
    page's largest at most, half of that on average or less, and the softmax
    averages the values' part of it."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                        "serve_kept_rows.py")
    spec = importlib.util.spec_from_file_location("serve_kept_rows", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    assert mod.main(format) < most
