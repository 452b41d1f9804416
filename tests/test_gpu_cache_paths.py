"""The cache's kernels on calls whose blocks have several items, or runs, each.

Attention is held to the bounds of test_gpu_cache.py, with the term for weights
below fp16's least step by kernel.  The few-query kernel holds a row's weights
with the largest at 2^14: one is off by 2^-25 at least steps of 2^-24, 2^-39 of
the largest, times a code of at most 448 < 2^9 for each of n tokens: 2^-30 n
max(p v_scale) / sum p.  In the many-query kernel a row's reference follows its
maximum once that has grown by 2^8, so the largest lies between 2^7 and 2^15 and
the term is up to 2^7 larger: 2^-23 n max(p v_scale) / sum p.  Codes and scales
are exact."""

import math

import pytest
import torch

import cache_reference as ref
from paper_2606_14782_gb300 import bacon, build
from test_gpu_cache import check_pages, fill, ints, shuffled

pytestmark = pytest.mark.gpu

FEW = 32  # rows of a request, on average, up to which the few-query kernel has the call


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    bacon.load()


def reference(cache, q, lengths, table, asked, causal):
    """In 64 bits, all units at once: out, lse, and for each output what bounds
    its error: sum p |v|, the largest sum |q k| scale, n max(p v_scale)."""
    R, H, p, d = lengths.shape[0], cache.kv_heads, cache.page, cache.head_dim
    G, n = cache.q_heads // H, lengths[:, 0].long()
    page = table[:, 0].clamp(min=0).long()
    k, v = (ref.value(c[page], cache.format) * s[page].double()[..., None, None]
            for c, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))
    k, v = (x.reshape(R, H, -1, d) for x in (k, v))
    size = cache.v_scale[page].double().repeat_interleave(p, dim=-1)
    pos = torch.arange(k.shape[2], device="cuda")
    none = (pos >= n[..., None])
    # (whatever lies beyond a unit's tokens stands for nothing)
    k, v = (x.masked_fill(none[..., None], 0) for x in (k, v))
    size = size.masked_fill(none, 0)
    most, a = max(max(asked), 1), torch.tensor(asked, device="cuda")
    j = torch.arange(most, device="cuda")
    start = a.cumsum(0) - a
    token = (start[:, None] + j).clamp(max=q.shape[0] - 1)
    x = q[token].double().view(R, most, H, G, d).permute(0, 2, 3, 1, 4)  # [R, H, G, Q, d]
    sees = (n[..., None] - a[:, None, None] + j + 1 if causal else n[..., None].expand(R, H, most))
    hidden = (pos >= sees[..., None])[:, :, None]  # [R, H, 1, Q, N]
    scale = 1 / math.sqrt(d)
    logits = (torch.einsum("rhgqd,rhnd->rhgqn", x, k) * scale).masked_fill(hidden, float("-inf"))
    lse = torch.logsumexp(logits, dim=-1)
    empty = (sees <= 0)[:, :, None].expand_as(lse)
    w = torch.where(empty[..., None], 0, torch.exp(logits - lse[..., None]))
    S = (torch.einsum("rhgqd,rhnd->rhgqn", x.abs(), k.abs()) * scale).masked_fill(hidden, 0).amax(-1)
    out = torch.einsum("rhgqn,rhnd->rhgqd", w, v)
    A = torch.einsum("rhgqn,rhnd->rhgqd", w, v.abs())
    low = n[..., None, None] * (w * size[:, :, None, None]).amax(-1)
    inside = j < a[:, None]

    def rows(t):  # [R, H, G, Q, ...] -> [tokens, Hq, ...]
        t = t.permute(0, 3, 1, 2, *range(4, t.dim()))
        return t.reshape(R, most, H * G, *t.shape[4:])[inside]

    return [rows(t) for t in (out, torch.where(empty, float("-inf"), lse), A, S, low)]


def check(cache, q, lengths, table, asked, causal, out, lse, many, nan=None):
    """nan [tokens, Hq]: the outputs that see a NaN (which the reference, given
    the codes without it, does not know of)."""
    want, z, A, S, low = reference(cache, q, lengths, table, asked, causal)
    u = 2.0 ** -8 if cache.dtype is torch.bfloat16 else 2.0 ** -11
    tiny = 2.0 ** -25 if cache.dtype is torch.float16 else 0.0
    bound = (u * want.abs() + tiny + (2.0 ** -11 + 2.0 ** -15 * S[..., None]) * A
             + 2.0 ** (-23 if many else -30) * low[..., None])
    off = (out.double() - want).abs()
    fine = (off <= bound).all(-1)
    empty = z.isinf()
    off = torch.where(empty, 0, (lse.double() - z).abs())
    close = off <= 2.0 ** -16 * S + 2.0 ** -20 * (1 + torch.where(empty, 0, z).abs())
    close &= (lse.isinf() & (lse < 0)) == empty
    if nan is None:
        assert bool(fine.all()) and bool(close.all())
    else:
        assert torch.equal(out.isnan().any(-1), nan)
        assert bool((fine | nan).all()) and bool(close.all())


def setting(R, H, G, d, page, format, dtype, lengths, asked, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = torch.tensor(lengths, dtype=torch.int32).view(R, 1, H)
    blocks = max(1, -(-int(n.max()) // page))
    cache = bacon.Cache(1, H, H * G, d, int(((n + page - 1) // page).sum()) + 5, page=page,
                        format=format, dtype=ref.DTYPES[dtype], max_requests=R, max_blocks=blocks)
    fill(cache, gen)
    table = shuffled(cache, R, n, seed)[0].cuda()
    # what no unit holds is NaN, or the lowest code
    pos = torch.arange(blocks * page, device="cuda")
    held = (pos < n.cuda()[..., None]).view(R, 1, H, blocks, page)
    used = torch.zeros(cache.pages, page, dtype=torch.bool, device="cuda")
    used[table[table >= 0].long()] = held[table >= 0]
    for codes, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        codes[~used] = 0x7F if format == "e4m3" else 0x80
        scale[~used.any(1)] = float("nan")
    q = torch.randn(sum(asked), H * G, d, generator=gen, device="cuda").to(cache.dtype)
    starts = None
    if len(set(asked)) > 1:
        starts = ints([sum(asked[:i]) for i in range(R + 1)])
    return cache, q, n.cuda(), table, starts


def sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


# kv-heads 16; (requests, query heads a kv-head, queries of a request): the
# columns of the few-query kernel's forms, or rows of the many-query kernel's items
FORMS = {"8 columns": (150, 2, [4]), "16 columns": (100, 4, [3]), "32 columns": (50, 8, [4]),
         "ragged, 32 columns": (60, 3, [0, 1, 18, 7, 3]), "one token": (150, 1, [1]),
         "160 rows": (50, 4, [40]), "ragged rows": (60, 4, [0, 1, 100, 33, 70, 64])}


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("d,page,format,dtype", [(64, 16, "e4m3", "fp16"), (128, 64, "int8", "bf16"),
                                                 (128, 16, "e4m3", "bf16"), (64, 32, "int8", "fp16")])
@pytest.mark.parametrize("causal", [True, False])
def test_blocks_of_several_items(form, d, page, format, dtype, causal):
    R, G, pattern = FORMS[form]
    H, gen = 16, torch.Generator().manual_seed(R + d)
    asked = [pattern[r % len(pattern)] for r in range(R)]
    rows = sum(asked) * G
    many = rows // R > FEW
    grid = sms() * (1 if many or rows // R > 16 else 2 if rows // R > 8 else 3)
    width = 256 if many else 8 if rows // R <= 8 else 16 if rows // R <= 16 else 32
    items = sum(-(-a * G // width) for a in asked) * H
    assert items >= 5 * grid
    # short units of every kind, a fifth of them empty
    lengths = torch.randint(0, 260, (R * H,), generator=gen)
    lengths[torch.rand(R * H, generator=gen) < 0.2] = 0
    cache, q, n, table, starts = setting(R, H, G, d, page, format, dtype, lengths.tolist(), asked, 1)
    out, lse = cache.attend(0, q, n, table, starts=starts, causal=causal, lse=True)
    again, z = cache.attend(0, q, n, table, starts=starts, causal=causal, lse=True)
    cache.sync()
    assert torch.equal(again, out) and torch.equal(z, lse)
    check(cache, q, n, table, asked, causal, out, lse, many)


@pytest.mark.parametrize("form", ["8 columns", "16 columns", "32 columns", "160 rows"])
@pytest.mark.parametrize("d", [64, 128])
def test_a_nan_stays_with_its_item(form, d):
    """NaN in V at the last token of every seventh unit: the last query sees it,
    those before it do not, and no later item of the block knows of it."""
    R, G, pattern = FORMS[form]
    H, gen = 16, torch.Generator().manual_seed(5)
    asked = [pattern[0]] * R
    lengths = torch.randint(pattern[0], 260, (R * H,), generator=gen)
    cache, q, n, table, _ = setting(R, H, G, d, 16, "e4m3", "bf16", lengths.tolist(), asked, 2)
    want, lse = cache.attend(0, q, n, table, lse=True)
    clean = cache.v.clone()
    nan = torch.zeros(sum(asked), H, G, dtype=torch.bool, device="cuda")
    for u in range(0, R * H, 7):
        r, h, at = u // H, u % H, int(lengths[u]) - 1
        cache.v[int(table[r, 0, h, at // 16]), at % 16, u % d] = 0x7F
        nan[(r + 1) * asked[0] - 1, h] = True
    out, z = cache.attend(0, q, n, table, lse=True)
    cache.sync()
    nan = nan.view(-1, H * G)
    assert torch.equal(out.isnan().any(-1), nan) and torch.equal(z, lse)
    assert torch.equal(out[~nan], want[~nan])
    # one dim of a row, and the others as they were
    assert torch.equal(out.isnan().sum(-1), nan.long())
    assert torch.equal(out[~out.isnan()], want[~out.isnan()])
    cache.v.copy_(clean)
    check(cache, q, n, table, asked, True, want, lse, form == "160 rows")


# ------------------------------------------------------------------- store

def odd(n, d, dtype, gen):
    """Rows of very different sizes; one in forty holds an infinity or NaN."""
    x = torch.randn(n, d, generator=gen) * torch.exp(2 * torch.randn(n, 1, generator=gen))
    for i in range(3, n, 40):
        x[i, i % d] = (float("inf"), float("nan"), -float("inf"))[i // 40 % 3]
    return x.to(ref.DTYPES[dtype])


@pytest.mark.parametrize("format", ["e4m3", "int8"])
@pytest.mark.parametrize("d,page,units,most", [(64, 16, 400, 40), (128, 32, 300, 90), (64, 64, 1200, 150),
                                               (64, 128, 1200, 300)])
def test_store_of_several_runs_a_block(format, d, page, units, most):
    """Units' rows one after the other: blocks of many runs, up to a window of a
    page's tokens, in which runs start in any word."""
    gen = torch.Generator().manual_seed(units)
    added = torch.randint(0, most, (1, 1, units), generator=gen, dtype=torch.int32)
    added[0, 0, ::9] = 1
    total = int(added.sum())
    window = total // (152 * 8)
    assert min(window, page) >= (page if most >= 150 else 2)
    need = int(((added + page - 1) // page).sum())
    dtype = "bf16" if d == 128 else "fp16"
    cache = bacon.Cache(1, units, units, d, need + 2, page=page, format=format,
                        dtype=ref.DTYPES[dtype], max_requests=1, max_blocks=-(-most // page))
    cache.k.fill_(0x7F), cache.v.fill_(0xFF)
    lengths, table, ring, state = cache.tables(1)
    slots, lengths, state = cache.plan(lengths, added.cuda(), table, ring, state, total)
    k, v = (odd(total, d, dtype, gen) for _ in range(2))
    cache.store(k.cuda(), v.cuda(), slots)
    pages = [ref.Pages(format, page, d) for _ in range(2)]
    for held, x in zip(pages, (k, v)):
        held.store(x, slots.tolist())
    check_pages(cache, pages, slots, None)


@pytest.mark.parametrize("format", ["e4m3", "int8"])
@pytest.mark.parametrize("d,page,R,H", [(64, 16, 700, 4), (128, 64, 400, 8)])
def test_append_of_several_runs_a_block(format, d, page, R, H):
    """A few tokens of many requests at once: a window's runs append to pages,
    whose older rows are quantised again where the new ones are larger."""
    gen = torch.Generator().manual_seed(R)
    cache = bacon.Cache(1, H, H, d, R * H * 3, page=page, format=format, max_requests=R, max_blocks=3)
    lengths, table, ring, state = cache.tables(R)
    pages = [ref.Pages(format, page, d) for _ in range(2)]
    for step, most in enumerate((page + 3, 4, 5)):
        asked = torch.randint(0, most, (R,), generator=gen, dtype=torch.int32)
        T = int(asked.sum())
        assert T * H >= 2 * 152 * 8  # windows of two tokens and more
        slots, lengths, state = cache.plan(lengths, asked.cuda(), table, ring, state, T)
        fused = torch.empty(T, 3 * H, d, dtype=torch.bfloat16, device="cuda")
        for i in range(2):
            x = odd(T * H, d, "bf16", gen).view(T, H, d) * (8.0 if step == 1 else 0.5)
            fused[:, (1 + i) * H:(2 + i) * H] = x.cuda()
        k, v = fused[:, H:2 * H], fused[:, 2 * H:]
        cache.store(k, v, slots[0])
        for h in range(H):
            mine = slots[0, :, h].tolist()
            for held, x in zip(pages, (k, v)):
                held.store(x[:, h].cpu(), mine)
        every = cache.locate(lengths, table, int(lengths.sum()))
        check_pages(cache, pages, every, None)


# ------------------------------------------------------------ after an error

@pytest.mark.parametrize("what", ["page", "negative page", "length", "negative length"])
@pytest.mark.parametrize("asked", [1, 60])
def test_a_reported_index_leaves_nothing_behind(what, asked):
    """The calls after a refused one, before and after the error is asked for,
    give what they gave before."""
    R, H, G = 3, 2, 4
    lengths = [[2900, 3000], [1, 17], [5000, 400]]
    flat = [n for r in lengths for n in r]
    cache, q, n, table, _ = setting(R, H, G, 64, 16, "e4m3", "bf16", flat, [asked] * R, 3)
    want, lse = cache.attend(0, q, n, table, lse=True)
    cache.sync()
    bad_n, bad = n.clone(), table.clone()
    if what == "page":
        bad[0, 0, 1, 100] = cache.pages
    elif what == "negative page":
        bad[2, 0, 0, 7] = -3
    elif what == "length":
        bad_n[0, 0, 0] = cache.max_blocks * 16 + 1
    else:
        bad_n[2, 0, 0] = -5
    cache.attend(0, q, bad_n, bad)
    out, z = cache.attend(0, q, n, table, lse=True)
    with pytest.raises(bacon.BaconError) as e:
        cache.sync()
    assert e.value.status == bacon.BACON_EINVAL
    assert torch.equal(out, want) and torch.equal(z, lse)
    out, z = cache.attend(0, q, n, table, lse=True)
    cache.sync()
    assert torch.equal(out, want) and torch.equal(z, lse)
