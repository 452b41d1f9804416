"""Measured operators: serving from the rows that a compression kept.

A prompt's kept K/V rows, whose number differs by kv-head when the head budgets
are shared inside a layer, are put in pages of 8-bit values; new tokens are
appended and attend to them.  A unit is one (request, layer, kv-head).  A page
holds `page` tokens of one unit, with one scale for K and one for V.  The
operators (`op`):

  plan    pages for the tokens that each unit is about to get, and the slots of
          these tokens: block tables and slot maps from lengths
  store   rows into their slots, quantised with the scale of their page, which
          grows when an appended row asks for it; and the touched pages back
          as values
  attend  the queries of one layer's new tokens over the units' pages

`own` chooses between the framework's calls and their plain form.
"""

import math

import torch

own = False

FLOOR = 2.0 ** -60  # the least scale of a page
FREE_PAGES = 37     # pages of a pool that nobody uses, at least


# ------------------------------------------------------------------ cases

def _plan(name, requests, layers, kv_heads, page, order, held, new):
    """order "units": `new` rows a unit on average, each unit its own number;
    "tokens": `new` tokens a request, the same in all its units."""
    c = dict(op="plan", requests=requests, layers=layers, kv_heads=kv_heads, page=page,
             order=order, held=held, new=new)
    return dict(c, name=name) if name else c


def _store(name, requests, layers, q_heads, kv_heads, head_dim, page, format, dtype, order, held,
           new):
    c = dict(op="store", requests=requests, layers=layers, q_heads=q_heads, kv_heads=kv_heads,
             head_dim=head_dim, page=page, format=format, dtype=dtype, order=order, held=held,
             new=new)
    return dict(c, name=name) if name else c


def _attend(name, requests, q_heads, kv_heads, head_dim, page, format, dtype, held, new,
            ragged=True, causal=True, layers=1):
    """`held` cached tokens a unit before the `new` ones a request."""
    c = dict(op="attend", requests=requests, layers=layers, q_heads=q_heads, kv_heads=kv_heads,
             head_dim=head_dim, page=page, format=format, dtype=dtype, held=held, new=new,
             ragged=ragged, causal=causal)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one decoding step of the screenshot requests: a token for every unit
        _plan("plan_step", 4, 28, 4, 64, "tokens", 1024, 1),
        # a batch of image prompts whose kept rows differ by head
        _plan("plan_prompts", 16, 32, 32, 64, "units", 0, 256),
        # one layer of a decoding step: a row at the end of each unit's last page
        _store("store_step", 32, 1, 32, 8, 128, 64, "e4m3", "bf16", "tokens", 1000, 1),
        # one layer of a few ragged follow-up turns
        _store("store_turn", 5, 1, 8, 2, 64, 32, "int8", "fp16", "tokens", 333, 700),
        # every kept row of four screenshot prompts
        _store("store_prompts", 4, 28, 28, 4, 128, 64, "e4m3", "bf16", "units", 0, 1024),
        # a toy model's first token: launches and latency are all there is
        _attend("decode_tiny", 1, 4, 4, 64, 16, "e4m3", "bf16", 64, 1, ragged=False, layers=2),
        # a token of four screenshot requests over their kept rows
        _attend("decode_gui", 4, 28, 4, 128, 64, "e4m3", "bf16", 1024, 1),
        # a batch of image requests of a multi-head model: many short units
        _attend("decode_mha", 24, 32, 32, 128, 32, "int8", "fp16", 256, 1),
        # a batch of long prompts that were not compressed: the most bytes
        _attend("decode_batch", 32, 28, 4, 128, 64, "e4m3", "bf16", 16384, 1),
        # four drafted tokens of each request checked at once
        _attend("draft_check", 8, 28, 4, 128, 64, "e4m3", "fp16", 4096, 4),
        # short follow-up turns of ragged length
        _attend("turn_short", 3, 12, 2, 64, 16, "int8", "bf16", 2000, 100),
        # a long follow-up turn over a long prompt: the most operations
        _attend("turn_long", 1, 28, 4, 128, 64, "e4m3", "bf16", 12288, 4096, ragged=False),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


HEADS = ((4, 4), (8, 8), (32, 32), (28, 4), (32, 8), (16, 4), (8, 2), (6, 2), (12, 2))
MOST_SLOTS = 16 * 32 * 32 * 256              # plan_prompts
MOST_ROWS = 4 * 28 * 4 * 1024 * 128          # store_prompts, in elements of K
MOST_CACHED = 32 * 4 * 16384 * 128           # decode_batch, in elements of K
MOST_PAIRS = 28 * 4096 * (12288 + 2048) * 128  # turn_long, in multiplications of q k


def draw(rng):
    while True:
        op = rng.choice(("plan", "store", "store", "attend", "attend", "attend", "attend"))
        q_heads, kv_heads = rng.choice(HEADS)
        head_dim = rng.choice((64, 128, 128))
        page = rng.choice((16, 32, 64, 64, 128))
        format, dtype = rng.choice(("e4m3", "int8")), rng.choice(("bf16", "bf16", "fp16"))
        requests = _log_int(rng, 1, 48)
        if op == "plan":
            layers = rng.randint(1, 32)
            order = rng.choice(("units", "tokens"))
            held = 0 if order == "units" else _log_int(rng, 1, 4096)
            new = _log_int(rng, 1, 2048)
            if requests * layers * kv_heads * (new + held // page) <= MOST_SLOTS // 2:
                return _plan(None, requests, layers, kv_heads, page, order, held, new)
        elif op == "store":
            order = rng.choice(("units", "tokens"))
            layers = rng.randint(1, 32) if order == "units" else 1
            held = 0 if order == "units" else _log_int(rng, 1, 4096)
            new = _log_int(rng, 1, 2048)
            rows = requests * layers * kv_heads * (2 * new + held) * head_dim
            if rows <= MOST_ROWS:
                return _store(None, requests, layers, q_heads, kv_heads, head_dim, page, format,
                              dtype, order, held, new)
        else:
            held = _log_int(rng, 1, 131072)
            new = rng.choice((1, 1, 1, _log_int(rng, 2, 8), _log_int(rng, 9, 4096)))
            ragged = rng.random() < 0.7
            # units are up to 1.7 times as long, requests ask up to twice as much
            longest = (1.7 if ragged else 1) * held + (2 if ragged else 1) * new
            cached = requests * kv_heads * longest * head_dim
            pairs = requests * q_heads * (2 if ragged else 1) * new * longest * head_dim
            if cached <= MOST_CACHED and pairs <= MOST_PAIRS:
                return _attend(None, requests, q_heads, kv_heads, head_dim, page, format, dtype,
                               held, new, ragged=ragged, causal=rng.random() < 0.8,
                               layers=rng.choice((1, 1, 3)))


# ----------------------------------------------------------------- inputs

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _counts(c):
    """(held [R, L, H], new) of a case; new is [R, L, H] for rows in units'
    order and [R] for tokens.  From the sizes alone, on the CPU: the same for
    every seed, so that work() knows them."""
    gen = torch.Generator().manual_seed(7)
    shape = (c["requests"], c["layers"], c["kv_heads"])

    def around(mean, shape, lo, hi):
        spread = lo + (hi - lo) * torch.rand(shape, generator=gen, dtype=torch.float64)
        return (mean * spread).round().to(torch.int64)

    ragged = c.get("ragged", True)
    held = around(c["held"], shape, 0.3, 1.7) if ragged else torch.full(shape, c["held"])
    if c.get("order") == "units":
        # a layer's budget shared by its heads: their counts add up to it
        new = around(c["new"], shape, 0.3, 1.7).clamp(max=c["new"] * c["kv_heads"])
        new[..., -1] = 0
        over = (new.cumsum(-1) - c["new"] * c["kv_heads"]).clamp(min=0)
        new = (new - over).clamp(min=0)
        new[..., -1] = c["new"] * c["kv_heads"] - new.sum(-1)
    elif ragged and c["new"] > 1:
        new = torch.randint(1, 2 * c["new"], (c["requests"],), generator=gen)
    else:
        new = torch.full((c["requests"],), c["new"])
    return held, new


def _after(c, held, new):
    return held + (new if new.dim() == 3 else new[:, None, None])


def _tables(c, lengths, widest, gen, dev):
    """A table [R, L, H, blocks] whose pages lie anywhere in the pool, the ring
    of the pages that nobody uses, and its state {next, count}."""
    p = c["page"]
    blocks = (lengths + p - 1) // p
    width = max(1, -(-int(widest.max()) // p))
    spare = int(((widest + p - 1) // p - blocks).sum()) + FREE_PAGES
    used = int(blocks.sum())
    pages = used + spare
    order = torch.randperm(pages, generator=gen, device=dev).to(torch.int32)
    blocks = blocks.to(dev)
    filled = torch.arange(width, device=dev) < blocks[..., None]
    table = torch.full(filled.shape, -1, dtype=torch.int32, device=dev)
    table[filled] = order[:used]
    # the ring's order starts somewhere in its middle
    start = pages // 3
    ring = torch.cat([order[used:], order[:used]]).roll(start)
    state = torch.tensor([start, spare], dtype=torch.int32, device=dev)
    return table, ring.contiguous(), state, pages


def _slots(table, page, first, count):
    """Slots of the positions [first, first + count) of each unit, one after
    another (plain indexing)."""
    first, count = first.reshape(-1), count.reshape(-1)
    unit = torch.repeat_interleave(torch.arange(count.numel(), device=table.device),
                                   count)
    at = torch.arange(unit.numel(), device=table.device) - (count.cumsum(0) - count)[unit]
    pos = first[unit] + at
    block = table.reshape(first.numel(), -1)[unit, pos // page].long()
    return (block * page + pos % page).int(), unit, at


def _scale(amax, format):
    """The scale of a page from the largest magnitude in it."""
    if format == "e4m3":  # the least power of two with amax <= 448 scale
        m, e = torch.frexp(amax)
        s = (e + 118 + (m > 0.875).int() << 23).view(torch.float32)  # bits of 2^(e - 9), or twice
    else:  # amax / 127, rounded up to eight significant bits
        # (by a tensor: a division by a number may multiply by its reciprocal)
        bits = (amax / torch.full_like(amax, 127)).view(torch.int32)
        s = ((bits + 0xFFFF) & ~0xFFFF).view(torch.float32)
    return torch.where(amax > 0, s, 0).clamp(min=FLOOR)


def _encode(x, scale, format):
    y = x / scale
    if format == "e4m3":
        return y.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    return y.round().clamp(-127, 127).to(torch.int8).view(torch.uint8)


def _decode(codes, format):
    kind = torch.float8_e4m3fn if format == "e4m3" else torch.int8
    return codes.view(kind).float()


def _pool(c, pages, gen, dev):
    """Rows of a cache in 8 bits; the sizes of the rows vary like those of keys."""
    x = torch.randn(pages, c["page"], c["head_dim"], generator=gen, device=dev)
    x *= torch.exp(0.4 * torch.randn(pages, c["page"], 1, generator=gen, device=dev))
    scale = _scale(x.abs().amax(dim=(1, 2)), c["format"])
    return _encode(x, scale[:, None, None], c["format"]), scale


def prepare(case, seed):
    c, dev = case, "cuda"
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    held, new = _counts(c)
    after = _after(c, held, new)
    s = dict(case=c)
    if c["op"] == "plan":
        s["table"], s["free"], s["state"], s["pages"] = _tables(c, held, after, gen, dev)
        s["lengths"], s["added"] = held.int().to(dev), new.int().to(dev)
        s["total"] = int(new.sum())  # the kept rows, or the new tokens, of the batch
        return s
    table, _, _, s["pages"] = _tables(c, after, after, gen, dev)
    s["table"], s["lengths"] = table, after.int().to(dev)
    s["k"], s["k_scale"] = _pool(c, s["pages"], gen, dev)
    s["v"], s["v_scale"] = _pool(c, s["pages"], gen, dev)
    d, H, dt = c["head_dim"], c["kv_heads"], DTYPES[c["dtype"]]
    if c["op"] == "attend":
        s["layer"] = c["layers"] // 2
        s["total"] = int(new.sum())
        q = torch.randn(s["total"], c["q_heads"], d, generator=gen, device=dev)
        s["q"] = q.to(dt)
        # where each request's queries start; equal numbers need no list
        s["starts"] = (torch.nn.functional.pad(new.cumsum(0), (1, 0)).int().to(dev)
                       if c["ragged"] and c["new"] > 1 else None)
        s["longest"], s["most"] = int(after.max()), int(new.max())
        return s
    every = _after(c, torch.zeros_like(held), new)
    slots, unit, at = _slots(table, c["page"], held.to(dev), every.to(dev))
    if c["order"] == "units":
        s["rows_k"], s["rows_v"] = (
            (torch.randn(slots.numel(), d, generator=gen, device=dev)
             * torch.exp(0.4 * torch.randn(slots.numel(), 1, generator=gen, device=dev))).to(dt)
            for _ in range(2))
        s["slots"] = slots
    else:
        # K and V are parts of a fused projection's rows
        total = int(new.sum())
        start = (new.cumsum(0) - new).to(dev)
        s["slots"] = torch.empty(total, H, dtype=torch.int32, device=dev)
        s["slots"][start[unit // H] + at, unit % H] = slots
        rows = torch.randn(total, c["q_heads"] + 2 * H, d, generator=gen, device=dev)
        rows *= torch.exp(0.4 * torch.randn(total, 1, 1, generator=gen, device=dev))
        rows = rows.to(dt)
        s["rows_k"] = rows[:, c["q_heads"]:c["q_heads"] + H]
        s["rows_v"] = rows[:, c["q_heads"] + H:]
    # every row of the pages that get one
    first = held // c["page"] * c["page"]
    s["touched"] = _slots(table, c["page"], first.to(dev), (after - first).to(dev))[0]
    return s


# ----------------------------------------------------------- the plain form

def _plain_plan(s):
    c = s["case"]
    p, shape = c["page"], s["lengths"].shape
    n = s["lengths"].reshape(-1).long()
    per_unit = s["added"].dim() == 3
    a = (s["added"] if per_unit else s["added"][:, None, None].expand(shape)).reshape(-1).long()
    have, want = (n + p - 1) // p, (n + a + p - 1) // p
    need = want - have
    rank = torch.arange(int(s["pages"]), device=n.device)
    start = need.cumsum(0) - need
    unit = torch.searchsorted(start + need, rank, right=True)
    inside = unit < n.numel()
    unit = unit.clamp(max=n.numel() - 1)
    column = have[unit] + rank - start[unit]
    page = s["free"][(s["state"][0].long() + rank) % s["pages"]]
    flat = s["table"].view(n.numel(), -1)
    flat[unit[inside], column[inside]] = page[inside]
    got = need.sum()
    state = torch.stack([(s["state"][0] + got) % s["pages"], s["state"][1] - got]).int()
    out = {"table": s["table"], "lengths": (n + a).int().view(shape), "state": state}
    if per_unit:
        out["slots"] = _slots(s["table"], p, n, a)[0]
        return out
    R, L, H = shape
    slots, unit, at = _slots(s["table"], p, n, a)
    request = unit // (L * H)
    begin = (s["added"].cumsum(0) - s["added"]).long()
    out["slots"] = torch.empty(L, s["total"], H, dtype=torch.int32, device=n.device)
    out["slots"][unit // H % L, begin[request] + at, unit % H] = slots
    return out


def _plain_store(codes, scale, rows, slots, c):
    """The new rows among the older ones of their pages, all quantised anew: a
    page whose scale stays gets the same codes again."""
    p, d, f = c["page"], c["head_dim"], c["format"]
    rows, slots = rows.reshape(-1, d).float(), slots.reshape(-1).long()
    page, inverse = torch.unique(slots // p, return_inverse=True)
    first = torch.full_like(page, p).scatter_reduce(0, inverse, slots % p, "amin")
    amax = rows.new_zeros(page.numel()).scatter_reduce(0, inverse, rows.abs().amax(-1), "amax")
    s = torch.where(first > 0, scale[page], 0).maximum(_scale(amax, f))
    x = _decode(codes[page], f) * scale[page][:, None, None]
    x[inverse, slots % p] = rows
    codes[page] = _encode(x, s[:, None, None], f)
    scale[page] = s


def _plain_load(codes, scale, slots, c):
    p = c["page"]
    x = _decode(codes.view(-1, c["head_dim"])[slots.long()], c["format"])
    return (x * scale[slots.long() // p][:, None]).to(DTYPES[c["dtype"]])


def _plain_attend(s):
    c = s["case"]
    R, H, p, d = c["requests"], c["kv_heads"], c["page"], c["head_dim"]
    G, N, Q, dev = c["q_heads"] // H, s["longest"], s["most"], s["q"].device
    blocks = -(-N // p)
    table = s["table"][:, s["layer"], :, :blocks].clamp(min=0).long()  # [R, H, blocks]
    n = s["lengths"][:, s["layer"]].long()

    def rows(codes, scale):
        x = _decode(codes[table], c["format"]) * scale[table][..., None, None]
        return x.view(R, H, blocks * p, d)

    pos = torch.arange(blocks * p, device=dev)
    k, v = rows(s["k"], s["k_scale"]), rows(s["v"], s["v_scale"])
    v = torch.where((pos < n[..., None])[..., None], v, 0)
    if s["starts"] is None:
        start, a = torch.arange(R, device=dev) * Q, torch.full((R,), Q, device=dev)
    else:
        start, a = s["starts"][:-1].long(), s["starts"].diff().long()
    j = torch.arange(Q, device=dev)
    token = (start[:, None] + j).clamp(max=s["total"] - 1)  # [R, Q]
    q = s["q"][token].float().view(R, Q, H, G, d).permute(0, 2, 3, 1, 4)
    x = torch.matmul(q.reshape(R, H, G * Q, d), k.transpose(-1, -2)).view(R, H, G, Q, -1)
    x *= 1.0 / math.sqrt(d)
    last = n[..., None] - a[:, None, None] + j if c["causal"] else (n[..., None] - 1).expand(
        R, H, Q)
    x.masked_fill_((pos > last[..., None])[:, :, None], float("-inf"))
    m = x.amax(-1, keepdim=True)
    x = torch.exp(x.sub_(torch.where(m.isinf(), 0, m)))
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(R, H, G * Q, -1), v).view(R, H, G, Q, d)
    o = o / torch.where(total > 0, total, 1)
    lse = (m + torch.log(total)).squeeze(-1)
    inside = j < a[:, None]  # [R, Q]
    o = o.permute(0, 3, 1, 2, 4).reshape(R, Q, H * G, d)[inside]
    lse = lse.permute(0, 3, 1, 2).reshape(R, Q, H * G)[inside]
    return {"out": o.to(DTYPES[c["dtype"]]), "lse": lse}


# ----------------------------------------------------------------- one pass

def _cache(s):
    """The program's handle on its pools, made at the first call."""
    if "cache" not in s:
        from paper_2606_14782_gb300 import bacon
        c = s["case"]
        pools = {n: s[n] for n in ("k", "v", "k_scale", "v_scale") if n in s}
        s["cache"] = bacon.Cache(c["layers"], c["kv_heads"], c.get("q_heads", c["kv_heads"]),
                                 c.get("head_dim", 64), s["pages"], page=c["page"],
                                 format=c.get("format", "e4m3"),
                                 dtype=DTYPES[c.get("dtype", "bf16")],
                                 max_requests=c["requests"], max_blocks=s["table"].shape[-1],
                                 **pools)
    return s["cache"]


def run(state):
    s, c = state, state["case"]
    if not own:
        if c["op"] == "plan":
            return _plain_plan(s)
        if c["op"] == "attend":
            return _plain_attend(s)
        _plain_store(s["k"], s["k_scale"], s["rows_k"], s["slots"], c)
        _plain_store(s["v"], s["v_scale"], s["rows_v"], s["slots"], c)
        return {"k": _plain_load(s["k"], s["k_scale"], s["touched"], c),
                "v": _plain_load(s["v"], s["v_scale"], s["touched"], c)}
    cache = _cache(s)
    if c["op"] == "plan":
        slots, lengths, st = cache.plan(s["lengths"], s["added"], s["table"], s["free"],
                                        s["state"], s["total"])
        return {"slots": slots, "table": s["table"], "lengths": lengths, "state": st}
    if c["op"] == "store":
        cache.store(s["rows_k"], s["rows_v"], s["slots"])
        k, v = cache.load(s["touched"])
        return {"k": k, "v": v}
    out, lse = cache.attend(s["layer"], s["q"], s["lengths"], s["table"], starts=s["starts"],
                            causal=c["causal"], lse=True)
    return {"out": out, "lse": lse}


def work(case):
    """Lengths, rows, codes, scales and queries read once, what they give
    written once; two products for every query and key that it sees."""
    c = case
    held, new = _counts(c)
    after = _after(c, held, new)
    p, units = c["page"], held.numel()
    if c["op"] == "plan":
        pages = int(((after + p - 1) // p - (held + p - 1) // p).sum())
        slots = int((after - held).sum())
        return {"bytes": 8 * units + 4 * new.numel() + 8 * pages + 4 * slots, "flops": 0}
    d = c["head_dim"]
    if c["op"] == "store":
        rows = int((after - held).sum())
        touched = int((after - held // p * p).sum())
        # K and V: new rows in 16 bits become 8; all rows of the pages leave in 16
        return {"bytes": 2 * d * (3 * rows + 3 * touched) + 4 * (rows + touched), "flops": 0}
    n, a = after[:, c["layers"] // 2].double(), new.double()[:, None]
    seen = a * n - (a * (a - 1) / 2 if c["causal"] else 0)
    tokens, G = int(n.sum()), c["q_heads"] // c["kv_heads"]
    pages = int(((after[:, c["layers"] // 2] + p - 1) // p).sum())
    return {"bytes": 2 * d * tokens + 12 * pages
            + int(new.sum()) * c["q_heads"] * (4 * d + 4),
            "flops": 4 * d * G * float(seen.sum())}


# ---------------------------------------------------- the definition in 64 bits

def _two_to(e):
    """2^e in 64 bits (a general power may round)."""
    return (e.to(torch.int64) + 1023 << 52).view(torch.float64)


def _exact_value(codes, format):
    """What an 8-bit code stands for, from its bits."""
    b = codes.to(torch.int64)
    if format == "int8":
        return torch.where(b > 127, b - 256, b).double()
    e, m = b >> 3 & 15, (b & 7).double()
    x = torch.where(e > 0, (8 + m) * _two_to(e - 10), m * 2.0 ** -9)
    x = torch.where((b & 127) == 127, float("nan"), x)
    return torch.where(b > 127, -x, x)


def _exact_round(y, format):
    """The nearest value that a code stands for, ties to the even code."""
    if format == "int8":
        return y.round().clamp(-127, 127)
    step = _two_to(torch.frexp(y.abs().clamp(min=2.0 ** -6)).exponent - 4)
    return ((y / step).round() * step).clamp(-448, 448)


def _exact_store(codes, scale, rows, slots, touched, c):
    p, d, f = c["page"], c["head_dim"], c["format"]
    rows, slots = rows.reshape(-1, d).double(), slots.reshape(-1).long()
    pages = scale.numel()
    x = _exact_value(codes, f) * scale.double()[:, None, None]
    big = torch.zeros(pages, p, dtype=torch.float64, device=rows.device)
    fresh = torch.zeros(pages, dtype=torch.bool, device=rows.device)
    big.view(-1)[slots] = rows.abs().amax(dim=1)
    fresh[slots[slots % p == 0] // p] = True
    amax = big.amax(dim=1)
    if f == "e4m3":
        want = _two_to((amax / 448).clamp(min=FLOOR).log2().ceil())
        want = torch.where(amax <= 224 * want, want / 2, want)  # log2 rounds
        want = torch.where(amax > 448 * want, want * 2, want).clamp(min=FLOOR)
    else:
        t = (amax / torch.full_like(amax, 127)).clamp(min=FLOOR)
        unit = _two_to(torch.frexp(t).exponent - 8)
        want = (t / unit).ceil() * unit
    s = torch.where(fresh, want, scale.double().maximum(want))
    x.view(-1, d)[slots] = rows
    t = touched.long()
    s = s[t // p][:, None]
    return _exact_round(x.view(-1, d)[t] / s, f) * s


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["op"] == "plan":
        p, pages = c["page"], s["pages"]
        n, a = s["lengths"].cpu(), s["added"].cpu()
        table, ring = s["table"].cpu(), s["free"].cpu()
        head, count = s["state"].tolist()
        R, L, H = n.shape
        a3 = a if a.dim() == 3 else a[:, None, None].expand(R, L, H)
        flat, rows, used = table.view(R * L * H, -1), [], 0
        for u, (have, more) in enumerate(zip(n.reshape(-1).tolist(), a3.reshape(-1).tolist())):
            lo, hi = -(-have // p), -(-(have + more) // p)
            flat[u, lo:hi] = ring[(head + used + torch.arange(hi - lo)) % pages]
            used += hi - lo
            pos = torch.arange(have, have + more)
            rows.append(flat[u, pos // p] * p + (pos % p).int())
        if a.dim() == 3:
            slots = torch.cat(rows)
        else:
            slots = torch.cat([torch.stack(rows[r * L * H:(r + 1) * L * H]).view(L, H, -1)
                               for r in range(R)], dim=2).transpose(1, 2)
        return {"slots": slots.contiguous(), "table": table, "lengths": n + a3,
                "state": torch.tensor([(head + used) % pages, count - used], dtype=torch.int32)}
    if c["op"] == "store":
        return {"k": _exact_store(s["k"], s["k_scale"], s["rows_k"], s["slots"], s["touched"], c),
                "v": _exact_store(s["v"], s["v_scale"], s["rows_v"], s["slots"], s["touched"], c)}
    R, H, d, l = c["requests"], c["kv_heads"], c["head_dim"], s["layer"]
    G, dev = c["q_heads"] // H, s["q"].device
    starts = (s["starts"].tolist() if s["starts"] is not None
              else [c["new"] * r for r in range(R + 1)])
    out = torch.zeros(s["total"], H, G, d, dtype=torch.float64, device=dev)
    lse = torch.empty(s["total"], H, G, dtype=torch.float64, device=dev)
    lengths = s["lengths"][:, l].tolist()
    for r in range(R):
        lo, a = starts[r], starts[r + 1] - starts[r]
        for h in range(H):
            n = lengths[r][h]
            page = s["table"][r, l, h, :-(-n // c["page"])].long()
            k, v = ((_exact_value(s[x][page], c["format"])
                     * s[x + "_scale"][page].double()[:, None, None]).reshape(-1, d)[:n]
                    for x in ("k", "v"))
            hidden = (torch.arange(n, device=dev)
                      > torch.arange(n - a, n, device=dev)[:, None]) if c["causal"] else None
            for g in range(G):
                x = s["q"][lo:lo + a, h * G + g].double() @ k.T / math.sqrt(d)
                if hidden is not None:
                    x.masked_fill_(hidden, float("-inf"))
                z = torch.logsumexp(x, dim=-1)
                lse[lo:lo + a, h, g] = z
                if n:
                    o = torch.exp(x - z[:, None]) @ v
                    out[lo:lo + a, h, g] = torch.where(z[:, None].isinf(), 0, o)
    return {"out": out.view(-1, H * G, d), "lse": lse.view(-1, H * G)}
