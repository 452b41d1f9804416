"""Measured operators: what a serving program does with a token between its
matrix products and the cache.

The operators (`op`):

  rotary  positions into Q and K of a fused projection's rows, after a norm of
          each head where the model has one; K may leave head by head, as the
          compression reads it
  write   the same for new tokens whose K, with its positions, and V go into
          the 8-bit pages of the cache in the same call
  norm    what lies between two blocks: the norm of a block's output, its gate,
          the residual sum, the norm before the next block
  logits  penalties for repeated tokens, biases, grammar masks, temperature,
          and the greedy token with its log-probability

`own` chooses between the framework's calls and their plain form.
"""

import math

import torch

own = False

FLOOR = 2.0 ** -60  # the least scale of a page
EPS = 1e-6


# ------------------------------------------------------------------ cases

def _rotary(name, requests, tokens, q_heads, kv_heads, head_dim, rotary_dim, interleaved, scaling,
            axes, norm, dtype, first, keys="tokens"):
    """`first`: about where the tokens stand.  keys "heads": K head by head."""
    c = dict(op="rotary", requests=requests, tokens=tokens, q_heads=q_heads, kv_heads=kv_heads,
             head_dim=head_dim, rotary_dim=rotary_dim, interleaved=interleaved, scaling=scaling,
             axes=axes, norm=norm, dtype=dtype, first=first, keys=keys)
    return dict(c, name=name) if name else c


def _write(name, requests, q_heads, kv_heads, head_dim, rotary_dim, interleaved, scaling, norm,
           page, format, dtype, held, new):
    c = dict(op="write", requests=requests, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim,
             rotary_dim=rotary_dim, interleaved=interleaved, scaling=scaling, axes=1, norm=norm,
             page=page, format=format, dtype=dtype, held=held, new=new)
    return dict(c, name=name) if name else c


def _norm(name, tokens, width, dtype, residual, post, pre, gate, gate_kind):
    """residual: the type of the residual sum; post, pre: the norms after and
    before a block; gate: its shape (a value for each channel, token, or both)."""
    c = dict(op="norm", tokens=tokens, width=width, dtype=dtype, residual=residual, post=post,
             pre=pre, gate=gate, gate_kind=gate_kind)
    return dict(c, name=name) if name else c


def _logits(name, requests, drafts, vocab, history, dtype, penalties, biases, grammar, write):
    """`drafts` rows a request, each with the ones before it in its history of
    about `history` tokens; write: the logits themselves are wanted too."""
    c = dict(op="logits", requests=requests, drafts=drafts, vocab=vocab, history=history,
             dtype=dtype, penalties=penalties, biases=biases, grammar=grammar, write=write)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one layer of one request's decoding step: launches and latency
        _rotary("rotary_token", 1, 1, 28, 4, 128, 128, False, "none", 1, False, "bf16", 4096),
        # ragged prompts end to end in one row of tokens, positions in a part of each head
        _rotary("rotary_part", 1, 5003, 12, 2, 64, 32, True, "rotations", 1, True, "fp16", 100000),
        # one layer of the screenshot prompts: three positions a token, K as the scoring reads it
        _rotary("rotary_prompts", 4, 16384, 28, 4, 128, 128, False, "none", 3, False, "bf16", 0,
                keys="heads"),
        # one layer of a decoding step: a row in each unit's last page
        _write("write_step", 32, 32, 8, 128, 128, False, "linear", True, 64, "e4m3", "bf16", 1000, 1),
        # one layer of ragged follow-up turns
        _write("write_turn", 5, 28, 4, 128, 128, False, "dims", False, 32, "int8", "fp16", 2000, 700),
        # one token between two blocks
        _norm("norm_token", 1, 3584, "bf16", "bf16", "none", "rms", "none", "linear"),
        # a narrow odd width, norms around the block, a gate a token, the sum in 32 bits
        _norm("norm_odd", 2049, 1111, "fp16", "fp32", "layer", "layer", "token", "sigmoid"),
        # the screenshot prompts between two blocks
        _norm("norm_prompts", 65536, 3584, "bf16", "bf16", "rms", "rms", "channel", "linear"),
        # one request's greedy token, nothing else wanted
        _logits("logits_token", 1, 1, 32000, 500, "bf16", True, 0, False, False),
        # drafted tokens under a grammar
        _logits("logits_drafts", 5, 4, 50021, 3000, "bf16", True, 37, True, True),
        # long histories of a few requests
        _logits("logits_long", 4, 1, 131072, 100000, "fp32", True, 300, False, True),
        # a full batch, everything asked for
        _logits("logits_batch", 256, 1, 131072, 6000, "fp32", True, 16, True, True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


HEADS = ((4, 4), (8, 8), (32, 32), (28, 4), (32, 8), (16, 4), (8, 2), (6, 2), (12, 2), (7, 1))
MOST = {"rotary": 4 * 16384 * 32 * 128 * 4, "write": 5 * 700 * 36 * 128 * 8,
        "norm": 65536 * 3584 * 8, "logits": 256 * 131072 * 8}


def draw(rng):
    while True:
        op = rng.choice(("rotary", "write", "norm", "logits"))
        q_heads, kv_heads = rng.choice(HEADS)
        head_dim = rng.choice((64, 128, 128))
        rotary_dim = rng.choice((head_dim, head_dim, head_dim, head_dim // 2, head_dim // 4,
                                 head_dim - 24))
        interleaved, norm = rng.random() < 0.4, rng.random() < 0.4
        scaling = rng.choice(("none", "linear", "base", "rotations", "dims"))
        dtype = rng.choice(("bf16", "bf16", "fp16"))
        if op == "rotary":
            wide = rng.choice((head_dim, head_dim, head_dim, 80, 256))
            c = _rotary(None, _log_int(rng, 1, 16), _log_int(rng, 1, 32768), q_heads, kv_heads,
                        wide, min(rotary_dim, wide), interleaved, scaling, rng.choice((1, 1, 3)),
                        norm, rng.choice((dtype, dtype, "fp32")), rng.choice((0, 1000, 1000000)),
                        rng.choice(("tokens", "heads")))
        elif op == "write":
            c = _write(None, _log_int(rng, 1, 48), q_heads, kv_heads, head_dim, rotary_dim,
                       interleaved, scaling, norm, rng.choice((16, 32, 64, 64, 128)),
                       rng.choice(("e4m3", "int8")), dtype, _log_int(rng, 1, 4096),
                       rng.choice((1, 1, _log_int(rng, 2, 1024))))
        elif op == "norm":
            gate = rng.choice(("none", "none", "channel", "token", "full"))
            c = _norm(None, _log_int(rng, 1, 32768),
                      rng.choice((8 * _log_int(rng, 4, 2048), _log_int(rng, 1, 16384))),
                      rng.choice((dtype, dtype, "fp32")), rng.choice(("same", "fp32")),
                      rng.choice(("none", "none", "rms", "layer")), rng.choice(("rms", "layer")),
                      gate, rng.choice(("linear", "sigmoid", "tanh", "silu")))
            if c["residual"] == "same":
                c["residual"] = c["dtype"]
        else:
            c = _logits(None, _log_int(rng, 1, 256), rng.choice((1, 1, rng.randint(2, 6))),
                        _log_int(rng, 1000, 262144), _log_int(rng, 1, 131072),
                        rng.choice((dtype, "fp32")), rng.random() < 0.8,
                        rng.choice((0, _log_int(rng, 1, 300))), rng.random() < 0.5,
                        rng.random() < 0.7)
            if not (c["penalties"] or c["biases"] or c["grammar"]):
                continue
        if work(c)["bytes"] <= MOST[op]:
            return c


# ----------------------------------------------------------------- inputs

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZES = {"bf16": 2, "fp16": 2, "fp32": 4}

# base of the frequencies, and for each way to scale them: by how much, the
# length trained for, the rotations between which it sets in, and the amplitude
BASE = 10000.0
SCALINGS = {"none": (1.0, 0, 0.0, 0.0, 1.0), "linear": (4.0, 0, 0.0, 0.0, 1.0),
            "base": (8.0, 0, 0.0, 0.0, 1.0), "rotations": (8.0, 8192, 1.0, 4.0, 1.0),
            "dims": (16.0, 4096, 1.0, 32.0, 0.1 * math.log(16.0) + 1.0)}


def _axes(c):
    """The position axis of each frequency: time, height and width in parts."""
    half = c["rotary_dim"] // 2
    if c["axes"] == 1:
        return None
    return [0 if 4 * i < half else 1 if 8 * i < 5 * half else 2 for i in range(half)]


def _around(mean, shape, lo, hi, seed):
    """Numbers around `mean`, from the sizes alone: the same for every seed, so
    that work() knows them."""
    gen = torch.Generator().manual_seed(seed)
    spread = lo + (hi - lo) * torch.rand(shape, generator=gen, dtype=torch.float64)
    return (mean * spread).round().to(torch.int64)


def _counts(c):
    """(held [R, H], new [R]) of a `write` case."""
    held = _around(c["held"], (c["requests"], c["kv_heads"]), 0.3, 1.7, 7)
    if c["new"] == 1:
        return held, torch.ones(c["requests"], dtype=torch.int64)
    return held, _around(c["new"], (c["requests"],), 0.5, 1.5, 8).clamp(min=1)


def _lengths(c):
    """History of each row, its prompt's part, and the row's request."""
    n = _around(c["history"], (c["requests"],), 0.2, 1.6, 9).clamp(min=1)
    n = n.clamp(max=1 << 18)
    prompt = (0.7 * n).long()
    request = torch.arange(c["requests"]).repeat_interleave(c["drafts"])
    ahead = torch.arange(c["drafts"]).repeat(c["requests"])
    return n[request] + ahead, prompt[request], request


def _rows(shape, gen, dtype):
    """A fused projection's rows; their sizes vary from token to token."""
    x = torch.randn(shape, generator=gen, device="cuda")
    x *= torch.exp(0.4 * torch.randn(shape[:-2] + (1, 1), generator=gen, device="cuda"))
    return x.to(dtype)


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


def _head_weights(s, c, gen):
    for n in ("q_weight", "k_weight"):
        s[n] = None
        if c["norm"]:
            x = 1 + 0.2 * torch.randn(c["head_dim"], generator=gen, device="cuda")
            s[n] = x.to(DTYPES[c["dtype"]])


def _prepare_rotary(c, gen):
    s, R, N, Hq, H = {}, c["requests"], c["tokens"], c["q_heads"], c["kv_heads"]
    rows = _rows((R, N, Hq + 2 * H, c["head_dim"]), gen, DTYPES[c["dtype"]])
    s["q"], s["k"] = rows[:, :, :Hq], rows[:, :, Hq:Hq + H]
    _head_weights(s, c, gen)
    start = torch.randint(0, c["first"] + 1, (R, 1), generator=gen, device="cuda")
    at = torch.arange(N, device="cuda")
    if c["axes"] == 1:
        s["positions"] = (start + at).int().contiguous()
    else:  # an image of 124 tokens a line after a few words
        place = (at - 16).clamp(min=0)
        text = at < 16
        s["positions"] = torch.stack([start + torch.where(text, at, 16),
                                      start + torch.where(text, at, 16 + place // 124),
                                      start + torch.where(text, at, 16 + place % 124)]).int()
    if c["keys"] == "heads":
        s["keys"] = torch.empty(R, H, N, c["head_dim"], dtype=DTYPES[c["dtype"]], device="cuda")
    return s


def _prepare_write(c, gen):
    dev, H, p, d = "cuda", c["kv_heads"], c["page"], c["head_dim"]
    held, new = _counts(c)
    after = held + new[:, None]
    blocks = (after + p - 1) // p
    s = {"pages": int(blocks.sum()) + 37, "total": int(new.sum())}
    order = torch.randperm(s["pages"], generator=gen, device=dev).to(torch.int32)
    filled = torch.arange(int(blocks.max()), device=dev) < blocks.to(dev)[..., None]
    table = torch.full(filled.shape, -1, dtype=torch.int32, device=dev)
    table[filled] = order[:int(blocks.sum())]

    def places(first, count):
        """Slots of the positions [first, first + count) of each unit."""
        first, count = first.reshape(-1).to(dev), count.reshape(-1).to(dev)
        unit = torch.repeat_interleave(torch.arange(count.numel(), device=dev), count)
        pos = first[unit] + torch.arange(unit.numel(), device=dev) - (count.cumsum(0) - count)[unit]
        return (table.view(count.numel(), -1)[unit, pos // p] * p + pos % p).int(), unit, pos

    slots, unit, pos = places(held, after - held)
    begin = (new.cumsum(0) - new).to(dev)
    token = begin[unit // H] + pos - held.reshape(-1).to(dev)[unit]
    s["slots"] = torch.empty(s["total"], H, dtype=torch.int32, device=dev)
    s["slots"][token, unit % H] = slots
    first = held // p * p
    s["touched"] = places(first, after - first)[0]  # every row of the pages that get one
    for n in ("k", "v"):
        x = torch.randn(s["pages"], p, d, generator=gen, device=dev)
        x *= torch.exp(0.4 * torch.randn(s["pages"], p, 1, generator=gen, device=dev))
        s[n + "_scale"] = _scale(x.abs().amax(dim=(1, 2)), c["format"])
        s[n] = _encode(x, s[n + "_scale"][:, None, None], c["format"])
    rows = _rows((s["total"], c["q_heads"] + 2 * H, d), gen, DTYPES[c["dtype"]])
    s["rows_q"], s["rows_k"], s["rows_v"] = rows.split((c["q_heads"], H, H), dim=1)
    _head_weights(s, c, gen)
    # the tokens stand behind whole prompts, not behind the rows kept of them
    start = torch.randint(0, 16384, (c["requests"],), generator=gen, device=dev)
    request = torch.repeat_interleave(torch.arange(c["requests"], device=dev), new.to(dev))
    s["positions"] = (start[request] + torch.arange(s["total"], device=dev) - begin[request]).int()
    return s


def _prepare_norm(c, gen):
    s, T, D, dt = {}, c["tokens"], c["width"], DTYPES[c["dtype"]]

    def weight(mean, spread):
        return (mean + spread * torch.randn(D, generator=gen, device="cuda")).to(dt)

    big = torch.exp(0.5 * torch.randn(D, generator=gen, device="cuda"))  # some channels are larger
    s["y"] = (torch.randn(T, D, generator=gen, device="cuda") * big).to(dt)
    s["x"] = (4 * torch.randn(T, D, generator=gen, device="cuda") * big).to(DTYPES[c["residual"]])
    for n in ("post", "pre"):
        s[n + "_weight"] = weight(1, 0.2) if c[n] != "none" else None
        s[n + "_bias"] = weight(0, 0.2) if c[n] == "layer" else None
    shape = {"none": None, "channel": (D,), "token": (T, 1), "full": (T, D)}[c["gate"]]
    s["gate"] = None if shape is None else torch.randn(shape, generator=gen, device="cuda").to(dt)
    s["scale"] = 0.75
    return s


def _prepare_logits(c, gen):
    s, dev, V = {}, "cuda", c["vocab"]
    lengths, prompt, request = _lengths(c)
    rows, longest = lengths.numel(), int(lengths.max())
    x = 2.5 * torch.randn(rows, V, generator=gen, device=dev)
    # the tokens of a text: few of them often; an image's places in it have none
    u = torch.rand(c["requests"], longest, generator=gen, device=dev, dtype=torch.float64)
    s["tokens"] = (V * u ** 3).int().clamp(max=V - 1)
    s["tokens"][:, :longest // 8] = -1
    # a model is inclined to say again what was said
    last = s["tokens"][:, -1:].long()[request.to(dev)]
    s["logits"] = x.scatter_add(1, last, torch.full_like(last, 8, dtype=torch.float32)).to(
        DTYPES[c["dtype"]])
    s["request"], s["prompt"], s["lengths"] = (t.int().to(dev) for t in (request, prompt, lengths))
    if not c["penalties"]:
        s["tokens"] = s["lengths"] = s["prompt"] = s["request"] = None

    def uniform(lo, hi):
        return lo + (hi - lo) * torch.rand(rows, generator=gen, device=dev)

    s["repetition"], s["frequency"], s["presence"] = (
        (uniform(1, 1.4), uniform(0, 0.5), uniform(-0.2, 1)) if c["penalties"] else (None,) * 3)
    s["temperature"] = uniform(0.5, 1.5) if c["write"] else None
    s["bias_tokens"] = s["bias_values"] = None
    if c["biases"]:
        # tokens of a row differ; some places of the list are unused
        step = max(1, V // c["biases"])
        at = torch.arange(c["biases"], device=dev) * step
        at = (at + torch.randint(0, step, (rows, c["biases"]), generator=gen, device=dev)) % V
        unused = torch.rand(rows, c["biases"], generator=gen, device=dev) < 0.2
        s["bias_tokens"] = torch.where(unused, -1, at).int()
        s["bias_values"] = 3 * torch.randn(rows, c["biases"], generator=gen, device=dev)
    s["mask"] = None
    if c["grammar"]:  # from nearly everything to a few tokens; nothing at all in a row that ended
        words = -(-V // 32)
        share = uniform(0, 1)[:, None] ** 4
        share[-1] = 0 if rows > 2 else 0.5
        allowed = torch.rand(rows, words * 32, generator=gen, device=dev) < share
        bits = allowed.view(rows, words, 32).long() << torch.arange(32, device=dev)
        bits = bits.sum(-1)
        s["mask"] = torch.where(bits >= 1 << 31, bits - (1 << 32), bits).int()
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"rotary": _prepare_rotary, "write": _prepare_write, "norm": _prepare_norm,
         "logits": _prepare_logits}[case["op"]](case, gen)
    s["case"] = case
    return s


# ----------------------------------------------------------- the plain form

def _plain_angles(c, positions):
    """cos and sin of each token's angles; far positions need 64 bits."""
    D, (factor, original, low, high, amplitude) = c["rotary_dim"], SCALINGS[c["scaling"]]
    i = torch.arange(D // 2, dtype=torch.float64, device=positions.device)
    theta = BASE ** (-2 * i / D)
    if c["scaling"] == "linear":
        theta = theta / factor
    elif c["scaling"] == "base":
        theta = (BASE * factor ** (D / (D - 2))) ** (-2 * i / D)
    elif c["scaling"] == "rotations":
        kept = ((original * theta / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
        theta = kept * theta + (1 - kept) * theta / factor
    elif c["scaling"] == "dims":
        at = [D * math.log(original / (2 * math.pi * r)) / (2 * math.log(BASE)) for r in (high, low)]
        first, last = max(math.floor(at[0]), 0), min(math.ceil(at[1]), D // 2 - 1)
        kept = 1 - ((i - first) / max(last - first, 0.5)).clamp(0, 1)
        theta = kept * theta + (1 - kept) * theta / factor
    p = positions.double()
    p = p[..., None] if c["axes"] == 1 else p[_axes(c)].movedim(0, -1)
    angle = p * theta
    return ((torch.cos(angle) * amplitude).float()[..., None, :],
            (torch.sin(angle) * amplitude).float()[..., None, :])


def _plain_rotate(x, weight, cos, sin, c):
    dtype, D, x = x.dtype, c["rotary_dim"], x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    if c["interleaved"]:
        a, b = x[..., 0:D:2], x[..., 1:D:2]
        y = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = x[..., :D // 2], x[..., D // 2:D]
        y = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((y, x[..., D:]), -1).to(dtype)


def _plain_rotary(s):
    c = s["case"]
    cos, sin = _plain_angles(c, s["positions"])
    k = _plain_rotate(s["k"], s["k_weight"], cos, sin, c)
    if c["keys"] == "heads":
        s["keys"].copy_(k.transpose(1, 2))
        k = s["keys"].transpose(1, 2)
    return {"q": _plain_rotate(s["q"], s["q_weight"], cos, sin, c), "k": k}


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


def _plain_write(s):
    c = s["case"]
    cos, sin = _plain_angles(c, s["positions"])
    k = _plain_rotate(s["rows_k"], s["k_weight"], cos, sin, c)
    _plain_store(s["k"], s["k_scale"], k, s["slots"], c)
    _plain_store(s["v"], s["v_scale"], s["rows_v"], s["slots"], c)
    return {"q": _plain_rotate(s["rows_q"], s["q_weight"], cos, sin, c),
            "k": _plain_load(s["k"], s["k_scale"], s["touched"], c),
            "v": _plain_load(s["v"], s["v_scale"], s["touched"], c)}


def _plain_normed(x, kind, weight, bias):
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    return x if bias is None else x + bias.float()


def _plain_norm(s):
    c, a = s["case"], s["y"].float()
    if c["post"] != "none":
        a = _plain_normed(a, c["post"], s["post_weight"], s["post_bias"])
    if s["gate"] is not None:
        g = s["gate"].float()
        if c["gate_kind"] == "tanh":
            g = torch.tanh(g)
        elif c["gate_kind"] != "linear":
            g = (1 if c["gate_kind"] == "sigmoid" else g) / (1 + torch.exp(-g))
        a = a * g
    total = s["x"].float() + s["scale"] * a
    return {"sum": total.to(s["x"].dtype),
            "normed": _plain_normed(total, c["pre"], s["pre_weight"], s["pre_bias"]).to(s["y"].dtype)}


def _plain_logits(s):
    c, x = s["case"], s["logits"].float()
    rows, V = x.shape
    if s["tokens"] is not None:
        longest = s["tokens"].shape[1]
        token = s["tokens"][s["request"].long()].long()
        at = torch.arange(longest, device=x.device)
        inside = (at < s["lengths"][:, None]) & (token >= 0) & (token < V)
        answer = inside & (at >= s["prompt"][:, None])
        one = torch.ones_like(token, dtype=torch.int32)
        none = torch.zeros(rows, V + 1, dtype=torch.int32, device=x.device)
        seen = none.scatter(1, torch.where(inside, token, V), one)[:, :V] > 0
        count = none.scatter_add(1, torch.where(answer, token, V), one)[:, :V].float()
        rep, freq, pres = (s[n][:, None] for n in ("repetition", "frequency", "presence"))
        x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
        x = torch.where(count > 0, x - (freq * count + pres), x)
    if s["bias_tokens"] is not None:
        at = s["bias_tokens"].long()
        more = torch.zeros(rows, V + 1, device=x.device)
        x = x + more.scatter(1, torch.where(at < 0, V, at), s["bias_values"])[:, :V]
    if s["mask"] is not None:
        v = torch.arange(V, device=x.device)
        allowed = (s["mask"][:, v // 32] >> (v % 32)) & 1
        x = x.masked_fill(allowed == 0, float("-inf"))
    top = x.amax(-1, keepdim=True)
    first = torch.where(x == top, torch.arange(V, device=x.device), V).amin(-1)
    ended = top[:, 0] == float("-inf")
    best = torch.where(ended, -1, first).int()
    if s["temperature"] is not None:
        x = x / s["temperature"][:, None]
    top = x.amax(-1)
    more = torch.log(torch.exp(x - torch.where(ended, 0, top)[:, None]).sum(-1))
    out = {"best": best, "logprob": torch.where(ended, float("-inf"), -more),
           "lse": torch.where(ended, float("-inf"), top + more)}
    if c["write"]:
        out["out"] = x
    return out


# ----------------------------------------------------------------- one pass

def _handle(s):
    """The program's handles and layers, made at the first call."""
    if "handle" not in s:
        from paper_2606_14782_gb300 import bacon
        c = s["case"]
        if c["op"] in ("rotary", "write"):
            factor, original, low, high, amplitude = SCALINGS[c["scaling"]]
            s["handle"] = bacon.Rotary(
                c["head_dim"], c["rotary_dim"], base=BASE, interleaved=c["interleaved"],
                scaling=None if c["scaling"] == "none" else c["scaling"], factor=factor,
                original=original, low=low, high=high, amplitude=amplitude, axes=_axes(c))
        if c["op"] == "write":
            s["cache"] = bacon.Cache(1, c["kv_heads"], c["q_heads"], c["head_dim"], s["pages"],
                                     page=c["page"], format=c["format"], dtype=DTYPES[c["dtype"]],
                                     max_requests=c["requests"], k=s["k"], v=s["v"],
                                     k_scale=s["k_scale"], v_scale=s["v_scale"])
        elif c["op"] == "norm":
            s["handle"] = bacon.BlockNorm(
                c["width"], pre=c["pre"], post=None if c["post"] == "none" else c["post"],
                gate=c["gate_kind"], scale=s["scale"], eps=EPS,
                **{n: s[n] for n in ("pre_weight", "pre_bias", "post_weight", "post_bias")})
        elif c["op"] == "logits":
            s["handle"] = bacon.Logits(c["vocab"])
    return s["handle"]


def run(state):
    s, c = state, state["case"]
    if not own:
        return {"rotary": _plain_rotary, "write": _plain_write, "norm": _plain_norm,
                "logits": _plain_logits}[c["op"]](s)
    h = _handle(s)
    if c["op"] == "rotary":
        k_out = s["keys"].transpose(1, 2) if c["keys"] == "heads" else None
        q, k = h.apply(s["q"], s["k"], s["positions"], q_weight=s["q_weight"],
                       k_weight=s["k_weight"], eps=EPS, k_out=k_out)
        return {"q": q, "k": k}
    if c["op"] == "write":
        q = s["cache"].store_rotated(h, s["rows_q"], s["rows_k"], s["rows_v"], s["positions"],
                                     s["slots"], q_weight=s["q_weight"], k_weight=s["k_weight"],
                                     eps=EPS)
        k, v = s["cache"].load(s["touched"])
        return {"q": q, "k": k, "v": v}
    if c["op"] == "norm":
        total, normed = h(s["y"], s["x"], s["gate"])
        return {"sum": total, "normed": normed}
    out, best, logprob, lse = h.process(
        s["logits"], tokens=s["tokens"], lengths=s["lengths"], prompt=s["prompt"],
        request=s["request"], repetition=s["repetition"], frequency=s["frequency"],
        presence=s["presence"], temperature=s["temperature"], bias_tokens=s["bias_tokens"],
        bias_values=s["bias_values"], mask=s["mask"], out=None if c["write"] else False)
    r = {"best": best, "logprob": logprob, "lse": lse}
    if c["write"]:
        r["out"] = out
    return r


def work(case):
    """Inputs read once, outputs written once."""
    c, e = case, SIZES[case["dtype"]]
    if c["op"] == "rotary":
        tokens = c["requests"] * c["tokens"]
        rows = tokens * (c["q_heads"] + c["kv_heads"])
        return {"bytes": 2 * e * rows * c["head_dim"] + 4 * c["axes"] * tokens,
                "flops": rows * (3 * c["rotary_dim"] + (4 * c["head_dim"] if c["norm"] else 0))}
    if c["op"] == "write":
        held, new = _counts(c)
        after, p, d, tokens = held + new[:, None], c["page"], c["head_dim"], int(new.sum())
        units = tokens * c["kv_heads"]
        touched = int((after - held // p * p).sum())
        # Q and the new rows of K and V in, Q out in 16 bits; the new codes; the
        # touched pages' rows back as values
        return {"bytes": 4 * d * tokens * c["q_heads"] + 2 * d * (3 * units + 3 * touched)
                + 4 * (tokens + units + touched),
                "flops": (tokens * c["q_heads"] + units) * 3 * c["rotary_dim"]}
    if c["op"] == "norm":
        n = c["tokens"] * c["width"]
        gate = {"none": 0, "channel": c["width"], "token": c["tokens"], "full": n}[c["gate"]]
        return {"bytes": 2 * e * n + 2 * SIZES[c["residual"]] * n + e * gate, "flops": 12 * n}
    lengths, _, request = _lengths(c)
    rows, V = lengths.numel(), c["vocab"]
    said = int(lengths[c["drafts"] - 1::c["drafts"]].sum()) if c["penalties"] else 0
    return {"bytes": rows * V * (e + (4 if c["write"] else 0)) + 4 * said + 8 * rows * c["biases"]
            + (rows * V // 8 if c["grammar"] else 0) + 12 * rows, "flops": 6 * rows * V}


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
    x = _exact_value(codes, f) * scale.double()[:, None, None]
    big = torch.zeros(scale.numel(), p, dtype=torch.float64, device=rows.device)
    fresh = torch.zeros(scale.numel(), dtype=torch.bool, device=rows.device)
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


def _exact_turn(c, positions, dev):
    """Each token's rotations as complex numbers, [..., 1, D / 2]."""
    D, (factor, original, low, high, amplitude) = c["rotary_dim"], SCALINGS[c["scaling"]]
    theta, axes = [], _axes(c) or [0] * (D // 2)
    for i in range(D // 2):
        b = BASE * factor ** (D / (D - 2)) if c["scaling"] == "base" else BASE
        t = math.exp(-2 * i / D * math.log(b))
        if c["scaling"] == "linear":
            t /= factor
        elif c["scaling"] == "rotations":
            share = min(1.0, max(0.0, (original * t / math.tau - low) / (high - low)))
            t *= share + (1 - share) / factor
        elif c["scaling"] == "dims":
            a, z = (D / 2 * math.log(original / math.tau / r) / math.log(BASE) for r in (high, low))
            a, z = max(0, math.floor(a)), min(D // 2 - 1, math.ceil(z))
            share = 1 - min(1.0, max(0.0, (i - a) / max(z - a, 0.5)))
            t *= share + (1 - share) / factor
        theta.append(t)
    p = positions.double() if c["axes"] == 3 else positions.double()[None]
    angle = torch.stack([p[a] * t for a, t in zip(axes, theta)], -1)
    return torch.polar(torch.full_like(angle, amplitude), angle).unsqueeze(-2)


def _exact_rotate(x, weight, turn, c):
    x, D = x.double(), c["rotary_dim"]
    if weight is not None:
        x = x / (x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt() * weight.double()
    y = x.clone()
    one, two = (slice(0, D, 2), slice(1, D, 2)) if c["interleaved"] else (slice(0, D // 2),
                                                                          slice(D // 2, D))
    z = torch.complex(x[..., one], x[..., two]) * turn
    y[..., one], y[..., two] = z.real, z.imag
    return y


def _exact_logits(c, s):
    outs = {"best": [], "logprob": [], "lse": [], "out": []}
    for r in range(s["logits"].shape[0]):
        x = s["logits"][r].double()
        V = x.numel()
        if s["tokens"] is not None:
            said = s["tokens"][int(s["request"][r]), :int(s["lengths"][r])].long()
            word = (said >= 0) & (said < V)
            every = torch.bincount(said[word], minlength=V) > 0
            said, word = said[int(s["prompt"][r]):], word[int(s["prompt"][r]):]
            times = torch.bincount(said[word], minlength=V).double()
            rep = s["repetition"][r].double()
            x = torch.where(every, torch.maximum(x, x * 0) / rep + torch.minimum(x, x * 0) * rep, x)
            x = x - s["frequency"][r].double() * times - s["presence"][r].double() * times.clamp(max=1)
        if s["bias_tokens"] is not None:
            used = s["bias_tokens"][r] >= 0
            x = x.index_add(0, s["bias_tokens"][r][used].long(), s["bias_values"][r][used].double())
        if s["mask"] is not None:
            bits = s["mask"][r].long()[:, None] >> torch.arange(32, device=x.device) & 1
            x[bits.reshape(-1)[:V] == 0] = -math.inf
        best = int(x.argmax()) if float(x.max()) > -math.inf else -1
        if s["temperature"] is not None:
            x = x / s["temperature"][r].double()
        z = torch.logsumexp(x, 0)
        outs["best"].append(best)
        outs["lse"].append(z)
        outs["logprob"].append(torch.log_softmax(x, 0)[best] if best >= 0 else z)
        if c["write"]:
            outs["out"].append(x)
    out = {n: torch.stack(outs[n]) for n in ("logprob", "lse")}
    out["best"] = torch.tensor(outs["best"], dtype=torch.int32)
    if c["write"]:
        out["out"] = torch.stack(outs["out"])
    return out


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["op"] in ("rotary", "write"):
        turn = _exact_turn(c, s["positions"], "cuda")
        pre = "rows_" if c["op"] == "write" else ""
        q = _exact_rotate(s[pre + "q"], s["q_weight"], turn, c)
        k = _exact_rotate(s[pre + "k"], s["k_weight"], turn, c)
        if c["op"] == "rotary":
            return {"q": q, "k": k}
        k = k.to(DTYPES[c["dtype"]])  # the rows that are stored have the cache's type
        return {"q": q,
                "k": _exact_store(s["k"], s["k_scale"], k, s["slots"], s["touched"], c),
                "v": _exact_store(s["v"], s["v_scale"], s["rows_v"], s["slots"], s["touched"], c)}
    if c["op"] == "logits":
        return _exact_logits(c, s)

    def normed(x, kind):
        w, b = s[kind + "_weight"], s[kind + "_bias"]
        if c[kind] == "layer":
            var, mean = torch.var_mean(x, dim=-1, correction=0, keepdim=True)
            return (x - mean) / (var + EPS).sqrt() * w.double() + b.double()
        return x / (x.square().sum(-1, keepdim=True) / c["width"] + EPS).sqrt() * w.double()

    a = normed(s["y"].double(), "post") if c["post"] != "none" else s["y"].double()
    if s["gate"] is not None:
        g = s["gate"].double()
        a = a * {"linear": g, "sigmoid": torch.sigmoid(g), "tanh": torch.tanh(g),
                 "silu": g * torch.sigmoid(g)}[c["gate_kind"]]
    total = torch.add(s["x"].double(), a, alpha=s["scale"])
    return {"sum": total, "normed": normed(total, "pre")}
