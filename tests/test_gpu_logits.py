"""Rules on logits against a plain reference.

Bounds, stated before the first run.  Penalties, biases and masks are single
roundings of fp32 that are stated, so a row without a temperature and its best
token are exact.  A temperature is a reciprocal and a product: 2^-22 of the value
(1.5 units in the last place, and the reference's).  Log-sums: a term's exponent
has two roundings of |x - top| / T, which weighs less than its exp, the
exponential unit 2^-22, and at most 2^7 sums in turn: 2^-16 of the sum, absolute
in the log; the value itself is off by 2^-22 of it."""

import math

import pytest
import torch

import step_reference as ref
from paper_2606_14782_gb300 import bacon, build

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
INF = math.inf


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    bacon.load()


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def floats(x):
    return torch.tensor(x, dtype=torch.float32, device="cuda")


def pack(allowed):
    """Bit masks int32 [rows, words] of allowed [rows, V]."""
    rows, V = allowed.shape
    words = -(-V // 32)
    a = torch.zeros(rows, words * 32, dtype=torch.int64)
    a[:, :V] = allowed
    bits = (a.view(rows, words, 32) << torch.arange(32)).sum(-1)
    return torch.where(bits >= 1 << 31, bits - (1 << 32), bits).int().cuda()


def draw(rows, V, dtype, seed, spread=3.0):
    gen = torch.Generator().manual_seed(seed)
    return (spread * torch.randn(rows, V, generator=gen)).to(DTYPES[dtype]).cuda()


def verify(out, best, logprob, lse, wanted, temperature=None, out_dtype=torch.float32, rows=None):
    """Against the rows under the rules on the CPU, before the temperature."""
    for r, x in enumerate(wanted):
        if rows is not None and r not in rows:
            continue
        t = 1.0 if temperature is None else float(temperature[r])
        if out is not None:
            y = (x.double() / t)
            got = out[r].cpu()
            if temperature is None:
                assert torch.equal(got.isnan(), x.isnan())
                assert torch.equal(got.nan_to_num(7.0), x.to(out_dtype).nan_to_num(7.0))
            else:
                rel = 2.0 ** -22 + {torch.float32: 0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[out_dtype]
                fine = y.isfinite()
                assert torch.equal(got.isfinite(), fine)
                assert bool(((got.double() - y).abs()[fine] <= rel * 1.01 * y.abs()[fine] + 2.0 ** -25).all())
        if best is None:
            continue
        b = ref.best_of(x)
        assert int(best[r]) == b
        if b < 0:
            assert float(lse[r]) == -INF and float(logprob[r]) == -INF
            continue
        z = torch.logsumexp(x.double() / t, 0)
        top = x[b].double() / t
        assert abs(float(lse[r]) - float(z)) <= 2.0 ** -16 + 2.0 ** -22 * (abs(float(z)) + abs(float(top)))
        assert abs(float(logprob[r]) - float(top - z)) <= 2.0 ** -16 * (1 + abs(float(top - z)) * 2.0 ** -6)


def everything(rows, V, dtype, seed, drafts=1, longest=60, grammar=True, biases=5):
    """Inputs of all rules, and each row's own rules on the CPU."""
    gen = torch.Generator().manual_seed(seed)
    requests = -(-rows // drafts)
    x = draw(rows, V, dtype, seed)
    tokens = (V * torch.rand(requests, longest, generator=gen) ** 3).int()
    tokens[torch.rand(requests, longest, generator=gen) < 0.1] = -1
    tokens[torch.rand(requests, longest, generator=gen) < 0.05] = V + 3
    request = torch.arange(rows) // drafts
    lengths = torch.randint(0, longest - drafts + 1, (requests,), generator=gen)[request] + torch.arange(rows) % drafts
    prompt = (lengths * torch.rand(rows, generator=gen)).int()
    rep = 1 + torch.rand(rows, generator=gen)
    freq, pres = torch.rand(rows, generator=gen), torch.rand(rows, generator=gen) - 0.3
    lists = torch.randint(-1, V, (rows, biases), generator=gen).int()
    values = torch.randn(rows, biases, generator=gen) * 4
    allowed = torch.rand(rows, V, generator=gen) < 0.6 if grammar else None
    kw = dict(tokens=tokens.cuda(), lengths=lengths.int().cuda(), prompt=prompt.cuda(), request=request.int().cuda(),
              repetition=rep.cuda(), frequency=freq.cuda(), presence=pres.cuda(), bias_tokens=lists.cuda(),
              bias_values=values.cuda(), mask=pack(allowed) if grammar else None)
    want = []
    for r in range(rows):
        given = {int(t): float(v) for t, v in zip(lists[r], values[r]) if t >= 0}  # the last of equals
        want.append(ref.rules(x[r].cpu(), tokens[request[r]][:lengths[r]].tolist(), int(prompt[r]), float(rep[r]),
                              float(freq[r]), float(pres[r]), given, allowed[r] if grammar else None))
    return x, kw, want


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("V", [1, 2, 31, 32, 100, 257, 1000, 4096, 4101, 32000, 50021])
@pytest.mark.parametrize("rows", [1, 5])
def test_all_rules(rows, V, dtype):
    x, kw, want = everything(rows, V, dtype, V + rows)
    h = bacon.Logits(V)
    verify(*h.process(x, **kw), want)
    t = 0.5 + torch.rand(rows, generator=torch.Generator().manual_seed(1))
    verify(*h.process(x, temperature=t.cuda(), **kw), want, t)
    out, best, logprob, lse = h.process(x, out=False, **kw)
    assert out is None
    verify(out, best, logprob, lse, want)
    out, best, _, _ = h.process(x, greedy=False, **kw)
    assert best is None
    verify(out, None, None, None, want)
    h.sync()


@pytest.mark.parametrize("drafts", [1, 3, 4])
def test_drafts_see_those_before_them(drafts):
    x, kw, want = everything(12, 5000, "bf16", drafts, drafts=drafts, longest=200)
    h = bacon.Logits(5000)
    verify(*h.process(x, **kw), want)
    h.sync()


@pytest.mark.parametrize("drop", ["history", "biases", "mask", "prompt", "penalties"])
def test_rules_one_by_one(drop):
    V = 3001
    x, kw, _ = everything(4, V, "fp32", 3, biases=9)
    if drop == "history":
        for n in ("tokens", "lengths", "prompt", "request", "repetition", "frequency", "presence"):
            kw[n] = None
    elif drop == "biases":
        kw["bias_tokens"] = kw["bias_values"] = None
    elif drop == "penalties":
        kw["repetition"] = kw["frequency"] = kw["presence"] = None
    else:
        kw[drop] = None
    want = []
    for r in range(4):
        history = kw["tokens"][r, :int(kw["lengths"][r])].tolist() if kw["tokens"] is not None else []
        given = {} if kw["bias_tokens"] is None else {
            int(t): float(v) for t, v in zip(kw["bias_tokens"][r], kw["bias_values"][r]) if t >= 0}
        allowed = None
        if kw["mask"] is not None:
            v = torch.arange(V)
            allowed = (kw["mask"][r].cpu()[v // 32] >> (v % 32)) & 1 > 0
        p = [float(kw[n][r]) if kw[n] is not None else d
             for n, d in (("repetition", 1.0), ("frequency", 0.0), ("presence", 0.0))]
        want.append(ref.rules(x[r].cpu(), history, int(kw["prompt"][r]) if kw["prompt"] is not None else 0, *p,
                              given, allowed))
    h = bacon.Logits(V)
    verify(*h.process(x, **kw), want)
    h.sync()


def test_long_histories_and_the_largest_vocabulary():
    V = 458752
    h = bacon.Logits(V)
    gen = torch.Generator().manual_seed(1)
    tokens = torch.randint(0, 50, (2, 300000), generator=gen).int()
    tokens[1, ::7] = V - 1
    x = draw(2, V, "bf16", 2)
    want = [ref.rules(x[r].cpu(), tokens[r, :n].tolist(), p, 1.3, 0.001, 0.2)
            for r, (n, p) in enumerate(((300000, 0), (299999, 150000)))]
    got = h.process(x, tokens=tokens.cuda(), lengths=ints([300000, 299999]), prompt=ints([0, 150000]),
                    repetition=floats([1.3] * 2), frequency=floats([0.001] * 2), presence=floats([0.2] * 2))
    verify(*got, want)
    h.sync()


def test_the_largest_vocabulary_in_many_rows():
    """Eight blocks of a row: the most shared memory."""
    V = 458752
    x = draw(20, V, "fp16", 1)
    tokens = torch.randint(0, V, (20, 50), generator=torch.Generator().manual_seed(2)).int()
    want = [ref.rules(x[r].cpu(), tokens[r].tolist(), 25, 2.0, 0.25, 0.5) for r in range(20)]
    h = bacon.Logits(V)
    got = h.process(x, tokens=tokens.cuda(), lengths=ints([50] * 20), prompt=ints([25] * 20),
                    repetition=floats([2.0] * 20), frequency=floats([0.25] * 20), presence=floats([0.5] * 20))
    verify(*got, want)
    h.sync()


def test_a_prompt_of_one_token_many_times():
    """An image's places: one number over and over, then a few words."""
    V = 2000
    x = draw(2, V, "fp32", 5)
    history = [7] * 30000 + [8, 7, 9, 9]
    tokens = ints([history, history])
    h = bacon.Logits(V)
    for start in (0, 1, 2, 3):  # lines that start anywhere
        room = torch.zeros(2, len(history) + 5, dtype=torch.int32, device="cuda")
        room[:, start:start + len(history)] = tokens
        line = room[:, start:start + len(history)]
        got = h.process(x, tokens=line, lengths=ints([30004, 17]), prompt=ints([30000, 17]), repetition=floats([1.5] * 2),
                        frequency=floats([0.5] * 2), presence=floats([0.25] * 2))
        want = [ref.rules(x[0].cpu(), history, 30000, 1.5, 0.5, 0.25), ref.rules(x[1].cpu(), [7] * 17, 17, 1.5, 0.5, 0.25)]
        verify(*got, want)
    h.sync()


@pytest.mark.parametrize("V", [33, 777, 4096, 50021, 131072])
@pytest.mark.parametrize("rows", [1, 3, 25])
def test_prompts_that_a_rows_blocks_share(V, rows):
    """Long prompts beside short ones, and rows left out, in one call."""
    gen = torch.Generator().manual_seed(V)
    tokens = (V * torch.rand(rows, 40001, generator=gen) ** 4).int()
    tokens[:, 5000:9000] = V + 7
    x = draw(rows, V, "bf16", 2)
    prompt = [20000 if r % 3 == 0 else 50 if r % 3 == 1 else 16383 + r % 2 for r in range(rows)]
    lengths = [p + 300 + r for r, p in enumerate(prompt)]
    want = [ref.rules(x[r].cpu(), tokens[r, :n].tolist(), p, 1.25, 0.01, 0.3) for r, (n, p) in enumerate(zip(lengths, prompt))]
    kw = dict(tokens=tokens.cuda(), prompt=ints(prompt), repetition=floats([1.25] * rows),
              frequency=floats([0.01] * rows), presence=floats([0.3] * rows))
    h = bacon.Logits(V)
    verify(*h.process(x, lengths=ints(lengths), **kw), want)
    out, best, _, _ = h.process(x, lengths=ints(lengths), greedy=False, **kw)
    verify(out, None, None, None, want)
    lengths[0] = -1
    out = torch.full((rows, V), 6.0, device="cuda")
    got = h.process(x, lengths=ints(lengths), out=out, **kw)
    assert bool((out[0] == 6).all())
    verify(*got, want, rows=range(1, rows))
    h.sync()


def test_no_history_and_no_list():
    V = 300
    x = draw(3, V, "bf16", 6)
    h = bacon.Logits(V)
    none = torch.empty(3, 0, dtype=torch.int32, device="cuda")
    empty = h.process(x, tokens=none, lengths=ints([0, 0, 0]), bias_tokens=none, bias_values=none.float())
    verify(*empty, [x[r].cpu().float() for r in range(3)])
    some = h.process(x, tokens=ints([[1, 2]] * 3), lengths=ints([0, 0, 0]), repetition=floats([3.0] * 3))
    verify(*some, [x[r].cpu().float() for r in range(3)])
    out = torch.full((3, V), 4.0, device="cuda")
    h.process(x, lengths=ints([0, -1, 0]), out=out)
    assert bool((out[1] == 4).all()) and torch.equal(out[2], x[2].float())
    h.sync()


def test_many_rows():
    x, kw, want = everything(300, 777, "bf16", 5)
    h = bacon.Logits(777)
    verify(*h.process(x, **kw), want)
    h.sync()


@pytest.mark.parametrize("V", [64, 1003])
def test_strides_in_place_and_types(V):
    x, kw, want = everything(6, V, "bf16", 9)
    h = bacon.Logits(V)
    wide = torch.full((6, V + 5), 3.0, dtype=torch.bfloat16, device="cuda")
    wide[:, :V] = x
    room = torch.full((6, V + 9), 2.0, dtype=torch.float32, device="cuda")
    out, *rest = h.process(wide[:, :V], out=room[:, :V], **kw)
    verify(out, *rest, want)
    assert bool((room[:, V:] == 2).all()) and bool((wide[:, V:] == 3).all())
    got = h.process(x, out=torch.empty_like(x), **kw)
    verify(*got, want, out_dtype=torch.bfloat16)
    y = x.clone()
    got = h.process(y, out=y, **kw)
    assert got[0] is y
    verify(*got, want, out_dtype=torch.bfloat16)
    one = x[:1].expand(6, V)
    kw1 = dict(kw, mask=kw["mask"][:1])
    out, best, _, _ = h.process(one, **kw1)
    again, best2, _, _ = h.process(one.contiguous(), **dict(kw, mask=kw["mask"][:1].expand(6, -1)))
    assert torch.equal(out, again) and torch.equal(best, best2)


def test_rows_with_nothing_left_and_rows_left_out():
    V = 200
    x, kw, want = everything(4, V, "fp32", 4)
    allowed = torch.ones(4, V, dtype=torch.bool)
    allowed[1] = False
    kw["mask"] = pack(allowed)
    kw["mask"][1, -1] = -256  # bits behind the vocabulary count for nothing
    kw["lengths"][2] = -1
    kw["bias_tokens"][2] = 10 ** 9  # nothing of a row that is left out is read
    h = bacon.Logits(V)
    out = torch.full((4, V), 5.0, device="cuda")
    got, best, logprob, lse = h.process(x, out=out, **kw)
    assert int(best[1]) == -1 and float(lse[1]) == -INF and float(logprob[1]) == -INF
    assert bool((out[1] == -INF).all()) and bool((out[2] == 5).all())
    h.sync()


def test_ties_go_to_the_lowest_token():
    V = 40000
    x = torch.zeros(3, V, dtype=torch.bfloat16, device="cuda")
    x[1, [39999, 20001, 777]] = 2
    x[2] = -0.0
    x[2, 12345:] = 0.0
    h = bacon.Logits(V)
    _, best, logprob, lse = h.process(x)
    assert best.tolist() == [0, 777, 0]
    assert abs(float(logprob[0]) + math.log(V)) < 1e-4 and abs(float(lse[0]) - math.log(V)) < 1e-4


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_values_that_are_not_finite(dtype):
    V = 500
    x = draw(6, V, dtype, 1)
    low = torch.finfo(DTYPES[dtype]).min
    x[0, 100:] = -INF                    # masked by the caller
    x[1, 3:] = low                       # or with the type's lowest value
    x[2, 7] = float("nan")               # in a place that the mask leaves out
    x[3, 9] = float("nan")               # and in one that it does not
    x[4, 11] = INF
    x[5] = -INF
    allowed = torch.ones(6, V, dtype=torch.bool)
    allowed[2, 7] = False
    allowed[0, :50] = False
    want = [ref.rules(x[r].cpu(), [1, 2, 200], 1, 1.5, 0.5, 0.5, {}, allowed[r]) for r in range(6)]
    h = bacon.Logits(V)
    tokens = ints([[1, 2, 200]] * 6)
    out, best, logprob, lse = h.process(x, tokens=tokens, lengths=ints([3] * 6), prompt=ints([1] * 6),
                                        repetition=floats([1.5] * 6), frequency=floats([0.5] * 6),
                                        presence=floats([0.5] * 6), mask=pack(allowed))
    verify(out, best, logprob, lse, want, rows=(0, 1, 2, 5))
    verify(out, None, None, None, want)
    assert int(best[3]) == ref.best_of(want[3]) and math.isnan(float(lse[3])) and math.isnan(float(logprob[3]))
    assert int(best[4]) == 11 and float(lse[4]) == INF
    h.sync()


def test_biases_that_ban_and_that_are_named_twice():
    V = 300
    x = draw(2, V, "fp32", 2)
    h = bacon.Logits(V)
    top = int(x[0].argmax())
    lists = ints([[top, 5, 5, 9, 5, -1, 250, 250], [-1] * 8])
    values = floats([[-INF, 1, 100, 2, -4, 77, 3, 4], [50.0] * 8])
    out, best, _, _ = h.process(x, bias_tokens=lists, bias_values=values)
    want = [ref.rules(x[0].cpu(), [], 0, biases={top: -INF, 5: -4.0, 9: 2.0, 250: 4.0}), x[1].cpu()]
    verify(out, best, *h.process(x, bias_tokens=lists, bias_values=values)[2:], want)
    many = torch.arange(2047, dtype=torch.int32, device="cuda")[None] % V
    given = torch.arange(2047, dtype=torch.float32, device="cuda")[None]
    out, *rest = h.process(x[:1], bias_tokens=many.contiguous(), bias_values=given)
    last = {t: float(max(i for i in range(2047) if i % V == t)) for t in range(V)}
    verify(out, *rest, [ref.rules(x[0].cpu(), [], 0, biases=last)])
    h.sync()


@pytest.mark.parametrize("change", [dict(lengths=11), dict(lengths=-2), dict(prompt=5), dict(prompt=-1),
                                    dict(request=2), dict(request=-1), dict(bias=-2), dict(bias=100),
                                    dict(repetition=0.0), dict(repetition=float("nan")), dict(temperature=-1.0),
                                    dict(temperature=0.0), dict(frequency=INF), dict(presence=float("nan"))])
def test_what_is_wrong_is_reported(change):
    V = 100
    x = draw(2, V, "fp32", 3)
    a = dict(lengths=4, prompt=2, request=0, bias=7, repetition=2.0, temperature=1.0, frequency=0.5, presence=0.25)
    b = {**a, **change}
    history = [1, 2, 3, 3, 4, 5, 6, 7, 8, 9]

    def call(c):
        return h.process(x, tokens=ints([history, history]), lengths=ints([4, c["lengths"]]),
                         prompt=ints([2, c["prompt"]]), request=ints([0, c["request"]]),
                         bias_tokens=ints([[7], [c["bias"]]]), bias_values=floats([[1.5], [1.5]]),
                         **{n: floats([a[n], c[n]]) for n in ("repetition", "temperature", "frequency", "presence")})

    h = bacon.Logits(V)
    got = call(b)
    with pytest.raises(bacon.BaconError):
        h.sync()
    h.sync()
    default = dict(repetition=1.0, temperature=1.0, frequency=0.0, presence=0.0)
    c = {**a, **{n: default[n] for n in change if n in default}}
    first = ref.rules(x[0].cpu(), history[:4], 2, 2.0, 0.5, 0.25, {7: 1.5})
    left = "bias" not in change and {7: 1.5} or {}
    lost = any(n in change for n in ("lengths", "prompt", "request"))
    second = ref.rules(x[1].cpu(), [] if lost else history[:4], 2, c["repetition"], c["frequency"], c["presence"], left)
    verify(*got, [first, second])


def test_no_rows_and_refusals():
    h = bacon.Logits(100)
    x = draw(3, 100, "fp32", 1)
    assert h.process(x[:0])[1].shape == (0,)
    history, n = ints([[1, 2]] * 3), ints([2] * 3)
    for args, kw in (((x[:, :50],), {}), ((x.double(),), {}), ((x.cpu(),), {}), ((x[0],), {}),
                     ((x.t().contiguous().t(),), {}), ((x,), dict(out=x[:2])), ((x,), dict(out=x.half())),
                     ((x,), dict(tokens=history, lengths=n.long())), ((x,), dict(tokens=history, lengths=n[:2])),
                     ((x,), dict(tokens=history.long(), lengths=n)), ((x,), dict(repetition=n)),
                     ((x,), dict(temperature=floats([1.0]))), ((x,), dict(mask=ints([[1] * 3] * 3))),
                     ((x,), dict(mask=ints([[1] * 4] * 2))), ((x,), dict(bias_tokens=n[:, None].contiguous())),
                     ((x,), dict(bias_tokens=n[:, None].contiguous(), bias_values=floats([[1.0]])))):
        with pytest.raises(ValueError):
            h.process(*args, **kw)
    with pytest.raises(bacon.BaconError):
        h.process(x, out=False, greedy=False)
    with pytest.raises(bacon.BaconError):
        h.process(x, tokens=history)
    with pytest.raises(bacon.BaconError):
        h.process(x, out=x[:1].expand(3, 100))
    h.close()
    with pytest.raises(bacon.BaconError):
        h.process(x)


def test_another_stream_and_a_graph():
    x, kw, want = everything(5, 4000, "bf16", 2)
    h = bacon.Logits(4000)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = h.process(x, stream=s, **kw)
    torch.cuda.current_stream().wait_stream(s)
    verify(*got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = h.process(x, **kw)
    other, more, want = everything(5, 4000, "bf16", 77)
    x.copy_(other)
    for n, t in more.items():
        kw[n].copy_(t)
    graph.replay()
    verify(*out, want)
    h.sync()


def test_the_same_every_time():
    x, kw, _ = everything(40, 30000, "fp32", 2, longest=3000)
    h = bacon.Logits(30000)
    first = h.process(x, **kw)
    for _ in range(3):
        for a, b in zip(first, h.process(x, **kw)):
            assert torch.equal(a, b)
