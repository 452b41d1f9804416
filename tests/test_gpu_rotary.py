"""Rotary rows against a plain 64-bit reference, and storing them against the two
calls that it stands for.

Bounds, stated before the first run.  An angle is off by 2^-33 of a turn from its
phase and by 2^-25 of at most half a turn from its rounding to fp32: below 2^-23.
Sine and cosine are off by two units in the last place at most (2^-23), their
product with the amplitude and the two products of a value by 2^-24 each: a value
is off by less than 2^-20 of A (|x| + |its pair|), and by the rounding of its type,
half a step: 2^-8 of the value for bf16, 2^-11 and at least 2^-25 for fp16, 2^-24
for fp32.  A norm's root (8 products in turn, 5 sums, a quotient, a root and the
products with it and the weight: under 20 roundings) adds 2^-19 of the same size."""

import pytest
import torch

import cache_reference
import step_reference as ref
from paper_2606_14782_gb300 import bacon, build

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
ROUND = {"bf16": (2.0 ** -8, 2.0 ** -134), "fp16": (2.0 ** -11, 2.0 ** -25), "fp32": (2.0 ** -24, 2.0 ** -150)}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    bacon.load()


def draw(shape, dtype, seed, scale=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(shape, generator=gen, device="cuda")
    return (x * scale * torch.exp(0.5 * torch.randn(shape[:-1] + (1,), generator=gen, device="cuda"))).to(DTYPES[dtype])


def places(shape, seed, far=5000):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-far, far, shape, generator=gen, device="cuda").int()


def close(got, want, size, dtype, norm=False):
    rel, least = ROUND[dtype]
    bound = (2.0 ** -20 + (2.0 ** -19 if norm else 0)) * size + rel * want.abs() * (1 + 2.0 ** -10) + least
    off = (got.double() - want).abs()
    assert got.shape == want.shape
    assert bool((off <= bound).all()), float((off / bound).max())


def check(handle, q, k, positions, dtype, axes=None, amplitude=1.0, qw=None, kw=None, eps=1e-6, offset=0.0,
          transposed=False, **outs):
    theta, inter = handle.frequencies, handle.interleaved_for_test
    got = handle.apply(q, k, positions, q_weight=qw, k_weight=kw, eps=eps, offset=offset,
                       transposed=transposed, **outs)
    for x, y, w in ((q, got[0], qw), (k, got[1], kw)):
        if x is None:
            assert y is None
            continue
        want, size = ref.rotate(x, positions, theta, inter, axes, amplitude, w, eps, offset, transposed)
        close(y, want, size, dtype, w is not None)
    return got


def rotary(*args, **kw):
    r = bacon.Rotary(*args, **kw)
    r.interleaved_for_test = kw.get("interleaved", False)
    return r


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,D", [(64, 64), (128, 128), (128, 32), (64, 40), (128, 104), (80, 80), (256, 64),
                                 (256, 256), (8, 8), (10, 6), (2, 2), (96, 2), (192, 96)])
def test_layouts(d, D, interleaved, dtype):
    r = rotary(d, D, interleaved=interleaved)
    for T, Hq, H in ((1, 4, 1), (7, 7, 1), (33, 28, 4)):
        q, k = draw((T, Hq, d), dtype, T), draw((T, H, d), dtype, T + 1)
        check(r, q, k, places((T,), T), dtype)
        qw, kw = draw((d,), dtype, 3), draw((d,), dtype, 4)
        check(r, q, k, places((T,), T), dtype, qw=qw, kw=kw)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_weights_of_one_and_in_fp32(dtype):
    r = rotary(128, interleaved=True)
    q, k = draw((19, 8, 128), dtype, 1), draw((19, 2, 128), dtype, 2)
    w = draw((128,), "fp32", 3)
    check(r, q, k, places((19,), 1), dtype, qw=w, offset=1.0, eps=1e-3)
    check(r, q, k, places((19,), 1), dtype, kw=w, offset=1.0)
    check(r, q, None, places((19,), 1), dtype, qw=w)
    check(r, None, k, places((19,), 1), dtype)


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions(interleaved):
    """2^31 positions of one radian: the phase is exact, the reference's own
    angle is off by 2^31 2^-53 of it, 2^-22, which is allowed for."""
    r = rotary(64, interleaved=interleaved, amplitude=1.5)
    p = torch.tensor([-2 ** 31, 2 ** 31 - 1, 10 ** 9, -1, 0, 1], dtype=torch.int32, device="cuda")
    x = draw((6, 3, 64), "fp32", 1)
    want, size = ref.rotate(x, p, r.frequencies, interleaved, None, 1.5)
    got, _ = r.apply(x, None, p)
    assert bool(((got.double() - want).abs() <= (2.0 ** -20 + 2.0 ** -21) * size + 2.0 ** -24 * want.abs()).all())
    assert torch.equal(rotary(64, amplitude=1.0).apply(x[4:5], None, p[4:5])[0], x[4:5])


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("R,N", [(1, 5), (3, 40), (2, 257)])
def test_axes_requests_and_head_major_keys(R, N, interleaved):
    axes = [i % 3 for i in range(20)] + [2, 1, 0, 0]
    r = rotary(64, 48, interleaved=interleaved, axes=axes)
    fused = draw((R, N, 12, 64), "bf16", 1)
    q, k = fused[:, :, :8], fused[:, :, 8:10]
    room = torch.full((R, 2, N + 3, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    got = check(r, q, k, places((3, R, N), 2), "bf16", axes=axes, k_out=room[:, :, :N].transpose(1, 2))
    assert got[1].data_ptr() == room.data_ptr()
    assert bool((room[:, :, N:] == 7).all())  # rows behind the last token are left as they were


@pytest.mark.parametrize("d,D,interleaved", [(64, 64, False), (128, 32, False), (64, 40, False),
                                             (64, 40, True), (64, 24, True)])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_in_place(d, D, interleaved, norm, dtype):
    r = rotary(d, D, interleaved=interleaved)
    fused = draw((9, 10, d), dtype, 5)
    q, k = fused[:, :6], fused[:, 6:8]
    p, w = places((9,), 1), draw((d,), dtype, 2) if norm else None
    want = r.apply(q, k, p, q_weight=w, k_weight=w)
    rest = fused[:, 8:].clone()
    got = r.apply(q, k, p, q_weight=w, k_weight=w, q_out=q, k_out=k)
    assert got[0].data_ptr() == q.data_ptr()
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(fused[:, 8:], rest)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,D", [(64, 64), (64, 20), (30, 12)])
def test_rows_that_start_anywhere(d, D, interleaved):
    """One value behind a multiple of 16 bytes, odd distances, shared rows."""
    r = rotary(d, D, interleaved=interleaved)
    flat = draw((20000,), "fp16", 1)
    q = flat[1:].as_strided((11, 3, d), (3 * d + 5, d + 1, 1))
    k = flat[3:].as_strided((11, 2, d), (0, d + 3, 1))  # the same two rows for every token
    room = torch.full((11 * 3 * (d + 2) + 7,), 9.0, dtype=torch.float16, device="cuda")
    out = room[1:].as_strided((11, 3, d), (3 * (d + 2), d + 2, 1))
    check(r, q, k, places((11,), 3), "fp16", q_out=out)
    touched = torch.zeros_like(room, dtype=torch.bool)
    touched[1:].as_strided((11, 3, d), (3 * (d + 2), d + 2, 1)).fill_(True)
    assert bool((room[~touched] == 9).all())


@pytest.mark.parametrize("d,D,interleaved", [(64, 64, False), (128, 32, False), (128, 128, True), (64, 16, True),
                                             (80, 48, False), (80, 40, True), (40, 16, False), (256, 96, False)])
@pytest.mark.parametrize("norm", [False, True])
def test_a_rows_bits_do_not_depend_on_how_it_is_read(d, D, interleaved, norm):
    """Rows one value off a multiple of 16 bytes are turned by other lanes."""
    r = rotary(d, D, interleaved=interleaved)
    x, p = draw((37, 3, d), "bf16", 1), places((37,), 2)
    w = draw((d,), "bf16", 3) if norm else None
    want = r.apply(x, None, p, q_weight=w)[0]
    room = torch.empty(37 * 3 * d + 1, dtype=torch.bfloat16, device="cuda")
    other = room[1:].view(37, 3, d)
    other.copy_(x)
    assert torch.equal(r.apply(other, None, p, q_weight=w)[0], want)
    assert torch.equal(r.apply(x[20:21], None, p[20:21], q_weight=w)[0], want[20:21])  # alone as among others


def test_what_does_not_turn_stays_bit_for_bit():
    for inter in (False, True):
        r = rotary(64, 32, interleaved=inter)
        x = draw((4, 2, 64), "bf16", 1)
        x[0, 0, 32:36] = torch.tensor([-0.0, float("inf"), float("nan"), -float("inf")])
        y, _ = r.apply(x, None, places((4,), 1))
        assert torch.equal(y[..., 32:].contiguous().view(torch.int16), x[..., 32:].contiguous().view(torch.int16))


def test_extreme_rows():
    """Rows whose squares pass fp32 have a norm; a row of zeros stays one; what
    is not finite stays in its row."""
    for inter, D in ((False, 64), (True, 64), (False, 40)):
        r = rotary(64, D, interleaved=inter)
        x = draw((5, 1, 64), "bf16", 1)
        x[0] = torch.where(x[0] > 0, 3e38, -2e38)
        x[1] = 0
        x[2] *= 1e-30
        x[3, 0, 7] = float("nan")
        w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
        y, _ = r.apply(x, None, places((5,), 1), q_weight=w)
        good = [0, 1, 2, 4]
        want, size = ref.rotate(x[good], places((5,), 1)[good], r.frequencies, inter, weight=w)
        close(y[good], want, size, "bf16", True)
        assert bool(y[3].isnan().all())


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,D", [(64, 64), (64, 24)])
def test_transposed_is_the_gradient(d, D, interleaved):
    r = rotary(d, D, interleaved=interleaved, amplitude=1.25)
    p, g, x = places((6,), 1), draw((6, 3, d), "fp32", 2), draw((6, 3, d), "fp32", 3)
    got = check(r, g, None, p, "fp32", amplitude=1.25, transposed=True)[0]
    v = x.double().requires_grad_()
    y, size = ref.rotate(v, p, r.frequencies, interleaved, None, 1.25)
    (y * g.double()).sum().backward()
    close(got, v.grad, ref.rotate(g, p, r.frequencies, interleaved, None, 1.25, transposed=True)[1], "fp32")
    # and against differences: the map is linear, so a step of any length does
    step = draw((6, 3, d), "fp32", 4)
    y0, y1 = (r.apply(t, None, p)[0].double() for t in (x, x + step))
    slope = float(((y1 - y0) * g.double()).sum())
    moved = (x + step).double() - x.double()
    # each of 1152 terms is off by 2^-19 of its size at most
    room = float((2.0 ** -19 * 1.25 * 2 * (x.abs() + step.abs()).double().amax() * g.abs().double()).sum())
    assert abs(slope - float((got.double() * moved).sum())) <= 2 * room


def test_differences_of_positions_move_rows():
    r = rotary(128)
    x, p, to = draw((8, 2, 128), "fp32", 1), places((8,), 1), places((8,), 2)
    there = r.apply(r.apply(x, None, p)[0], None, to - p)[0]
    want, size = ref.rotate(x, to, r.frequencies, False)
    # two calls: the bound of each
    assert bool(((there.double() - want).abs() <= 2.0 ** -18 * size).all())


def test_large_and_many():
    r = rotary(128)
    q, k = draw((3, 2801, 28, 128), "bf16", 1), draw((3, 2801, 4, 128), "bf16", 2)
    check(r, q, k, places((3, 2801), 1), "bf16")
    w = draw((128,), "bf16", 1)
    check(r, q, k, places((3, 2801), 1), "bf16", qw=w, kw=w)


def test_offsets_beyond_32_bits():
    base = torch.zeros(2 ** 31 + 4096, dtype=torch.bfloat16, device="cuda")
    x = base[2 ** 31:].view(2, 16, 128)
    x.copy_(draw((2, 16, 128), "bf16", 1))
    far = base.as_strided((2, 16, 128), (2 ** 31, 128, 1), 0)  # token 1 lies 4 GB behind token 0
    far[0].copy_(x[1])
    r = rotary(128)
    check(r, far, None, places((2,), 1), "bf16")


def test_no_tokens():
    r = rotary(64)
    q = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    y, z = r.apply(q, q[:, :2], torch.empty(0, dtype=torch.int32, device="cuda"))
    assert y.shape == (0, 4, 64) and z.shape == (0, 2, 64)


def test_refusals():
    r = rotary(64)
    q, p = draw((4, 2, 64), "bf16", 1), places((4,), 1)
    for bad in (dict(q=q[..., :32]), dict(q=q.double()), dict(positions=p.long()), dict(positions=p[:3]),
                dict(positions=p.cpu()), dict(k=q[:3]), dict(k=q.half()), dict(q=q.transpose(1, 2)),
                dict(q_weight=torch.ones(32, dtype=torch.bfloat16, device="cuda")),
                dict(q_weight=torch.ones(64, dtype=torch.float16, device="cuda")),
                dict(q_weight=torch.ones(64, device="cuda"), k_weight=torch.ones(64, device="cuda").bfloat16()),
                dict(q_out=torch.empty(4, 2, 64, device="cuda")), dict(q=q[0])):
        with pytest.raises(ValueError):
            r.apply(**{**dict(q=q, k=q, positions=p), **bad})
    shared = q[:1].expand(4, 2, 64)
    with pytest.raises(bacon.BaconError):
        r.apply(q, None, p, q_out=shared)
    with pytest.raises(bacon.BaconError):
        r.apply(q, None, p, q_weight=torch.ones(64, device="cuda"), transposed=True)


def test_another_stream_a_graph_and_a_closed_handle():
    r, w = rotary(128, 96), draw((128,), "bf16", 9)
    q, k, p = draw((50, 8, 128), "bf16", 1), draw((50, 2, 128), "bf16", 2), places((50,), 3)
    want = r.apply(q, k, p, q_weight=w)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = r.apply(q, k, p, q_weight=w, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = r.apply(q, k, p, q_weight=w)
    r.close()
    other, there = draw((50, 8, 128), "bf16", 7), places((50,), 8)
    q.copy_(other)
    p.copy_(there)
    graph.replay()
    again = rotary(128, 96).apply(other, k, there, q_weight=w)
    assert torch.equal(out[0], again[0]) and torch.equal(out[1], again[1])


# ------------------------------------------------- rows into the 8-bit cache

def pages(R, H, d, page, format, dtype, held, seed):
    """A cache of one layer whose units hold `held` tokens, and its tables."""
    cache = bacon.Cache(1, H, H, d, pages=R * H * (held // page + 12), page=page, format=format,
                        dtype=DTYPES[dtype], max_requests=R, max_blocks=held // page + 12)
    lengths, table, ring, state = cache.tables(R)
    if held:
        added = torch.full((R,), held, dtype=torch.int32, device="cuda")
        slots, lengths, state = cache.plan(lengths, added, table, ring, state, R * held)
        cache.store(draw((R * held, H, d), dtype, seed, 0.1), draw((R * held, H, d), dtype, seed + 1, 0.1), slots[0])
    return cache, lengths, table, ring, state


@pytest.mark.parametrize("format", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d,D,interleaved", [(64, 64, False), (128, 128, False), (128, 128, True), (128, 104, False),
                                             (64, 16, False), (64, 22, True), (128, 18, False)])
@pytest.mark.parametrize("page,held,new,norm", [(16, 0, 1, False), (64, 37, 1, True), (128, 5, 70, False),
                                                (32, 61, 45, True)])
def test_rotated_store_is_the_two_calls(format, dtype, d, D, interleaved, page, held, new, norm):
    R, H, Hq = 3, 2, 6
    r = rotary(d, D, interleaved=interleaved)
    one, lengths, table, ring, state = pages(R, H, d, page, format, dtype, held, 1)
    two = pages(R, H, d, page, format, dtype, held, 1)[0]
    n = torch.tensor([new, 1, max(1, new - 2)], dtype=torch.int32, device="cuda")
    T = int(n.sum())
    slots, lengths, state = one.plan(lengths, n, table, ring, state, T)
    fused = draw((T, Hq + 2 * H, d), dtype, 5)
    q, k, v = fused.split((Hq, H, H), dim=1)
    p = places((T,), 4)
    w = dict(q_weight=draw((d,), dtype, 7), k_weight=draw((d,), dtype, 8), offset=0.5) if norm else {}
    got = one.store_rotated(r, q, k, v, p, slots[0], **w)
    qr, kr = r.apply(q, k, p, **w)
    two.store(kr, v, slots[0])
    one.sync()
    two.sync()
    assert torch.equal(got, qr)
    used = table[table >= 0].long()
    assert used.numel()
    for a, b in ((one.k_scale, two.k_scale), (one.v_scale, two.v_scale)):
        assert torch.equal(a[used], b[used])
    rows = slots[0].reshape(-1).long()
    for a, b in ((one.k, two.k), (one.v, two.v)):
        assert torch.equal(a.view(-1, d)[rows], b.view(-1, d)[rows])
    every = one.locate(lengths, table, int(lengths.sum()))
    for a, b in zip(one.load(every), two.load(every)):
        assert torch.equal(a, b)


def test_rotated_store_takes_axes_no_queries_and_many():
    axes = [0] * 16 + [1] * 24 + [2] * 24
    r = rotary(128, axes=axes)
    one, lengths, table, ring, state = pages(4, 4, 128, 64, "e4m3", "bf16", 0, 1)
    two = pages(4, 4, 128, 64, "e4m3", "bf16", 0, 1)[0]
    n = torch.tensor([700, 1, 333, 64], dtype=torch.int32, device="cuda")
    T = int(n.sum())
    slots, lengths, state = one.plan(lengths, n, table, ring, state, T)
    q, k, v = draw((T, 28, 128), "bf16", 1), draw((T, 4, 128), "bf16", 2), draw((T, 4, 128), "bf16", 3)
    p = places((3, T), 1)
    out = torch.empty_like(q)
    assert one.store_rotated(r, None, k, v, p, slots[0]) is None
    assert one.store_rotated(r, q, k, v, p, slots[0], q_out=out) is out
    qr, kr = r.apply(q, k, p)
    two.store(kr, v, slots[0])
    assert torch.equal(out, qr)
    every = one.locate(lengths, table, int(lengths.sum()))
    for a, b in zip(one.load(every), two.load(every)):
        assert torch.equal(a, b)
    # the values themselves, against the rows: half a step of the codes
    want = ref.rotate(k, p, r.frequencies, False, axes)[0]
    kl = one.load(slots[0])[0].double()
    scale = one.k_scale[slots[0].long() // 64].double()[..., None]
    assert bool(((kl - want).abs() <= want.abs() * (2.0 ** -4 + 2.0 ** -7) + scale * 2.0 ** -10 + 2.0 ** -20 * 20).all())


def test_rotated_store_of_bad_slots_and_padding():
    r = rotary(64)
    cache, lengths, table, ring, state = pages(1, 1, 64, 16, "e4m3", "bf16", 0, 1)
    q, k, p = draw((3, 2, 64), "bf16", 1), draw((3, 1, 64), "bf16", 2), places((3,), 1)
    before = cache.k.clone()
    none = torch.full((3, 1), -1, dtype=torch.int32, device="cuda")
    got = cache.store_rotated(r, q, k, k, p, none)  # a padded batch: Q turns, nothing is stored
    cache.sync()
    assert torch.equal(cache.k, before) and torch.equal(got, r.apply(q, None, p)[0])
    cache.store_rotated(r, q, k, k, p, torch.full((3, 1), 1 << 30, dtype=torch.int32, device="cuda"))
    with pytest.raises(bacon.BaconError):
        cache.sync()
    cache.sync()


def test_rotated_store_refusals():
    cache, *_ = pages(1, 2, 64, 16, "e4m3", "bf16", 0, 1)
    r, k, p = rotary(64), draw((3, 2, 64), "bf16", 1), places((3,), 1)
    slots = torch.full((3, 2), -1, dtype=torch.int32, device="cuda")
    for bad in (dict(k=k[:2]), dict(q=k[:2]), dict(q=k.half()), dict(positions=p.long()), dict(slots=slots[:2]),
                dict(positions=p[:2]), dict(q_out=k[:, :1]), dict(k_weight=k[0, 0, :32])):
        with pytest.raises(ValueError):
            cache.store_rotated(**{**dict(rotary=r, q=k, k=k, v=k, positions=p, slots=slots), **bad})
    with pytest.raises(bacon.BaconError):
        cache.store_rotated(rotary(128), None, k, k, p, slots)
    empty = k[:0]
    assert cache.store_rotated(r, empty, empty, empty, p[:0], slots[:0]).shape == (0, 2, 64)
