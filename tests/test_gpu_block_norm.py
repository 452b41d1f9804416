"""The step between two blocks against a plain 64-bit reference.

Bounds, stated before the first run.  A norm's sums have at most 40 products in
turn and 10 sums, its root, quotient and products under 10 roundings more: each
value is off by less than 2^-18 of its size, and, with a mean, by 2^-18 of the
mean magnitude as the norm scales it.  An activation is off by 2^-21 of the
gate's size.  The residual sum adds two roundings.  An error in s reaches n by
the norm's factor, once directly and once through the root and the mean.  Each
output is rounded to its type: half a step."""

import pytest
import torch

import step_reference as ref
from paper_2606_14782_gb300 import bacon, build

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
ROUND = {torch.bfloat16: (2.0 ** -8, 2.0 ** -134), torch.float16: (2.0 ** -11, 2.0 ** -25),
         torch.float32: (2.0 ** -24, 2.0 ** -150)}
STEP = 2.0 ** -18


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    bacon.load()


def draw(shape, dtype, seed, spread=0.5):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(shape, generator=gen, device="cuda")
    return (x * torch.exp(spread * torch.randn(shape[-1:], generator=gen, device="cuda"))).to(DTYPES[dtype])


def norm_with_bound(v, off, kind, w, b, eps, offset):
    """The norm of v in 64 bits and how far it may be off when v is by `off`."""
    c = v - v.mean(-1, keepdim=True) if kind == "layer" else v
    inv = 1 / ((c * c).mean(-1, keepdim=True) + eps).sqrt()
    weight = 1.0 if w is None else (offset + w.double()).abs()
    shift = off.mean(-1, keepdim=True) + STEP * v.abs().mean(-1, keepdim=True) if kind == "layer" else 0.0
    root = (off * off).mean(-1, keepdim=True).sqrt() * inv + STEP
    y = ref.normed(v, kind, w, b, eps, offset)
    bias = 0.0 if b is None else 2.0 ** -23 * b.double().abs()
    return y, weight * inv * (off + shift + c.abs() * (root + STEP)) + 2.0 ** -23 * y.abs() + bias


def check(width, y, x=None, gate=None, post=None, pre="rms", weights=None, kind="linear", scale=1.0, eps=1e-6,
          offset=0.0, **outs):
    weights = weights or {}
    layer = bacon.BlockNorm(width, pre=pre, post=post, gate=kind, scale=scale, eps=eps, offset=offset, **weights)
    a, off = y.double(), torch.zeros_like(y, dtype=torch.float64)
    given = [None if t is None else t.clone() for t in (y, x, gate)]
    total, normed = layer(y, x, gate, **outs)
    y, x, gate = given
    a = y.double()
    if post:
        a, off = norm_with_bound(a, off, post, weights.get("post_weight"), weights.get("post_bias"), eps, offset)
    if gate is not None:
        g = ref.GATES[kind](gate.double())
        off = off * g.abs() + a.abs() * (2.0 ** -21 * g.abs() + 2.0 ** -23 * g.abs())
        a = a * g
    s = scale * a if x is None else x.double() + scale * a
    off = abs(scale) * off + 2.0 ** -23 * (abs(scale) * a.abs() + s.abs())
    if total is not None:
        rel, least = ROUND[total.dtype]
        assert bool(((total.double() - s).abs() <= off + rel * s.abs() * (1 + 2.0 ** -10) + least).all())
    if pre:
        n, far = norm_with_bound(s, off, pre, weights.get("pre_weight"), weights.get("pre_bias"), eps, offset)
        rel, least = ROUND[normed.dtype]
        bound = far + rel * n.abs() * (1 + 2.0 ** -10) + least
        assert bool(((normed.double() - n).abs() <= bound).all()), float(((normed.double() - n).abs() / bound).max())
    return total, normed


WIDTHS = [1, 2, 7, 8, 64, 255, 256, 520, 1000, 1024, 1030, 1111, 2048, 3584, 4100, 8192, 8200, 12288, 16384, 16391,
          20000, 32768, 32767]


@pytest.mark.parametrize("dtype,residual", [("bf16", "bf16"), ("bf16", "fp32"), ("fp16", "fp16"), ("fp16", "fp32"),
                                            ("fp32", "fp32")])
@pytest.mark.parametrize("width", WIDTHS)
def test_everything_at_once(width, dtype, residual):
    T = 6 if width > 2000 else 37
    w = {n: draw((width,), dtype, i) for i, n in enumerate(("post_weight", "pre_weight", "post_bias", "pre_bias"))}
    y, x, g = draw((T, width), dtype, 7), draw((T, width), residual, 8), draw((T, width), dtype, 9)
    check(width, y, x, g, post="rms", pre="layer", weights=w, kind="sigmoid", scale=0.5)
    check(width, y, x, None, post="layer", pre="rms", weights=w)
    check(width, y, x, g[0], pre="rms", weights={"pre_weight": w["pre_weight"]}, kind="silu", scale=-1.5, offset=1.0)


@pytest.mark.parametrize("kind", list(ref.GATES))
@pytest.mark.parametrize("width", [96, 1111])
@pytest.mark.parametrize("shape", ["channel", "token", "full"])
def test_gates(kind, width, shape):
    T = 21
    g = draw({"channel": (width,), "token": (T, 1), "full": (T, width)}[shape], "bf16", 3, 1.0) * 3
    y, x = draw((T, width), "bf16", 1), draw((T, width), "bf16", 2)
    check(width, y, x, g, kind=kind)
    check(width, y, None, g, kind=kind, pre=None)
    check(width, y.view(3, 7, width), x.view(3, 7, width), g if shape == "channel" else g.view(3, 7, -1), kind=kind)


def test_a_norm_alone_and_a_sum_alone():
    y, x = draw((5, 640), "bf16", 1), draw((5, 640), "fp32", 2)
    total, n = check(640, y)
    assert total is None and n.dtype is torch.bfloat16
    total, n = check(640, y, x, pre=None)
    assert n is None and total.dtype is torch.float32
    total, _ = check(640, y, sum_out=torch.empty_like(y))
    assert torch.equal(total, y)
    w = {"pre_weight": draw((640,), "fp32", 3), "pre_bias": draw((640,), "fp32", 4)}
    check(640, y, x, pre="layer", weights=w)


@pytest.mark.parametrize("width", [40, 700, 1111, 5000, 20001])
def test_strides_and_places(width):
    """Rows apart, starting anywhere, and what lies between them."""
    T, gap = 9, 13
    for lead in (0, 1, 5):
        for apart in (width + gap, width + 8):
            flat = draw((1, T * (apart + 16) + lead), "bf16", 1)[0]
            y = flat[lead:].as_strided((T, width), (apart, 1))
            x = draw((T, width), "bf16", 2)
            room = torch.full((T * apart + lead + 8,), 5.0, dtype=torch.bfloat16, device="cuda")
            out = room[lead:].as_strided((T, width), (apart, 1))
            check(width, y, x, sum_out=out)
            touched = torch.zeros_like(room, dtype=torch.bool)
            touched[lead:].as_strided((T, width), (apart, 1)).fill_(True)
            assert bool((room[~touched] == 5).all())
            check(width, y, y, norm_out=out)
    one = draw((1, width), "bf16", 3).expand(T, width)  # one row for every token
    check(width, one, one)


@pytest.mark.parametrize("width", [64, 1111, 3584, 20000])
def test_in_place(width):
    y, x, g = draw((7, width), "bf16", 1), draw((7, width), "bf16", 2), draw((7, width), "bf16", 3)
    want = check(width, y, x, g, post="rms", kind="tanh")
    a, b = y.clone(), x.clone()
    got = check(width, a, b, g, post="rms", kind="tanh", sum_out=b, norm_out=a)
    assert got[0] is b and got[1] is a
    assert torch.equal(a, want[1]) and torch.equal(b, want[0])


@pytest.mark.parametrize("width", [64, 1111, 5000, 20000])
@pytest.mark.parametrize("pre", ["rms", "layer"])
def test_extreme_rows(width, pre):
    """Squares beyond fp32, all zeros, tiny values; what is not finite stays in
    its row."""
    y = draw((6, width), "bf16", 1)
    y[0] = torch.where(y[0] > 0, 3e38, -2.5e38)
    y[1] = 0
    y[2] *= 1e-32
    y[3, width // 2] = float("nan")
    good = [0, 1, 2, 5]
    _, n = bacon.BlockNorm(width, pre=pre)(y)
    v = y.double()[good]
    # sizes near 3e38 and a mean of them: the bound is relative to the row
    want = ref.normed(v, pre, None, None, 1e-6, 0.0)
    big = v.abs().amax(-1, keepdim=True) / ((v * v).mean(-1, keepdim=True) + 1e-6).sqrt().clamp(min=1e-3)
    assert bool(((n.double()[good] - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -15 * (1 + big)).all())
    assert bool(n[3].isnan().all()) and bool(n[5].isfinite().all())
    gate = torch.full((6, 1), -float("inf"), dtype=torch.bfloat16, device="cuda")
    total, _ = bacon.BlockNorm(width, pre=None, gate="silu")(y[5:], None, gate[5:])
    assert bool((total == 0).all())  # silu at minus infinity


@pytest.mark.parametrize("width", [8, 16, 24, 40, 64, 128, 200])
@pytest.mark.parametrize("pre", ["rms", "layer"])
def test_extreme_rows_beside_others(width, pre):
    """Rows that share a warp: one that is gone through again, one of NaN, one of
    infinities, and those beside them as if they were alone."""
    for T in (1, 3, 13, 1000):
        y = draw((T, width), "bf16", T)
        x, g = draw((T, width), "fp32", 2), draw((T, 1), "bf16", 3)
        for r, v in ((1, 3e38), (4, float("nan")), (6, float("inf"))):
            if r < T:
                y[r] = v
                y[r, 0] = -1
        layer = bacon.BlockNorm(width, pre=pre)
        _, n = layer(y)
        total, m = layer(y, x, g)
        for r in (0, 2, 5, 7, T - 1):
            if r < T and r not in (1, 4, 6):
                assert torch.equal(layer(y[r:r + 1])[1], n[r:r + 1])
                assert all(torch.equal(a, b[r:r + 1]) for a, b in
                           zip(layer(y[r:r + 1], x[r:r + 1], g[r:r + 1]), (total, m)))
        if T > 6:
            want = ref.normed(y[1].double(), pre, None, None, 1e-6, 0.0)
            # 3e38 in all but one place: the mean is off by 2^-18 of it, the root by 2^-18
            assert bool(((n[1].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -12).all())
            assert bool(n[4].isnan().all()) and bool(n[6].isnan().any())


def test_large_means():
    """Values of 1000 +- 1: the mean is taken off before squares are summed."""
    for width in (512, 8192):
        y = 1000 + draw((4, width), "fp32", 1, 0.0)
        _, n = bacon.BlockNorm(width, pre="layer")(y)
        want = ref.normed(y.double(), "layer", None, None, 1e-6, 0.0)
        # the mean of values of 1000 in fp32: 50 roundings of 2^-24 1000 at most
        assert bool(((n.double() - want).abs() <= 2.0 ** -16 * want.abs() + 60 * 2.0 ** -24 * 1000).all())


@pytest.mark.parametrize("width", [64, 600, 1111, 2048, 3584, 8192, 12000, 20000])
def test_a_row_is_the_same_among_others_and_every_time(width):
    y, x = draw((1301, width), "bf16", 1), draw((1301, width), "bf16", 2)
    layer = bacon.BlockNorm(width, post="rms", pre="layer")
    whole, again = layer(y, x), layer(y, x)
    for part in (slice(77, 78), slice(1100, 1301)):
        for a, b, c in zip(whole, again, layer(y[part], x[part])):
            assert torch.equal(a, b) and torch.equal(a[part], c)


def test_offsets_beyond_32_bits():
    y = torch.empty(2 ** 31 // 4096 + 3, 4096, dtype=torch.bfloat16, device="cuda")
    y.fill_(1.0)
    y[-1] = draw((4096,), "bf16", 1)
    layer = bacon.BlockNorm(4096)
    layer(y, norm_out=y)
    n = y[-1]
    want = ref.normed(draw((4096,), "bf16", 1).double(), "rms", None, None, 1e-6, 0.0)
    assert bool(((n.double() - want).abs() <= (2.0 ** -8 + STEP) * want.abs() * 1.01).all())
    assert bool((y[:-1] == 1.0).all())


def test_no_tokens_and_refusals():
    layer = bacon.BlockNorm(64)
    y = draw((4, 64), "bf16", 1)
    assert layer(y[:0])[1].shape == (0, 64)
    for args in ((y[:, :32],), (y.double(),), (y, y[:3]), (y, y.half()), (y, y, y[:, :3]), (y, y, y.float()),
                 (y.t().contiguous().t(),)):
        with pytest.raises(ValueError):
            layer(*args)
    for kw in (dict(norm_out=y[:3]), dict(norm_out=y.float()), dict(sum_out=y.half())):
        with pytest.raises(ValueError):
            layer(y, y, **kw)
    with pytest.raises(ValueError):
        bacon.BlockNorm(64, pre=None)(y, y, norm_out=y)
    with pytest.raises(ValueError):
        bacon.BlockNorm(64, pre_weight=y[0, :32])(y)
    with pytest.raises(ValueError):
        bacon.BlockNorm(64, pre_weight=y[0].half())(y)
    with pytest.raises(bacon.BaconError):
        bacon.BlockNorm(64, pre=None)(y)  # nothing is wanted
    with pytest.raises(bacon.BaconError):
        bacon.BlockNorm(64, eps=0.0)(y)
    with pytest.raises(bacon.BaconError):
        layer(y, norm_out=y[:1].expand(4, 64))


def test_another_stream_and_a_graph():
    layer = bacon.BlockNorm(1111, post="layer")
    y, x = draw((30, 1111), "fp16", 1), draw((30, 1111), "fp16", 2)
    want = layer(y, x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = layer(y, x, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer(y, x)
    y.copy_(draw((30, 1111), "fp16", 5))
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(layer(y, x), out))
