"""Rows with infinities and NaN: the log-sum-exp is an infinity's, unless there is NaN."""

import pytest
import torch

from paper_2606_14782_gb300 import bacon, build

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("vocab", [7, 1000, 32000, 50021, 131072])
@pytest.mark.parametrize("temperature", [None, 0.5, 3e38])
def test_rows_with_infinities(vocab, dtype, temperature):
    build.build()
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    last, mid = vocab - 1, vocab // 2
    given = [{}, {3: INF}, {3: INF, last: INF}, {3: NAN}, {3: INF, mid: NAN}, {mid: NAN, last: INF}, {0: INF, 1: NAN},
             {0: NAN, 1: INF}, {last - 1: INF, last: -INF}, {mid: -INF}, {mid: NAN, last: -INF}]
    x = torch.randn(len(given), vocab, generator=gen, device="cuda").to(dtype)
    for r, row in enumerate(given):
        for at, v in row.items():
            x[r, at] = v
    handle = bacon.Logits(vocab)
    t = None if temperature is None else torch.full((len(given),), temperature, device="cuda")
    out, best, logprob, lse = handle.process(x, temperature=t)
    handle.sync()
    z = x.double() / (temperature or 1.0)
    want = z.logsumexp(-1)
    assert torch.equal(lse.isnan(), want.isnan()) and torch.equal(lse == INF, want == INF)
    ok = want.isfinite()
    # a sum of 2^17 values in chains of 2^10 at most, a logarithm and a sum
    assert bool(((lse.double() - want)[ok].abs() <= 2.0 ** -13 + 2.0 ** -22 * want[ok].abs()).all())
    for r, row in enumerate(given):
        top = x[r].double().nan_to_num(nan=-INF, posinf=INF).max()
        assert int(best[r]) == int((x[r] == top).nonzero()[0])
        # an infinity's share of an infinity is not a number
        assert bool(logprob[r].isnan()) == any(v == INF or v != v for v in row.values())
    handle.close()


def test_masked_infinities_do_not_count():
    vocab = 5000
    x = torch.zeros(4, vocab, device="cuda")
    x[0, 10], x[0, 11], x[1, 10], x[2, 11] = INF, NAN, INF, NAN
    words = torch.full((4, (vocab + 31) // 32), -1, dtype=torch.int32, device="cuda")
    words[:, 0] = ~(1 << 10 | 1 << 11)
    words[3] = 0
    handle = bacon.Logits(vocab)
    _, best, logprob, lse = handle.process(x, mask=words)
    assert best.tolist() == [0, 0, 0, -1] and bool(lse[:3].isfinite().all()) and lse[3].item() == -INF
    want = torch.log(torch.tensor(vocab - 2.0, dtype=torch.float64))
    # vocab - 2 ones add up exactly: a logarithm
    assert bool(((lse[:3].double().cpu() - want).abs() <= 2.0 ** -20 * want).all())
    assert torch.equal(logprob[:3], -lse[:3])
    handle.close()
