"""Histories of no entries: a length that is not 0 is outside them, and is reported."""

import pytest
import torch

from paper_2606_14782_gb300 import bacon, build

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [100, 50021, 131072])
def test_histories_without_entries(vocab):
    build.build()
    rows = 3
    x = torch.randn(rows, vocab, device="cuda")
    none = torch.empty(rows, 0, dtype=torch.int32, device="cuda")
    penalty = torch.full((rows,), 1.5, device="cuda")
    handle = bacon.Logits(vocab)
    want = handle.process(x)

    def call(*lengths):
        return handle.process(x, tokens=none, lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"),
                              repetition=penalty)

    assert all(torch.equal(a, b) for a, b in zip(call(0, 0, 0), want))
    handle.sync()
    # left out, as any history that is not what its length says
    assert all(torch.equal(a, b) for a, b in zip(call(0, 5, 0), want))
    with pytest.raises(bacon.BaconError):
        handle.sync()
    handle.sync()
    nobody = none[:0]  # no lines at all
    lengths = torch.zeros(rows, dtype=torch.int32, device="cuda")
    assert all(torch.equal(a, b) for a, b in zip(handle.process(x, tokens=nobody, lengths=lengths), want))
    handle.sync()
    handle.process(x, tokens=nobody, lengths=lengths + 1)
    with pytest.raises(bacon.BaconError):
        handle.sync()
    handle.close()
