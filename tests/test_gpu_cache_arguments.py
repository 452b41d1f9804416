"""Host tensors given to the 8-bit cache's calls are refused before anything is
launched, outputs among them."""

import pytest
import torch

from paper_2606_14782_gb300 import bacon, build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    bacon.load()


def test_host_outputs_and_inputs_are_refused():
    cache = bacon.Cache(1, 2, 4, 64, 16, page=16, max_requests=2, max_blocks=4)
    lengths, table, ring, state = cache.tables(2)
    slots, lengths, state = cache.plan(lengths, None, table, ring, state, 2)
    kv = torch.randn(2, 2, 64, device="cuda").to(torch.bfloat16)
    cache.store(kv, kv, slots[0])
    q = torch.randn(2, 4, 64, device="cuda").to(torch.bfloat16)
    want, lse = cache.attend(0, q, lengths, table, lse=True)
    flat = slots.view(-1)
    rows = cache.load(flat)
    for call in (lambda: cache.attend(0, q, lengths, table, out=want.cpu()),
                 lambda: cache.attend(0, q, lengths, table, lse=lse.cpu()),
                 lambda: cache.attend(0, q.cpu(), lengths, table),
                 lambda: cache.attend(0, q, lengths.cpu(), table),
                 lambda: cache.load(flat, k_out=rows[0].cpu()),
                 lambda: cache.load(flat, v_out=rows[1].cpu()),
                 lambda: cache.load(flat.cpu()),
                 lambda: cache.store(kv.cpu(), kv, slots[0]),
                 lambda: cache.plan(lengths, None, table, ring, state, 2, slots=slots.cpu()),
                 lambda: cache.locate(lengths, table, 2, slots=flat[:2].cpu()),
                 lambda: cache.release(torch.ones(2, dtype=torch.int32), lengths, table, ring, state),
                 lambda: bacon.Cache(1, 2, 4, 64, 16, page=16, k=cache.k.cpu())):
        with pytest.raises(ValueError):
            call()
    again, z = cache.attend(0, q, lengths, table, out=torch.empty_like(want),
                            lse=torch.empty_like(lse))
    cache.sync()
    assert torch.equal(again, want) and torch.equal(z, lse)
