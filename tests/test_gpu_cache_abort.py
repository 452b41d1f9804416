"""Failure detection of the cache's attention in the middle of a block's work.

As in test_gpu_cache_faults.py, with the withheld load in a later tile of a
block that has many tiles, or several items: stages are in use again, later
loads are on their way and later items still to come when the waits run out.
BACON_FAULT=missing_page:<tile> is read when the cache is created; nothing
faults or traps.  The error comes back once, the cache stays usable, and what it
computes next is bit for bit what a fresh cache computes."""

import os
import subprocess
import sys
import textwrap

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = textwrap.dedent("""
    import os, sys, time
    sys.path.insert(0, {root!r})
    import torch
    from paper_2606_14782_gb300 import bacon, build

    build.build()
    gen = torch.Generator(device="cuda").manual_seed(1)
    R, H, G, d, page, asked, held = {shape}
    blocks = -(-held // page)
    pages = R * H * blocks

    def cache(like=None):
        pools = {{}} if like is None else dict(k=like.k, v=like.v, k_scale=like.k_scale,
                                               v_scale=like.v_scale)
        return bacon.Cache(1, H, H * G, d, pages, page=page, format="int8", max_requests=R,
                           max_blocks=blocks, **pools)

    c = cache()                          # BACON_FAULT is set: one fault pending
    os.environ.pop("BACON_FAULT")
    for codes, scale in ((c.k, c.k_scale), (c.v, c.v_scale)):
        codes.copy_(torch.randint(0, 256, codes.shape, generator=gen, device="cuda"))
        scale.fill_(0.01)
    table = torch.randperm(pages, generator=gen, device="cuda").int().view(R, 1, H, blocks)
    lengths = torch.full((R, 1, H), held, dtype=torch.int32, device="cuda")
    q = torch.randn(R * asked, H * G, d, generator=gen, device="cuda").to(torch.bfloat16)
    t0 = time.time()
    c.attend(0, q, lengths, table)
    try:
        c.sync()
        print("STATUS", 0)
    except bacon.BaconError as e:
        print("STATUS", e.status)
    print("SECONDS", round(time.time() - t0, 2))
    out, lse = c.attend(0, q, lengths, table, lse=True)
    c.sync()
    fresh = cache(c)
    want, z = fresh.attend(0, q, lengths, table, lse=True)
    fresh.sync()
    print("SAME", int(torch.equal(out, want)), int(torch.equal(lse, z)), int(torch.isfinite(out).all()))
""")

LONG = (40, 4, 7, 128, 64, 1, 5500)      # about 30 tiles a block, one or two items
SHORT = (40, 32, 1, 128, 64, 1, 300)     # 5 tiles an item, 14 a block
TURNS = (4, 2, 7, 128, 64, 90, 16000)    # about 20 tiles a block
SHORT_TURNS = (120, 8, 4, 64, 32, 60, 250)  # 2 tiles an item, 12 or 13 a block


@pytest.mark.parametrize("shape,tile", [(LONG, 1), (LONG, 11), (LONG, 29), (SHORT, 4), (SHORT, 9),
                                        (TURNS, 1), (TURNS, 10), (TURNS, 19), (SHORT_TURNS, 3),
                                        (SHORT_TURNS, 8)])
def test_a_page_missing_later_times_out_and_the_cache_recovers(shape, tile):
    env = dict(os.environ, BACON_FAULT=f"missing_page:{tile}")
    proc = subprocess.run([sys.executable, "-c", CHILD.format(root=ROOT, shape=shape)], env=env,
                          capture_output=True, text=True, timeout=300)
    assert proc.returncode == 0, proc.stderr[-2000:]
    lines = dict(line.split(" ", 1) for line in proc.stdout.splitlines() if " " in line)
    from paper_2606_14782_gb300 import bacon
    assert int(lines["STATUS"]) == bacon.BACON_ETIMEOUT, proc.stdout
    assert float(lines["SECONDS"]) < 30.0, proc.stdout     # bounded waits, no hang
    assert lines["SAME"].split() == ["1", "1", "1"], proc.stdout
