"""Failure detection of the cache's attention: a pipeline wait that runs out is
reported, not hung.

Every wait is bounded (about a second of clock cycles).  When one runs out, the
block raises its abort flag, its roles end, its copies in flight are waited for,
tensor memory is freed, and bacon_cache_sync reports BACON_ETIMEOUT.  The fault
is injected on the host: with BACON_FAULT=missing_page set when the cache is
created, its next attention withholds one load of 16 rows, so that its waiters
wait for data that never comes.  Nothing faults or traps.  The test runs in a
child process and checks that the error comes back, that the cache stays usable
and that its next call matches a fresh cache bit for bit.
"""

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
    R, H, G, d, page, asked, held = 3, 2, 7, 128, 32, {asked}, 700
    blocks = -(-(held + asked) // page)

    def cache(like=None):
        pools = {{}} if like is None else dict(k=like.k, v=like.v, k_scale=like.k_scale,
                                               v_scale=like.v_scale)
        return bacon.Cache(1, H, H * G, d, R * H * blocks, page=page, max_requests=R,
                           max_blocks=blocks, **pools)

    c = cache()                          # BACON_FAULT is set: one fault pending
    os.environ.pop("BACON_FAULT")
    lengths, table, ring, state = c.tables(R)
    added = torch.full((R, 1, H), held + asked, dtype=torch.int32, device="cuda")
    n = int(added.sum())
    slots, lengths, state = c.plan(lengths, added, table, ring, state, n)
    rows = [torch.randn(n, d, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2)]
    c.store(*rows, slots)
    c.sync()
    q = torch.randn(R * asked, H * G, d, generator=gen, device="cuda").to(torch.bfloat16)
    t0 = time.time()
    c.attend(0, q, lengths, table)
    try:
        c.sync()
        print("STATUS", 0)
    except bacon.BaconError as e:
        print("STATUS", e.status)
    print("SECONDS", round(time.time() - t0, 2))
    out = c.attend(0, q, lengths, table)
    c.sync()
    fresh = cache(c)
    want = fresh.attend(0, q, lengths, table)
    fresh.sync()
    print("SAME", int(torch.equal(out, want)), int(torch.isfinite(out).all()))
""")


@pytest.mark.parametrize("asked", [1, 90])  # either kernel
def test_a_missing_page_times_out_and_the_cache_recovers(asked):
    env = dict(os.environ, BACON_FAULT="missing_page")
    proc = subprocess.run([sys.executable, "-c", CHILD.format(root=ROOT, asked=asked)], env=env,
                          capture_output=True, text=True, timeout=300)
    assert proc.returncode == 0, proc.stderr[-2000:]
    lines = dict(line.split(" ", 1) for line in proc.stdout.splitlines() if " " in line)
    from paper_2606_14782_gb300 import bacon
    assert int(lines["STATUS"]) == bacon.BACON_ETIMEOUT, proc.stdout
    assert float(lines["SECONDS"]) < 30.0, proc.stdout     # bounded waits, no hang
    assert lines["SAME"].split() == ["1", "1"], proc.stdout
