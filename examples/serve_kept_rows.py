"""Serving from the rows that a compression kept.

Two prompts are compressed with head budgets shared inside each layer, so that
every head keeps its own number of rows.  The kept rows go into pages of 8-bit
values; then a few tokens are decoded, one of the prompts gets a follow-up turn
and is finished.  What a model would compute between the calls (projections of
the new tokens) is drawn at random here.  The last layer's attention is compared
with a dense one over the same rows in 16 bits, so that the difference shows
what the 8-bit pages cost.

    python examples/serve_kept_rows.py [e4m3|int8]
"""

import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2606_14782_gb300 import bacon, workloads  # noqa: E402

PAGE, DECODED, TURN = 64, 8, 40


def dense(q, k, v, ahead):
    """Attention of q [a, Hq, d] over lists of rows per kv-head, the last
    `ahead` of them the queries' own tokens."""
    out = torch.empty_like(q, dtype=torch.float32)
    group = q.shape[1] // len(k)
    for h in range(len(k)):
        x = torch.einsum("agd,nd->gan", q[:, h * group:(h + 1) * group].float(), k[h].float())
        x = x / q.shape[-1] ** 0.5
        hidden = torch.ones(ahead, ahead, dtype=torch.bool, device=q.device).triu(1)
        x[:, :, x.shape[-1] - ahead:].masked_fill_(hidden, float("-inf"))
        out[:, h * group:(h + 1) * group] = torch.einsum("gan,nd->agd", x.softmax(-1), v[h].float())
    return out


def main(format="e4m3"):
    wl = workloads.CONFIGS["tiny"].with_(q_heads=28, kv_heads=4, head_dim=128, seq_len=2000,
                                         visual=(16, 1900), requests=2, layers=3)
    budget, R, L, H = 300, wl.requests, wl.layers, wl.kv_heads
    x = workloads.generate(wl, seed=1, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(2)

    # the end of the prefill: kept rows, heads in order, and their numbers
    ctx = bacon.Context(L, H, wl.q_heads, wl.head_dim, wl.window, wl.pool, budget,
                        max_seq_len=wl.seq_len, max_requests=R)
    k, v, _, counts = ctx.compress_adaptive(x.qwin, x.k, x.v, budget)
    ctx.sync()

    # pages for them; the tables stay on the GPU, and so do the lengths
    tokens = R * L * H * budget
    pages = tokens // PAGE + R * L * H * (2 + (DECODED + TURN) // PAGE)
    cache = bacon.Cache(L, H, wl.q_heads, wl.head_dim, pages, page=PAGE, format=format,
                        max_requests=R, max_blocks=-(-(H * budget + DECODED + TURN) // PAGE))
    lengths, table, ring, state = cache.tables(R)
    slots, lengths, state = cache.plan(lengths, counts, table, ring, state, tokens)
    cache.store(k.view(tokens, -1), v.view(tokens, -1), slots)

    # the last layer's rows in 16 bits, to compare with
    kept = [[list(t.split(counts[r, L - 1].tolist())) for t in (k[r, L - 1], v[r, L - 1])]
            for r in range(R)]
    worst = 0.0

    def step(asked):
        """One forward pass of asked[r] new tokens of each request."""
        nonlocal lengths, state, worst
        T = sum(asked)
        starts = torch.tensor([0] + asked).cumsum(0).int().cuda()
        added = torch.tensor(asked, dtype=torch.int32, device="cuda")
        slots, lengths, state = cache.plan(lengths, added, table, ring, state, T)
        for l in range(L):
            fused = torch.randn(T, wl.q_heads + 2 * H, wl.head_dim, generator=gen, device="cuda")
            fused = (fused / wl.head_dim ** 0.5).to(torch.bfloat16)  # like the prompt's rows
            q, new = fused[:, :wl.q_heads], fused[:, wl.q_heads:].split(H, dim=1)
            cache.store(*new, slots[l])
            out = cache.attend(l, q, lengths, table, starts=starts)
        for r in range(R):
            mine = slice(int(starts[r]), int(starts[r + 1]))
            if asked[r] == 0:
                continue
            for rows, t in zip(kept[r], new):
                rows[:] = [torch.cat([rows[h], t[mine, h]]) for h in range(H)]
            want = dense(q[mine], *kept[r], asked[r])
            off = (out[mine].float() - want).norm() / want.norm()
            worst = max(worst, float(off))

    for _ in range(DECODED):
        step([1] * R)
    step([TURN, 1])
    cache.sync()
    free = int(state[1])
    cache.release(torch.tensor([1, 0], dtype=torch.int32, device="cuda"), lengths, table, ring, state)
    cache.sync()
    print(f"{format}: {tokens} kept rows in {pages} pages of {PAGE}; {DECODED} tokens and a turn of "
          f"{TURN} attended; difference from 16-bit rows {worst:.4f}; {int(state[1]) - free} pages "
          f"given back")
    return worst


if __name__ == "__main__":
    main(*sys.argv[1:])
