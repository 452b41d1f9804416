"""Serving from the rows that a compression kept.

Two prompts are compressed with head budgets shared inside each layer, so that
every head keeps its own number of rows.  The kept rows go into pages of 8-bit
values; then a few tokens are decoded, one of the prompts gets a follow-up turn
and is finished.  Around the cache runs a small model of random weights: norms
between its blocks, positions behind the whole prompt (not behind the rows that
were kept) put into Q and K as K is stored, and the next token by the rules on
the logits.  The last layer's attention is compared with a dense one over the
same rows in 16 bits, so that the difference shows what the 8-bit pages cost.

    python examples/serve_kept_rows.py [e4m3|int8]
"""

import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2606_14782_gb300 import bacon, workloads  # noqa: E402

PAGE, DECODED, TURN, WIDTH, VOCAB = 64, 8, 40, 512, 1000


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

    # the model: random weights of sizes that give rows like the prompt's
    def weight(rows, columns, size):
        return (size * torch.randn(rows, columns, generator=gen, device="cuda")).to(torch.bfloat16)

    d = wl.head_dim
    embedding = weight(VOCAB, WIDTH, 1.0)
    project = [weight(WIDTH, (wl.q_heads + 2 * H) * d, (WIDTH * d) ** -0.5) for _ in range(L)]
    back = [weight(wl.q_heads * d, WIDTH, (wl.q_heads * d) ** -0.5) for _ in range(L)]
    unembed = weight(WIDTH, VOCAB, WIDTH ** -0.5)
    between = [bacon.BlockNorm(WIDTH) for _ in range(L + 1)]
    rotary = bacon.Rotary(d)
    rules = bacon.Logits(VOCAB)
    place = torch.full((R,), wl.seq_len, dtype=torch.int32, device="cuda")
    said = torch.full((R, DECODED + TURN + 2), -1, dtype=torch.int32, device="cuda")
    count = torch.zeros(R, dtype=torch.int32, device="cuda")
    penalty = torch.full((R,), 1.2, device="cuda")

    def step(asked, tokens):
        """One forward pass of asked[r] new tokens of each request; returns each
        request's next token."""
        nonlocal lengths, state, worst, place
        T = sum(asked)
        starts = torch.tensor([0] + asked).cumsum(0).int().cuda()
        added = torch.tensor(asked, dtype=torch.int32, device="cuda")
        request = torch.repeat_interleave(torch.arange(R, device="cuda"), added.long(), output_size=T)
        at = torch.arange(T, dtype=torch.int32, device="cuda") - starts[request] + place[request]
        place = place + added
        slots, lengths, state = cache.plan(lengths, added, table, ring, state, T)
        y, total = embedding[tokens], None
        for l in range(L):
            total, n = between[l](y, total, sum_out=None if l else torch.empty_like(y))
            fused = (n @ project[l]).view(T, wl.q_heads + 2 * H, d)
            q, k, v = fused.split((wl.q_heads, H, H), dim=1)
            q = cache.store_rotated(rotary, q, k, v, at, slots[l])
            out = cache.attend(l, q, lengths, table, starts=starts)
            y = out.view(T, -1) @ back[l]
        new = rotary.apply(None, k, at)[1], v
        for r in range(R):
            mine = slice(int(starts[r]), int(starts[r + 1]))
            if asked[r] == 0:
                continue
            for rows, t in zip(kept[r], new):
                rows[:] = [torch.cat([rows[h], t[mine, h]]) for h in range(H)]
            want = dense(q[mine], *kept[r], asked[r])
            off = (out[mine].float() - want).norm() / want.norm()
            worst = max(worst, float(off))
        last = starts[1:].long() - 1  # each request's last token (all have one)
        _, n = between[L](y[last], total[last])
        _, best, _, _ = rules.process(n @ unembed, tokens=said, lengths=count, repetition=penalty,
                                      out=False)
        said[torch.arange(R, device="cuda"), count.long()] = best
        count.add_(1)
        return best.long()

    token = torch.zeros(R, dtype=torch.int64, device="cuda")
    for _ in range(DECODED):
        token = step([1] * R, token)
    turn = torch.randint(0, VOCAB, (TURN,), generator=gen, device="cuda")
    step([TURN, 1], torch.cat([turn, token[1:]]))
    rules.sync()
    cache.sync()
    free = int(state[1])
    cache.release(torch.tensor([1, 0], dtype=torch.int32, device="cuda"), lengths, table, ring, state)
    cache.sync()
    print(f"{format}: {tokens} kept rows in {pages} pages of {PAGE}; {DECODED} tokens and a turn of "
          f"{TURN} attended, tokens {said[0, :DECODED].tolist()}; difference from 16-bit rows {worst:.4f}; {int(state[1]) - free} pages "
          f"given back")
    return worst


if __name__ == "__main__":
    main(*sys.argv[1:])
