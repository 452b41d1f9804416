"""A decoding step's calls one after the other, as a program makes them: every
call's result against the plain 64-bit reference of that call on the inputs that
it got, and the whole step captured, replayed and compared with the same step
made call by call.  Bounds are those of the calls' own tests."""

import pytest
import torch

import step_reference as ref
import test_gpu_block_norm as norms
import test_gpu_logits as logits_test
import test_gpu_rotary as rotary_test
from paper_2606_14782_gb300 import bacon, build

pytestmark = pytest.mark.gpu

R, L, HQ, H, D, WIDTH, VOCAB, HELD = 3, 2, 8, 2, 64, 320, 1003, 50


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    bacon.load()


class Model:
    def __init__(self):
        gen = torch.Generator(device="cuda").manual_seed(1)

        def draw(*shape, size=1.0):
            return (size * torch.randn(shape, generator=gen, device="cuda")).to(torch.bfloat16)

        self.embedding = draw(VOCAB, WIDTH)
        self.project = [draw(WIDTH, (HQ + 2 * H) * D, size=WIDTH ** -0.5) for _ in range(L)]
        self.back = [draw(HQ * D, WIDTH, size=(HQ * D) ** -0.5) for _ in range(L)]
        self.weights = [1 + draw(WIDTH, size=0.1) for _ in range(2 * L + 2)]
        self.gate = draw(WIDTH)
        self.between = [bacon.BlockNorm(WIDTH, pre_weight=self.weights[2 * l], post="rms" if l else None,
                                        post_weight=self.weights[2 * l + 1] if l else None, gate="tanh", scale=0.5)
                        for l in range(L + 1)]
        self.qw, self.kw = 1 + draw(D, size=0.1), 1 + draw(D, size=0.1)
        self.rotary = bacon.Rotary(D, 48, scaling="linear", factor=2.0)
        self.rotary.interleaved_for_test = False
        self.rules = bacon.Logits(VOCAB)
        self.cache = bacon.Cache(L, H, HQ, D, pages=R * L * H * 8, page=16, max_requests=R, max_blocks=8)
        lengths, self.table, self.ring, state = self.cache.tables(R)
        added = torch.full((R,), HELD, dtype=torch.int32, device="cuda")
        slots, self.lengths, self.state = self.cache.plan(lengths, added, self.table, self.ring, state, R * HELD)
        for l in range(L):
            self.cache.store(draw(R * HELD, H, D), draw(R * HELD, H, D), slots[l])
        self.tokens = torch.zeros(R, dtype=torch.int64, device="cuda")
        self.place = torch.tensor([700, 5000, 123456], dtype=torch.int32, device="cuda")
        self.said = torch.full((R, 20), -1, dtype=torch.int32, device="cuda")
        self.count = torch.zeros(R, dtype=torch.int32, device="cuda")
        self.two = torch.full((R,), 2.0, device="cuda")
        self.half = torch.full((R,), 0.5, device="cuda")
        allowed = torch.rand(R, VOCAB, generator=torch.Generator().manual_seed(3)) < 0.5
        self.allowed, self.mask = allowed, logits_test.pack(allowed)

    def step(self, check=False):
        """One token of every request; the state moves on in place."""
        slots, lengths, state = self.cache.plan(self.lengths, None, self.table, self.ring, self.state, R)
        y, total = self.embedding[self.tokens], self.embedding[self.tokens]
        for l in range(L):
            gate = self.gate if l else None
            before = total
            total, n = self.between[l](y, total, gate)
            if check:
                self.check_norm(l, y, before, gate, total, n)
            fused = (n @ self.project[l]).view(R, HQ + 2 * H, D)
            q, k, v = fused.split((HQ, H, H), dim=1)
            turned = self.cache.store_rotated(self.rotary, q, k, v, self.place, slots[l], q_weight=self.qw,
                                              k_weight=self.kw)
            if check:
                rotary_test.check(self.rotary, q, k, self.place, "bf16", qw=self.qw, kw=self.kw)
                assert torch.equal(turned, self.rotary.apply(q, None, self.place, q_weight=self.qw)[0])
            out = self.cache.attend(l, turned, lengths, self.table)
            if check:
                self.check_attend(l, turned, out, lengths)
            y = out.view(R, -1) @ self.back[l]
        before = total
        total, n = self.between[L](y, total, self.gate)
        if check:
            self.check_norm(L, y, before, self.gate, total, n)
        x = n @ self.embedding.T
        got = self.rules.process(x, tokens=self.said, lengths=self.count, repetition=self.two, frequency=self.half,
                                 mask=self.mask)
        if check:
            want = [ref.rules(x[r].cpu(), self.said[r, :int(self.count[r])].tolist(), 0, 2.0, 0.5, 0.0, {},
                              self.allowed[r]) for r in range(R)]
            logits_test.verify(*got, want)
        self.lengths.copy_(lengths)
        self.state.copy_(state)
        self.said.scatter_(1, self.count.long()[:, None], got[1][:, None])
        self.count.add_(1)
        self.place.add_(1)
        self.tokens.copy_(got[1])
        return got

    def check_norm(self, l, y, x, gate, total, n):
        w = {"pre_weight": self.weights[2 * l]}
        if l:
            w["post_weight"] = self.weights[2 * l + 1]
        again = norms.check(WIDTH, y, x, gate, post="rms" if l else None, weights=w, kind="tanh", scale=0.5)
        assert torch.equal(again[0], total) and torch.equal(again[1], n)

    def check_attend(self, l, q, out, lengths):
        """Over the cache's values: the softmax's weights have 11 bits, the output 8."""
        for r in range(R):
            for h in range(H):
                one = torch.zeros_like(lengths)
                one[r, l, h] = lengths[r, l, h]
                rows = int(lengths[r, l, h])
                k, v = self.cache.load(self.cache.locate(one, self.table, rows))
                x = q[r, h * 4:h * 4 + 4].double() @ k.double().T / D ** 0.5
                want = x.softmax(-1) @ v.double()
                size = x.softmax(-1) @ v.double().abs()
                off = (out[r, h * 4:h * 4 + 4].double() - want).abs()
                # bf16's half step, the weights' 2^-11, and v rounded to 16 bits by load: 2^-8
                assert bool((off <= 2.0 ** -8 * want.abs() + (2.0 ** -10 + 2.0 ** -8) * size + 1e-6).all())


def test_every_call_of_a_step():
    m = Model()
    for _ in range(4):
        m.step(check=True)
    m.cache.sync()
    m.rules.sync()
    assert int(m.count[0]) == 4 and bool((m.tokens >= 0).all())


def test_a_captured_step_is_the_same():
    eager, captured = Model(), Model()
    a = [tuple(t.clone() for t in eager.step()) for _ in range(5)]
    first = tuple(t.clone() for t in captured.step())  # handles and libraries warm
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = captured.step()
    b = [first]
    for _ in range(4):
        graph.replay()
        b.append(tuple(t.clone() for t in got))
    captured.cache.sync()
    captured.rules.sync()
    for x, y in zip(a, b):
        assert all(torch.equal(s, t) for s, t in zip(x, y))
    assert torch.equal(eager.said, captured.said) and torch.equal(eager.lengths, captured.lengths)


def test_two_handles_and_two_graphs():
    """Two captured steps of two programs, replayed in turn: nothing is shared."""
    one, two = Model(), Model()
    two.place += 17
    one.step(), two.step()
    graphs = []
    for m in (one, two):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = m.step()
        graphs.append((g, got))
    alone = Model()
    alone.step()
    for _ in range(3):
        graphs[0][0].replay()
        graphs[1][0].replay()
        want = alone.step()
        assert all(torch.equal(s, t) for s, t in zip(graphs[0][1], want))
