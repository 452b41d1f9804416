"""Model of what the cache's attention kernels do when a load never comes, run
on the CPU.

A block has a warp that loads (tiles of pages into a ring of stages, or into one
raw buffer each for K and V that other warps convert; the query rows of an item
into two slots) and warps that compute.  One load is withheld: its bytes are
expected on the barrier and never arrive.  Waits are bounded and end early when
the block's abort flag is set, except the last ones of the loading warp; a wait
tests a parity, so it also returns when the barrier is a phase behind or ahead.
Whatever the interleaving, every warp has to finish, no barrier may be armed
again while its phase is open, and when the block ends no copy may be on its way
into its shared memory.  `old` is the protocol that looked at the flag only
while it waited and waited for its copies only when the loading warp itself had
given up; the model finds its faults."""

import random

import pytest


class Bar:
    """An mbarrier: a phase ends with `count` arrivals and no copy expected."""

    def __init__(self, count, name):
        self.count, self.pending, self.tx = count, count, 0
        self.phase, self.name = 0, name

    def _close(self):
        if self.pending == 0 and self.tx == 0:
            self.phase += 1
            self.pending = self.count

    def expect(self):
        self.tx += 1

    def arrive(self):
        if self.pending == 0:
            raise Fault(f"{self.name}: armed again while its phase is open")
        self.pending -= 1
        self._close()

    def land(self):
        self.tx -= 1
        self._close()


class Fault(Exception):
    pass


class Block:
    """Bounded waits, copies on their way and the roles' interleaving."""

    def __init__(self, seed, slow, limit=250):
        self.rnd = random.Random(seed)
        self.slow, self.limit = slow, limit  # the odds that a copy lands in a step
        self.copies, self.commits, self.abort, self.gave_up = [], [], False, False

    def copy(self, bar, withheld):
        bar.expect()
        if not withheld:
            self.copies.append(bar)

    def wait(self, bar, k, flag=True):
        """Whether phase k was seen to be over.  (A copy that was asked for takes
        microseconds of the second that a wait may last; other warps' waits may
        have started long before it, so theirs are shorter here.)"""
        polls = 0
        while (bar.phase & 1) == (k & 1):
            if (flag and self.abort) or polls > (self.limit if flag else 20 * self.limit):
                return False
            polls += 1
            yield
        return True

    def give_up(self):
        self.abort = self.gave_up = True

    def run(self, roles):
        live = list(roles)
        for _ in range(2000000):
            if not live:
                if self.copies:
                    return "a copy was on its way when the block ended"
                return None if self.gave_up else "nobody noticed"
            x = self.rnd.random()
            if self.copies and x < self.slow:
                self.copies.pop(self.rnd.randrange(len(self.copies))).land()
                continue
            if self.commits and x < 0.5:
                self.commits.pop(0).arrive()
                continue
            i = self.rnd.randrange(len(live))
            try:
                next(live[i])
            except StopIteration:
                live.pop(i)
            except Fault as f:
                return str(f)
        return "deadlock"


# ----------------------------------------------- few queries: ring of stages

def few(items, missing, seed, old, slow, stages=3, warps=4):
    """items: tiles of each item of the block."""
    b = Block(seed, slow)
    full = [Bar(1, f"full{i}") for i in range(stages)]
    empty = [Bar(warps, f"empty{i}") for i in range(stages)]
    q_full = [Bar(1, f"q_full{i}") for i in range(2)]
    q_empty = [Bar(warps, f"q_empty{i}") for i in range(2)]
    meet = Bar(warps, "named barrier")
    quit = [False]

    def load():
        issued = asked = 0
        stop = False
        for tiles in items:
            there = yield from b.wait(q_empty[asked & 1], (asked >> 1) - 1)
            if not there or (b.abort and not old):
                stop = True
                break
            b.copy(q_full[asked & 1], False)
            yield
            q_full[asked & 1].arrive()
            asked += 1
            for _ in range(tiles):
                s = issued % stages
                there = yield from b.wait(empty[s], issued // stages - 1)
                if not there or (b.abort and not old):
                    stop = True
                    break
                b.copy(full[s], issued == missing)
                yield
                full[s].arrive()
                issued += 1
            if stop:
                break
        if stop:
            b.give_up()
        if stop or not old:
            for i in range(max(0, issued - stages), issued):
                yield from b.wait(full[i % stages], i // stages, flag=False)
            for i in range(max(0, asked - 2), asked):
                yield from b.wait(q_full[i & 1], i >> 1, flag=False)

    def together(n):
        """The n-th meeting of the warps (not bounded)."""
        meet.arrive()
        while meet.phase <= n:
            yield

    def compute(w):
        met = seq = 0
        for k, tiles in enumerate(items):
            there = yield from b.wait(q_full[k & 1], k >> 1)
            if not there:
                b.give_up()
            if w == 0:
                quit[0] = not there
            yield from together(met)
            met += 1
            if quit[0]:
                return
            q_empty[k & 1].arrive()
            for i in range(tiles):
                s = (seq + i) % stages
                there = yield from b.wait(full[s], (seq + i) // stages)
                if not there:
                    b.give_up()
                yield
                empty[s].arrive()
            seq += tiles
            for _ in range(2):  # the joining
                yield from together(met)
                met += 1

    return b.run([load()] + [compute(w) for w in range(warps)])


# ------------------------------------- many queries: raw tiles and converters

def many(items, missing, seed, old, slow):
    """One row tile, two warps of each converting role, two of the softmax."""
    b = Block(seed, slow)
    raw = {x: (Bar(1, f"raw{x}_full"), Bar(2, f"raw{x}_empty")) for x in "kv"}
    made = {x: [Bar(2, f"{x}_full{i}") for i in range(2)] for x in "kv"}
    used = {x: [Bar(1, f"{x}_empty{i}") for i in range(2)] for x in "kv"}
    s_full, o_full, q_full = Bar(1, "s_full"), Bar(1, "o_full"), Bar(2, "q_full")
    p_full, drain = Bar(2, "p_full"), Bar(1, "drain")
    meta = [Bar(1, f"meta{i}") for i in range(4)]
    item_full = [Bar(1, f"item_full{i}") for i in range(2)]
    item_done = [Bar(2, f"item_done{i}") for i in range(2)]
    meet, quit, ended = Bar(2, "named barrier"), [False], Bar(8, "end of the block")

    def wait(bar, k):
        there = yield from b.wait(bar, k)
        if not there:
            b.give_up()
        return there

    def end():
        ended.arrive()
        while ended.phase == 0:
            yield

    def load():
        seq = keys = values = 0
        good = True
        for k, tiles in enumerate(items):
            good = yield from wait(item_done[k & 1], (k >> 1) - 1)
            if not good or (b.abort and not old):
                good = False
                break
            item_full[k & 1].arrive()
            for _ in range(tiles):
                for x in "kv":
                    good = yield from wait(raw[x][1], seq - 1)
                    if not good:
                        break
                    b.copy(raw[x][0], x == "k" and seq == missing)
                    yield
                    raw[x][0].arrive()
                    if x == "k":
                        keys += 1
                        yield
                        meta[seq & 3].arrive()
                    else:
                        values += 1
                if not good:
                    break
                seq += 1
            if not good:
                break
        if old and not good:
            yield from b.wait(raw["k"][0], seq, flag=False)
            if seq:
                yield from b.wait(raw["v"][0], seq - 1, flag=False)
        if not old:
            if keys:
                yield from b.wait(raw["k"][0], keys - 1, flag=False)
            if values:
                yield from b.wait(raw["v"][0], values - 1, flag=False)
        yield from end()

    def convert(x):
        seq = 0
        for k, tiles in enumerate(items):
            if x == "v":
                if not (yield from wait(item_full[k & 1], k >> 1)):
                    yield from end()
                    return
            for _ in range(tiles):
                good = yield from wait(raw[x][0], seq)
                good = good and (yield from wait(used[x][seq & 1], (seq >> 1) - 1))
                if not good:
                    yield from end()
                    return
                yield
                made[x][seq & 1].arrive()
                raw[x][1].arrive()
                seq += 1
        yield from end()

    def issue():
        seq = p = 0
        good = True
        for k, tiles in enumerate(items):
            good = yield from wait(item_full[k & 1], k >> 1)
            good = good and (yield from wait(q_full, k))
            good = good and (yield from wait(made["k"][seq & 1], seq >> 1))
            if not good:
                break
            b.commits += [s_full, used["k"][seq & 1]]
            for i in range(tiles):
                good = yield from wait(made["v"][seq & 1], seq >> 1)
                if i + 1 < tiles:
                    good = good and (yield from wait(made["k"][(seq + 1) & 1], (seq + 1) >> 1))
                good = good and (yield from wait(p_full, p))
                if not good:
                    break
                p += 1
                b.commits.append(used["v"][seq & 1])
                if i + 1 < tiles:
                    b.commits += [s_full, used["k"][(seq + 1) & 1]]
                else:
                    b.commits.append(o_full)
                seq += 1
            if not good:
                break
        b.commits.append(drain)
        if not (yield from b.wait(drain, 0, flag=False)):
            raise Fault("the products issued did not end")
        yield from end()

    def softmax(w):
        met = seq = s = 0
        for k, tiles in enumerate(items):
            there = yield from wait(item_full[k & 1], k >> 1)
            if w == 0:
                quit[0] = not there or (b.abort and not old)
            meet.arrive()
            while meet.phase <= met:
                yield
            met += 1
            if quit[0]:
                break
            yield
            if q_full.pending == 0:
                raise Fault("queries of two items at once")
            q_full.arrive()
            for _ in range(tiles):
                yield from wait(meta[seq & 3], seq >> 2)
                yield from wait(s_full, s)
                seq, s = seq + 1, s + 1
                yield
                p_full.arrive()
            yield from wait(o_full, k)
            yield
            item_done[k & 1].arrive()
        yield from end()

    return b.run([load(), issue()] + [convert(x) for x in "kkvv"] + [softmax(w) for w in range(2)])


WORK = [[1], [2], [3], [4, 2], [1, 1, 1, 1, 1], [7], [2, 9, 1], [12, 3]]
CASES = [(w, m) for w in WORK for m in sorted({0, 1, sum(w) // 2, sum(w) - 1}) if m < sum(w)]


@pytest.mark.parametrize("kernel", [few, many])
@pytest.mark.parametrize("items,missing", CASES)
def test_the_block_ends_without_a_copy_on_its_way(kernel, items, missing):
    for seed in range(6):
        for slow in (0.3, 0.03, 0.004):
            fault = kernel(items, missing, seed, False, slow)
            assert fault is None, (seed, slow, fault)


@pytest.mark.parametrize("kernel", [few, many])
def test_the_model_finds_the_old_protocols_copies(kernel):
    faults = {kernel(items, missing, seed, True, 0.004)
              for items, missing in CASES for seed in range(6)}
    assert "a copy was on its way when the block ended" in faults, faults


def test_the_model_finds_a_stage_that_is_armed_again():
    faults = {few(items, missing, seed, True, 0.3)
              for items, missing in CASES for seed in range(6)}
    assert any(f and "armed again" in f for f in faults), faults
