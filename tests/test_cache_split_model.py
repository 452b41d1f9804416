"""Model of how the cache's attention deals its tiles to blocks, run on the CPU:
every part of a cut item belongs to a block that runs and finishes it, and every
slot of partial sums that is written or read exists.  That holds for query
ranges that follow one another; for overlapping ones it does not (the model
shows a call whose items need more blocks than run), so that such a call has to
be refused as a whole."""

import random

import pytest

SMS = 152


def items_of(starts, lengths, group, rows, tile, causal=True):
    """Tiles of every item (rows of a unit's queries), in the kernel's order."""
    out = []
    for r, units in enumerate(lengths):
        asked = starts[r + 1] - starts[r]
        for n in units:
            for block in range(-(-max(asked, 0) * group // rows)):
                last = min(asked - 1, (block * rows + rows - 1) // group)
                seen = max(0, n - asked + last + 1) if causal else n
                out.append(max(1, -(-seen // tile)))
    return out


def deal(items, expected, grid, least):
    """[(first block, parts)] of every item, and the number of blocks."""
    total = sum(items)
    if expected * 4 <= grid and total <= 16 * grid:
        run = max(least, -(-total // (grid - expected)))
        out, at = [], 0
        for tiles in items:
            parts = -(-tiles // run)
            out.append((at, parts))
            at += parts
        return out, at
    blocks = min(total, grid)
    share, more = divmod(total, blocks) if blocks else (0, 0)

    def owner(t):
        long = (share + 1) * more
        return t // (share + 1) if t < long else more + (t - long) // share

    out, at = [], 0
    for tiles in items:
        out.append((owner(at), owner(at + tiles - 1) - owner(at) + 1))
        at += tiles
    return out, blocks


def fits(starts, lengths, group, rows, tile, grid, least, requests):
    tokens = starts[-1]
    heads = len(lengths[0])
    expected = (tokens * group // rows + requests) * heads
    parts, blocks = deal(items_of(starts, lengths, group, rows, tile), expected, grid, least)
    return blocks <= grid and all(f + n <= grid for f, n in parts)


KERNELS = [(8, 64, 3 * SMS, 1), (16, 64, 2 * SMS, 1), (32, 128, SMS, 1), (256, 128, SMS, 2)]


@pytest.mark.parametrize("rows,tile,grid,least", KERNELS)
def test_parts_lie_in_the_grid(rows, tile, grid, least):
    rng = random.Random(rows)
    for _ in range(400):
        R, H, group = rng.randint(1, 40), rng.randint(1, 8), rng.randint(1, 12)
        most = rng.choice([1, 4, 60, 500])
        asked = [rng.randint(0, most) for _ in range(R)]
        starts = [sum(asked[:i]) for i in range(R + 1)]
        longest = rng.choice([0, 3, 200, 5000, 60000])
        lengths = [[rng.randint(0, longest) for _ in range(H)] for _ in range(R)]
        assert fits(starts, lengths, group, rows, tile, grid, least, R), (starts, lengths, group)


def test_overlapping_ranges_would_not_fit():
    R, asked = 24, 300
    starts = [0 if r % 2 == 0 else asked for r in range(R)] + [asked]
    lengths = [[2500] for _ in range(R)]
    assert not fits(starts, lengths, 7, 256, 128, SMS, 2, R)
