"""Frequencies scaled over a ramp of pairs ("dims") against the header's definition:
the ramp's end is the pair that turns `low` times over the original length, rounded up,
and may lie behind the last pair.  No GPU is needed."""

import math

import pytest

from paper_2606_14782_gb300 import bacon, build


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()


def defined(D, base, factor, original, low, high):
    def pair(turns):  # original base^(-2 i / D) = 2 pi turns
        return D / 2 * math.log(original / (math.tau * turns), base)
    first, last = max(0, math.floor(pair(high))), math.ceil(pair(low))
    for i in range(D // 2):
        theta = base ** (-2 * i / D)
        kept = min(1.0, max(0.0, 1 - (i - first) / max(last - first, 0.5)))
        yield kept * theta + (1 - kept) * theta / factor


@pytest.mark.parametrize("D,base,factor,original,low,high,end", [
    (128, 1e4, 4.0, 131072, 1.0, 32.0, 70), (64, 1e4, 16.0, 65536, 1.0, 32.0, 33),
    (16, 1e4, 4.0, 32768, 1.0, 32.0, 8), (128, 500.0, 8.0, 32768, 1.0, 32.0, 89),
    (128, 1e4, 16.0, 4096, 1.0, 32.0, 46), (64, 1e6, 40.0, 100, 1.0, 32.0, 7),
    (128, 1e4, 8.0, 1 << 30, 1.0, 32.0, 132)])
def test_ramp_ends_where_it_ends(D, base, factor, original, low, high, end):
    """log and pow in 64 bits, times a ramp up to 2^7 pairs long: 2^-40 of the value."""
    assert math.ceil(D / 2 * math.log(original / (math.tau * low), base)) == end
    got = bacon.Rotary(D, base=base, scaling="dims", factor=factor, original=original, low=low, high=high).frequencies
    for g, w in zip(got, defined(D, base, factor, original, low, high)):
        assert abs(g - w) <= 2.0 ** -40 * w


def test_far_ramps_keep_a_part_of_the_last_pair():
    plain = bacon.Rotary(64).frequencies[-1]
    last = bacon.Rotary(64, scaling="dims", factor=16.0, original=65536).frequencies[-1]
    assert last > 3 * plain / 16
    # all pairs turn more than `high` times: nothing is scaled
    far = bacon.Rotary(64, scaling="dims", factor=16.0, original=1e12)
    assert far.frequencies == bacon.Rotary(64).frequencies
