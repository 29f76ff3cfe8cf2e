"""The bands of scaled frequencies at their edges (host, no GPU): contexts so long that every frequency turns often, or so short that
none does."""
import math

import pytest
import torch


@pytest.fixture(scope="module")
def frequencies():
    from paper_2608_00029_b200 import build, nova_rope
    build.build()
    return nova_rope.nova_rope_frequencies


@pytest.mark.parametrize("kind", ["bands", "yarn"])
@pytest.mark.parametrize("rotary,base,original,low,high", [
    (64, 10.0, 32768, 1.0, 32.0),      # the slowest turns 600 times: none is scaled
    (64, 10000.0, 2**40, 1.0, 32.0),
    (2, 10000.0, 8192, 1.0, 32.0),     # a single pair
    (64, 10000.0, 128, 32.0, 64.0),    # the fastest turns 20 times: all are
    (64, 10000.0, 4, 1.0, 32.0),
    (2, 500.0, 6, 1.0, 2.0),
    (64, 10000.0, 4096, 1.0, 32.0),    # ordinary ones
    (128, 500000.0, 8192, 1.0, 4.0),
    (96, 100.0, 300, 2.0, 3.0),
])
def test_what_turns_often_stays_and_what_does_not_is_divided(frequencies, kind, rotary, base, original, low, high):
    f, _ = frequencies(rotary, base, kind, 8.0, original, low, high)
    plain = base ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / rotary)
    turns = original * plain / (2 * math.pi)
    ratio = f.double() / plain
    often, seldom = turns >= high * (1 + 1e-9), turns <= low * (1 - 1e-9)
    assert ((ratio - 1).abs()[often] <= 2.0**-23).all()
    assert ((ratio * 8 - 1).abs()[seldom] <= 2.0**-23).all()
    assert (ratio >= 1 / 8 - 1e-6).all() and (ratio <= 1 + 1e-6).all()
