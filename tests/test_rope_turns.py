"""The turns of a position: the nearest multiple of 2^-64 at every frequency, and so the promised angle at any position."""
from __future__ import annotations

from fractions import Fraction

import numpy as np
import pytest

import paper_2512_18337_b200 as S
from tests.test_step_host import TWO_PI

FREQUENCIES = [0.0, 5e-324, 2.0 ** -70, 1e-9, 0.3, 1.0, 6.283185307179586, -100.25, 800.0, 1e3, 54321.0625, 999_983.7, -777_777.7, 1e6, -1e6]


@pytest.mark.parametrize("f", FREQUENCIES)
def test_nearest(f):
    got = int(S.sam_rope_turns([f])[0])
    off = (Fraction(got, 1 << 64) - Fraction(f) / TWO_PI) % 1
    # TWO_PI has 60 digits: what it adds for 2^20 radians lies below 2^-170
    assert min(off, 1 - off) <= Fraction(1, 1 << 65) + Fraction(1, 1 << 150)


@pytest.mark.parametrize("f", FREQUENCIES)
def test_any_position(f):
    turns = int(S.sam_rope_turns([f])[0])
    for p in (1, 250_000, (1 << 31) - 1, -(1 << 31), -7):
        off = (Fraction(turns * p, 1 << 64) - Fraction(f) * p / TWO_PI) % 1
        assert min(off, 1 - off) < Fraction(1, 1 << 25)


def test_many_at_once():
    rng = np.random.default_rng(0)
    f = rng.uniform(-1, 1, 64) * 10.0 ** rng.uniform(-12, 6, 64)
    assert [int(t) for t in S.sam_rope_turns(f)] == [int(S.sam_rope_turns([x])[0]) for x in f]
