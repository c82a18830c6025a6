"""A scale that is no number is refused: no weights follow from it."""
from __future__ import annotations

import ctypes as C

import pytest

import paper_2512_18337_b200 as S
from tests.test_cache_host import _struct


@pytest.mark.parametrize("scale", [float("nan"), float("inf"), float("-inf")])
def test_scales_that_are_not_finite_are_refused(scale):
    lib = S.binding._load()
    c = C.addressof(s := _struct())
    for B, Q in ((1, 1), (1, 64), (0, 1)):
        assert lib.sam_cache_attend(c, 0, 16, 0, 0, 0, 0, B, Q, 4, None, None, scale, 0, 16, 0, 0, 0, None, 256, 1 << 40, None) == -1
    del s
