"""High frequencies at far positions: angles taken exactly, in fractions, as the reference."""
from __future__ import annotations

from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2512_18337_b200 as S
from tests.test_gpu_cache_attend import DEV, _i32
from tests.test_gpu_rotated import ROTATION, _check_queries, _empty_cache
from tests.test_step_host import TWO_PI

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("f", [1e3, 54321.0625, 999_983.7, -777_777.7, 1e6])
def test_far_positions_of_high_frequencies(f):
    positions = [0, 1, 250_000, (1 << 30) - 1, (1 << 31) - 1, -1, -(1 << 31)]
    Q = len(positions)
    c, _ = _empty_cache([0], Q, 16, 1, 64)
    rope = S.SamRope(np.full(16, f), device=DEV)
    rng = np.random.default_rng(0)
    q = torch.from_numpy(rng.standard_normal((1, Q, 3, 64))).to(DEV, torch.float16)
    k = torch.zeros(1, Q, 1, 64, dtype=torch.float16, device=DEV)
    got = c.append_rotated(0, q, k, k, rope, positions=_i32([positions]))
    # the angle modulo a turn, exactly; as a float64 it is off by 2^-52 of itself
    angle = np.array([float((Fraction(f) * p / TWO_PI) % 1 * TWO_PI) for p in positions])[:, None, None]
    x = q[0].double().cpu().numpy()
    a, b = x[..., :16], x[..., 16:32]
    y, size = x.copy(), np.zeros_like(x)
    y[..., :16], y[..., 16:32] = a * np.cos(angle) - b * np.sin(angle), b * np.cos(angle) + a * np.sin(angle)
    size[..., :16] = size[..., 16:32] = np.abs(a) + np.abs(b)
    # turns are off by half of 2^-64 each position, 2^-34 of a turn after 2^31, and 2^-32 of a turn is cut off
    _check_queries(got[0], y, size * (1 + 2 * np.pi * 2.0 ** -31 / ROTATION), "fp16")
