"""Muon's update of matrices that one direction makes up, with the first two steps at once, against the formula in 64 bits."""
import math

import pytest
import torch

from tests.test_gpu_muon import norm, orthogonal, randn, update_of

pytestmark = pytest.mark.gpu
H = 2.0 ** -11                                       # half a step of fp16


@pytest.mark.parametrize("shapes", [[(700, 2500)] * 12, [(2500, 700)] * 12, [(1500, 9000)] * 2 + [(1500, 5000)], [(2048, 8000)]])
def test_one_direction(shapes):
    """X = s u v^T: a matrix M = m u u^T whose elements are rounded, each by at most H, leaves |E u| <= m H sqrt(sum u_j^4 / 3) = m H / sqrt(n) in the direction that it moves u to (u of normal elements,
    roundings uniform within half a step).  Over s = 1.11 behind two steps, the weights m are 10.8 for Q, and for what comes before it, carried through the derivatives, 7.6 (A), 4.4 (B), 4.7 (C),
    1.6 (A of the second step), 1.3 (B1); for X's own operand 10.8 sqrt(n / k).  Their root of squares is 16 to 18; three steps apart add about 10.  In all 20 H / sqrt(n), and 40 is allowed.  (A
    rounding of B A that is added as 2 a B A has a weight of 53 by itself: 2.74 * 2 a * 2.8.)"""
    gs = [randn(3 * k, r, 1) @ randn(3 * k + 1, 1, c) for k, (r, c) in enumerate(shapes)]
    xs, opt = update_of(gs)
    assert opt._work.numel() > sum(6 * g.numel() for g in gs) + 8 * sum(min(s) ** 2 for s in shapes)          # (two steps at once: the two square matrices more)
    for k in {0, len(gs) - 1}:
        want, _ = orthogonal(gs[k] * 0.05 * 1.95)
        off = norm(xs[k].double() - want) / norm(want)
        print(shapes[k], "off by %.2g, allowed %.2g" % (off, 40 * H / math.sqrt(min(shapes[k]))))
        assert off <= 40 * H / math.sqrt(min(shapes[k]))
