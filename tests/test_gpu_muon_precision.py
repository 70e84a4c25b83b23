"""How far Muon's updates may be from the formula in 64 bits, in absolute terms: whatever the kernel's own roundings are."""
import pytest
import torch

import paper_2512_20953_amd as P
from tests.test_gpu_muon import F32, low_rank, norm, orthogonal, randn, update_of

pytestmark = pytest.mark.gpu
H = 2.0 ** -11                                       # half a step of fp16


def off(x, want):
    return norm(x.double() - want) / norm(want)


@pytest.mark.parametrize("make", [randn, low_rank])
@pytest.mark.parametrize("r,c", [(17, 3000), (24, 100), (64, 64), (100, 37), (128, 128), (130, 2049), (2049, 130), (256, 256), (200, 520), (250, 8000)])
def test_operands_in_22_bits(make, r, c):
    """Of a step A, B and X are rounded to 22 bits, by at most 2^-22 of an element (2^-22 / sqrt 3 in root of squares, 2^-22 the three together), and sums of up to 2049 products are fp32, 32 of them
    exact, 2^-24 sqrt(64) = 2^-21: 2.2 of 2^-22.  Four more steps carry that on by up to 140 along the smallest singular values, while X's norm grows from 1 to 0.7 sqrt(n) or more, 5.6 for n = 64:
    2.2 * 2^-22 * 140 / 5.6 = 1.3e-5, of later steps a tenth of it more: 2^-16.  (Of fewer rows the singular values begin larger and are carried on less.)  Without any one of the six products of an
    upper by a lower half the random ones are 4e-5 to 2e-3 off."""
    g = randn(r + c, r, c) if make is randn else low_rank(r + c, r, c)
    (x,), _ = update_of([g])
    want, _ = orthogonal(g * 0.05 * 1.95)
    print("%d x %d %s: off by %.2g" % (r, c, make.__name__, off(x, want)))
    assert off(x, want) <= 2.0 ** -16


# At the singular values that the last steps leave, 0.7 to 1.2, an element's part B X has the weight 2.74, and with it the roundings of B and of X's operand; A's is carried on with
# 4.78 - 4.06 s^2 = 2.8 at most, X's operand in A with twice half of that: sqrt(2 * 2.74^2 + 2 * 2.8^2) = 5.5 roundings of H / sqrt(3) over a value of 0.7 or more, 4.5 H, in every element at
# its largest; the steps before are carried on by slopes below 1 there and are of roundings of numbers between powers of two, 0.72 of the largest: 5 H in all.  Where eight directions make a matrix up the
# others grow to that size in the last two steps only; eight of 64 or more directions are sqrt(1 / 8) of the norm: 2 H.
RANDOM, FEW = 5 * H, 2 * H


@pytest.mark.parametrize("shapes", [[(64, 64)], [(257, 300)], [(300, 1000), (1000, 300)], [(512, 512)], [(700, 2500)] * 12, [(1500, 1500)], [(2500, 4300)], [(512, 1000)] * 24, [(2048, 8000)]])
@pytest.mark.parametrize("make,room", [(randn, RANDOM), (low_rank, FEW)])
def test_operands_in_11_bits(make, room, shapes):
    """bf16 gradients and parameters with a copy in fp32 for the larger ones; the smallest in bf16, for which half a step of 2^-8 of each element is left."""
    gs = [make(3 * k, r, c) for k, (r, c) in enumerate(shapes)]
    if min(shapes[0]) <= 256:
        ps = [torch.zeros(g.shape, dtype=torch.bfloat16, device="cuda") for g in gs]
        P.Muon(ps, gs, scale=1.0).step(1.0)
        xs, room = [-p.double() for p in ps], room + 2.0 ** -8
    else:
        xs, _ = update_of(gs)
    for k in {0, len(gs) // 2, len(gs) - 1}:
        want, _ = orthogonal(gs[k] * 0.05 * 1.95)
        print(shapes[k], make.__name__, "off by %.2g, allowed %.2g" % (off(xs[k], want), room))
        assert off(xs[k], want) <= room


def test_large_matrices_that_are_not_worked_on_together():
    """2^26 elements each, four to a group: every one against the formula, as a whole and in tiles of 256 x 256 (a wrong tile is off by its own norm)"""
    n = 8192
    gs = [randn(k, n, n) for k in range(2)]
    wants = []
    for g in gs:
        x = (g * (0.05 * 1.95)).double()
        x /= norm(x) + 1e-7
        for _ in range(5):
            a = x @ x.T.contiguous()
            b = torch.addmm(a, a, a, beta=-4.7750, alpha=2.0315)
            x = torch.addmm(x, b, x, beta=3.4445)
            del a, b
        wants.append(x)
    order = [0, 1, 1, 0, 0]
    ps = [torch.zeros(n, n, dtype=F32, device="cuda") for _ in order]
    P.Muon(ps, [gs[k] for k in order], scale=1.0).step(1.0)
    tiles = lambda t: t.view(n // 256, 256, n // 256, 256).square().sum(dim=(1, 3)).sqrt()      # noqa: E731
    for p, k in zip(ps, order):
        d = p.double().neg_().sub_(wants[k])
        print("off by %.2g, the worst tile by %.2g" % (norm(d) / norm(wants[k]), (tiles(d) / tiles(wants[k])).max().item()))
        assert norm(d) <= RANDOM * norm(wants[k])
        assert (tiles(d) <= 2 * RANDOM * tiles(wants[k])).all()


def test_what_shares_a_call_changes_roundings_alone():
    """Alone, beside a large matrix and beside many: other tiles, the first two steps at once or not.  Each form is within its room, so that two are within the sum of both."""
    g = randn(1, 700, 2500)
    want, _ = orthogonal(g * 0.05 * 1.95)
    for others in ([], [(2048, 8000)], [(700, 2500)] * 11, [(300, 310)] * 3):
        xs, _ = update_of([g] + [randn(5 + k, *s) for k, s in enumerate(others)])
        again, _ = update_of([g] + [randn(55 + k, *s) for k, s in enumerate(others)])
        assert off(xs[0], want) <= RANDOM
        assert torch.equal(xs[0], again[0])          # whatever the others hold
