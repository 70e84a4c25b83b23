"""The loss of logits with its gradient through the C ABI against a plain form in 64 bits."""
import math

import pytest
import torch

import paper_2512_20953_amd as P

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


def half_step(t):
    return torch.finfo(t).eps / 2


def randn(seed, *shape, dtype=F32, std=1.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype).cuda()


def targets_of(seed, T, V, bits=64, none=0):
    g = torch.Generator().manual_seed(seed)
    t = torch.randint(0, V, (T,), generator=g)
    if none:
        t[torch.rand(T, generator=g) < 1 / none] = -1
    return t.to(torch.int32 if bits == 32 else torch.int64).cuda()


def check(z, target, loss, grad, scale):
    T, V = z.shape
    if T == 0:
        return
    zd, live, at = z.double(), target >= 0, target.long().clamp_min(0)[:, None]
    top = zd.amax(1, keepdim=True)
    far = top - zd                                    # an exponent's argument is off by 3 U times that, exp2 by 2 U more; -infinity gives 0 exactly
    e = (-far).exp()
    S = e.sum(1, keepdim=True)
    rel = torch.where(e > 0, 3 * U * torch.where(far.isfinite(), far, 0.0) + 4 * U, 0.0)
    rel_s = (e * rel).sum(1, keepdim=True) / S * 2 + (V / 1024 + 200) * U       # (twice: a wave's sum is brought to the block's maximum by one more exponential)
    want = (top + S.log() - zd.gather(1, at))[:, 0]
    room = rel_s[:, 0] + 4 * U * ((top - zd.gather(1, at))[:, 0].abs() + S.log()[:, 0].abs() + 1)
    assert (loss.double()[~live] == 0).all()
    assert ((loss.double() - want).abs()[live] <= room[live]).all()
    if grad is None:
        return
    p = e / S
    hit = torch.zeros_like(p).scatter_(1, at, 1.0)
    g = torch.where(live[:, None], (p - hit) * scale, 0.0)
    tiny = torch.finfo(grad.dtype).smallest_normal * half_step(grad.dtype) * 2 + 2.0 ** -126      # (the hardware's exp2 flushes below 2^-126)
    room = abs(scale) * (p * (rel + rel_s + 4 * U) + hit * 2 * U) + g.abs() * half_step(grad.dtype) * (1 + 2 ** -8) + tiny
    assert ((grad.double() - g).abs() <= room).all()


SHAPES = [(1, 1), (3, 2), (5, 7), (4, 64), (9, 512), (7, 1000), (40, 4001), (3, 4104), (5, 8192), (6, 16379), (3, 32000), (4, 50257), (2, 65528), (2, 65537), (2, 131071), (1, 131088), (2, 200003), (300, 96), (0, 9)]


@pytest.mark.parametrize("kind,bits", [(BF, 64), (F32, 32)])
@pytest.mark.parametrize("T,V", SHAPES)
def test_loss_and_gradient(T, V, kind, bits):
    z, t = randn(T + V, T, V, dtype=kind, std=3.0), targets_of(V, T, V, bits, none=4 if T > 4 else 0)
    loss, g = torch.full((T,), 7.0, device="cuda"), torch.full_like(z, 7.0)
    scale = 1 / max(T, 1)
    P.cross_entropy(z, t, loss, g, scale=scale)
    check(z, t, loss, g, scale)
    alone = torch.empty_like(loss)
    P.cross_entropy(z, t, alone)
    assert torch.equal(alone, loss)
    own = z.clone()
    P.cross_entropy(own, t, alone, own, scale=torch.tensor([scale], device="cuda"))
    assert torch.equal(own, g) and torch.equal(alone, loss)


@pytest.mark.parametrize("V", [50, 777, 5001, 40000])
@pytest.mark.parametrize("shift", [0, 1, 3, 7])
def test_rows_that_begin_anywhere(V, shift):
    T = 6
    for ld_z, ld_g, other in ((V + 9, V + 9, shift), (V + 9, V + 5, 0), (V, V + 8, 2)):
        zw, gw = torch.full((T * ld_z + 16,), 9.0, dtype=BF, device="cuda"), torch.full((T * ld_g + 16,), 7.0, dtype=BF, device="cuda")
        z, g = zw[shift:shift + T * ld_z].view(T, ld_z)[:, :V], gw[other:other + T * ld_g].view(T, ld_g)[:, :V]
        z.copy_(randn(V + shift, T, V, std=2.0))
        t, loss = targets_of(3, T, V), torch.empty(T, device="cuda")
        t[0], t[1] = 0, V - 1
        P.cross_entropy(z, t, loss, g, scale=0.25)
        check(z, t, loss, g, 0.25)
        left = gw.clone()
        left[other:other + T * ld_g].view(T, ld_g)[:, :V] = 7.0
        assert (left == 7).all()                       # nothing beside the rows
        if ld_z == ld_g and other == shift:
            want, before = g.clone(), zw.clone()
            P.cross_entropy(z, t, loss, z, scale=0.25)
            assert torch.equal(z, want)
            before[shift:shift + T * ld_z].view(T, ld_z)[:, :V] = want
            assert torch.equal(zw, before)


@pytest.mark.parametrize("kind", [BF, F32])
@pytest.mark.parametrize("V", [5, 300, 3000, 20000, 140000])
def test_masked_logits(V, kind):
    T = 8
    z, t = randn(V, T, V, dtype=kind), torch.zeros(T, dtype=torch.int64, device="cuda")
    low, inf = torch.finfo(kind).min, float("inf")
    z[0, 1:] = -inf                                    # the target alone: loss 0
    z[1, 1:] = low
    z[2] = low                                         # every logit the lowest: all alike
    z[3, 2:] = -inf
    z[4, 0] = -inf                                     # the target cannot be: an infinite loss, finite gradients
    z[5] = -inf                                        # nothing can be
    z[6, V - 1] = inf
    z[7, V // 2] = float("nan")
    loss, g = torch.empty(T, device="cuda"), torch.empty_like(z)
    P.cross_entropy(z, t, loss, g)
    assert loss[0] == loss[1] == 0 and (g[:2] == 0).all()
    assert math.isclose(loss[2].item(), math.log(V), rel_tol=(V / 1024 + 210) * U) and ((g[2, 1:].double() * V - 1).abs() <= half_step(kind) + (V / 1024 + 210) * U).all()
    check(z[3:4], t[3:4], loss[3:4], g[3:4], 1.0)
    assert loss[4] == inf and g[4].isfinite().all() and g[4, 0] == -1
    check(z[4:5], torch.ones_like(t[:1]), *one_more(z[4:5], torch.ones_like(t[:1])), 1.0)
    assert loss[5:].isnan().all() and g[5].isnan().all() and g[6].isnan().all() and g[7].isnan().all()


def one_more(z, t):
    loss, g = torch.empty(z.shape[0], device="cuda"), torch.empty_like(z)
    P.cross_entropy(z, t, loss, g)
    return loss, g


def test_targets_that_are_none():
    T, V = 9, 1003
    z, t = randn(1, T, V, dtype=BF), targets_of(2, T, V)
    t[1], t[3], t[5], t[7] = -1, -2, V, 2 ** 32 + 3
    loss, g = one_more(z, t)
    assert loss[1] == 0 and (g[1] == 0).all()
    assert loss[[3, 5, 7]].isnan().all() and g[[3, 5, 7]].isnan().all()
    keep = [0, 2, 4, 6, 8]
    check(z[keep], t[keep], loss[keep], g[keep], 1.0)
    z[1] = float("nan")
    loss, g = one_more(z, t)
    assert loss[1] == 0 and (g[1] == 0).all()          # a row without a target is not looked at


def test_rows_far_into_large_logits():
    """Elements behind the 2^31st, in place"""
    T, V = 45000, 50257
    z = torch.zeros(T, V, dtype=BF, device="cuda")
    far = [0, 42731, T - 1]
    z[far] = randn(1, 3, V, dtype=BF, std=2.0)
    keep, t = z[far].clone(), targets_of(2, T, V)
    loss = torch.empty(T, device="cuda")
    P.cross_entropy(z, t, loss, z)
    check(keep, t[far], loss[far], z[far], 1.0)


def test_captured_with_a_scale_on_the_device():
    T, V = 70, 9001
    z, t, scale = randn(1, T, V, dtype=BF), targets_of(2, T, V, none=5), torch.tensor([0.5], device="cuda")
    loss, g = torch.empty(T, device="cuda"), torch.empty_like(z)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        P.cross_entropy(z, t, loss, g, scale=scale, stream=s)
    for rep in range(3):
        scale.fill_(1.0 / (rep + 1))
        g.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        check(z, t, loss, g, 1.0 / (rep + 1))
        z.add_(0.25)                                   # (a shift of all logits changes neither but for their rounding)


def test_gradient_against_differences():
    T, V, h = 3, 11, 1 / 32
    z, t = randn(1, T, V), targets_of(2, T, V)
    _, g = one_more(z, t)
    for c in range(V):
        e = torch.zeros(V, device="cuda")
        e[c] = h
        num = (one_more(z + e, t)[0].double() - one_more(z - e, t)[0].double()) / (2 * h)
        # the loss is off by about 210 U + 8 U on either side; its third derivative by a logit is at most 1/4
        assert ((num - g[:, c].double()).abs() <= 2 * 260 * U / (2 * h) + h * h / 24 + 220 * U).all()
