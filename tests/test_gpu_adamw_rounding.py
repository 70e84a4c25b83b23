"""The random rounding of 8-bit states over many steps: by other bits in every step, eager with default arguments and replayed.

Rounded by independent bits, a stored moment keeps the expectation of its recursion.  For a gradient that stays the same the deviation of one element settles at the variance of
a step's rounding, at most a quarter of the distance of two codes squared, over 1 - beta^2.  That distance is at most an eighth of the value's binade; a value near x stays below 2 x, so
x / 4 is taken: a standard deviation of x / 8 / sqrt(1 - beta^2), 0.29 x for beta = 0.9 and 0.40 x for 0.95.  The mean over N elements is asked for within 6 times that over sqrt N."""
import math

import pytest
import torch

import paper_2512_20953_amd as P

pytestmark = pytest.mark.gpu
DEV = "cuda"
B1, B2, G, N, STEPS = 0.9, 0.95, 0.37, 32 * 1024, 200


def _from_far():
    """An optimizer whose moments come from a gradient twice as large: m = 2 G, v = 4 G^2 as they are stored."""
    grads = [torch.full((N,), 2 * G, device=DEV)]
    first = P.AdamW([torch.zeros(N, device=DEV)], grads, betas=(0.0, 0.0), state_bits=8)
    first.step(0.0, 1)
    return P.AdamW([torch.zeros(N, device=DEV)], [torch.full((N,), G, device=DEV)], betas=(B1, B2), state_bits=8,
                   **{k: getattr(first, k) for k in ("m", "v", "m_scale", "v_scale")})


def _values(opt):
    out = [[torch.empty(t.numel(), dtype=torch.bfloat16, device=DEV) for t in opt.params] for _ in range(2)]
    opt.state_values(*out)
    return [[t.double().cpu() for t in o] for o in out]


def _state(opt):
    return [t.clone() for k in ("m", "v", "m_scale", "v_scale") for t in getattr(opt, k)]


def _check_means(opt):
    (m,), (v,) = _values(opt)
    for got, far, want, beta in ((m, 2 * G, G, B1), (v, 4 * G * G, G * G, B2)):
        mean = want + (far - want) * beta ** STEPS
        assert abs(got.mean().item() - mean) <= 6 * want / 8 / math.sqrt((1 - beta * beta) * N) + 2 ** -3 * far * beta ** STEPS, (got.mean().item(), mean)


def test_moments_reach_their_mean_eager_and_replayed():
    eager, opt = _from_far(), _from_far()
    for a, b in zip(_state(eager), _state(opt)):
        assert torch.equal(a, b)
    lr, count = torch.zeros(1, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            opt.step(lr, count)
        for step in range(1, STEPS + 1):
            count.fill_(step)
            g.replay()
            eager.step(0.0, step)
            if step % 50 == 1:
                torch.cuda.synchronize()
                assert all(torch.equal(a, b) for a, b in zip(_state(opt), _state(eager))), step     # a number from the device is that from the host
    torch.cuda.synchronize()
    _check_means(eager)
    _check_means(opt)
    del g


def test_steps_from_one_state_round_differently():
    base = _from_far()
    count = torch.zeros(1, dtype=torch.int32, device=DEV)

    def after(step, **kw):
        state = {k: [t.clone() for t in getattr(base, k)] for k in ("m", "v", "m_scale", "v_scale")}
        opt = P.AdamW([torch.zeros(N, device=DEV)], base.grads, betas=(B1, B2), state_bits=8, **state)
        opt.step(0.0, count.fill_(step) if kw.pop("device", False) else step, **kw)
        return _state(opt)

    same = lambda a, b: all(torch.equal(x, y) for x, y in zip(a, b))   # noqa: E731
    assert same(after(5), after(5)) and same(after(5), after(5, device=True))
    for kw in ({}, dict(device=True), dict(device=True, seed=3)):
        a, b = after(5, **kw), after(6, **kw)
        assert not torch.equal(a[0], b[0]) and not torch.equal(a[1], b[1])
    assert same(after(5, seed=3, device=True), after(2, seed=8)) and same(after(2, seed=8), after(900, seed=8))   # a number beside a number stands alone
    assert same(after(7, seed=-2, device=True), after(1, seed=5)) and same(after(7, seed=2 ** 32 - 2, device=True), after(1, seed=5))


def test_a_capture_that_would_repeat_its_bits_is_refused():
    b8, b32 = (P.AdamW([torch.zeros(64, device=DEV)], [torch.ones(64, device=DEV)], state_bits=n) for n in (8, 32))
    lr, count = torch.zeros(1, device=DEV), torch.ones(1, dtype=torch.int32, device=DEV)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            for a in ((1e-3, 1), (lr, 1)):
                with pytest.raises(P.AhError, match="step_dev"):
                    b8.step(*a, seed=4)
                b32.step(*a)
            b8.step(lr, count)
        g.replay()
    torch.cuda.synchronize()
    assert not (b8.m[0] == 0).any() and not (b32.m[0] == 0).any()
    b8.step(1e-3, 1)                                        # not captured: any number will do
    torch.cuda.synchronize()
    del g
