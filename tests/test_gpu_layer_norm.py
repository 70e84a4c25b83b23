"""Layer norm, forward and backward, through the C ABI against plain forms in 64 bits."""
import pytest
import torch

import paper_2512_20953_amd as P

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32
DEPTH = 48           # roundings of a sum over a row: up to 16 elements a lane, 6 steps of a wave, 16 waves
EPS = 1e-5


def half_step(t):
    return torch.finfo(t).eps / 2


def randn(seed, *shape, dtype=F32, std=1.0, mean=0.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * std + mean).to(dtype).cuda()


def padded(t, ld):
    wide = torch.full((t.shape[0], ld), 7.0, dtype=t.dtype, device=t.device)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def mean_abs(t):
    return t.abs().mean(1, keepdim=True)


class Plain:
    """Statistics in 64 bits, and how far fp32 may be off them"""

    def __init__(self, x, rms, eps=EPS):
        self.x = x.double()
        m = torch.zeros_like(self.x[:, :1]) if rms else self.x.mean(1, keepdim=True)
        self.d = self.x - m
        self.r = (self.d.square().mean(1, keepdim=True) + eps).rsqrt()
        self.e_mean = torch.zeros_like(m) if rms else (DEPTH + 2) * U * mean_abs(self.x)
        # the mean square is off by 2 |d| e_mean and its roundings, r by half of that relative to it
        self.rel_r = self.e_mean * mean_abs(self.d) * self.r.square() + self.e_mean.square() * self.r.square() + (DEPTH / 2 + 8) * U
        self.e_d = self.e_mean + U * self.d.abs()


SHAPES = [(1, 1), (3, 2), (5, 7), (2, 64), (9, 512), (7, 520), (6, 1000), (33, 1001), (4, 1024), (5, 2048), (3, 2500), (17, 4096), (2, 4100), (3, 8192), (2, 16384), (2, 16383), (1500, 128), (0, 40)]


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("kind,param", [(BF, BF), (F32, F32), (BF, F32)])
@pytest.mark.parametrize("T,w", SHAPES)
def test_forward(T, w, kind, param, rms):
    x = padded(randn(w + T, T, w, dtype=kind, std=2.0, mean=0.7), w + (8 if w % 16 == 0 else 3))
    gain, bias = randn(1, w, dtype=param, mean=1.0, std=0.3), randn(2, w, dtype=param)
    for g, b in ((gain, bias), (None, None), (gain, None)):
        y = padded(torch.zeros(T, w, dtype=kind, device="cuda"), w + (8 if w % 16 == 0 else 3))
        P.layer_norm_fwd(x, g, b, y, eps=EPS, rms=rms)
        q = Plain(x, rms)
        gd, bd = (torch.ones(w, device="cuda") if g is None else g).double(), (torch.zeros(w, device="cuda") if b is None else b).double()
        n = q.d * q.r * gd
        want = n + bd
        room = gd.abs() * q.r * (q.e_d + q.d.abs() * q.rel_r) + 3 * U * (n.abs() + want.abs()) + half_step(kind) * want.abs()
        assert ((y.double() - want).abs() <= room * 1.01 + 1e-38).all()


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("kind,param", [(BF, BF), (F32, F32), (F32, BF)])
@pytest.mark.parametrize("T,w", SHAPES)
def test_backward(T, w, kind, param, rms):
    ld = w + (8 if w % 16 == 0 else 3)
    x, dy = padded(randn(w + T, T, w, dtype=kind, std=2.0, mean=0.7), ld), padded(randn(w + T + 1, T, w, dtype=kind), ld)
    gain = randn(1, w, dtype=param, mean=1.0, std=0.3)
    for g, beta in ((gain, 0), (gain, 1), (None, 0)):
        dx = padded(torch.zeros(T, w, dtype=kind, device="cuda"), ld)
        dg, db = randn(3, w), randn(4, w)
        old_g, old_b = (dg.double(), db.double()) if beta else (0.0, 0.0)
        if not beta:
            dg.fill_(float("nan"))
            db.fill_(float("nan"))
        work = torch.full((P.layer_norm_bwd_workspace(T, w),), 255, dtype=torch.uint8, device="cuda")
        P.layer_norm_bwd(x, g, dy, dx, dg, db, work, eps=EPS, rms=rms, beta=beta)
        q = Plain(x, rms)
        gd, yd = (torch.ones(w, device="cuda") if g is None else g).double(), dy.double()
        v = yd * gd
        mv = torch.zeros_like(q.r) if rms else v.mean(1, keepdim=True)
        along = (q.d * v).mean(1, keepdim=True)
        k = along * q.r.square()
        want = q.r * (v - mv - q.d * k)
        e_along = q.e_mean * mean_abs(v) + (DEPTH + 4) * U * mean_abs(q.d * v)
        e_k = q.r.square() * (e_along + along.abs() * (2 * q.rel_r + 4 * U))
        e_inner = 2 * U * v.abs() + (DEPTH + 3) * U * mean_abs(v) * (not rms) + q.d.abs() * e_k + k.abs() * q.e_d + 4 * U * (v.abs() + mv.abs() + (q.d * k).abs())
        room = q.r * e_inner + want.abs() * (q.rel_r + 2 * U) + half_step(kind) * want.abs()
        assert ((dx.double() - want).abs() <= room * 1.01 + 1e-38).all()
        n = q.d * q.r
        e_n = q.r * q.e_d + n.abs() * (q.rel_r + 2 * U)
        room_g = ((yd.abs() * e_n).sum(0) + (T + 4) * U * (yd * n).abs().sum(0)) * 1.01 + 2 * U * (old_g.abs() if beta else 0.0)
        assert ((dg.double() - (yd * n).sum(0) - old_g).abs() <= room_g + 1e-38).all()
        room_b = (T + 4) * U * yd.abs().sum(0) + 2 * U * (old_b.abs() if beta else 0.0)
        assert ((db.double() - yd.sum(0) - old_b).abs() <= room_b + 1e-38).all()


def test_in_place_and_without_a_gradient():
    T, w = 700, 264
    x, dy, gain, bias = randn(1, T, w, dtype=BF), randn(2, T, w, dtype=BF), randn(3, w, dtype=BF), randn(4, w, dtype=BF)
    y, dx, dg, db = torch.empty_like(x), torch.empty_like(x), torch.empty(w, device="cuda"), torch.empty(w, device="cuda")
    work = torch.empty(P.layer_norm_bwd_workspace(T, w), dtype=torch.uint8, device="cuda")
    P.layer_norm_fwd(x, gain, bias, y)
    P.layer_norm_bwd(x, gain, dy, dx, dg, db, work)
    z = x.clone()
    P.layer_norm_fwd(z, gain, bias, z)
    assert torch.equal(z, y)
    for other in (x.clone(), dy.clone()):
        a, b = (other, dy) if torch.equal(other, x) else (x, other)
        g2 = torch.empty_like(dg)
        P.layer_norm_bwd(a, gain, b, other, g2, None, work)
        assert torch.equal(other, dx) and torch.equal(g2, dg)
    b2, z = torch.empty_like(db), torch.empty_like(dx)
    P.layer_norm_bwd(x, gain, dy, z, None, b2, work)
    assert torch.equal(z, dx) and torch.equal(b2, db)
    P.layer_norm_bwd(x, gain, dy, z, None, None, work)


@pytest.mark.parametrize("w", [256, 1001, 4096, 8200])
def test_rows_do_not_reach_each_other_and_captured(w):
    T = 1300
    x, dy, gain = randn(1, T, w, dtype=BF), randn(2, T, w, dtype=BF), randn(3, w, dtype=BF)
    y0, dx0 = torch.empty_like(x), torch.empty_like(x)
    dg, db = torch.empty(w, device="cuda"), torch.empty(w, device="cuda")
    work = torch.empty(P.layer_norm_bwd_workspace(T, w), dtype=torch.uint8, device="cuda")
    P.layer_norm_fwd(x, gain, None, y0)
    P.layer_norm_bwd(x, gain, dy, dx0, dg, db, work)
    want = dg.clone(), db.clone()
    bad = x.clone()
    bad[[0, 77, T - 1], 5] = float("nan")
    bad[500] = float("inf")
    y, dx = torch.empty_like(x), torch.empty_like(x)
    P.layer_norm_fwd(bad, gain, None, y)
    P.layer_norm_bwd(bad, gain, dy, dx, dg, db, work)
    rows = torch.ones(T, dtype=torch.bool, device="cuda")
    rows[[0, 77, T - 1, 500]] = False
    assert torch.equal(y[rows], y0[rows]) and torch.equal(dx[rows], dx0[rows])
    assert y[~rows].isnan().any(1).all() and dx[~rows].isnan().any(1).all() and dg.isnan().any()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        P.layer_norm_fwd(x, gain, None, y, stream=s)
        P.layer_norm_bwd(x, gain, dy, dx, dg, db, work, stream=s)
    for rep in range(3):
        y.zero_(), dx.zero_(), dg.zero_(), db.zero_()
        work.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, y0) and torch.equal(dx, dx0) and torch.equal(dg, want[0]) and torch.equal(db, want[1]), rep


def test_large_means_and_constant_rows():
    """A row far from zero keeps its variance (squares are taken around the mean); one whose elements are all alike comes out as its bias."""
    w = 1024
    x = (randn(1, 8, w) + 1000.0)
    y = torch.empty_like(x)
    P.layer_norm_fwd(x, None, None, y)
    q = Plain(x, False)
    assert ((y.double() - q.d * q.r).abs() <= 1.01 * (q.r * (q.e_d + q.d.abs() * q.rel_r)) + 4 * U * (q.d * q.r).abs()).all()
    x.fill_(-3.5)
    b = randn(2, w)
    P.layer_norm_fwd(x, None, b, y)
    assert torch.equal(y, b.expand_as(y))


def test_gradient_against_differences():
    """Central differences of sum(y dy) over a step h in x, gain and bias: the error of y (about 16 U |y|) over h, and h^2 / 6 times the third derivative (of n by x: at most 15 r^3 a term)."""
    T, w, h, eps = 4, 9, 1 / 32, 0.1
    x, dy, gain, bias = randn(1, T, w), randn(2, T, w), randn(3, w, mean=1.0, std=0.3), randn(4, w)
    for rms in (False, True):
        dx, dg, db = torch.empty_like(x), torch.empty(w, device="cuda"), torch.empty(w, device="cuda")
        P.layer_norm_bwd(x, gain, dy, dx, dg, db, torch.empty(P.layer_norm_bwd_workspace(T, w), dtype=torch.uint8, device="cuda"), eps=eps, rms=rms)

        def f(a, g, b):
            y = torch.empty_like(a)
            P.layer_norm_fwd(a, g, b, y, eps=eps, rms=rms)
            return (y.double() * dy.double()).sum(1)
        r3 = Plain(x, rms, eps).r.max().item() ** 3
        size = (dy.double().abs() * gain.double().abs()).sum(1).max().item()
        for c in range(w):
            e = torch.zeros(w, device="cuda")
            e[c] = h
            room = size * 15 * r3 * h * h / 6 + 64 * U * (size * 4 + dy.abs().sum(1).max().item() * 4) / h
            for got, num in ((dx[:, c], f(x + e, gain, bias) - f(x - e, gain, bias)), (dg[c], (f(x, gain + e, bias) - f(x, gain - e, bias)).sum()),
                             (db[c], (f(x, gain, bias + e) - f(x, gain, bias - e)).sum())):
                assert ((got.double() - num / (2 * h)).abs() <= room * T).all()
