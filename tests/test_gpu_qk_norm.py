"""Norms of the query and key heads with the rotation against their definition in 64 bits, element by element.

Tolerances.  The result is rounded to bf16 once (2^-8 of itself); what comes before is fp32: products and sums of two terms, a mean over a head, a
reciprocal root, below 1e-6 of the terms' magnitudes together; 1e-5 of those.  The gains' gradients are fp32 sums: 1e-5 of the sum of magnitudes."""
import pytest
import torch

import paper_2512_20953_amd as P

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _case(T, nh, nkv, d, seed, pad=8, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    w = (nh + nkv) * d
    x = (scale * torch.randn(T, w + pad, generator=g)).bfloat16().to(DEV)[:, :w]
    dy = torch.randn(T, w + 2 * pad, generator=g).bfloat16().to(DEV)[:, pad:pad + w]
    gains = [(1 + 0.3 * torch.randn(d, generator=g)).bfloat16().to(DEV) for _ in range(2)]
    return x, dy, gains


def _table(n, d, base=10000.0):
    t = torch.empty(n, d // 2, 2, device=DEV)
    P.rope_table(t, d, base)
    return t


def _reference(x, dy, gains, table, pos, nh, nkv, d, eps):
    """y, dx and the gains' gradients with the magnitudes that their fp32 errors go by."""
    T, h, n = x.shape[0], d // 2, nh + nkv
    gain = torch.cat([gains[0].double().expand(nh, d), gains[1].double().expand(nkv, d)])
    X, DY = x.double().reshape(T, n, d), dy.double().reshape(T, n, d)
    cos = sin = None
    if table is not None:
        cos, sin = table.double()[pos][:, None, :, 0], table.double()[pos][:, None, :, 1]
    turn = lambda a, s: a if table is None else torch.cat([a[..., :h] * cos - s * a[..., h:] * sin, a[..., h:] * cos + s * a[..., :h] * sin], -1)  # noqa: E731
    r = 1 / torch.sqrt((X * X).mean(-1, keepdim=True) + eps)
    norm = X * r * gain
    both = norm.abs() + torch.cat([norm[..., h:], norm[..., :h]], -1).abs()
    dn = turn(DY, -1)
    xr, w = X * r, dn * gain
    dx = r * (w - xr * (w * xr).mean(-1, keepdim=True))
    dn_size = DY.abs() + torch.cat([DY[..., h:], DY[..., :h]], -1).abs()
    size = r * (dn_size * gain.abs() + xr.abs() * (dn_size * gain.abs() * xr.abs()).mean(-1, keepdim=True))
    dg, dg_size = (dn * xr).sum(0), (dn_size * xr.abs()).sum(0)
    flat = lambda t: t.reshape(T, -1)  # noqa: E731
    return (flat(turn(norm, 1)), flat(both)), (flat(dx), flat(size)), [(dg[a:b].sum(0), dg_size[a:b].sum(0)) for a, b in ((0, nh), (nh, n))]


def _within(got, ref, size, rounded):
    room = (2 ** -8 * ref.abs() if rounded else 0) + 1e-5 * size + 1e-30
    assert ((got.double() - ref).abs() <= room).all(), ((got.double() - ref).abs() / room).max().item()


@pytest.mark.parametrize("T,S,nh,nkv,d", [
    (1, 1, 1, 0, 64), (1, 1, 32, 8, 128), (3, 2, 0, 1, 128), (5, 5, 1, 1, 64), (7, 4, 3, 1, 64), (64, 64, 4, 4, 64), (129, 43, 5, 2, 128), (200, 100, 16, 3, 64),
    (333, 111, 9, 9, 128), (1000, 1000, 2, 1, 64), (5000, 2500, 12, 4, 128)])
@pytest.mark.parametrize("rotate", ["rows", "positions", "not"])
def test_forward_and_backward(T, S, nh, nkv, d, rotate):
    x, dy, gains = _case(T, nh, nkv, d, T + d)
    table = None if rotate == "not" else _table(S + 3, d)
    pos = torch.arange(T, device=DEV) % S
    positions = None
    if rotate == "positions":
        pos = torch.randint(0, S + 3, (T,), generator=torch.Generator().manual_seed(1)).to(DEV)
        positions = pos.int()
    (y, ysize), (dx, dxsize), dg = _reference(x, dy, gains, table, pos, nh, nkv, d, 1e-6)
    w = (nh + nkv) * d
    out = torch.full((T, w + 16), float("nan"), dtype=torch.bfloat16, device=DEV)
    P.qk_norm_rope_fwd(x, *gains, table, out[:, 8:8 + w], S, nh, nkv, d, positions=positions)
    _within(out[:, 8:8 + w], y, ysize, True)
    assert torch.isnan(out[:, :8]).all() and torch.isnan(out[:, 8 + w:]).all()
    out.fill_(float("nan"))
    got = [torch.full((d,), 3.0, device=DEV) for _ in range(2)]
    work = torch.full((P.qk_norm_rope_bwd_workspace(T, nh, nkv, d),), 255, dtype=torch.uint8, device=DEV)
    for beta in (0, 1):
        P.qk_norm_rope_bwd(x, *gains, table, dy, out[:, 8:8 + w], *got, work, S, nh, nkv, d, positions=positions, beta=beta)
    _within(out[:, 8:8 + w], dx, dxsize, True)
    assert torch.isnan(out[:, :8]).all() and torch.isnan(out[:, 8 + w:]).all()
    for g, (ref, size), n in zip(got, dg, (nh, nkv)):
        if n:
            _within(g, 2 * ref, 2 * size, False)
        else:
            assert (g == 3).all()                   # no such heads: left alone


def test_in_place_and_the_same_bits_every_time():
    T, S, nh, nkv, d = 700, 100, 6, 2, 64
    x, dy, gains = _case(T, nh, nkv, d, 5, pad=0)
    table = _table(S, d)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    work = torch.empty(P.qk_norm_rope_bwd_workspace(T, nh, nkv, d), dtype=torch.uint8, device=DEV)
    dg = torch.empty(4, d, device=DEV)
    P.qk_norm_rope_fwd(x, *gains, table, y, S, nh, nkv, d)
    dyc = dy.contiguous()
    P.qk_norm_rope_bwd(x, *gains, table, dyc, dx, dg[0], dg[1], work, S, nh, nkv, d)
    twice = dyc.clone()
    P.qk_norm_rope_bwd(x, *gains, table, twice, twice, dg[2], dg[3], work, S, nh, nkv, d)
    assert torch.equal(twice, dx) and torch.equal(dg[:2], dg[2:])
    over = x.clone()
    P.qk_norm_rope_bwd(over, *gains, table, dyc, over, dg[2], dg[3], work, S, nh, nkv, d)
    assert torch.equal(over, dx)
    z = x.clone()
    P.qk_norm_rope_fwd(z, *gains, table, z, S, nh, nkv, d)
    assert torch.equal(z, y)


def test_no_rows_zero_rows_and_tiny_rows():
    d = 128
    x, dy, gains = _case(4, 2, 1, d, 8)
    work = torch.empty(P.qk_norm_rope_bwd_workspace(4, 2, 1, d), dtype=torch.uint8, device=DEV)
    dg = torch.full((2, d), 5.0, device=DEV)
    P.qk_norm_rope_fwd(x[:0], *gains, None, x[:0], 1, 2, 1, d)
    P.qk_norm_rope_bwd(x[:0], *gains, None, dy[:0], dy[:0], dg[0], dg[1], work, 1, 2, 1, d)
    assert (dg == 0).all()                           # the sum over no rows
    P.qk_norm_rope_bwd(x[:0], *gains, None, dy[:0], dy[:0], dg[0].fill_(5), dg[1].fill_(5), work, 1, 2, 1, d, beta=1)
    assert (dg == 5).all()
    x = torch.zeros(4, 3 * d, dtype=torch.bfloat16, device=DEV)
    x[1] = 1e-12
    x[2] = 1e4
    y, dx = torch.empty_like(x), torch.empty_like(x)
    pos = torch.zeros(4, dtype=torch.long, device=DEV)
    (ry, sy), (rdx, sdx), _ = _reference(x, dy, gains, None, pos, 2, 1, d, 1e-6)
    P.qk_norm_rope_fwd(x, *gains, None, y, 1, 2, 1, d)
    P.qk_norm_rope_bwd(x, *gains, None, dy, dx, dg[0], dg[1], work, 1, 2, 1, d)
    _within(y, ry, sy, True)
    _within(dx, rdx, sdx, True)


def test_positions_outside_the_table_show():
    T, nh, nkv, d = 6, 2, 1, 64
    x, _, gains = _case(T, nh, nkv, d, 2)
    y = torch.empty(T, 3 * d, dtype=torch.bfloat16, device=DEV)
    pos = torch.tensor([0, -1, 3, 4, 2, 1 << 30], dtype=torch.int32, device=DEV)
    P.qk_norm_rope_fwd(x, *gains, _table(4, d), y, 4, nh, nkv, d, positions=pos)
    bad = torch.tensor([False, True, False, True, False, True], device=DEV)
    assert torch.isnan(y[bad].float()).all() and torch.isfinite(y[~bad].float()).all()


def test_table_is_the_angles_in_64_bits():
    n, d = 5000, 128
    theta = 10000.0 ** (-2 * torch.arange(d // 2, dtype=torch.float64) / d)
    a = torch.arange(n, dtype=torch.float64)[:, None] * theta
    got = _table(n, d).cpu().double()
    # the angle's own error (a few roundings of 2^-53 at angles up to 5000) is far below fp32's half step
    assert (got[..., 0] - a.cos()).abs().max() <= 2 ** -24 and (got[..., 1] - a.sin()).abs().max() <= 2 ** -24


def test_a_captured_pass_replays():
    T, S, nh, nkv, d = 300, 100, 4, 2, 64
    x, dy, gains = _case(T, nh, nkv, d, 5)
    table = _table(S, d)
    w = (nh + nkv) * d
    y, dx = torch.empty(2, T, w, dtype=torch.bfloat16, device=DEV)
    dg = torch.empty(2, d, device=DEV)
    work = torch.empty(P.qk_norm_rope_bwd_workspace(T, nh, nkv, d), dtype=torch.uint8, device=DEV)

    def call():
        P.qk_norm_rope_fwd(x, *gains, table, y, S, nh, nkv, d)
        P.qk_norm_rope_bwd(x, *gains, table, dy, dx, dg[0], dg[1], work, S, nh, nkv, d)

    call()
    torch.cuda.synchronize()
    want = [t.clone() for t in (y, dx, dg)]
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            call()
        for _ in range(3):
            for t in (y, dx, dg):
                t.fill_(float("nan"))
            work.fill_(255)
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip((y, dx, dg), want))


def test_refusals():
    T, S, nh, nkv, d = 8, 8, 2, 1, 64
    x, dy, gains = _case(T, nh, nkv, d, 5)
    y, table = torch.empty(T, 3 * d, dtype=torch.bfloat16, device=DEV), _table(S, d)
    call = lambda x=x, g=gains[0], t=table, y=y, S=S, **kw: P.qk_norm_rope_fwd(x, g, gains[1], t, y, S, nh, nkv, d, **kw)  # noqa: E731
    call()
    for bad in (dict(x=x.float()), dict(x=x[:, :128]), dict(y=y[:4]), dict(g=gains[0].float()), dict(g=gains[0][:32]), dict(t=table[:4]), dict(t=table.double()),
                dict(t=table[..., 0]), dict(S=0), dict(eps=0.0), dict(positions=torch.zeros(T, device=DEV)), dict(positions=torch.zeros(4, dtype=torch.int32, device=DEV))):
        with pytest.raises(P.AhError):
            call(**bad)
    with pytest.raises(P.AhError, match="too few"):
        P.qk_norm_rope_bwd(x, *gains, table, dy, y, *torch.empty(2, d, device=DEV), torch.empty(8, dtype=torch.uint8, device=DEV), S, nh, nkv, d)
