"""The optimizer step by the momentum's orthogonal factor, through the binding, against the formula in 64 bits."""
import math

import pytest
import torch

import paper_2512_20953_amd as P

pytestmark = pytest.mark.gpu
A, B, C = 3.4445, -4.7750, 2.0315
U, H = 2.0 ** -24, 2.0 ** -11                        # half a step of fp32, of fp16
BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64


def randn(seed, *shape, dtype=F32, std=1.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype).cuda()


def low_rank(seed, r, c, rank=8, noise=0.05):
    return randn(seed, r, rank) @ randn(seed + 1, rank, c) + noise * randn(seed + 2, r, c)


def normed(u, eps):
    x = u.double()
    x = x if x.shape[0] <= x.shape[1] else x.T.contiguous()
    return x / (torch.linalg.matrix_norm(x) + eps)


def orthogonal(u, eps=1e-7, steps=5, pair=False):
    """The polynomial of u in 64 bits, and the same with the kernel's roundings (operands in fp16, X as two fp16 numbers) of sums in 64 bits.  pair: with the first two steps at
    once, (a + B1)(a + B) = a^2 + Q, in which the second step's A is (a + B) A (a + B)."""
    x = y = normed(u, eps)
    f16 = lambda t: t.half().double()                  # noqa: E731
    split = lambda t: (f16(64 * t), f16((64 * t - f16(64 * t)) * 2048))   # noqa: E731
    hi, lo = split(y.float().double())
    mirrored = lambda t: t.tril() + t.tril(-1).T       # noqa: E731
    for k in range(steps):
        q = x @ x.T.contiguous()
        x = A * x + (B * q + C * (q @ q)) @ x
        if pair and k == 1:
            continue
        a, by = f16(hi @ hi.T.contiguous() / 4), A
        b = f16(B * a + C * (a @ a) / 1024)
        if pair and k == 0 and steps > 1:
            c = mirrored(f16(b @ a / 1024))
            a = mirrored(f16(A * A * a + 2 * A * c + b @ c / 1024))
            b1 = f16(B * a + C * (a @ a) / 1024)
            b, by = mirrored(f16(A * (b + b1) + b1 @ b / 1024)), A * A
        y = (by * (hi + lo / 2048) + b @ hi / 1024) / 64
        hi, lo = split(y)
    turn = (lambda t: t) if u.shape[0] <= u.shape[1] else (lambda t: t.T)
    return turn(x), turn((hi + lo / 2048) / 64)


def norm(t):
    return torch.linalg.matrix_norm(t).item()


def room_of(want, rounded):
    """How far from `want` the kernel may be, by how far the rounded form is.

    The kernel's sums are in fp32: off by about U sqrt(k / 32) of an element, they take one in a thousand or so to the other side of an fp16 rounding.  That moves a first step
    by sqrt(12 / 1000) = 0.11 of what all of its roundings (uniform within half a step) make, and every step behind it carries a difference on by up to 3.44 = the polynomial's slope at 0,
    four steps by 140: by the end the two forms' roundings are two draws of one distribution, not the same ones.  What they leave is a sum of many small errors; it is
    largest along the smallest singular values, and along one of them still a vector of at least n independent parts (n: the smaller side), whose length varies by 1 / sqrt(2 n): 0.09
    for n = 64, so that 1.5 times the other's length is five such deviations.  Of fewer than 64 rows or columns hardly a rounding goes to the other side (5 steps of a few hundred at a thousandth
    each), and one that does adds at most one whole step to the half steps that all others are off by: 3 times.  Beside that 2^-14 of the whole: fp32's own roundings, 2 U carried on by 3.44^5 = 480."""
    return (1.5 if min(want.shape) >= 64 else 3.0) * norm(rounded - want) + 2.0 ** -14 * norm(want)


def one_step(u, eps=1e-7):
    """How far a single step may be off, whatever the roundings: the operand's (H |X|, twice in A), A's and B's own, sums over k terms in fp32, the halves of X (2^-22)."""
    x = normed(u, eps)
    (n, k), f, s, tiny = x.shape, norm(x), torch.linalg.matrix_norm(x, ord=2).item(), math.sqrt(x.numel()) * 2.0 ** -31
    q = x @ x.T.contiguous()
    b = B * q + C * (q @ q)
    fa, fb, sb, g = norm(q), norm(b), torch.linalg.matrix_norm(b, ord=2).item(), norm(A * x + b @ x)
    e_a = 2 * s * (H * f + tiny) + k * U * f * f + H * fa + n * 2.0 ** -35
    e_b = (abs(B) + 2 * C * s * s) * e_a + C * n * U * fa * fa + (H + 8 * U) * fb + n * 2.0 ** -35
    return 1.05 * (e_b * s + sb * (H * f + tiny) + n * U * fb * f + 8 * U * (A * f + g) + 2.0 ** -21 * (A * f + g) + tiny)


def update_of(gs, **kw):
    """The updates X of matrices whose gradients are gs: parameters 0, momentum 0, lr 1, scale 1"""
    ps = [torch.zeros(g.shape, device="cuda") for g in gs]
    opt = P.Muon(ps, gs, scale=1.0, **kw)
    opt.step(1.0)
    return [-p for p in ps], opt


SIZES = [(1, 1), (1, 7), (5, 3), (64, 64), (100, 37), (128, 300), (257, 129), (300, 1000), (1000, 260), (512, 512), (130, 2049)]


@pytest.mark.parametrize("r,c", SIZES)
@pytest.mark.parametrize("make", [randn, low_rank])
def test_update(r, c, make):
    g = make(r + c, r, c)
    (x,), opt = update_of([g])
    want, rounded = orthogonal(g * 0.05 * 1.95)
    print("%d x %d: off by %.2g, of %.2g, the rounded form by %.2g; from that %.2g" % (r, c, norm(x.double() - want), norm(want), norm(rounded - want), norm(x.double() - rounded)))
    assert norm(x.double() - want) <= room_of(want, rounded)
    # m = 0.05 g: 0.05 as fp32 holds it (1 - 0.95), one product and one sum
    assert ((opt.m[0].double() - 0.05 * g.double()).abs() <= 4 * U * 0.05 * g.double().abs()).all()


def test_tiles_of_a_large_call_and_matrices_of_unlike_sizes():
    for shapes in ([(2500, 4300)], [(512, 1000)] * 25 + [(3, 5), (1000, 520), (1, 1)], [(4400, 2304), (300, 2000)]):
        gs = [randn(k, r, c, std=10.0 ** (k % 5 - 2)) for k, (r, c) in enumerate(shapes)]
        xs, _ = update_of(gs)
        for k in {0, len(gs) // 2, len(gs) - 3, len(gs) - 2, len(gs) - 1} & set(range(len(gs))):
            room = max(room_of(*orthogonal(gs[k] * 0.05 * 1.95, pair=pair)) for pair in (False, True))       # (sizes decide, here of either kind)
            want, _ = orthogonal(gs[k] * 0.05 * 1.95)
            assert norm(xs[k].double() - want) <= room, (k, shapes[k])


@pytest.mark.parametrize("make", [randn, low_rank])
@pytest.mark.parametrize("shapes", [[(1, 1), (1, 7), (9, 40)], [(24, 100), (64, 64), (100, 37)], [(130, 2049)], [(256, 256)], [(300, 1000), (8000, 250), (200, 520), (17, 30000)], [(128, 130)] * 26])
def test_small_matrices_are_not_rounded_to_sixteen_bits(shapes, make):
    """Of at most 256 rows or columns.  Operands are kept in 22 bits: A, B and X of a step are off by a few of 2^-22 and, as sums in fp32, of U each, 16 U of X together.  Four more steps carry
    that on by up to 140, the five steps' shares are independent: 16 U 140 sqrt(5) = 2^-11.7, of an X whose norm is 2 or more (fewer than eight singular values: none small enough to be carried
    on so far).  Operands in 11 bits would leave 1e-3 to 3e-3."""
    gs = [make(3 * k, r, c) for k, (r, c) in enumerate(shapes)]
    xs, _ = update_of(gs)
    for k, s in enumerate(shapes):
        if min(s) > 256:
            continue
        want, _ = orthogonal(gs[k] * 0.05 * 1.95)
        off = norm(xs[k].double() - want) / norm(want)
        print(s, "off by %.2g" % off)
        assert off <= 2.0 ** -12, (k, s)


@pytest.mark.parametrize("make", [randn, low_rank])
@pytest.mark.parametrize("shapes,steps", [([(2048, 8000)], 5), ([(9000, 1500)] * 2 + [(1500, 5000)], 5), ([(700, 2500)] * 12, 5), ([(700, 2500)] * 12, 2), ([(700, 2500)] * 12, 3), ([(2304, 9000)] * 2, 4)])
def test_many_more_columns_than_rows(shapes, steps, make):
    """Where the first two steps are taken at once"""
    gs = [make(3 * k, r, c) for k, (r, c) in enumerate(shapes)]
    xs, opt = update_of(gs, ns_steps=steps)
    n = sum(min(s) ** 2 for s in shapes)
    assert opt._work.numel() > sum(6 * g.numel() for g in gs) + 8 * n          # (the two square matrices more that this takes)
    for k in {0, len(gs) - 1}:
        want, rounded = orthogonal(gs[k] * 0.05 * 1.95, steps=steps, pair=True)
        print(shapes[k], steps, "off by %.2g, the rounded form by %.2g, of %.2g" % (norm(xs[k].double() - want), norm(rounded - want), norm(want)))
        assert norm(xs[k].double() - want) <= room_of(want, rounded), (k, shapes[k])


@pytest.mark.parametrize("steps", [1, 2, 5, 9])
def test_singular_values(steps):
    g = randn(steps, 200, 333)
    (x,), _ = update_of([g], ns_steps=steps)
    want, rounded = orthogonal(g * 0.05 * 1.95, steps=steps)
    assert norm(x.double() - want) <= room_of(want, rounded)
    if steps >= 5:      # what the documentation says of the factor
        s = torch.linalg.svdvals(x.double().cpu())
        assert 0.68 <= s.min() and s.max() <= 1.21


@pytest.mark.parametrize("r,c", SIZES + [(2, 100000), (70000, 3), (1, 131072)])
@pytest.mark.parametrize("rank", [1, 3, 0])
def test_one_step(r, c, rank):
    """Of matrices with few directions, whose singular values are large from the start, and of others"""
    g = randn(r + c, r, rank) @ randn(1, rank, c) if rank else randn(r + c, r, c)
    (x,), _ = update_of([g], ns_steps=1)
    want, rounded = orthogonal(g * 0.05 * 1.95, steps=1)
    # (the product that made a matrix of few directions is the gradient as it is; u = 0.0975 g is rounded four times)
    assert norm(x.double() - want) <= one_step(g * 0.05 * 1.95) + 8 * U * A * norm(want)
    if max(r, c) < 10000:       # (longer sums than that are off by more than an operand's rounding leaves in them)
        assert norm(x.double() - want) <= room_of(want, rounded)


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("param,grad,master", [(BF, F32, False), (BF, BF, True), (F32, BF, False), (F32, F32, False), (BF, F32, True)])
def test_step(param, grad, master, nesterov):
    shapes, lr, wd, mu = [(96, 200), (130, 70), (64, 64)], 0.01, 0.1, 0.9
    ps = [randn(k, *s, dtype=param, std=0.02) for k, s in enumerate(shapes)]
    gs = [randn(k + 10, *s, dtype=grad) for k, s in enumerate(shapes)]
    ms = [randn(k + 20, *s) for k, s in enumerate(shapes)]
    before, m0 = [p.double().clone() for p in ps], [m.double().clone() for m in ms]
    opt = P.Muon(ps, gs, momentum=mu, nesterov=nesterov, weight_decay=[wd, 0.0, wd], scale=[None, 2.0, 0.5], master=master, m=ms)
    opt.step(lr)
    for k, (r, c) in enumerate(shapes):
        g = gs[k].double()
        m = m0[k] + (1 - mu) * (g - m0[k])
        assert ((ms[k].double() - m).abs() <= 4 * U * (m0[k].abs() + g.abs())).all()
        u = m + (1 - mu) * (g - m) if nesterov else m
        x, rounded = orthogonal(u)
        room = room_of(x, rounded)
        scale = (0.2 * math.sqrt(max(r, c)), 2.0, 0.5)[k]
        want = before[k] * (1 - lr * (wd, 0.0, wd)[k]) - lr * scale * x
        out = (opt.master[k] if master else ps[k]).double()
        step = torch.finfo(BF).eps / 2 if param is BF and not master else 0.0
        # u itself is off by 8 U (|m| + |g|) relative to its norm, which the polynomial carries on by at most 3.4445^5
        e_u = 8 * U * math.sqrt(((m0[k].abs() + g.abs()) ** 2).sum().item()) / torch.linalg.matrix_norm(u).item() * 3.4445 ** 5
        assert torch.linalg.matrix_norm(out - want).item() <= lr * scale * (room + e_u) + torch.linalg.matrix_norm((4 * U + step) * (before[k].abs() + want.abs())).item()
        if master:
            assert torch.equal(ps[k], opt.master[k].to(BF))


def test_columns_of_wider_matrices():
    r, widths = 150, (64, 70, 33)
    wide = lambda seed, dt: randn(seed, r + 2, sum(widths) + 9, dtype=dt)   # noqa: E731
    P0, G0, M0, Q0 = wide(1, BF), wide(2, F32), wide(3, F32), wide(4, F32)
    cut = lambda t: [t[1:-1, a:a + w] for a, w in ((2, 64), (66, 70), (140, 33))]   # noqa: E731
    apart = [x.contiguous() for x in cut(P0)], [x.contiguous() for x in cut(G0)], [x.contiguous() for x in cut(M0)], [x.contiguous() for x in cut(Q0)]
    keep = [t.clone() for t in (P0, G0, M0, Q0)]
    for p, g, m, q in ((*map(cut, (P0, G0, M0, Q0)),), apart):
        P.Muon(p, g, weight_decay=0.1, m=m, master=q).step(0.02)
    for t, old, new in zip((P0, G0, M0, Q0), keep, apart):
        for x, y in zip(cut(t), new):
            assert torch.equal(x, y)
        for x, y in zip(cut(t), cut(old)):
            x.copy_(y)
        assert torch.equal(t, old)                     # nothing beside the blocks


def test_sizes_of_gradients_and_none():
    """The update does not depend on the gradient's size, from 1e-18 (an eps far below) to 1e30; a gradient of zeros gives none."""
    g = randn(1, 80, 120)
    (want,), _ = update_of([g], eps=1e-37)
    for power in (-60, -40, 40, 100):                  # powers of two, eps far below half a step of the norm: the same bits
        (x,), _ = update_of([g * 2.0 ** power], eps=1e-37)
        assert torch.equal(x, want)
    (x,), _ = update_of([torch.zeros_like(g)])
    assert (x == 0).all()
    (x,), _ = update_of([g * 1e-9])                    # a norm of about 1e-8 beside an eps of 1e-7
    ref, rounded = orthogonal(g * 1e-9 * 0.05 * 1.95)
    assert norm(x.double() - ref) <= room_of(ref, rounded)


def test_what_is_not_finite_stays_in_its_matrix():
    gs = [randn(k, 70, 90) for k in range(4)]
    clean, _ = update_of([g.clone() for g in gs])
    gs[1][3, 4], gs[2][5] = float("nan"), float("inf")
    xs, _ = update_of(gs)
    assert torch.equal(xs[0], clean[0]) and torch.equal(xs[3], clean[3])
    assert xs[1].isnan().all() and xs[2].isnan().all()


def test_what_the_scratch_memory_held_and_matrices_without_elements():
    shapes = [(200, 333), (0, 7), (64, 64), (5, 0), (300, 40)]
    gs = [randn(k, *s) for k, s in enumerate(shapes)]
    clean, _ = update_of([g for g in gs if g.numel()])
    ps = [torch.zeros_like(g) for g in gs]
    opt = P.Muon(ps, gs, scale=1.0)
    opt._work.fill_(255)
    opt.step(1.0)
    assert all(torch.equal(-p, x) for p, x in zip([p for p in ps if p.numel()], clean))
    P.Muon([torch.zeros(0, 3, device="cuda")], [torch.zeros(0, 3, device="cuda")]).step(1.0)


@pytest.mark.parametrize("kind", ["fp32", "master", "bf16"])
@pytest.mark.parametrize("shapes", [[(64, 64), (200, 333), (300, 40), (1, 9)], [(700, 2500)] * 6 + [(30, 70), (256, 300), (257, 300), (300, 1000)], [(100, 90)] * 30 + [(2048, 8000)]])
def test_small_and_large_matrices_of_each_type(shapes, kind):
    """In scratch memory that held NaN, and nothing behind its end is written.  bf16 parameters: 2^-8 of each element more."""
    gs = [randn(k, r, c) for k, (r, c) in enumerate(shapes)]
    ps = [torch.zeros(*s, dtype=F32 if kind == "fp32" else BF, device="cuda") for s in shapes]
    opt = P.Muon(ps, gs, scale=1.0, master=kind == "master" or None)
    need = opt._work.numel()
    opt._work = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")
    opt.step(1.0)
    assert (opt._work[need:] == 255).all()
    xs = [-p.double() for p in (opt.master if kind == "master" else ps)]
    for k, s in {s: (k, s) for k, s in enumerate(shapes)}.values():
        want, rounded = orthogonal(gs[k] * 0.05 * 1.95)
        room = room_of(want, rounded)
        if min(s) > 300:
            room = max(room, room_of(*orthogonal(gs[k] * 0.05 * 1.95, pair=True)))
        if kind != "bf16" and min(s) <= 256:
            room = 2.0 ** -12 * norm(want)
        if kind == "bf16":
            room += 2.0 ** -8 * (norm(want) + room)
        assert norm(xs[k] - want) <= room, (k, s)
        if kind == "master":
            assert torch.equal(opt.master[k].to(BF), ps[k])


def test_more_matrices_than_are_worked_on_together():
    """2^26 elements each: four to a group, in one call; a matrix comes out the same wherever it stands"""
    n = 8192
    g = [randn(k, n, n) for k in range(2)]
    ps = [torch.zeros(n, n, device="cuda") for _ in range(5)]
    P.Muon(ps, [g[0], g[1], g[1], g[0], g[0]], scale=1.0).step(1.0)
    assert torch.equal(ps[0], ps[3]) and torch.equal(ps[0], ps[4]) and torch.equal(ps[1], ps[2])
    x = -ps[0][:, :512].double()                       # 512 of the columns of a factor whose singular values are 0.68 .. 1.21: theirs are at most that, and not 0
    s = torch.linalg.eigvalsh(x.T @ x).sqrt()
    assert 0 < s.min() and s.max() <= 1.21


def test_factor_of_the_gradients_norm():
    ps, gs = [randn(1, 60, 100), randn(2, 100, 30)], [randn(3, 60, 100, std=5.0), randn(4, 100, 30, std=5.0)]
    out, work = torch.empty(2, device="cuda"), torch.empty(P.grad_norm_workspace(2), dtype=torch.uint8, device="cuda")
    P.grad_norm(gs, out, work, 1.0)
    size = math.sqrt(sum(g.double().square().sum().item() for g in gs))
    assert math.isclose(out[0].item(), size, rel_tol=2 * U) and math.isclose(out[1].item(), 1 / size, rel_tol=4 * U)
    assert torch.equal(P.AdamW([p.clone() for p in ps], gs).grad_norm(1.0), out)
    out[1] = 2.0 ** -6                                 # a power of two: the gradients' bits stay
    a, b = [p.clone() for p in ps], [p.clone() for p in ps]
    oa, ob = P.Muon(a, gs), P.Muon(b, [g * 2.0 ** -6 for g in gs])
    oa.step(0.1, grad_norm=out)
    ob.step(0.1)
    assert all(torch.equal(x, y) for x, y in zip(a + oa.m, b + ob.m))
    out[1] = float("nan")
    keep = [t.clone() for t in a + oa.m]
    oa.step(0.1, grad_norm=out)
    assert all(torch.equal(x, y) for x, y in zip(a + oa.m, keep))


def test_captured_and_on_two_streams():
    shapes = [(200, 700), (300, 128), (64, 65)]
    make = lambda: ([randn(k, *s, dtype=BF) for k, s in enumerate(shapes)], [randn(k + 9, *s) for k, s in enumerate(shapes)])   # noqa: E731
    (pe, ge), (pg, gg), (p1, g1), (p2, g2) = make(), make(), make(), make()
    eager, graphed = P.Muon(pe, ge, weight_decay=0.1, master=True), P.Muon(pg, gg, weight_decay=0.1, master=True)
    lr = torch.tensor([0.02], device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        graphed.step(lr, stream=s)
    for rep in range(3):
        lr.fill_(0.02 / (rep + 1))
        graph.replay()
        torch.cuda.synchronize()
        eager.step(float(lr.item()))
        assert all(torch.equal(x, y) for x, y in zip(pe + eager.m + eager.master, pg + graphed.m + graphed.master)), rep
        for x, y in zip(ge, gg):
            x.neg_(), y.neg_()
    one, two = P.Muon(p1, g1), P.Muon(p2, g2)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(4):
        one.step(0.02, stream=s1)
        two.step(0.02, stream=s2)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(p1 + one.m, p2 + two.m))


@pytest.mark.parametrize("shapes", [[(700, 2500)] * 6 + [(40, 90), (300, 310)], [(1500, 1500), (250, 80)]])
def test_captured_groups_of_unlike_matrices(shapes):
    """The groups follow each other in the same scratch memory, the first two steps at once or not"""
    make = lambda: ([randn(k, *s) for k, s in enumerate(shapes)], [randn(k + 9, *s) for k, s in enumerate(shapes)])   # noqa: E731
    (pe, ge), (pg, gg) = make(), make()
    eager, graphed = P.Muon(pe, ge), P.Muon(pg, gg)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        graphed.step(0.02, stream=s)
    for rep in range(3):
        graph.replay()
        torch.cuda.synchronize()
        eager.step(0.02)
        assert all(torch.equal(x, y) for x, y in zip(pe + eager.m, pg + graphed.m)), rep
        for x, y in zip(ge, gg):
            x.neg_(), y.neg_()


def test_tensors_that_overlap_are_refused():
    f = lambda *s: torch.zeros(*s, device="cuda")      # noqa: E731
    p, q, g, w = f(32, 48), f(32, 48), f(32, 48), f(32, 96)
    P.Muon([w[:, :48], w[:, 48:]], [g, g])             # columns beside each other, a gradient twice
    P.Muon([w[:, :48]], [w[:, 48:]])
    for params, grads, kw in (([p, p], [g, g], {}), ([p], [p], {}), ([w[:, :48], w[:, 47:95]], [g, g], {}), ([p, q], [g, g], dict(m=[q, f(32, 48)])), ([p], [g], dict(m=[g])),
                              ([w[:, :48], w.view(64, 48)[:32]], [g, g], {}), ([w[:16, 60:], w.view(-1)[90:90 + 36].view(1, 36)], [g[:16, :36], g[:1, :36]], {})):
        with pytest.raises(P.AhError, match="overlap"):
            P.Muon(params, grads, **kw)
