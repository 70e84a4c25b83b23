"""Windowed attention with visible first tokens against its definition in 64 bits, element by element.

Tolerances.  Rounded to bf16 (at most 2^-8 of the value each): a probability before its product with V or dO, dS before its products with K and Q,
and the result.  So |o - ref| <= 2^-8 (sum_j p_ij |v_j| + |ref|), |dv| likewise with |do|, |dq - ref| <= 2^-8 (sum_j |ds_ij| |k_j| / sqrt d + |ref|),
|dk| likewise with |q|.  The rest is fp32 (hardware exponential of an argument of a few dozen: 1e-6 of a probability or so; dP - delta: 1e-6 of the sum of its
terms' magnitudes): 2 % on top of the former, and 1e-5 of sum p (|do| |v| + |do| |o|) |k|.  Log-sum-exp: 2e-6 of its size and of the largest score.
The backward reference starts from the kernel's own o and lse: they are inputs."""
import math

import pytest
import torch

import paper_2512_20953_amd as P

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _inputs(T, wq, wk, pad, seed):
    g = torch.Generator().manual_seed(seed)
    big = torch.randn(T, wq + 2 * wk + pad, generator=g).bfloat16().to(DEV)
    do = torch.randn(T, wq + pad, generator=g).bfloat16().to(DEV)[:, :wq]
    return big[:, :wq], big[:, wq:wq + wk], big[:, wq + wk:wq + 2 * wk], do


def _run(q, k, v, do, n_seq, S, nh, nkv, d, W, sinks, offsets=None):
    """Results in strided buffers of NaN, so that what was not written shows."""
    nan = lambda w: torch.full((q.shape[0], w + 24), float("nan"), dtype=torch.bfloat16, device=DEV)[:, 8:8 + w]  # noqa: E731
    o, dq, dk, dv = nan(nh * d), nan(nh * d), nan(nkv * d), nan(nkv * d)
    lse = torch.full((n_seq, nh, S), float("nan"), device=DEV)
    work = torch.full((P.attention_window_bwd_workspace(n_seq, S, nh, nkv, d, W, sinks),), 255, dtype=torch.uint8, device=DEV)
    P.attention_window_fwd(q, k, v, o, lse, n_seq, S, nh, nkv, d, W, sinks, offsets)
    P.attention_window_bwd(q, k, v, o, lse, do, dq, dk, dv, work, n_seq, S, nh, nkv, d, W, sinks, offsets)
    torch.cuda.synchronize()
    return o, lse, dq, dk, dv


def _check(q, k, v, do, o, lse, dq, dk, dv, spans, nh, nkv, d, W, sinks):
    rep, sc = nh // nkv, 1 / math.sqrt(d)
    for b, (r0, r1) in enumerate(spans):
        n = r1 - r0
        if n == 0:
            continue
        at = torch.arange(n, device=DEV)
        gap = at[:, None] - at
        hidden = (gap < 0) | ((gap >= W) & (at >= sinks))
        for kh in range(nkv):
            kc = slice(kh * d, kh * d + d)
            K, V = k[r0:r1, kc].double(), v[r0:r1, kc].double()
            sums = [torch.zeros(n, d, dtype=torch.float64, device=DEV) for _ in range(5)]   # dk, its bound twice over, dv, its bound
            for h in range(kh * rep, kh * rep + rep):
                qc = slice(h * d, h * d + d)
                Q, DO, O = (t[r0:r1, qc].double() for t in (q, do, o))
                s = (Q @ K.T * sc).masked_fill(hidden, -math.inf)
                ref_lse, p = torch.logsumexp(s, 1), torch.softmax(s, 1)
                got = lse[b, h, :n].double()
                room = 2e-6 * (1 + ref_lse.abs() + s.masked_fill(hidden, 0).abs().amax(1))
                assert ((got - ref_lse).abs() <= room).all(), ("lse", b, h, (got - ref_lse).abs().max().item())
                ref = p @ V
                _within("o", O, ref, 2 ** -8 * (p @ V.abs() + ref.abs()), b, h)
                p = torch.exp(s - got[:, None])
                dp, delta = DO @ V.T, (DO * O).sum(1, keepdim=True)
                slack = p * (DO.abs() @ V.abs().T + (DO * O).abs().sum(1, keepdim=True)) * 1e-5
                ds = p * (dp - delta)
                ref = ds @ K * sc
                _within("dq", dq[r0:r1, qc].double(), ref, 2 ** -8 * (ds.abs() @ K.abs() * sc + ref.abs()) + slack @ K.abs() * sc, b, h)
                sums[0] += ds.T @ Q * sc
                sums[1] += ds.abs().T @ Q.abs() * sc
                sums[2] += slack.T @ Q.abs() * sc
                sums[3] += p.T @ DO
                sums[4] += p.T @ DO.abs()
            _within("dk", dk[r0:r1, kc].double(), sums[0], 2 ** -8 * (sums[1] + sums[0].abs()) + sums[2], b, kh)
            _within("dv", dv[r0:r1, kc].double(), sums[3], 2 ** -8 * (sums[4] + sums[3].abs()), b, kh)


def _within(what, got, ref, room, b, h):
    bad = ~((got - ref).abs() <= 1.02 * room + 1e-30)
    assert not bad.any(), (what, b, h, bad.nonzero()[:4].tolist(), ((got - ref).abs() / (room + 1e-30)).max().item())


CASES = [  # n_seq, S, heads, key heads, head_dim, window, sinks
    (1, 1, 1, 1, 64, 1, 0), (2, 1, 4, 2, 128, 5, 3), (3, 2, 2, 1, 64, 1, 0), (1, 31, 3, 3, 128, 8, 2), (2, 63, 4, 1, 64, 64, 0), (1, 64, 2, 2, 128, 63, 64),
    (1, 65, 2, 1, 128, 64, 1), (2, 127, 4, 2, 64, 65, 0), (1, 128, 6, 2, 128, 1, 0), (1, 128, 3, 1, 64, 128, 0), (1, 129, 4, 4, 128, 33, 5),
    (1, 200, 4, 2, 64, 1000, 1000), (1, 257, 2, 1, 128, 96, 65), (2, 333, 6, 3, 64, 100, 0), (1, 500, 2, 2, 128, 128, 130), (1, 640, 4, 1, 64, 256, 4),
    (1, 1000, 4, 2, 128, 16, 3),       # far queries of the first keys in shares
    (1, 1500, 2, 1, 64, 40, 200),      # two blocks of first keys in shares
    (1, 1111, 1, 1, 128, 64, 1),
    (3, 700, 8, 8, 64, 1, 33),
    (2, 2050, 2, 2, 128, 300, 7),
]


@pytest.mark.parametrize("n_seq,S,nh,nkv,d,W,sinks", CASES)
def test_sequences_of_one_length(n_seq, S, nh, nkv, d, W, sinks):
    x = _inputs(n_seq * S, nh * d, nkv * d, 8 * (S % 3), S)
    out = _run(*x, n_seq, S, nh, nkv, d, W, sinks)
    _check(*x, *out, [(b * S, b * S + S) for b in range(n_seq)], nh, nkv, d, W, sinks)


@pytest.mark.parametrize("lengths,behind,nh,nkv,d,W,sinks", [
    ([1], 0, 2, 1, 64, 4, 1), ([0, 1, 0], 2, 2, 2, 128, 4, 1), ([5, 0, 64, 200, 1, 0], 7, 4, 2, 64, 32, 2), ([129, 128, 127, 2], 0, 3, 1, 128, 50, 0),
    ([1000, 3, 90], 5, 4, 2, 64, 20, 3), ([300, 1301], 1, 2, 2, 128, 64, 70)])
def test_packed_sequences(lengths, behind, nh, nkv, d, W, sinks):
    ends = [sum(lengths[:k]) for k in range(len(lengths) + 1)]
    T, S = ends[-1] + behind, max(lengths)
    x = _inputs(T, nh * d, nkv * d, 0, T)
    x[0][ends[-1]:], x[1][ends[-1]:], x[2][ends[-1]:], x[3][ends[-1]:] = (float("nan"),) * 4     # rows of no sequence are not read
    out = _run(*x, len(lengths), S, nh, nkv, d, W, sinks, torch.tensor(ends, dtype=torch.int32, device=DEV))
    _check(*x, *out, list(zip(ends, ends[1:])), nh, nkv, d, W, sinks)
    for t in (out[0], *out[2:]):
        assert torch.isnan(t[ends[-1]:]).all()                                                  # nor written
    for b, n in enumerate(lengths):
        assert torch.isnan(out[1][b, :, n:]).all()
    # a longest length that is an upper bound only changes no row
    more = _run(*x, len(lengths), S + 150, nh, nkv, d, W, sinks, torch.tensor(ends, dtype=torch.int32, device=DEV))
    for a, t in zip(out[:1] + out[2:3], more[:1] + more[2:3]):
        assert torch.equal(a[:ends[-1]], t[:ends[-1]])


def test_a_window_of_the_whole_sequence_is_causal_attention():
    B, S, nh, d = 2, 256, 3, 64
    T, w = B * S, nh * d
    qkv = torch.randn(T, 3 * w, generator=torch.Generator().manual_seed(1)).bfloat16().to(DEV)
    o, want = torch.empty(2, T, w, dtype=torch.bfloat16, device=DEV)
    lse, lse_want = torch.empty(2, B, nh, S, device=DEV)
    P.attention_fwd(qkv, want, lse_want, B, S, nh, d, True)
    P.attention_window_fwd(qkv[:, :w], qkv[:, w:2 * w], qkv[:, 2 * w:], o, lse, B, S, nh, nh, d, 1 << 30, 0)
    assert (o.float() - want.float()).norm() <= 2 ** -7 * want.float().norm()                   # (rounded in another order)
    assert (lse - lse_want).abs().max() <= 2e-5


def test_offsets_outside_the_buffers_are_cut():
    nh, d, T = 2, 64, 100
    x = _inputs(T, nh * d, nh * d, 0, 3)
    cut = _run(*x, 3, 64, nh, nh, d, 16, 2, torch.tensor([-5, 40, 90, 2000], dtype=torch.int32, device=DEV))
    good = _run(*x, 3, 64, nh, nh, d, 16, 2, torch.tensor([0, 40, 90, 100], dtype=torch.int32, device=DEV))
    for a, b in zip(cut, good):
        assert torch.equal(torch.nan_to_num(a.float(), nan=7.0), torch.nan_to_num(b.float(), nan=7.0))
    back = _run(*x, 2, 64, nh, nh, d, 16, 2, torch.tensor([50, 20, 60], dtype=torch.int32, device=DEV))     # a length below 0 is none
    assert torch.isfinite(back[0][20:60].float()).all() and torch.isnan(back[0][:20].float()).all()


@pytest.mark.parametrize("bad", [float("inf"), float("nan"), -3.0e38])
@pytest.mark.parametrize("at,W,sinks,d", [(300, 60, 2, 64), (20, 60, 2, 128), (40, 1, 5, 64), (100, 130, 70, 128)])
def test_what_nobody_sees_reaches_nobody(at, W, sinks, d, bad):
    """A key and value that are not finite: queries at .. at + W - 1 see them, also where they share a tile with the first tokens, which all later ones see."""
    S, nh = 900, 2
    x = _inputs(S, nh * d, nh * d, 0, 9)
    clean = _run(*x, 1, S, nh, nh, d, W, sinks)
    y = [t.clone() for t in x]
    y[1][at], y[2][at] = bad, bad
    o, lse, dq, dk, dv = _run(*y, 1, S, nh, nh, d, W, sinks)
    keep = torch.ones(S, dtype=torch.bool, device=DEV)
    # a block of 128 queries from q0 on walks the whole tile of 64 keys that holds `at` while q0 < at + W + 63: up to query at + W + 189
    keep[max(0, at - 192):at + W + 192] = False
    assert keep.sum() > 200
    for t, c in ((o, clean[0]), (dq, clean[2])):
        assert torch.equal(t[keep], c[keep])
    assert torch.equal(lse[:, :, keep], clean[1][:, :, keep])


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_a_bad_query_reaches_its_own_keys(bad):
    """A query and output gradient that are not finite: keys at - W + 1 .. at and the first tokens see them."""
    S, nh, d, W, sinks, at = 1000, 2, 64, 60, 2, 600
    x = _inputs(S, nh * d, nh * d, 0, 9)
    clean = _run(*x, 1, S, nh, nh, d, W, sinks)
    y = [t.clone() for t in x]
    y[0][at], y[3][at] = bad, bad
    out = _run(*y, 1, S, nh, nh, d, W, sinks)
    keep = torch.ones(S, dtype=torch.bool, device=DEV)
    keep[at - W - 192:at + 192] = False
    keep[:sinks + 192] = False
    for k in (3, 4):
        assert torch.equal(out[k][keep], clean[k][keep])
    keep[:sinks + 192] = True
    assert torch.equal(out[0][keep], clean[0][keep]) and torch.equal(out[2][keep], clean[2][keep])


def test_the_same_bits_every_time_and_two_streams_at_once():
    S, nh, nkv, d, W, sinks = 1500, 4, 2, 128, 100, 5
    x = _inputs(S, nh * d, nkv * d, 0, 4)
    first = _run(*x, 1, S, nh, nkv, d, W, sinks)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    torch.cuda.synchronize()
    for s in streams:
        with torch.cuda.stream(s):
            o, dq, dk, dv = (torch.empty_like(t) for t in (first[0], *first[2:]))
            lse = torch.empty_like(first[1])
            work = torch.empty(P.attention_window_bwd_workspace(1, S, nh, nkv, d, W, sinks), dtype=torch.uint8, device=DEV)
            P.attention_window_fwd(*x[:3], o, lse, 1, S, nh, nkv, d, W, sinks)
            P.attention_window_bwd(*x[:3], o, lse, x[3], dq, dk, dv, work, 1, S, nh, nkv, d, W, sinks)
            outs.append((o, lse, dq, dk, dv, work))
    torch.cuda.synchronize()
    for out in outs:
        assert all(torch.equal(a, b) for a, b in zip(out, first))


def test_a_captured_pass_replays():
    S, nh, nkv, d, W, sinks = 700, 2, 1, 64, 50, 3
    x = _inputs(S, nh * d, nkv * d, 0, 6)
    want = _run(*x, 1, S, nh, nkv, d, W, sinks)
    o, dq, dk, dv = (torch.empty_like(t) for t in (want[0], *want[2:]))
    lse = torch.empty_like(want[1])
    work = torch.empty(P.attention_window_bwd_workspace(1, S, nh, nkv, d, W, sinks), dtype=torch.uint8, device=DEV)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            P.attention_window_fwd(*x[:3], o, lse, 1, S, nh, nkv, d, W, sinks)
            P.attention_window_bwd(*x[:3], o, lse, x[3], dq, dk, dv, work, 1, S, nh, nkv, d, W, sinks)
        for _ in range(3):
            for t in (o, lse, dq, dk, dv):
                t.fill_(float("nan"))
            work.fill_(255)
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip((o, lse, dq, dk, dv), want))


def test_gradients_against_differences():
    """Directional derivatives of sum(o * do) in fp64 differences of the definition agree with the kernel's gradients to the rounding of bf16."""
    S, nh, nkv, d, W, sinks = 90, 2, 1, 64, 20, 3
    x = _inputs(S, nh * d, nkv * d, 0, 11)
    _, _, dq, dk, dv = _run(*x, 1, S, nh, nkv, d, W, sinks)
    at = torch.arange(S, device=DEV)
    gap = at[:, None] - at
    hidden = (gap < 0) | ((gap >= W) & (at >= sinks))

    def loss(q, k, v):
        total = 0
        for h in range(nh):
            c, kc = slice(h * d, h * d + d), slice(h // (nh // nkv) * d, h // (nh // nkv) * d + d)
            p = torch.softmax((q[:, c] @ k[:, kc].T / math.sqrt(d)).masked_fill(hidden, -math.inf), 1)
            total = total + ((p @ v[:, kc]) * x[3][:, c].double()).sum()
        return total.item()

    base = [t.double() for t in x[:3]]
    g = torch.Generator().manual_seed(2)
    for k, grad in enumerate((dq, dk, dv)):
        u = torch.randn(base[k].shape, generator=g).double().to(DEV)
        up, down = list(base), list(base)
        up[k], down[k] = base[k] + 1e-4 * u, base[k] - 1e-4 * u
        want = (loss(*up) - loss(*down)) / 2e-4
        # errors of single elements are independent and below 3 * 2^-8 of their size: their sum against a random direction is off by a few times that of the norm
        assert abs((grad.double() * u).sum().item() - want) <= 5 * 3 * 2 ** -8 * grad.double().norm().item()


def test_refusals():
    x = _inputs(64, 128, 128, 0, 1)
    o, lse = torch.empty(64, 128, dtype=torch.bfloat16, device=DEV), torch.empty(1, 2, 64, device=DEV)
    call = lambda **kw: P.attention_window_fwd(*[kw.pop(n, t) for n, t in zip(("q", "k", "v", "o", "lse"), (*x[:3], o, lse))],  # noqa: E731
                                               *[kw.pop(n, t) for n, t in zip(("B", "S", "nh", "nkv", "d", "W"), (1, 64, 2, 2, 64, 8))], **kw)
    call()
    for bad in (dict(q=x[0].float()), dict(q=x[0].T), dict(k=x[1][:, :64]), dict(v=x[2][:32]), dict(o=o[:, ::2]), dict(lse=lse[..., :32]), dict(S=63), dict(S=65),
                dict(q=torch.empty(64, 132, dtype=torch.bfloat16, device=DEV)[:, :128]), dict(q=torch.empty(64, 136, dtype=torch.bfloat16, device=DEV)[:, 4:132]),
                dict(offsets=torch.zeros(3, dtype=torch.int32, device=DEV)), dict(offsets=torch.zeros(2, dtype=torch.int64, device=DEV)), dict(W=0), dict(nkv=3),
                dict(sinks=-1)):
        with pytest.raises(P.AhError):
            call(**bad)
    work = torch.empty(8, dtype=torch.uint8, device=DEV)
    with pytest.raises(P.AhError, match="too few"):
        P.attention_window_bwd(*x[:3], o, lse, x[3], *[torch.empty_like(o) for _ in range(3)], work, 1, 64, 2, 2, 64, 8)
