"""Embedding and its gradient through the C ABI against plain forms in 64 bits."""
import math

import pytest
import torch

import paper_2512_20953_amd as P

pytestmark = pytest.mark.gpu
U = 2.0 ** -24                                       # half a step of fp32
BF, F32 = torch.bfloat16, torch.float32


def half_step(t):
    return torch.finfo(t).eps / 2


def randn(seed, *shape, dtype=F32, std=1.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype).cuda()


def tokens_of(seed, T, V, bits=64, none=0, hot=0):
    g = torch.Generator().manual_seed(seed)
    t = torch.randint(0, V, (T,), generator=g)
    if hot:
        t[torch.rand(T, generator=g) < 0.7] = hot % V
    if none:
        t[torch.rand(T, generator=g) < 1 / none] = -1
    return t.to(torch.int32 if bits == 32 else torch.int64).cuda()


def padded(t, ld, at=0):
    """t as columns of a wider matrix, from column `at` on"""
    wide = torch.full((t.shape[0], ld), 7.0, dtype=t.dtype, device=t.device)
    wide[:, at:at + t.shape[1]] = t
    return wide[:, at:at + t.shape[1]]


FWD = [  # T, V, width, table, rows, bits, scale, positions, extra columns
    (1, 1, 1, BF, BF, 64, 1.0, 0, 0), (1, 7, 4096, BF, BF, 32, 1.0, 0, 0), (130, 50, 64, BF, F32, 64, 8.0, 0, 0), (257, 33, 1001, F32, BF, 32, 0.5, 100, 0),
    (64, 11, 2056, F32, F32, 64, 3.0, 64, 8), (300, 1000, 24, BF, BF, 64, 2.0, 7, 5), (5, 3, 65536, BF, BF, 64, 1.0, 2, 0), (0, 5, 16, BF, BF, 64, 1.0, 0, 0)]


@pytest.mark.parametrize("T,V,w,tt,at,bits,scale,pos,extra", FWD)
def test_rows_of_the_table(T, V, w, tt, at, bits, scale, pos, extra):
    table, tok = padded(randn(1, V, w, dtype=tt), w + extra, extra // 2), tokens_of(2, T, V, bits, none=5)
    pt = padded(randn(3, pos, w, dtype=tt), w + 2 * extra) if pos else None
    y = padded(torch.zeros(T, w, dtype=at, device="cuda"), w + extra)
    P.embedding_fwd(table, tok, y, scale=scale, pos_table=pt, seq_len=pos)
    e = torch.where((tok >= 0)[:, None], table.double()[tok.long().clamp_min(0)], 0.0) * scale if T else y.double()
    want = e + pt.double()[torch.arange(T) % pos] if pos else e
    # the product and the sum are rounded to fp32, the result to its type
    room = U * e.abs() + 2 * U * want.abs() + half_step(at) * want.abs() * (1 + 1e-6)
    assert ((y.double() - want).abs() <= room).all()


def test_positions_of_their_own_and_what_is_no_token():
    T, V, w, n = 200, 40, 72, 30
    table, pt, tok = randn(1, V, w, dtype=BF), randn(2, n, w, dtype=BF), tokens_of(3, T, V, 32)
    pos = torch.randint(0, n, (T,), generator=torch.Generator().manual_seed(4)).int().cuda()
    tok[3], tok[5], tok[7], tok[9] = V, -2, -1, 2 ** 31 - 1
    pos[11], pos[13] = n, -1
    y = torch.zeros(T, w, dtype=BF, device="cuda")
    P.embedding_fwd(table, tok, y, pos_table=pt, positions=pos)
    bad = torch.zeros(T, dtype=torch.bool, device="cuda")
    bad[[3, 5, 9, 11, 13]] = True
    assert torch.equal(y.isnan().all(1), bad) and torch.equal(y.isnan().any(1), bad)
    assert torch.equal(y[7], pt[pos[7].item()])
    ok = ~bad & (tok >= 0)
    want = table.float()[tok.long().clamp(0, V - 1)] + pt.float()[pos.long().clamp(0, n - 1)]
    assert torch.equal(y[ok], want.to(BF)[ok])
    wide = tok.long()
    wide[3] = 2 ** 32 + 1                            # not token 1
    P.embedding_fwd(table, wide, y)
    assert y[3].isnan().all() and torch.equal(y[0], table[tok[0].item()])


def check_bwd(tok, dy, V, scale, beta, ld=0, seed=5):
    T, w = dy.shape
    d = padded(randn(seed, V, w), ld or w)
    before = d.double().clone() if beta else torch.zeros(V, w, dtype=torch.float64, device="cuda")
    work = torch.full((P.embedding_bwd_workspace(T, V, w),), 0xC3, dtype=torch.uint8, device="cuda")
    if not beta:
        d.fill_(float("nan"))
    P.embedding_bwd(tok, dy, d, work, scale=scale, beta=beta)
    ok = (tok >= 0) & (tok < V)
    at, rows = tok[ok].long(), dy.double()[ok]
    total = torch.zeros(V, w, dtype=torch.float64, device="cuda").index_add_(0, at, rows) * scale
    size = torch.zeros(V, w, dtype=torch.float64, device="cuda").index_add_(0, at, rows.abs()) * abs(scale)
    n = torch.bincount(at, minlength=V).double()[:, None]
    # n - 1 sums, the scale and the last sum, each rounded once
    room = (n + 2) * U * (size + before.abs())
    assert ((d.double() - before - total).abs() <= room).all()
    untouched = (n == 0)[:, 0]
    assert torch.equal(d.double()[untouched], before[untouched])
    return d


BWD = [  # T, V, width, type, bits, scale, beta, none, hot
    (1, 1, 1, F32, 64, 1.0, 0, 0, 0), (1, 5, 16, BF, 32, 2.0, 1, 0, 0), (31, 4, 8, BF, 64, 1.0, 0, 0, 0), (32, 1, 264, BF, 64, 1.0, 1, 0, 0),
    (33, 300, 1001, F32, 32, 0.5, 0, 3, 0), (1000, 17, 64, BF, 64, 1.0, 1, 4, 0), (4096, 255, 40, BF, 32, 1.0, 0, 0, 3), (4097, 256, 33, F32, 64, 1.0, 0, 0, 255),
    (5000, 257, 2056, BF, 64, 1.0, 1, 7, 9), (9000, 70000, 24, BF, 32, 1.0, 0, 0, 66000), (70000, 3, 16, F32, 64, 1.0, 0, 0, 1), (9, 20, 8, BF, 64, 1.0, 0, 1, 0),
    (300000, 1000, 8, BF, 32, 1.0, 1, 50, 0), (16384, 70000, 8, F32, 32, 1.0, 0, 9, 4), (16385, 70000, 8, F32, 32, 1.0, 0, 9, 4), (3, 200000, 1, F32, 64, 1.0, 0, 0, 0),
    (40, 30, 5000, F32, 64, 1.0, 0, 4, 0), (100, 9, 8200, BF, 64, 1.0, 0, 0, 3), (40, 5, 65536, BF, 32, 1.0, 1, 3, 0),
    (50, 3, 65535, F32, 32, 1.0, 0, 3, 0)]


@pytest.mark.parametrize("T,V,w,kind,bits,scale,beta,none,hot", BWD)
def test_gradient_of_the_table(T, V, w, kind, bits, scale, beta, none, hot):
    check_bwd(tokens_of(T, T, V, bits, none, hot), padded(randn(T + 1, T, w, dtype=kind), w + (8 if w % 16 == 8 else 0)), V, scale, beta)


@pytest.mark.parametrize("V,w", [(50, 64), (50, 33)])
def test_gradient_beside_other_columns_and_no_rows(V, w):
    tok, dy = tokens_of(1, 400, V, none=6), randn(2, 400, w, dtype=BF)
    for beta in (0, 1):
        d = check_bwd(tok, dy, V, 1.0, beta, ld=w + 8)
        assert (d.as_strided((V, 8), d.stride(), d.storage_offset() + w) == 7).all()
    d = randn(3, V, w)
    want = d.clone()
    work = torch.empty(P.embedding_bwd_workspace(0, V, w), dtype=torch.uint8, device="cuda")
    P.embedding_bwd(tok[:0], dy[:0], d, work, beta=1)
    assert torch.equal(d, want)
    P.embedding_bwd(tok[:0], dy[:0], d, work, beta=0)
    assert (d == 0).all()


def test_gradient_is_the_same_every_time_and_captured():
    T, V, w = 6000, 500, 136
    tok, dy = tokens_of(1, T, V, hot=5), randn(2, T, w, dtype=BF)
    work = torch.empty(P.embedding_bwd_workspace(T, V, w), dtype=torch.uint8, device="cuda")
    first = torch.empty(V, w, device="cuda")
    P.embedding_bwd(tok, dy, first, work)
    d, y = torch.empty_like(first), torch.empty(T, w, dtype=F32, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        P.embedding_bwd(tok, dy, d, work, stream=s)
        P.embedding_fwd(d, tok, y, scale=2.0, stream=s)
    for rep in range(3):
        d.fill_(float("nan"))
        work.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(d, first), rep
        assert torch.equal(y, 2 * first[tok.long()]), rep
        again = torch.empty_like(first)
        P.embedding_bwd(tok, dy, again, work)
        torch.cuda.synchronize()
        assert torch.equal(again, first), rep


def test_padding_reads_nothing():
    """Rows of dy and of the table that belong to no token may hold anything"""
    T, V, w = 900, 70, 40
    tok, dy, table = tokens_of(1, T, V, none=3), randn(2, T, w, dtype=BF), randn(3, V, w, dtype=BF)
    tok[tok == 0] = 1
    dy[tok < 0], table[0] = float("nan"), float("inf")
    y, d = torch.empty_like(dy), torch.empty(V, w, device="cuda")
    P.embedding_fwd(table, tok, y)
    P.embedding_bwd(tok, dy, d, torch.empty(P.embedding_bwd_workspace(T, V, w), dtype=torch.uint8, device="cuda"))
    assert (y[tok < 0] == 0).all() and y.isfinite().all() and d.isfinite().all() and (d[0] == 0).all()


@pytest.mark.parametrize("T", [700, 20000])
def test_rows_far_into_a_large_table(T):
    """Elements behind the 2^31st, of the table and of its gradient"""
    V, w = 1100000, 2048
    table = torch.zeros(V, w, dtype=BF, device="cuda")
    tok = V - 1 - torch.arange(T, device="cuda") // 2 * 37
    table[tok] = randn(1, T, w, dtype=BF)
    y = torch.empty(T, w, dtype=BF, device="cuda")
    P.embedding_fwd(table, tok, y)
    assert torch.equal(y, table[tok])
    del table
    dy, d = randn(2, T, w, dtype=BF), torch.full((V, w), 7.0, device="cuda")
    P.embedding_bwd(tok, dy, d, torch.empty(P.embedding_bwd_workspace(T, V, w), dtype=torch.uint8, device="cuda"))
    assert torch.equal(d[tok[::2]], dy[::2].float() + dy[1::2].float())
    d[tok] = 0
    assert not d.any()


def test_a_row_that_is_not_finite_reaches_its_token_alone():
    T, V, w = 3000, 90, 72
    tok, dy = tokens_of(1, T, V), randn(2, T, w, dtype=BF)
    dy[100], dy[2000, 3] = float("nan"), float("inf")
    d = torch.empty(V, w, device="cuda")
    P.embedding_bwd(tok, dy, d, torch.empty(P.embedding_bwd_workspace(T, V, w), dtype=torch.uint8, device="cuda"))
    bad = ~d.isfinite()
    want = torch.zeros_like(bad)
    want[tok[100].item()] = True
    want[tok[2000].item(), 3] = True
    assert torch.equal(bad, want)


def test_gradient_against_differences():
    T, V, w, h = 12, 5, 3, 1 / 64
    table, tok, dy = randn(1, V, w).round(decimals=2), tokens_of(2, T, V, none=4), randn(3, T, w)
    d = torch.empty(V, w, device="cuda")
    P.embedding_bwd(tok, dy, d, torch.empty(P.embedding_bwd_workspace(T, V, w), dtype=torch.uint8, device="cuda"), scale=1.5)

    def f(t):
        y = torch.empty(T, w, device="cuda")
        P.embedding_fwd(t, tok, y, scale=1.5)
        return (y.double() * dy.double()).sum().item()
    for v in range(V):
        for c in range(w):
            up, down = table.clone(), table.clone()
            up[v, c] += h
            down[v, c] -= h
            # y is off by 2 U (|table| + h) 1.5 in each of at most T terms on either side, the table's own steps likewise
            room = T * 8 * U * 4 * 1.5 * dy.abs().max().item() / (2 * h) + (T + 2) * U * 1.5 * dy.abs().sum().item()
            assert math.isclose((f(up) - f(down)) / (up[v, c] - down[v, c]).double().item(), d[v, c].item(), abs_tol=room)
