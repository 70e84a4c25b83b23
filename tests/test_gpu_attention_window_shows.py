"""What is not finite shows in every row that sees it (the other side, that it reaches no others, is in test_gpu_attention_window.py), and an infinitely low score counts as nothing."""
import math

import pytest
import torch

import paper_2512_20953_amd as P
from tests.test_gpu_attention_window import _inputs, _run

pytestmark = pytest.mark.gpu
DEV = "cuda"
CASES = [(300, 700, 60, 2, 64, 2, 1), (5, 700, 60, 8, 128, 2, 2), (127, 400, 1, 0, 64, 3, 1), (64, 333, 130, 70, 128, 2, 1), (0, 200, 200, 0, 64, 2, 2), (199, 200, 50, 3, 128, 4, 2)]


def _sees(S, W, sinks):
    at = torch.arange(S, device=DEV)
    gap = at[:, None] - at
    return (gap >= 0) & ((gap < W) | (at < sinks))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("at,S,W,sinks,d,nh,nkv", CASES)
def test_a_key_or_value_shows_in_the_rows_that_see_it(at, S, W, sinks, d, nh, nkv, bad):
    x = _inputs(S, nh * d, nkv * d, 0, 9)
    rows = _sees(S, W, sinks)[:, at]
    for which in (1, 2):
        y = [t.clone() for t in x]
        y[which][at, :d] = bad                              # of the first key head
        o, lse, dq, dk, dv = _run(*y, 1, S, nh, nkv, d, W, sinks)
        for h in range(nh):
            c = slice(h * d, h * d + d)
            if h < nh // nkv:
                assert not torch.isfinite(o[rows, c].float()).any() and not torch.isfinite(dq[rows, c].float()).any(), (which, h)
                if which == 1:
                    assert not torch.isfinite(lse[0, h, rows]).any()
            else:
                assert torch.isfinite(o[:, c].float()).all() and torch.isfinite(dq[:, c].float()).all()
        assert not torch.isfinite(dk[at, :d].float()).any()             # its own gradient, through the probabilities' sums
        if which == 1:
            assert not torch.isfinite(dv[at, :d].float()).any()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("at,S,W,sinks,d,nh,nkv", CASES)
def test_a_query_or_output_gradient_shows_in_the_keys_that_it_sees(at, S, W, sinks, d, nh, nkv, bad):
    x = _inputs(S, nh * d, nkv * d, 0, 9)
    keys = _sees(S, W, sinks)[at]
    for which in (0, 3):
        y = [t.clone() for t in x]
        y[which][at, :d] = bad
        o, lse, dq, dk, dv = _run(*y, 1, S, nh, nkv, d, W, sinks)
        assert not torch.isfinite(dq[at, :d].float()).any()
        assert not torch.isfinite(dk[keys, :d].float()).any() and not torch.isfinite(dv[keys, :d].float()).any()
        if which == 0:
            assert not torch.isfinite(o[at, :d].float()).any() and not torch.isfinite(lse[0, 0, at])


@pytest.mark.parametrize("at,S,W,sinks,d,nh,nkv", [c for c in CASES if c[2] > 1])
def test_a_score_of_minus_infinity_counts_as_nothing(at, S, W, sinks, d, nh, nkv):
    """One column of a key infinite: where the query's sign makes its score -inf the row is as without that key (first rows, that see no other, apart), else NaN."""
    x = [t.clone() for t in _inputs(S, nh * d, nkv * d, 0, 9)]
    x[1][at, 3] = float("inf")
    o, lse, *_ = _run(*x, 1, S, nh, nkv, d, W, sinks)
    sees = _sees(S, W, sinks)
    rows = sees[:, at]
    for h in range(nh // nkv):
        c = slice(h * d, h * d + d)
        s = (x[0][:, c].double() @ x[1][:, :d].double().T / math.sqrt(d)).masked_fill(~sees, -math.inf)
        low = rows & (s[:, at] == -math.inf) & (sees.sum(1) > 1)
        assert at == S - 1 or low.any()
        p = torch.softmax(s, 1)
        ref, got = p @ x[2][:, :d].double(), o[:, c].double()
        room = 1.02 * 2 ** -8 * (p @ x[2][:, :d].double().abs() + ref.abs())
        assert ((got - ref).abs() <= room)[low].all() and torch.isfinite(lse[0, h, low]).all()
        assert not torch.isfinite(got[rows & ~low]).any()
