"""Calls at the edges of what the operators of include/ah_ops.h document, through the C ABI with made-up addresses (nothing is launched) and through the binding."""
import ctypes as C

import pytest
import torch

import paper_2512_20953_amd as P
from paper_2512_20953_amd import binding as B

EINVAL = 1


@pytest.mark.parametrize("max_norm", [1e-50, 1e-46, 1e-40])
def test_a_limit_that_fp32_does_not_hold_is_refused(max_norm):
    # (1e-50 rounds to 0, which would stand for no limit; subnormals lose digits of the factor)
    assert B.lib.ah_grad_norm(None, 0, 1, max_norm, 256, 256, None) == EINVAL


@pytest.mark.parametrize("eps", [1e-45, 1e-39])
def test_a_subnormal_epsilon_of_the_norms_is_refused(eps):
    c = B._QkNormConfig(struct_size=C.sizeof(B._QkNormConfig), rows=10, seq_len=5, n_heads=4, n_kv_heads=2, head_dim=64, n_pos=5, eps=eps, gain_q=256, gain_k=256, cos_sin=256)
    assert B.lib.ah_qk_norm_rope_fwd(C.byref(c), None, None, None) == EINVAL
    assert b"eps" in B.lib.ah_last_error()


def test_a_window_that_32_bits_do_not_hold_is_everything():
    most = 2 ** 31 - 1
    for window, sinks in ((2 ** 32 + 5, 0), (2 ** 40, 2 ** 33 + 1), (2 ** 31, 3)):
        c = B._window_config(1, 100, 2, 2, 64, window, sinks)
        assert c.window == most and c.sinks == min(sinks, most)
    c = B._window_config(1, 100, 2, 2, 64, -2 ** 33 + 7, 0)
    assert c.window < 1                                           # refused, not taken for 7


@pytest.mark.parametrize("written,read,ok", [
    ([(0, 8), (8, 16)], [(16, 32)], True),
    ([(0, 8), (0, 8)], [], False),                     # the same tensor twice
    ([(0, 64), (8, 16)], [], False),                   # one inside another
    ([(0, 8)], [(16, 32), (16, 32), (20, 24)], True),  # gradients may be shared
    ([(24, 28)], [(0, 32)], False), ([(0, 32)], [(24, 28)], False), ([(30, 40)], [(0, 32), (8, 12)], False), ([(32, 40)], [(0, 32), (8, 12)], True),
    ([(5, 5), (0, 8)], [(0, 0)], True),                # nothing overlaps nothing
])
def test_tensors_that_overlap(written, read, ok):
    assert B._apart(written, read) == ok


@pytest.mark.gpu
def test_adamw_refuses_tensors_that_overlap():
    n = 256
    f = lambda: torch.zeros(n, device="cuda")          # noqa: E731
    p, q, g = f(), f(), f()
    P.AdamW([p, q], [g, g])                            # the same gradient for both
    for params, grads, kw in (([p, p], [g, g], {}), ([p, p[8:]], [g, g[8:]], {}), ([p], [p], {}), ([p, q], [g, g], dict(m=[q, f()])),
                              ([p], [g], dict(m=[p])), ([p], [g], dict(m=[g])), ([p, q], [g, g], dict(v=[q, f()]))):
        with pytest.raises(P.AhError, match="overlap"):
            P.AdamW(params, grads, **kw)
    m = f()
    with pytest.raises(P.AhError, match="overlap"):
        P.AdamW([p], [g], m=[m], v=[m])


@pytest.mark.gpu
@pytest.mark.parametrize("window,sinks", [(256, 0), (256, 3), (1000, 300)])
def test_a_stage_with_a_window_of_its_whole_sequence_has_causal_attention(window, sinks):
    results = []
    for kw in ({}, dict(attn_window=window, attn_sinks=sinks)):
        cfg = B.StageConfig.make(arch="llama", n_layers=1, hidden=256, n_heads=4, head_dim=64, ffn=512, seq=256, mb=2, qk_norm=1, **kw)
        st = P.Stage(cfg)
        g = torch.Generator().manual_seed(3)
        st.params.copy_((0.04 * torch.randn(st.params.shape, generator=g)).bfloat16())
        x, dy = (torch.randn(512, 256, generator=g).bfloat16().cuda() for _ in range(2))
        y, dx = torch.empty_like(x), torch.empty_like(x)
        st.forward(0, x, y)
        st.zero_grads()
        st.backward(0, dy, dx)
        torch.cuda.synchronize()
        results.append((y.cpu(), dx.cpu(), st.grads.cpu().clone()))
    for a, b in zip(*results):
        assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("n_seq,S,W,d", [(7, 1, 123, 64), (3, 1, 4, 128), (2, 200, 1, 64), (1, 130, 1, 128)])
def test_a_query_that_sees_itself_alone_has_no_gradient(n_seq, S, W, d):
    """P = 1, o = v, so that dS = dO v - sum(o dO) is 0: what is left is the rounding of two fp32 sums of d products, each at most d 2^-24 of the sum of their
    magnitudes; P is 1 within 2^-10 (the exponent's argument, below 2^7 in magnitude, is formed from three roundings), dS is rounded by 2^-8 more, and a key has 3 queries: 2 covers both factors."""
    nh, nk, T = 9, 3, n_seq * S
    g = torch.Generator().manual_seed(S + d)
    q, k, v, do = (torch.randn(T, n * d, generator=g).bfloat16().cuda() for n in (nh, nk, nk, nh))
    o, lse = torch.empty_like(q), torch.empty(n_seq, nh, S, device="cuda")
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    work = torch.empty(P.attention_window_bwd_workspace(n_seq, S, nh, nk, d, W), dtype=torch.uint8, device="cuda")
    P.attention_window_fwd(q, k, v, o, lse, n_seq, S, nh, nk, d, W)
    P.attention_window_bwd(q, k, v, o, lse, do, dq, dk, dv, work, n_seq, S, nh, nk, d, W)
    heads = lambda t, n: t.double().cpu().reshape(T, n, d)                    # noqa: E731
    assert torch.equal(heads(o, nh), heads(v, nk).repeat_interleave(nh // nk, 1))
    room = 2 * 2 * d * 2.0 ** -24 * (heads(o, nh) * heads(do, nh)).abs().sum(-1, keepdim=True) / d ** 0.5
    assert (heads(dq, nh).abs() <= room * heads(k, nk).repeat_interleave(nh // nk, 1).abs()).all()
    assert (heads(dk, nk).abs() <= (room * heads(q, nh).abs()).reshape(T, nk, nh // nk, d).sum(2)).all()
