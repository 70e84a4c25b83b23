"""Arguments of the binding that the library's fields, or their types, do not hold: none may be taken for another one."""
import pytest

import paper_2512_20953_amd as P
from paper_2512_20953_amd import binding as B


def _stage(**kw):
    return B.StageConfig.make(**{**dict(arch="llama", n_layers=1, hidden=256, n_heads=4, head_dim=64, ffn=384, seq=256, mb=1), **kw})


@pytest.mark.parametrize("window,sinks", [(2 ** 32 + 5, 0), (2 ** 40, 2 ** 33 + 1), (2 ** 31, 3), (2 ** 63, 2 ** 63)])
def test_a_stage_window_that_32_bits_do_not_hold_is_everything(window, sinks):
    c = _stage(attn_window=window, attn_sinks=sinks)
    assert c.attn_window == 2 ** 31 - 1 and c.attn_sinks == min(sinks, 2 ** 31 - 1)
    assert B.query_sizes(c) == B.query_sizes(_stage())


def test_a_stage_window_below_zero_is_refused():
    for kw in (dict(attn_window=-2 ** 33 + 7), dict(attn_window=7, attn_sinks=-2 ** 33 + 7)):
        with pytest.raises(P.AhError):
            B.query_sizes(_stage(**kw))


@pytest.mark.parametrize("kw", [dict(n_seq=2 ** 32 + 1), dict(seq_len=2 ** 32 + 64), dict(nh=2 ** 32 + 4, nh_kv=2 ** 32 + 4), dict(d=2 ** 32 + 64), dict(seq_len=-2 ** 32 + 64)])
def test_windowed_attention_refuses_sizes_that_its_fields_do_not_hold(kw):
    with pytest.raises(P.AhError):
        P.attention_window_bwd_workspace(**{**dict(n_seq=1, seq_len=64, nh=4, nh_kv=4, d=64, window=8, sinks=2), **kw})


@pytest.mark.parametrize("kw", [dict(rows=2 ** 32 + 5), dict(rows=-2 ** 32 + 5), dict(nh=2 ** 32 + 5), dict(nh_kv=2 ** 32 + 5), dict(d=2 ** 32 + 64)])
def test_norms_refuse_sizes_that_their_fields_do_not_hold(kw):
    with pytest.raises(P.AhError):
        P.qk_norm_rope_bwd_workspace(**{**dict(rows=5, nh=2, nh_kv=2, d=64), **kw})


@pytest.mark.gpu
@pytest.mark.parametrize("seq_len", [2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 63])
def test_a_sequence_longer_than_all_rows_has_their_positions(seq_len):
    import torch
    T, d = 20, 64
    g = torch.Generator().manual_seed(1)
    x = torch.randn(T, 2 * d, generator=g).bfloat16().cuda()
    gain = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    table = torch.empty(T, d // 2, 2, device="cuda")
    P.rope_table(table, d)
    y, want = torch.empty_like(x), torch.empty_like(x)
    P.qk_norm_rope_fwd(x, gain, gain, table, want, T, 1, 1, d)
    P.qk_norm_rope_fwd(x, gain, gain, table, y, seq_len, 1, 1, d)
    assert torch.equal(y, want)


@pytest.mark.gpu
@pytest.mark.parametrize("beta", [0.5, 0.99, -0.5, 2, 2 ** 32, float("nan")])
def test_norms_add_to_their_gains_gradients_or_not(beta):
    import torch
    T, d = 4, 64
    x = torch.ones(T, 2 * d, dtype=torch.bfloat16, device="cuda")
    gain = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    dx, dg = torch.full_like(x, 7), torch.full((2, d), 3.0, device="cuda")
    work = torch.empty(P.qk_norm_rope_bwd_workspace(T, 1, 1, d), dtype=torch.uint8, device="cuda")
    with pytest.raises(P.AhError):
        P.qk_norm_rope_bwd(x, gain, gain, None, x, dx, dg[0], dg[1], work, T, 1, 1, d, beta=beta)
    assert (dx == 7).all() and (dg == 3).all()


def test_norms_in_place_go_row_for_row():
    """Rows written at another distance than they are read would overwrite rows that are still to be read (made-up addresses: a call that is not refused reaches no device here)."""
    c = dict(struct_size=B._QK_SIZE, rows=10, seq_len=5, n_heads=4, n_kv_heads=2, head_dim=64, n_pos=5, eps=1e-6, gain_q=256, gain_k=256)
    fwd = lambda **kw: B.lib.ah_qk_norm_rope_fwd(B._QkNormConfig(**c, **kw), 256, 256, None)  # noqa: E731
    bwd = lambda x, dy, dx, **kw: B.lib.ah_qk_norm_rope_bwd(B._QkNormConfig(**c, **kw), x, dy, dx, 256, 256, 0, 256, None)  # noqa: E731
    assert fwd(ld_x=392) == fwd(ld_y=392) == fwd(ld_x=392, ld_y=400) == 1
    assert bwd(256, 512, 256, ld_x=392) == bwd(256, 512, 256, ld_dx=392) == bwd(512, 256, 256, ld_y=392) == bwd(512, 256, 256, ld_dx=392) == 1
    assert b"stride" in B.lib.ah_last_error()
