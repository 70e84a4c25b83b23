"""Calls that the operators of include/ah_ops.h refuse, through the C ABI with made-up addresses (nothing is launched) and through the binding."""
import ctypes as C

import pytest
import torch

import paper_2512_20953_amd as P
from paper_2512_20953_amd import binding as B

OK, EINVAL, EUNSUPPORTED = 0, 1, 5


def _window(**kw):
    c = dict(struct_size=C.sizeof(B._WindowConfig), n_seq=2, seq_len=100, n_heads=4, n_kv_heads=2, head_dim=64, window=8, sinks=2)
    return B._WindowConfig(**{**c, **kw})


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=8), EINVAL), (dict(head_dim=96), EUNSUPPORTED), (dict(n_seq=0), EINVAL), (dict(seq_len=0), EINVAL), (dict(n_kv_heads=3), EINVAL),
    (dict(n_kv_heads=0), EINVAL), (dict(window=0), EINVAL), (dict(sinks=-1), EINVAL), (dict(rows=199), EINVAL), (dict(rows=-1), EINVAL),
    (dict(offsets=256), EINVAL), (dict(offsets=258, rows=10), EINVAL), (dict(ld_q=255), EINVAL), (dict(ld_q=260), EINVAL), (dict(ld_k=120), EINVAL),
    (dict(ld_o=1 << 24), EINVAL), (dict(seq_len=1 << 25), EUNSUPPORTED), (dict(n_seq=1 << 20, seq_len=4096), EUNSUPPORTED)])
def test_window_configurations(kw, status):
    c = _window(**kw)
    assert B.lib.ah_attention_window_fwd(C.byref(c), 256, 256, 256, 256, 256, None) == status
    assert B.lib.ah_attention_window_bwd(C.byref(c), *[256] * 10, None) == status


def test_window_pointers():
    c = _window()
    for k in range(5):
        for bad in (None, 264 if k < 4 else 258):
            assert B.lib.ah_attention_window_fwd(C.byref(c), *[bad if i == k else 256 for i in range(5)], None) == EINVAL
    for k in range(10):
        for bad in (None, 258):
            assert B.lib.ah_attention_window_bwd(C.byref(c), *[bad if i == k else 256 for i in range(10)], None) == EINVAL
    assert B.lib.ah_attention_window_bwd(C.byref(c), *[256] * 9, 272, None) == EINVAL       # a workspace is 256-byte aligned
    assert B.lib.ah_attention_window_bwd(C.byref(_window(ld_dv=136 - 1)), *[256] * 10, None) == EINVAL
    assert B.lib.ah_attention_window_fwd(None, 256, 256, 256, 256, 256, None) == EINVAL
    assert B.lib.ah_attention_window_bwd_workspace(C.byref(c), None) == EINVAL


def test_window_workspace_holds_row_sums_and_the_shares_of_the_first_keys():
    n = lambda **kw: P.attention_window_bwd_workspace(**{**dict(n_seq=2, seq_len=100, nh=4, nh_kv=2, d=64, window=8, sinks=0), **kw})  # noqa: E731
    sums = 2 * ((2 * 4 * 100 * 4 + 255) // 256 * 256)
    shares = n() - sums                                                    # a launch that small shares each key block's walk: [sequence, key head][share][100 keys]...
    assert shares > 0 and shares % (2 * 2 * 100 * 2 * 64 * 4) == 0
    assert n(n_seq=300) == 2 * 300 * 4 * 100 * 4   # ... one that fills the chip does not
    far = n(seq_len=4000, sinks=4) - n(seq_len=4000)
    assert far > 0 and far % (2 * 2 * 4 * 2 * 64 * 4) == 0                 # [sequence, key head][share][4 keys][dk, dv][64] fp32
    assert n(seq_len=4000, sinks=4, window=4000) == n(seq_len=4000, window=4000)   # nobody lies behind the window
    with pytest.raises(P.AhError):
        n(d=80)


def _qk(**kw):
    c = dict(struct_size=C.sizeof(B._QkNormConfig), rows=10, seq_len=5, n_heads=4, n_kv_heads=2, head_dim=64, n_pos=5, eps=1e-6, gain_q=256, gain_k=256, cos_sin=256)
    return B._QkNormConfig(**{**c, **kw})


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=8), EINVAL), (dict(head_dim=32), EUNSUPPORTED), (dict(rows=-1), EINVAL), (dict(rows=(1 << 25) + 1), EUNSUPPORTED),
    (dict(n_heads=0, n_kv_heads=0), EINVAL), (dict(n_heads=-1), EINVAL), (dict(eps=0.0), EINVAL), (dict(eps=float("nan")), EINVAL),
    (dict(gain_q=None), EINVAL), (dict(gain_k=None), EINVAL), (dict(gain_q=264), EINVAL), (dict(cos_sin=264), EINVAL), (dict(positions=258), EINVAL),
    (dict(ld_x=376), EINVAL), (dict(ld_x=388), EINVAL), (dict(n_pos=0), EINVAL), (dict(n_pos=4), EINVAL), (dict(seq_len=0), EINVAL)])
def test_qk_norm_configurations(kw, status):
    c = _qk(**kw)
    assert B.lib.ah_qk_norm_rope_fwd(C.byref(c), 256, 256, None) == status
    assert B.lib.ah_qk_norm_rope_bwd(C.byref(c), 256, 256, 256, 256, 256, 0, 256, None) == status


def test_qk_norm_pointers_and_nothing_to_do():
    c = _qk()
    fwd, bwd = B.lib.ah_qk_norm_rope_fwd, B.lib.ah_qk_norm_rope_bwd
    assert fwd(C.byref(c), None, 256, None) == fwd(C.byref(c), 256, 264, None) == EINVAL
    for k in range(5):
        args = [256] * 5
        args[k] = None
        assert bwd(C.byref(c), *args, 0, 256, None) == EINVAL
    assert bwd(C.byref(c), *[256] * 5, 2, 256, None) == EINVAL
    assert bwd(C.byref(c), *[256] * 5, 0, 8, None) == EINVAL
    assert fwd(C.byref(_qk(rows=0)), None, None, None) == OK
    for a in ((256, 0, 64, 1e4), (256, 5, 63, 1e4), (256, 5, 64, 0.0), (None, 5, 64, 1e4), (256, 5, 64, float("inf"))):
        assert B.lib.ah_rope_table(*a, None) == EINVAL


def _adam(**kw):
    c = dict(struct_size=C.sizeof(B._AdamWConfig), param_type=0, grad_type=1, state_bits=32, lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, step=1)
    return B._AdamWConfig(**{**c, **kw})


def _tensor(**kw):
    return (B._AdamWTensor * 1)(B._AdamWTensor(**{**dict(param=256, grad=256, m=256, v=256, n=8), **kw}))


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=8), EINVAL), (dict(param_type=2), EINVAL), (dict(grad_type=-1), EINVAL), (dict(state_bits=16), EUNSUPPORTED), (dict(lr=-1.0), EINVAL),
    (dict(lr=float("nan")), EINVAL), (dict(beta1=1.0), EINVAL), (dict(beta2=-0.1), EINVAL), (dict(eps=0.0), EINVAL), (dict(eps=1e-38), EINVAL), (dict(step=0), EINVAL),
    (dict(lr_dev=258), EINVAL), (dict(step_dev=258), EINVAL), (dict(grad_norm=258), EINVAL)])
def test_adamw_configurations(kw, status):
    assert B.lib.ah_adamw_step(C.byref(_adam(**kw)), _tensor(), 1, None) == status


@pytest.mark.parametrize("kw,cfg,status", [
    (dict(param=None), {}, EINVAL), (dict(grad=None), {}, EINVAL), (dict(m=None), {}, EINVAL), (dict(v=None), {}, EINVAL),
    (dict(), dict(state_bits=8), EINVAL), (dict(m_scale=256), dict(state_bits=8), EINVAL), (dict(param=257), {}, EINVAL), (dict(grad=258), {}, EINVAL),
    (dict(m=258), {}, EINVAL), (dict(master=258), {}, EINVAL), (dict(master=256), dict(param_type=1), EINVAL), (dict(weight_decay=float("inf")), {}, EINVAL),
    (dict(n=(1 << 34) + 1), {}, EUNSUPPORTED)])
def test_adamw_tensors(kw, cfg, status):
    assert B.lib.ah_adamw_step(C.byref(_adam(**cfg)), _tensor(**kw), 1, None) == status


def test_adamw_lists():
    step, norm, values = B.lib.ah_adamw_step, B.lib.ah_grad_norm, B.lib.ah_adamw_state_values
    two = (B._AdamWTensor * 2)(_tensor()[0], _tensor(master=256)[0])
    assert step(C.byref(_adam()), two, 2, None) == EINVAL                 # a master copy for one of them only
    assert step(None, two, 2, None) == step(C.byref(_adam()), None, 1, None) == step(C.byref(_adam()), two, -1, None) == EINVAL
    assert step(C.byref(_adam()), _tensor(n=0, param=None), 1, None) == OK and step(C.byref(_adam()), None, 0, None) == OK
    for a in ((_tensor(grad=None), 1, 1, 1.0, 256, 256), (_tensor(), 1, 2, 1.0, 256, 256), (_tensor(), 1, 1, -1.0, 256, 256),
              (_tensor(), 1, 1, float("nan"), 256, 256), (_tensor(), 1, 1, 1.0, None, 256), (_tensor(), 1, 1, 1.0, 256, 260)):
        assert norm(*a, None) == EINVAL
    out = (C.c_void_p * 1)(256)
    assert values(_tensor(), 1, out, out, None) == EINVAL                 # no scales: not 8-bit states
    assert values(_tensor(m_scale=256, v_scale=256), 1, out, None, None) == EINVAL
    assert values(_tensor(m_scale=256, v_scale=256), 1, out, (C.c_void_p * 1)(257), None) == EINVAL


def test_the_binding_takes_no_host_memory():
    t, f = torch.zeros(4, 256, dtype=torch.bfloat16), torch.zeros(4, 4, 64)
    with pytest.raises(P.AhError, match="not in device memory"):
        P.attention_window_fwd(t, t, t, t, f, 1, 4, 4, 4, 64, 2)
    with pytest.raises(P.AhError, match="not in device memory"):
        P.qk_norm_rope_fwd(t, t[0, :64], t[0, :64], None, t, 4, 2, 2, 64)
    with pytest.raises(P.AhError, match="not in device memory"):
        P.AdamW([f], [f])
    with pytest.raises(P.AhError, match="0 parameters"):
        P.AdamW([], [])
    with pytest.raises(P.AhError, match="state_bits"):
        P.AdamW([f], [f], state_bits=4)
