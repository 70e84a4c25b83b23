"""Calls that Muon, the embedding, the layer norm and the loss refuse, through the C ABI with made-up addresses (nothing is launched) and through the binding."""
import ctypes as C

import pytest
import torch

import paper_2512_20953_amd as P
from paper_2512_20953_amd import binding as B

OK, EINVAL, EUNSUPPORTED = 0, 1, 5
NAN, INF = float("nan"), float("inf")


def _embedding(**kw):
    c = dict(struct_size=B._EMBED_SIZE, rows=10, vocab=20, width=16, token_bits=64, scale=1.0)
    return B._EmbeddingConfig(**{**c, **kw})


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=8), EINVAL), (dict(rows=-1), EINVAL), (dict(vocab=0), EINVAL), (dict(width=0), EINVAL), (dict(rows=(1 << 25) + 1), EUNSUPPORTED),
    (dict(vocab=(1 << 30) + 1), EUNSUPPORTED), (dict(width=65537), EUNSUPPORTED), (dict(table_type=2), EINVAL), (dict(act_type=-1), EINVAL), (dict(token_bits=16), EINVAL),
    (dict(scale=NAN), EINVAL), (dict(scale=INF), EINVAL), (dict(ld_table=15), EINVAL), (dict(ld_act=15), EINVAL), (dict(ld_act=-16), EINVAL), (dict(ld_table=(1 << 31) + 1), EINVAL)])
def test_embedding_configurations(kw, status):
    c = _embedding(**kw)
    assert B.lib.ah_embedding_fwd(C.byref(c), 256, 256, 256, None) == status
    assert B.lib.ah_embedding_bwd(C.byref(c), 256, 256, 256, 0, 256, None) == status


@pytest.mark.parametrize("kw", [dict(n_pos=0), dict(n_pos=9), dict(n_pos=10, seq_len=0), dict(n_pos=10, ld_pos=8), dict(n_pos=10, pos_table=257), dict(n_pos=10, positions=258)])
def test_embedding_positions(kw):
    c = _embedding(**{**dict(pos_table=256, seq_len=100), **kw})
    assert B.lib.ah_embedding_fwd(C.byref(c), 256, 256, 256, None) == EINVAL


def test_embedding_pointers_and_nothing_to_do():
    fwd, bwd, c = B.lib.ah_embedding_fwd, B.lib.ah_embedding_bwd, _embedding()
    for k in range(3):
        for bad in (None, 257):
            assert fwd(C.byref(c), *[bad if i == k else 256 for i in range(3)], None) == EINVAL
            assert bwd(C.byref(c), *[bad if i == k else 256 for i in range(3)], 0, 256, None) == EINVAL
    assert bwd(C.byref(c), 256, 256, 256, 2, 256, None) == EINVAL
    for work in (None, 264):
        assert bwd(C.byref(c), 256, 256, 256, 0, work, None) == EINVAL
    assert fwd(C.byref(_embedding(rows=0)), None, None, None, None) == OK
    assert bwd(C.byref(_embedding(rows=0)), None, None, 256, 1, 256, None) == OK
    assert fwd(None, 256, 256, 256, None) == bwd(None, 256, 256, 256, 0, 256, None) == EINVAL
    assert B.lib.ah_embedding_bwd_workspace(C.byref(c), None) == EINVAL


def _norm(**kw):
    c = dict(struct_size=B._NORM_SIZE, rows=10, width=16, eps=1e-5, gain=256, bias=256)
    return B._LayerNormConfig(**{**c, **kw})


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=8), EINVAL), (dict(rows=-1), EINVAL), (dict(width=0), EINVAL), (dict(width=16385), EUNSUPPORTED), (dict(rows=(1 << 25) + 1), EUNSUPPORTED), (dict(rms=2), EINVAL),
    (dict(act_type=2), EINVAL), (dict(param_type=2), EINVAL), (dict(eps=0.0), EINVAL), (dict(eps=1e-39), EINVAL), (dict(eps=NAN), EINVAL), (dict(eps=INF), EINVAL),
    (dict(gain=257), EINVAL), (dict(bias=258, param_type=1), EINVAL), (dict(ld_x=15), EINVAL), (dict(ld_y=15), EINVAL), (dict(ld_dx=15), EINVAL)])
def test_layer_norm_configurations(kw, status):
    c = _norm(**kw)
    assert B.lib.ah_layer_norm_fwd(C.byref(c), 256, 256, None) == status
    assert B.lib.ah_layer_norm_bwd(C.byref(c), 256, 256, 256, 256, 256, 0, 256, None) == status


def test_layer_norm_pointers_places_and_nothing_to_do():
    fwd, bwd, c = B.lib.ah_layer_norm_fwd, B.lib.ah_layer_norm_bwd, _norm()
    for k in range(2):
        assert fwd(C.byref(c), *[None if i == k else 256 for i in range(2)], None) == fwd(C.byref(c), *[257 if i == k else 256 for i in range(2)], None) == EINVAL
    for k in range(3):
        for bad in (None, 257):
            assert bwd(C.byref(c), *[bad if i == k else 256 for i in range(3)], 256, 256, 0, 256, None) == EINVAL
    for dg, db, beta, work in ((258, 256, 0, 256), (256, 258, 0, 256), (256, 256, 2, 256), (256, 256, 0, None), (256, 256, 0, 264)):
        assert bwd(C.byref(c), 256, 256, 256, dg, db, beta, work, None) == EINVAL
    assert fwd(C.byref(_norm(ld_x=24)), 256, 256, None) == bwd(C.byref(_norm(ld_dx=24)), 256, 512, 256, 256, 256, 0, 256, None) == EINVAL
    assert bwd(C.byref(_norm(ld_y=24)), 512, 256, 256, 256, 256, 0, 256, None) == EINVAL
    assert fwd(C.byref(_norm(rows=0)), None, None, None) == OK
    assert fwd(None, 256, 256, None) == B.lib.ah_layer_norm_bwd_workspace(C.byref(c), None) == EINVAL


def _loss(**kw):
    c = dict(struct_size=B._LOSS_SIZE, rows=10, vocab=16, target_bits=64, scale=1.0)
    return B._CrossEntropyConfig(**{**c, **kw})


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=8), EINVAL), (dict(rows=-1), EINVAL), (dict(vocab=0), EINVAL), (dict(rows=(1 << 25) + 1), EUNSUPPORTED), (dict(vocab=(1 << 24) + 1), EUNSUPPORTED),
    (dict(act_type=2), EINVAL), (dict(target_bits=8), EINVAL), (dict(scale=NAN), EINVAL), (dict(scale_dev=258), EINVAL), (dict(ld_logits=15), EINVAL), (dict(ld_grad=15), EINVAL)])
def test_cross_entropy_configurations(kw, status):
    assert B.lib.ah_cross_entropy(C.byref(_loss(**kw)), 256, 256, 256, 512, None) == status


def test_cross_entropy_pointers_and_nothing_to_do():
    f, c = B.lib.ah_cross_entropy, _loss()
    for k in range(3):
        for bad in (None, 257):
            assert f(C.byref(c), *[bad if i == k else 256 for i in range(3)], 512, None) == EINVAL
    assert f(C.byref(c), 256, 256, 256, 257, None) == EINVAL
    assert f(C.byref(_loss(ld_logits=24)), 256, 256, 256, 256, None) == f(C.byref(_loss(ld_grad=24)), 256, 256, 256, 256, None) == EINVAL
    assert f(C.byref(_loss(rows=0)), None, None, None, None, None) == OK
    assert f(None, 256, 256, 256, None, None) == EINVAL


def _muon(c=None, **kw):
    cfg = B._MuonConfig(**{**dict(struct_size=C.sizeof(B._MuonConfig), nesterov=1, ns_steps=5, lr=0.1, momentum=0.9, eps=1e-7), **(c or {})})
    m = B._MuonMatrix(**{**dict(param=256, grad=256, momentum=256, rows=8, cols=16, scale=1.0), **kw})
    return B.lib.ah_muon_step(C.byref(cfg), C.byref(m), 1, 256, None)


@pytest.mark.parametrize("kw", [
    dict(struct_size=8), dict(param_type=2), dict(grad_type=2), dict(nesterov=2), dict(ns_steps=0), dict(ns_steps=33), dict(lr=-1.0), dict(lr=NAN), dict(momentum=1.0),
    dict(momentum=-0.1), dict(eps=0.0), dict(eps=1e-38), dict(eps=INF), dict(lr_dev=258), dict(grad_norm=258)])
def test_muon_configurations(kw):
    assert _muon(kw) == EINVAL


@pytest.mark.parametrize("kw,status", [
    (dict(param=None), EINVAL), (dict(grad=None), EINVAL), (dict(momentum=None), EINVAL), (dict(param=257), EINVAL), (dict(momentum=258), EINVAL), (dict(master=258), EINVAL),
    (dict(rows=-1), EINVAL), (dict(cols=-1), EINVAL), (dict(rows=32769, cols=40000), EUNSUPPORTED), (dict(cols=131073), EUNSUPPORTED), (dict(ld_param=15), EINVAL),
    (dict(ld_grad=15), EINVAL), (dict(ld_momentum=15), EINVAL), (dict(ld_master=15), EINVAL), (dict(weight_decay=NAN), EINVAL), (dict(scale=INF), EINVAL)])
def test_muon_matrices(kw, status):
    assert _muon(**kw) == status


def test_muon_lists():
    assert _muon(dict(param_type=1), master=256) == EINVAL
    assert _muon(rows=0) == _muon(cols=0) == OK        # nothing to do
    cfg = B._MuonConfig(struct_size=C.sizeof(B._MuonConfig), nesterov=1, ns_steps=5, lr=0.1, momentum=0.9, eps=1e-7)
    m = B._MuonMatrix(param=256, grad=256, momentum=256, rows=8, cols=16, scale=1.0)
    two = (B._MuonMatrix * 2)(m, B._MuonMatrix(param=256, grad=256, momentum=256, master=256, rows=8, cols=16, scale=1.0))
    assert B.lib.ah_muon_step(C.byref(cfg), two, 2, 256, None) == EINVAL                   # a master copy for one of them
    assert B.lib.ah_muon_step(C.byref(cfg), C.byref(m), -1, 256, None) == B.lib.ah_muon_step(C.byref(cfg), None, 1, 256, None) == EINVAL
    assert B.lib.ah_muon_step(C.byref(cfg), C.byref(m), 1, None, None) == B.lib.ah_muon_step(C.byref(cfg), C.byref(m), 1, 264, None) == EINVAL
    assert B.lib.ah_muon_step(None, C.byref(m), 1, 256, None) == B.lib.ah_muon_workspace(C.byref(m), 1, None) == EINVAL


def test_muon_workspace_is_that_of_its_largest_group():
    def need(*shapes):
        n = C.c_uint64()
        assert B.lib.ah_muon_workspace((B._MuonMatrix * len(shapes))(*[B._MuonMatrix(rows=r, cols=c) for r, c in shapes]), len(shapes), n) == OK
        return n.value
    one = need((4096, 11008))
    assert one >= 6 * 4096 * 11008 + 4 * 4096 ** 2 and need((11008, 4096)) == one
    assert need((4096, 11008), (4096, 11008)) > 1.9 * one
    assert need(*[(4096, 11008)] * 40) == need(*[(4096, 11008)] * 5)       # 2^28 elements at a time
    assert need((0, 5)) == 256 and need(*[(8, 8)] * 1000) == need(*[(8, 8)] * 24)


@pytest.mark.parametrize("call", [
    lambda: P.embedding_bwd_workspace(2 ** 32 + 5, 10, 8), lambda: P.embedding_bwd_workspace(5, 2 ** 32 + 10, 8), lambda: P.embedding_bwd_workspace(5, 10, 2 ** 32 + 8),
    lambda: P.embedding_bwd_workspace(-2 ** 32 + 5, 10, 8), lambda: P.layer_norm_bwd_workspace(2 ** 32 + 5, 8), lambda: P.layer_norm_bwd_workspace(5, 2 ** 32 + 8),
    lambda: P.grad_norm_workspace(-1)])
def test_sizes_that_the_fields_do_not_hold(call):
    with pytest.raises(P.AhError):
        call()


def test_tensors_of_the_host_are_refused():
    z, t, i = torch.zeros(4, 8), torch.zeros(4), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: P.embedding_fwd(z, i, z), lambda: P.embedding_bwd(i, z, z, t), lambda: P.layer_norm_fwd(z, None, None, z), lambda: P.layer_norm_bwd(z, None, z, z, t, t, t),
                 lambda: P.cross_entropy(z, i, t), lambda: P.Muon([z], [z.clone()]), lambda: P.grad_norm([z], t, t)):
        with pytest.raises(P.AhError, match="device"):
            call()


@pytest.mark.parametrize("written,read,ok", [
    ([(0, 4, 8, 8), (32, 4, 8, 8)], [], True), ([(0, 4, 8, 8), (24, 4, 8, 8)], [], False),
    ([(0, 4, 8, 32), (8, 4, 8, 32), (16, 4, 16, 32)], [], True),          # columns beside each other
    ([(0, 4, 12, 32), (8, 4, 8, 32)], [], False), ([(16, 4, 16, 32), (40, 4, 8, 32)], [], True), ([(16, 4, 16, 32), (24 + 32, 4, 8, 32)], [], False),
    ([(0, 4, 8, 32)], [(0, 4, 8, 32)], False), ([(0, 4, 8, 32)], [(8, 4, 8, 32), (8, 4, 8, 32)], True),
    ([(0, 4, 8, 32), (8, 4, 8, 24)], [], False),                          # rows at other distances: taken for overlapping
    ([(0, 0, 8, 8), (0, 4, 8, 8)], [(4, 4, 0, 8)], True)])
def test_matrices_that_overlap(written, read, ok):
    assert B._matrices_apart(written, read) == ok
