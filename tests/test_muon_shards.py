"""Stage.muon() over a stage of a tensor-parallel group, which holds shards of its matrices."""
import pytest
import torch

import paper_2512_20953_amd as P


def test_a_shards_factor_is_asked_for():
    stage = P.Stage.__new__(P.Stage)                   # (the configuration alone: nothing else is looked at)
    stage.cfg = P.StageConfig.make(tp=2)
    for call in (lambda: stage.muon(), lambda: stage.muon(0.1, scale=1.0), lambda: stage.muon(shards=False)):
        with pytest.raises(P.AhError, match="shard"):
            call()


@pytest.mark.gpu
def test_shards_step_as_matrices_of_their_own():
    stage = P.Stage(P.StageConfig.make(n_layers=1, hidden=512, n_heads=8, head_dim=64, ffn=1024, tp=2))
    with pytest.raises(P.AhError, match="shard"):
        stage.muon()
    opt = stage.muon(shards=True, weight_decay=0.0, scale=1.0)
    # query, key and value blocks and the first MLP matrix of half the columns, the other two of half the rows
    assert [tuple(p.shape) for p in opt.params] == [(512, 256)] * 3 + [(256, 512), (512, 512), (512, 512)]
    gen = torch.Generator(device="cuda").manual_seed(1)
    stage.grads.normal_(generator=gen)
    single = P.Muon([torch.zeros(512, 256, dtype=torch.bfloat16, device="cuda")], [opt.grads[1].contiguous()], scale=1.0)
    opt.step(1.0)
    single.step(1.0)
    # the same formula whatever stands beside it; 2^-8: bf16's steps, 4e-3: of the products' operands in either group
    assert torch.linalg.matrix_norm(opt.params[1].double() - single.params[0].double()) <= (2 ** -8 + 8e-3) * torch.linalg.matrix_norm(single.params[0].double())
