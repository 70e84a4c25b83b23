"""The operators around a stage together, as a whole small model trains: embedding -> Stage -> layer norm -> logits of the same table -> loss, all gradients, and the step
(Muon over the stage's matrices, AdamW over everything else).  Against the stage's oracle and plain forms of the ends in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2512_20953_amd as P
from oracle import stage_ref as R
from synth import stage_inputs as SI
from tests import gpu_util as U
from tests.test_gpu_muon import norm, orthogonal, room_of

pytestmark = pytest.mark.gpu
V = 384
MAX_NORM = 0.05


class Model:
    """Buffers of a training step, and the step"""

    def __init__(self, w):
        cfg, self.oracle_cfg = U.make_cfgs(dict(w, n_mb=1))
        self.stage, self.w, self.rms = P.Stage(cfg), w, w["arch"] == "llama"
        self.params = [SI.draw_layer_params(w, l, perturb_vectors=True) for l in range(w["n_layers"])]
        U.load_params(self.stage, self.params)
        h, T = w["hidden"], w["mb"] * w["seq"]
        g = torch.Generator().manual_seed(1)
        bf = lambda *s, std=1.0, mean=0.0: (torch.randn(*s, generator=g) * std + mean).bfloat16().cuda()   # noqa: E731
        self.scale = 1.0 if not self.rms else h ** 0.5
        self.table, self.pos = bf(V, h, std=1.0 / self.scale), None if self.rms else bf(w["seq"], h, std=0.5)
        self.gain, self.bias = bf(h, std=0.2, mean=0.3), None if self.rms else bf(h, std=0.2)
        self.tokens = torch.randint(0, V, (T,), generator=g).cuda()
        self.targets = torch.randint(0, V, (T,), generator=g).cuda()
        self.tokens[::17] = -1
        self.targets[::17] = -1
        self.live = int((self.targets >= 0).sum())
        rows = lambda n=h: torch.empty(T, n, dtype=torch.bfloat16, device="cuda")   # noqa: E731
        self.x, self.y, self.n, self.logits, self.dn, self.dy, self.dx = rows(), rows(), rows(), rows(V), rows(), rows(), rows()
        self.loss = torch.empty(T, device="cuda")
        f = lambda t: None if t is None else torch.full(t.shape, float("nan"), device="cuda")   # noqa: E731
        self.d_table, self.d_pos, self.d_gain, self.d_bias = f(self.table), f(self.pos), f(self.gain), f(self.bias)
        self.positions = (torch.arange(T) % w["seq"]).int().cuda()
        byte = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")   # noqa: E731
        self.work_e, self.work_p, self.work_n = byte(P.embedding_bwd_workspace(T, V, h)), byte(P.embedding_bwd_workspace(T, w["seq"], h)), byte(P.layer_norm_bwd_workspace(T, h))
        ends = [(p, d) for p, d in ((self.table, self.d_table), (self.pos, self.d_pos), (self.gain, self.d_gain), (self.bias, self.d_bias)) if p is not None]
        self.muon, self.vectors = self.stage.muon(master=True), self.stage.adamw(matrices=False)
        self.ends = P.AdamW([p for p, _ in ends], [d for _, d in ends])
        self.all_grads = [self.stage.grads] + [d for _, d in ends]
        self.norm, self.work_g = torch.empty(2, device="cuda"), byte(P.grad_norm_workspace(len(self.all_grads)))

    def gradients(self, s=None):
        eps = 1e-6 if self.rms else 1e-5
        P.embedding_fwd(self.table, self.tokens, self.x, scale=self.scale, pos_table=self.pos, seq_len=self.w["seq"], stream=s)
        self.stage.forward(0, self.x, self.y, s)
        P.layer_norm_fwd(self.y, self.gain, self.bias, self.n, eps=eps, rms=self.rms, stream=s)
        P.gemm_nt(self.n, self.table, self.logits, stream=s)
        P.cross_entropy(self.logits, self.targets, self.loss, self.logits, scale=1.0 / self.live, stream=s)     # the gradient takes the logits' place
        P.gemm_nn(self.logits, self.table, None, self.dn, stream=s)
        P.gemm_tn(self.logits, self.n, self.d_table, 0, stream=s)
        P.layer_norm_bwd(self.y, self.gain, self.dn, self.dy, self.d_gain, self.d_bias, self.work_n, eps=eps, rms=self.rms, stream=s)
        self.stage.zero_grads(s)
        self.stage.backward(0, self.dy, self.dx, s)
        P.embedding_bwd(self.tokens, self.dx, self.d_table, self.work_e, scale=self.scale, beta=1, stream=s)
        if self.pos is not None:
            P.embedding_bwd(self.positions, self.dx, self.d_pos, self.work_p, stream=s)

    def step(self, k, s=None):
        P.grad_norm(self.all_grads, self.norm, self.work_g, MAX_NORM, stream=s)
        self.muon.step(0.01, grad_norm=self.norm, stream=s)
        self.vectors.step(0.01, k, grad_norm=self.norm, stream=s)
        self.ends.step(0.01, k, grad_norm=self.norm, stream=s)

    def state(self):
        return [self.stage.params, self.table, self.gain] + [t for t in (self.pos, self.bias) if t is not None] + self.muon.m + self.muon.master + self.ends.m + self.vectors.v


def in_64_bits(m):
    """(loss of every row, gradients) through the oracle and plain forms"""
    t = lambda x: None if x is None else x.double().cpu()   # noqa: E731
    table, pos, gain, bias = t(m.table), t(m.pos), t(m.gain), t(m.bias)
    tok, tgt = m.tokens.cpu(), m.targets.cpu()
    on, ok = (tok >= 0)[:, None], tgt >= 0
    x = torch.where(on, table[tok.clamp_min(0)], 0.0) * m.scale
    if pos is not None:
        x = x + pos[m.positions.cpu().long()]
    ps = [{k: v.astype(np.float64) for k, v in p.items()} for p in m.params]
    y, caches, _ = R.stage_fwd(m.oracle_cfg, ps, x.numpy())
    leaves = [v.clone().requires_grad_() for v in (torch.from_numpy(y), gain, table)] + [None if bias is None else bias.clone().requires_grad_()]
    yy, g, e, b = leaves
    d = yy if m.rms else yy - yy.mean(1, keepdim=True)
    n = d * (d.square().mean(1, keepdim=True) + (1e-6 if m.rms else 1e-5)).rsqrt() * g + (0 if b is None else b)
    loss = torch.where(ok, -torch.log_softmax(n @ e.T, 1).gather(1, tgt.clamp_min(0)[:, None])[:, 0], 0.0)
    (loss.sum() / m.live).backward()
    grads = R.zero_grads_like(ps)
    dx = torch.from_numpy(R.stage_bwd(m.oracle_cfg, ps, caches, yy.grad.numpy(), grads))
    d_table = e.grad.index_add(0, tok.clamp_min(0), torch.where(on, dx, 0.0) * m.scale)
    out = {"table": d_table, "gain": g.grad, "dx": dx}
    if b is not None:
        out |= {"bias": b.grad, "pos": torch.zeros_like(pos).index_add(0, m.positions.cpu().long(), dx)}
    return loss.detach(), out, grads


@pytest.mark.parametrize("arch", ["gpt", "llama"])
def test_gradients_of_a_whole_model(arch):
    w = dict(SI.WORKLOADS["tiny"], arch=arch, ffn=1024)
    m = Model(w)
    m.gradients()
    loss, ends, grads = in_64_bits(m)
    # the stage's own gates: its activations and gradients in bf16; the loss follows the logits, which are rounded like any other activation
    assert U.rel_l2(m.loss.double().cpu(), loss) <= U.ACT_TOL
    for name, got in (("table", m.d_table), ("gain", m.d_gain), ("bias", m.d_bias), ("pos", m.d_pos), ("dx", m.dx)):
        if got is not None:
            assert U.rel_l2(got.double().cpu(), ends[name]) <= U.GRAD_TOL, name
    for l, layer in enumerate(grads):
        for name, ref in layer.items():
            assert U.rel_l2(m.stage.grad_view(l, name).double().cpu().reshape(ref.shape), ref) <= U.GRAD_TOL, (l, name)


@pytest.mark.parametrize("arch", ["gpt", "llama"])
def test_a_step_of_all_optimizers(arch):
    m = Model(dict(SI.WORKLOADS["tiny"], arch=arch, ffn=1024))
    m.gradients()
    before = {(l, n): m.stage.param_view(l, n).clone() for l in range(2) for n in ("wqkv", "wo", "w1", "w2", "ln1_g")}
    m.step(1)
    total = torch.cat([g.double().reshape(-1) for g in m.all_grads]).norm().item()
    assert abs(m.norm[0].item() / total - 1) <= 2.0 ** -23
    assert len(m.muon.params) == 2 * (7 if arch == "llama" else 6)
    k = 0
    for l in range(2):
        for name in ("wqkv", "wo", "w1", "w2"):
            old, g = before[l, name].double(), m.stage.grad_view(l, name).double()
            blocks = 3 if name == "wqkv" else 2 if arch == "llama" and name == "w1" else 1
            for a, u in zip(old.split(old.shape[1] // blocks, 1), g.split(old.shape[1] // blocks, 1)):
                x, rounded = orthogonal(u * m.norm[1].double().item() * 0.0975)
                by = 0.01 * 0.2 * max(a.shape) ** 0.5
                assert norm(m.muon.master[k].double() - (a * (1 - 0.001) - by * x)) <= by * (room_of(x, rounded) + 2.0 ** -12 * norm(x)) + 2.0 ** -22 * norm(a), (l, name)
                assert torch.equal(m.muon.params[k], m.muon.master[k].bfloat16())
                k += 1
        assert not torch.equal(before[l, "ln1_g"], m.stage.param_view(l, "ln1_g"))
    assert k == len(m.muon.params)


@pytest.mark.parametrize("arch", ["gpt", "llama"])
def test_captured_training_steps(arch):
    w = dict(SI.WORKLOADS["tiny"], arch=arch, ffn=1024)
    eager, graphed = Model(w), Model(w)
    s = torch.cuda.Stream()
    graphed.gradients(s)                               # creates what the library keeps, outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        graphed.gradients(s)
        P.grad_norm(graphed.all_grads, graphed.norm, graphed.work_g, MAX_NORM, stream=s)
        graphed.muon.step(0.01, grad_norm=graphed.norm, stream=s)
    for rep in range(3):
        graph.replay()
        torch.cuda.synchronize()
        eager.gradients()
        P.grad_norm(eager.all_grads, eager.norm, eager.work_g, MAX_NORM)
        eager.muon.step(0.01, grad_norm=eager.norm)
        torch.cuda.synchronize()
        for a, b in zip(eager.state() + eager.all_grads + [eager.loss], graphed.state() + graphed.all_grads + [graphed.loss]):
            assert torch.equal(a, b), rep
    del graph
    torch.cuda.synchronize()
