"""Stages with a sliding window, visible first tokens and normed heads, and whole training iterations with the optimizer: the operators of ah_ops.h as
a stage uses them, against the layer's definition in 64 bits (autograd on the CPU).

Tolerances as for the other stages (normalised L2: activations 2e-2, gradients 3e-2, every tensor): the options add a rounding or two of 2^-8 per
element at most to the dozen that a layer has."""
import ctypes as C
import math

import pytest
import torch

import paper_2512_20953_amd as P
from paper_2512_20953_amd.binding import StageConfig, query_sizes
from tests import gpu_util as U

BASE = dict(n_layers=2, hidden=256, n_heads=4, head_dim=64, ffn=384, seq=256, mb=2)
NAMES = {"gpt": ["ln1_g", "ln1_b", "wqkv", "bqkv", "wo", "bo", "ln2_g", "ln2_b", "w1", "b1", "w2", "b2"], "llama": ["ln1_g", "wqkv", "wo", "ln2_g", "wgu", "wd"]}
NAMES["bert"] = NAMES["gpt"]


def test_a_configuration_that_ends_before_the_new_fields_is_taken():
    new = StageConfig.make(arch="llama", **BASE)
    old = StageConfig.make(arch="llama", **BASE, attn_window=9, qk_norm=1)     # (what lies behind its end is not read)
    old.struct_size = StageConfig.attn_window.offset
    assert query_sizes(old) == query_sizes(new)


@pytest.mark.parametrize("kw,status", [(dict(attn_window=-1), 1), (dict(attn_sinks=3), 1), (dict(attn_window=8, attn_sinks=-1), 1), (dict(qk_norm=2), 1),
                                       (dict(arch="bert", attn_window=8), 5)])
def test_refusals(kw, status):
    with pytest.raises(P.AhError) as e:
        query_sizes(StageConfig.make(**{**BASE, "arch": "gpt", **kw}))
    assert e.value.status == status


def test_sizes():
    T, h = BASE["seq"] * BASE["mb"], BASE["hidden"]
    a, b = query_sizes(StageConfig.make(arch="gpt", **BASE)), query_sizes(StageConfig.make(arch="gpt", qk_norm=1, **BASE))
    assert b["param_elems"] - a["param_elems"] == 2 * 2 * 128
    assert b["activation_bytes_per_layer_per_slot"] - a["activation_bytes_per_layer_per_slot"] == 4 * T * h


class Reference:
    """The stage's layers in fp64 with autograd."""

    def __init__(self, cfg, arch, stage):
        self.cfg, self.arch = cfg, arch
        names = NAMES[arch] + (["qn_g", "kn_g"] if cfg.qk_norm else [])
        self.p = [{n: stage.param_view(l, n).double().cpu().requires_grad_() for n in names} for l in range(cfg.n_layers)]

    def norm(self, x, p, which):
        eps = 1e-6 if self.arch == "llama" else 1e-5
        if self.arch == "llama":
            return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * p[which + "_g"]
        c = x - x.mean(-1, keepdim=True)
        return c * torch.rsqrt((c * c).mean(-1, keepdim=True) + eps) * p[which + "_g"] + p[which + "_b"]

    def attention(self, a, p):
        c = self.cfg
        B, S, nh, d = c.microbatch_size, c.seq_len, c.n_heads, c.head_dim
        qkv = a @ p["wqkv"] + (p["bqkv"] if "bqkv" in p else 0)
        q, k, v = (t.reshape(B, S, nh, d).transpose(1, 2) for t in qkv.split(nh * d, dim=-1))
        if c.qk_norm:
            eps = 1e-6 if self.arch == "llama" else 1e-5
            q, k = (t * torch.rsqrt((t * t).mean(-1, keepdim=True) + eps) * p[g] for t, g in ((q, "qn_g"), (k, "kn_g")))
        if self.arch == "llama":
            theta = 10000.0 ** (-2 * torch.arange(d // 2, dtype=torch.float64) / d)
            ang = torch.arange(S, dtype=torch.float64)[:, None] * theta
            turn = torch.polar(torch.ones_like(ang), ang)
            def rot(t):
                z = torch.complex(t[..., :d // 2], t[..., d // 2:]) * turn
                return torch.cat([z.real, z.imag], -1)
            q, k = rot(q), rot(k)
        i, j = torch.arange(S)[:, None], torch.arange(S)[None]
        W = c.attn_window or S
        hidden = torch.zeros(S, S, dtype=torch.bool) if self.arch == "bert" else (j > i) | ((i - j >= W) & (j >= c.attn_sinks))
        s = (q @ k.transpose(-1, -2) / math.sqrt(d)).masked_fill(hidden, -math.inf)
        return (torch.softmax(s, -1) @ v).transpose(1, 2).reshape(B * S, nh * d)

    def __call__(self, x):
        for p in self.p:
            m = x + self.attention(self.norm(x, p, "ln1"), p) @ p["wo"] + (p["bo"] if "bo" in p else 0)
            n = self.norm(m, p, "ln2")
            if self.arch == "llama":
                g, u = (n @ p["wgu"]).chunk(2, -1)
                x = m + (torch.nn.functional.silu(g) * u) @ p["wd"]
            else:
                x = m + torch.nn.functional.gelu(n @ p["w1"] + p["b1"], approximate="tanh") @ p["w2"] + p["b2"]
        return x


def _stage(arch, **kw):
    cfg = StageConfig.make(arch=arch, **{**BASE, **kw})
    st = P.Stage(cfg)
    g = torch.Generator().manual_seed(5)
    for l in range(cfg.n_layers):
        for n in NAMES[arch] + (["qn_g", "kn_g"] if cfg.qk_norm else []):
            v = st.param_view(l, n)
            r = torch.randn(v.shape, generator=g)
            v.copy_((1 + 0.2 * r if n.endswith("_g") else 0.1 * r if v.dim() == 1 else 0.04 * r).bfloat16())
    return cfg, st


def _draw(cfg, k, seed=9):
    g = torch.Generator().manual_seed(seed)
    T, h = cfg.microbatch_size * cfg.seq_len, cfg.hidden
    return [tuple(torch.randn(T, h, generator=g).bfloat16() for _ in range(2)) for _ in range(k)]


def _l2(got, ref):
    ref = ref.double().cpu().reshape(-1)
    return ((got.double().cpu().reshape(-1) - ref).norm() / ref.norm()).item()


CASES = [("llama", dict(attn_window=50, attn_sinks=3, qk_norm=1)), ("llama", dict(qk_norm=1, recompute=1)), ("gpt", dict(attn_window=100)),
         ("gpt", dict(qk_norm=1, attn_window=33, attn_sinks=70, wgrad_group=2)), ("bert", dict(qk_norm=1)),
         ("llama", dict(attn_window=40, attn_sinks=2, qk_norm=1, head_dim=128, n_heads=2, residual_fp32=1, recompute=1)),
         ("gpt", dict(attn_window=1000, attn_sinks=5, qk_norm=1, side=True)), ("llama", dict(attn_window=20, attn_sinks=1, qk_norm=1, wgrad_group=3, side=True))]


@pytest.mark.gpu
@pytest.mark.parametrize("arch,kw", CASES)
def test_stage_against_its_definition(arch, kw, monkeypatch):
    if kw.get("side"):
        monkeypatch.setenv("AH_SIDE_STREAM_MIN_GFLOP", "0")     # a stage this small keeps one stream otherwise
        monkeypatch.setenv("AH_DEFER_WGRADS", "0")
    kw = {k: v for k, v in kw.items() if k != "side"}
    K = 3
    cfg, st = _stage(arch, n_mb=K, max_in_flight=max(1, kw.get("wgrad_group", 0)), **kw)
    ref = Reference(cfg, arch, st)
    st.zero_grads()
    for m, (x, dy) in enumerate(_draw(cfg, K)):
        xd, dyd = x.cuda(), dy.cuda()
        y, dx = torch.empty_like(xd), torch.empty_like(xd)
        slot = m % cfg.max_in_flight
        st.forward(slot, xd, y)
        st.backward(slot, dyd, dx)
        torch.cuda.synchronize()
        x64 = x.double().requires_grad_()
        out = ref(x64)
        out.backward(dy.double())
        assert _l2(y, out.detach()) <= U.ACT_TOL and _l2(dx, x64.grad) <= U.ACT_TOL, (m, _l2(y, out.detach()), _l2(dx, x64.grad))
    st.flush_grads()
    torch.cuda.synchronize()
    errors = {(l, n): _l2(st.grad_view(l, n), t.grad) for l, p in enumerate(ref.p) for n, t in p.items()}
    assert max(errors.values()) <= U.GRAD_TOL, errors
    st.close()


@pytest.mark.gpu
def test_without_the_options_a_stage_keeps_its_bits():
    """A window that hides nothing and no norms: attention by other kernels, everything else the same; off, the very same bits as a stage made without the fields."""
    outs = []
    for end in (StageConfig.attn_window.offset, C.sizeof(StageConfig)):
        cfg, st = _stage("llama")
        old = StageConfig.make(arch="llama", **BASE)
        old.struct_size = end
        st2 = P.Stage(old)
        st2.params.copy_(st.params)
        x, dy = (t.cuda() for t in _draw(cfg, 1)[0])
        y, dx = torch.empty_like(x), torch.empty_like(x)
        st2.forward(0, x, y)
        st2.backward(0, dy, dx)
        torch.cuda.synchronize()
        outs.append((y, dx, st2.grads.clone()))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.gpu
def test_trace_names_the_new_sites_and_keeps_the_bits():
    cfg, st = _stage("llama", attn_window=50, attn_sinks=3, qk_norm=1)
    x, dy = (t.cuda() for t in _draw(cfg, 1)[0])
    y, dx = torch.empty_like(x), torch.empty_like(x)
    st.forward(0, x, y)
    st.backward(0, dy, dx)
    torch.cuda.synchronize()
    want = (y.clone(), dx.clone(), st.grads.clone())
    st.zero_grads()
    st.trace_begin()
    st.forward(0, x, y)
    st.backward(0, dy, dx)
    sites = {s["name"]: s for s in st.trace_end()}
    assert all(torch.equal(a, b) for a, b in zip(want, (y, dx, st.grads)))
    assert sites["qk_norm_fwd"]["launches"] == sites["qk_norm_bwd"]["launches"] == 2 and sites["gemm_nn.qkv_fwd"]["launches"] == 4 and "rope" not in sites
    S, W, n = 256, 50, 3
    pairs = sum(sum(1 for j in range(i + 1) if i - j < W or j < n) for i in range(S))
    assert sites["attention_fwd"]["flops_per_launch"] == 4 * 64 * pairs * 4 * 2
    T, h, F = 512, 256, 384
    assert sum(s["flops_per_launch"] * s["launches"] for s in sites.values() if s["name"] == "gemm_nn.qkv_fwd") == 2 * 2 * T * h * 3 * h


@pytest.mark.gpu
@pytest.mark.parametrize("bits,master,group", [(32, True, 0), (8, True, 2), (8, False, 0)])
def test_iterations_with_the_optimizer(bits, master, group):
    """Three iterations of two micro-batches, gradient norm, clipping and step, everything enqueued on one stream: the parameters are those of the step's formula on the
    stage's own gradients, and the loss sum(y * dy) goes the way that its gradient says."""
    cfg, st = _stage("llama", n_layers=1, n_mb=2, max_in_flight=2, wgrad_group=group, attn_window=60, attn_sinks=2, qk_norm=1)
    opt = st.adamw(weight_decay=0.1, state_bits=bits, master=master, betas=(0.9, 0.95))
    assert len(opt.params) == 8 and sum(p.numel() for p in opt.params) == sum(st.param_view(0, n).numel() for n in NAMES["llama"] + ["qn_g", "kn_g"])
    batch = [tuple(t.cuda() for t in b) for b in _draw(cfg, 2)]
    m = [torch.zeros(p.numel(), dtype=torch.float64) for p in opt.params]
    v = [torch.zeros(p.numel(), dtype=torch.float64) for p in opt.params]
    losses = []
    for it in range(1, 4):
        before = [(opt.master if master else opt.params)[k].double().cpu() for k in range(8)]
        st.zero_grads()
        ys = []
        for s, (x, dy) in enumerate(batch):
            y, dx = torch.empty_like(x), torch.empty_like(x)
            st.forward(s, x, y)
            st.backward(s, dy, dx)
            ys.append(y)
        st.flush_grads()
        norm = opt.grad_norm(1.0)
        opt.step(1e-3, it, grad_norm=norm, seed=it)
        torch.cuda.synchronize()
        losses.append(sum((y.double() * dy.double()).sum().item() for y, (_, dy) in zip(ys, batch)))
        grads = [g.double().cpu() for g in opt.grads]
        want = math.sqrt(sum((g * g).sum().item() for g in grads))
        assert abs(norm[0].item() - want) <= 2 ** -22 * want
        factor = norm[1].item()
        for k, name in enumerate(NAMES["llama"] + ["qn_g", "kn_g"]):
            m[k] = 0.9 * m[k] + 0.1 * factor * grads[k]
            v[k] = 0.95 * v[k] + 0.05 * (factor * grads[k]) ** 2
            update = 1e-3 * (m[k] / (1 - 0.9 ** it)) / (torch.sqrt(v[k] / (1 - 0.95 ** it)) + 1e-8)
            ref = before[k] * (1 - 1e-3 * (0.1 if opt.params[k].numel() > 256 else 0)) - update
            got = (opt.master if master else opt.params)[k].double().cpu()
            # 8-bit states go on from rounded moments: taken over from the optimizer below, so that each step is checked by itself
            room = 1e-4 * update.abs() + 1e-6 * ref.abs() + (0 if master else 2 ** -8 * ref.abs()) + 1e-12
            assert ((got - ref).abs() <= room).all(), (it, name, ((got - ref).abs() / room).max().item())
        if bits == 8:
            out = [[torch.empty(p.numel(), dtype=torch.bfloat16, device="cuda") for p in opt.params] for _ in range(2)]
            opt.state_values(*out)
            m, v = ([t.double().cpu() for t in o] for o in out)
        if master:
            assert all(torch.equal(a, b.bfloat16()) for a, b in zip(opt.params, opt.master))
    st.close()
