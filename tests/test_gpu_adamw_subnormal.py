"""Second moments below 2^-126 divide a step like any others: it matters where eps is smaller still.

The moments are the kernel's own (or their IEEE fp32 recursion from what 8-bit states stand for); the update then goes through a hardware root and reciprocal (1 ulp each), three
roundings of fp32 and lr / (1 - beta1^t) and 1 / sqrt(1 - beta2^t) in fp32: below 8 x 2^-23 of itself."""
import pytest
import torch

import paper_2512_20953_amd as P

pytestmark = pytest.mark.gpu
DEV = "cuda"
B1, B2, LR = 0.9, 0.95, 1e-2


def _check(got, m, v, step, eps):
    want = -LR / (1 - B1 ** step) * m.double() / (torch.sqrt(v.double() / (1 - B2 ** step)) + eps)
    assert ((got.double().cpu() - want).abs() <= 2 ** -20 * want.abs()).all(), ((got.double().cpu() - want).abs() / want.abs()).max().item()


@pytest.mark.parametrize("eps", [1e-37, 1e-30, 1e-20, 1e-8])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_states_in_32_bits(eps, dtype):
    grad = (10.0 ** torch.linspace(-21.5, -16, 999)).to(dtype).to(DEV)        # v from 5e-45 on
    p = torch.zeros(999, device=DEV)
    opt = P.AdamW([p], [grad], betas=(B1, B2), eps=eps)
    for step in (1, 2):
        p.zero_()
        opt.step(LR, step)
        m, v = opt.m[0].cpu(), opt.v[0].cpu()
        assert (v > 0).all() and (v < 2.0 ** -126).sum() > 400
        _check(p, m, v, step, eps)


@pytest.mark.parametrize("eps", [1e-37, 1e-30, 8e-12, 8.2e-12, 1e-8])   # (from 8.13e-12 on subnormals are below half a unit of it)
def test_states_in_8_bits(eps):
    n = 640
    grad = torch.full((n,), 1e-19, device=DEV)
    p = torch.zeros(n, device=DEV)
    opt = P.AdamW([p], [grad], betas=(B1, B2), eps=eps, state_bits=8)
    opt.step(LR, 1)
    out = [[torch.empty(n, dtype=torch.bfloat16, device=DEV)] for _ in range(2)]
    opt.state_values(*out)
    m, v = (o[0].float().cpu() for o in out)
    assert (m > 0).all() and (v > 0).all() and (v < 2.0 ** -126).all()
    p.zero_()
    grad.zero_()
    opt.step(LR, 2)
    c1, c2 = torch.tensor(1 - B1, dtype=torch.float32), torch.tensor(1 - B2, dtype=torch.float32)
    _check(p, m + c1 * (0 - m), v + c2 * (0 - v), 2, eps)
