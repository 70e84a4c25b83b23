"""AdamW over parameters that autograd knows: the copies that it makes are plain tensors, and a step leaves the graph alone."""
import pytest
import torch

import paper_2512_20953_amd as P

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 32])
def test_parameters_that_need_gradients(bits):
    p = torch.nn.Parameter(torch.linspace(-1, 1, 96).bfloat16().cuda())
    q = p.detach().clone()
    g = torch.linspace(1, 2, 96).cuda()
    a, b = (P.AdamW([t], [g], state_bits=bits, master=True) for t in (p, q))
    assert not a.master[0].requires_grad and a.master[0].grad_fn is None and not a.master[0]._base.requires_grad
    for opt in (a, b):
        opt.step(1e-2, 1)
    assert torch.equal(p.detach(), q) and torch.equal(a.master[0], b.master[0])
    p.float().sum().backward()
    assert (p.grad == 1).all()


def test_states_in_8_bits_come_with_their_scales():
    n, f = 96, lambda k: [torch.ones(k, dtype=torch.uint8, device="cuda")]      # noqa: E731
    p, g = [torch.zeros(n, device="cuda")], [torch.ones(n, device="cuda")]
    for kw in (dict(m=f(n)), dict(v=f(n)), dict(m=f(n), v=f(n)), dict(m=f(n), v=f(n), m_scale=f(3)), dict(m_scale=f(3)), dict(v_scale=f(3))):
        with pytest.raises(P.AhError, match="scales"):
            P.AdamW(p, g, state_bits=8, **kw)
    P.AdamW(p, g, state_bits=8, m=f(n), v=f(n), m_scale=f(3), v_scale=f(3))
