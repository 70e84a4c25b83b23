"""A stage made from a configuration that ends before its latest fields does not read what lies behind that end."""
import ctypes as C

import pytest
import torch

import paper_2512_20953_amd as P
from paper_2512_20953_amd.binding import StageConfig

pytestmark = pytest.mark.gpu
BASE = dict(arch="llama", n_layers=1, hidden=256, n_heads=4, head_dim=64, ffn=384, seq=256, mb=1)


def _run(cfg):
    st = P.Stage(cfg)
    g = torch.Generator().manual_seed(3)
    st.params.copy_((0.04 * torch.randn(st.params.shape, generator=g)).bfloat16())
    x, dy = (torch.randn(256, 256, generator=g).bfloat16().cuda() for _ in range(2))
    y, dx = torch.empty_like(x), torch.empty_like(x)
    st.forward(0, x, y)
    st.backward(0, dy, dx)
    torch.cuda.synchronize()
    return y, dx, st.grads.clone()


def test_fields_behind_the_end_are_not_read():
    plain, short, whole = StageConfig.make(**BASE), StageConfig.make(**BASE, attn_window=9, attn_sinks=2, qk_norm=1), StageConfig.make(**BASE, attn_window=9, attn_sinks=2)
    short.struct_size = StageConfig.attn_window.offset
    assert plain.struct_size == C.sizeof(StageConfig)
    want = _run(plain)
    assert all(torch.equal(a, b) for a, b in zip(_run(short), want))
    assert not torch.equal(_run(whole)[0], want[0])                    # (read, they would change the results)
