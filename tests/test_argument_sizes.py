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
