"""The gradient of a table whose tokens are few: the zeros of the other rows, through the binding."""
import time

import pytest
import torch

import paper_2512_20953_amd as P

pytestmark = pytest.mark.gpu
F32 = torch.float32


def scratch(T, V, w):
    return torch.empty(P.embedding_bwd_workspace(T, V, w), dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("T", [0, 1, 300, 2000, 20000])
@pytest.mark.parametrize("V,w,gap,shift", [(1, 1, 0, 1), (1, 3, 0, 3), (1, 700, 5, 2), (5, 1, 0, 1), (3, 2, 0, 2), (900, 17, 0, 3), (901, 33, 0, 1), (77, 64, 0, 2), (40, 65, 3, 0), (40, 66, 3, 3),
                                           (300, 1, 1, 1), (300, 1, 6, 3), (30, 1300, 2, 1), (6, 4099, 4, 2), (15999, 3, 0, 1), (12000, 18, 3, 2), (16001, 65, 0, 3), (50000, 5, 0, 1), (20000, 7, 2, 1)])
def test_every_element_is_written_and_none_beside_them(T, V, w, gap, shift):
    """Tables that begin `shift` elements behind 16 bytes, with rows `gap` elements apart"""
    ld = w + gap
    buf = torch.full((shift + V * ld + 64,), 7.0, device="cuda")
    d = buf[shift:].as_strided((V, w), (ld, 1))
    want = torch.full_like(buf, 7.0)
    inside = want[shift:].as_strided((V, w), (ld, 1))
    g = torch.Generator().manual_seed(T + V + w)
    tok = torch.randint(0, V, (T,), generator=g).cuda()
    dy = torch.randint(-8, 9, (T, w), generator=g).float().cuda()           # whole numbers: their sums are the same in any order
    inside.zero_()
    inside.index_add_(0, tok, dy)
    d.fill_(float("nan"))
    P.embedding_bwd(tok, dy, d, scratch(T, V, w))
    assert torch.equal(buf, want)


@pytest.mark.parametrize("T,V,w", [(222, 70000, 3800), (222, 70000, 3801), (16, 91583, 2176)])
def test_few_tokens_take_hardly_longer_than_the_zeros(T, V, w):
    """Beside the table's zeros, 0.8 GB and more, what few tokens add is two short launches: at most a quarter longer than a fill of the table."""
    tok, dy = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(1)).cuda(), torch.randn(T, w, device="cuda")
    d, work = torch.empty(V, w, device="cuda"), scratch(T, V, w)

    def seconds(call):
        torch.cuda.synchronize()
        t = time.perf_counter()
        for _ in range(10):
            call()
        torch.cuda.synchronize()
        return time.perf_counter() - t
    bwd, fill = lambda: P.embedding_bwd(tok, dy, d, work), lambda: d.zero_()    # noqa: E731
    both = [(seconds(bwd), seconds(fill)) for _ in range(8)][1:]
    a, b = (min(x) for x in zip(*both))
    print("%d tokens, %d x %d: %.0f us, the zeros alone %.0f" % (T, V, w, a * 1e5, b * 1e5))
    assert a <= 1.25 * b
