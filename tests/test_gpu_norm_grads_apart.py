"""Gradients of scales and of shifts that would be written to the same elements are refused."""
import pytest
import torch

import paper_1907_09356_b200 as choco
from test_gpu_group_norm import DEV

pytestmark = pytest.mark.gpu


def rows(G, at, n, ld, c):
    return G.as_strided((n, c), (ld, 1), at)


@pytest.mark.parametrize("n,ld,c", [(3, 40, 8), (1, 8, 8), (3, 16, 8), (3, 8, 8), (4, 21, 6)])
def test_rows_that_meet(n, ld, c):
    x = torch.randn((n, 2, 5, c), device=DEV)
    stats = [torch.zeros((n, 2, 2), device=DEV), torch.ones((n, 2, 2), device=DEV)]
    gn = choco.GroupNorm(n, c, 2, max_images=2)
    G = torch.zeros(2 * n * ld + 2 * c, device=DEV)
    for first, second in [(0, k) for k in range(n * ld + 3)] + [(k, 0) for k in range(1, n * ld + 3)]:
        dw, db = rows(G, first, n, ld, c), rows(G, second, n, ld, c)
        elements = lambda at: {at + i * ld + k for i in range(n) for k in range(c)}  # noqa: E731
        G.zero_()
        if elements(first) & elements(second):
            with pytest.raises(choco.ChocoError) as err:
                gn.backward(x, x, None, None, *stats, None, dw, db)
            assert err.value.code == -1 and not G.any()
        else:
            gn.backward(x, x, None, None, *stats, None, dw, db)
            assert float((dw - (x * x).sum((1, 2))).abs().max()) < 1e-4 and float((db - x.sum((1, 2))).abs().max()) < 1e-4
    gn.close()
