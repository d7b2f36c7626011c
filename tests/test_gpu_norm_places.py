"""Group norm where arrays lie in one another: sets of channels of a wider array, and the same array under another view."""
import pytest
import torch

import paper_1907_09356_b200 as choco
from test_gpu_group_norm import DEV, F32, close, forward

pytestmark = pytest.mark.gpu


def check(x, y):
    n, c = x.shape[0], x.shape[-1]
    x0 = x.clone()
    gn = choco.GroupNorm(n, c, 4)
    gn.forward(x, None, None, y)
    flat = lambda t: t.reshape(n, t.shape[1], -1, c)  # noqa: E731
    close(flat(y), forward(flat(x0), torch.ones((n, c), device=DEV), torch.zeros((n, c), device=DEV), 4, "none")[0], 2.0 ** -18)
    gn.close()
    return x0


@pytest.mark.parametrize("shape", [(2, 3, 1, 32), (1, 3, 1, 32), (2, 1, 1, 32), (1, 1, 1, 32), (1, 1, 7, 32), (2, 1, 7, 32)])
def test_sets_of_channels(shape):
    """Of images of one pixel as well."""
    gen = torch.Generator(device=DEV).manual_seed(61)
    for low, high in (((0, 16), (16, 32)), ((16, 32), (0, 16)), ((0, 12), (20, 32))):
        both = torch.randn(shape, generator=gen, device=DEV)
        x = both[..., low[0]:low[1]]
        x0 = check(x, both[..., high[0]:high[1]])
        assert torch.equal(x, x0)


def test_in_place_under_another_view():
    """Strides of axes with one element say nothing."""
    gen = torch.Generator(device=DEV).manual_seed(62)
    for shape, strides in (((1, 4, 6, 16), (7, 96, 16, 1)), ((2, 1, 6, 16), (96, 5, 16, 1)), ((2, 4, 1, 16), (64, 16, 3, 1))):
        x = torch.randn(shape, generator=gen, device=DEV)
        check(x, x.as_strided(shape, strides))


def test_places_that_meet_are_refused():
    memory = torch.zeros(4000, device=DEV)
    gn = choco.GroupNorm(2, 8, 2)
    x = memory.as_strided((2, 3, 1, 8), (96, 32, 32, 1))
    for offset, strides in ((4, (96, 32, 32, 1)), (28, (96, 32, 32, 1)), (8, (96, 16, 16, 1)), (8, (192, 32, 32, 1))):
        with pytest.raises(choco.ChocoError):
            gn.forward(x, None, None, memory.as_strided((2, 3, 1, 8), strides, offset))
    odd = memory.as_strided((2, 3, 5, 8), (500, 165, 33, 1)), memory.as_strided((2, 3, 5, 8), (500, 165, 33, 1), 16)
    with pytest.raises(choco.ChocoError):                            # 500 is no multiple of 33: the second worker's pixels lie elsewhere
        gn.forward(odd[0], None, None, odd[1])
    assert not memory.any()
    gn.close()
