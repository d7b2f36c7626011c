"""Group norm's statistics where the first pixels of an image are not like the rest of it."""
import pytest
import torch

import paper_1907_09356_b200 as choco
from test_gpu_group_norm import BF16, DEV, F16, F32, close, forward

pytestmark = pytest.mark.gpu


def images(shape, kind, dtype):
    """Noise of deviation 1 about an offset, whose first pixels lie elsewhere; in `dtype`'s own values."""
    gen = torch.Generator(device=DEV).manual_seed(21)
    offset, first, count = {"spike30": (0.0, 30.0, 1), "spike100": (0.0, 100.0, 1), "spike1000": (0.5, 1000.0, 1), "corner100": (100.0, 0.0, 1),
                            "corner1000": (1000.0, 0.0, 1), "border": (200.0, 0.0, 300), "spread": (3.0, -500.0, 9)}[kind]
    x = torch.randn(shape, generator=gen, device=DEV) + offset
    x[:, :, :count] = first
    if kind == "spread":                                             # the last pixels and some between as well
        x[:, :, -5:] = first
        x[:, :, shape[2] // 3] = first
    return x.to(dtype), offset


# kept in a block's shared memory, in a cluster's, read twice in part (accesses of 16, 8 and 2 or 4 bytes), slices gone through in rounds
SHAPES = [((2, 2, 300, 16), 4), ((1, 2, 12_544, 16), 8), ((1, 1, 12_544, 64), 32), ((1, 1, 100_000, 48), 6), ((1, 1, 400_000, 16), 4), ((1, 2, 50_001, 15), 5),
          ((1, 1, 30_000, 34), 17), ((1, 1, 700, 2048), 1), ((1, 1, 3000, 1200), 1), ((1, 1, 40, 2047), 1)]


@pytest.mark.parametrize("kind", ["spike30", "spike100", "spike1000", "corner100", "corner1000", "border", "spread"])
@pytest.mark.parametrize("shape,groups", SHAPES)
def test_first_pixels_unlike_the_rest(shape, groups, kind):
    if kind == "border" and shape[2] <= 600:
        shape = (*shape[:2], 900, shape[3])
    for dtype in (F32, BF16, F16):
        x, offset = images(shape, kind, dtype)
        gn = choco.GroupNorm(shape[0], shape[3], groups)
        y, mean, rstd = torch.empty_like(x), torch.empty((*shape[:2], groups), device=DEV), torch.empty((*shape[:2], groups), device=DEV)
        gn.forward(x, None, None, y, mean, rstd)
        one = torch.ones((shape[0], shape[3]), device=DEV)
        want = forward(x, one, one * 0, groups, "none")
        # sums of squares about points that lie within the values they are taken of lose a few roundings of float32, however far the first
        # pixel is: the bounds of ordinary images
        close(mean, want[1], 2.0 ** -20, want[1].abs() + 1 / want[2])
        close(rstd, want[2], 2.0 ** -20)
        # the mean is rounded to float32 before it is taken away: half a unit of it, in units of the deviation (1 at least)
        close(y, want[0], torch.finfo(dtype).eps / 2 + 2.0 ** -18 + offset * 2.0 ** -24)
        gn.close()
