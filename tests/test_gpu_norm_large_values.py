"""Group norm of values at the end of their type's range: what is subtracted first is formed without leaving it."""
import pytest
import torch

import paper_1907_09356_b200 as choco
from test_gpu_group_norm import BF16, DEV, F16, F32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,value", [(F32, 3.0e38), (F32, -1.5e38), (BF16, 3.0e38), (F16, 65504.0)])
@pytest.mark.parametrize("pixels", [1, 50, 3000])
def test_constant_images(dtype, value, pixels):
    x = torch.full((1, 2, pixels, 16), value, device=DEV).to(dtype)
    x[:, 1] /= 2
    y, mean, rstd = torch.empty_like(x), torch.empty((1, 2, 4), device=DEV), torch.empty((1, 2, 4), device=DEV)
    gn = choco.GroupNorm(1, 16, 4, eps=0.25)
    gn.forward(x, None, None, y, mean, rstd)
    assert torch.equal(mean, x[:, :, 0, ::4].float()) and torch.equal(rstd, torch.full_like(rstd, 2.0)) and not y.any()
    gn.close()


def test_one_infinity_makes_an_infinite_mean():
    for at in (0, 1, 7, 20):                                         # among the pixels that are looked at first, and not
        x = torch.randn((1, 1, 50, 8), device=DEV)
        x[0, 0, at, 2] = float("inf")
        y, mean = torch.empty_like(x), torch.empty((1, 1, 2), device=DEV)
        gn = choco.GroupNorm(1, 8, 2)
        gn.forward(x, None, None, y, mean)
        assert y[..., :4].isnan().all() and y[..., 4:].isfinite().all() and not mean[0, 0, 0].isfinite() and mean[0, 0, 1].isfinite()
        gn.close()
