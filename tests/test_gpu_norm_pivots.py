"""Group norm's statistics over very many small groups, among which every distance of the first pixel from the others occurs."""
import pytest
import torch

import paper_1907_09356_b200 as choco
from test_gpu_group_norm import BF16, DEV, F16, F32, close, statistics

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pixels", [4, 16, 61, 300])
@pytest.mark.parametrize("per", [1, 2])
def test_many_groups(pixels, per):
    gen = torch.Generator(device=DEV).manual_seed(81)
    images, c = 600_000 // pixels, 64
    for dtype in (F32, BF16, F16):
        x = (torch.randn((1, images, pixels, c), generator=gen, device=DEV) * 3 + torch.randn(c, generator=gen, device=DEV)).to(dtype)
        mean, rstd = torch.empty((1, images, c // per), device=DEV), torch.empty((1, images, c // per), device=DEV)
        gn = choco.GroupNorm(1, c, c // per)
        gn.forward(x, None, None, torch.empty_like(x), mean, rstd)
        m, r = statistics(x, c // per)
        # 1.5 R roundings of rstd with R = 8 (and a few of its own): below 2^-20; the mean: as many of the deviation
        close(mean, m, 2.0 ** -20, m.abs() + 1 / r)
        assert float((rstd.double() / r - 1).abs().max()) < 2.0 ** -20
        gn.close()
