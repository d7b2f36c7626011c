"""Group norm of channel counts that have few divisors, up to the most channels that there may be."""
import time

import pytest
import torch

import paper_1907_09356_b200 as choco
from test_gpu_group_norm import BF16, DEV, F32, inputs, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape,groups", [((1, 2, 30, 2053), 2053), ((2, 1, 9, 4099), 4099), ((1, 1, 40, 6159), 3), ((1, 1, 5, 1 << 20), 1 << 10), ((1, 1, 16, 1048573), 1048573)])
def test_many_channels(shape, groups):
    gen = torch.Generator(device=DEV).manual_seed(71)
    if shape[3] // groups > 2048:
        with pytest.raises(choco.ChocoError):
            choco.GroupNorm(shape[0], shape[3], groups)
        return
    gn = choco.GroupNorm(shape[0], shape[3], groups, max_images=shape[1], activation="relu")
    for dtype in (F32, BF16):
        run(gn, *inputs(shape, gen, dtype, dtype), groups, "relu")
    gn.close()


def test_calls_do_not_search_through_all_channels():
    """1048573 is prime: a call looks for divisors below the widest slice only, well under the time of as many divisions as channels."""
    c = 1048573
    x, y = torch.zeros((1, 1, 1, c), device=DEV), torch.empty((1, 1, 1, c), device=DEV)
    gn = choco.GroupNorm(1, c, c)
    gn.forward(x, None, None, y)
    torch.cuda.synchronize()
    took = []
    for _ in range(20):
        t = time.perf_counter()
        gn.forward(x, None, None, y)
        took.append(time.perf_counter() - t)
        torch.cuda.synchronize()
    assert min(took) < 1e-3                                          # (a million 64-bit remainders take several milliseconds)
    gn.close()
