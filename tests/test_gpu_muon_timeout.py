"""Waits of Muon's kernels that run out: counted, sat out and reported, whatever roles of a block they are of.

No GPU is stalled for this.  The handle's test hook sets the polls after which a wait counts as run out to zero; the second, bounded
part of every wait then sees what the first would have seen."""
import pytest
import torch

import paper_1907_09356_b200 as choco
from test_gpu_muon import DEV, F32, exact, gradient, most_off, off

pytestmark = pytest.mark.gpu

# one block; single blocks, X X^T whole and split along K; pairs, whole and split; all of them in one list
LISTS = [[(64, 576)], [(100, 700)], [(100, 3000)], [(300, 300)], [(650, 2600)], [(16, 27), (100, 3000), (3000, 90), (700, 4200), (260, 6000)]]


def timed_out(call):
    with pytest.raises(choco.ChocoError) as err:
        call()
    assert err.value.code == choco.ERR_TIMEOUT


@pytest.mark.parametrize("products", [1, 3])
@pytest.mark.parametrize("shapes", LISTS)
def test_waits_that_run_out_are_reported(shapes, products):
    gen = torch.Generator(device=DEV).manual_seed(41)
    ins = [gradient(s, gen) for s in shapes]
    outs = [torch.empty(s, device=DEV) for s in shapes]
    o = choco.Orthogonalizer(ins, outs, products=products)
    o.apply()
    o.status()
    choco.choco_debug_muon_set_wait_polls(o.handle, 0)
    o.apply()
    timed_out(o.status)
    torch.cuda.synchronize()                                         # the device is alive and well
    o.close()
    fresh = choco.Orthogonalizer(ins, outs, products=products)
    fresh.apply()
    fresh.status()
    fresh.close()
    for u, v in zip(ins, outs):
        assert off(v, exact(u)) < most_off(products, 5, F32)
