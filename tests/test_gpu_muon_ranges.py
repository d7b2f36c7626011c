"""Muon's momentum lies apart from what a step reads and writes."""
import pytest
import torch

import paper_1907_09356_b200 as choco
from test_gpu_muon import DEV, gradient

pytestmark = pytest.mark.gpu


def test_momentum_that_meets_other_arrays_is_refused():
    gen = torch.Generator(device=DEV).manual_seed(51)
    shape, off = (20, 64), [0, 1280]
    memory = torch.zeros(8 * 1280, device=DEV)
    X, G, C = (memory[k * 2560:k * 2560 + 2560].view(2, 1280) for k in range(3))
    G.copy_(gradient((2, *shape), gen).flatten(1))
    for start in (0, 1276, 2556, 2560, 3000, 5116, 5120, 7676):      # in X, G and C, and across their ends
        if start % 4 == 0:
            opt = choco.Muon(X, G, off, [shape], copy=C, states=memory[start:start + 2560])
            before = memory.clone()
            with pytest.raises(choco.ChocoError) as err:
                opt.step(0.1)
            assert err.value.code == -1 and torch.equal(memory, before)
            opt.close()
    opt = choco.Muon(X, G, off, [shape], copy=C, states=memory[7680:])
    opt.step(0.1)                                                    # right behind them
    x0 = X.clone()
    choco.choco_muon_set_grads(opt.handle, [memory[7680:].data_ptr(), G[1].data_ptr()])
    with pytest.raises(choco.ChocoError):
        opt.step(0.1)                                                # new gradients lie in it
    choco.choco_muon_set_grads(opt.handle, [G[1].data_ptr(), G[0].data_ptr()])
    opt.step(0.1)
    opt.status()
    assert X.isfinite().all() and not torch.equal(X, x0)
    opt.close()
