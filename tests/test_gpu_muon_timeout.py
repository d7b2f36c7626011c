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


@pytest.mark.parametrize("shapes", LISTS)
def test_nothing_is_written_after_a_wait_ran_out(shapes):
    gen = torch.Generator(device=DEV).manual_seed(42)
    off_ = [0]
    for r, c in shapes:
        off_.append(off_[-1] + r * c)
    X = torch.randn((2, off_[-1]), generator=gen, device=DEV)
    G, C = torch.randn(X.shape, generator=gen, device=DEV), torch.zeros(X.shape, dtype=torch.bfloat16, device=DEV)
    opt = choco.Muon(X, G, off_, shapes, copy=C)
    opt.step(0.02)
    opt.status()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):                       # of healthy calls
        opt.step(0.02)
    x0, c0 = X.clone(), C.clone()
    choco.choco_debug_muon_set_wait_polls(opt.handle, 0)
    opt.step(0.02)
    if len(shapes) == 1:                                             # (of several, those that were done before may have been written)
        assert torch.equal(X, x0) and torch.equal(C, c0)
    x1, c1, m1 = X.clone(), C.clone(), opt.m.clone()
    choco.choco_debug_muon_set_wait_polls(opt.handle, 1 << 22)
    opt.step(0.02)                                                   # enqueued: nobody has looked yet
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(X, x1) and torch.equal(C, c1) and torch.equal(opt.m, m1)
    timed_out(opt.status)
    for call in (lambda: opt.step(0.02), opt.status, lambda: choco.choco_muon_orthogonalize(opt.handle),
                 lambda: choco.choco_muon_set_grads(opt.handle, [G.data_ptr()] * opt.handle.n_matrices)):
        timed_out(call)
    torch.cuda.synchronize()
    assert torch.equal(X, x1) and torch.equal(opt.m, m1)
    del graph
    opt.close()
    again = choco.Muon(X, G, off_, shapes, copy=C)                   # a fresh handle carries on
    again.step(0.02)
    again.status()
    assert X.isfinite().all() and not torch.equal(X, x1)
    again.close()
