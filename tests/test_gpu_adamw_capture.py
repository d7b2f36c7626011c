"""AdamW steps captured in a graph: every replay is a step of its own.  Tolerances are those of test_gpu_adamw,
whose Run gives the step in 64 bits for each worker's own number of steps."""
import numpy as np
import pytest
import torch

import paper_1907_09356_b200 as choco
from test_gpu_adamw import BF16, DEV, Run, U

pytestmark = pytest.mark.gpu


def gradients(r, seed):
    r.G[:, :r.d].normal_(0.0, 0.01, generator=torch.Generator(device=DEV).manual_seed(seed))


def graph_of(call):
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    return graph


@pytest.mark.parametrize("bits", [32, 8])
def test_replays_are_the_steps_of_direct_calls(bits):
    a, b = Run(2, [500, 300], bits, copy=BF16), Run(2, [500, 300], bits, copy=BF16)
    graph = graph_of(lambda: b.opt.step(1e-3))
    assert list(b.opt.get_steps()) == [0, 0]                     # a capture is no step
    for t in range(1, 6):
        for r in (a, b):
            gradients(r, t)
        want = b.ref(1e-3, t)
        a.opt.step(1e-3)
        graph.replay()
        b.check(None, want)
        assert list(b.opt.get_steps()) == [t, t]
        assert torch.equal(a.X, b.X) and torch.equal(a.opt.m, b.opt.m) and torch.equal(a.opt.v, b.opt.v) and torch.equal(a.copy, b.copy)
    for r in (a, b):
        r.opt.close()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("sizes", [[300, 2049, 5], [4096, 40_000, 256 * 33_000]])
def test_replays_and_direct_calls_alternate_and_groups_sit_out(bits, sizes):
    """A worker's gradient overflows now and then, in a replay or in a direct call; the counts are set anew on the
    way.  The longer list takes several launches a step.  The parameters stay within ref()'s bound; moments do not
    depend on the number of steps and equal those of a run of direct calls bit for bit."""
    r, twin = Run(3, sizes, bits, copy=BF16), Run(3, sizes, bits, copy=BF16)
    norm, factor = torch.zeros(3, device=DEV), torch.zeros(3, device=DEV)

    def one(run):
        run.opt.grad_norm(0.5, norm, factor)
        run.opt.step(1e-3, factor)

    graph = graph_of(lambda: one(r))
    taken = np.array([0, 0, 0])
    for t, how in enumerate("drrdrrrdSrdr"):
        if how == "S":
            taken = np.array([4, 700, 2])
            r.opt.set_steps(taken)
            continue
        moving = [0, 1, 2]
        for run in (r, twin):
            gradients(run, t)
            if t in (2, 3, 10):
                run.G[1, 2] = float("inf")
                moving = [0, 2]
        one(twin)                                                # leaves the factors that ref() needs
        kept = r.X[1].clone()
        x, _, _, _, bound = r.ref(1e-3, [int(taken[i]) + (i in moving) for i in range(3)], factor)
        graph.replay() if how == "r" else one(r)
        taken[moving] += 1
        lim = 1.01 * (bound + 2 * U * x.abs()) + 1e-38
        assert bool(((r.X[:, :r.d].double() - x).abs() <= lim)[moving].all())
        assert torch.equal(r.copy[:, :r.d], r.X[:, :r.d].to(BF16))
        if 1 not in moving:
            assert torch.equal(r.X[1], kept)
        for a, b in zip((r.opt.m, r.opt.v, r.opt.m_scale, r.opt.v_scale), (twin.opt.m, twin.opt.v, twin.opt.m_scale, twin.opt.v_scale)):
            assert a is None or torch.equal(a, b)
        assert list(r.opt.get_steps()) == list(taken)
    for run in (r, twin):
        run.opt.close()


def test_two_steps_in_one_graph():
    a, b = Run(2, [500, 300]), Run(2, [500, 300])
    graph = graph_of(lambda: (b.opt.step(1e-3), b.opt.step(1e-3)))
    for _ in range(3):
        graph.replay()
    for _ in range(6):
        a.opt.step(1e-3)
    assert torch.equal(a.X, b.X) and torch.equal(a.opt.m, b.opt.m) and list(b.opt.get_steps()) == [6, 6]
    for r in (a, b):
        r.opt.close()


def test_gradients_that_would_move_chunks_under_a_graph_are_refused():
    r = Run(1, [5000])
    store = torch.randn(5008, device=DEV)
    at = lambda shift: [store[shift:shift + 5000].data_ptr()]  # noqa: E731
    choco.choco_adamw_set_grads(r.opt.handle, at(1))
    choco.choco_adamw_set_grads(r.opt.handle, at(0))
    graph = graph_of(lambda: r.opt.step(1e-3))
    with pytest.raises(choco.ChocoError) as e:
        choco.choco_adamw_set_grads(r.opt.handle, at(1))
    assert e.value.code == -6
    for shift in (4, 0):                                         # these stay on 16-byte boundaries
        choco.choco_adamw_set_grads(r.opt.handle, at(shift))
        r.G[0, :5000] = store[shift:shift + 5000]                # what ref() looks at
        want = r.ref(1e-3, int(r.opt.get_steps()[0]) + 1)
        graph.replay()
        r.check(None, want)
    r.opt.close()
