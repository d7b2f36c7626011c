"""Orthogonalised updates and Muon against the formulas in float64."""
import math

import numpy as np
import pytest
import torch

import paper_1907_09356_b200 as choco

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
USUAL = choco.MUON_COEFFICIENTS

# How far a result may be off, as 2-norm over the result's.  A step multiplies small singular values, and with them what is
# wrong in their directions, by up to 3.4445, so an error e of every step grows to e (3.4445 + 3.4445^2 + ...).  With three
# products a step rounds X, S and B to 22 bits and adds up in float32: e = 2^-19 takes in all of them.  With one product
# e = 2^-11 and the same sum says nothing (0.33); but roundings are independent of each other and few directions are small: float16
# rounding put into a float64 run of these sizes gives 0.0008 .. 0.0017, and 0.004 is asked for.
def most_off(products, steps, out):
    growth = sum(USUAL[0] ** k for k in range(1, steps + 1))
    return (growth * 2.0 ** -19 if products == 3 else 0.004) + torch.finfo(out).eps / 2


def exact(u, steps=5, coefficients=USUAL):
    u = u.double()
    tall = u.shape[-2] > u.shape[-1]
    x = u.mT if tall else u
    norm = torch.linalg.matrix_norm(x, keepdim=True)
    x = x / torch.where(norm > 0, norm, 1.0)
    a, b, c = coefficients
    for _ in range(steps):
        s = x @ x.mT
        x = a * x + (b * s + c * s @ s) @ x
    return x.mT if tall else x


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


def gradient(shape, gen, size=1e-3, dtype=F32):
    *batch, r, c = shape
    rank = min(4, r, c)
    u = torch.randn(shape, generator=gen, device=DEV) * (0.3 * size)
    u += torch.randn((*batch, r, rank), generator=gen, device=DEV) * size @ torch.randn((*batch, rank, c), generator=gen, device=DEV)
    return u.to(dtype)


SHAPES = [(1, 1), (1, 7), (300, 1), (2, 2), (5, 64), (16, 27), (64, 65), (127, 129), (128, 128), (129, 128), (64, 576), (576, 64), (255, 257), (257, 300),
          (130, 1000), (384, 640), (500, 129), (1000, 1001), (2600, 650)]


@pytest.mark.parametrize("products", [1, 3])
@pytest.mark.parametrize("shape", SHAPES)
def test_orthogonalized_matrices(shape, products):
    gen = torch.Generator(device=DEV).manual_seed(1)
    u = gradient(shape, gen)
    for steps in (1, 5):
        out = torch.full(shape, float("nan"), device=DEV)
        o = choco.Orthogonalizer([u], [out], steps=steps, products=products)
        o.apply()
        o.status()
        o.close()
        assert off(out, exact(u, steps)) < most_off(products, steps, F32)


@pytest.mark.parametrize("source", [F32, BF16, F16])
@pytest.mark.parametrize("target", [F32, BF16, F16])
def test_types(source, target):
    gen = torch.Generator(device=DEV).manual_seed(2)
    for shape in ((40, 90), (2, 150, 260), (260, 300)):
        u = gradient(shape, gen, dtype=source)
        out = torch.empty(shape, dtype=target, device=DEV)
        o = choco.Orthogonalizer([u], [out])
        o.apply()
        o.close()
        want = exact(u)
        products = 1 if target == BF16 and min(shape[-2:]) > 128 else 3
        assert off(out, want) < most_off(products, 5, target)


@pytest.mark.parametrize("size", [1e-30, 1e-24, 1e25, 1e36])
def test_gradients_of_any_size(size):
    """Squares of these leave float32."""
    gen = torch.Generator(device=DEV).manual_seed(3)
    for shape in ((30, 50), (200, 140)):
        u = torch.randn(shape, generator=gen, device=DEV) * size
        out = torch.empty(shape, device=DEV)
        o = choco.Orthogonalizer([u], [out])
        o.apply()
        o.close()
        assert off(out, exact(u)) < most_off(3, 5, F32)


def test_zeros_and_what_is_no_number_stay_in_their_matrices():
    gen = torch.Generator(device=DEV).manual_seed(4)
    for shape in ((20, 40), (150, 300)):
        u = gradient((5, *shape), gen)
        u[1] = 0
        u[2, 3, 4] = float("nan")
        u[3, 0, 0] = float("inf")
        out = torch.full_like(u, 7.0)
        o = choco.Orthogonalizer([u], [out])
        o.apply()
        o.status()
        o.close()
        assert torch.equal(out[1], torch.zeros_like(out[1]))
        assert not out[2].isfinite().all() and not out[3].isfinite().all()
        for k in (0, 4):
            assert off(out[k], exact(u[k])) < most_off(3, 5, F32)


@pytest.mark.parametrize("shape", [(37, 60), (60, 37), (200, 333), (333, 200)])
def test_rows_with_gaps(shape):
    """Matrices that are parts of wider arrays: nothing else of these is written, nothing else read."""
    gen = torch.Generator(device=DEV).manual_seed(5)
    for gap in (1, 4, 8):
        wide = torch.full((shape[0] + 2, shape[1] + gap), float("nan"), device=DEV)
        u = wide[1:-1, gap:]
        u.copy_(gradient(shape, gen))
        into = torch.full((shape[0] + 2, shape[1] + gap + 3), 5.0, device=DEV)
        out = into[1:-1, 2:2 + shape[1]]
        o = choco.Orthogonalizer([u], [out])
        o.apply()
        o.close()
        assert off(out, exact(u)) < most_off(3, 5, F32)
        out.fill_(5.0)
        assert torch.equal(into, torch.full_like(into, 5.0))


@pytest.mark.parametrize("coefficients,steps", [((1.5, -0.5, 0.0), 3), ((1.875, -1.25, 0.375), 2), (USUAL, 0), (USUAL, 7)])
def test_polynomials(coefficients, steps):
    gen = torch.Generator(device=DEV).manual_seed(6)
    for shape in ((50, 80), (140, 260)):
        u = gradient(shape, gen)
        out = torch.empty_like(u)
        o = choco.Orthogonalizer([u], [out], steps=steps, coefficients=coefficients)
        o.apply()
        o.close()
        # (each step magnifies what is wrong by a at most)
        growth = sum(coefficients[0] ** k for k in range(1, steps + 1)) + 1
        assert off(out, exact(u, steps, coefficients)) < growth * 2.0 ** -19


def test_singular_values_come_near_one():
    gen = torch.Generator(device=DEV).manual_seed(7)
    u = torch.randn((128, 512), generator=gen, device=DEV)
    out = torch.empty_like(u)
    choco.Orthogonalizer([u], [out]).apply()
    s = torch.linalg.svdvals(out.double())
    assert 0.6 < float(s.min()) and float(s.max()) < 1.3


def test_a_matrix_does_not_depend_on_the_others():
    """Nor on the order of the list, on what ran before, or on the time; more than one workspace's worth among them."""
    gen = torch.Generator(device=DEV).manual_seed(8)
    shapes = [(2048, 2048)] * 30 + [(64, 576)] * 3 + [(100, 3000), (300, 100), (128, 1152), (1, 1), (700, 65)]
    ins = [gradient(s, gen) for s in shapes]
    outs = [torch.empty_like(u) for u in ins]
    together = choco.Orthogonalizer(ins, outs)
    together.apply()
    together.apply()
    together.status()
    back = [torch.empty_like(u) for u in ins]
    other = choco.Orthogonalizer(ins[::-1], back[::-1])
    other.apply()
    for a, b in zip(outs, back):
        assert torch.equal(a, b)
    assert off(outs[3], exact(ins[3])) < most_off(3, 5, F32) and off(outs[29], exact(ins[29])) < most_off(3, 5, F32)
    together.close()
    other.close()


def network(n, gen, x=F32, g=F32, copy=None, tail=3):
    """Rows of X and G with matrices, biases and a ragged rest between them."""
    shapes = [(16, 27), None, (40, 100), (130, 260), None, (300, 17), (1, 9)]
    sizes = [s[0] * s[1] if s else 11 for s in shapes]
    layer_off = np.concatenate([[0], np.cumsum(sizes)])
    d = int(layer_off[-1]) + tail
    X = (torch.randn((n, d), generator=gen, device=DEV) * 0.05).to(x)
    G = torch.randn((n, d), generator=gen, device=DEV) * 1e-3
    for k, s in enumerate(shapes):
        if s:
            G[:, layer_off[k]:layer_off[k + 1]] = gradient((n, *s), gen).view(n, -1)
    return X, G.to(g), layer_off, shapes, None if copy is None else torch.zeros((n, d), dtype=copy, device=DEV)


def want_step(X, m, G, layer_off, shapes, offsets, factor, lr, decay, beta, nesterov, scale=None):
    """(x, m) in float64; the moments of matrix k of worker i start at offsets[i * matrices + k]."""
    x, m = X.double(), m.double()
    which = [k for k, s in enumerate(shapes) if s]
    for i in range(X.shape[0]):
        c = 1.0 if factor is None else float(factor[i])
        if not math.isfinite(c):
            continue
        for j, k in enumerate(which):
            (r, q), here = shapes[k], slice(int(layer_off[k]), int(layer_off[k + 1]))
            at = int(offsets[i * len(which) + j])
            g = c * G[i, here].double()
            part = m[at:at + r * q]
            part.mul_(beta).add_(g, alpha=1 - beta)
            u = beta * part + (1 - beta) * g if nesterov else part
            s = math.sqrt(max(1.0, r / q)) if scale is None else scale
            x[i, here] -= lr * (s * exact(u.view(r, q)).reshape(-1) + decay * x[i, here])
    return x, m


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("x,g,copy", [(F32, F32, None), (F32, BF16, BF16), (BF16, BF16, None), (F16, F32, F32)])
def test_steps(x, g, copy, nesterov):
    gen = torch.Generator(device=DEV).manual_seed(9)
    X, G, layer_off, shapes, C = network(3, gen, x, g, copy)
    opt = choco.Muon(X, G, layer_off, shapes, weight_decay=0.1, copy=C, beta=0.9, nesterov=nesterov)
    gaps = torch.ones(opt.elements, dtype=torch.bool, device=DEV)
    which = [s for s in shapes if s] * 3
    for at, (r, q) in zip(opt.offsets, which):
        gaps[at:at + r * q] = False
    assert int(gaps.sum()) > 0
    opt.m[gaps] = 123.0
    factor = torch.tensor([1.0, 0.3, 2.0], device=DEV)
    for step in range(3):
        before, m0 = X.clone(), opt.m.clone()
        opt.step(0.02, factor)
        opt.status()
        want, m = want_step(before, m0, G, layer_off, shapes, opt.offsets, factor, 0.02, 0.1, 0.9, nesterov)
        # m: two roundings; x: that of the result, and those of O, of which 0.02 s is taken (x has 0.05, O up to 1/sqrt(9))
        assert float((opt.m.double() - m).abs().max()) <= 4 * 2.0 ** -24 * float(m[~gaps].abs().max())
        o = 0.02 * 5 * most_off(3 if x != BF16 else 1, 5, F32)
        assert float((X.double() - want).abs().max()) <= torch.finfo(x).eps / 2 * float(want.abs().max()) + o
        touched = torch.zeros(X.shape[1], dtype=torch.bool, device=DEV)
        for k, s in enumerate(shapes):
            if s:
                touched[layer_off[k]:layer_off[k + 1]] = True
        assert torch.equal(X[:, ~touched], before[:, ~touched])
        assert torch.equal(opt.m[gaps], torch.full_like(opt.m[gaps], 123.0))
        if C is not None:
            assert float((C[:, touched].double() - want[:, touched]).abs().max()) <= torch.finfo(C.dtype).eps / 2 * float(want.abs().max()) + o
            assert torch.equal(C[:, ~touched], torch.zeros_like(C[:, ~touched]))
        G.copy_(G.flip(0))
    opt.close()


@pytest.mark.parametrize("bad", [float("inf"), float("nan"), float("-inf")])
def test_a_worker_whose_factor_is_no_number_is_left_as_it_is(bad):
    gen = torch.Generator(device=DEV).manual_seed(10)
    X, G, layer_off, shapes, C = network(3, gen, copy=BF16)
    G[1] = float("nan")
    opt = choco.Muon(X, G, layer_off, shapes, weight_decay=0.1, copy=C)
    opt.m.normal_(generator=gen)
    x0, m0 = X.clone(), opt.m.clone()
    opt.step(0.1, torch.tensor([1.0, bad, 0.5], device=DEV))
    per = len([s for s in shapes if s])
    here = slice(int(opt.offsets[per]), int(opt.offsets[2 * per]))
    assert torch.equal(X[1], x0[1]) and torch.equal(opt.m[here], m0[here]) and not C[1].any()
    assert X[[0, 2]].isfinite().all() and not torch.equal(X[0], x0[0]) and not torch.equal(X[2], x0[2])
    opt.close()


def test_captured_steps():
    """Replays take the momentum further, and two handles' graphs on one stream do not disturb each other."""
    gen = torch.Generator(device=DEV).manual_seed(11)
    X, G, layer_off, shapes, _ = network(2, gen)
    runs = []
    for captured in (False, True):
        xs, opts = [X.clone(), X.clone() * 2], []
        for x in xs:
            opts.append(choco.Muon(x, G, layer_off, shapes, weight_decay=0.01))
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            if captured:
                graphs = []
                for opt in opts:
                    graph = torch.cuda.CUDAGraph()
                    with torch.cuda.graph(graph, stream=side):
                        opt.step(0.02)
                    graphs.append(graph)
                for _ in range(3):
                    for graph in graphs:
                        graph.replay()
            else:
                for _ in range(3):
                    for opt in opts:
                        opt.step(0.02)
        torch.cuda.synchronize()
        runs.append([*xs, *(o.m.clone() for o in opts)])
        for opt in opts:
            opt.close()
    for a, b in zip(*runs):
        assert torch.equal(a, b)


def test_new_gradients():
    gen = torch.Generator(device=DEV).manual_seed(12)
    for shape in ((40, 64), (200, 260)):
        u, v = gradient(shape, gen), torch.empty(shape[0] * shape[1] + 1, device=DEV)[1:].view(shape)
        v.copy_(gradient(shape, gen))
        out = torch.empty(shape, device=DEV)
        o = choco.Orthogonalizer([u], [out])
        choco.choco_muon_set_grads(o.handle, [v.data_ptr()])
        o.apply()
        assert off(out, exact(v)) < most_off(3, 5, F32)
        with pytest.raises(choco.ChocoError):
            choco.choco_muon_set_grads(o.handle, [out.data_ptr()])   # what the call writes
        o.close()


def test_refusals():
    a, b = torch.zeros((8, 8), device=DEV), torch.zeros((8, 8), device=DEV)
    for ins, outs in (([a], [a]), ([a], [b[:, :4]]), ([a, b], [torch.empty_like(a), a]), ([a], [b.t()]), ([], []), ([a[0]], [b[0]]), ([a.double()], [b]),
                      ([a.cpu()], [b]), ([a, a], [b, b]), ([a], [a[1:]])):
        with pytest.raises(choco.ChocoError):
            choco.Orthogonalizer(ins, outs)
    X, G = torch.zeros((2, 20), device=DEV), torch.zeros((2, 20), device=DEV)
    for off_, shapes in (([0, 12, 20], [(3, 4)]), ([0, 12, 20], [(3, 5), None]), ([0, 12, 20], [None, None]), ([0, 12, 21], [(3, 4), None]), ([1, 13, 20], [(3, 4), None])):
        with pytest.raises(choco.ChocoError):
            choco.Muon(X, G, off_, shapes)
    with pytest.raises(choco.ChocoError):
        choco.Muon(X, X, [0, 20], [(4, 5)])
    opt = choco.Muon(X, G, [0, 20], [(4, 5)])
    for lr in (float("nan"), -1.0, float("inf"), 1e39):
        with pytest.raises(choco.ChocoError):
            opt.step(lr)
    with pytest.raises(choco.ChocoError):
        opt.step(0.1, torch.zeros(1, device=DEV))
    with pytest.raises(choco.ChocoError):
        choco.choco_muon_step(opt.handle, opt.m[:-1], 0.1)
    opt.step(0.0)
    assert not X.any()
    opt.close()


def test_empty_matrices():
    u, z = torch.ones((3, 4), device=DEV), torch.zeros((0, 4), device=DEV)
    out = torch.empty_like(u)
    o = choco.Orthogonalizer([z, u, torch.zeros((2, 5, 0), device=DEV)], [z.clone(), out, torch.zeros((2, 5, 0), device=DEV)])
    o.apply()
    assert off(out, exact(u)) < most_off(3, 5, F32)
    only = choco.Orthogonalizer([z], [z.clone()])
    only.apply()
    only.status()
