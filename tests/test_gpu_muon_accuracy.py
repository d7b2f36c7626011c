"""How near Muon's products come to the formula in float64: bounds that tell three products from one, and sums that leave tensor
memory from sums that stay."""
import pytest
import torch

import paper_1907_09356_b200 as choco
from test_gpu_muon import BF16, DEV, F16, F32, USUAL, exact, gradient, off

pytestmark = pytest.mark.gpu


def most_off(u, steps=5):
    """Bound for three products, as 2-norm over the result's.  A step adds errors of e |X| to X (as 2-norms), which later steps magnify by
    the polynomial's largest slope, 3.4445, at most.  e: numbers of 22 bits (2^-22), and float32 sums that are cut towards
    zero, by half a unit (2^-24) of sums that are half as large on average, four times for every 64 of K, 1, 2 or 4 of which are
    added up before the sums are rounded: 2^-23 each."""
    x = u.double()
    x = x / torch.linalg.matrix_norm(x)
    x = x.mT if x.shape[0] > x.shape[1] else x
    k = x.shape[1]
    e = 2.0 ** -22 + (4 if k > 64 * 63 else 2 if k > 64 * 15 else 1) * 2.0 ** -23
    a, b, c = USUAL
    total = 0.0
    for step in range(steps + 1):
        size = float(x.norm())
        total += e * size * a ** (steps - step)
        if step < steps:
            s = x @ x.mT
            x = a * x + (b * s + c * s @ s) @ x
    return total / size


def orthogonalized(u, dtype=F32, **kw):
    out = torch.full(u.shape, float("nan"), dtype=dtype, device=DEV)
    o = choco.Orthogonalizer([u], [out], **kw)
    o.apply()
    o.status()
    o.close()
    return out


# in a block's shared memory; single blocks, X X^T whole and split along K; pairs, whole and split; K from 64 steps of 64 on
SHAPES = [(64, 576), (48, 100), (127, 129), (100, 700), (100, 3000), (3000, 100), (17, 5000), (128, 9000), (255, 257), (200, 2000), (650, 2600), (2600, 650), (260, 6000),
          (4096, 4096), (1100, 4200)]


@pytest.mark.parametrize("shape", SHAPES)
def test_three_products_carry_22_bits(shape):
    gen = torch.Generator(device=DEV).manual_seed(31)
    u = gradient(shape, gen)
    assert off(orthogonalized(u), exact(u)) < most_off(u) + 2.0 ** -24


@pytest.mark.parametrize("shape", [(64, 576), (100, 3000), (150, 260), (650, 2600), (300, 300)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_as_many_bits_as_float32_unless_asked_otherwise(shape, dtype):
    """Whatever the result's type: it is rounded once, at the end."""
    gen = torch.Generator(device=DEV).manual_seed(32)
    u = gradient(shape, gen, dtype=dtype)
    out = orthogonalized(u, dtype)
    assert torch.equal(out, orthogonalized(u, dtype, products=3))
    assert torch.equal(out, orthogonalized(u).to(dtype))
    # elements that the error b takes across the middle between two numbers of the type end one unit (eps) off: a share of 2 b / eps of
    # them at most, as numbers lie eps / 2 apart or more
    b, eps = most_off(u) + 2.0 ** -24, torch.finfo(dtype).eps
    assert off(out, exact(u).to(dtype)) < b + (min(1.0, 4 * b / eps)) ** 0.5 * eps


def test_one_product_when_asked():
    gen = torch.Generator(device=DEV).manual_seed(33)
    u = gradient((300, 700), gen)
    assert 1e-4 < off(orthogonalized(u, products=1), exact(u)) < 0.004


def test_updates_of_a_step():
    """x0 - x of a step that starts from zeros is lr s O, matrix by matrix."""
    gen = torch.Generator(device=DEV).manual_seed(34)
    shapes = [(64, 576), (100, 1500), (500, 333)]
    off_ = [0]
    for r, c in shapes:
        off_.append(off_[-1] + r * c)
    G = torch.cat([gradient(s, gen).flatten() for s in shapes])[None].repeat(2, 1)
    G[1] = G[1].flip(0)
    for dtype in (F32, BF16):
        X = torch.zeros(G.shape, dtype=dtype, device=DEV)
        opt = choco.Muon(X, G, off_, shapes, lr_scale=1.0, nesterov=False)
        opt.step(1.0)
        opt.status()
        for i in range(2):
            for k, s in enumerate(shapes):
                u = G[i, off_[k]:off_[k + 1]].view(s)
                got = -X[i, off_[k]:off_[k + 1]].view(s)
                b, eps = most_off(u) + 2.0 ** -22, torch.finfo(dtype).eps
                assert off(got, exact(u).to(dtype)) < b + (min(1.0, 4 * b / eps)) ** 0.5 * eps
        opt.close()
