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
