"""AdamW at the ends of the range: gradients with subnormal squares and an eps far below them, norms that float32
cannot hold."""
import numpy as np
import pytest
import torch

import paper_1907_09356_b200 as choco
from test_gpu_adamw import B1, B2, DEV, U

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [1e-30, 2.0 ** -126])
def test_gradients_with_subnormal_squares(bits, eps):
    """First step from zeroed moments: m / sqrt(v) is the sign, whatever the size, so x moves by -lr sign.  v is
    rounded to the subnormal grid, 2^-149 apart, twice; its root is off by half of that share of v, m and the
    quotient by the roundings of test_gpu_adamw or the approximations' 2^-22 each (four of them)."""
    d, lr = 1000, 1e-2
    gen = torch.Generator(device=DEV).manual_seed(1)
    size = torch.logspace(-19, -17, d, dtype=torch.float64, device=DEV)
    sign = torch.where(torch.rand(d, generator=gen, device=DEV) < 0.5, -1.0, 1.0)
    G = (size * sign).float()[None]
    X = torch.zeros((1, d), device=DEV)
    opt = choco.AdamW(X, G, [0, d], eps=eps, beta1=B1, beta2=B2, state_bits=bits)
    opt.step(lr)
    v = (1 - B2) * G.double() ** 2
    share = 0.5 * 2 * 2.0 ** -149 / v + 20 * U + (4 * 2.0 ** -22 if bits == 8 else 0.0)
    assert bool(((X.double() / (-lr * sign.double()) - 1).abs() <= 1.01 * share).all())
    for _ in range(3):
        opt.step(lr)
    assert bool(torch.isfinite(X).all()) and float(X.abs().max()) < 40 * lr   # nothing is divided by eps alone
    opt.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_the_smallest_eps_divides_zeros(bits):
    """m = v = 0 with the smallest eps allowed: 0 / eps is 0."""
    eps = 2.0 ** -126 if bits == 8 else 1e-44
    X = torch.ones((2, 700), device=DEV)
    G = torch.zeros((2, 700), device=DEV)
    G[1, ::3] = 1e-3
    opt = choco.AdamW(X, G, np.array([0, 300, 700]), eps=eps, state_bits=bits)
    for _ in range(3):
        opt.step(1e-2)
    assert bool((X[0] == 1).all()) and bool(torch.isfinite(X).all())
    still = torch.ones(700, dtype=torch.bool, device=DEV)
    still[::3] = False
    assert bool((X[1][still] == 1).all()) and bool((X[1][~still] < 1).all())
    opt.close()


def test_a_norm_beyond_float32_is_infinite_and_its_factor_nan():
    """Finite gradients whose norm only float64 can hold: the group sits the step out, as it does with infinite ones.
    One whose norm is just below float32's largest number, 3.4028e38, keeps its factor; unscale counts."""
    G = torch.zeros((4, 300), device=DEV)
    G[0, :2] = 3e38                                              # norm 4.2e38
    G[1, :2] = 2.4e38                                            # 3.394e38
    G[2, :] = 3e38                                               # 5.2e39, times unscale 1.3e39 and 5.2e37
    G[3, 7] = 1.0
    X = torch.ones((4, 300), device=DEV)
    opt = choco.AdamW(X, G, [0, 300])
    norm, factor = torch.zeros(4, device=DEV), torch.zeros(4, device=DEV)
    for unscale, over in ((1.0, [0, 2]), (0.25, [2]), (0.01, [])):
        opt.grad_norm(1.0, norm, factor, unscale)
        for k in range(4):
            want = float(G[k].double().norm()) * unscale
            if k in over:
                assert float(norm[k]) == float("inf") and bool(torch.isnan(factor[k]))
            else:
                assert abs(float(norm[k]) - want) <= 2 * U * want and bool(torch.isfinite(factor[k]))
        kept = X.clone()
        opt.step(1e-3, factor)
        for k in over:
            assert torch.equal(X[k], kept[k])
    opt.close()


def test_a_learning_rate_that_float32_cannot_hold_is_refused():
    X, G = torch.ones((1, 300), device=DEV), torch.ones((1, 300), device=DEV)
    opt = choco.AdamW(X, G, [0, 300])
    for lr in (1e39, 3.41e38, 1.7e308, -1.0, float("nan"), float("inf")):
        with pytest.raises(choco.ChocoError) as e:
            opt.step(lr)
        assert e.value.code == -1
    assert bool((X == 1).all()) and list(opt.get_steps()) == [0]
    opt.close()
