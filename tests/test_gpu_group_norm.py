"""Group norm with an activation and its gradients against the formulas in float64."""
import math

import pytest
import torch

import paper_1907_09356_b200 as choco

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
EPS = 1e-5


def act(z, kind):
    return {"none": lambda: z, "relu": lambda: z.clamp(min=0), "silu": lambda: z * torch.sigmoid(z), "gelu": lambda: z * torch.special.ndtr(z)}[kind]()


def statistics(x, groups):
    g = x.double().unflatten(-1, (groups, -1))
    var, mean = torch.var_mean(g, dim=(2, 4), correction=0)
    return mean, 1 / torch.sqrt(var + EPS)


def normalized(x, mean, rstd):
    spread = lambda t: t.double().repeat_interleave(x.shape[-1] // t.shape[-1], dim=-1)[:, :, None]  # noqa: E731
    return (x.double() - spread(mean)) * spread(rstd)


def forward(x, w, b, groups, kind):
    """(y, mean, rstd) in float64, x [n, images, pixels, channels]."""
    mean, rstd = statistics(x, groups)
    per = lambda t: t.double()[:, None, None]  # noqa: E731
    return act(normalized(x, mean, rstd) * per(w) + per(b), kind), mean, rstd


def close(got, want, unit, scale=None):
    """Within `unit` of the value or of the array's mean size, whichever is larger."""
    want = want.double()
    size = want.abs().clamp(min=float(want.square().mean().sqrt())) if scale is None else scale
    assert got.isfinite().all()
    assert float(((got.double() - want).abs() / size).max()) < unit


@pytest.mark.parametrize("kind", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("shape,groups", [((2, 3, 49, 64), 16), ((1, 1, 1024, 16), 4), ((3, 2, 100, 15), 5)])
def test_forward(shape, groups, kind):
    gen = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn(shape, generator=gen, device=DEV) * 2 + 1
    w, b = torch.randn((shape[0], shape[3]), generator=gen, device=DEV), torch.randn((shape[0], shape[3]), generator=gen, device=DEV)
    y, mean, rstd = torch.empty_like(x), torch.empty((*shape[:2], groups), device=DEV), torch.empty((*shape[:2], groups), device=DEV)
    gn = choco.GroupNorm(shape[0], shape[3], groups, activation=kind)
    gn.forward(x, w, b, y, mean, rstd)
    want = forward(x, w, b, groups, kind)
    # xhat is off by a few roundings of values up to about 4, and z by those of w xhat and b
    close(y, want[0], 64 * 2.0 ** -24)
    close(mean, want[1], 16 * 2.0 ** -24)
    close(rstd, want[2], 16 * 2.0 ** -24)
    gn.close()
