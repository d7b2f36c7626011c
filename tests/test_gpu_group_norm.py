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
    close(mean, want[1], 16 * 2.0 ** -24, want[1].abs() + 1 / want[2])
    close(rstd, want[2], 16 * 2.0 ** -24)
    gn.close()


def gradients(x, dy, w, b, mean, rstd, kind):
    """(dx, dw, db) in float64 from the statistics as they are given, x and dy [n, images, pixels, channels]."""
    groups = mean.shape[-1]
    xhat = normalized(x, mean, rstd)
    per = lambda t: t.double()[:, None, None]  # noqa: E731
    z = (per(w) * xhat + per(b))
    s = torch.sigmoid(z)
    slope = {"none": lambda: torch.ones_like(z), "relu": lambda: (z > 0).double(), "silu": lambda: s + z * s * (1 - s),
             "gelu": lambda: torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)}[kind]()
    dz = dy.double() * slope
    db, dw = dz.sum((1, 2)), (dz * xhat).sum((1, 2))
    dz = dz * per(w)
    split = lambda t: t.unflatten(-1, (groups, -1))  # noqa: E731
    over = lambda t: split(t).mean((2, 4)).repeat_interleave(x.shape[-1] // groups, dim=-1)[:, :, None]  # noqa: E731
    scale = rstd.double().repeat_interleave(x.shape[-1] // groups, dim=-1)[:, :, None]
    return (dz - over(dz) - xhat * over(dz * xhat)) * scale, dw, db


def inputs(shape, gen, x=F32, y=F32, param=F32, pitch=0, offset=0.5):
    n, images, pixels, c = shape
    wide = lambda t: torch.zeros((n, images, pixels, c + pitch), dtype=t, device=DEV)[..., pitch // 2:pitch // 2 + c]  # noqa: E731
    a, dy = wide(x), wide(y)
    v = torch.randn(shape, generator=gen, device=DEV) * (torch.rand(c, generator=gen, device=DEV) + 0.5) + torch.randn(c, generator=gen, device=DEV) * offset
    a.copy_(v)
    dy.copy_(torch.randn(shape, generator=gen, device=DEV))
    row = torch.randn((n, 2 * c + 3), generator=gen, device=DEV).to(param)
    return a, dy, row[:, :c], row[:, c:2 * c], wide(y), wide(x)


def run(gn, a, dy, w, b, y, dx, groups, kind, add=None):
    """Both directions, compared with the formulas."""
    n, images, pixels, c = a.shape
    mean, rstd = torch.empty((n, images, groups), device=DEV), torch.empty((n, images, groups), device=DEV)
    one = torch.ones((n, c), device=DEV)
    wv, bv = one if w is None else w, one * 0 if b is None else b
    gn.forward(a, w, b, y, mean, rstd)
    want = forward(a, wv, bv, groups, kind)
    unit = lambda t: torch.finfo(t).eps / 2  # noqa: E731
    # float32 inside: xhat off by some roundings of |x - mean| rstd, of which there are up to about 6
    inside = 2.0 ** -18
    close(y, want[0], unit(y.dtype) + inside)
    # the mean is p + sum(x - p) / N with p a value of the channel: its roundings are units of |x - p|, that is of the deviation, and of the
    # mean itself, however near to 0 that is
    close(mean, want[1], 2.0 ** -20, want[1].abs() + 1 / want[2])
    close(rstd, want[2], 2.0 ** -20)
    G = torch.zeros((n, 2 * c + 5), device=DEV) if add is None else torch.randn((n, 2 * c + 5), device=DEV).to(add)
    dw, db, G0 = G[:, 2:2 + c], G[:, 2 + c:2 + 2 * c], G.clone()
    gn.backward(a, dy, w, b, mean, rstd, dx, dw, db, accumulate=add is not None)
    gx, gw, gb = gradients(a, dy, wv, bv, mean, rstd, kind)
    if pixels * c // groups >= 16:          # (of fewer values dx all but cancels)
        close(dx, gx, unit(dx.dtype) + 4 * inside)
    # sums of images x pixels terms of size 1: float32 partial sums of a few hundred, joined in float64
    total = float(images * pixels) ** 0.5
    for got, wanted, before in ((dw, gw, G0[:, 2:2 + c]), (db, gb, G0[:, 2 + c:2 + 2 * c])):
        wanted = wanted + (before.double() if add is not None else 0)
        assert float((got.double() - wanted).abs().max()) < 2.0 ** -19 * 4 * total + unit(got.dtype) * float(wanted.abs().max())
    assert torch.equal(G[:, :2], G0[:, :2]) and torch.equal(G[:, 2 + 2 * c:], G0[:, 2 + 2 * c:])
    return mean, rstd


SHAPES = [((1, 1, 1, 1), 1), ((2, 3, 1, 8), 8), ((2, 2, 1, 64), 4), ((1, 2, 49, 2048), 32), ((2, 1, 7, 96), 32), ((3, 2, 100, 15), 5), ((1, 3, 64, 33), 1), ((2, 2, 50, 66), 11),
          ((1, 1, 5000, 8), 2), ((1, 2, 33, 2048), 1), ((1, 2, 20, 2047), 1), ((2, 1, 12544, 16), 16), ((1, 1, 3, 4096), 64), ((1, 2, 300, 1200), 4), ((9, 5, 64, 64), 16)]


@pytest.mark.parametrize("kind", ["relu", "silu"])
@pytest.mark.parametrize("shape,groups", SHAPES)
def test_shapes(shape, groups, kind):
    gen = torch.Generator(device=DEV).manual_seed(2)
    gn = choco.GroupNorm(shape[0], shape[3], groups, max_images=shape[1], activation=kind)
    for x in (F32, BF16):
        run(gn, *inputs(shape, gen, x, x), groups, kind)
    gn.close()


@pytest.mark.parametrize("x", [F32, BF16, F16])
@pytest.mark.parametrize("y", [F32, BF16, F16])
@pytest.mark.parametrize("kind", ["none", "relu", "silu", "gelu"])
def test_types(x, y, kind):
    gen = torch.Generator(device=DEV).manual_seed(3)
    for shape, groups in (((2, 2, 70, 40), 5), ((2, 2, 30, 21), 7)):
        for param in (F32, x):
            gn = choco.GroupNorm(shape[0], shape[3], groups, max_images=2, activation=kind)
            run(gn, *inputs(shape, gen, x, y, param), groups, kind, add=None if param == F32 else y)
            gn.close()


@pytest.mark.parametrize("pitch", [2, 8, 13, 64])
@pytest.mark.parametrize("x", [F32, F16])
def test_channels_of_wider_arrays(x, pitch):
    """What lies between the channels that are meant is neither read nor written."""
    gen = torch.Generator(device=DEV).manual_seed(4)
    shape, groups = (2, 2, 60, 32), 8
    gn = choco.GroupNorm(2, 32, groups, max_images=2, activation="relu")
    a, dy, w, b, y, dx = inputs(shape, gen, x, x, F32, pitch)
    for t in (a, dy, y, dx):
        t._base[..., :pitch // 2] = float("nan")
        t._base[..., pitch // 2 + 32:] = float("nan")
    run(gn, a, dy, w, b, y, dx, groups, "relu")
    for t in (y, dx):
        assert t._base[..., :pitch // 2].isnan().all() and t._base[..., pitch // 2 + 32:].isnan().all()
    gn.close()


def test_images_larger_than_what_a_cluster_keeps():
    gen = torch.Generator(device=DEV).manual_seed(5)
    for shape, groups, x in (((1, 2, 40_000, 64), 1, F32), ((1, 1, 100_000, 48), 2, BF16), ((1, 1, 50_001, 33), 1, F16)):
        gn = choco.GroupNorm(1, shape[3], groups, max_images=2, activation="relu")
        run(gn, *inputs(shape, gen, x, x), groups, "relu")
        gn.close()


@pytest.mark.parametrize("offset", [30.0, 1000.0])
def test_means_far_from_zero(offset):
    """x = offset + noise: the statistics lose nothing that x has."""
    gen = torch.Generator(device=DEV).manual_seed(6)
    shape, groups = (1, 2, 500, 32), 8
    x = torch.randn(shape, generator=gen, device=DEV) + offset
    mean, rstd = torch.empty((1, 2, groups), device=DEV), torch.empty((1, 2, groups), device=DEV)
    y = torch.empty_like(x)
    gn = choco.GroupNorm(1, 32, groups)
    gn.forward(x, None, None, y, mean, rstd)
    want = forward(x, torch.ones((1, 32), device=DEV), torch.zeros((1, 32), device=DEV), groups, "none")
    close(mean, want[1], 2.0 ** -22, want[1].abs() + 1 / want[2])
    close(rstd, want[2], 2.0 ** -20)
    # the mean is rounded to float32 before it is taken away: half a unit of it, in units of the deviation (which is 1)
    close(y, want[0], 2.0 ** -18 + offset * 2.0 ** -24)
    gn.close()


def test_constant_images_and_no_parameters():
    x = torch.full((2, 2, 10, 16), 3.0, device=DEV)
    x[1] = -7.25
    y, mean, rstd = torch.empty_like(x), torch.empty((2, 2, 4), device=DEV), torch.empty((2, 2, 4), device=DEV)
    gn = choco.GroupNorm(2, 16, 4, max_images=2, eps=0.25)
    gn.forward(x, None, None, y, mean, rstd)
    assert torch.equal(mean[0], torch.full_like(mean[0], 3.0)) and torch.equal(mean[1], torch.full_like(mean[1], -7.25))
    assert torch.equal(rstd, torch.full_like(rstd, 2.0)) and not y.any()
    gen = torch.Generator(device=DEV).manual_seed(7)
    a, dy, w, b, y, dx = inputs((2, 2, 40, 16), gen)
    other = choco.GroupNorm(2, 16, 4, max_images=2, activation="silu")
    for weight, bias in ((None, None), (w, None), (None, b)):
        run(other, a, dy, weight, bias, y, dx, 4, "silu")
    shared = w[:1].expand(2, 16)                                     # one scale for all workers
    run(other, a, dy, shared, shared, y, dx, 4, "silu")
    for g in (gn, other):
        g.close()


def test_several_axes_of_pixels_and_missing_outputs():
    gen = torch.Generator(device=DEV).manual_seed(8)
    a, dy, w, b, y, dx = inputs((2, 3, 35, 24), gen)
    gn = choco.GroupNorm(2, 24, 6, max_images=3, activation="gelu")
    mean, rstd = run(gn, a, dy, w, b, y, dx, 6, "gelu")
    y2, dx2 = torch.empty((2, 3, 5, 7, 24), device=DEV), torch.empty((2, 3, 7, 5, 24), device=DEV).transpose(2, 3).contiguous()
    square = lambda t: t.unflatten(2, (5, 7))  # noqa: E731
    gn.forward(square(a), w, b, y2)                                   # inference: no statistics kept
    assert torch.equal(y2.flatten(2, 3), y)
    dw, db = torch.empty((2, 24), device=DEV), torch.empty((2, 24), device=DEV)
    gn.backward(square(a), square(dy), w, b, mean, rstd, dx2, None, None)
    assert torch.equal(dx2.flatten(2, 3), dx)
    gn.backward(a, dy, w, b, mean, rstd, None, dw, None)
    gn.backward(a, dy, w, b, mean, rstd, None, None, db)
    _, gw, gb = gradients(a, dy, w, b, mean, rstd, "gelu")
    close(dw, gw, 2.0 ** -16)
    close(db, gb, 2.0 ** -16)
    gn.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_in_place(dtype):
    gen = torch.Generator(device=DEV).manual_seed(9)
    for shape, groups in (((2, 3, 3000, 64), 8), ((1, 1, 40_000, 64), 1)):
        a, dy, w, b, y, dx = inputs(shape, gen, dtype, dtype)
        gn = choco.GroupNorm(shape[0], 64, groups, max_images=3, activation="relu")
        mean, rstd = run(gn, a, dy, w, b, y, dx, groups, "relu")
        same = a.clone()
        gn.forward(same, w, b, same)
        assert torch.equal(same, y)
        for over in (dy, a):
            x_, dy_ = a.clone(), dy.clone()
            to = dy_ if over is dy else x_
            gn.backward(x_, dy_, w, b, mean, rstd, to, None, None)
            assert torch.equal(to, dx)
        gn.close()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_relu_is_open_where_z_of_these_statistics_is(dtype):
    """z within float32's roundings of 0 and exactly 0, with scales of both signs and of 0."""
    gen = torch.Generator(device=DEV).manual_seed(10)
    n, images, pixels, c, groups = 2, 2, 400, 32, 8
    x = torch.randn((n, images, pixels, c), generator=gen, device=DEV).to(dtype)
    mean, rstd = (t.float() for t in statistics(x, groups))
    w = torch.randn((n, c), generator=gen, device=DEV)
    w[:, 3], w[:, 7] = 0, -0.0
    # borders at values that x has: z = 0 there up to the rounding of b, on one side or the other
    pick = x[:, 0, 5].double()
    spread = lambda t: t[:, 0].double().repeat_interleave(c // groups, dim=-1)  # noqa: E731
    b = (-(pick - spread(mean)) * spread(rstd) * w.double()).float()
    b[:, 7] = 1.0
    b[:, 11], mean[:, :, 11 // (c // groups)] = 0.0, x[:, :, 9, 11].float()  # z = 0 exactly
    dy = torch.ones_like(x)
    dw, db = torch.empty((n, c), device=DEV), torch.empty((n, c), device=DEV)
    gn = choco.GroupNorm(n, c, groups, max_images=images, activation="relu")
    gn.backward(x, dy, w, b, mean, rstd, None, dw, db)
    want = gradients(x, dy, w, b, mean, rstd, "relu")[2]
    assert torch.equal(db.double(), want)                            # whole numbers: how many are open
    assert 0 < float(want[:, 7].min()) == images * pixels and float(want[:, 3].max()) in (0.0, float(images * pixels))
    gn.close()


@pytest.mark.parametrize("kind", ["none", "silu", "gelu", "relu"])
def test_gradients_against_differences(kind):
    """Along random directions the loss <r, y> changes as dx, dw and db say (differences of the formula in float64)."""
    gen = torch.Generator(device=DEV).manual_seed(11)
    shape, groups = (2, 2, 60, 12), 3
    x, r, w, b, y, dx = inputs(shape, gen)
    if kind == "relu":                                               # away from the border, where there is no derivative
        b.copy_(torch.where(b > 0, 9.0, -9.0))
        b[:, 0] = 0.3
    mean, rstd = torch.empty((2, 2, groups), device=DEV), torch.empty((2, 2, groups), device=DEV)
    dw, db = torch.empty((2, 12), device=DEV), torch.empty((2, 12), device=DEV)
    gn = choco.GroupNorm(2, 12, groups, max_images=2, activation=kind)
    gn.forward(x, w, b, y, mean, rstd)
    gn.backward(x, r, w, b, mean, rstd, dx, dw, db)
    loss = lambda xx, ww, bb: float((forward(xx, ww, bb, groups, kind)[0] * r.double()).sum())  # noqa: E731
    h = 1e-6
    for which, grad in ((0, dx), (1, dw), (2, db)):
        args = [x.double(), w.double(), b.double()]
        v = torch.randn(args[which].shape, generator=gen, device=DEV, dtype=torch.float64)
        up, down = list(args), list(args)
        up[which], down[which] = args[which] + h * v, args[which] - h * v
        slope = (loss(*up) - loss(*down)) / (2 * h)
        size = float((grad.double().norm() * v.norm()))
        # differences: h^2 of a third derivative and 1e-16 / h of the loss; float32 gradients: 2^-16 of their size
        assert abs(slope - float((grad.double() * v).sum())) < 2e-5 * size + 1e-5
    gn.close()


def test_what_is_no_number_stays_in_its_group():
    gen = torch.Generator(device=DEV).manual_seed(12)
    shape, groups = (2, 3, 50, 16), 4
    x, dy, w, b, y, dx = inputs(shape, gen)
    x[0, 1, 7, 5], x[1, 0, 3, 0] = float("nan"), float("inf")
    mean, rstd = torch.empty((2, 3, groups), device=DEV), torch.empty((2, 3, groups), device=DEV)
    gn = choco.GroupNorm(2, 16, groups, max_images=3, activation="relu")
    gn.forward(x, w, b, y, mean, rstd)
    bad = torch.zeros((2, 3, 50, 16), dtype=torch.bool, device=DEV)
    bad[0, 1, :, 4:8] = bad[1, 0, :, 0:4] = True
    assert y[bad].isnan().all() and y[~bad].isfinite().all()
    gn.backward(x, dy, w, b, mean, rstd, dx, None, None)
    assert dx[~bad].isfinite().all() and not dx[bad].isfinite().any()
    gn.close()


def test_same_bits_every_time_captured_and_on_another_stream():
    gen = torch.Generator(device=DEV).manual_seed(13)
    for shape, groups, dtype in (((2, 4, 3136, 64), 32, BF16), ((3, 5, 64, 24), 8, F32)):
        x, dy, w, b, y, dx = inputs(shape, gen, dtype, dtype)
        c = shape[3]
        gn = choco.GroupNorm(shape[0], c, groups, max_images=shape[1], activation="silu")

        def calls(stream=None):
            out = [torch.empty_like(x), torch.empty((*shape[:2], groups), device=DEV), torch.empty((*shape[:2], groups), device=DEV), torch.empty_like(x),
                   torch.ones((shape[0], c), device=DEV), torch.ones((shape[0], c), device=DEV)]
            torch.cuda.synchronize()
            gn.forward(x, w, b, out[0], out[1], out[2], stream=stream)
            gn.backward(x, dy, w, b, out[1], out[2], out[3], out[4], out[5], accumulate=True, stream=stream)
            return out
        want = calls()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        for _ in range(3):
            for a, e in zip(calls(side), want):
                side.synchronize()
                assert torch.equal(a, e)
        graph = torch.cuda.CUDAGraph()
        out = [torch.empty_like(t) for t in want]
        with torch.cuda.graph(graph, stream=side):
            gn.forward(x, w, b, out[0], out[1], out[2])
            gn.backward(x, dy, w, b, out[1], out[2], out[3], out[4], out[5], accumulate=True)
        out[4].fill_(1.0)
        out[5].fill_(1.0)
        graph.replay()
        torch.cuda.synchronize()
        for a, e in zip(out, want):
            assert torch.equal(a, e)
        gn.close()


def test_sizes_of_zero():
    gn = choco.GroupNorm(2, 8, 2, max_images=4, activation="relu")
    for shape in ((2, 0, 5, 8), (2, 3, 0, 8)):
        x = torch.zeros(shape, device=DEV)
        stats = torch.zeros((2, shape[1], 2), device=DEV)
        gn.forward(x, None, None, x.clone(), stats, stats.clone())
        dw = torch.full((2, 8), 3.0, device=DEV)
        gn.backward(x, x, None, None, stats, stats, x.clone(), dw, None, accumulate=True)
        assert torch.equal(dw, torch.full_like(dw, 3.0))
        gn.backward(x, x, None, None, stats, stats, x.clone(), dw, None)
        assert not dw.any()
    gn.close()


def test_refusals():
    gn = choco.GroupNorm(2, 8, 2, max_images=2, activation="relu")
    x, y = torch.zeros((2, 2, 6, 8), device=DEV), torch.zeros((2, 2, 6, 8), device=DEV)
    w, s = torch.zeros((2, 8), device=DEV), torch.zeros((2, 2, 2), device=DEV)
    flat = torch.zeros(2 * 2 * 6 * 8 + 8, device=DEV)
    shifted = flat[8:].view(2, 2, 6, 8)
    bad_forward = [
        (x, w, w, y[:, :1], s, s), (x[..., :4], w, w, y[..., :4], s, s), (x, w[:, :4], w, y, s, s), (x, w, w[:1], y, s, s), (x, w, w.half(), y, s, s),
        (x, w, w, y, s[:, :1], s), (x, w, w, y, s.double(), s), (x.cpu(), w, w, y, s, s), (x, w, w, y.cpu(), s, s), (x, w.cpu(), w, y, s, s), (x.double(), w, w, y, s, s),
        (flat[:-8].view(2, 2, 6, 8), w, w, shifted, s, s), (x, w, w, x[:, :1].expand(2, 2, 6, 8), s, s), (x.transpose(2, 3), w, w, y, s, s),
        (x, w, w, torch.zeros((2, 2, 6, 8), device=DEV).as_strided((2, 2, 6, 8), (96, 48, 4, 1)), s, s), (x[0], w, w, y[0], s, s)]
    for args in bad_forward:
        with pytest.raises(choco.ChocoError):
            gn.forward(*args)
    big = torch.zeros((2, 3, 6, 8), device=DEV)
    bad_backward = [
        (x, y[:, :1], w, w, s, s, None, w, w), (x, y, w, w, None, s, None, w, w), (x, y, w, w, s, s, torch.zeros_like(x).half(), w, w),
        (x, y, w, w, s, s, None, w[:, :4], w), (x, y, w, w, s, s, None, w[:1].expand(2, 8), None), (flat[:-8].view(2, 2, 6, 8), y, w, w, s, s, shifted, None, None),
        (big, big, w, w, torch.zeros((2, 3, 2), device=DEV), torch.zeros((2, 3, 2), device=DEV), None, w, w)]      # more than max_images
    for args in bad_backward:
        with pytest.raises(choco.ChocoError):
            gn.backward(*args)
    for kw in (dict(groups=3), dict(groups=0), dict(channels=0), dict(n=0), dict(max_images=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(activation="tanh"),
               dict(channels=4096, groups=1), dict(channels=1 << 21, groups=1 << 20), dict(n=70000)):
        with pytest.raises(choco.ChocoError):
            choco.GroupNorm(**{**dict(n=2, channels=8, groups=2), **kw})
    gn.forward(x, w, w, y, s, s.clone())                              # and in order
    gn.close()


def test_two_sets_of_channels_of_one_array():
    """y behind x in the same pixels, as a network's concatenated features are."""
    gen = torch.Generator(device=DEV).manual_seed(14)
    both = torch.randn((2, 2, 30, 32), generator=gen, device=DEV)
    x, y = both[..., :16], both[..., 16:]
    x0 = x.clone()
    gn = choco.GroupNorm(2, 16, 4)
    gn.forward(x, None, None, y)
    want = forward(x0, torch.ones((2, 16), device=DEV), torch.zeros((2, 16), device=DEV), 4, "none")[0]
    close(y, want, 2.0 ** -18)
    assert torch.equal(x, x0)
    gn.close()
