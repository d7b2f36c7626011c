"""AdamW over tensor lists, its 8-bit moments and the gradient norms, against 64-bit arithmetic.

Tolerances, from the order of operations choco.h gives; U = 2^-24, w the parameter type's rounding.
  m: every term is a product of rounded factors:        4 U (|b1 m| + |(1 - b1) g'|)            =: em
  v: at most six roundings of non-negative terms:       6 U v
  x: the quotient's denominator is off by at most 8 U, so the step is off by
     em / den * size + 12 U |m / den| size, the decay by 7 U |x lr wd|, and the sum is rounded to
     float32 and to the type: (w + U) |x|.
Products of roundings are covered by a factor of 1.01.  A code k of 8 bits is the nearest on the scale
of square roots: half a step, 0.5 / 127 sqrt(a), plus 0.001 steps for the roundings of y (a few U
times at most 255) plus what em moves the root by, at most sqrt(em).
"""
import ctypes

import numpy as np
import pytest
import torch

import paper_1907_09356_b200 as choco
import workloads

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
W = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
B1, B2, EPS = 0.9, 0.999, 1e-8
BLOCK = choco.ADAMW_BLOCK


def values(code, scale, kind):
    k = code.double().view(-1, BLOCK)
    r = k * k.abs() * scale.double()[:, None]
    return (r if kind == "m" else r * r).view(-1)


class Run:
    """Rows of X and G cut into layers, with everything a step needs; ref() gives the step in 64 bits."""

    def __init__(self, n, sizes, bits=32, x=F32, g=F32, copy=None, head=0, decay=None, lr_scale=None, seed=1, gsd=1e-2, step=0):
        self.n, self.sizes, self.bits, self.copy = n, list(sizes), bits, None
        off = workloads.layer_offsets(sizes)
        self.off, d = off, int(off[-1])
        gen = torch.Generator(device=DEV).manual_seed(seed)
        rnd = lambda *s: torch.randn(s, generator=gen, device=DEV)  # noqa: E731
        pad = lambda dt: torch.full((n, d + head + 3), 9.0, dtype=dt, device=DEV)  # noqa: E731
        self.Xs, self.Gs = pad(x), pad(g)
        self.X, self.G = self.Xs[:, head:], self.Gs[:, head:]
        self.X[:, :d] = rnd(n, d).to(x)
        self.G[:, :d] = (gsd * rnd(n, d)).to(g)
        if copy is not None:
            self.copys = pad(copy)
            self.copy = self.copys[:, head:]
        L = len(sizes)
        self.decay = np.asarray([0.1 * (i % 2) for i in range(L)] if decay is None else decay, dtype=np.float64)
        self.lr_scale = np.asarray([1.0 + (i % 3) for i in range(L)] if lr_scale is None else lr_scale, dtype=np.float64)
        self.opt = choco.AdamW(self.X, self.G, off, self.decay, self.lr_scale, self.copy, B1, B2, EPS, bits, step=step)
        self.e = self.opt.elements
        where = [self.opt.offsets[i * L + l] + np.arange(sizes[l]) for i in range(n) for l in range(L)]
        self.where = torch.from_numpy(np.concatenate(where).astype(np.int64)).to(DEV)   # coordinate -> place in m, v
        self.d = d
        self.wd = torch.from_numpy(np.repeat(self.decay, sizes)).to(DEV)
        self.ls = torch.from_numpy(np.repeat(self.lr_scale, sizes)).to(DEV)

    def moments(self):
        if self.bits == 32:
            return self.opt.m.double(), self.opt.v.double()
        return values(self.opt.m, self.opt.m_scale, "m"), values(self.opt.v, self.opt.v_scale, "v")

    def randomise(self, seed=3):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        live = torch.zeros(self.e, dtype=torch.bool, device=DEV)
        live[self.where] = True
        if self.bits == 32:
            self.opt.m.copy_(torch.randn(self.e, generator=gen, device=DEV) * 1e-2 * live)
            self.opt.v.copy_(torch.randn(self.e, generator=gen, device=DEV) ** 2 * 1e-4 * live)
        else:
            self.opt.m.copy_(torch.randint(-127, 128, (self.e,), generator=gen, device=DEV) * live)
            self.opt.v.copy_(torch.randint(0, 256, (self.e,), generator=gen, device=DEV) * live)
            self.opt.m_scale.copy_(torch.rand(self.e // BLOCK, generator=gen, device=DEV) * 1e-6)
            self.opt.v_scale.copy_(torch.rand(self.e // BLOCK, generator=gen, device=DEV) * 1e-7)

    def ref(self, lr, t, factor=None):
        """(x, m, v, em, bound of x) in 64 bits; t: one number or one per worker."""
        n, d = self.n, self.d
        m0, v0 = self.moments()
        m0, v0 = m0[self.where].view(n, d), v0[self.where].view(n, d)
        x, g = self.X[:, :d].double(), self.G[:, :d].double()
        if factor is not None:
            g = g * factor.double()[:, None]
        t = torch.as_tensor(t, dtype=torch.float64, device=DEV).expand(n)[:, None]
        m = B1 * m0 + (1 - B1) * g
        v = B2 * v0 + (1 - B2) * g * g
        em = 4 * U * ((B1 * m0).abs() + ((1 - B1) * g).abs())
        den = (v / (1 - B2 ** t)).sqrt() + EPS
        size = lr * self.ls / (1 - B1 ** t)
        new = x - (m / den * size + x * (lr * self.ls * self.wd))
        bound = em / den * size + 12 * U * (m / den).abs() * size + 7 * U * (x * lr * self.ls * self.wd).abs()
        return new, m, v, em, bound

    def check(self, before, want, workers=None):
        """The state now against ref()'s answer (for some workers, or for all)."""
        n, d = self.n, self.d
        x, m, v, em, bound = want
        rows = torch.arange(n, device=DEV) if workers is None else torch.as_tensor(workers, device=DEV)
        got = self.X[:, :d].double()
        w = W[self.X.dtype]
        sub = 6e-8 if self.X.dtype == F16 else 1e-38
        lim = 1.01 * (bound + (w + U) * x.abs()) + sub
        assert bool(((got - x).abs() <= lim)[rows].all()), float(((got - x).abs() / lim)[rows].max())
        if self.copy is not None:
            wc = W[self.copy.dtype]
            lim = 1.01 * (bound + (wc + U) * x.abs()) + 6e-8
            assert bool(((self.copy[:, :d].double() - x).abs() <= lim)[rows].all())
        gm, gv = (a[self.where].view(n, d) for a in self.moments())
        if self.bits == 32:
            assert bool(((gm - m).abs() <= 1.01 * em + 1e-44)[rows].all())
            assert bool(((gv - v).abs() <= 1.01 * 6 * U * v + 1e-44)[rows].all())
        else:
            self.check_codes(gm, gv, m, v, em, rows)
        # gaps and whatever surrounds the rows are untouched
        gap = torch.ones(self.e, dtype=torch.bool, device=DEV)
        gap[self.where] = False
        assert not bool(self.opt.m[gap].any()) and not bool(self.opt.v[gap].any())
        assert bool((self.Xs[:, d + self.X.storage_offset():] == 9.0).all())

    def check_codes(self, gm, gv, m, v, em, rows):
        n, d = self.n, self.d
        live = torch.zeros((n, d), dtype=torch.bool, device=DEV)
        live[rows] = True

        def padded(a):
            p = torch.zeros(self.e, dtype=torch.float64, device=DEV)
            p[self.where] = a.reshape(-1)
            return p.view(-1, BLOCK)

        for got, want, err, levels in ((gm, m, em, 127), (gv.sqrt(), v.sqrt(), 4 * U * v.sqrt(), 255)):
            top = padded(want.abs()).max(1, keepdim=True).values
            g, a, e = padded(got), padded(want), padded(err)
            code = padded(live.double()) > 0
            lim = (0.5 + 1e-3) / levels * top.sqrt() + e.sqrt() + 1e-15
            if levels == 255:                                     # a small v keeps the code 1
                lim = torch.where((a > 0) & (g.sqrt() * levels <= 1.001 * top.sqrt()), lim * 2.01, lim)
            far = (g.abs().sqrt() - a.abs().sqrt()).abs() - lim
            assert bool((far[code] <= 0).all()), float(far[code].max())
            assert bool(((g * a >= 0) | (a.abs() <= e))[code].all())
            if levels == 255:
                assert bool((g[code & (a > 1e-22)] > 0).all())
        for scale, want, levels in ((self.opt.m_scale, m.abs(), 127), (self.opt.v_scale, v.sqrt(), 255)):
            top = padded(want).max(1).values.clamp(min=1e-30)
            own = (padded(live.double()) > 0).any(1)
            assert bool(((scale.double() * levels ** 2 - top).abs() <= 10 * U * top + 1e-36)[own].all())


RAGGED = [1, 2, 0, 255, 256, 257, 31, 2047, 2048, 2049, 8, 5000, 12]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("x,g,copy", [(F32, F32, None), (F32, BF16, BF16), (F32, F16, F16), (BF16, BF16, None), (F16, F32, None),
                                      (BF16, F32, F16)])
@pytest.mark.parametrize("head", [0, 1, 2, 4])
def test_step_types_sizes_and_alignments(bits, x, g, copy, head):
    r = Run(3, RAGGED, bits, x, g, copy, head, step=4)
    r.randomise()
    want = r.ref(1e-3, 5)
    r.opt.step(1e-3)
    r.check(None, want)
    r.opt.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_from_a_fresh_state(bits):
    r = Run(2, [300, 4096, 7], bits, copy=BF16)
    for t in range(1, 7):
        r.G[:, :r.d].normal_(0.0, 0.01, generator=torch.Generator(device=DEV).manual_seed(t))
        want = r.ref(2e-3, t)
        r.opt.step(2e-3)
        r.check(None, want)
    assert list(r.opt.get_steps()) == [6, 6]
    r.opt.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_vectors_of_whole_blocks(bits):
    """Aligned tensors of whole blocks (the fast path) beside unaligned ones in the same list."""
    r = Run(2, [256, 4096, 1 << 16, 3, 512, 2048], bits, step=9)
    r.randomise()
    want = r.ref(1e-3, 10)
    r.opt.step(1e-3)
    r.check(None, want)
    r.opt.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_zero_gradients_and_moments(bits):
    """0 / (0 + eps): nothing moves but the decay, and nothing is NaN; blocks of zeros keep codes 0."""
    r = Run(2, [300, 256], bits, decay=[0.1, 0.0])
    r.G.zero_()
    want = r.ref(1e-2, 1)
    r.opt.step(1e-2)
    r.check(None, want)
    assert not bool(r.opt.m.any()) and not bool(r.opt.v.any())
    r.opt.close()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("scale", [1e-12, 1e6])
def test_extreme_gradients(bits, scale):
    r = Run(2, [700, 256], bits, gsd=scale, step=2)
    want = r.ref(1e-3, 3)
    r.opt.step(1e-3)
    r.check(None, want)
    r.opt.close()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_groups_with_overflowed_gradients_sit_out(bits, bad):
    """Worker 1's gradient overflows in step 2: it keeps everything, its step number included, and its
    later steps use its own bias corrections."""
    r = Run(3, [300, 2049, 5], bits, copy=BF16)
    norm, factor = torch.zeros(3, device=DEV), torch.zeros(3, device=DEV)
    taken = [0, 0, 0]
    for t in range(1, 5):
        r.G[:, :r.d].normal_(0.0, 0.01, generator=torch.Generator(device=DEV).manual_seed(t))
        if t == 2:
            r.G[1, 2100] = bad
        r.opt.grad_norm(0.1, norm, factor)
        if t == 2:
            assert bool(torch.isnan(factor[1])) and bool(torch.isfinite(factor[[0, 2]]).all())
        kept = [a.clone() for a in (r.X, r.copy, *r.moments())]
        moving = [0, 2] if t == 2 else [0, 1, 2]
        want = r.ref(1e-3, [taken[i] + (i in moving) for i in range(3)], factor)
        r.opt.step(1e-3, factor)
        for i in moving:
            taken[i] += 1
        r.check(None, want, moving)
        if t == 2:
            L = len(r.sizes)
            own = slice(int(r.opt.offsets[L]), int(r.opt.offsets[2 * L]))
            assert torch.equal(r.X[1], kept[0][1]) and torch.equal(r.copy[1], kept[1][1])
            for a, b in zip(r.moments(), kept[2:]):
                assert torch.equal(a[own], b[own])
    assert list(r.opt.get_steps()) == taken == [4, 3, 4]
    r.opt.close()


def test_resume_gives_the_same_bits():
    for bits in (32, 8):
        a, b = Run(2, [500, 300], bits), Run(2, [500, 300], bits)
        grads = [torch.randn(a.G.shape, generator=torch.Generator(device=DEV).manual_seed(t), device=DEV) for t in range(6)]
        for t in range(6):
            a.G.copy_(grads[t])
            a.opt.step(1e-3)
        for t in range(3):
            b.G.copy_(grads[t])
            b.opt.step(1e-3)
        states = [s.clone() for s in (b.opt.m, b.opt.v, b.opt.m_scale, b.opt.v_scale) if s is not None]
        c = choco.AdamW(b.X, b.G, b.off, b.decay, b.lr_scale, beta1=B1, beta2=B2, eps=EPS, state_bits=bits, states=states)
        c.set_steps(b.opt.get_steps())
        for t in range(3, 6):
            b.G.copy_(grads[t])
            c.step(1e-3)
        assert torch.equal(a.X, b.X) and torch.equal(a.opt.m, c.m) and torch.equal(a.opt.v, c.v)
        for o in (a.opt, b.opt, c):
            o.close()


@pytest.mark.parametrize("g", [F32, BF16, F16])
@pytest.mark.parametrize("head", [0, 1, 2])
@pytest.mark.parametrize("sizes", [RAGGED, [1], [100_003], [16384, 16384 * 5 + 1, 3]])
def test_grad_norm(g, head, sizes):
    """Sums are exact to about 2^-50; what is left are the roundings of the results: 2 U, and for
    the factor the product with it."""
    r = Run(4, sizes, 32, F32, g, None, head)
    norm, factor = torch.zeros(4, device=DEV), torch.zeros(4, device=DEV)
    want = r.G[:, :r.d].double().norm(dim=1)
    for clip, unscale in ((0.25, 1.0), (0.0, 1.0), (1e9, 0.5), (0.25, 1.0 / 1024)):
        r.opt.grad_norm(clip, norm, factor, unscale)
        n = want * unscale
        f = unscale * (torch.clamp(clip / (n + 1e-6), max=1.0) if clip else torch.ones_like(n))
        assert bool(((norm.double() - n).abs() <= 2 * U * n).all())
        assert bool(((factor.double() - f).abs() <= 3 * U * f).all())
    r.opt.close()


def test_grad_norm_range():
    """Values whose squares leave float32's range, zeros, and infinities of one group only."""
    r = Run(4, [1000], 32)
    norm, factor = torch.zeros(4, device=DEV), torch.zeros(4, device=DEV)
    r.G[0] = 1e30
    r.G[1] = 1e-30
    r.G[2] = 0.0
    r.G[3, 5] = float("inf")
    r.opt.grad_norm(1.0, norm, factor)
    root = 1000 ** 0.5
    assert abs(float(norm[0]) / (1e30 * root) - 1) < 1e-6 and abs(float(norm[1]) / (1e-30 * root) - 1) < 1e-6
    assert float(norm[2]) == 0.0 and float(factor[1]) == 1.0 and float(factor[2]) == 1.0
    assert abs(float(factor[0]) * 1e30 * root - 1) < 1e-6
    assert float(norm[3]) == float("inf") and bool(torch.isnan(factor[3]))
    again = [norm.clone(), factor.clone()]
    r.opt.grad_norm(1.0, norm, factor)
    assert torch.equal(norm, again[0]) and torch.equal(factor[:3], again[1][:3])
    r.opt.close()


def test_norms_of_a_list_without_parameters():
    G = torch.randn((3, 1000), device=DEV)
    opt = choco.AdamW(None, G, [0, 400, 1000])
    norm, factor = torch.zeros(3, device=DEV), torch.zeros(3, device=DEV)
    opt.grad_norm(1.0, norm, factor)
    assert bool(((norm.double() - G.double().norm(dim=1)).abs() <= 2 * U * norm.double()).all())
    with pytest.raises(choco.ChocoError):
        opt.step(1e-3)
    opt.close()


def test_separate_tensors_groups_in_any_order_and_new_gradients():
    """Tensors that are no rows of one array, of mixed types, groups interleaved, one group empty."""
    gen = torch.Generator(device=DEV).manual_seed(1)
    shapes = [(40, 50), (7,), (300, 3), (1,), (128, 16)]
    types = [(F32, F32), (BF16, BF16), (F32, BF16), (F16, F32), (F32, F16)]
    group = [2, 0, 2, 0, 3]
    xs = [torch.randn(s, generator=gen, device=DEV).to(t[0]) for s, t in zip(shapes, types)]
    gs = [(torch.randn(s, generator=gen, device=DEV) * 0.01).to(t[1]) for s, t in zip(shapes, types)]
    rec = np.zeros(5, dtype=choco.ADAMW_TENSOR)
    for i in range(5):
        rec[i] = (xs[i].data_ptr(), gs[i].data_ptr(), 0, xs[i].numel(), choco._dtype(xs[i]), choco._dtype(gs[i]), 0, group[i],
                  0.05, 1.0)
    opt = choco.choco_adamw_init(rec, 4, B1, B2, EPS, 32)
    e, off = choco.choco_adamw_state_size(opt, 5)
    assert list(off) == [0, 2048, 2304, 3328, 3584] and e == 3584 + 2048
    m, v = torch.zeros(e, device=DEV), torch.zeros(e, device=DEV)
    norm, factor = torch.zeros(4, device=DEV), torch.zeros(4, device=DEV)
    for t in (1, 2):
        if t == 2:                                               # the gradients move to new arrays
            gs = [(g.double() * -3).to(g.dtype) for g in gs]
            choco.choco_adamw_set_grads(opt, [g.data_ptr() for g in gs])
        choco.choco_adamw_grad_norm(opt, 0.1, norm, factor)
        for k in range(4):
            want = torch.cat([gs[i].double().reshape(-1) for i in range(5) if group[i] == k] or [torch.zeros(1, device=DEV)]).norm()
            assert abs(float(norm[k]) - float(want)) <= 2 * U * float(want)
        old = [(x.double(), m[o:o + x.numel()].double(), v[o:o + x.numel()].double()) for x, o in zip(xs, off)]
        choco.choco_adamw_step(opt, m, v, None, None, 1e-2, factor)
        for i, (x0, m0, v0) in enumerate(old):
            g = gs[i].double().reshape(-1) * factor[group[i]].double()
            mn, vn = B1 * m0 + (1 - B1) * g, B2 * v0 + (1 - B2) * g * g
            step = (mn / (1 - B1 ** t)) / ((vn / (1 - B2 ** t)).sqrt() + EPS)
            want = x0.reshape(-1) - 1e-2 * (step + 0.05 * x0.reshape(-1))
            em = 4 * U * ((B1 * m0).abs() + ((1 - B1) * g).abs())
            lim = 1e-2 * (em / (mn.abs() + 1e-300) + 13 * U) * step.abs() + (W[xs[i].dtype] + 2 * U) * want.abs() + 6e-8 * (xs[i].dtype == F16)
            assert bool(((xs[i].double().reshape(-1) - want).abs() <= 1.01 * lim).all())
    assert list(choco.choco_adamw_get_steps(opt, 4)) == [2, 2, 2, 2]
    choco.choco_adamw_destroy(opt)


@pytest.mark.parametrize("bits", [32, 8])
def test_new_gradients_at_other_alignments(bits):
    """A gradient that moves to an address off a 16-byte boundary, and back: other accesses, same results."""
    r = Run(1, [5000], bits, step=1)
    r.randomise()
    store = torch.randn(5008, device=DEV)
    for shift in (0, 1, 2, 4, 3, 0):
        g = store[shift:shift + 5000]
        choco.choco_adamw_set_grads(r.opt.handle, [g.data_ptr()])
        r.G[0, :5000] = g                                        # what ref() looks at
        t = int(r.opt.get_steps()[0]) + 1
        want = r.ref(1e-3, t)
        r.opt.step(1e-3)
        r.check(None, want)
    norm, factor = torch.zeros(1, device=DEV), torch.zeros(1, device=DEV)
    r.opt.grad_norm(1.0, norm, factor)
    assert abs(float(norm) / float(store[:5000].double().norm()) - 1) <= 2 * U
    r.opt.close()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_read_state(bits, dtype):
    r = Run(2, [300, 4096, 7], bits, step=3)
    r.randomise()
    m, v = torch.empty(r.e, dtype=dtype, device=DEV), torch.empty(r.e, dtype=dtype, device=DEV)
    r.opt.read_state(m, v)
    for got, want in zip((m, v), r.moments()):
        assert bool(((got.double() - want).abs() <= (W[dtype] + 4 * U) * want.abs() + (6e-8 if dtype == F16 else 1e-38)).all())
    only = torch.empty(r.e, dtype=dtype, device=DEV)
    r.opt.read_state(None, only)
    assert torch.equal(only, v)
    r.opt.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_follows_a_run_in_64_bits(bits):
    """400 steps on a quadratic beside the formula in 64 bits.  With 32-bit moments a step is off by
    some 20 U of its size, so the loss after 400 of them by less than 400 * 2 * 20 U = 1e-3 of the start's.
    With 8 bits a moment is off by up to 1 / k of itself, a few per cent, one way as often as the
    other: the loss stays within twice that of the run in 64 bits."""
    n, d = 2, 3000
    X, G = torch.randn((n, d), device=DEV), torch.zeros((n, d), device=DEV)
    target = torch.randn((n, d), device=DEV)
    h = torch.rand((n, d), device=DEV) + 0.1
    opt = choco.AdamW(X, G, [0, 1000, d], state_bits=bits)
    x, m, v = X.double(), torch.zeros((n, d), dtype=torch.float64, device=DEV), torch.zeros((n, d), dtype=torch.float64, device=DEV)
    loss = lambda a: float((h.double() * (a.double() - target.double()) ** 2).sum())  # noqa: E731
    start = loss(X)
    for t in range(1, 401):
        lr = 0.02 * (1 - (t - 1) / 400)
        torch.mul(h, X - target, out=G)
        opt.step(lr)
        g = h.double() * (x - target.double())
        m, v = B1 * m + (1 - B1) * g, B2 * v + (1 - B2) * g * g
        x = x - lr * (m / (1 - B1 ** t)) / ((v / (1 - B2 ** t)).sqrt() + EPS)
    if bits == 32:
        assert abs(loss(X) - loss(x)) <= 1e-3 * start
    else:
        assert loss(X) <= 2 * loss(x)
    opt.close()


@pytest.mark.parametrize("bits", [8, 32])
def test_offsets_beyond_32_bits(bits):
    """One tensor of more than 2^32 elements (or, with 32-bit moments, bytes beyond 2^33): its last
    elements come out as those of a short tensor with the same values."""
    size = (1 << 32) + 1000 if bits == 8 else (1 << 31) + 1000
    tail = 1000 + 256
    X = torch.zeros((1, size), dtype=BF16, device=DEV)
    G = torch.zeros((1, size), dtype=BF16, device=DEV)
    X[0, -tail:] = torch.randn(tail, device=DEV)
    G[0, -tail:] = torch.randn(tail, device=DEV)
    x, g = X[:, -tail:].clone(), G[:, -tail:].clone()
    big = choco.AdamW(X, G, [0, size], weight_decay=0.1, state_bits=bits)
    small = choco.AdamW(x, g, [0, tail], weight_decay=0.1, state_bits=bits)
    norm, factor = torch.zeros(2, device=DEV), torch.zeros(2, device=DEV)
    big.grad_norm(1.0, norm[:1], factor[:1])
    small.grad_norm(1.0, norm[1:], factor[1:])
    assert abs(float(norm[0]) / float(norm[1]) - 1) < 4 * U
    for _ in range(2):
        big.step(1e-2, factor[1:])
        small.step(1e-2, factor[1:])
    assert torch.equal(X[:, -tail:], x)
    assert torch.equal(big.m[size - tail:size], small.m[:tail]) and torch.equal(big.v[size - tail:size], small.v[:tail])
    big.close()
    small.close()


def test_another_stream_and_capture():
    a, b = Run(2, [500, 300], 8, copy=BF16), Run(2, [500, 300], 8, copy=BF16)
    na, fa, nb, fb = (torch.zeros(2, device=DEV) for _ in range(4))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    a.opt.grad_norm(0.1, na, fa, stream=side)
    a.opt.step(1e-3, fa, stream=side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.opt.grad_norm(0.1, nb, fb)
        b.opt.step(1e-3, fb)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(na, nb) and torch.equal(a.X, b.X) and torch.equal(a.opt.m, b.opt.m) and torch.equal(a.copy, b.copy)
    a.opt.close()
    b.opt.close()


def test_refusals():
    r = Run(2, [300], 8)
    o, lib, h = r.opt, choco.load(), r.opt.handle
    p = lambda t: t.data_ptr()  # noqa: E731
    f = torch.ones(2, device=DEV)
    step = lambda **k: lib.choco_adamw_step(k.get("h", h), k.get("m", p(o.m)), k.get("v", p(o.v)), k.get("ms", p(o.m_scale)),  # noqa: E731
                                            k.get("vs", p(o.v_scale)), k.get("lr", 1e-3), k.get("f", p(f)), None)
    for bad in (dict(h=None), dict(m=None), dict(v=None), dict(ms=None), dict(vs=None), dict(lr=-1.0), dict(lr=float("nan"))):
        assert step(**bad) == -1, bad
    for bad in (dict(m=p(o.m) + 8), dict(v=p(o.v) + 1), dict(ms=p(o.m_scale) + 2), dict(f=p(f) + 1)):
        assert step(**bad) == -5, bad
    norm = lambda **k: lib.choco_adamw_grad_norm(k.get("h", h), k.get("c", 1.0), k.get("u", 1.0), k.get("n", p(f)),  # noqa: E731
                                                 k.get("f", p(f)), None)
    for bad in (dict(h=None), dict(c=-1.0), dict(c=float("nan")), dict(u=0.0), dict(u=float("inf")), dict(n=None), dict(f=None)):
        assert norm(**bad) == -1, bad
    assert norm(n=p(f) + 1) == -5
    assert lib.choco_adamw_read_state(h, p(o.m), p(o.v), None, p(o.v_scale), p(f), None, 0, None) == -1
    assert lib.choco_adamw_read_state(h, p(o.m), p(o.v), p(o.m_scale), p(o.v_scale), p(f), None, 4, None) == -1
    assert lib.choco_adamw_set_grads(h, None, None) == -1
    bad = np.array([p(r.G), 0], dtype=np.uint64)
    assert lib.choco_adamw_set_grads(h, bad.ctypes.data, None) == -1
    bad = np.array([p(r.G), p(r.G) + 2], dtype=np.uint64)
    assert lib.choco_adamw_set_grads(h, bad.ctypes.data, None) == -5
    steps = np.array([3, -1], dtype=np.int64)
    assert lib.choco_adamw_set_steps(h, steps.ctypes.data, None) == -1
    assert list(o.get_steps()) == [0, 0] and not bool(o.m.any())     # nothing above did anything
    for kw in (dict(states=(o.m, o.v)), dict(states=(o.m.float(), o.v, o.m_scale, o.v_scale)),
               dict(states=(o.m[:-256], o.v, o.m_scale, o.v_scale))):
        with pytest.raises(choco.ChocoError):
            choco.AdamW(r.X, r.G, r.off, state_bits=8, **kw)
    with pytest.raises(choco.ChocoError):
        choco.AdamW(r.X, r.G.double(), r.off)
    with pytest.raises(choco.ChocoError):
        choco.AdamW(r.X, r.G, [0, 100_000])
    with pytest.raises(choco.ChocoError):
        o.read_state(torch.empty(10, device=DEV), None)
    for call in (lambda: choco.AdamW(r.X.cpu(), r.G, r.off), lambda: choco.AdamW(r.X, r.G.cpu(), r.off),
                 lambda: o.step(1e-3, f.cpu()), lambda: o.grad_norm(1.0, f, f.cpu())):   # nothing of them reaches a kernel
        with pytest.raises(choco.ChocoError):
            call()
    o.close()
