"""8-bit moments rounded at random: neighbouring codes, the right expected value, averages that v follows, and the
same bits every time.

Tolerances.  A code is one of the two next to k = levels sqrt(|m| / top) (sqrt(v) for v), whose roundings move k by
1e-3 at most (as in test_gpu_adamw), plus what m's own error moves the root by.  Shares of N rounded elements are
binomial: 6 standard deviations.
"""
import numpy as np
import pytest
import torch

import paper_1907_09356_b200 as choco
from test_gpu_adamw import B1, B2, BF16, BLOCK, DEV, F32, RAGGED, Run, U, values

pytestmark = pytest.mark.gpu


def random_run(seed=7, **kw):
    r = Run(bits=8, **kw)
    choco.choco_adamw_set_rounding(r.opt.handle, True, seed)
    return r


def state(opt):
    return [opt.m, opt.v, opt.m_scale, opt.v_scale]


@pytest.mark.parametrize("x,g,copy", [(F32, F32, None), (F32, BF16, BF16), (BF16, BF16, None)])
@pytest.mark.parametrize("head", [0, 1])
@pytest.mark.parametrize("sizes", [RAGGED, [40_960], [256 * 40_000, 700]])
def test_codes_are_neighbours_of_the_value(x, g, copy, head, sizes):
    r = random_run(n=2 if len(sizes) > 2 else 1, sizes=sizes, x=x, g=g, copy=copy, head=head, step=4)
    r.randomise()
    want = r.ref(1e-3, 5)
    r.opt.step(1e-3)
    new, m, v, em, bound = want
    lim = 1.01 * (bound + (2.0 ** -8 if x == BF16 else 2 * U) * new.abs()) + 1e-38
    assert bool(((r.X[:, :r.d].double() - new).abs() <= lim).all())
    if copy is not None:
        assert torch.equal(r.copy[:, :r.d], r.X[:, :r.d].to(copy))

    def padded(a):
        p = torch.zeros(r.e, dtype=torch.float64, device=DEV)
        p[r.where] = a.reshape(-1)
        return p.view(-1, BLOCK)

    for code, value, err, levels in ((r.opt.m, m, em, 127), (r.opt.v, v.sqrt(), 4 * U * v.sqrt(), 255)):
        a, e, k = padded(value), padded(err), code.double().view(-1, BLOCK)
        top = a.abs().max(1, keepdim=True).values.clamp(min=1e-30)
        at, slack = levels * (a.abs() / top).sqrt(), 1e-3 + levels * (e / top).sqrt()
        low, high = torch.floor(at - slack), torch.ceil(at + slack)
        if levels == 255:
            high = torch.where(a > 0, high.clamp(min=1), high)
            assert bool((k[a > 0] >= 1).all())
        assert bool(((k.abs() >= low) & (k.abs() <= high.clamp(max=levels))).all())
        assert bool(((k * a >= 0) | (a.abs() <= e)).all())
    gap = torch.ones(r.e, dtype=torch.bool, device=DEV)
    gap[r.where] = False
    assert not bool(r.opt.m[gap].any()) and not bool(r.opt.v[gap].any())
    r.opt.close()


@pytest.mark.parametrize("small", [0.7, 0.2, 0.03, 0.0041])
@pytest.mark.parametrize("shift", [0, 1])
def test_the_expected_value_is_the_value(small, shift):
    """A million elements of one size beside the largest of their block, one step from zeros: the mean of the values
    their codes stand for is the value, for m and for v; a share p goes up, with p (1 - p) / N its variance."""
    blocks = 4096
    d = blocks * BLOCK
    G = torch.full((1, d + 1), small, device=DEV)[:, shift:shift + d]
    G[:, ::BLOCK] = 1.0
    G[:, 1::2] *= -1
    X = torch.zeros((1, d), device=DEV)
    opt = choco.AdamW(X, G, [0, d], state_bits=8, rounding="random", seed=11)
    opt.step(1e-3)
    rest = torch.ones(d, dtype=torch.bool, device=DEV)
    rest[::BLOCK] = False
    count = int(rest.sum())
    for code, scale, kind, levels, ratio in ((opt.m, opt.m_scale, "m", 127, small), (opt.v, opt.v_scale, "v", 255, small)):
        k = levels * ratio ** 0.5                                # of m and of sqrt(v): both are `small` of the largest
        power = 2 if kind == "m" else 4
        low = np.floor(k)
        p = (k ** power - low ** power) / ((low + 1) ** power - low ** power)
        up = float((code[rest].double().abs() > low).double().mean())
        assert bool(((code[rest].double().abs() - low) * (code[rest].double().abs() - low - 1) == 0).all())
        # the value is off by some 20 U, that is of a step k / power times as much; 16 bits make p a multiple of 2^-16
        assert abs(up - p) <= 6 * (p * (1 - p) / count) ** 0.5 + 20 * U * k + 2.0 ** -16
        assert bool((torch.sign(values(code, scale, "m")[rest]) == torch.sign(G.reshape(-1)[rest])).all()) or kind == "v"
    opt.close()


def test_v_follows_its_average():
    """Half of every block's gradients become ten times smaller after 3000 steps.  The noise of v's rounding is, per
    element, sqrt(2 / k) of v (k codes below, 1 / (1 - beta2) / 2 steps of a share of a code each), about 0.2, so the sum
    over 8192 elements is known to 0.2 %; ten times that is allowed.  Nearest codes give 1.3 and over 100 times."""
    d = 64 * BLOCK
    part = (torch.arange(d, device=DEV) % BLOCK) < BLOCK // 2
    G, X = torch.zeros((1, d), device=DEV), torch.zeros((1, d), device=DEV)
    opt = choco.AdamW(X, G, [0, d], state_bits=8, rounding="random", seed=3)
    v = torch.zeros(d, dtype=torch.float64, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(5)
    for t in range(8000):
        G.normal_(0.0, 1e-2, generator=gen)
        if t >= 3000:
            G[0, part] *= 0.1
        opt.step(1e-4)
        v.mul_(B2).addcmul_(G[0].double(), G[0].double(), value=1 - B2)
        if t in (2999, 7999):
            stored = values(opt.v, opt.v_scale, "v")
            for which in (part, ~part):
                assert abs(float(stored[which].sum() / v[which].sum()) - 1) < 0.02
    opt.close()


def run_steps(sizes, seed, head=0, steps=6, graph=False, resume=0):
    r = random_run(seed=seed, n=2, sizes=sizes, head=head)
    opts = [r.opt]
    replay = None
    if graph:
        replay = torch.cuda.CUDAGraph()
        with torch.cuda.graph(replay):
            r.opt.step(1e-3)
    for t in range(steps):
        if resume and t == resume:
            c = choco.AdamW(r.X, r.G, r.off, r.decay, r.lr_scale, beta1=B1, beta2=B2, state_bits=8, states=[a.clone() for a in state(r.opt)],
                            step=t, rounding="random", seed=seed)
            opts.append(c)
        r.G[:, :r.d].normal_(0.0, 0.01, generator=torch.Generator(device=DEV).manual_seed(t))
        replay.replay() if graph else opts[-1].step(1e-3)
    torch.cuda.synchronize()
    got = [r.X[:, :r.d].clone()] + [a.clone() for a in state(opts[-1])]
    for o in opts:
        o.close()
    return got


@pytest.mark.parametrize("sizes", [[300, 4096, 7], [256 * 18_000, 5000]])
def test_the_same_bits_every_time(sizes):
    """Run again, resumed, replayed from a graph, and with rows that start elsewhere (single accesses): equal.
    Another seed: not."""
    want = run_steps(sizes, 7)
    for other in (run_steps(sizes, 7), run_steps(sizes, 7, resume=3), run_steps(sizes, 7, graph=True), run_steps(sizes, 7, head=1)):
        for a, b in zip(want, other):
            assert torch.equal(a, b)
    assert not torch.equal(want[2], run_steps(sizes, 8)[2])


def test_refusals_and_the_way_back():
    r = Run(1, [300], 32)
    with pytest.raises(choco.ChocoError) as e:
        choco.choco_adamw_set_rounding(r.opt.handle, True, 1)
    assert e.value.code == -6
    with pytest.raises(choco.ChocoError):
        choco.AdamW(r.X, r.G, r.off, state_bits=32, rounding="random")
    with pytest.raises(choco.ChocoError):
        choco.AdamW(r.X, r.G, r.off, state_bits=8, rounding="up")
    r.opt.close()
    r, s = random_run(n=1, sizes=[300]), Run(1, [300], 8)
    assert choco.load().choco_adamw_set_rounding(r.opt.handle, 2, 1) == -1 and choco.load().choco_adamw_set_rounding(None, 1, 1) == -1
    choco.choco_adamw_set_rounding(r.opt.handle, False)
    r.opt.step(1e-3)
    s.opt.step(1e-3)
    assert all(torch.equal(a, b) for a, b in zip(state(r.opt), state(s.opt)))
    r.opt.close()
    s.opt.close()
