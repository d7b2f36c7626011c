"""AdamW over lists of nothing but whole aligned blocks, longer than a chunk: every element is updated once.

Tolerances are those of test_gpu_adamw; lists that are cut differently (or run again) give the same
bits, since a block's update looks at nothing outside it.
"""
import numpy as np
import pytest
import torch

import paper_1907_09356_b200 as choco
from test_gpu_adamw import B1, B2, BF16, DEV, EPS, F16, F32, Run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("sizes", [[2048], [4096], [1280, 65536], [1024, 256, 2816, 1536]])
def test_short_lists(bits, sizes):
    r = Run(1, sizes, bits, step=4)
    r.randomise()
    want = r.ref(1e-3, 5)
    r.opt.step(1e-3)
    r.check(None, want)
    r.opt.close()


def state_of(opt):
    return [a for a in (opt.m, opt.v, opt.m_scale, opt.v_scale) if a is not None]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("n,sizes", [(2, [4096]), (3, [2048, 5120, 1280]), (2, [9 << 20, 1024 * 5 + 256])])
def test_workers_together_and_alone_and_again(bits, n, sizes):
    """One list for all workers, one for each, and the same once more: short lists and one beyond them."""
    d = sum(sizes)
    off = np.concatenate([[0], np.cumsum(sizes)])
    gen = torch.Generator(device=DEV).manual_seed(2)
    X0 = torch.randn((n, d), generator=gen, device=DEV)
    G = torch.randn((n, d), generator=gen, device=DEV) * 0.01
    results = []
    for parts in ([slice(0, n)], [slice(i, i + 1) for i in range(n)], [slice(0, n)]):
        X = X0.clone()
        opts = [choco.AdamW(X[p], G[p], off, 0.1, state_bits=bits) for p in parts]
        for _ in range(3):
            for o in opts:
                o.step(1e-3)
        results.append([X] + [torch.cat(a) for a in zip(*(state_of(o) for o in opts))])
        for o in opts:
            o.close()
    for other in results[1:]:
        for a, b in zip(results[0], other):
            assert torch.equal(a, b)


@pytest.mark.parametrize("bits", [32, 8])
def test_one_pair_of_types_has_whole_blocks_only(bits):
    """A list of three pairs of types, one of them without a ragged end, against a list for each tensor."""
    gen = torch.Generator(device=DEV).manual_seed(3)
    sizes, types = [5000, 4096, 2300], [(F32, F32), (BF16, F32), (F16, BF16)]
    x0 = [torch.randn(s, generator=gen, device=DEV).to(t[0]) for s, t in zip(sizes, types)]
    gs = [(torch.randn(s, generator=gen, device=DEV) * 0.01).to(t[1]) for s, t in zip(sizes, types)]

    def steps(which):
        xs = [x.clone() for x in x0]
        rec = np.zeros(len(which), dtype=choco.ADAMW_TENSOR)
        for k, i in enumerate(which):
            rec[k] = (xs[i].data_ptr(), gs[i].data_ptr(), 0, sizes[i], choco._dtype(xs[i]), choco._dtype(gs[i]), 0, 0, 0.05, 1.0)
        opt = choco.choco_adamw_init(rec, 1, B1, B2, EPS, bits)
        e, off = choco.choco_adamw_state_size(opt, len(which))
        new = lambda count, dtype: torch.zeros(count, dtype=dtype, device=DEV)  # noqa: E731
        m, v = (new(e, F32), new(e, F32)) if bits == 32 else (new(e, torch.int8), new(e, torch.uint8))
        ms, vs = (None, None) if bits == 32 else (new(e // 256, F32), new(e // 256, F32))
        for _ in range(3):
            choco.choco_adamw_step(opt, m, v, ms, vs, 1e-2)
        torch.cuda.synchronize()
        choco.choco_adamw_destroy(opt)
        return {i: (xs[i], m[o:o + sizes[i]], v[o:o + sizes[i]]) for i, o in zip(which, off)}

    together = steps([0, 1, 2])
    for i in range(3):
        for a, b in zip(together[i], steps([i])[i]):
            assert torch.equal(a, b)


@pytest.mark.parametrize("bits", [32, 8])
def test_new_gradients_make_a_list_aligned(bits):
    r = Run(1, [8192], bits, step=1)
    r.randomise()
    store = torch.randn(8200, device=DEV)
    for shift in (1, 0, 3, 4):
        g = store[shift:shift + 8192]
        choco.choco_adamw_set_grads(r.opt.handle, [g.data_ptr()])
        r.G[0, :8192] = g                                        # what ref() looks at
        want = r.ref(1e-3, int(r.opt.get_steps()[0]) + 1)
        r.opt.step(1e-3)
        r.check(None, want)
    r.opt.close()
