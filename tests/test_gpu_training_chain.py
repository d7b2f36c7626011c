"""Lookup, gradient, norms and AdamW enqueued back to back, where every kernel may start while the one
before it ends, against the same calls with a wait for the device after each."""
import pytest
import torch

import paper_1907_09356_b200 as choco
from test_gpu_embedding import BF16, DEV, F32, tokens_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab,dim,tail,count", [(300, 50, 1777, 600), (2000, 131, 40_001, 200)])
def test_chained_calls_see_what_the_call_before_wrote(bits, dtype, vocab, dim, tail, count):
    """Rows off 16-byte boundaries: memory sectors that two blocks of threads share are written by one
    and read by the other in the next call."""
    n, off = 3, [0, vocab * dim, vocab * dim + tail]
    gen = torch.Generator(device=DEV).manual_seed(1)
    X0 = (torch.randn((n, off[2] + 1), generator=gen, device=DEV) * 0.1).to(dtype)
    G0 = (torch.randn((n, off[2] + 1), generator=gen, device=DEV) * 0.01).to(F32)
    tok = tokens_of(n, count, vocab, "zipf", 3)

    def steps(wait):
        X, G = X0.clone()[:, 1:], G0.clone()[:, 1:]
        emb = choco.Embedding(n, vocab, dim, count, table_ld=off[2] + 1)
        opt = choco.AdamW(X, G, off, 0.01, state_bits=bits)
        rows = torch.zeros((n, count, dim), dtype=dtype, device=DEV)
        norm, factor = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
        torch.cuda.synchronize()
        for _ in range(25):
            for call in (lambda: emb.forward(X, tok, rows), lambda: emb.backward(tok, rows, G, accumulate=True),
                         lambda: opt.grad_norm(1.0, norm, factor), lambda: opt.step(1e-3, factor), lambda: opt.step(1e-3)):
                call()
                if wait:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        result = [X.clone(), G.clone(), rows, norm, factor, opt.m, opt.v]
        emb.close()
        opt.close()
        return result

    want = steps(True)
    for _ in range(3):
        for a, b in zip(steps(False), want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("bits", [32, 8])
def test_a_new_handle_on_another_stream(bits):
    """The tables of a handle are on the device when its init returns: the first calls may be on any stream,
    with nothing between that waits.  A thousand tensors make the copy a long one."""
    n, sizes = 40, [700 + k for k in range(26)]
    off = [0]
    for s in sizes:
        off.append(off[-1] + s)
    gen = torch.Generator(device=DEV).manual_seed(4)
    X0, G = torch.randn((n, off[-1]), generator=gen, device=DEV), torch.randn((n, off[-1]), generator=gen, device=DEV) * 0.01
    side = torch.cuda.Stream()
    results = []
    for k in range(12):
        X = X0.clone()
        norm, factor = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
        e = n * sum((s + 255) // 256 * 256 for s in sizes)
        zeros = lambda count, t: torch.zeros(count, dtype=t, device=DEV)  # noqa: E731
        states = (zeros(e, F32), zeros(e, F32)) if bits == 32 else (zeros(e, torch.int8), zeros(e, torch.uint8), zeros(e // 256, F32),
                                                                    zeros(e // 256, F32))
        torch.cuda.synchronize()
        opt = choco.AdamW(X, G, off, 0.01, state_bits=bits, states=states)
        opt.grad_norm(1.0, norm, factor, stream=side)
        opt.step(1e-3, factor, stream=side)
        side.synchronize()
        results.append((X, norm, factor, *states))
        opt.close()
    for other in results[1:]:
        for a, b in zip(results[0], other):
            assert torch.equal(a, b)
