"""The gradient of more tokens than a cluster of blocks orders, sorted in global memory with one to four passes: the
result lies in the other pair of buffers each time."""
import pytest
import torch

import paper_1907_09356_b200 as choco
from test_gpu_embedding import DEV, F32, check_grad, table_in, tokens_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [1, 200, 255, 256, 65535, 65536, 70_000, 128_256, (1 << 24) - 1, 1 << 24])
def test_passes_of_the_global_sort(vocab):
    n, dim, counts = 1 if vocab > 1 << 20 else 2, 4, (131_073, 150_001)
    emb = choco.Embedding(n, vocab, dim, max(counts))
    for count, kind in zip(counts, ("uniform", "outside")):
        tok = tokens_of(n, count, vocab, kind, count)
        tok[:, 5], tok[:, count - 1] = vocab - 1, 0
        dout = torch.randn((n, count, dim), generator=torch.Generator(device=DEV).manual_seed(3), device=DEV)
        for accumulate in (False, True):
            G, view = table_in(n, vocab, dim, dim, vocab * dim, 0, F32, 6)
            before = view.clone()
            emb.backward(tok, dout, G, accumulate=accumulate)
            check_grad(view, tok, dout, 1.0, before if accumulate else None)
    emb.close()


@pytest.mark.parametrize("vocab", [300, 100_000])
def test_sorted_in_global_memory_and_in_a_cluster(vocab):
    """One handle, with the same tokens twice and without: sums of the first 131072 tokens, ordered by a cluster, and
    of those with a tail of tokens that stand for nothing, sorted in global memory."""
    n, dim, count = 1, 8, 131_072
    emb = choco.Embedding(n, vocab, dim, count + 999)
    tok = tokens_of(n, count, vocab, "uniform", 1)
    longer = torch.cat([tok, torch.full((n, 999), -1, device=DEV)], dim=1)
    dout = torch.randn((n, count + 999, dim), generator=torch.Generator(device=DEV).manual_seed(3), device=DEV)
    results = []
    for t, d in ((tok, dout[:, :count]), (longer, dout)):
        G, view = table_in(n, vocab, dim, dim, vocab * dim, 0, F32, 6)
        emb.backward(t, d, G)
        check_grad(view, t, d, 1.0, None)
        results.append(view.clone())
    if vocab > 1000:                                             # runs short enough to be added up in one piece
        assert torch.equal(*results)
    emb.close()
