"""The gradient of the lookup across the sizes at which its way of ordering tokens changes: one launch
(up to 256 tokens per worker), a cluster of blocks (up to 131072), a sort in global memory; one handle
through all of them in turn, so that what one call leaves behind meets the next."""
import pytest
import torch

import paper_1907_09356_b200 as choco
from test_gpu_embedding import DEV, F32, BF16, check_grad, ref_lookup, table_in, tokens_of

pytestmark = pytest.mark.gpu


def one(emb, n, vocab, dim, count, kind, accumulate, dtype=F32, gdtype=F32):
    tok = tokens_of(n, count, vocab, kind, count, torch.int32)
    dout = torch.randn((n, count, dim), generator=torch.Generator(device=DEV).manual_seed(count), device=DEV).to(dtype)
    G, view = table_in(n, vocab, dim, dim, vocab * dim, 0, gdtype, 6)
    before = view.clone()
    emb.backward(tok, dout, G, accumulate=accumulate)
    check_grad(view, tok, dout, 1.0, before if accumulate else None)


@pytest.mark.parametrize("n,counts", [(1, [131073, 256, 131072, 257, 5, 140000, 8192, 8193, 65537, 1024, 1025, 0, 131071]),
                                      (5, [300, 20000, 255, 1, 40000, 2049, 16385, 512])])
@pytest.mark.parametrize("vocab", [700, 40000])
def test_one_handle_through_all_sizes(n, counts, vocab):
    dim = 8
    emb = choco.Embedding(n, vocab, dim, max(counts))
    for k, count in enumerate(counts):
        one(emb, n, vocab, dim, count, "zipf" if k % 3 else "ragged", accumulate=k % 4 == 3)
    emb.close()


@pytest.mark.parametrize("kind", ["same", "two", "none", "outside", "uniform"])
@pytest.mark.parametrize("count", [255, 257, 3000, 20000, 133000])
def test_extreme_token_lists(kind, count):
    emb = choco.Embedding(2, 999, 12, count)
    for accumulate in (False, True):
        one(emb, 2, 999, 12, count, kind, accumulate)
    emb.close()


@pytest.mark.parametrize("n", [16, 40, 150])
def test_many_workers(n):
    for count in (3, 260, 2500):
        emb = choco.Embedding(n, 333, 20, count)
        one(emb, n, 333, 20, count, "zipf", False, BF16)
        one(emb, n, 333, 20, count, "ragged", True, BF16)
        emb.close()


@pytest.mark.parametrize("dim", [4, 100, 1024, 1500, 2050])
@pytest.mark.parametrize("gdtype", [F32, BF16])
def test_long_runs_over_many_columns(dim, gdtype):
    """Runs of thousands of rows, added up by several warps and blocks, in rows of every width."""
    emb = choco.Embedding(1, 64, dim, 9000)
    for accumulate in (False, True):
        one(emb, 1, 64, dim, 9000, "zipf", accumulate, BF16, gdtype)
    emb.close()


@pytest.mark.parametrize("vocab", [1 << 18, (1 << 18) - 1, 1 << 20, 511, 512, 513])
def test_vocabularies_at_the_digits_limits(vocab):
    emb = choco.Embedding(1, vocab, 4, 5000)
    one(emb, 1, vocab, 4, 5000, "uniform", False)
    one(emb, 1, vocab, 4, 5000, "outside", False)
    emb.close()


@pytest.mark.parametrize("count", [1, 40, 300, 9000])
@pytest.mark.parametrize("accumulate", [False, True])
def test_broadcast_gradients_and_shared_tokens(count, accumulate):
    """One row of dout for every token (a mean's gradient), one batch for all workers, the same tokens for
    all workers: expanded tensors, with strides of zero."""
    n, vocab, dim = 3, 50, 24
    gen = torch.Generator(device=DEV).manual_seed(1)
    tok = tokens_of(n, count, vocab, "zipf", count)
    shared = tokens_of(1, count, vocab, "ragged", count).expand(n, count)
    row = torch.randn((n, 1, dim), generator=gen, device=DEV).expand(n, count, dim)
    batch = torch.randn((1, count, dim), generator=gen, device=DEV).expand(n, count, dim)
    emb = choco.Embedding(n, vocab, dim, count)
    for t in (tok, shared):
        for dout in (row, batch):
            G, view = table_in(n, vocab, dim, dim, vocab * dim, 0, F32, 6)
            before = view.clone()
            emb.backward(t, dout, G, accumulate=accumulate)
            check_grad(view, t, dout, 1.0, before if accumulate else None)
        X, xview = table_in(n, vocab, dim, dim, vocab * dim, 0, F32, 7)
        out = torch.empty((n, count, dim), device=DEV)
        emb.forward(X, t, out)
        assert torch.equal(out.double(), ref_lookup(xview, t, 1.0))
    emb.close()
