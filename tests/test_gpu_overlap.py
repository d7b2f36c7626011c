"""Arrays that a call would write twice at once are refused: rows of a lookup's output, tensors of an AdamW list."""
import itertools

import numpy as np
import pytest
import torch

import paper_1907_09356_b200 as choco
from test_gpu_embedding import BF16, DEV, ref_lookup, table_in, tokens_of

pytestmark = pytest.mark.gpu


def overlaps(n, count, dim, ld, row):
    places = (ld * np.arange(n)[:, None, None] + row * np.arange(count)[None, :, None] + np.arange(dim)).reshape(-1)
    return len(np.unique(places)) < len(places)


@pytest.mark.parametrize("n,count,dim", [(1, 3, 4), (2, 1, 4), (2, 3, 4), (3, 4, 5), (5, 2, 3), (4, 7, 2)])
def test_lookup_takes_every_layout_of_separate_rows_and_no_other(n, count, dim):
    """All strides up to what lies clear of overlaps: worker after worker, token after token, and between."""
    vocab = 9
    X, view = table_in(n, vocab, dim, dim, vocab * dim, 0, torch.float32, 1)
    tok = tokens_of(n, count, vocab, "outside", 2)
    want = ref_lookup(view, tok, 1.0).float()
    emb = choco.Embedding(n, vocab, dim, 0)
    taken = 0
    for ld, row in itertools.product(range(0, count * (dim + 3) + 2), range(dim, n * (dim + 2) + 2)):
        store = torch.full((ld * (n - 1) + row * (count - 1) + dim,), 55.0, device=DEV)
        out = store.as_strided((n, count, dim), (ld, row, 1))
        if overlaps(n, count, dim, ld, row):
            with pytest.raises(choco.ChocoError):
                emb.forward(X, tok, out)
            assert bool((store == 55.0).all())
        else:
            emb.forward(X, tok, out)
            assert torch.equal(out, want)
            taken += 1
    assert taken > 0
    emb.close()


def test_lookup_refuses_an_expanded_output():
    X = torch.zeros((3, 40), device=DEV)
    tok = torch.zeros((3, 6), dtype=torch.int64, device=DEV)
    emb = choco.Embedding(3, 5, 8, 0)
    for out in (torch.zeros((1, 6, 8), device=DEV).expand(3, 6, 8), torch.zeros((3, 1, 8), device=DEV).expand(3, 6, 8)):
        with pytest.raises(choco.ChocoError):
            emb.forward(X, tok, out)
    emb.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_refuses_tensors_that_share_memory(bits):
    X, G, C = torch.zeros((3, 600), device=DEV), torch.zeros((3, 600), device=DEV), torch.zeros((3, 600), dtype=BF16, device=DEV)
    off = [0, 100, 600]
    new = lambda x, g, c=None: choco.AdamW(x, g, off, copy=c, state_bits=bits)  # noqa: E731
    flat = torch.zeros(2000, device=DEV)
    for bad in ((X[:1].expand(3, 600), G, None),                                     # one row for all workers
                (flat.as_strided((3, 600), (599, 1)), G, None),                      # the last element of a row is the next one's first
                (X, G, C[:1].expand(3, 600)),
                (X, X, None),                                                        # gradients in the parameters' place
                (X, X[:1].expand(3, 600), None), (X, G, X.view(BF16)[:, 600:])):
        with pytest.raises(choco.ChocoError) as e:
            new(*bad)
        assert e.value.code == -1
    opt = new(X, G[:1].expand(3, 600), C)                                            # one gradient for all workers
    with pytest.raises(choco.ChocoError):
        choco.choco_adamw_set_grads(opt.handle, [X.data_ptr()] * 6)
    choco.choco_adamw_set_grads(opt.handle, [G.data_ptr()] * 6)
    opt.step(1e-3)
    opt.close()
    norms = choco.AdamW(None, G[:1].expand(3, 600), off)
    norms.close()
