"""Token lookup and its gradient against a plain implementation in 64 bits.

Tolerances, from the arithmetic.  u = 2^-24 is float32's rounding, w the output type's.  A lookup
rounds a product and then to the output type: (u + w) |value|.  A gradient element is a float32 sum
of k terms in some order, a product with the scale, a sum with the old value and one rounding:
(k + 3) u (|scale| sum |term| + |old|) + w |result|.  Both are taken with a factor of 1.01 for products
of roundings, plus the type's smallest subnormal.
"""
import ctypes

import numpy as np
import pytest
import torch

import paper_1907_09356_b200 as choco

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
W = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SUB = {torch.float32: 1e-44, torch.bfloat16: 1e-40, torch.float16: 6e-8}
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def tokens_of(n, count, vocab, kind, seed, dtype=torch.int64):
    g = torch.Generator().manual_seed(seed)
    if kind == "uniform":
        t = torch.randint(0, vocab, (n, count), generator=g)
    elif kind == "zipf":
        p = 1.0 / torch.arange(1, vocab + 1, dtype=torch.float64)
        t = torch.multinomial(p.expand(n, -1), max(count, 1), replacement=True, generator=g)[:, :count]
        t = torch.randperm(vocab, generator=g)[t]
    elif kind == "same":
        t = torch.full((n, count), vocab // 2)
    elif kind == "two":                                       # two tokens in turn: no two neighbours alike
        t = (torch.arange(count) % 2 * (vocab - 1)).repeat(n, 1)
    elif kind == "none":
        t = torch.full((n, count), -1)
    elif kind == "ragged":                                    # every worker's batch ends elsewhere
        t = torch.randint(0, vocab, (n, count), generator=g)
        for i in range(n):
            t[i, count * i // n:] = -1
    elif kind == "outside":                                   # tokens out of range on either side
        t = torch.randint(-vocab, 2 * vocab, (n, count), generator=g)
        if dtype == torch.int64 and count > 2:
            t[:, 0], t[:, 1] = 2 ** 40 + 1, -2 ** 40
    return t.to(dtype).to(DEV)


def table_in(n, vocab, dim, row, ld, head, dtype, seed):
    """A [n, ld] array whose columns from `head` on hold the tables; everything else is a sentinel."""
    X = torch.full((n, ld + head), 77.0, dtype=dtype, device=DEV)
    view = X[:, head:].as_strided((n, vocab, dim), (ld + head, row, 1), X.storage_offset() + head)
    g = torch.Generator(device=DEV).manual_seed(seed)
    view.copy_(torch.randn((n, vocab, dim), generator=g, device=DEV))
    return X, view


def ref_lookup(view, tok, scale):
    n, vocab, dim = view.shape
    t = tok.long()
    ok = (t >= 0) & (t < vocab)
    rows = view.double()[torch.arange(n, device=DEV)[:, None], t.clamp(0, vocab - 1)] * scale
    return torch.where(ok[..., None], rows, torch.zeros_like(rows))


def ref_grad(shape, tok, dout, scale, padding=-1):
    """(sum, sum of magnitudes, number of terms) per row, in float64."""
    n, vocab, dim = shape
    t = tok.long()
    ok = (t >= 0) & (t < vocab) & (t != padding)
    at = (t.clamp(0, vocab - 1) + vocab * torch.arange(n, device=DEV)[:, None])[ok]
    d = dout.double()[ok] * scale
    out = []
    for v in (d, d.abs()):
        out.append(torch.zeros((n * vocab, dim), dtype=torch.float64, device=DEV).index_add_(0, at, v).view(n, vocab, dim))
    k = torch.zeros(n * vocab, dtype=torch.float64, device=DEV).index_add_(0, at, torch.ones_like(at, dtype=torch.float64))
    return out[0], out[1], k.view(n, vocab, 1)


def close(got, want, bound):
    err = (got.double() - want).abs()
    assert bool((err <= 1.01 * bound).all()), float((err / bound.clamp(min=1e-300)).max())


def check_grad(view, tok, dout, scale, before, padding=-1):
    total, mag, k = ref_grad(view.shape, tok, dout, scale, padding)
    w, sub = W[view.dtype], SUB[view.dtype]
    old = torch.zeros_like(total) if before is None else before.double()
    want = total + old
    close(view, want, (k + 3) * U * (mag + old.abs()) * (k > 0) + w * want.abs() * (k > 0) + sub * (k > 0))
    untouched = (k == 0).expand_as(want)
    if before is None:
        assert not bool(view[untouched].any())
    else:
        assert torch.equal(view[untouched], before[untouched])


DIMS = [1, 2, 3, 8, 31, 50, 64, 128, 130, 200, 257, 650, 1024, 1100]


@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (F16, F32), (F32, BF16)])
def test_lookup_dims_and_types(dim, types):
    n, vocab, count = 3, 57, 41
    tok = tokens_of(n, count, vocab, "outside", dim)
    X, view = table_in(n, vocab, dim, dim, vocab * dim, 0, types[0], 1)
    out = torch.full((n, count, dim), float("nan"), dtype=types[1], device=DEV)
    emb = choco.Embedding(n, vocab, dim, 0, scale=1.7)
    emb.forward(X, tok, out)
    want = ref_lookup(view, tok, float(np.float32(1.7)))
    close(out, want, (U + W[types[1]]) * want.abs() + SUB[types[1]])
    emb.close()


@pytest.mark.parametrize("count", [0, 1, 2, 7, 8, 9, 255, 1000])
@pytest.mark.parametrize("index", [torch.int32, torch.int64])
def test_lookup_lengths(count, index):
    n, vocab, dim = 2, 300, 72
    tok = tokens_of(n, count, vocab, "zipf", count, index)
    X, view = table_in(n, vocab, dim, dim, vocab * dim, 0, F32, 1)
    out = torch.full((n, count, dim), float("nan"), device=DEV)
    emb = choco.Embedding(n, vocab, dim, 0)
    emb.forward(X, tok, out)
    want = ref_lookup(view, tok, 1.0)
    assert torch.equal(out.double(), want)
    emb.close()


@pytest.mark.parametrize("row,extra,head,pitch", [(50, 0, 0, 0), (51, 3, 1, 1), (56, 8, 4, 6), (64, 0, 2, 14), (52, 4, 8, 2)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides_and_offsets(row, extra, head, pitch, dtype):
    """Rows further apart than they are long, tables at odd offsets of X, outputs with a pitch."""
    n, vocab, dim, count = 3, 40, 50, 33
    ld = vocab * row + extra
    tok = tokens_of(n, count, vocab, "outside", row)
    X, view = table_in(n, vocab, dim, row, ld, head, dtype, 3)
    emb = choco.Embedding(n, vocab, dim, 64, table_row=row, table_ld=ld + head, scale=0.5)
    store = torch.full((n, count + 2, dim + pitch), 55.0, dtype=dtype, device=DEV)
    out = store[:, 1:count + 1, :dim] if pitch else store[:, :count, :dim]
    emb.forward(X[:, head:], tok, out)
    want = ref_lookup(view, tok, 0.5)
    close(out, want, (U + W[dtype]) * want.abs())
    mark = torch.full_like(store, 55.0)
    (mark[:, 1:count + 1, :dim] if pitch else mark[:, :count, :dim]).copy_(out)
    assert torch.equal(mark, store)                           # nothing written between or behind the rows
    for accumulate in (False, True):
        G, gview = table_in(n, vocab, dim, row, ld, head, F32, 4)
        before = gview.clone()
        emb.backward(tok, out, G[:, head:], accumulate=accumulate)
        check_grad(gview, tok, out, 0.5, before if accumulate else None)
        H, hview = table_in(n, vocab, dim, row, ld, head, F32, 4)
        hview.copy_(gview)
        assert torch.equal(H, G)                              # gaps and everything before the tables untouched
    emb.close()


@pytest.mark.parametrize("kind", ["uniform", "zipf", "same", "two", "none", "ragged", "outside"])
@pytest.mark.parametrize("count", [1, 2, 33, 257, 2047, 2048, 2049, 6000])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_lengths_and_repeats(kind, count, accumulate):
    n, vocab, dim = 3, 310, 40
    tok = tokens_of(n, count, vocab, kind, count)
    dout = torch.randn((n, count, dim), generator=torch.Generator(device=DEV).manual_seed(5), device=DEV)
    # what masked positions hold is nothing to go by
    t = tok.long()
    dout[(t < 0) | (t >= vocab)] = float("nan")
    dout[:, -1][(t[:, -1] < 0)] = float("inf")
    G, view = table_in(n, vocab, dim, dim, vocab * dim, 0, F32, 6)
    before = view.clone()
    emb = choco.Embedding(n, vocab, dim, count, scale=1.3)
    emb.backward(tok, dout, G, accumulate=accumulate)
    check_grad(view, tok, dout, float(np.float32(1.3)), before if accumulate else None)
    emb.close()


@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("types", [(F32, F32), (BF16, F32), (F16, BF16), (F32, F16)])
def test_gradient_dims_and_types(dim, types):
    n, vocab, count = 2, 37, 333
    tok = tokens_of(n, count, vocab, "zipf", dim, torch.int32)
    dout = torch.randn((n, count, dim), generator=torch.Generator(device=DEV).manual_seed(5), device=DEV).to(types[0])
    for accumulate in (False, True):
        G, view = table_in(n, vocab, dim, dim, vocab * dim, 0, types[1], 6)
        before = view.clone()
        emb = choco.Embedding(n, vocab, dim, 400, scale=0.25)
        emb.backward(tok, dout, G, accumulate=accumulate)
        check_grad(view, tok, dout, 0.25, before if accumulate else None)
        emb.close()


@pytest.mark.parametrize("vocab", [1, 2, 255, 256, 257, 65535, 65536, 65537, 1 << 17])
def test_gradient_vocabularies(vocab):
    n, dim, count = 2, 8, 5000
    for kind in ("uniform", "zipf"):
        tok = tokens_of(n, count, vocab, kind, vocab)
        tok[:, 0], tok[:, 1] = vocab - 1, 0
        dout = torch.randn((n, count, dim), generator=torch.Generator(device=DEV).manual_seed(7), device=DEV)
        G, view = table_in(n, vocab, dim, dim, vocab * dim, 0, F32, 8)
        emb = choco.Embedding(n, vocab, dim, count)
        emb.backward(tok, dout, G)
        check_grad(view, tok, dout, 1.0, None)
        emb.close()


@pytest.mark.parametrize("n,count", [(1, 40000), (1, 70000), (9, 9000), (40, 300)])
@pytest.mark.parametrize("dim,dtype", [(24, BF16), (150, F32)])
def test_gradient_large_batches(n, count, dim, dtype):
    vocab = 4000
    tok = tokens_of(n, count, vocab, "zipf", count, torch.int32)
    dout = torch.randn((n, count, dim), generator=torch.Generator(device=DEV).manual_seed(5), device=DEV).to(dtype)
    emb = choco.Embedding(n, vocab, dim, count)
    for accumulate in (False, True):
        G, view = table_in(n, vocab, dim, dim, vocab * dim, 0, F32, 6)
        before = view.clone()
        emb.backward(tok, dout, G, accumulate=accumulate)
        check_grad(view, tok, dout, 1.0, before if accumulate else None)
        again = G.clone()
        view.copy_(before)
        emb.backward(tok, dout, G, accumulate=accumulate)
        assert torch.equal(again, G)                          # the same bits every time
    emb.close()


def test_capacity_can_exceed_the_batch_and_batches_can_vary():
    n, vocab, dim = 2, 500, 16
    emb = choco.Embedding(n, vocab, dim, 5000)
    for count in (5000, 3, 2100, 0, 700, 1):
        tok = tokens_of(n, count, vocab, "zipf", count)
        dout = torch.randn((n, count, dim), device=DEV)
        G, view = table_in(n, vocab, dim, dim, vocab * dim, 0, F32, 6)
        emb.backward(tok, dout, G)
        check_grad(view, tok, dout, 1.0, None)
    emb.close()


def test_padding_token_is_looked_up_but_gets_no_gradient():
    n, vocab, dim, count, pad = 2, 20, 12, 90, 4
    tok = tokens_of(n, count, vocab, "zipf", 1)
    tok[:, ::3] = pad
    X, view = table_in(n, vocab, dim, dim, vocab * dim, 0, F32, 6)
    emb = choco.Embedding(n, vocab, dim, count, padding=pad)
    out = torch.empty((n, count, dim), device=DEV)
    emb.forward(X, tok, out)
    assert torch.equal(out.double(), ref_lookup(view, tok, 1.0))
    dout = torch.randn((n, count, dim), device=DEV)
    G, gview = table_in(n, vocab, dim, dim, vocab * dim, 0, F32, 7)
    emb.backward(tok, dout, G)
    check_grad(gview, tok, dout, 1.0, None, padding=pad)
    assert not bool(gview[:, pad].any())
    emb.close()


def test_gradient_against_differences():
    """f(W) = <lookup(W), dout> is linear in W, so a central difference with a step of 1 is the
    gradient up to the roundings of the two lookups: a scaled table entry of magnitude up to B is
    rounded to within u B, and so is every one of the k places it appears at."""
    n, vocab, dim, count, scale = 2, 11, 6, 64, 0.75
    tok = tokens_of(n, count, vocab, "ragged", 2)
    X, view = table_in(n, vocab, dim, dim, vocab * dim, 0, F32, 6)
    dout = torch.randn((n, count, dim), device=DEV)
    emb = choco.Embedding(n, vocab, dim, count, scale=scale)
    G, gview = table_in(n, vocab, dim, dim, vocab * dim, 0, F32, 7)
    emb.backward(tok, dout, G)
    _, mag, k = ref_grad(view.shape, tok, dout, scale)
    out = torch.empty((n, count, dim), device=DEV)

    def f():
        emb.forward(X, tok, out)
        return (out.double() * dout.double()).sum()

    for i in range(n):
        for r in range(vocab):
            for c in range(0, dim, 2):
                old = view[i, r, c].clone()
                view[i, r, c] = old + 1
                up, top = f(), view[i, r, c].double()
                view[i, r, c] = old - 1
                down, low = f(), view[i, r, c].double()
                view[i, r, c] = old
                big = (old.abs() + 1).double()
                slope = (up - down) / (top - low)
                bound = 4 * U * big * mag[i, r, c] + (k[i, r, 0] + 3) * U * mag[i, r, c] + 1e-12
                assert abs(float(gview[i, r, c]) - float(slope)) <= float(bound)
    emb.close()


def test_offsets_beyond_32_bits():
    n, vocab, dim, count = 2, 3, 40, 8
    ld = (1 << 32) + 8
    X = torch.empty((n, ld), dtype=BF16, device=DEV)
    row = (1 << 31)                                            # rows of one table billions of elements apart
    view = X.as_strided((n, vocab - 1, dim), (ld, row, 1))
    view.copy_(torch.randn((n, vocab - 1, dim), device=DEV))
    tok = tokens_of(n, count, vocab - 1, "uniform", 1)
    emb = choco.Embedding(n, vocab - 1, dim, count, table_row=row, table_ld=ld)
    out = torch.empty((n, count, dim), dtype=BF16, device=DEV)
    emb.forward(X, tok, out)
    assert torch.equal(out.double(), ref_lookup(view, tok, 1.0))
    emb.backward(tok, out, X)
    check_grad(view, tok, out, 1.0, None)
    emb.close()


def test_another_stream_and_capture():
    n, vocab, dim, count = 2, 400, 48, 700
    X, view = table_in(n, vocab, dim, dim, vocab * dim, 0, F32, 6)
    G, gview = table_in(n, vocab, dim, dim, vocab * dim, 0, F32, 7)
    tok = tokens_of(n, count, vocab, "zipf", 3)
    out = torch.empty((n, count, dim), device=DEV)
    emb = choco.Embedding(n, vocab, dim, count)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    emb.forward(X, tok, out, stream=side)
    emb.backward(tok, out, G, stream=side)
    side.synchronize()
    assert torch.equal(out.double(), ref_lookup(view, tok, 1.0))
    check_grad(gview, tok, out, 1.0, None)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        emb.forward(X, tok, out)
        emb.backward(tok, out, G)
    view.mul_(-2.0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out.double(), ref_lookup(view, tok, 1.0))
    check_grad(gview, tok, out, 1.0, None)
    emb.close()


def test_refusals():
    n, vocab, dim = 2, 10, 8
    emb = choco.Embedding(n, vocab, dim, 16)
    X = torch.zeros((n, vocab * dim), device=DEV)
    tok = torch.zeros((n, 4), dtype=torch.int64, device=DEV)
    out = torch.zeros((n, 4, dim), device=DEV)
    lib, h = choco.load(), emb.handle
    p = lambda t: t.data_ptr()  # noqa: E731
    fwd = lambda **k: lib.choco_embedding_forward(  # noqa: E731
        k.get("h", h), k.get("table", p(X)), k.get("td", 0), k.get("tok", p(tok)), k.get("bits", 64), k.get("count", 4),
        k.get("tld", 4), k.get("out", p(out)), k.get("od", 0), k.get("row", dim), k.get("ld", 4 * dim), None)
    bwd = lambda **k: lib.choco_embedding_backward(  # noqa: E731
        k.get("h", h), k.get("tok", p(tok)), k.get("bits", 64), k.get("count", 4), k.get("tld", 4), k.get("dout", p(out)),
        k.get("dd", 0), k.get("row", dim), k.get("ld", 4 * dim), k.get("grad", p(X)), k.get("gd", 0), 0, None)
    assert fwd() == 0 and bwd() == 0
    for bad in (dict(h=None), dict(tok=None), dict(bits=16), dict(count=-1), dict(tld=3), dict(row=dim - 1), dict(ld=-1)):
        assert fwd(**bad) == -1 and bwd(**bad) == -1, bad
    for bad in (dict(table=None), dict(td=3), dict(out=None), dict(od=-1)):
        assert fwd(**bad) == -1, bad
    for bad in (dict(grad=None), dict(dd=7), dict(dout=None), dict(gd=3)):
        assert bwd(**bad) == -1, bad
    assert fwd(table=p(X) + 2) == -5 and fwd(out=p(out) + 1, od=1) == -5 and fwd(tok=p(tok) + 4) == -5
    assert bwd(grad=p(X) + 2) == -5 and bwd(dout=p(out) + 3) == -5 and bwd(tok=p(tok) + 4) == -5
    assert bwd(count=17, tld=17) == -7                          # more tokens than the workspace holds
    assert fwd(count=1 << 31, tld=1 << 31) == -7
    assert lib.choco_embedding_destroy(None) == -1
    with pytest.raises(choco.ChocoError):
        emb.forward(X, tok, torch.zeros((n, 4, dim + 1), device=DEV))
    with pytest.raises(choco.ChocoError):
        emb.forward(X.double(), tok, out)
    with pytest.raises(choco.ChocoError):
        emb.forward(X, tok.to(torch.int16), out)
    with pytest.raises(choco.ChocoError):
        emb.backward(tok, out[:, :3], X)
    for bad in ((X.cpu(), tok, out), (X, tok.cpu(), out), (X, tok, out.cpu())):   # nothing of them reaches a kernel
        with pytest.raises(choco.ChocoError):
            emb.forward(*bad)
        with pytest.raises(choco.ChocoError):
            emb.backward(bad[1], bad[2], bad[0])
    torch.cuda.synchronize()
    emb.close()
