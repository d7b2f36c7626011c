"""Cases for the training-side operators: token lookup, its gradient, gradient norms and AdamW.

Every case is the work of one pass for `n` workers at once.  Parameters, gradients and the token
table live where a decentralised run has them: in the dense rows of X and G, [n, ld] float32 (or
a 16-bit array of the same shape), one row per worker, a layer of the row per parameter tensor.

  lookup       out[i, t] = scale * table_i[token[i, t]]; tokens outside the vocabulary give zeros
  lookup_grad  grad_i[r] (+)= scale * sum over t with token[i, t] = r of dout[i, t]
  grad_norm    the 2-norm of every worker's gradient and the factor that clips it
  adamw        one AdamW step over all layers of all workers; moments in 32 or in 8 bits

Moments in 8 bits are held in blocks of 256 elements of a tensor: a block keeps a float32 scale and
a code k for every element, nearest on the scale of square roots, of m (signed, k up to 127) and of
sqrt(v) (k up to 255).  They come back as the values they stand for.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 256          # elements of a tensor that share a scale
NORM_EPS = 1e-6      # added to the norm before the clipping factor is formed
TINY = 1e-30         # smallest largest-value a block is scaled by
BETA1, BETA2, EPS = 0.9, 0.999, 1e-8
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2, "": 0}
LSTM_ROW = 28_950_000  # coordinates of a worker with the language model of the 32-node graph


def _device():
    return torch.device("cuda" if torch.cuda.is_available() else "cpu")


def _f32(v):
    return float(np.float32(v))


# --------------------------------------------------------------------------- cases


def listed():
    return [
        # one new token for each of eight workers' models: nothing but latency
        dict(name="lookup_one_token", op="lookup", n=8, tokens=1, vocab=33278, dim=650, ld=LSTM_ROW, table="f32", out="f32",
             index="i64", scale=1.0, masked=0.0),
        # the language-model run: 64 sequences of 35 tokens for each of 8 workers, rows of 2600 bytes
        # (every other one off a 16-byte boundary)
        dict(name="lookup_lstm", op="lookup", n=8, tokens=2240, vocab=33278, dim=650, ld=LSTM_ROW, table="f32", out="f32",
             index="i64", scale=1.0, masked=0.02),
        # one model, a large batch, 16-bit copy of the table, scaled by sqrt(dim)
        dict(name="lookup_large_bf16", op="lookup", n=1, tokens=262144, vocab=50000, dim=1024, ld=50000 * 1024, table="bf16",
             out="bf16", index="i32", scale=32.0, masked=0.1),
        # a small tied table: the lookup's gradient is added to the output layer's
        dict(name="lookup_grad_tied_small", op="lookup_grad", n=4, tokens=128, vocab=2000, dim=200, ld=500_003, dout="f32",
             grad="f32", index="i64", scale=1.0, masked=0.05, add=True),
        # the gradient of lookup_lstm, written into the rows of G (most rows are zeros)
        dict(name="lookup_grad_lstm", op="lookup_grad", n=8, tokens=2240, vocab=33278, dim=650, ld=LSTM_ROW, dout="f32",
             grad="f32", index="i64", scale=1.0, masked=0.02, add=False),
        # one model, a large batch: frequent tokens have thousands of rows to add up
        dict(name="lookup_grad_large_bf16", op="lookup_grad", n=1, tokens=131072, vocab=50000, dim=1024, ld=50000 * 1024,
             dout="bf16", grad="f32", index="i32", scale=32.0, masked=0.1, add=False),
        # every worker's norm over the ResNet-20-sized vector cut into its 65 tensors
        dict(name="grad_norm_small", op="grad_norm", n=8, layers="resnet20", d=272474, grad="f32", clip=0.25),
        # and over the LSTM-sized one
        dict(name="grad_norm_large", op="grad_norm", n=16, layers="even", d=LSTM_ROW, grad="f32", clip=0.25),
        # 520 ragged tensors, most of them tiny
        dict(name="adamw_32_small", op="adamw", bits=32, n=8, layers="resnet20", d=272474, x="f32", grad="f32", copy="", clip=0.0,
             t=3),
        # the language-model run: norms, clipping factors, AdamW and the 16-bit copy of the new weights
        dict(name="adamw_32_clip_large", op="adamw", bits=32, n=16, layers="even", d=LSTM_ROW, x="f32", grad="f32", copy="bf16",
             clip=0.25, t=1000),
        # 8-bit moments on a small model, 16-bit weights
        dict(name="adamw_8_small_bf16", op="adamw", bits=8, n=4, layers="resnet20", d=272474, x="bf16", grad="bf16", copy="",
             clip=0.0, t=3),
        # 8-bit moments on the ResNet-50-sized vector cut into its 161 tensors, 16-bit gradients
        dict(name="adamw_8_large", op="adamw", bits=8, n=8, layers="resnet50", d=25_557_032, x="f32", grad="bf16", copy="bf16",
             clip=0.0, t=1000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["lookup", "lookup_grad", "grad_norm", "adamw", "adamw"])
    f = lambda: rng.choice(["f32", "f32", "bf16", "f16"])  # noqa: E731
    if op in ("lookup", "lookup_grad"):
        n, vocab, dim = _log(rng, 1, 32), _log(rng, 300, 60000), _log(rng, 48, 1400)
        dim = dim if rng.random() < 0.3 else dim // 8 * 8
        vocab = max(300, min(vocab, 200_000_000 // (n * dim)))
        tokens = max(1, min(_log(rng, 1, 200_000), 200_000_000 // (n * dim)))
        c = dict(op=op, n=n, tokens=tokens, vocab=vocab, dim=dim, ld=vocab * dim + rng.choice([0, 0, 16, 1000, 4099]),
                 index=rng.choice(["i32", "i64"]), scale=rng.choice([1.0, _f32(math.sqrt(dim))]), masked=rng.choice([0.0, 0.02, 0.3]))
        if op == "lookup":
            c["table"] = f()
            c["out"] = c["table"] if rng.random() < 0.6 else f()
        else:
            c["dout"], c["grad"], c["add"] = f(), rng.choice(["f32", "f32", "f32", "bf16"]), rng.random() < 0.4
        return c
    layers = rng.choice(["resnet20", "even", "even", "resnet50"])
    d = {"resnet20": 272474, "resnet50": 25_557_032}.get(layers) or _log(rng, 500, LSTM_ROW)
    n = min(_log(rng, 1, 64), max(1, 200_000_000 // d))
    c = dict(op=op, n=n, layers=layers, d=d, grad=f(), clip=rng.choice([0.0, 0.25, 1.0]) if op == "adamw" else rng.choice([0.25, 1.0]))
    if op == "adamw":
        c["bits"] = rng.choice([8, 32])
        if c["bits"] == 8:
            c["clip"] = 0.0
        c["x"] = rng.choice(["f32", "f32", "f32", "bf16", "f16"])
        c["copy"] = rng.choice(["", "bf16", "f16"]) if c["x"] == "f32" else ""
        c["t"] = _log(rng, 1, 100_000)
    return c


# --------------------------------------------------------------------------- inputs


def _generator(seed):
    return torch.Generator(device=_device()).manual_seed(int(seed))


def _normal(g, shape, dtype, sd):
    out = torch.empty(shape, dtype=dtype, device=_device())
    return out.normal_(0.0, sd, generator=g)


def _tokens(case, g):
    """Tokens with Zipf's frequencies over a shuffled vocabulary; each masked one is -1 (padding of ragged batches)."""
    dev, vocab = _device(), case["vocab"]
    cdf = (1.0 / torch.arange(1, vocab + 1, dtype=torch.float64, device=dev)).cumsum(0)
    names = torch.randperm(vocab, generator=g, device=dev)
    u = torch.rand((case["n"], case["tokens"]), generator=g, dtype=torch.float64, device=dev) * cdf[-1]
    tok = names[torch.searchsorted(cdf, u).clamp_(max=vocab - 1)]
    drop = torch.rand(tok.shape, generator=g, device=dev) < case["masked"]
    return tok.masked_fill_(drop, -1).to(torch.int32 if case["index"] == "i32" else torch.int64).contiguous()


def _sizes(case):
    """Lengths of a worker's tensors."""
    d = case["d"]
    if case["layers"] == "even":  # a table of three quarters of the row and eight equal layers, cut at multiples of 512 where that fits
        unit = 512 if d >= 65536 else 1
        part = d // 32 // unit * unit
        return [d - 8 * part] + [part] * 8 if part else [d]
    import workloads
    return {"resnet20": workloads.resnet20_layer_sizes, "resnet50": workloads.resnet50_layer_sizes}[case["layers"]]()


def _plan(case):
    """Where the tensors of a row start, where their moments start, and what decay each has (none for short ones)."""
    sizes = np.asarray(_sizes(case), dtype=np.int64)
    off = np.concatenate([[0], np.cumsum(sizes)])
    padded = -(-sizes // BLOCK) * BLOCK
    state = np.concatenate([[0], np.cumsum(padded)])
    decay = np.where(sizes >= 512, 0.01, 0.0)
    return off, state, decay


def _places(off, state):
    """For every coordinate of a row the place of its moments; None where the two are the same."""
    if off[-1] == state[-1]:
        return None
    shift = np.repeat(state[:-1] - off[:-1], np.diff(off))
    return torch.from_numpy(shift).to(_device()) + torch.arange(int(off[-1]), device=_device())


def prepare(case, seed):
    g, dev = _generator(seed), _device()
    n = case["n"]
    st = {"case": case}
    if case["op"] in ("lookup", "lookup_grad"):
        vocab, dim, ld = case["vocab"], case["dim"], case["ld"]
        off = ld - vocab * dim if case["op"] == "lookup" or not case["add"] else 0
        st["off"] = off
        st["tokens"] = _tokens(case, g)
        if case["op"] == "lookup":
            st["X"] = _normal(g, (n, ld), TYPES[case["table"]], 0.1)
            st["table"] = st["X"][:, off:]
            st["out"] = torch.empty((n, case["tokens"], dim), dtype=TYPES[case["out"]], device=dev)
        else:
            st["G"] = _normal(g, (n, ld), TYPES[case["grad"]], 0.01) if case["add"] else torch.zeros((n, ld), dtype=TYPES[case["grad"]], device=dev)
            st["grad"] = st["G"][:, off:]
            st["dout"] = _normal(g, (n, case["tokens"], dim), TYPES[case["dout"]], 0.01)
        if own:
            import paper_1907_09356_b200 as choco
            st["emb"] = choco.Embedding(n, vocab, dim, case["tokens"], table_ld=ld, scale=case["scale"])
        return st
    off, state, decay = _plan(case)
    d, e = int(off[-1]), int(state[-1])
    st["G"] = _normal(g, (n, d), TYPES[case["grad"]], 0.001)
    st["G"] *= torch.rand((n, 1), generator=g, device=dev).mul_(2).to(st["G"].dtype)
    st["norm"] = torch.empty(n, dtype=torch.float32, device=dev)
    st["factor"] = torch.rand(n, generator=g, device=dev)
    if case["op"] == "grad_norm":
        if own:
            import paper_1907_09356_b200 as choco
            st["opt"] = choco.AdamW(None, st["G"], off, weight_decay=decay, beta1=BETA1, beta2=BETA2, eps=EPS)
        return st
    st["X"] = _normal(g, (n, d), TYPES[case["x"]], 0.05)
    st["copy"] = torch.empty((n, d), dtype=TYPES[case["copy"]], device=dev) if case["copy"] else None
    st["places"] = _places(off, state)
    st["decay"] = torch.from_numpy(np.repeat(decay.astype(np.float32), np.diff(off))).to(dev)
    m = _normal(g, (n, e), torch.float32, 0.0003)
    v = _normal(g, (n, e), torch.float32, 1.0).abs_().add_(0.01).mul_(1e-6)
    if st["places"] is not None:  # nothing behind a tensor's last element
        gap = torch.ones(e, dtype=torch.bool, device=dev).index_fill_(0, st["places"], False)
        m, v = m.masked_fill_(gap, 0.0), v.masked_fill_(gap, 0.0)
    if case["bits"] == 32:
        st["m"], st["v"] = m, v
    else:
        st["m"], st["m_scale"] = _code_m(m)
        st["v"], st["v_scale"] = _code_v(v)
        st["m_out"] = torch.empty((n, e), dtype=torch.bfloat16, device=dev)
        st["v_out"] = torch.empty((n, e), dtype=torch.bfloat16, device=dev)
    del m, v
    st["t"] = case["t"]
    if own:
        import paper_1907_09356_b200 as choco
        states = (st["m"], st["v"]) if case["bits"] == 32 else (st["m"], st["v"], st["m_scale"], st["v_scale"])
        st["opt"] = choco.AdamW(st["X"], st["G"], off, weight_decay=decay, copy=st["copy"], beta1=BETA1, beta2=BETA2, eps=EPS,
                                state_bits=case["bits"], states=states, step=case["t"] - 1)
    return st


# --------------------------------------------------------------------------- plain forms


def _edges(levels):
    """The values, on the scale of squares, from which on the codes 1 .. levels are the nearest."""
    k = torch.arange(1, levels + 1, dtype=torch.float32, device=_device()) - 0.5
    return k * k


def _code(y, levels):
    """The nearest code on the scale of square roots, of y in [0, levels ^ 2]."""
    return torch.bucketize(y, _edges(levels), out_int32=True, right=True)


def _scales(a, levels):
    """A block's scale and the factor that takes its values to [0, levels ^ 2], from its largest value."""
    a = a.clamp(min=TINY)
    return a * _f32(1.0 / levels ** 2), torch.full_like(a, float(levels ** 2)) / a


def _code_m(m):
    b = m.view(-1, BLOCK)
    a = b.abs()
    scale, inv = _scales(a.amax(1), 127)
    k = _code(a.mul_(inv[:, None]), 127)
    return torch.where(b < 0, -k, k).to(torch.int8).view(m.shape), scale


def _code_v(v):
    b = v.view(-1, BLOCK)
    r = b.sqrt()
    scale, inv = _scales(r.amax(1), 255)
    k = _code(r.mul_(inv[:, None]), 255)
    return torch.maximum(k, (b > 0).to(torch.int32)).to(torch.uint8).view(v.shape), scale


def _value_m(code, scale):
    k = code.view(-1, BLOCK).float()
    return (k * k.abs() * scale[:, None]).view(code.shape)


def _value_v(code, scale):
    k = code.view(-1, BLOCK).float()
    r = k * k * scale[:, None]
    return (r * r).view(code.shape)


def _plain_lookup(st, case):
    n, vocab, dim, off = case["n"], case["vocab"], case["dim"], st["off"]
    table = st["X"][:, off:off + vocab * dim].unflatten(1, (vocab, dim))
    tok = st["tokens"].long()
    there = (tok >= 0) & (tok < vocab)
    rows = table[torch.arange(n, device=tok.device)[:, None], tok.clamp(0, vocab - 1)].float() * case["scale"]
    st["out"].copy_(rows.masked_fill_(~there[..., None], 0.0))
    return st["out"]


def _plain_lookup_grad(st, case):
    n, vocab, dim, off = case["n"], case["vocab"], case["dim"], st["off"]
    tok = st["tokens"].long()
    there = (tok >= 0) & (tok < vocab)
    at = (tok.clamp(0, vocab - 1) + vocab * torch.arange(n, device=tok.device)[:, None]).reshape(-1)
    rows = st["dout"].float().masked_fill_(~there[..., None], 0.0) if st["dout"].dtype != torch.float32 else st["dout"].masked_fill(~there[..., None], 0.0)
    total = torch.zeros((n * vocab, dim), dtype=torch.float32, device=tok.device).index_add_(0, at, rows.view(-1, dim)).mul_(case["scale"])
    grad = st["G"][:, off:off + vocab * dim]
    grad.copy_(grad.float().add_(total.view(n, -1)) if case["add"] else total.view(n, -1))
    return grad


def _plain_norm(st, case):
    grad = st["G"].float()
    norm = (grad * grad).sum(1).sqrt()
    return norm, (case["clip"] / (norm + NORM_EPS)).clamp(max=1.0)


def _plain_adamw(st, case):
    t, lr = st["t"], 1e-3
    places, x = st["places"], st["X"].float()
    out = {}
    factor = st["factor"]
    if case["clip"]:
        out["norm"], factor = _plain_norm(st, case)
    grad = st["G"].float() * factor[:, None]
    gs = grad if places is None else torch.zeros(st["m"].shape, device=grad.device).index_copy_(1, places, grad)
    m, v = (st["m"], st["v"]) if case["bits"] == 32 else (_value_m(st["m"], st["m_scale"]), _value_v(st["v"], st["v_scale"]))
    m = m * _f32(BETA1) + gs * _f32(1 - BETA1)
    v = v * _f32(BETA2) + (gs * _f32(1 - BETA2)) * gs
    den = v.sqrt() * _f32(1 / math.sqrt(1 - BETA2 ** t)) + _f32(EPS)
    ratio = m / den
    if places is not None:
        ratio = ratio.index_select(1, places)
    x -= ratio * _f32(lr / (1 - BETA1 ** t)) + x * (st["decay"] * _f32(lr))
    st["X"].copy_(x)
    if st["copy"] is not None:
        st["copy"].copy_(x)
        out["copy"] = st["copy"]
    st["t"] = t + 1
    out["x"] = st["X"]
    if case["bits"] == 32:
        st["m"], st["v"] = m, v
        return {**out, "m": m, "v": v}
    st["m"], st["m_scale"] = _code_m(m)
    st["v"], st["v_scale"] = _code_v(v)
    st["m_out"].copy_(_value_m(st["m"], st["m_scale"]))
    st["v_out"].copy_(_value_v(st["v"], st["v_scale"]))
    return {**out, "m": st["m_out"], "v": st["v_out"]}


# --------------------------------------------------------------------------- one pass


def run(st):
    case = st["case"]
    if not own:
        if case["op"] == "grad_norm":
            return dict(zip(("norm", "factor"), _plain_norm(st, case)))
        return {"lookup": _plain_lookup, "lookup_grad": _plain_lookup_grad, "adamw": _plain_adamw}[case["op"]](st, case)
    if case["op"] == "lookup":
        st["emb"].forward(st["table"], st["tokens"], st["out"])
        return st["out"]
    if case["op"] == "lookup_grad":
        st["emb"].backward(st["tokens"], st["dout"], st["grad"], accumulate=case["add"])
        return st["grad"][:, :case["vocab"] * case["dim"]]
    opt = st["opt"]
    if case["op"] == "grad_norm":
        opt.grad_norm(case["clip"], st["norm"], st["factor"])
        return {"norm": st["norm"], "factor": st["factor"]}
    out = {}
    if case["clip"]:
        opt.grad_norm(case["clip"], st["norm"], st["factor"])
        out["norm"] = st["norm"]
    opt.step(1e-3, st["factor"])
    if st["copy"] is not None:
        out["copy"] = st["copy"]
    out["x"] = st["X"]
    if case["bits"] == 32:
        return {**out, "m": st["m"], "v": st["v"]}
    opt.read_state(st["m_out"], st["v_out"])
    return {**out, "m": st["m_out"], "v": st["v_out"]}


# --------------------------------------------------------------------------- what a pass cannot do without


def _distinct(case):
    """Expected number of different tokens of one worker's batch."""
    p = 1.0 / np.arange(1, case["vocab"] + 1)
    return float(np.sum(-np.expm1(case["tokens"] * (1 - case["masked"]) * np.log1p(-p / p.sum()))))


def work(case):
    n = case["n"]
    if case["op"] in ("lookup", "lookup_grad"):
        dim, total = case["dim"], n * case["tokens"]
        kept, rows = total * (1 - case["masked"]), n * _distinct(case)
        index = total * (4 if case["index"] == "i32" else 8)
        if case["op"] == "lookup":
            return {"bytes": index + rows * dim * SIZE[case["table"]] + total * dim * SIZE[case["out"]], "flops": kept * dim}
        written = 2 * rows if case["add"] else n * case["vocab"]
        return {"bytes": index + kept * dim * SIZE[case["dout"]] + written * dim * SIZE[case["grad"]], "flops": (kept + rows) * dim}
    count = n * int(sum(_sizes(case)))
    if case["op"] == "grad_norm":
        return {"bytes": count * SIZE[case["grad"]] + 8 * n, "flops": 2 * count}
    moments = 16 if case["bits"] == 32 else 4 + 16 / BLOCK + 4  # read and written; 8 bits: and their values written
    return {"bytes": count * (2 * SIZE[case["x"]] + SIZE[case["grad"]] + SIZE[case["copy"]] + moments), "flops": count * (16 if case["clip"] else 14)}


# --------------------------------------------------------------------------- in 64 bits


def _exact_codes(value, levels):
    """(codes, scales) of non-negative values from the definition."""
    b = value.reshape(-1, BLOCK)
    top = b.max(dim=1, keepdim=True).values.clamp(min=TINY)
    return torch.floor(torch.sqrt(b / top) * levels + 0.5), top / levels ** 2


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    n = case["n"]
    if case["op"] == "lookup":
        vocab, dim, off = case["vocab"], case["dim"], st["off"]
        out = torch.zeros((n, case["tokens"], dim), dtype=torch.float64, device=_device())
        for i in range(n):
            table = st["X"][i, off:off + vocab * dim].view(vocab, dim)
            keep = st["tokens"][i] >= 0
            out[i, keep] = case["scale"] * table[st["tokens"][i][keep].long()].double()
        return out
    if case["op"] == "lookup_grad":
        vocab, dim, off = case["vocab"], case["dim"], st["off"]
        out = st["G"][:, off:off + vocab * dim].double()
        if not case["add"]:
            out.zero_()
        for i in range(n):
            keep = st["tokens"][i] >= 0
            out[i].view(vocab, dim).index_add_(0, st["tokens"][i][keep].long(), st["dout"][i][keep].double(), alpha=case["scale"])
        return out
    g = st["G"].double()
    norm = torch.linalg.vector_norm(g, dim=1)
    factor = torch.minimum(torch.ones_like(norm), case["clip"] / (norm + NORM_EPS))
    if case["op"] == "grad_norm":
        return {"norm": norm, "factor": factor}
    out = {"norm": norm} if case["clip"] else {}
    g *= (factor if case["clip"] else st["factor"].double())[:, None]
    off, state, decay = _plan(case)
    x, e, t = st["X"].double(), int(state[-1]), case["t"]
    if case["bits"] == 32:
        m, v = st["m"].double(), st["v"].double()
    else:
        k = st["m"].double().view(-1, BLOCK)
        m = (k.sign() * k ** 2 * st["m_scale"].double()[:, None]).view(n, e)
        v = ((st["v"].double().view(-1, BLOCK) ** 2 * st["v_scale"].double()[:, None]) ** 2).view(n, e)
    for a, b, s, w in zip(off[:-1], off[1:], state[:-1], decay):  # tensor by tensor
        gl, ml, vl, xl = g[:, a:b], m[:, s:s + b - a], v[:, s:s + b - a], x[:, a:b]
        ml.mul_(BETA1).add_(gl, alpha=1 - BETA1)
        vl.mul_(BETA2).addcmul_(gl, gl, value=1 - BETA2)
        step = (ml / (1 - BETA1 ** t)) / ((vl / (1 - BETA2 ** t)).sqrt() + EPS)
        xl.sub_(1e-3 * (step + float(w) * xl))
    out["x"] = x
    if st["copy"] is not None:
        out["copy"] = x
    if case["bits"] == 8:
        km, sm = _exact_codes(m.abs(), 127)
        kv, sv = _exact_codes(v.sqrt(), 255)
        kv = torch.maximum(kv, (v.view(-1, BLOCK) > 0).double())
        m = (m.view(-1, BLOCK).sign() * km ** 2 * sm).view(n, e)
        v = ((kv ** 2 * sv) ** 2).view(n, e)
    return {**out, "m": m, "v": v}
