"""Cases for what a network between lookup and optimizer needs: group norm with an activation, forward and
backward, and Muon's orthogonalised updates.

Every case is one pass for `n` workers at once.  Parameters and gradients live in the dense rows of X and G,
[n, ld], one row per worker, a layer of the row per parameter tensor.

  orthogonalize  O = p(p(...p(U / |U|))) of every matrix of a list, p(X) = a X + (b A + c A^2) X with A = X X^T of
                 the smaller side: five products' worth of steps that bring all singular values near 1
  muon           one step over the matrices of all workers: m = beta m + (1 - beta) c g, u = beta m + (1 - beta) c g,
                 x = x - (lr s O(u) + x lr decay) with s = sqrt(max(1, rows / cols))
  norm           y = act(w (x - mean) rstd + b), channels last; mean and 1 / sqrt(var + eps) over the pixels of an image
                 and the channels of a group
  norm_grad      its gradients: dx for every element, dw and db for every channel of every worker
"""
import math

import numpy as np
import torch

own = False

BLOCK = 256                             # matrices start on multiples of this in the momentum
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
STEPS, BETA, LR, DECAY = 5, 0.95, 0.02, 0.01
EPS = 1e-5                              # of group norm
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2, "": 0}


def _device():
    return torch.device("cuda" if torch.cuda.is_available() else "cpu")


def _f32(v):
    return float(np.float32(v))


# --------------------------------------------------------------------------- cases


def listed():
    return [
        # one filter bank of the ResNet-20, by itself: nothing but latency
        dict(name="orthogonalize_filters_small", op="orthogonalize", matrices="1:64x576", input="f32", output="f32"),
        # the four gate matrices of the language model's LSTM (width 650) for each of eight workers
        dict(name="orthogonalize_lstm_bf16", op="orthogonalize", matrices="32:2600x650", input="bf16", output="bf16"),
        # one large square matrix in single precision
        dict(name="orthogonalize_square_large", op="orthogonalize", matrices="1:4096x4096", input="f32", output="f32"),
        # every matrix of the ResNet-20 of eight workers: 176 of 10 x 64 up to 64 x 576
        dict(name="muon_resnet20", op="muon", n=8, layers="resnet20", x="f32", grad="f32", copy="", clip=True),
        # every matrix of the ResNet-50 of four workers, 64 x 147 up to 2048 x 1024, with a 16-bit copy
        dict(name="muon_resnet50", op="muon", n=4, layers="resnet50", x="f32", grad="bf16", copy="bf16", clip=True),
        # ragged matrices, wide, tall and single rows, 16-bit weights
        dict(name="muon_ragged_bf16", op="muon", n=3, layers="650x650,2600x650,333x1001,17x5000,1x300,129x127", x="bf16", grad="bf16",
             copy="", clip=False),
        # one image of the CIFAR network's first stage: nothing but latency
        dict(name="norm_one_image", op="norm", n=1, images=1, pixels=1024, channels=16, groups=4, act="relu", x="f32", y="f32", param="f32",
             pitch=0),
        # that stage for eight workers with batches of 128
        dict(name="norm_resnet20", op="norm", n=8, images=128, pixels=1024, channels=16, groups=8, act="relu", x="f32", y="f32",
             param="f32", pitch=0),
        # the ResNet-50's stem, 112 x 112 pixels of 64 channels, in 16 bits
        dict(name="norm_stem_bf16", op="norm", n=2, images=64, pixels=12544, channels=64, groups=32, act="relu", x="bf16", y="bf16",
             param="f32", pitch=0),
        # the CIFAR network's last stage, 8 x 8 pixels of 64 channels
        dict(name="norm_grad_small", op="norm_grad", n=8, images=32, pixels=64, channels=64, groups=16, act="relu", x="f32", y="f32",
             param="f32", pitch=0, add=False),
        # the ResNet-50's last stage, 7 x 7 pixels, with a smooth activation, added to earlier gradients
        dict(name="norm_grad_odd_f16", op="norm_grad", n=4, images=32, pixels=49, channels=2048, groups=32, act="silu", x="f16", y="f16",
             param="f16", pitch=0, add=True),
        # the ResNet-50's first stage, 56 x 56 pixels of 256 channels
        dict(name="norm_grad_stage_bf16", op="norm_grad", n=2, images=64, pixels=3136, channels=256, groups=32, act="relu", x="bf16",
             y="bf16", param="f32", pitch=0, add=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _products(rows, cols):
    """Operations of the steps on one matrix; symmetric products count one half."""
    m, k = min(rows, cols), max(rows, cols)
    return STEPS * (3 * m * m * k + m * m * m)


def draw(rng):
    op = rng.choice(["orthogonalize", "muon", "norm", "norm_grad"])
    f = lambda: rng.choice(["f32", "f32", "bf16", "f16"])  # noqa: E731
    if op in ("orthogonalize", "muon"):
        most, left = _products(4096, 4096), 60_000_000
        shapes = []
        for _ in range(rng.choice([1, 1, 2, 4])):
            a, b = _log(rng, 1, 2048), _log(rng, 1, 8192)
            a = a // 16 * 16 if a >= 64 and rng.random() < 0.5 else a
            shapes.append((a, b) if rng.random() < 0.6 else (b, a))
        count = _log(rng, 1, 64)
        elements, flops = sum(a * b for a, b in shapes), sum(_products(a, b) for a, b in shapes)
        count = max(1, min(count, int(most // flops), left // elements))
        if op == "orthogonalize":
            return dict(op=op, matrices=",".join("%d:%dx%d" % (count, a, b) for a, b in shapes), input=f(), output=f())
        x = f()
        return dict(op=op, n=count, layers=",".join("%dx%d" % s for s in shapes), x=x, grad=f(), copy=rng.choice(["", "bf16"]) if x == "f32" else "",
                    clip=rng.random() < 0.5)
    per, groups = _log(rng, 1, 64), _log(rng, 1, 64)
    if rng.random() < 0.6:
        per, groups = 1 << (per.bit_length() - 1), 1 << (groups.bit_length() - 1)
    channels = per * groups
    pixels = rng.choice([_log(rng, 1, 12544), _log(rng, 1, 112) ** 2])
    n, images = _log(rng, 1, 16), _log(rng, 1, 128)
    most = 100_000_000
    pixels = max(-(-16 // per), min(pixels, most // channels))   # of fewer values a group's gradient all but cancels
    images = max(1, min(images, most // (channels * pixels)))
    n = max(1, min(n, most // (channels * pixels * images)))
    x = f()
    c = dict(op=op, n=n, images=images, pixels=pixels, channels=channels, groups=groups, act=rng.choice(["none", "relu", "relu", "silu", "gelu"]),
             x=x, y=x if rng.random() < 0.7 else f(), param=rng.choice(["f32", x]), pitch=rng.choice([0, 0, 0, 8, channels]))
    if op == "norm_grad":
        c["add"] = rng.random() < 0.3
    return c


# --------------------------------------------------------------------------- inputs


def _generator(seed):
    return torch.Generator(device=_device()).manual_seed(int(seed))


def _normal(g, shape, sd):
    return torch.empty(shape, dtype=torch.float32, device=_device()).normal_(0.0, sd, generator=g)


def _matrices(case):
    """(count, rows, cols) of a list of matrices."""
    part = lambda t: (int(t.partition(":")[0]), *(int(v) for v in t.partition(":")[2].split("x")))  # noqa: E731
    return list(map(part, case["matrices"].split(",")))


def _layers(case):
    """(lengths of a worker's tensors, the shape of each that is a matrix or None)."""
    if not case["layers"].startswith("resnet"):
        shapes = list(map(lambda t: tuple(int(v) for v in t.split("x")), case["layers"].split(",")))
        return [a * b for a, b in shapes], shapes
    import workloads
    sizes = {"resnet20": workloads.resnet20_layer_sizes, "resnet50": workloads.resnet50_layer_sizes}[case["layers"]]()
    # filters, scale, shift of one convolution after another, then the classifier and its bias: a matrix has as
    # many rows as the tensor behind it elements
    return sizes, [(sizes[k + 1], s // sizes[k + 1]) if k % 3 == 0 else None for k, s in enumerate(sizes)]


def _gradients(g, count, rows, cols, size):
    """Matrices as gradients are: a few strong directions on a broad floor."""
    rank = min(8, rows, cols)
    out = _normal(g, (count, rows, cols), 0.3 * size)
    left, right = _normal(g, (count, rows, rank), size), _normal(g, (count, rank, cols), 1.0)
    return out.add_(left @ (right * (0.5 ** torch.arange(rank, device=out.device))[:, None]))


def _plan(case):
    """Offsets of a row's tensors, and for every matrix its layer and where its momentum starts."""
    sizes, shapes = _layers(case)
    off = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int64)
    where, at = [], 0
    for k, s in enumerate(shapes):
        if s is not None:
            where.append((k, s, at))
            at += -(-s[0] * s[1] // BLOCK) * BLOCK
    return off, shapes, where, at


def _prepare_muon(case, g, st):
    off, shapes, where, e = _plan(case)
    n, d = case["n"], int(off[-1])
    X, G, m = _normal(g, (n, d), 0.05), _normal(g, (n, d), 1e-3), torch.zeros((n, e), dtype=torch.float32, device=_device())
    for k, (rows, cols), at in where:
        G[:, off[k]:off[k + 1]] = _gradients(g, n, rows, cols, 1e-3).view(n, -1)
        m[:, at:at + rows * cols] = _gradients(g, n, rows, cols, 5e-4).view(n, -1)
    st.update(X=X.to(TYPES[case["x"]]), G=G.to(TYPES[case["grad"]]), m=m, where=where, off=off)
    st["copy"] = X.to(TYPES[case["copy"]]) if case["copy"] else None
    st["factor"] = torch.rand(n, generator=g, device=_device()) if case["clip"] else None
    if own:
        import paper_1907_09356_b200 as choco
        st["opt"] = choco.Muon(st["X"], st["G"], off, shapes, weight_decay=DECAY, copy=st["copy"], beta=BETA, states=m.view(-1))


def _pixels(case, g, dtype, like=None):
    """An array [n, images, pixels, channels]; with a pitch, a slice of the channels of a wider one."""
    shape = (case["n"], case["images"], case["pixels"], case["channels"])
    wide = torch.empty((*shape[:3], shape[3] + case["pitch"]), dtype=dtype, device=_device())
    part = wide[..., :shape[3]]
    if like is not None:
        part.copy_(like)
    elif g is not None:
        part.copy_(_normal(g, shape, 1.0))
    return part


def _prepare_norm(case, g, st):
    n, c, k = case["n"], case["channels"], case["groups"]
    # channels of convolutions: each has its own size and offset
    x = _normal(g, (n, case["images"], case["pixels"], c), 1.0)
    x *= torch.rand(c, generator=g, device=_device()).add_(0.5)
    x += _normal(g, (c,), 0.5)
    st["x"] = _pixels(case, None, TYPES[case["x"]], x)
    del x
    param = TYPES[case["param"]]
    # scale and shift behind one another in the workers' rows, as the layers of a network are
    row = 2 * c + 3
    st["X"] = torch.zeros((n, row), dtype=param, device=_device())
    st["weight"], st["bias"] = st["X"][:, :c], st["X"][:, c:2 * c]
    st["weight"].copy_(_normal(g, (n, c), 0.2) + 1.0)
    st["bias"].copy_(_normal(g, (n, c), 0.2))
    stats = (n, case["images"], k)
    st["mean"], st["rstd"] = (torch.empty(stats, dtype=torch.float32, device=_device()) for _ in range(2))
    if case["op"] == "norm":
        st["y"] = _pixels(case, None, TYPES[case["y"]])
    else:
        x = st["x"].double().unflatten(3, (k, -1)) if st["x"].numel() < 30_000_000 else st["x"].float().unflatten(3, (k, -1))
        mean = x.mean(dim=(2, 4))
        var = (x - mean[:, :, None, :, None]).square_().mean(dim=(2, 4))
        st["mean"].copy_(mean)
        st["rstd"].copy_((var + EPS).rsqrt())
        del x
        st["dy"] = _pixels(case, g, TYPES[case["y"]])
        st["dx"] = _pixels(case, None, TYPES[case["x"]])
        st["G"] = _normal(g, (n, row), 1.0).to(torch.float32) if case["add"] else torch.zeros((n, row), device=_device())
        st["dweight"], st["dbias"] = st["G"][:, :c], st["G"][:, c:2 * c]
    if own:
        import paper_1907_09356_b200 as choco
        st["norm"] = choco.GroupNorm(n, c, k, max_images=case["images"], eps=EPS, activation=case["act"])


def prepare(case, seed):
    g, st = _generator(seed), {"case": case}
    if case["op"] == "muon":
        _prepare_muon(case, g, st)
    elif case["op"] == "orthogonalize":
        st["in"] = [_gradients(g, *s, 1e-3).to(TYPES[case["input"]]) for s in _matrices(case)]
        st["out"] = [torch.empty_like(u, dtype=TYPES[case["output"]]) for u in st["in"]]
        if own:
            import paper_1907_09356_b200 as choco
            st["orthogonalizer"] = choco.Orthogonalizer(st["in"], st["out"])
    else:
        _prepare_norm(case, g, st)
    return st


# --------------------------------------------------------------------------- plain forms


def _plain_orthogonal(u):
    """[count, rows, cols] in 32 bits."""
    tall = u.shape[1] > u.shape[2]
    x = (u.mT if tall else u).contiguous()
    norm = (x * x).sum(dim=(1, 2), keepdim=True).sqrt()
    x = x / torch.where(norm > 0, norm, 1.0)
    a, b, c = COEFFICIENTS
    for _ in range(STEPS):
        s = x @ x.mT
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.mT if tall else x


def _plain_muon(st, case):
    n, off = case["n"], st["off"]
    for k, (rows, cols), at in st["where"]:
        x = st["X"][:, off[k]:off[k + 1]]
        g = st["G"][:, off[k]:off[k + 1]].float()
        if st["factor"] is not None:
            g = g * st["factor"][:, None]
        m = st["m"][:, at:at + rows * cols]
        m.copy_(m * _f32(BETA) + g * _f32(1 - BETA))
        o = _plain_orthogonal((m * _f32(BETA) + g * _f32(1 - BETA)).view(n, rows, cols)).reshape(n, -1)
        new = x.float()
        new = new - (o * _f32(LR * math.sqrt(max(1.0, rows / cols))) + new * _f32(LR * DECAY))
        x.copy_(new)
        if st["copy"] is not None:
            st["copy"][:, off[k]:off[k + 1]] = new
    return _muon_outputs(st)


def _muon_outputs(st):
    out = {"x": st["X"], "m": st["m"]}
    if st["copy"] is not None:
        out["copy"] = st["copy"]
    return out


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "silu":
        return z / (1 + (-z).exp())
    return z * (0.5 * (1 + (z * math.sqrt(0.5)).erf())) if act == "gelu" else z


def _act_grad(z, act):
    if act == "silu":
        s = 1 / (1 + (-z).exp())
        return s * (1 + z * (1 - s))
    if act == "gelu":
        return 0.5 * (1 + (z * math.sqrt(0.5)).erf()) + z * (z * z * -0.5).exp() * (1 / math.sqrt(2 * math.pi))
    return torch.ones_like(z)


def _wide(v):
    """Of groups (n, images, groups) or of channels (n, channels), for arrays [n, images, pixels, groups, channels of one]."""
    return v[:, :, None, :, None]


def _plain_norm(st, case):
    k = case["groups"]
    x = st["x"].float().unflatten(3, (k, -1))
    mean = x.mean(dim=(2, 4))
    x = x - _wide(mean)
    rstd = (x.square().mean(dim=(2, 4)) + EPS).rsqrt()
    per = lambda t: t.float().unflatten(1, (k, -1))[:, None, None]  # noqa: E731
    z = x.mul_(_wide(rstd)).mul_(per(st["weight"])).add_(per(st["bias"]))
    st["y"].copy_(_act(z, case["act"]).flatten(3))
    st["mean"].copy_(mean)
    st["rstd"].copy_(rstd)
    return {"y": st["y"], "mean": st["mean"], "rstd": st["rstd"]}


def _open(st, case, xhat):
    """Where z > 0, in 64 bits: next to that border 32 would put some elements on the other side."""
    k = case["groups"]
    per = lambda t: t.double().unflatten(1, (k, -1))[:, None, None]  # noqa: E731
    z = xhat.double() if xhat is not None else (st["x"].double().unflatten(3, (k, -1)) - _wide(st["mean"].double())).mul_(_wide(st["rstd"].double()))
    return z.mul_(per(st["weight"])).add_(per(st["bias"])) > 0


def _plain_norm_grad(st, case):
    k = case["groups"]
    xhat = (st["x"].float().unflatten(3, (k, -1)) - _wide(st["mean"])).mul_(_wide(st["rstd"]))
    dz = st["dy"].float().unflatten(3, (k, -1))
    w = st["weight"].float().unflatten(1, (k, -1))[:, None, None]
    if case["act"] == "relu":
        dz = torch.where(_open(st, case, None), dz, 0.0)
    elif case["act"] != "none":
        dz = dz * _act_grad(xhat * w + st["bias"].float().unflatten(1, (k, -1))[:, None, None], case["act"])
    db, dw = dz.sum(dim=(1, 2)).flatten(1), (dz * xhat).sum(dim=(1, 2)).flatten(1)
    dz = dz * w
    first, second = dz.mean(dim=(2, 4)), (dz * xhat).mean(dim=(2, 4))
    dx = dz.sub_(_wide(first)).sub_(xhat.mul_(_wide(second))).mul_(_wide(st["rstd"]))
    st["dx"].copy_(dx.flatten(3))
    st["dweight"].copy_(st["dweight"] + dw if case["add"] else dw)
    st["dbias"].copy_(st["dbias"] + db if case["add"] else db)
    return {"dx": st["dx"], "dweight": st["dweight"], "dbias": st["dbias"]}


# --------------------------------------------------------------------------- one pass


def run(st):
    case = st["case"]
    if not own:
        if case["op"] == "orthogonalize":
            return list(map(lambda u, o: o.copy_(_plain_orthogonal(u.float())), st["in"], st["out"]))
        return {"muon": _plain_muon, "norm": _plain_norm, "norm_grad": _plain_norm_grad}[case["op"]](st, case)
    if case["op"] == "orthogonalize":
        st["orthogonalizer"].apply()
        return st["out"]
    if case["op"] == "muon":
        st["opt"].step(LR, st["factor"])
        return _muon_outputs(st)
    if case["op"] == "norm":
        st["norm"].forward(st["x"], st["weight"], st["bias"], st["y"], st["mean"], st["rstd"])
        return {"y": st["y"], "mean": st["mean"], "rstd": st["rstd"]}
    st["norm"].backward(st["x"], st["dy"], st["weight"], st["bias"], st["mean"], st["rstd"], st["dx"], st["dweight"], st["dbias"],
                        accumulate=case["add"])
    return {"dx": st["dx"], "dweight": st["dweight"], "dbias": st["dbias"]}


# --------------------------------------------------------------------------- what a pass cannot do without


def work(case):
    if case["op"] == "orthogonalize":
        elements = sum(k * a * b for k, a, b in _matrices(case))
        return {"bytes": elements * (SIZE[case["input"]] + SIZE[case["output"]]), "flops": sum(k * _products(a, b) for k, a, b in _matrices(case))}
    if case["op"] == "muon":
        shapes = [s for s in _layers(case)[1] if s is not None]
        elements = case["n"] * sum(a * b for a, b in shapes)
        each = 2 * SIZE[case["x"]] + SIZE[case["grad"]] + SIZE[case["copy"]] + 8
        return {"bytes": elements * each, "flops": case["n"] * sum(_products(a, b) for a, b in shapes)}
    rows = case["n"] * case["images"]
    elements = rows * case["pixels"] * case["channels"]
    params, stats = 2 * case["n"] * case["channels"], 8 * rows * case["groups"]
    if case["op"] == "norm":
        return {"bytes": elements * (SIZE[case["x"]] + SIZE[case["y"]]) + params * SIZE[case["param"]] + stats, "flops": 8 * elements}
    grads = params * (8 if case["add"] else 4)
    return {"bytes": elements * (2 * SIZE[case["x"]] + SIZE[case["y"]]) + params * SIZE[case["param"]] + grads + stats, "flops": 16 * elements}


# --------------------------------------------------------------------------- in 64 bits


def _exact_orthogonal(u):
    """One matrix: the odd polynomial on it, from its smaller side."""
    if u.shape[0] > u.shape[1]:
        return _exact_orthogonal(u.t()).t()
    size = torch.linalg.matrix_norm(u)
    y = u / size if float(size) > 0 else u
    a, b, c = COEFFICIENTS
    one = torch.eye(u.shape[0], dtype=torch.float64, device=u.device)
    for _ in range(STEPS):
        square = y @ y.t()
        y = (a * one + square @ (b * one + c * square)) @ y
    return y


def _exact_muon(st, case):
    x, m = st["X"].double(), st["m"].double()
    grad = st["G"].double()
    if st["factor"] is not None:
        grad = grad * st["factor"].double()[:, None]
    for i in range(case["n"]):
        for k, (rows, cols), at in st["where"]:
            here = slice(int(st["off"][k]), int(st["off"][k + 1]))
            mi = m[i, at:at + rows * cols]
            mi += (1 - BETA) * (grad[i, here] - mi)
            u = mi + (1 - BETA) * (grad[i, here] - mi)
            o = _exact_orthogonal(u.view(rows, cols)).reshape(-1)
            x[i, here] = x[i, here] * (1 - LR * DECAY) - LR * max(1.0, rows / cols) ** 0.5 * o
    out = {"x": x, "m": m}
    if st["copy"] is not None:
        out["copy"] = st["copy"].double()
        for k, _, _ in st["where"]:
            here = slice(int(st["off"][k]), int(st["off"][k + 1]))
            out["copy"][:, here] = x[:, here]
    return out


def _exact_norm(st, case):
    n, c, k = case["n"], case["channels"], case["groups"]
    y = torch.empty(st["y"].shape, dtype=torch.float64, device=_device())
    mean, rstd = (torch.empty(st["mean"].shape, dtype=torch.float64, device=_device()) for _ in range(2))
    for i in range(n):
        x = st["x"][i].double().reshape(case["images"], case["pixels"], k, c // k).transpose(1, 2)   # images, groups, pixels, channels of a group
        var, mu = torch.var_mean(x, dim=(2, 3), correction=0)
        mean[i], rstd[i] = mu, 1 / torch.sqrt(var + EPS)
        z = ((x - mu[..., None, None]) * rstd[i][..., None, None]).transpose(1, 2).flatten(2)
        z = z * st["weight"][i].double() + st["bias"][i].double()
        y[i] = {"none": lambda v: v, "relu": torch.relu, "silu": lambda v: v * torch.sigmoid(v),
                "gelu": lambda v: v * torch.special.ndtr(v)}[case["act"]](z)
    return {"y": y, "mean": mean, "rstd": rstd}


def _exact_norm_grad(st, case):
    n, c, k = case["n"], case["channels"], case["groups"]
    dx = torch.empty(st["dx"].shape, dtype=torch.float64, device=_device())
    dweight, dbias = st["dweight"].double(), st["dbias"].double()
    if not case["add"]:
        dweight, dbias = torch.zeros_like(dweight), torch.zeros_like(dbias)
    for i in range(n):
        spread = lambda t: t.double().repeat_interleave(c // k, dim=-1)[:, None]  # noqa: E731  a group's value for each of its channels
        scale = spread(st["rstd"][i])
        xhat = (st["x"][i].double() - spread(st["mean"][i])) * scale
        w = st["weight"][i].double()
        z = w * xhat + st["bias"][i].double()
        sig = torch.sigmoid(z) if case["act"] == "silu" else None
        slope = {"none": lambda: 1.0, "relu": lambda: (z > 0).double(), "silu": lambda: sig + z * sig * (1 - sig),
                 "gelu": lambda: torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)}[case["act"]]()
        dz = st["dy"][i].double() * slope
        del z, sig, slope
        dbias[i] += dz.sum(dim=(0, 1))
        dweight[i] += (dz * xhat).sum(dim=(0, 1))
        dz *= w
        over = lambda t: t.sum(dim=1).unflatten(1, (k, c // k)).mean(dim=2) / case["pixels"]  # noqa: E731
        dx[i] = (dz - spread(over(dz)) - xhat * spread(over(dz * xhat))) * scale
    return {"dx": dx, "dweight": dweight, "dbias": dbias}


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "orthogonalize":
        return [torch.stack([_exact_orthogonal(u.double()) for u in us]) for us in st["in"]]
    return {"muon": _exact_muon, "norm": _exact_norm, "norm_grad": _exact_norm_grad}[case["op"]](st, case)
