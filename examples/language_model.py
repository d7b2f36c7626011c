"""A small language model trained by n workers that gossip: token lookup, tied output layer, gradient
of the lookup, per-worker clipping, AdamW and the CHOCO-Gossip step, all on the rows of X and G.

    python examples/language_model.py [--workers 8] [--steps 200] [--bits 8] [--q topk]

The model is a bigram model: logits = scale * E[token] W E^T with one table E for input and output and a
square matrix W, trained on the sequences of a random Markov chain, every worker on a chain of its
own with a shared part.  Its three products are library products; what the library of this
repository does is the rest of the step.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1907_09356_b200 as choco  # noqa: E402
import workloads  # noqa: E402


def train(workers=8, steps=200, bits=32, q="topk", vocab=512, dim=64, batch=16, length=33, lr=3e-3, gamma=None, clip=1.0, seed=0,
          log=None):
    """Returns (mean loss per step, consensus distance per step)."""
    if gamma is None:       # consensus stepsizes in the stable range of each operator
        gamma = {"topk": 0.1, "randk": 0.03, "qsgd": 0.1, "sign": 0.4, "identity": 1.0}[q]
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    w = workloads.ring(workers)
    sizes = [vocab * dim, dim * dim, dim]                       # table, matrix, bias of the hidden layer
    off = workloads.layer_offsets(sizes)
    d = int(off[-1])
    X = (torch.randn(d, generator=gen, device=dev) * 0.05).repeat(workers, 1)   # all start from one model
    X[:, off[1]:off[2]] += torch.eye(dim, device=dev).reshape(-1)
    X[:, off[2]:] = 0
    Xhat, S, G = torch.zeros_like(X), torch.zeros_like(X), torch.zeros_like(X)
    # a chain whose next token is one of four; the workers prefer different ones of them
    successors = torch.randint(0, vocab, (vocab, 4), generator=gen, device=dev)
    prefer = torch.softmax(torch.randn((workers, 4), generator=gen, device=dev), dim=1)

    count = batch * (length - 1)
    scale = dim ** 0.5
    emb = choco.Embedding(workers, vocab, dim, count, table_ld=d, scale=scale)
    opt = choco.AdamW(X, G, off, weight_decay=[0.01, 0.01, 0.0], state_bits=bits, rounding="random" if bits == 8 else "nearest", seed=seed)
    kw = dict(k=max(1, d // 20)) if q in ("topk", "randk") else dict(s=16, bucket=512) if q == "qsgd" else {}
    gossip = choco.Choco(w, d, q, seed=seed, **kw)
    choco.choco_set_carry(gossip.ctx, False)                    # AdamW changes X between two gossip steps
    norm, factor = torch.zeros(workers, device=dev), torch.zeros(workers, device=dev)
    rows = torch.empty((workers, count, dim), device=dev)
    E = X[:, :off[1]].unflatten(1, (vocab, dim))
    W = X[:, off[1]:off[2]].unflatten(1, (dim, dim))
    bias = X[:, off[2]:]
    worker = torch.arange(workers, device=dev)[:, None]
    losses, distances = [], []
    for t in range(steps):
        seq = torch.randint(0, vocab, (workers, batch, 1), generator=gen, device=dev)
        for _ in range(length - 1):
            pick = torch.multinomial(prefer, batch, replacement=True, generator=gen)
            seq = torch.cat([seq, successors[seq[:, :, -1], pick][:, :, None]], dim=2)
        tokens, target = seq[:, :, :-1].reshape(workers, -1).contiguous(), seq[:, :, 1:].reshape(workers, -1)

        emb.forward(X, tokens, rows)                            # scale * E[token]
        hidden = rows @ W + bias[:, None]
        logp = torch.log_softmax(hidden @ E.transpose(1, 2), dim=2)
        losses.append(float(-logp.gather(2, target[..., None]).mean()))
        dlogits = logp.exp_()
        dlogits[worker, torch.arange(count, device=dev), target] -= 1
        dlogits /= count
        dhidden = dlogits @ E
        G[:, :off[1]] = (dlogits.transpose(1, 2) @ hidden).flatten(1)   # the output layer's part of the table's gradient
        G[:, off[1]:off[2]] = (rows.transpose(1, 2) @ dhidden).flatten(1)
        G[:, off[2]:] = dhidden.sum(1)
        emb.backward(tokens, dhidden @ W.transpose(1, 2), G, accumulate=True)   # and the lookup's, added to it
        opt.grad_norm(clip, norm, factor)
        opt.step(lr, factor)
        gossip.gossip_step(X, Xhat, S, gamma)
        distances.append(choco.choco_consensus_error(gossip.ctx, X))
        if log and (t % 20 == 0 or t == steps - 1):
            log(f"step {t:4d}  loss {losses[-1]:.4f}  consensus distance {distances[-1]:.4f}  largest norm {float(norm.max()):.3f}")
    emb.close()
    opt.close()
    gossip.close()
    return np.asarray(losses), np.asarray(distances)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--workers", type=int, default=8)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--bits", type=int, choices=(8, 32), default=32)
    ap.add_argument("--q", choices=sorted(choco.Q_KINDS), default="topk")
    a = ap.parse_args()
    train(a.workers, a.steps, a.bits, a.q, log=print)
