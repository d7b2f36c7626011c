"""A small convolutional network trained by n workers that gossip: group norm in place of batch statistics (each worker
sees mostly classes of its own), per-worker clipping, Muon for the filters and the classifier, AdamW for scales, shifts and
biases, and the CHOCO-Gossip step, all on the rows of X and G.

    python examples/image_model.py [--workers 8] [--steps 100] [--q topk]

Two 3x3 convolutions (as products with unfolded pixels, library products), each followed by group norm and relu, the mean over
the pixels and a classifier, on images of ten classes: a class is a random pattern, an image the pattern with noise.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1907_09356_b200 as choco  # noqa: E402
import workloads  # noqa: E402

CLASSES = 10


def unfold(x):
    """[n, b, h, w, c] -> [n, b, h, w, 9 c]: the 3x3 neighbours of every pixel, zeros outside."""
    h, w = x.shape[2:4]
    wide = torch.nn.functional.pad(x, (0, 0, 1, 1, 1, 1))
    return torch.cat([wide[:, :, i:i + h, j:j + w] for i in range(3) for j in range(3)], dim=-1)


def fold(cols):
    """The transpose of unfold."""
    n, b, h, w, c = cols.shape
    wide = torch.zeros((n, b, h + 2, w + 2, c // 9), dtype=cols.dtype, device=cols.device)
    for k, part in enumerate(cols.split(c // 9, dim=-1)):
        wide[:, :, k // 3:k // 3 + h, k % 3:k % 3 + w] += part
    return wide[:, :, 1:-1, 1:-1]


class ImageModel:
    """The network's parameters are the layers of a row of X, its gradients those of a row of G."""

    def __init__(self, workers, batch, widths=(16, 32), groups=4):
        self.n, self.batch = workers, batch
        self.shapes, self.norms, c = [], [], 3
        for width in widths:                                    # filters, scale, shift
            self.shapes += [(width, 9 * c), None, None]
            self.norms.append(choco.GroupNorm(workers, width, groups, max_images=batch, activation="relu"))
            c = width
        self.widths = widths
        self.shapes += [(CLASSES, c), None]
        sizes = []
        for k, s in enumerate(self.shapes):
            sizes.append(s[0] * s[1] if s else self.shapes[k - 1 if self.shapes[k - 1] else k - 2][0])
        self.off = workloads.layer_offsets(sizes)

    def layer(self, rows, k):
        part = rows[:, self.off[k]:self.off[k + 1]]
        return part.unflatten(1, self.shapes[k]) if self.shapes[k] else part

    def init(self, gen, device):
        X = torch.zeros(int(self.off[-1]), device=device)
        for k, s in enumerate(self.shapes):
            here = slice(int(self.off[k]), int(self.off[k + 1]))
            if s:
                X[here] = torch.randn(s[0] * s[1], generator=gen, device=device) / s[1] ** 0.5
            elif k % 3 == 1 and k < 3 * len(self.widths):
                X[here] = 1.0                                   # scales
        return X.repeat(self.n, 1)                              # all start from one model

    def gradients(self, X, G, images, labels):
        """Writes the gradient of the mean loss into G; returns the loss of every worker.  images [n, batch, h, w, 3]."""
        n, b, h, w = images.shape[:4]
        stats = [[torch.empty((n, b, gn.groups), device=X.device) for _ in range(2)] for gn in self.norms]
        x, kept = images, []
        for k, gn in enumerate(self.norms):
            cols = unfold(x).flatten(1, 3)
            z = (cols @ self.layer(X, 3 * k).mT).unflatten(1, (b, h, w))
            x = torch.empty_like(z)
            gn.forward(z, self.layer(X, 3 * k + 1), self.layer(X, 3 * k + 2), x, *stats[k])
            kept.append((cols, z))
        last = 3 * len(self.norms)
        mean = x.mean(dim=(2, 3))
        logp = torch.log_softmax(mean @ self.layer(X, last).mT + self.layer(X, last + 1)[:, None], dim=2)
        loss = -logp.gather(2, labels[..., None]).mean(dim=(1, 2))
        d = logp.exp().scatter_add_(2, labels[..., None], torch.full(labels.shape, -1.0, device=X.device)[..., None]) / b
        self.layer(G, last).copy_(d.mT @ mean)
        self.layer(G, last + 1).copy_(d.sum(1))
        dx = (d @ self.layer(X, last))[:, :, None, None].expand_as(x) / (h * w)
        for k in reversed(range(len(self.norms))):
            cols, z = kept[k]
            dx = dx.contiguous()
            self.norms[k].backward(z, dx, self.layer(X, 3 * k + 1), self.layer(X, 3 * k + 2), *stats[k], dx, self.layer(G, 3 * k + 1),
                                   self.layer(G, 3 * k + 2))   # in place: dx now is the convolution's
            dz = dx.flatten(1, 3)
            self.layer(G, 3 * k).copy_(dz.mT @ cols)
            if k > 0:
                dx = fold((dz @ self.layer(X, 3 * k)).unflatten(1, (b, h, w)))
        return loss

    def close(self):
        for gn in self.norms:
            gn.close()


def train(workers=8, steps=100, q="topk", batch=32, size=12, lr=0.02, gamma=None, clip=1.0, seed=0, log=None):
    """Returns (mean loss per step, consensus distance per step)."""
    if gamma is None:       # consensus stepsizes in the stable range of each operator
        gamma = {"topk": 0.1, "randk": 0.03, "qsgd": 0.1, "sign": 0.4, "identity": 1.0}[q]
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    model = ImageModel(workers, batch)
    X = model.init(gen, dev)
    d = X.shape[1]
    G, Xhat, S = torch.zeros_like(X), torch.zeros_like(X), torch.zeros_like(X)
    patterns = torch.randn((CLASSES, size, size, 3), generator=gen, device=dev)
    prefer = torch.softmax(2 * torch.randn((workers, CLASSES), generator=gen, device=dev), dim=1)   # the workers' data differ

    others = [k for k, s in enumerate(model.shapes) if s is None]
    norms = choco.AdamW(None, G, model.off)                     # clipping looks at all layers
    muon = choco.Muon(X, G, model.off, model.shapes, weight_decay=0.01)
    adamw = choco.AdamW(X, G, model.off, layers=others)
    kw = dict(k=max(1, d // 20)) if q in ("topk", "randk") else dict(s=16, bucket=512) if q == "qsgd" else {}
    gossip = choco.Choco(workloads.ring(workers), d, q, seed=seed, **kw)
    choco.choco_set_carry(gossip.ctx, False)                    # the optimizers change X between two gossip steps
    norm, factor = torch.zeros(workers, device=dev), torch.zeros(workers, device=dev)
    losses, distances = [], []
    for t in range(steps):
        labels = torch.multinomial(prefer, batch, replacement=True, generator=gen)
        images = patterns[labels] + torch.randn((workers, batch, size, size, 3), generator=gen, device=dev)
        losses.append(float(model.gradients(X, G, images, labels).mean()))
        norms.grad_norm(clip, norm, factor)
        muon.step(lr, factor)
        adamw.step(0.1 * lr, factor)
        gossip.gossip_step(X, Xhat, S, gamma)
        distances.append(choco.choco_consensus_error(gossip.ctx, X))
        if log and (t % 20 == 0 or t == steps - 1):
            log(f"step {t:4d}  loss {losses[-1]:.4f}  consensus distance {distances[-1]:.4f}  largest norm {float(norm.max()):.3f}")
    muon.status()
    for part in (model, norms, muon, adamw, gossip):
        part.close()
    return np.asarray(losses), np.asarray(distances)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--workers", type=int, default=8)
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--q", choices=sorted(choco.Q_KINDS), default="topk")
    a = ap.parse_args()
    train(a.workers, a.steps, a.q, log=print)
