"""The example that runs group norm, clipping, Muon, AdamW and gossip together: its gradients, and the calls back to back."""
import math
import os
import sys

import pytest
import torch

import paper_1907_09356_b200 as choco

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))
pytestmark = pytest.mark.gpu


def batch_of(model, gen, size=9):
    images = torch.randn((model.n, model.batch, size, size, 3), generator=gen, device="cuda")
    return images, torch.randint(0, 10, (model.n, model.batch), generator=gen, device="cuda")


def test_gradients_are_those_of_the_model():
    import image_model
    gen = torch.Generator(device="cuda").manual_seed(1)
    model = image_model.ImageModel(3, 5)
    X = model.init(gen, "cuda")
    X += 0.1 * torch.randn(X.shape, generator=gen, device="cuda")
    G = torch.full_like(X, float("nan"))
    images, labels = batch_of(model, gen)
    loss = model.gradients(X, G, images, labels)

    rows = X.double().requires_grad_()
    x = images.double()
    for k, gn in enumerate(model.norms):
        cols = image_model.unfold(x)
        z = torch.einsum("nbhwc,noc->nbhwo", cols, model.layer(rows, 3 * k))
        g = z.unflatten(-1, (gn.groups, -1))
        mean = g.mean(dim=(2, 3, 5), keepdim=True)
        z = ((g - mean) / torch.sqrt((g - mean).square().mean(dim=(2, 3, 5), keepdim=True) + 1e-5)).flatten(4)
        per = lambda j: model.layer(rows, j)[:, None, None, None]  # noqa: E731
        x = torch.relu(z * per(3 * k + 1) + per(3 * k + 2))
    logits = torch.einsum("nbc,noc->nbo", x.mean(dim=(2, 3)), model.layer(rows, 6)) + model.layer(rows, 7)[:, None]
    want = torch.nn.functional.cross_entropy(logits.flatten(0, 1), labels.flatten(), reduction="none").view(3, 5).mean(1)
    want.sum().backward()
    assert float((loss.double() - want.detach()).abs().max()) < 1e-5
    # float32 products over up to 405 terms, two layers deep, and the few relus within a rounding of 0 of either side
    assert float((G.double() - rows.grad).abs().max()) < 1e-3 * float(rows.grad.abs().max())
    assert float((G.double() - rows.grad).norm()) < 1e-4 * float(rows.grad.norm())
    model.close()


@pytest.mark.parametrize("q", ["topk", "sign"])
def test_it_runs(q):
    import image_model
    losses, distances = image_model.train(workers=4, steps=30, q=q, batch=8)
    assert len(losses) == 30 and all(math.isfinite(v) for v in losses) and all(math.isfinite(v) for v in distances)


def test_calls_back_to_back_see_what_the_call_before_wrote():
    """Every kernel may start while the one before it ends: against the same calls with a wait for the device after each."""
    import image_model
    gen = torch.Generator(device="cuda").manual_seed(2)
    model = image_model.ImageModel(4, 6, widths=(24, 40), groups=8)
    X0 = model.init(gen, "cuda")
    X0 += 0.1 * torch.randn(X0.shape, generator=gen, device="cuda")
    z0 = torch.randn((4, 6, 200, 24), generator=gen, device="cuda")
    others = [k for k, s in enumerate(model.shapes) if s is None]

    def steps(wait):
        X, G, z = X0.clone(), X0.flip(1).contiguous() * 0.01, z0.clone()
        y, dz = torch.empty_like(z), torch.empty_like(z)
        mean, rstd = torch.empty((4, 6, 8), device="cuda"), torch.empty((4, 6, 8), device="cuda")
        norm, factor = torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda")
        norms, adamw = choco.AdamW(None, G, model.off), choco.AdamW(X, G, model.off, layers=others)
        muon = choco.Muon(X, G, model.off, model.shapes, weight_decay=0.01)
        wide = choco.Orthogonalizer([z.view(4, -1, 200 * 6)[:, :20]], [y.view(4, -1, 200 * 6)[:, :20]])
        w, b, dw, db = (model.layer(t, k) for t in (X, G) for k in (1, 2))
        gn = model.norms[0]
        for _ in range(10):
            for call in (lambda: gn.forward(z, w, b, y, mean, rstd), lambda: gn.backward(z, y, w, b, mean, rstd, dz, dw, db, accumulate=True),
                         lambda: wide.apply(), lambda: gn.backward(z, y, w, b, mean, rstd, dz, dw, db, accumulate=True), lambda: norms.grad_norm(1.0, norm, factor),
                         lambda: muon.step(0.02, factor), lambda: adamw.step(1e-3, factor), lambda: muon.step(0.01)):
                call()
                if wait:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        muon.status()
        out = [X.clone(), G.clone(), y, dz, mean, rstd, norm, factor, muon.m.clone(), adamw.m.clone(), adamw.v.clone()]
        for part in (norms, adamw, muon, wide):
            part.close()
        return out

    want = steps(True)
    for _ in range(3):
        for a, e in zip(steps(False), want):
            assert torch.equal(a, e)
    model.close()


def test_the_matrix_of_the_language_model_by_muon():
    import language_model
    losses, distances = language_model.train(workers=4, steps=20, vocab=128, dim=32, optimizer="muon")
    assert all(math.isfinite(v) for v in losses) and all(math.isfinite(v) for v in distances)
