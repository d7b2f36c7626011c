"""Group norm and Muon where offsets of elements pass 32 bits."""
import pytest
import torch

import paper_1907_09356_b200 as choco

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, F16 = torch.float32, torch.float16


@pytest.mark.parametrize("axis", [0, 1, 2])
def test_group_norm_of_pixels_far_apart(axis):
    """The same values, near each other and far apart along one axis, give the same bits."""
    shape, groups = (2, 2, 5, 16), 4
    gen = torch.Generator(device=DEV).manual_seed(1)
    near = torch.randn(shape, generator=gen, device=DEV).to(F16)
    dy = torch.randn(shape, generator=gen, device=DEV).to(F16)
    w, b = torch.randn((2, 16), generator=gen, device=DEV), torch.randn((2, 16), generator=gen, device=DEV)
    strides = [160, 80, 16, 1]
    strides[axis] = (1 << 32) // (shape[axis] - 1) + 4096          # the last of the axis starts behind 2^32 elements
    for k in range(axis):                                          # axes outside of it are strewn between
        strides[k] = 1024 * (k + 1)
    memory = torch.empty(strides[axis] * (shape[axis] - 1) + 8192, dtype=F16, device=DEV)
    far = memory.as_strided(shape, strides)
    far.copy_(near)
    gn = choco.GroupNorm(2, 16, groups, max_images=2, activation="silu")
    out = {}
    for name, x in (("near", near.clone()), ("far", far)):
        y, mean, rstd = torch.empty_like(near), torch.empty((2, 2, groups), device=DEV), torch.empty((2, 2, groups), device=DEV)
        dx, dw, db = torch.empty_like(near), torch.empty_like(w), torch.empty_like(b)
        gn.forward(x, w, b, y, mean, rstd)
        gn.backward(x, dy, w, b, mean, rstd, dx, dw, db)
        gn.forward(x, w, b, x)                                     # and written far apart
        out[name] = (y, mean, rstd, dx, dw, db, x.clone(memory_format=torch.contiguous_format))
    for a, c in zip(out["near"], out["far"]):
        assert a.isfinite().all() and torch.equal(a, c)
    assert torch.equal(out["near"][0], out["near"][6])
    gn.close()


@pytest.mark.parametrize("shape", [(12, 200), (200, 12), (140, 300), (300, 140)])
def test_muon_of_rows_far_apart(shape):
    rows, cols = shape
    pitch = (1 << 32) // (rows - 1) + 512
    memory = torch.empty(pitch * (rows - 1) + 512, dtype=F16, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(2)
    u = torch.randn(shape, generator=gen, device=DEV).to(F16)
    far = memory.as_strided(shape, (pitch, 1))
    far.copy_(u)
    near, back = torch.empty(shape, dtype=F32, device=DEV), torch.empty(shape, dtype=F32, device=DEV)
    for a, o in ((u, near), (far, back)):
        op = choco.Orthogonalizer([a], [o])
        op.apply()
        op.status()
        op.close()
    assert near.isfinite().all() and torch.equal(near, back)
    op = choco.Orthogonalizer([u], [far])                          # and written far apart
    op.apply()
    op.status()
    op.close()
    # (aligned and other accesses add up alike, so it is the same float32 result, rounded)
    assert torch.equal(far.contiguous(), near.to(F16))
