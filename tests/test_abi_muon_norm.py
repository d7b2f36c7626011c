"""The calls of Muon and of group norm reject bad arguments on the host, before they touch a device (no GPU needed)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_1907_09356_b200 as choco
from paper_1907_09356_b200 import build as choco_build


@pytest.fixture(scope="module")
def lib():
    choco_build.build()
    return choco.load()


def _muon(lib, matrix=None, n=1, beta=0.95, abc=choco.MUON_COEFFICIENTS, nesterov=1, steps=5, products=0, groups=2, more=None):
    t = np.zeros(2 if more else 1, dtype=choco.MUON_MATRIX)
    t["x"], t["g"], t["rows"], t["cols"], t["lr_scale"] = 1 << 20, 1 << 30, 10, 20, 1.0
    for k, v in (matrix or {}).items():
        t[0][k] = v
    for k, v in (more or {}).items():
        t[1][k] = v
    p = choco.choco_muon_params(beta, *abc, nesterov, steps, products, groups)
    h = ctypes.c_void_p()
    rc = lib.choco_muon_init(ctypes.byref(h), len(t) if n else 0, t.ctypes.data, ctypes.byref(p))
    assert h.value is None or rc == 0
    if h.value:
        lib.choco_muon_destroy(h)
    return rc


@pytest.mark.parametrize("kw,code", [
    (dict(n=0), -1), (dict(beta=1.0), -1), (dict(beta=-0.1), -1), (dict(beta=float("nan")), -1), (dict(nesterov=2), -1), (dict(steps=-1), -1), (dict(steps=65), -1),
    (dict(products=2), -6), (dict(groups=0), -1), (dict(abc=(float("nan"), 0, 0)), -1), (dict(abc=(4.0, 0.0, 0.0)), -1), (dict(abc=(1.5, -20.0, 0.0)), -1),
    (dict(abc=(1.0, 1.0, 1.0)), -1), (dict(matrix=dict(rows=-1)), -1), (dict(matrix=dict(cols=-1)), -1), (dict(matrix=dict(x=0)), -1), (dict(matrix=dict(g=0)), -1),
    (dict(matrix=dict(x_ld=19)), -1), (dict(matrix=dict(g_ld=19)), -1), (dict(matrix=dict(copy_ld=-1)), -1), (dict(matrix=dict(group=2)), -1),
    (dict(matrix=dict(group=-1)), -1), (dict(matrix=dict(x_dtype=3)), -1), (dict(matrix=dict(g_dtype=-1)), -1), (dict(matrix=dict(copy_dtype=4)), -1),
    (dict(matrix=dict(weight_decay=-1.0)), -1), (dict(matrix=dict(weight_decay=1e39)), -1), (dict(matrix=dict(lr_scale=float("inf"))), -1),
    (dict(matrix=dict(x=(1 << 20) + 2)), -5), (dict(matrix=dict(g=(1 << 30) + 1, g_dtype=1)), -5), (dict(matrix=dict(rows=1 << 15, cols=1 << 15)), -7),
    (dict(matrix=dict(rows=1, cols=(1 << 30) + 1)), -7), (dict(matrix=dict(x_ld=1 << 39)), -7), (dict(matrix=dict(g=1 << 20)), -1),
    (dict(matrix=dict(copy=(1 << 20) + 400)), -1), (dict(more=dict(x=(1 << 20) + 796)), -1), (dict(more=dict(x=1 << 25, g=(1 << 20) + 4)), -1)])
def test_muon_refusals(lib, kw, code):
    assert _muon(lib, **kw) == code


@pytest.mark.parametrize("kw", [dict(), dict(more=dict(x=(1 << 20) + 800)), dict(abc=(1.5, -0.5, 0.0)), dict(abc=(2.0, -1.5, 0.5)), dict(steps=0, abc=(0.0, 0.0, 0.0)),
                                dict(matrix=dict(rows=0, x=0, g=0)), dict(more=dict(x=1 << 25, g=(1 << 30) + 4))])
def test_muon_takes_what_is_in_order(lib, kw):
    assert _muon(lib, **kw) in (0, -3, -4)       # (there may be no device to go on with)


def test_muon_null_pointers(lib):
    assert lib.choco_muon_init(None, 1, None, None) == -1
    h, e = ctypes.c_void_p(), ctypes.c_int64()
    assert lib.choco_muon_init(ctypes.byref(h), 1, None, None) == -1
    assert lib.choco_muon_destroy(None) == -1 and lib.choco_muon_state_size(None, ctypes.byref(e), None) == -1
    assert lib.choco_muon_step(None, None, 0.1, None, None) == -1 and lib.choco_muon_orthogonalize(None, None) == -1
    assert lib.choco_muon_set_grads(None, None, None) == -1 and lib.choco_muon_status(None, None) == -1


def test_records_match_the_structs():
    d = np.dtype(choco.MUON_MATRIX)
    assert d.itemsize == 96
    assert [d.fields[f][1] for f in ("x", "g", "copy", "rows", "cols", "x_ld", "g_ld", "copy_ld", "x_dtype", "g_dtype", "copy_dtype", "group", "weight_decay",
                                     "lr_scale")] == [0, 8, 16, 24, 32, 40, 48, 56, 64, 68, 72, 76, 80, 88]
    assert ctypes.sizeof(choco.choco_muon_params) == 48 and ctypes.sizeof(choco.choco_group_norm_params) == 40
    assert ctypes.sizeof(choco.choco_pixels) == 40


@pytest.mark.parametrize("kw,code", [
    (dict(n=0), -1), (dict(groups=0), -1), (dict(groups=3), -1), (dict(channels=0), -1), (dict(max_images=-1), -1), (dict(eps=-1.0), -1), (dict(eps=1e39), -1),
    (dict(eps=float("nan")), -1), (dict(activation=4), -1), (dict(activation=-1), -1), (dict(n=65536), -7), (dict(channels=1 << 21, groups=1 << 20), -7),
    (dict(channels=2049, groups=1), -7), (dict(max_images=1 << 31), -7), (dict(max_images=1 << 62), -7)])
def test_group_norm_refusals(lib, kw, code):
    a = dict(n=2, groups=2, channels=8, max_images=0, eps=1e-5, activation=1, unused=0)
    a.update(kw)
    p = choco.choco_group_norm_params(*[a[f] for f, _ in choco.choco_group_norm_params._fields_])
    h = ctypes.c_void_p()
    assert lib.choco_group_norm_init(ctypes.byref(h), ctypes.byref(p)) == code and h.value is None


def test_group_norm_null_pointers(lib):
    h = ctypes.c_void_p()
    assert lib.choco_group_norm_init(None, None) == -1 and lib.choco_group_norm_init(ctypes.byref(h), None) == -1
    assert lib.choco_group_norm_destroy(None) == -1
    assert lib.choco_group_norm_forward(None, 1, 1, None, None, None, None, 0, 0, None, None, None) == -1
    assert lib.choco_group_norm_backward(None, 1, 1, None, None, None, None, None, 0, 0, None, None, None, None, 0, 0, 0, None) == -1


# --------------------------------------------------------------------------- what the binding checks by itself


@pytest.fixture
def no_library(monkeypatch):
    def no_call():
        raise AssertionError("the library was called")
    monkeypatch.setattr(choco, "load", no_call)


def refused(call, match):
    with pytest.raises(choco.ChocoError, match=match):
        call()


def test_momentum_is_that_of_the_list(no_library):
    h = choco.MuonHandle()
    h.describe(-1, 3, 2, 512)
    for bad in (None, torch.zeros(511), torch.zeros(512, dtype=torch.float64), torch.zeros(512, dtype=torch.float16), torch.zeros(1024)[::2]):
        refused(lambda: choco.choco_muon_step(h, bad, 0.1), "momentum must be|are not supported")
    refused(lambda: choco.choco_muon_step(h, torch.zeros(512), 0.1, torch.zeros(1)), "one element for each of 2 groups")
    refused(lambda: choco.choco_muon_set_grads(h, [4096] * 2), "3 matrices")
    with pytest.raises(AssertionError):
        choco.choco_muon_step(h, torch.zeros(512), 0.1, torch.zeros(2))


def norm(n=2, channels=8, groups=4):
    h = choco.GroupNormHandle()
    h.describe(-1, n, channels, groups)
    return h


def test_arrays_of_pixels(no_library):
    h = norm()
    x = torch.zeros((2, 3, 4, 5, 8))
    p, images, pixels = choco._pixels_of(h, "x", x)
    assert (p.worker, p.image, p.pixel, p.dtype, images, pixels) == (480, 160, 8, 0, 3, 20)
    p, images, pixels = choco._pixels_of(h, "x", torch.zeros((2, 3, 20, 11))[..., 1:9])
    assert (p.worker, p.image, p.pixel, images, pixels) == (660, 220, 11, 3, 20)
    p, images, pixels = choco._pixels_of(h, "x", x[:, :, :, :1])     # one column of pixels
    assert (p.pixel, pixels) == (40, 4)
    p, images, pixels = choco._pixels_of(h, "x", torch.zeros((2, 1, 20, 8), dtype=torch.bfloat16).expand(2, 3, 20, 8))
    assert (p.image, p.dtype) == (0, 1)
    for bad in (x[:1], x[..., :4], x.transpose(3, 4), x[:, :, :, ::2].transpose(2, 3), x[:, :, :, :3], x[0, 0, 0], torch.zeros((2, 8))):
        refused(lambda: choco._pixels_of(h, "x", bad), "must be|must have one stride")
    h.device = 1
    refused(lambda: choco._pixels_of(h, "x", x), "handle's GPU")


def test_parameters_and_statistics(no_library):
    h, x = norm(), torch.zeros((2, 3, 20, 8))
    w, row = torch.zeros((2, 8)), torch.zeros((2, 40))
    assert choco._channels_of(h, "w", None, None) == (8, 0) and choco._channels_of(h, "w", row[:, 3:11], row[:, 11:19]) == (40, 0)
    assert choco._channels_of(h, "w", w[:1].expand(2, 8), None) == (0, 0)
    for bad in ((w, row[:, :8]), (w, w.half()), (w[:1], None), (w[:, :7], None), (w.t(), None), (torch.zeros((2, 16))[:, ::2], None)):
        refused(lambda: choco._channels_of(h, "w", *bad), "must be|have one type")
    s = torch.zeros((2, 3, 4))
    for bad in (torch.zeros((2, 3, 3)), torch.zeros((2, 2, 4)), s.double(), torch.zeros((2, 3, 8))[..., ::2]):
        refused(lambda: choco.choco_group_norm_forward(h, x, w, w, x.clone(), bad, s), "mean and rstd|are not supported")
        refused(lambda: choco.choco_group_norm_backward(h, x, x.clone(), w, w, s, bad, None, None, None), "mean and rstd|are not supported")
    refused(lambda: choco.choco_group_norm_backward(h, x, x.clone(), w, w, None, s, None, None, None), "are needed")
    refused(lambda: choco.choco_group_norm_forward(h, x, w, w, x[:, :2], s, s), "shape of x")
    refused(lambda: choco.choco_group_norm_init(2, 8, 4, activation="swish"), "activations are")
    with pytest.raises(AssertionError):
        choco.choco_group_norm_forward(h, x, w, None, x.clone(), s, None)


def test_layers_of_an_adamw_list():
    class Rows:                                                  # rows on a GPU, as far as the list looks
        is_cuda, shape, device, dtype = True, (2, 30), "cuda:0", torch.float32

        def get_device(self):
            return 0

        def dim(self):
            return 2

        def stride(self, k):
            return (30, 1)[k]

        def data_ptr(self):
            return 4096

        def element_size(self):
            return 4

    every = choco.adamw_layer_tensors(None, Rows(), [0, 10, 15, 30])
    some = choco.adamw_layer_tensors(None, Rows(), [0, 10, 15, 30], layers=[0, 2])
    assert np.array_equal(some.reshape(2, 2), every.reshape(2, 3)[:, [0, 2]])
    for bad in ([], [3], [-1], [1, 1]):
        refused(lambda: choco.adamw_layer_tensors(None, Rows(), [0, 10, 15, 30], layers=bad), "layers must be")
