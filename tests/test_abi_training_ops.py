"""The init calls of the token tables and of AdamW reject bad arguments on the host, before they
touch a device (no GPU needed)."""
import ctypes

import numpy as np
import pytest

import paper_1907_09356_b200 as choco
from paper_1907_09356_b200 import build as choco_build


@pytest.fixture(scope="module")
def lib():
    choco_build.build()
    return choco.load()


def _embedding(lib, **kw):
    a = dict(n=2, scale=1.0, vocab=10, dim=8, table_row=0, table_ld=0, max_tokens=16, padding=-1)
    a.update(kw)
    p = choco.choco_embedding_params(*[a[f] for f, _ in choco.choco_embedding_params._fields_])
    h = ctypes.c_void_p()
    rc = lib.choco_embedding_init(ctypes.byref(h), ctypes.byref(p))
    assert h.value is None or rc == 0
    return rc


@pytest.mark.parametrize("kw,code", [
    (dict(n=0), -1), (dict(vocab=0), -1), (dict(dim=0), -1), (dict(max_tokens=-1), -1), (dict(scale=float("nan")), -1),
    (dict(scale=float("inf")), -1), (dict(table_row=7), -1), (dict(table_ld=79), -1), (dict(table_row=9, table_ld=88), -1),
    (dict(n=65536), -7), (dict(vocab=0x7fffffff), -7), (dict(dim=(1 << 24) + 1), -7), (dict(max_tokens=1 << 30), -7),
    (dict(max_tokens=1 << 31, n=1), -7), (dict(max_tokens=1 << 62, n=4), -7)])
def test_embedding_refusals(lib, kw, code):
    assert _embedding(lib, **kw) == code


def test_embedding_null_pointers(lib):
    assert lib.choco_embedding_init(None, None) == -1
    h = ctypes.c_void_p()
    assert lib.choco_embedding_init(ctypes.byref(h), None) == -1
    assert lib.choco_embedding_destroy(None) == -1


def _adamw(lib, tensor=None, n=1, groups=2, beta1=0.9, beta2=0.999, eps=1e-8, bits=32):
    t = np.zeros(1, dtype=choco.ADAMW_TENSOR)
    t["x"], t["g"], t["numel"], t["lr_scale"] = 4096, 8192, 100, 1.0
    for k, v in (tensor or {}).items():
        t[k] = v
    p = choco.choco_adamw_params(beta1, beta2, eps, bits, groups)
    h = ctypes.c_void_p()
    rc = lib.choco_adamw_init(ctypes.byref(h), n, t.ctypes.data, ctypes.byref(p))
    assert h.value is None or rc == 0
    return rc


@pytest.mark.parametrize("kw,code", [
    (dict(n=0), -1), (dict(groups=0), -1), (dict(beta1=1.0), -1), (dict(beta1=-0.1), -1), (dict(beta2=1.0), -1),
    (dict(beta2=float("nan")), -1), (dict(eps=0.0), -1), (dict(eps=1e-60), -1), (dict(eps=float("inf")), -1), (dict(bits=16), -6),
    (dict(tensor=dict(group=2)), -1), (dict(tensor=dict(group=-1)), -1), (dict(tensor=dict(numel=-1)), -1),
    (dict(tensor=dict(g=0)), -1), (dict(tensor=dict(x_dtype=3)), -1), (dict(tensor=dict(g_dtype=-1)), -1),
    (dict(tensor=dict(copy_dtype=9)), -1), (dict(tensor=dict(weight_decay=-1.0)), -1),
    (dict(tensor=dict(weight_decay=float("nan"))), -1), (dict(tensor=dict(lr_scale=float("inf"))), -1),
    (dict(tensor=dict(x=4098)), -5), (dict(tensor=dict(g=8193, g_dtype=1)), -5), (dict(tensor=dict(copy=4097, copy_dtype=2)), -5),
    (dict(tensor=dict(numel=(1 << 38) + 1)), -1)])
def test_adamw_refusals(lib, kw, code):
    assert _adamw(lib, **kw) == code


def test_adamw_null_pointers(lib):
    assert lib.choco_adamw_init(None, 1, None, None) == -1
    h = ctypes.c_void_p()
    assert lib.choco_adamw_init(ctypes.byref(h), 1, None, None) == -1
    e = ctypes.c_int64()
    assert lib.choco_adamw_destroy(None) == -1
    assert lib.choco_adamw_state_size(None, ctypes.byref(e), None) == -1
    assert lib.choco_adamw_step(None, None, None, None, None, 1e-3, None, None) == -1
    assert lib.choco_adamw_grad_norm(None, 1.0, 1.0, None, None, None) == -1
    assert lib.choco_adamw_read_state(None, None, None, None, None, None, None, 0, None) == -1


def test_record_matches_the_struct():
    """Field order and sizes of choco_adamw_tensor: 4 pointers or 64-bit values, 4 ints, 2 doubles."""
    d = np.dtype(choco.ADAMW_TENSOR)
    assert d.itemsize == 64
    assert [d.fields[f][1] for f in ("x", "g", "copy", "numel", "x_dtype", "g_dtype", "copy_dtype", "group", "weight_decay",
                                     "lr_scale")] == [0, 8, 16, 24, 32, 36, 40, 44, 48, 56]
