"""Matrices whose rows span more than an address can are refused on the host (no GPU needed): their ranges could not be compared."""
import pytest

import paper_1907_09356_b200 as choco
from paper_1907_09356_b200 import build as choco_build
from test_abi_muon_norm import _muon


@pytest.fixture(scope="module")
def lib():
    choco_build.build()
    return choco.load()


@pytest.mark.parametrize("which", ["x_ld", "g_ld", "copy_ld"])
def test_spans(lib, which):
    tall = dict(rows=1 << 26, cols=1)
    # 2^26 rows that are 2^38 elements apart: 2^66 bytes; x then ends, modulo 2^64, before it begins
    assert _muon(lib, matrix={**tall, which: 1 << 38}, more=dict(x=1 << 40, g=1 << 41)) == -7
    assert _muon(lib, matrix={**tall, which: (1 << 14) + 1}, more=dict(x=1 << 50, g=1 << 51)) == -7
    assert _muon(lib, matrix=dict(rows=1, cols=20, **{which: 1 << 38})) in (0, -3, -4)
    assert _muon(lib, matrix=dict(rows=1 << 16, cols=1, x=1 << 45, g=1 << 46, **{which: 1 << 24}), more=dict(x=1 << 20, g=1 << 21)) in (0, -3, -4)
