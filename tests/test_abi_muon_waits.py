"""The calls about waits that ran out reject bad handles on the host (no GPU needed)."""
import pytest

import paper_1907_09356_b200 as choco
from paper_1907_09356_b200 import build as choco_build


@pytest.fixture(scope="module")
def lib():
    choco_build.build()
    return choco.load()


def test_null_handles(lib):
    assert lib.choco_debug_muon_set_wait_polls(None, 0) == -1 and lib.choco_muon_status(None, None) == -1
