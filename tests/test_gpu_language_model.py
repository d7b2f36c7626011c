"""The example that runs lookup, its gradient, clipping, AdamW and gossip together learns its chain."""
import math
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits,q", [(32, "topk"), (8, "sign"), (8, "qsgd")])
def test_the_workers_learn_and_stay_together(bits, q):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import language_model
    losses, distances = language_model.train(workers=4, steps=150, bits=bits, q=q, vocab=128, dim=32)
    # an untrained model knows nothing: log(128) within the noise of its small weights; the chain has
    # four successors a token, so a model that has learned them is near log(4) or below; half-way
    # between the two is well on its way
    assert abs(losses[0] - math.log(128)) < 0.5
    assert losses[-10:].mean() < 0.5 * (math.log(128) + math.log(4))
    assert all(math.isfinite(v) for v in distances)
