"""Images of more pixels than a kernel's threads can count are refused before a launch."""
import pytest
import torch

import paper_1907_09356_b200 as choco
from test_gpu_group_norm import DEV

pytestmark = pytest.mark.gpu


def test_steps_that_cannot_be_counted():
    """One pixel of 2047 channels, repeated 2^31 - 1 times: sixteen rounds of 2^28 steps."""
    c = 2047
    x = torch.zeros((1, 1, 1, c), device=DEV).expand(1, 1, 2 ** 31 - 1, c)
    stats = [torch.zeros((1, 1, 1), device=DEV), torch.ones((1, 1, 1), device=DEV)]
    gn = choco.GroupNorm(1, c, 1, max_images=1)
    db = torch.full((1, c), 3.0, device=DEV)
    with pytest.raises(choco.ChocoError) as err:
        gn.backward(x, x, None, None, *stats, None, None, db)
    assert err.value.code == -7 and torch.equal(db, torch.full_like(db, 3.0))
    few = x[:, :, :1000]
    gn.backward(few, few, None, None, *stats, None, None, db)
    assert not db.any()
    gn.close()
