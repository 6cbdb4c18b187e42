"""GPU: a query that is NaN gives NaN in its own row, whatever CTAs its keys are cut over (16-bit and 8-bit caches)."""
import math

import pytest
import torch

from test_gpu_chunk_q8 import Inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("block", [0, 16])
@pytest.mark.parametrize("n,kv", [([40], [1000]), ([300], [1500]), ([1], [4000]), ([130, 5], [900, 3000])])
def test_a_row_of_nan_is_nan_however_its_keys_are_cut(block, n, kv):
    """Its keys lie in tiles that it sees in part, and each of them may be another CTA's."""
    x = Inputs(n, kv, 4, 1, 128, 64, block, seed=3)
    rows = sorted({0, sum(n) // 2, sum(n) - 1})
    for i, row in enumerate(rows):
        x.Q[row, i % 4, 3] = math.nan
    O, lse, status = x.run(window=100, sinks=0)
    marked = torch.zeros(lse.shape, dtype=torch.bool)
    for i, row in enumerate(rows):
        marked[row, i % 4] = True
    O, lse = O.cpu(), lse.cpu()
    assert status == 0 and bool(torch.isnan(O[marked]).all()) and bool(torch.isnan(lse[marked]).all())
    assert bool(torch.isfinite(O[~marked]).all()) and bool(torch.isfinite(lse[~marked]).all())
