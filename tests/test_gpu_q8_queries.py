"""GPU: queries that are not finite, through both kernels of the attention over a cache in 8 bits: what their formula gives, in
their own row alone.

An infinite element makes a row's scores infinite, of both signs: no softmax of them exists (NaN); under a cap they are the cap
or its negative. Tolerances: those of test_gpu_chunk_q8.py.
"""
import math

import pytest
import torch

from test_gpu_chunk_q8 import Inputs, attend64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,kv", [([40, 1], [200, 500]), ([300], [10]), ([1, 1], [200, 500]), ([2, 1], [3000, 0])])
@pytest.mark.parametrize("page,d,block", [(0, 64, 32), (32, 128, 16)])
@pytest.mark.parametrize("opts", [dict(), dict(bias=True), dict(softcap=10.0), dict(softcap=1000.0), dict(window=100, sinks=3)])
def test_rows_of_queries_that_are_not_finite(n, kv, page, d, block, opts):
    Hq, Hkv = 4, 2
    opts = dict(opts)
    if opts.pop("bias", False):
        opts["slopes"] = torch.tensor([0.5, 0.1, 0.01, 0.001])
    x = Inputs(n, kv, Hq, Hkv, d, page, block, seed=d + len(n), q_scale=2.0)
    finite = x.Q.clone()
    infinite = [(0, 1, 5, math.inf), (1 if sum(n) > 1 else 0, 2, 0, -math.inf)]
    for row, h, i, v in infinite:
        x.Q[row, h, i] = v
    x.Q[0, 3, 7] = math.nan
    marked = torch.zeros(x.Q.shape[:2], dtype=torch.bool)
    for row, h, _, _ in infinite:
        marked[row, h] = True
    marked[0, 3] = True

    O, lse, status = x.run(**opts)
    assert status == 0
    O, lse = O.double().cpu(), lse.double().cpu()
    want, A, want_lse, top, mag = attend64(finite.double(), x.keys, x.values, n, kv, d ** -0.5, **opts)
    delta = 2.0 ** -12 + 2.0 ** -17 * mag + 2.0 ** -20 * top
    extra = max(a + b for a, b in zip(n, kv)) * 2.0 ** -23 * 2.0 ** x.top_exp

    def close(rows, want, A, want_lse):
        bound = (2.0 ** -11 * 1.01 + 2 * delta) * A + 2.0 ** -8 * 1.01 * want.abs() + extra
        assert bool(((O - want).abs() <= bound)[rows].all())
        assert bool(((lse - want_lse).abs() <= delta + 1e-5 * want_lse.abs())[rows].all())

    close(~marked, want, A, want_lse)
    assert bool(torch.isnan(O[0, 3]).all()) and bool(torch.isnan(lse[0, 3]))
    if "softcap" not in opts:
        assert bool(torch.isnan(O[marked]).all()) and bool(torch.isnan(lse[marked]).all())
    else:
        marked[0, 3] = False
        capped = attend64(x.Q.double(), x.keys, x.values, n, kv, d ** -0.5, **opts)
        close(marked, *capped[:3])
