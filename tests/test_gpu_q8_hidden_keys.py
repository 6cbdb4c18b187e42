"""GPU: attention over a cache in 8 bits where blocks of keys are hidden, from all rows or from some: neither their codes nor
their exponents reach a row that does not see them.

Tolerances: those of test_gpu_chunk_q8.py, row by row: the last term takes the largest exponent of V that the row sees, since
a probability's rounding counts against the largest term of its own row.
"""
import math

import pytest
import torch

from test_gpu_chunk_q8 import Inputs, attend64

pytestmark = pytest.mark.gpu


def hide(x, a, b, page):
    """Keys [a, b) of sequence 0 (whole blocks): NaN codes, the largest exponent bytes; pages of nothing else do not exist."""
    for t in x.dev[:2]:
        raw = t.view(torch.uint8)
        for k in range(a, b):
            if page:
                raw[x.table[0, k // page], :, k % page] = 0x7f
            else:
                raw[0, :, k] = 0x7f
    for t in x.dev[2:4]:
        for k in range(a, b, x.block):
            if page:
                t[x.table[0, k // page], :, k % page // x.block] = 255
            else:
                t[0, :, k // x.block] = 255
    if page:
        for i in range(-(-a // page), b // page):
            x.dev[-1][0, i] = (-5, 1 << 20)[i % 2]


# sequences beside it without new tokens: none (the many-row kernel), or so many that the few-row kernel takes the call
@pytest.mark.parametrize("idle", [0, 70])
@pytest.mark.parametrize("page,d,block", [(0, 128, 16), (0, 64, 64), (16, 64, 16), (32, 128, 32), (64, 128, 64), (64, 64, 16),
                                          (192, 64, 32)])
@pytest.mark.parametrize("opts", [dict(), dict(softcap=20.0), dict(bias=True)])
def test_padding_blocks_need_not_be_initialised(idle, page, d, block, opts):
    """Whole blocks of padding among the new tokens, that no row sees, inside a tile and up to its edges."""
    n, kv, Hq = [312] + [0] * idle, [200] + [3] * idle, 3
    x = Inputs(n, kv, Hq, 1, d, page, block, seed=block + d)
    at = torch.arange(200, 512)
    first = torch.zeros(312, dtype=torch.int32)
    for a, b in ((256, 256 + block), (320, 320 + block), (448, 512)):
        first[at >= b] = b
        first[(at >= a) & (at < b)] = 1 << 20  # padding: sees nothing, and nothing behind it sees it
        hide(x, a, b, page)
    opts = dict(opts, first_key=first)
    if opts.pop("bias", False):
        opts["slopes"] = torch.tensor([0.5, 0.1, 0.01])
    x.check(**opts)


@pytest.mark.parametrize("idle", [0, 70])
@pytest.mark.parametrize("page,d,block", [(0, 64, 16), (64, 128, 16), (32, 128, 32), (64, 64, 64)])
@pytest.mark.parametrize("louder", [20, 40])
@pytest.mark.parametrize("mask", ["causal", "window", "documents", "sinks"])
def test_values_of_hidden_keys_cost_no_precision(idle, page, d, block, louder, mask):
    """A block of values 2^20 or 2^40 above the others, in the tile of rows that do not see it: later tokens, ones behind the
    window, ones of another document."""
    T, kv, Hq, Hkv = 240, 90, 4, 1
    a = 192
    b = a + block
    x = Inputs([T] + [0] * idle, [kv] + [3] * idle, Hq, Hkv, d, page, block, seed=louder + d, exps=(119, 121))
    x.values[0][:, a:b] *= 2.0 ** louder
    for k in range(a, b, block):
        if page:
            x.dev[3][x.table[0, k // page], :, k % page // block] += louder
        else:
            x.dev[3][0, :, k // block] += louder
    pos = torch.arange(kv, kv + T)
    sees, opts = pos >= a, {}
    if mask in ("window", "sinks"):
        opts = dict(window=24, sinks=6 if mask == "sinks" else 0)
        sees &= pos - 24 < b - 1
    if mask == "documents":
        first = torch.where(pos >= b, b, torch.where(pos >= a, a, 0)).to(torch.int32)
        opts = dict(first_key=first)
        sees &= first < b
    O, lse, status = x.run(**opts)
    assert status == 0
    want, A, want_lse, top, mag = attend64(x.Q.double(), x.keys, x.values, x.n, x.kv, d ** -0.5, **opts)
    delta = 2.0 ** -12 + 2.0 ** -17 * mag + 2.0 ** -20 * top
    largest = torch.exp2(torch.where(sees, 120.0 + louder, 120.0) - 127)[:, None, None]
    bound = (2.0 ** -11 * 1.01 + 2 * delta) * A + 2.0 ** -8 * 1.01 * want.abs() + (kv + T) * 2.0 ** -23 * largest
    O, lse = O.double().cpu(), lse.double().cpu()
    over = (O - want).abs() - bound
    assert bool(torch.isfinite(O).all()) and bool((over <= 0).all()), "rows %s" % (over > 0).any(-1).any(-1).nonzero().view(-1).tolist()
    assert bool(((lse - want_lse).abs() <= delta + 1e-5 * want_lse.abs()).all())


def test_hidden_exponents_change_nothing():
    """A row's result is the same to the bit whatever the exponents of blocks that it does not see."""
    x = Inputs([200], [100], 4, 1, 128, 64, 16, seed=3, exps=(119, 121))
    want = x.run()
    last = x.dev[3][x.table[0, 4]]  # keys 256 to 319: rows below 256 do not see them
    for byte in (0, 67, 119, 150, 255):
        last.fill_(byte)
        x.dev[3][x.table[0, 4]] = last
        O, lse, status = x.run()
        assert status == 0 and torch.equal(O[:156], want[0][:156]) and torch.equal(lse[:156], want[1][:156])
        assert math.isfinite(float(O.float().abs().max()))
