"""GPU: attention of a chunk where a CTA works through runs of many key tiles (libraspec_chunk_attn[_paged]), against the
definition in 64 bits: biases, caps and masks in the loop over tiles, the reference of the softmax raised within a run,
whole items taken in step, and plans of more blocks than the plan kernel has threads.

The tolerances are those of the other chunk attention tests: 2^-12 times the scale of queries and keys for a score, and
for a bias of size b three roundings of it, 3 x 2^-24 b.
"""
import math

import numpy as np
import pytest
import torch

from helpers import cuda
from paper_2608_08721_gb300 import binding as lr
from test_gpu_chunk_attn import assert_close, attend64, inputs, run

pytestmark = pytest.mark.gpu

KEYS = 128  # of a tile


def items(n, kv, Hq, Hkv, window=0):
    """(key tiles of all blocks and kv heads, blocks)"""
    per = 2 * (128 // (Hq // Hkv))
    tiles = blocks = 0
    for m, k in zip(n, kv):
        for j in range(0, m, per):
            lo = max(0, k + j - window + 1) if window else 0
            hi = k + min(m, j + per)
            tiles += (hi + KEYS - 1) // KEYS - lo // KEYS
            blocks += 1
    return tiles * Hkv, blocks


def sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


def reference(Q, keys, values, n, kv, kv_heads, g, **opts):
    """attend64 on the device, for the query heads of some kv heads."""
    heads = [h * g + i for h in kv_heads for i in range(g)]
    o = {k: (v.to(cuda()) if isinstance(v, torch.Tensor) else v) for k, v in opts.items()}
    if o.get("slopes") is not None:
        o["slopes"] = o["slopes"][heads]
    with torch.device(cuda()):
        out = attend64(Q[:, heads].to(cuda()).double(), [k[kv_heads].to(cuda()) for k in keys],
                       [v[kv_heads].to(cuda()) for v in values], n, kv, Q.shape[2] ** -0.5, **o)
    return heads, [x.cpu() for x in out]


def bias_scale(slopes, keys):
    """What a bias adds to a score's rounding, in units of 2^-12."""
    return 3 * 2.0 ** -24 * float(slopes.abs().max()) * keys * 2.0 ** 12


@pytest.mark.parametrize("d,page", [(64, 16), (128, 64)])
@pytest.mark.parametrize("opts", [dict(bias=0.25), dict(bias=-0.3), dict(cap=5.0, window=1000),
                                  dict(bias=0.01, cap=20.0, docs=True, prefix=True), dict(window=2000, docs=True)])
def test_masks_caps_and_biases_over_runs_of_tiles(opts, d, page):
    """Pages that no row sees, and rows past the keys of a sequence, hold no numbers."""
    n, kv, Hq, Hkv = [4000, 1, 777], [1500, 3000, 0], 8, 4
    tiles, _ = items(n, kv, Hq, Hkv, opts.get("window", 0))
    assert tiles >= 8 * sms()  # (runs of eight tiles on average)
    Q, K, V, table, cu, kvl, keys, values = inputs(n, kv, Hq, Hkv, d, page, 61, extra=300, fill=float("nan"))
    o, scale = dict(softcap=opts.get("cap", 0.0), window=opts.get("window", 0)), 1.0
    if "bias" in opts:
        o["slopes"] = opts["bias"] * torch.exp2(-torch.arange(Hq) / 2.0)
        scale += bias_scale(o["slopes"], 5500)
    if opts.get("docs"):
        first = torch.zeros(sum(n), dtype=torch.int32)
        first[1000:4000] = torch.arange(1000, 4000, dtype=torch.int32) // 700 * 700 + 1500
        first[4001:] = 100
        o["first_key"] = torch.minimum(first, torch.cat([torch.arange(k, k + m) for m, k in zip(n, kv)]).int())
    if opts.get("prefix"):
        o["prefix_len"] = torch.tensor([3000, 2000, 333], dtype=torch.int32)
    O, lse, status = run(Q, K, V, table, cu, kvl, **o)
    assert status == 0
    heads, want = reference(Q, keys, values, n, kv, [1, 3], Hq // Hkv, **o)
    assert_close(O[:, heads], lse[:, heads], *want, q_scale=scale)


@pytest.mark.parametrize("d,page,n,kv", [(64, 0, [3000], [2000]), (128, 32, [2500], [3000]),
                                         (64, 64, [1] * 40, [9000] * 40), (128, 0, [3, 20] * 10, [6000] * 20)])
def test_maxima_that_rise_within_a_run(d, page, n, kv):
    """Keys that grow along the sequence: rows' maxima rise by more than 2^8 from tile to tile, also in the second half
    of runs, so that O and the sums are rescaled many times; both for pairs of row tiles and for single ones."""
    Hq, Hkv, q_scale, k_scale = 4, 2, 3.0, 5.0
    assert items(n, kv, Hq, Hkv)[0] >= 8 * sms()
    Q, K, V, table, cu, kvl, keys, values = inputs(n, kv, Hq, Hkv, d, 0, 67, q_scale=q_scale)
    N = [a + b for a, b in zip(n, kv)]
    keys = [(x * torch.linspace(0.02, 1.0, x.shape[1])[None, :, None] ** 2 * k_scale).to(torch.bfloat16).double()
            for x in keys]
    Q, K, V, table, cu, kvl, _, _ = inputs(n, kv, Hq, Hkv, d, page, 67, q_scale=q_scale)
    for b in range(len(n)):
        at = torch.arange(N[b])
        if page:
            K[table[b, at // page].long(), :, at % page] = keys[b].transpose(0, 1).to(torch.bfloat16)
            V[table[b, at // page].long(), :, at % page] = values[b].transpose(0, 1).to(torch.bfloat16)
        else:
            K[b, :, :N[b]], V[b, :, :N[b]] = keys[b].to(torch.bfloat16), values[b].to(torch.bfloat16)
    # the last row's maximum over the keys so far, tile by tile: it rises by 8 in log 2 four times at least
    s = (Q[-1, 0].double() @ keys[-1][0].T) * d ** -0.5 * math.log2(math.e)
    top = torch.cummax(torch.stack([x.max() for x in s.split(KEYS)]), 0).values
    ref, rises = top[0], 0
    for m in top[1:]:
        if m > ref + 8:
            ref, rises = m, rises + 1
    assert rises >= 4
    O, lse, status = run(Q, K, V, table, cu, kvl)
    assert status == 0
    heads, want = reference(Q, keys, values, n, kv, [0, 1], Hq // Hkv)
    assert_close(O[:, heads], lse[:, heads], *want, q_scale=q_scale * k_scale)


def plan_head(ws):
    """What the plan kernel wrote: tiles, blocks, blocks of two row tiles, whole items of each CTA."""
    head = ws.buf[256:280].cpu().numpy()
    return int(head[:8].view(np.int64)[0]), *(int(x) for x in head[8:20].view(np.int32))


@pytest.mark.parametrize("d,kv", [(128, 16600), (64, 33100)])
@pytest.mark.parametrize("table", [False, True])
def test_blocks_of_a_long_cache_in_step(d, kv, table):
    """Keys that L2 does not hold, with more items than CTAs: whole items first, the rest cut; planned in registers, and
    (with first keys) in the table."""
    n, Hq, Hkv = [640], 64, 8
    Q, K, V, bt, cu, kvl, keys, values = inputs(n, [kv], Hq, Hkv, d, 128, 71)
    opts = dict(first_key=torch.full((640,), 5, dtype=torch.int32)) if table else {}
    ws = lr.ChunkWorkspace(640, 1, Hq, Hkv, d)
    O, lse, status = run(Q, K, V, bt, cu, kvl, ws=ws, **opts)
    assert status == 0
    tiles, blocks = items(n, [kv], Hq, Hkv)
    assert blocks >= 2 and blocks * Hkv >= sms() and (kv + 640 + KEYS - 1) // KEYS * Hkv * KEYS * d * 4 > 64 << 20
    if table:
        assert plan_head(ws) == (tiles // Hkv, blocks, blocks, blocks * Hkv // sms())
    heads, want = reference(Q, keys, values, n, [kv], [0, 7], Hq // Hkv, **opts)
    assert_close(O[:, heads], lse[:, heads], *want)


@pytest.mark.parametrize("first", [False, True])
def test_more_blocks_than_the_plan_has_threads(first):
    r = np.random.default_rng(5)
    B = 1500
    n, kv = [1] * B, r.integers(0, 400, B).tolist()
    n[700], n[1400] = 300, 200
    assert items(n, kv, 2, 1)[1] > 1024
    Q, K, V, table, cu, kvl, keys, values = inputs(n, kv, 2, 1, 64, 16, 73)
    opts = {}
    if first:
        pos = torch.cat([torch.arange(k, k + m) for m, k in zip(n, kv)])
        opts["first_key"] = (pos * torch.rand(len(pos), generator=torch.Generator().manual_seed(2))).to(torch.int32)
    ws = lr.ChunkWorkspace(sum(n), B, 2, 1, 64)
    O, lse, status = run(Q, K, V, table, cu, kvl, ws=ws, **opts)
    assert status == 0 and plan_head(ws)[1] == items(n, kv, 2, 1)[1]
    assert_close(O, lse, *attend64(Q.double(), keys, values, n, kv, 0.125, **opts))
