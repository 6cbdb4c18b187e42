"""GPU: attention of a ragged chunk over the cache (libraspec_chunk_attn[_paged]) against the definition in 64 bits.

Tolerances, from the arithmetic: a probability enters the second product as bf16 (8 significant bits: off by 2^-8 of
itself at most), so O moves by at most 2^-8 A with A = sum p |v| / sum p; the result's own rounding adds 2^-8 |O|. A
score is a binary32 sum of 64 or 128 exact products, below 2^-12 off at the sizes here (times the scale of the queries),
which moves lse by as much and O by 2 A times it.
"""
import math

import numpy as np
import pytest
import torch

from helpers import cuda
from paper_2608_08721_gb300 import binding as lr

pytestmark = pytest.mark.gpu


def attend64(Q, keys, values, n, kv, scale, softcap=0.0, slopes=None, window=0, first_key=None, prefix_len=None):
    """Q [T, Hq, d]; keys[b], values[b] [Hkv, >= N_b, d] float64. Returns O, A [T, Hq, d] and lse [T, Hq]."""
    T, Hq, d = Q.shape
    O, A = torch.zeros((T, Hq, d), dtype=torch.float64), torch.zeros((T, Hq, d), dtype=torch.float64)
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64)
    at = 0
    for b in range(len(n)):
        N = kv[b] + n[b]
        k = torch.arange(N)[None]
        p = torch.arange(kv[b], N)[:, None]
        see = k <= p
        if prefix_len is not None:
            see = see | (k < int(prefix_len[b]))
        if window:
            see = see & (k > p - window)
        rows = slice(at, at + n[b])
        if first_key is not None:
            see = see & (k >= first_key[rows][:, None])
        for h in range(Hq):
            kvh = h // (Hq // keys[b].shape[0])
            # a key that no row sees may hold anything
            K = torch.where(see.any(0)[:, None], keys[b][kvh, :N], 0.0)
            V = torch.where(see.any(0)[:, None], values[b][kvh, :N], 0.0)
            s = Q[rows, h] @ K.T * scale
            if softcap:
                s = softcap * torch.tanh(s / softcap)
            if slopes is not None:
                s = s - float(slopes[h]) * (p - k).abs()
            s = s.masked_fill(~see, -math.inf)
            lse[rows, h] = torch.logsumexp(s, dim=-1) if N else -math.inf
            w = torch.exp(s - torch.nan_to_num(lse[rows, h], neginf=0.0)[:, None])
            O[rows, h], A[rows, h] = w @ V, w @ V.abs()
        at += n[b]
    return O, A, lse


def inputs(n, kv, Hq, Hkv, d, page, seed, q_scale=1.0, extra=0, fill=None):
    """Packed queries and caches; `fill`: what cache rows past a sequence's keys hold."""
    g = torch.Generator().manual_seed(seed)
    B, T = len(n), int(sum(n))
    N = [a + b for a, b in zip(n, kv)]
    Q = (torch.randn((T, Hq, d), generator=g) * q_scale).to(torch.bfloat16)
    keys = [torch.randn((Hkv, x, d), generator=g).to(torch.bfloat16) for x in N]
    values = [torch.randn((Hkv, x, d), generator=g).to(torch.bfloat16) for x in N]
    table = None
    if page:
        per = max(1, (max(N) + extra + page - 1) // page)
        pages = B * per + 3
        table = torch.randperm(pages, generator=g)[:B * per].view(B, per).to(torch.int32)
        K, V = (torch.randn((pages, Hkv, page, d), generator=g).to(torch.bfloat16) for _ in range(2))
    else:
        K, V = (torch.randn((B, Hkv, max(1, max(N) + extra), d), generator=g).to(torch.bfloat16) for _ in range(2))
    if fill is not None:
        K.fill_(fill)
        V.fill_(fill)
    for b in range(B):
        if page:
            for i in range((N[b] + page - 1) // page):
                m = min(page, N[b] - i * page)
                K[table[b, i], :, :m] = keys[b][:, i * page:i * page + m]
                V[table[b, i], :, :m] = values[b][:, i * page:i * page + m]
        else:
            K[b, :, :N[b]], V[b, :, :N[b]] = keys[b], values[b]
    cu = torch.from_numpy(np.concatenate([[0], np.cumsum(n)]).astype(np.int32))
    return Q, K, V, table, cu, torch.tensor(kv, dtype=torch.int32), [k.double() for k in keys], [v.double() for v in values]


def run(Q, K, V, table, cu, kvl, ws=None, **opts):
    T, Hq, d = Q.shape
    ws = ws or lr.ChunkWorkspace(T, len(kvl), Hq, K.shape[1], d)
    dev = {k: v.to(cuda()) if isinstance(v, torch.Tensor) else v for k, v in opts.items()}
    O = torch.full((T, Hq, d), 7.0, dtype=torch.bfloat16, device=cuda())
    lse = torch.full((T, Hq), 7.0, device=cuda())
    args = [K.to(cuda()), V.to(cuda())] + ([table.to(cuda())] if table is not None else [])
    fn = lr.libraspec_chunk_attn if table is None else lr.libraspec_chunk_attn_paged
    fn(Q.to(cuda()), *args, cu.to(cuda()), kvl.to(cuda()), ws, O=O, lse=lse, **dev)
    status = lr.libraspec_get_status(ws)
    return O, lse, status


def assert_close(O, lse, want, A, want_lse, q_scale=1.0):
    delta = 2.0 ** -12 * q_scale
    O, lse = O.double().cpu(), lse.double().cpu()
    bound = 2.0 ** -8 * 1.01 * (A + want.abs()) + 2 * delta * A
    assert bool(torch.isfinite(O).all())
    over = (O - want).abs() - bound
    assert bool((over <= 0).all()), "O over its bound by %.3e at %s" % (over.max(), np.unravel_index(int(over.argmax()), over.shape))
    empty = torch.isinf(want_lse)
    assert torch.equal(empty, torch.isinf(lse)) and bool((O[empty] == 0).all())
    assert bool(((lse - want_lse)[~empty].abs() <= delta + 1e-5 * want_lse[~empty].abs()).all())


def check(n, kv, Hq, Hkv, d, page, seed=0, q_scale=1.0, extra=5, fill=None, **opts):
    Q, K, V, table, cu, kvl, keys, values = inputs(n, kv, Hq, Hkv, d, page, seed, q_scale, extra, fill)
    O, lse, status = run(Q, K, V, table, cu, kvl, **opts)
    assert status == 0
    want, A, want_lse = attend64(Q.double(), keys, values, n, kv, d ** -0.5, **opts)
    assert_close(O, lse, want, A, want_lse, q_scale)


# lengths: one token, the edges of a 128-key tile and of a row tile, none at all, blocks of two row tiles
LENGTHS = [([1], [0]), ([1], [127]), ([1], [128]), ([1, 1, 1], [511, 0, 63]), ([5], [2000]), ([129], [0]),
           ([0, 3, 0, 70], [4, 126, 9, 60]), ([64, 65, 1], [1, 190, 255]), ([300, 2], [100, 700])]


@pytest.mark.parametrize("n,kv", LENGTHS)
@pytest.mark.parametrize("Hq,Hkv,d,page", [(8, 2, 64, 0), (8, 1, 128, 64), (7, 1, 128, 16), (2, 2, 64, 96), (4, 4, 128, 0)])
def test_lengths_heads_and_pages(n, kv, Hq, Hkv, d, page):
    check(n, kv, Hq, Hkv, d, page, seed=len(n) + Hq)


@pytest.mark.parametrize("Hq,Hkv", [(33, 1), (64, 1), (100, 1), (128, 1), (28, 4)])
def test_query_heads_per_kv_head(Hq, Hkv):
    check([3, 1], [100, 300], Hq, Hkv, 64, 32, seed=Hq)


@pytest.mark.parametrize("opts", [dict(window=1), dict(window=5), dict(window=128), dict(window=100000),
                                  dict(softcap=2.0), dict(softcap=30.0, window=77), dict(bias=True),
                                  dict(bias=True, softcap=10.0), dict(prefix=True), dict(prefix=True, window=40),
                                  dict(docs=True), dict(docs=True, prefix=True, bias=True, softcap=5.0, window=200)])
@pytest.mark.parametrize("page,d", [(0, 64), (32, 128)])
def test_masks_caps_and_biases(opts, page, d):
    n, kv = [140, 1, 37], [200, 333, 0]
    o = {k: v for k, v in opts.items() if k in ("window", "softcap")}
    if opts.get("bias"):
        o["slopes"] = torch.tensor([2.0 ** -i for i in range(1, 9)])
    if opts.get("prefix"):
        o["prefix_len"] = torch.tensor([250, 1000, -3], dtype=torch.int32)
    if opts.get("docs"):
        first = torch.zeros(sum(n), dtype=torch.int32)
        first[60:140] = 260
        first[141:] = torch.arange(37, dtype=torch.int32) // 10 * 10
        o["first_key"] = first
    check(n, kv, 8, 2, d, page, seed=11, **o)


def test_rows_that_see_nothing():
    """Documents that begin after the row: alone in their block, beside others, and whole blocks of them."""
    n, kv = [200, 1, 3], [10, 130, 0]
    first = torch.zeros(204, dtype=torch.int32)
    first[3], first[70:140], first[200], first[201:] = 14, 100000, 131, 2**31 - 1
    check(n, kv, 8, 2, 64, 0, first_key=first)
    check(n, kv, 8, 1, 128, 16, first_key=first, slopes=torch.full((8,), 0.5), softcap=20.0)
    # a later document first: the order of the starts does not matter
    first[:200] = torch.randint(0, 210, (200,), generator=torch.Generator().manual_seed(6), dtype=torch.int32)
    check(n, kv, 8, 2, 64, 16, first_key=first)


@pytest.mark.parametrize("fill", [float("nan"), float("inf"), -3.0e38])
@pytest.mark.parametrize("page", [0, 16, 128])
@pytest.mark.parametrize("opts", [dict(), dict(softcap=3.0), dict(slopes=torch.full((8,), 0.3))])
def test_unwritten_cache_rows_take_no_part(fill, page, opts):
    check([1, 70, 3], [40, 130, 255], 8, 2, 128, page, fill=fill, extra=200, **opts)


def test_window_and_documents_leave_old_pages_unread():
    """Pages below every row's first key are gone: their entries point nowhere, and what a partly seen page holds below
    it is not a number."""
    n, kv, page = [33, 1], [500, 300], 16
    Q, K, V, table, cu, kvl, keys, values = inputs(n, kv, 4, 1, 64, page, 3)
    opts = dict(window=50, first_key=torch.cat([torch.full((33,), 470), torch.tensor([0])]).to(torch.int32))
    want = attend64(Q.double(), keys, values, n, kv, 0.125, **opts)
    for b, lowest in ((0, 470), (1, 300 - 50 + 1)):
        for x in (K, V):
            x[table[b, lowest // page].long(), :, :lowest % page] = float("nan")
        table[b, :lowest // page] = -1
        table[b, (kv[b] + n[b] + page - 1) // page:] = 10**6
    O, lse, status = run(Q, K, V, table, cu, kvl, **opts)
    assert status == 0
    assert_close(O, lse, *want)


@pytest.mark.parametrize("q_scale", [8.0, 40.0])
def test_large_scores_raise_the_reference(q_scale):
    """Peaked rows: the running maximum rises by far more than 2^8 between tiles."""
    check([40, 1], [900, 1500], 8, 2, 64, 0, seed=21, q_scale=q_scale)
    check([150], [300], 4, 2, 128, 64, seed=22, q_scale=q_scale)


@pytest.mark.parametrize("softcap,q_scale", [(0.01, 1.0), (1.0, 30.0), (50.0, 8.0), (1000.0, 40.0)])
def test_caps_far_below_and_above_the_scores(softcap, q_scale):
    check([70, 1], [200, 600], 8, 2, 64, 0, seed=24, q_scale=q_scale, softcap=softcap)


@pytest.mark.parametrize("n,kv", [([1], [40000]), ([2, 1], [9000, 20000]), ([600], [3000])])
def test_blocks_cut_over_many_ctas(n, kv):
    check(n, kv, 8, 2, 64, 64, seed=31)


def test_results_do_not_change_from_run_to_run_nor_with_what_the_workspace_served():
    n, kv = [1, 400, 9], [3000, 1000, 5000]
    a = inputs(n, kv, 8, 2, 128, 64, 5)[:6]
    other = inputs([3, 3], [50, 8000], 4, 2, 64, 0, 6)[:6]
    ws = lr.ChunkWorkspace(512, 8, 8, 1, 128)
    O, lse, status = run(*a, ws=ws)
    assert status == 0
    for _ in range(4):
        assert run(*other, ws=ws)[2] == 0
        O2, lse2, _ = run(*a, ws=ws)
        assert torch.equal(O, O2) and torch.equal(lse, lse2)


def test_dense_and_paged_agree_exactly():
    n, kv, page = [70, 1], [200, 999], 32
    Q, K, V, table, cu, kvl, keys, values = inputs(n, kv, 8, 2, 64, page, 8)
    Kd, Vd = (x[table.long()].permute(0, 2, 1, 3, 4).reshape(2, 2, -1, 64).contiguous() for x in (K, V))
    O, lse, _ = run(Q, K, V, table, cu, kvl)
    Od, lsed, _ = run(Q, Kd, Vd, None, cu, kvl)
    assert torch.equal(O, Od) and torch.equal(lse, lsed)


def test_chunks_equal_the_whole_prompt():
    """A prompt in one call, in chunks, and token by token: the same rows within twice the tolerance."""
    N, Hq, Hkv, d = 150, 4, 2, 64
    Q, K, V, _, _, _, keys, values = inputs([N], [0], Hq, Hkv, d, 0, 12)
    want, A, want_lse = attend64(Q.double(), keys, values, [N], [0], d ** -0.5)
    for step in (N, 64, 7, 1):
        for lo in range(0, N, step):
            m = min(step, N - lo)
            O, lse, status = run(Q[lo:lo + m], K, V, None, torch.tensor([0, m], dtype=torch.int32),
                                 torch.tensor([lo], dtype=torch.int32))
            assert status == 0
            assert_close(O, lse, want[lo:lo + m], A[lo:lo + m], want_lse[lo:lo + m])


@pytest.mark.parametrize("softcap", [0.0, 20.0])
def test_non_finite_inputs_stay_in_their_rows(softcap):
    """A NaN query makes its own rows NaN and no others."""
    n, kv = [5, 130], [700, 0]
    Q, K, V, table, cu, kvl, keys, values = inputs(n, kv, 8, 2, 64, 0, 13)
    want, A, want_lse = attend64(Q.double(), keys, values, n, kv, 0.125, softcap=softcap)
    Q[2, 3, 5], Q[40, 0] = float("nan"), float("nan")
    O, lse, status = run(Q, K, V, table, cu, kvl, softcap=softcap)
    bad = torch.zeros((135, 8), dtype=torch.bool)
    bad[2, 3] = bad[40, 0] = True
    assert bool(torch.isnan(O.cpu()[bad]).all()) and bool(torch.isnan(lse.cpu()[bad]).all())
    O, lse = (torch.where(bad.view(135, 8, *[1] * (x.dim() - 2)), y, x.double().cpu()) for x, y in
              ((O, want), (lse, want_lse)))
    assert_close(O, lse, want, A, want_lse)


def test_offsets_beyond_32_bits():
    """Pages past 2^31 elements of the pool."""
    Hkv, page, d, n, kv = 8, 256, 128, [2], [600]
    per = 3
    pages = 2**31 // (Hkv * page * d) + per
    Q, K, V, table, cu, kvl, keys, values = inputs(n, kv, 8, Hkv, d, page, 14)
    Kb, Vb = (torch.zeros((pages, Hkv, page, d), dtype=torch.bfloat16, device=cuda()) for _ in range(2))
    for i in range(per):
        Kb[pages - 1 - i], Vb[pages - 1 - i] = K[table[0, i].long()].to(cuda()), V[table[0, i].long()].to(cuda())
    far = torch.arange(pages - 1, pages - 1 - per, -1, dtype=torch.int32)[None]
    O, lse, status = run(Q, Kb, Vb, far.contiguous(), cu, kvl)
    assert status == 0
    assert_close(O, lse, *attend64(Q.double(), keys, values, n, kv, d ** -0.5))


def test_violations_set_status_and_spare_the_other_sequences():
    n, kv = [2, 3, 4], [10, 20, 30]
    Q, K, V, table, cu, kvl, keys, values = inputs(n, kv, 4, 2, 64, 16, 15, extra=0)
    want, A, want_lse = attend64(Q.double(), keys, values, n, kv, 0.125)
    bad = kvl.clone()
    bad[1] = 46  # 49 keys, the table holds 48
    O, lse, status = run(Q, K, V, table, cu, bad)
    assert status == lr.ST_KV_OVERFLOW
    for rows in (slice(0, 2), slice(5, 9)):
        assert_close(O[rows], lse[rows], want[rows], A[rows], want_lse[rows])
    assert bool((O[2:5] == 7).all()) and bool((lse[2:5] == 7).all())
    bad[1] = -1
    assert run(Q, K, V, table, cu, bad)[2] == lr.ST_KV_OVERFLOW
    O, lse, status = run(Q, K, V, table, torch.tensor([0, 2, 1, 1], dtype=torch.int32), kvl)
    assert status == lr.ST_BAD_LENGTH
    assert_close(O[:2], lse[:2], want[:2], A[:2], want_lse[:2])
    assert run(Q, K, V, table, torch.tensor([0, 2, 5, 10], dtype=torch.int32), kvl)[2] == lr.ST_BAD_LENGTH
    table[2, 1] = -1
    O, lse, status = run(Q, K, V, table, cu, kvl)
    assert status == lr.ST_BAD_PAGE
    assert_close(O[:5], lse[:5], want[:5], A[:5], want_lse[:5])


@pytest.mark.parametrize("d,page", [(128, 128), (64, 16)])
def test_decode_batch_of_uneven_lengths(d, page):
    """Every CTA works through pieces of several sequences, each with a last tile of its own length."""
    r = np.random.default_rng(7)
    kv = np.exp(r.uniform(math.log(100), math.log(4000), 48)).astype(int).tolist()
    check([1] * 48, kv, 8, 4, d, page, seed=43, fill=float("nan"))


@pytest.mark.parametrize("d", [64, 128])
def test_short_items_back_to_back(d):
    """Items of one to three key tiles, single rows and pairs in turn: 200 calls on end, each with the first's result."""
    r = np.random.default_rng(11)
    n = np.where(r.random(400) < 0.8, 1, r.integers(2, 60, 400)).tolist()
    kv = r.integers(0, 300, 400).tolist()
    Q, K, V, table, cu, kvl, keys, values = inputs(n, kv, 16, 4, d, 32, 47)
    dev = [x.to(cuda()) for x in (Q, K, V, table, cu, kvl)]
    ws = lr.ChunkWorkspace(sum(n), 400, 16, 4, d)
    first, _ = lr.libraspec_chunk_attn_paged(*dev, ws)
    for _ in range(200):
        O, lse = lr.libraspec_chunk_attn_paged(*dev, ws, want_lse=True)
    assert lr.libraspec_get_status(ws) == 0
    assert torch.equal(O, first)
    assert_close(O, lse, *attend64(Q.double(), keys, values, n, kv, d ** -0.5))


def test_many_sequences():
    """More sequences than the plan's threads; some without new tokens."""
    r = np.random.default_rng(3)
    B = 1300
    n, kv = r.integers(0, 3, B).tolist(), r.integers(0, 40, B).tolist()
    check(n, kv, 2, 1, 64, 16, seed=41)


def test_stream_and_graph():
    """On a stream of its own, eagerly and as a captured graph replayed on new contents."""
    n, kv = [3, 90], [200, 40]
    Q, K, V, table, cu, kvl, keys, values = inputs(n, kv, 8, 2, 64, 64, 17)
    dev = [x.to(cuda()) for x in (Q, K, V, table, cu, kvl)]
    ws = lr.ChunkWorkspace(93, 2, 8, 2, 64)
    O, lse = torch.empty_like(dev[0]), torch.empty((93, 8), device=cuda())
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    call = lambda: lr.libraspec_chunk_attn_paged(*dev, ws, O=O, lse=lse, window=64, stream=s)  # noqa: E731
    call()
    s.synchronize()
    eager, eager_lse = O.clone(), lse.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call()
    O.zero_()
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(O, eager) and torch.equal(lse, eager_lse)
    dev[5].copy_(torch.tensor([77, 5], dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    assert lr.libraspec_get_status(ws) == 0
    want = attend64(Q.double(), keys, values, n, [77, 5], 0.125, window=64)
    assert_close(O, lse, *want)


def test_outputs_belong_to_the_stream_of_the_call():
    """A call on another stream makes its outputs there: memory that the current stream has given back, and may still be
    working on, is not written by it."""
    s, d = torch.cuda.Stream(), 64
    X = torch.randn((300, 12, d), device=cuda(), dtype=torch.bfloat16)
    pos = torch.arange(300, dtype=torch.int32, device=cuda())
    cu, kvl = torch.tensor([0, 300], dtype=torch.int32, device=cuda()), torch.zeros(1, dtype=torch.int32, device=cuda())
    Kd, Vd = (torch.zeros((1, 2, 300, d), dtype=torch.bfloat16, device=cuda()) for _ in range(2))
    fr, ws = lr.RopeFreqs(d), lr.ChunkWorkspace(300, 1, 8, 2, d)
    q, k, v = X[:, :8], X[:, 8:10], X[:, 10:]
    Q = q.contiguous()
    torch.cuda.synchronize()
    calls = [lambda st: [lr.libraspec_rope(Q, pos, fr, stream=st)],
             lambda st: [lr.libraspec_rope_append(q, k, v, Kd, Vd, cu, kvl, fr, ws, stream=st)],
             lambda st: list(lr.libraspec_chunk_attn(Q, Kd, Vd, cu, kvl, ws, want_lse=True, stream=st))]
    for call in calls:
        here = call(None)
        torch.cuda.synchronize()
        want = [(x.data_ptr(), x.clone()) for x in here]
        del here  # their memory is the first that the current stream hands out again
        there = call(s)
        torch.cuda.synchronize()
        for x in there:
            assert all(x.data_ptr() != p for p, _ in want)
        assert all(torch.equal(x, w) for x, (_, w) in zip(there, want))
        del there


@pytest.mark.parametrize("softcap", [1e-39, 1e-30, 100.0, 300.0, 1e3, 1e5, 1e7, 1e20, 3e38])
@pytest.mark.parametrize("q_scale,bias", [(1.0, False), (8.0, True)])
def test_caps_of_any_size(softcap, q_scale, bias):
    """The cap's error is relative to the capped score, not to the cap: a cap far above the scores leaves them as they
    are; scores of zero stay zero under the smallest cap."""
    n, kv, d = [70, 1], [200, 600], 64
    Q, K, V, table, cu, kvl, keys, values = inputs(n, kv, 8, 2, d, 0, 25, q_scale=q_scale)
    Q[3], Q[70, 2] = 0.0, 0.0
    o = dict(slopes=torch.tensor([2.0 ** -i for i in range(1, 9)])) if bias else {}
    softcap = float(np.float32(softcap))
    O, lse, status = run(Q, K, V, table, cu, kvl, softcap=softcap, **o)
    assert status == 0
    assert_close(O, lse, *attend64(Q.double(), keys, values, n, kv, d ** -0.5, softcap=softcap, **o), q_scale=q_scale)


@pytest.mark.parametrize("n,kv", [([1, 33], [199, 100]), ([70, 1], [58, 127]), ([300, 5], [0, 128])])
@pytest.mark.parametrize("page", [0, 16, 48])
def test_blocks_that_see_nothing_read_nothing(n, kv, page):
    """A sequence of which no row sees a key: its pages need not exist, and nothing is reported."""
    Q, K, V, table, cu, kvl, keys, values = inputs(n, kv, 8, 2, 64, page, 19)
    first = torch.cat([torch.full((n[0],), 2**31 - 1), torch.zeros(n[1], dtype=torch.int64)]).to(torch.int32)
    if page:
        K[table[0].long()], V[table[0].long()] = float("nan"), float("nan")
        table[0] = 10**6
    else:
        K[0], V[0] = float("nan"), float("nan")
    O, lse, status = run(Q, K, V, table, cu, kvl, first_key=first)
    assert status == 0
    assert_close(O, lse, *attend64(Q.double(), keys, values, n, kv, 0.125, first_key=first))


@pytest.mark.parametrize("d,page", [(64, 0), (128, 16), (64, 48)])
@pytest.mark.parametrize("opts", [dict(), dict(slopes=torch.full((8,), 0.5), softcap=20.0), dict(prefix=True)])
def test_keys_of_rows_that_see_nothing_need_not_exist(d, page, opts):
    """Padding within a sequence: rows that see no key, whose own keys no other row sees. Neither what their cache rows
    hold (not a number), nor the pages that hold nothing else, take part: whole blocks of them, at the end of a block,
    and between rows of the same block that see keys on both sides."""
    n, kv, Hq, Hkv = [200, 1, 3], [10, 130, 0], 8, 2
    Q, K, V, table, cu, kvl, keys, values = inputs(n, kv, Hq, Hkv, d, page, 77, extra=40)
    first = torch.zeros(204, dtype=torch.int32)
    first[40:120] = 100000        # positions 50 .. 129: in two or three blocks
    first[120:190] = 130          # the rows behind them start over
    first[190:200] = 2**31 - 1    # the sequence's end
    first[200] = 131              # a decode step that sees nothing
    first[201:] = 3
    o = {k: v for k, v in opts.items() if k != "prefix"}
    if opts.get("prefix"):        # what is seen below 171 is seen as far as there; and a gap behind it
        o["prefix_len"] = torch.tensor([171, 0, 0], dtype=torch.int32)
        first[:30], first[30:40] = 100000, 150
        first[165:176], first[176:190] = 100000, 186
    want = attend64(Q.double(), keys, values, n, kv, d ** -0.5, first_key=first, **o)
    at = 0
    for b in range(3):
        N = n[b] + kv[b]
        k, p = torch.arange(N)[None], torch.arange(kv[b], N)[:, None]
        hi = torch.maximum(p + 1, o["prefix_len"][b] if "prefix_len" in o else torch.tensor(0))
        seen = ((k >= first[at:at + n[b]][:, None]) & (k < hi)).any(0)
        assert not bool(seen.all())
        at += n[b]
        for s in range(N):
            if not seen[s]:
                (K[table[b, s // page], :, s % page] if page else K[b, :, s])[:] = float("nan")
                (V[table[b, s // page], :, s % page] if page else V[b, :, s])[:] = float("nan")
        if page:
            for i in range(table.shape[1]):
                if not bool(seen[i * page:(i + 1) * page].any()):
                    table[b, i] = 10**6
    O, lse, status = run(Q, K, V, table, cu, kvl, first_key=first, **o)
    assert status == 0
    assert_close(O, lse, *want)
