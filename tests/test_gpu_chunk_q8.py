"""GPU: attention of a chunk over a cache in 8 bits (libraspec_chunk_attn_q8[_paged]) and in a window with sinks
(libraspec_sink_attn[_paged]), against the definition in 64 bits.

Tolerances, from the arithmetic. Over 8 bits: a query's elements are off by up to 2^-17 of the largest of their row. A score is
a binary32 sum of 64 or 128 exact products, off by up to 2^-17 of the sum of their magnitudes; its exponent takes a few
roundings more of 2^-24 of its size. A probability (times its value's scale) enters the second product as f16: off by 2^-11 of itself, or by 2^-25 where it
is below 2^-14, against a largest of 2^7 at least; with N keys and 2^e the largest scale that moves O by up to N 2^-23 2^e.
So with A = sum p |v| / sum p, and delta the scores' error, O is off by (2^-11 + 2 delta) A + N 2^-23 2^e and its own
rounding, 2^-8 |O|. In 16 bits: 2^-8 for 2^-11, and no last term (test_gpu_chunk_attn.py).
"""
import math

import numpy as np
import pytest
import torch

from helpers import cuda
from paper_2608_08721_gb300 import binding as lr

pytestmark = pytest.mark.gpu


def attend64(Q, keys, values, n, kv, scale, softcap=0.0, slopes=None, window=0, sinks=0, first_key=None, prefix_len=None):
    """Q [T, Hq, d]; keys[b], values[b] [Hkv, N_b, d] float64. Returns O, A [T, Hq, d], lse [T, Hq], the largest score,
    and the largest sum of magnitudes of a score's products, with the row's largest added to each of its elements."""
    T, Hq, d = Q.shape
    O, A = torch.zeros((T, Hq, d), dtype=torch.float64), torch.zeros((T, Hq, d), dtype=torch.float64)
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64)
    at, top, mag = 0, 0.0, 0.0
    for b in range(len(n)):
        N = kv[b] + n[b]
        k, p = torch.arange(N)[None], torch.arange(kv[b], N)[:, None]
        see = k <= p
        if prefix_len is not None:
            see = see | (k < int(prefix_len[b]))
        if window:
            see = see & ((k > p - window) | (k < sinks))
        rows = slice(at, at + n[b])
        if first_key is not None:
            see = see & (k >= first_key[rows][:, None])
        for h in range(Hq):
            kvh = h // (Hq // keys[b].shape[0])
            K = torch.where(see.any(0)[:, None], keys[b][kvh, :N], 0.0)  # a key that no row sees may hold anything
            V = torch.where(see.any(0)[:, None], values[b][kvh, :N], 0.0)
            s = Q[rows, h] @ K.T * scale
            if N and n[b]:
                q = Q[rows, h].abs()
                mag = max(mag, float(((q + q.amax(-1, keepdim=True)) @ K.abs().T * scale).max()))
            if softcap:
                s = softcap * torch.tanh(s / softcap)
            if slopes is not None:
                s = s - float(slopes[h]) * (p - k).abs()
            if see.any():
                top = max(top, float(s[see].abs().max()))
            s = s.masked_fill(~see, -math.inf)
            lse[rows, h] = torch.logsumexp(s, dim=-1) if N else -math.inf
            w = torch.exp(s - torch.nan_to_num(lse[rows, h], neginf=0.0)[:, None])
            O[rows, h], A[rows, h] = w @ V, w @ V.abs()
        at += n[b]
    return O, A, lse, top, mag


class Inputs:
    """Queries and a cache, in 8 bits (block > 0) or 16, dense or paged; what is not a sequence's key holds NaN."""

    def __init__(self, n, kv, Hq, Hkv, d, page, block, seed=0, q_scale=1.0, exps=(119, 124), extra=5):
        g = torch.Generator().manual_seed(seed)
        self.n, self.kv, self.block = n, kv, block
        B, T = len(n), int(sum(n))
        N = [a + b for a, b in zip(n, kv)]
        self.Q = (torch.randn((T, Hq, d), generator=g) * q_scale).to(torch.bfloat16)
        unit = block or 1
        cap = (max(1, max(N) + extra) + unit - 1) // unit * unit
        if page:
            per = (cap + page - 1) // page
            planes, rows = B * per + 3, page
            self.table = torch.randperm(planes, generator=g)[:B * per].view(B, per).to(torch.int32)
        else:
            planes, rows, self.table = B, cap, None
        self.keys, self.values, self.dev, self.top_exp = [[] for _ in n], [[] for _ in n], [], 0
        scales = []
        for which in (self.keys, self.values):
            if block:
                x = (torch.randn((planes, Hkv, rows, d), generator=g) * 50).clamp(-440, 440).to(torch.float8_e4m3fn)
                e = torch.randint(*exps, (planes, Hkv, rows // block), generator=g)
                v = x.float() * torch.exp2(e.float() - 127).repeat_interleave(block, 2)[..., None]
                self.top_exp = int(e.max()) - 127
                e = e.to(torch.uint8)
            else:
                x = torch.randn((planes, Hkv, rows, d), generator=g).to(torch.bfloat16)
                v, e = x.float(), None
            used = torch.zeros((planes, rows), dtype=torch.bool)
            for b in range(B):
                if page:
                    m = (N[b] + page - 1) // page
                    ids = self.table[b, :m].long()
                    which[b] = v[ids].transpose(0, 1).reshape(Hkv, -1, d)[:, :N[b]].double()
                    for i in range(m):
                        used[ids[i], :min(page, N[b] - i * page)] = True
                else:
                    which[b] = v[b, :, :N[b]].double()
                    used[b, :N[b]] = True
            if block:
                raw = x.view(torch.uint8)
                raw.masked_fill_(~used[:, None, :, None], 0x7f)
                blocks = used.view(planes, rows // block, block).any(2)
                e.masked_fill_(~blocks[:, None], 255)
                scales.append(e.to(cuda()))
            else:
                x.masked_fill_(~used[:, None, :, None], math.nan)
            self.dev.append(x.to(cuda()))
        self.dev += scales
        if page:
            table = self.table.clone()
            for b in range(B):
                table[b, (N[b] + page - 1) // page:] = 1 << 20  # pages of no key need not exist
            self.dev.append(table.to(cuda()))
        self.cu = torch.from_numpy(np.concatenate([[0], np.cumsum(n)]).astype(np.int32))
        self.kvl = torch.tensor(kv, dtype=torch.int32)
        self.heads = (T, B, Hq, Hkv, d)

    def run(self, ws=None, **opts):
        T, B, Hq, Hkv, d = self.heads
        ws = ws or lr.ChunkWorkspace(T, B, Hq, Hkv, d)
        dev = {k: v.to(cuda()) if isinstance(v, torch.Tensor) else v for k, v in opts.items()}
        O = torch.full((T, Hq, d), 7.0, dtype=torch.bfloat16, device=cuda())
        lse = torch.full((T, Hq), 7.0, device=cuda())
        name = ("libraspec_chunk_attn_q8" if self.block else "libraspec_sink_attn") + ("" if self.table is None else "_paged")
        getattr(lr, name)(self.Q.to(cuda()), *self.dev, self.cu.to(cuda()), self.kvl.to(cuda()), ws, O=O, lse=lse, **dev)
        return O, lse, lr.libraspec_get_status(ws)

    def check(self, **opts):
        O, lse, status = self.run(**opts)
        assert status == 0
        d = self.heads[-1]
        want, A, want_lse, top, mag = attend64(self.Q.double(), self.keys, self.values, self.n, self.kv, d ** -0.5, **opts)
        delta = 2.0 ** -12 + 2.0 ** -17 * mag + 2.0 ** -20 * top
        O, lse = O.double().cpu(), lse.double().cpu()
        bound = ((2.0 ** -11 if self.block else 2.0 ** -8) * 1.01 + 2 * delta) * A + 2.0 ** -8 * 1.01 * want.abs()
        if self.block:
            bound += max(a + b for a, b in zip(self.n, self.kv)) * 2.0 ** -23 * 2.0 ** self.top_exp
        assert bool(torch.isfinite(O).all())
        over = (O - want).abs() - bound
        assert bool((over <= 0).all()), "O over its bound by %.3e at %s" % (over.max(), np.unravel_index(int(over.argmax()), over.shape))
        empty = torch.isinf(want_lse)
        assert torch.equal(empty, torch.isinf(lse)) and bool((O[empty] == 0).all())
        assert bool(((lse - want_lse)[~empty].abs() <= delta + 1e-5 * want_lse[~empty].abs()).all())


# lengths: one token, the edges of a 128-key tile and of a row tile, none at all, blocks of two row tiles
LENGTHS = [([1], [0]), ([1], [127]), ([1], [128]), ([1, 1, 1], [511, 0, 63]), ([5], [2000]), ([129], [0]),
           ([0, 3, 0, 70], [4, 126, 9, 60]), ([64, 65, 1], [1, 190, 255]), ([300, 2], [100, 700])]


@pytest.mark.parametrize("n,kv", LENGTHS)
@pytest.mark.parametrize("Hq,Hkv,d,page,block", [(8, 2, 64, 0, 16), (8, 1, 128, 64, 32), (7, 1, 128, 16, 16), (2, 2, 64, 192, 64),
                                                 (4, 4, 128, 0, 64)])
def test_lengths_heads_and_pages(n, kv, Hq, Hkv, d, page, block):
    Inputs(n, kv, Hq, Hkv, d, page, block, seed=len(n) + Hq).check()


@pytest.mark.parametrize("Hq,Hkv", [(33, 1), (64, 1), (100, 1), (128, 1), (28, 4)])
def test_query_heads_per_kv_head(Hq, Hkv):
    Inputs([3, 1], [100, 300], Hq, Hkv, 64, 32, 16, seed=Hq).check()


def options(name, n, kv, Hq):
    opts = dict(name)
    g = torch.Generator().manual_seed(4)
    T = sum(n)
    if opts.pop("bias", False):
        opts["slopes"] = torch.exp2(-8.0 * torch.arange(1, Hq + 1) / Hq).float()
    if opts.pop("prefix", False):
        opts["prefix_len"] = torch.tensor([a + m // 2 for a, m in zip(kv, n)], dtype=torch.int32)
    if opts.pop("docs", False):  # some rows start behind themselves and see nothing
        opts["first_key"] = torch.cat([torch.randint(0, a + m + 5, (m,), generator=g) for a, m in zip(kv, n)]).to(torch.int32)
        assert len(opts["first_key"]) == T
    return opts


@pytest.mark.parametrize("opts", [dict(window=1), dict(window=5, sinks=1), dict(window=128, sinks=130), dict(window=100000, sinks=7),
                                  dict(sinks=9), dict(softcap=2.0), dict(softcap=30.0, window=77, sinks=4), dict(softcap=1e4),
                                  dict(bias=True), dict(bias=True, window=60, sinks=3), dict(bias=True, softcap=10.0),
                                  dict(softcap=500.0, bias=True, window=90, sinks=40), dict(prefix=True),
                                  dict(prefix=True, window=40, sinks=2), dict(docs=True),
                                  dict(docs=True, prefix=True, bias=True, softcap=5.0, window=200), dict(docs=True, softcap=300.0),
                                  dict(window=0, sinks=0, docs=True, prefix=True)])
@pytest.mark.parametrize("page,d,block", [(0, 64, 32), (32, 128, 16), (16, 64, 16)])
def test_options(opts, page, d, block):
    n, kv, Hq = [70, 1, 0, 200], [300, 411, 3, 5], 6
    Inputs(n, kv, Hq, 2, d, page, block, seed=3, q_scale=2.0).check(**options(opts, n, kv, Hq))


@pytest.mark.parametrize("window,sinks", [(1, 1), (5, 1), (64, 128), (100, 129), (128, 300), (1000, 3), (10, 1000), (7, 0)])
@pytest.mark.parametrize("page,d,block", [(0, 64, 0), (48, 128, 0), (64, 128, 16)])
def test_sinks(window, sinks, page, d, block):
    """Sinks of one tile and more, up to and beyond the window; tokens before and behind them; keys between are not read."""
    Inputs([1, 150, 40, 3], [900, 700, 0, 128], 4, 1, d, page, block, seed=window).check(window=window, sinks=sinks)


@pytest.mark.parametrize("opts", [dict(softcap=20.0), dict(softcap=1e3), dict(bias=True), dict(prefix=True), dict(bias=True, softcap=20.0),
                                  dict(bias=True, softcap=1e3)])
def test_sinks_in_16_bits_beside_other_options(opts):
    n, kv, Hq = [130, 1, 9], [1100, 777, 0], 8
    Inputs(n, kv, Hq, 2, 64, 16, 0, seed=9, q_scale=3.0).check(window=200, sinks=20, **options(opts, n, kv, Hq))


def test_keys_between_the_sinks_and_the_window_take_no_part():
    """They, and their pages, need not exist: NaN there, and block-table entries out of range."""
    for block in (0, 16):
        x = Inputs([2], [2000], 4, 2, 64, 16, block, seed=1)
        want = x.run(window=50, sinks=10)
        page = x.table[0]
        for p in range(1, (2000 - 50) // 16):
            for t in x.dev[:2]:
                t.view(torch.uint8)[page[p]] = 0x7f if block else 0xff
            x.dev[-1][0, p] = -5
        got = x.run(window=50, sinks=10)
        assert got[2] == 0 and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("exps", [(67, 68), (100, 150), (118, 125), (186, 188)])
@pytest.mark.parametrize("opts", [dict(), dict(softcap=20.0)])
def test_scales_over_their_whole_range(exps, opts):
    """Scales of 2^-60 to 2^60 (queries scaled so that scores stay moderate), and scales 2^50 apart in one sequence."""
    q = 2.0 ** (127 - 6 - (exps[0] + exps[1]) // 2)
    x = Inputs([40, 1], [200, 500], 4, 2, 64, 32, 16, seed=2, q_scale=min(max(q, 2.0 ** -66), 2.0 ** 54), exps=exps)
    if exps[1] - exps[0] > 40:  # (keys 2^50 apart: one row's scores all but vanish beside another's)
        x.Q *= 2.0 ** -20
    x.check(**opts)


@pytest.mark.parametrize("q_scale", [0.0, 1e-30, 1e-3, 30.0])
def test_query_magnitudes(q_scale):
    x = Inputs([40, 1], [200, 500], 4, 2, 128, 32, 16, seed=2, q_scale=q_scale)
    x.Q[3] *= 1e-6  # a row far below its neighbours keeps its bits
    x.check()


def test_scales_beyond_the_range_are_read_as_its_ends():
    x = Inputs([5], [100], 2, 1, 64, 0, 16, seed=5, exps=(187, 188), q_scale=2.0 ** -66)
    want = x.run()
    for t in x.dev[2:]:
        t[t == 187] = 250
    got = x.run()
    assert got[2] == 0 and torch.equal(got[0], want[0])


def test_equals_the_attention_of_the_cache_read_back():
    """The values are exact in bf16, so the 16-bit calls on what is read back differ by their own roundings of P alone."""
    n, kv, Hq, Hkv, d = [200, 1, 31], [300, 1500, 0], 8, 2, 128
    x = Inputs(n, kv, Hq, Hkv, d, 64, 16, seed=8)
    N = [a + b for a, b in zip(n, kv)]
    ws = lr.ChunkWorkspace(sum(n), 3, Hq, Hkv, d)
    cu = torch.tensor(np.concatenate([[0], np.cumsum(N)]), dtype=torch.int32, device=cuda())
    zero = torch.zeros(3, dtype=torch.int32, device=cuda())
    K, V = lr.libraspec_kv_read_q8_paged(*x.dev, cu, zero, sum(N), ws)
    cap = max(N)
    Kc, Vc = (torch.zeros((3, Hkv, cap, d), dtype=torch.bfloat16, device=cuda()) for _ in "KV")
    pos = torch.zeros(sum(N), dtype=torch.int32, device=cuda())  # (no rotation)
    lr.libraspec_rope_append(None, K, V, Kc, Vc, cu, zero, lr.RopeFreqs(d), ws, pos=pos)
    O16, lse16 = lr.libraspec_chunk_attn(x.Q.to(cuda()), Kc, Vc, x.cu.to(cuda()), x.kvl.to(cuda()), ws, want_lse=True)
    O8, lse8, status = x.run(ws)
    assert status == 0
    assert float((O8.double() - O16.double()).norm() / O16.double().norm()) < 2.0 ** -8
    assert bool(((lse8 - lse16).abs() <= 2.0 ** -12 + 1e-5 * lse16.abs()).all())


@pytest.mark.parametrize("block", [0, 16])
def test_results_do_not_change_from_run_to_run(block):
    x = Inputs([300, 1, 1, 17], [100, 4000, 9000, 600], 8, 2, 128, 64, block, seed=6)
    ws = lr.ChunkWorkspace(sum(x.n), 4, 8, 2, 128)
    first = x.run(ws, window=5000, sinks=4)
    for _ in range(3):
        again = x.run(ws, window=5000, sinks=4)
        assert again[2] == 0 and torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_many_sequences_and_a_plan_of_its_own_launch():
    r = np.random.default_rng(5)
    B = 600
    Inputs(r.integers(0, 3, B).tolist(), r.integers(0, 300, B).tolist(), 4, 2, 64, 16, 16, seed=7).check(window=100, sinks=2)


def test_long_runs_of_tiles():
    """More tiles than any ring holds, for both streams and for one, over several items of a CTA."""
    Inputs([1, 260], [40000, 5000], 4, 1, 64, 64, 16, seed=3).check()
    Inputs([2], [30000], 2, 1, 128, 0, 64, seed=4).check()


def test_lengths_out_of_range_are_reported():
    x = Inputs([3, 4], [10, 20], 4, 2, 64, 16, 16)
    x.cu = torch.tensor([0, 3, 9], dtype=torch.int32)
    O, _, status = x.run()
    assert status == lr.ST_BAD_LENGTH and bool((O[3:] == 7).all())
    x = Inputs([3, 4], [10, 20], 4, 2, 64, 16, 16)
    x.kvl = torch.tensor([10, 1000], dtype=torch.int32)
    O, _, status = x.run()
    assert status == lr.ST_KV_OVERFLOW and bool((O[3:] == 7).all())
    x = Inputs([3, 4], [10, 20], 4, 2, 64, 16, 16)
    want = x.run()
    x.dev[-1][1, 0] = -1
    O, _, status = x.run()
    assert status == lr.ST_BAD_PAGE and torch.equal(O[:3], want[0][:3])


# ------------------------------------------------------------------------------------ few rows: a decode step, a few tokens each
FEW = [([1, 2, 0, 1], [300, 411, 3, 0]), ([1] * 5, [127, 128, 129, 15, 16]), ([2, 0, 1], [700, 5, 2100]), ([3, 0, 0], [1000, 4, 4])]


@pytest.mark.parametrize("n,kv", FEW)
@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (8, 2), (7, 1), (16, 2), (11, 1), (16, 1)])
@pytest.mark.parametrize("page,d,block", [(0, 64, 32), (32, 128, 16), (0, 128, 64), (16, 64, 16)])
def test_few_rows(n, kv, Hq, Hkv, page, d, block):
    Inputs(n, kv, Hq, Hkv, d, page, block, seed=Hq + d).check()


@pytest.mark.parametrize("opts", [dict(window=1), dict(window=5, sinks=1), dict(window=128, sinks=130), dict(window=100000, sinks=7),
                                  dict(softcap=2.0), dict(softcap=30.0, window=77, sinks=4), dict(softcap=1e4), dict(bias=True),
                                  dict(bias=True, window=60, sinks=3), dict(softcap=500.0, bias=True, window=90, sinks=40),
                                  dict(prefix=True), dict(prefix=True, window=40, sinks=2), dict(docs=True),
                                  dict(docs=True, prefix=True, bias=True, softcap=5.0, window=200)])
@pytest.mark.parametrize("Hq,page,d,block", [(4, 0, 64, 32), (4, 32, 128, 16), (14, 16, 64, 16), (14, 64, 128, 64)])
def test_few_rows_and_options(opts, Hq, page, d, block):
    n, kv = [2, 1, 0, 1, 1], [300, 411, 3, 0, 1500]
    Inputs(n, kv, Hq, 2, d, page, block, seed=3, q_scale=2.0).check(**options(opts, n, kv, Hq))


@pytest.mark.parametrize("exps", [(67, 68), (100, 150), (186, 188)])
def test_few_rows_and_scales_over_their_whole_range(exps):
    q = 2.0 ** (127 - 6 - (exps[0] + exps[1]) // 2)
    x = Inputs([1, 1], [200, 500], 4, 2, 128, 32, 16, seed=2, q_scale=min(max(q, 2.0 ** -66), 2.0 ** 54), exps=exps)
    if exps[1] - exps[0] > 40:
        x.Q *= 2.0 ** -20
    x.check()


def test_few_rows_of_long_caches():
    """Items of several CTAs, more pieces than a warp looks up at once; the same bits from run to run."""
    x = Inputs([1, 1, 2], [40000, 9000, 17], 4, 1, 64, 64, 16, seed=3)
    x.check()
    x = Inputs([1, 1], [30000, 12345], 8, 1, 128, 0, 64, seed=4)
    x.check()
    first = x.run()
    assert all(torch.equal(a, b) for a, b in zip(first[:2], x.run()[:2]))


def test_few_rows_of_many_sequences():
    r = np.random.default_rng(6)
    B = 700
    Inputs(r.integers(0, 3, B).tolist(), r.integers(0, 300, B).tolist(), 4, 1, 64, 16, 16, seed=7).check(window=100, sinks=2)


def test_few_and_many_rows_share_a_workspace():
    """Calls of both kernels in turn on one workspace, as steps of a server make them."""
    big, few = Inputs([300, 40], [500, 90], 8, 2, 128, 64, 16, seed=1), Inputs([1, 1], [4000, 2500], 8, 2, 128, 64, 16, seed=2)
    ws = lr.ChunkWorkspace(340, 2, 8, 2, 128)
    want = [x.run() for x in (big, few)]
    for _ in range(2):
        for x, w in zip((big, few), want):
            got = x.run(ws)
            assert got[2] == 0 and torch.equal(got[0], w[0]) and torch.equal(got[1], w[1])


@pytest.mark.parametrize("n,kv", [([1, 40, 1, 2, 1, 0, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1], [700, 900, 5, 300] + [64 * i for i in range(12)]),
                                  ([3, 5, 4, 4, 4, 2], [100, 1000, 0, 33, 500, 127]), ([17, 0, 0, 0, 0, 1, 1], [300, 4, 5, 6, 7, 8, 2000]),
                                  ([1] * 60 + [150] + [1, 0, 3] * 30, [7 * i for i in range(151)]),
                                  ([0] * 99 + [300] + [0] * 40, [3] * 99 + [80] + [0] * 40)])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 1, 128), (8, 2, 64), (14, 2, 64)])
@pytest.mark.parametrize("opts", [dict(), dict(window=100, sinks=5), dict(docs=True)])
def test_chunks_beside_decoding_sequences(n, kv, Hq, Hkv, d, opts):
    """More new tokens than sequences, on average few enough for the few-row kernel: it takes all, or (of the last, with 4
    or 7 heads for each of the cache's) those that fit its blocks."""
    Inputs(n, kv, Hq, Hkv, d, 32, 16, seed=5).check(**options(opts, n, kv, Hq))


@pytest.mark.parametrize("block,n", [(16, [1, 1]), (16, [40, 7]), (0, [40, 1])])
def test_rows_behind_the_last_sequence_are_left_alone(block, n):
    x = Inputs(n, [100, 50], 4, 2, 64, 16, block, seed=2)
    T, B, Hq, Hkv, d = x.heads
    want, want_lse, _ = x.run(window=60, sinks=3)
    x.Q = torch.cat([x.Q, torch.full((5, Hq, d), math.nan, dtype=torch.bfloat16)])
    x.heads = (T + 5, B, Hq, Hkv, d)
    O, lse, status = x.run(window=60, sinks=3)
    # (blocks may be cut elsewhere: the results of other kernels' parts differ in their last bits)
    assert status == 0 and bool((O[T:] == 7).all()) and bool((lse[T:] == 7).all())
    assert bool(((O[:T].float() - want.float()).abs() <= 2.0 ** -6 * want.float().abs() + 1e-3).all())
    assert bool(((lse[:T] - want_lse).abs() <= 1e-3).all())


@pytest.mark.parametrize("block,n", [(16, [1, 1, 1]), (16, [200, 1, 30]), (16, [3, 9, 1]), (0, [200, 1, 30]),
                                     (16, [1, 150, 1] + [1] * 77)])
def test_as_a_graph(block, n):
    """Captured once, replayed on other queries and lengths in the same buffers: what eager calls give."""
    B = len(n)
    x = Inputs(n, [900, 700, 64] + [9] * (B - 3), 8, 2, 64, 64, block, seed=4)
    T, B, Hq, Hkv, d = x.heads
    fn = lr.libraspec_chunk_attn_q8_paged if block else lr.libraspec_sink_attn_paged
    ws, cu, kvl, Q = lr.ChunkWorkspace(T, B, Hq, Hkv, d), x.cu.to(cuda()), x.kvl.to(cuda()), x.Q.to(cuda())

    def call():
        return fn(Q, *x.dev, cu, kvl, ws, window=500, sinks=4, want_lse=True)

    call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = call()
    for lengths in ([900, 700, 64], [3, 640, 0], [899, 1, 63]):
        kvl[:3].copy_(torch.tensor(lengths, dtype=torch.int32))
        Q.copy_(torch.randn(Q.shape, device=cuda()))
        graph.replay()
        got = [t.clone() for t in out]
        want = call()
        assert lr.libraspec_get_status(ws) == 0
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_call_on_another_stream():
    x = Inputs([50, 1, 1, 2], [900, 700, 64, 5], 8, 2, 128, 64, 16, seed=4)
    T, B, Hq, Hkv, d = x.heads
    ws, cu, kvl, Q = lr.ChunkWorkspace(T, B, Hq, Hkv, d), x.cu.to(cuda()), x.kvl.to(cuda()), x.Q.to(cuda())
    want = lr.libraspec_chunk_attn_q8_paged(Q, *x.dev, cu, kvl, ws)[0].clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = lr.libraspec_chunk_attn_q8_paged(Q, *x.dev, cu, kvl, ws, stream=side)[0]
    side.synchronize()
    assert torch.equal(got, want)


def test_a_cache_whose_offsets_pass_32_bits():
    """Keys and codes beyond 2^32 bytes: appended, read back and attended to, by both kernels, at the end of 18 million keys
    (in a window, with sinks)."""
    Hq, Hkv, d, block, S = 4, 2, 128, 64, 18_000_000 // 64 * 64
    codes = [torch.empty((1, Hkv, S, d), dtype=torch.float8_e4m3fn, device=cuda()) for _ in "KV"]
    exps = [torch.zeros((1, Hkv, S // block), dtype=torch.uint8, device=cuda()) for _ in "KV"]
    assert codes[0].numel() > 2 ** 32
    g = torch.Generator().manual_seed(1)
    ws, freqs, window, sinks = lr.ChunkWorkspace(300, 1, Hq, Hkv, d), lr.RopeFreqs(d), 200, 10

    def step(at, n):
        x = torch.randn((n, Hq + 2 * Hkv, d), generator=g).to(torch.bfloat16).to(cuda())
        cu, kv = torch.tensor([0, n], dtype=torch.int32, device=cuda()), torch.tensor([at], dtype=torch.int32, device=cuda())
        pos = torch.zeros(n, dtype=torch.int32, device=cuda())  # (no rotation: the values are the inputs')
        q = lr.libraspec_rope_append_q8(x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], *codes, *exps, cu, kv, freqs, ws, pos=pos)
        K, V = lr.libraspec_kv_read_q8(*codes, *exps, cu, kv, n, ws)
        O, _ = lr.libraspec_chunk_attn_q8(q, *codes, *exps, cu, kv, ws, window=window, sinks=sinks)
        assert lr.libraspec_get_status(ws) == 0
        assert bool(((K.float() - x[:, Hq:Hq + Hkv].float()).abs() <= 2.0 ** -4 * x[:, Hq:Hq + Hkv].float().abs() + 2.0 ** -13).all())
        return q.double().cpu(), K.double().cpu(), V.double().cpu(), O.double().cpu()

    _, K0, V0, _ = step(0, 16)
    end = S - 300
    _, K1, V1, _ = step(end - 256, 256)
    for n in (299, 1):
        q, K2, V2, O = step(end, n)
        keys, values = torch.cat([K0[:sinks], K1, K2]), torch.cat([V0[:sinks], V1, V2])
        pos = torch.cat([torch.arange(sinks), torch.arange(end - 256, end + n)])
        p = torch.arange(end, end + n)[:, None]
        see = (pos <= p) & ((pos > p - window) | (pos < sinks))
        for h in range(Hq):
            s = (q[:, h] @ keys[:, h // 2].T * d ** -0.5).masked_fill(~see, -math.inf)
            w = s.softmax(-1)
            v = values[:, h // 2]
            assert bool(((O[:, h] - w @ v).abs() <= 2.0 ** -7 * (w @ v.abs())).all())


@pytest.mark.parametrize("n,kv", [([1], [70000]), ([2], [9000]), ([4, 1], [3000, 40000]), ([1, 1, 1], [1030, 0, 20000])])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 1, 128), (16, 1, 64), (3, 1, 128)])
@pytest.mark.parametrize("opts", [dict(), dict(window=30000, sinks=200)])
def test_rows_in_many_parts(n, kv, Hq, Hkv, d, opts):
    """Few rows over long caches: up to every CTA has a part of a row's keys; parts are merged in groups."""
    Inputs(n, kv, Hq, Hkv, d, 0, 64, seed=6).check(**options(opts, n, kv, Hq))


@pytest.mark.parametrize("kv", [1030, 9 * 128 - 1, 17 * 128 - 5])
def test_a_last_group_of_one_part(kv):
    """Nine or seventeen parts of a row: the last is a group by itself. Calls on two sets of queries in turn give the same
    each time (nothing is read of what the call before left)."""
    x = Inputs([1, 1], [kv, 20000], 3, 1, 128, 0, 64, seed=8)
    T, B, Hq, Hkv, d = x.heads
    ws, cu, kvl, Q = lr.ChunkWorkspace(T, B, Hq, Hkv, d), x.cu.to(cuda()), x.kvl.to(cuda()), x.Q.to(cuda())
    x.check()
    both = [Q, torch.randn(Q.shape, device=cuda(), dtype=torch.bfloat16)]
    runs = [lr.libraspec_chunk_attn_q8(both[i % 2], *x.dev, cu, kvl, ws, want_lse=True) for i in range(600)]
    for i in range(2, 600):
        assert all(torch.equal(a, b) for a, b in zip(runs[i], runs[i % 2]))


def test_two_calls_at_once():
    """Two streams, a workspace each."""
    both = [Inputs(n, kv, 8, 2, 128, 64, 16, seed=i) for i, (n, kv) in enumerate([([1, 1, 1], [3000, 5, 900]),
                                                                                  ([200, 1], [700, 2000])])]
    args, want = [], []
    for x in both:
        T, B, Hq, Hkv, d = x.heads
        args.append((x.Q.to(cuda()), *x.dev, x.cu.to(cuda()), x.kvl.to(cuda()), lr.ChunkWorkspace(T, B, Hq, Hkv, d)))
        want.append(lr.libraspec_chunk_attn_q8_paged(*args[-1], want_lse=True))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in both]
    got = [[lr.libraspec_chunk_attn_q8_paged(*a, want_lse=True, stream=s) for a, s in zip(args, streams)] for _ in range(20)]
    torch.cuda.synchronize()
    for pair in got:
        for (O, lse), (O1, lse1) in zip(pair, want):
            assert torch.equal(O, O1) and torch.equal(lse, lse1)
    assert all(lr.libraspec_get_status(a[-1]) == 0 for a in args)
