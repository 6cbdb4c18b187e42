"""GPU: query and key heads normed and rotated (libraspec_qk_norm_rope), the append to a cache in 8 bits
(libraspec_rope_append_q8[_paged]) and its read-back (libraspec_kv_read_q8[_paged]), against their definitions in 64 bits.

Tolerances, from the arithmetic. The rotation: 4e-6 of a pair's length (test_gpu_rope.py). The norm before it: a sum of
squares in chains of up to 32 roundings and five more over the lanes, 2^-24 each and halved by the root, the root to 2 ulp,
two products: below 32 roundings, 2e-6 of the value. A bf16 result adds 2^-8 of the value. Codes are rounded from a value
that far off: they lie between the codes of the two ends; and an exponent between those of the largest magnitude's ends.
"""
import math

import numpy as np
import pytest
import torch

from helpers import cuda
from paper_2608_08721_gb300 import binding as lr
from test_gpu_rope import freqs64, rotate64

pytestmark = pytest.mark.gpu
ROPE, NORM = 4e-6, 2e-6


def norm64(x, w, eps):
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w


def weights(d, seed):
    return [1.0 + 0.5 * torch.randn(d, generator=torch.Generator().manual_seed(seed + i)) for i in range(2)]


def assert_normed(got, want, length, dtype, rot):
    bound = (ROPE + NORM) * length + NORM * want.abs() + (2.0 ** -8 * 1.001 * want.abs() if dtype == torch.bfloat16 else 0.0)
    err = (got.double().cpu() - want).abs()
    assert bool((err <= bound).all()), "max %.3e over the bound by %.3e" % (err.max(), (err - bound).max())


@pytest.mark.parametrize("d,rot,Hq,Hk,T", [(128, 128, 32, 8, 64), (64, 64, 8, 2, 1), (128, 64, 7, 1, 33), (128, 24, 3, 0, 19),
                                           (64, 58, 0, 2, 5), (128, 2, 1, 1, 3), (256, 256, 5, 3, 9), (36, 20, 3, 2, 11),
                                           (512, 512, 2, 1, 4), (512, 512, 20, 20, 3), (96, 96, 40, 8, 7), (2, 2, 3, 4, 5)])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_rope(d, rot, Hq, Hk, T, inter, dtype):
    g = torch.Generator().manual_seed(d * rot + Hq)
    x = (torch.randn((T, Hq + Hk, d), generator=g) * torch.exp(torch.randn((T, Hq + Hk, 1), generator=g))).to(dtype)
    pos = torch.randint(0, 131072, (T,), generator=g, dtype=torch.int32)
    wq, wk = weights(d, 3)
    norm = lr.QkNorm(wq.to(cuda()), wk.to(cuda()), 1e-5)
    y = lr.libraspec_qk_norm_rope(x.to(cuda()), Hq, norm, pos.to(cuda()), lr.RopeFreqs(rot, magnitude=1.25), interleaved=inter)
    z = torch.cat([norm64(x[:, :Hq].double(), wq.double(), 1e-5), norm64(x[:, Hq:].double(), wk.double(), 1e-5)], 1)
    want, length = rotate64(z, pos.numpy(), freqs64(rot), inter, 1.25)
    assert y.dtype == dtype
    assert_normed(y, want, length, dtype, rot)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset", [0, 1])
def test_norm_rope_strided_in_place_and_unaligned(dtype, offset):
    """Queries and keys within a wider projection, in place: the rest of the row stays; also at an odd offset."""
    g = torch.Generator().manual_seed(3)
    T, H, d, width = 21, 6, 64, 11 * 64 + 8
    buf = torch.randn((T, width), generator=g).to(dtype)
    dev = buf.to(cuda())
    at = slice(128 + offset, 128 + offset + H * d)
    view, x = dev[:, at].unflatten(1, (H, d)), buf[:, at].unflatten(1, (H, d)).double()
    pos = torch.arange(7, 7 + T, dtype=torch.int32)
    wq, wk = weights(d, 5)
    out = lr.libraspec_qk_norm_rope(view, 4, lr.QkNorm(wq.to(cuda()), wk.to(cuda())), pos.to(cuda()), lr.RopeFreqs(d), Y=view)
    assert out is view
    z = torch.cat([norm64(x[:, :4], wq.double(), 1e-6), norm64(x[:, 4:], wk.double(), 1e-6)], 1)
    want, length = rotate64(z, pos.numpy(), freqs64(d), False)
    assert_normed(view, want, length, dtype, d)
    same = torch.ones(width, dtype=torch.bool)
    same[at] = False
    assert torch.equal(dev.cpu()[:, same], buf[:, same])


def test_norm_rope_of_zeros_and_tiny_heads():
    """The mean square of the first vanishes beside eps; a head of zeros stays zero."""
    x = torch.zeros((3, 2, 64))
    x[1] = 1e-8
    x[2] = 3.0
    one = torch.ones(64, device=cuda())
    y = lr.libraspec_qk_norm_rope(x.to(cuda()), 1, lr.QkNorm(one, one, 1e-6), torch.zeros(3, dtype=torch.int32, device=cuda()),
                                  lr.RopeFreqs(64)).cpu()
    assert bool((y[0] == 0).all())
    assert torch.allclose(y[1], torch.tensor(1e-5), rtol=1e-5, atol=0) and torch.allclose(y[2], torch.tensor(1.0), rtol=1e-6)


# ------------------------------------------------------------------------------------------------------- the cache in 8 bits
def to_e4m3(x):
    """Nearest e4m3 value, ties to even, saturating."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))).clamp_min(-6) - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


def exponent(amax):
    return (torch.floor(torch.log2(amax.double().clamp_min(2.0 ** -100))) - 7).clamp(-60, 60)


class Cache:
    """A cache in 8 bits on the device, dense or paged, with random contents, and what it held at the start."""

    def __init__(self, B, Hkv, d, cap, block, page, seed):
        g = torch.Generator().manual_seed(seed)
        self.B, self.Hkv, self.d, self.block, self.page = B, Hkv, d, block, page
        if page:
            per = (cap + page - 1) // page
            planes, rows = B * per + 3, page
            self.table = torch.randperm(planes, generator=g)[:B * per].view(B, per).to(torch.int32)
        else:
            planes, rows, self.table = B, (cap + block - 1) // block * block, None
        self.codes = [(torch.randn((planes, Hkv, rows, d), generator=g) * 60).clamp(-440, 440).to(torch.float8_e4m3fn) for _ in "KV"]
        self.exps = [torch.randint(115, 122, (planes, Hkv, rows // block), generator=g).to(torch.uint8) for _ in "KV"]
        self.dev = [t.to(cuda()) for t in self.codes + self.exps]
        self.dev_table = [] if self.table is None else [self.table.to(cuda())]

    def where(self, b, key):
        return (b, key) if not self.page else (int(self.table[b, key // self.page]), key % self.page)

    def rows(self, codes, exps, b, a, e):
        """Values of keys [a, e) of sequence b, [e - a, Hkv, d] float64, and the exponents of their rows."""
        if e <= a:
            return torch.zeros((0, self.Hkv, self.d), dtype=torch.float64), torch.zeros((0, self.Hkv), dtype=torch.float64)
        at = [self.where(b, k) for k in range(a, e)]
        p, r = torch.tensor([x for x, _ in at]), torch.tensor([x for _, x in at])
        ex = exps[p, :, r // self.block].double() - 127
        return codes.float()[p, :, r].double() * torch.exp2(ex)[..., None], ex


def append(cache, qkv, Hq, cu, kv, freqs, norm=None, inter=False, ws=None, pos=None, queries=True):
    Hkv = cache.Hkv
    ws = ws or lr.ChunkWorkspace(1, 1, 1, 1, 64)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    fn = lr.libraspec_rope_append_q8_paged if cache.page else lr.libraspec_rope_append_q8
    out = fn(q if queries else None, k, v, *cache.dev, *cache.dev_table, cu.to(cuda()), kv.to(cuda()), freqs, ws, norm=norm,
             interleaved=inter, pos=pos)
    return out, lr.libraspec_get_status(ws)


def check_cache(cache, name, new, slack, n, kv, before):
    """new [T, Hkv, d] float64 with slack (how far the kernel's value may be off); before: (codes, exponents) on the CPU."""
    which = "KV".index(name)
    codes, exps = cache.dev[which].cpu(), cache.dev[2 + which].cpu()
    old_codes, old_exps = before[which], before[2 + which]
    touched = torch.zeros((codes.shape[0], codes.shape[2]), dtype=torch.bool)
    touched_e = torch.zeros((exps.shape[0], exps.shape[2]), dtype=torch.bool)
    at = 0
    for b in range(len(n)):
        a, e = kv[b], kv[b] + n[b]
        for first in range(a // cache.block * cache.block, e, cache.block) if n[b] else ():
            lo, hi = max(first, a), min(first + cache.block, e)
            x, s = new[at + lo - a:at + hi - a], slack[at + lo - a:at + hi - a]
            low, high = exponent((x.abs() - s).clamp_min(0).amax((0, 2))), exponent((x.abs() + s).amax((0, 2)))
            p, r = cache.where(b, first)
            touched_e[p, r // cache.block] = True
            touched[p, r:r + hi - first] = True
            got = exps[p, :, r // cache.block].double() - 127
            if first < a:
                had, had_e = cache.rows(old_codes, old_exps, b, first, a)
                low, high = torch.maximum(low, had_e[0]), torch.maximum(high, had_e[0])
                want = to_e4m3(had / torch.exp2(got)[:, None])
                assert torch.equal(codes[p, :, r:r + a - first].double().transpose(0, 1), want), "rows that the block had"
            assert bool(((got >= low) & (got <= high)).all()), (name, b, first, got, low, high)
            c = codes[p, :, r + lo - first:r + hi - first].double().transpose(0, 1)
            scale = torch.exp2(got)[:, None]
            ends = to_e4m3((x - s) / scale), to_e4m3((x + s) / scale)
            assert bool(((c >= ends[0]) & (c <= ends[1])).all()), (name, b, first)
        at += n[b]
    rest = ~touched[:, None, :].expand(-1, cache.Hkv, -1)
    assert torch.equal(codes.view(torch.uint8)[rest], old_codes.view(torch.uint8)[rest]), "rows of no new token changed"
    rest = ~touched_e[:, None, :].expand(-1, cache.Hkv, -1)
    assert torch.equal(exps[rest], old_exps[rest])


def check_append(n, kv, Hq, Hkv, d, block, page, dtype=torch.bfloat16, rot=None, inter=False, norm=False, seed=0, scale=1.0,
                 offset=0, extra=7):
    rot = rot or d
    g = torch.Generator().manual_seed(seed)
    T = sum(n)
    cache = Cache(len(n), Hkv, d, max(a + b for a, b in zip(n, kv)) + extra, block, page, seed)
    before = [t.cpu().clone() for t in cache.dev]
    wide = (torch.randn((T, (Hq + 2 * Hkv) * d + offset), generator=g) * scale).to(dtype)
    x = wide[:, offset:].unflatten(1, (Hq + 2 * Hkv, d))
    dev = wide.to(cuda())[:, offset:].unflatten(1, (Hq + 2 * Hkv, d))
    cu = torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=torch.int32)
    wq, wk = weights(d, seed)
    nm = lr.QkNorm(wq.to(cuda()), wk.to(cuda()), 1e-5) if norm else None
    Qo, status = append(cache, dev, Hq, cu, torch.tensor(kv, dtype=torch.int32), lr.RopeFreqs(rot), nm, inter)
    assert status == 0
    pos = np.concatenate([np.arange(a, a + m) for a, m in zip(kv, n)])
    q, k, v = x[:, :Hq].double(), x[:, Hq:Hq + Hkv].double(), x[:, Hq + Hkv:].double()
    if norm:
        q, k = norm64(q, wq.double(), 1e-5), norm64(k, wk.double(), 1e-5)
    f = freqs64(rot)
    wq_, lq = rotate64(q, pos, f, inter)
    wk_, lk = rotate64(k, pos, f, inter)
    assert_normed(Qo, wq_, lq, torch.bfloat16, rot)
    slack = ROPE * lk + (NORM * (lk + wk_.abs()) if norm else 0.0)
    check_cache(cache, "K", wk_, slack, n, kv, before)
    check_cache(cache, "V", v, torch.zeros_like(v), n, kv, before)
    return cache


# new tokens and lengths: one token at a block's first, last and middle row, none, blocks filled up and begun, whole blocks
RAGGED = [([1], [0]), ([1], [15]), ([1], [16]), ([1, 1, 1, 1], [511, 0, 63, 40]), ([5], [62]), ([129], [0]),
          ([0, 3, 0, 70], [4, 126, 9, 60]), ([64, 65, 1], [1, 190, 255]), ([300, 2], [100, 7]), ([16, 64, 32], [16, 64, 32])]


@pytest.mark.parametrize("n,kv", RAGGED)
@pytest.mark.parametrize("Hq,Hkv,d,block,page", [(8, 2, 64, 16, 0), (7, 1, 128, 64, 64), (4, 2, 128, 32, 96), (2, 2, 64, 64, 0),
                                                 (8, 4, 128, 16, 16)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_append_lengths_blocks_and_pages(n, kv, Hq, Hkv, d, block, page, dtype):
    check_append(n, kv, Hq, Hkv, d, block, page, dtype, norm=d == 128, seed=len(n) + block)


@pytest.mark.parametrize("d,rot", [(128, 128), (128, 64), (128, 122), (64, 24), (64, 58), (128, 2)])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dtype,offset", [(torch.float32, 0), (torch.bfloat16, 0), (torch.bfloat16, 3), (torch.float32, 1)])
def test_append_rotated_parts_layouts_and_alignment(d, rot, inter, dtype, offset):
    check_append([33, 1, 70], [5, 100, 0], 5, 2, d, 32, 32, dtype, rot=rot, inter=inter, norm=inter, seed=rot, offset=offset)


@pytest.mark.parametrize("scale", [1e-30, 1e-6, 100.0, 1e15, 1e30])
def test_append_magnitudes(scale):
    """Blocks that had tokens of another magnitude grow (their codes are rounded again, down to zero) or keep their scale."""
    check_append([20, 3, 1], [70, 40, 9], 2, 2, 64, 32, 0, torch.float32, seed=5, scale=scale)


def test_append_many_heads_and_sequences():
    r = np.random.default_rng(3)
    B = 300
    check_append(r.integers(0, 4, B).tolist(), r.integers(0, 70, B).tolist(), 40, 3, 64, 16, 16, seed=11)


def test_append_in_steps_holds_what_one_step_holds():
    """128 tokens at once and in steps of 1 to 50: the same codes, but for scales that grew later (magnitudes rise with the
    position here, so nearly every step grows them) and values below 2^-6 of a scale, which were rounded twice."""
    g = torch.Generator().manual_seed(0)
    T, Hkv, d, block = 128, 2, 64, 32
    x = torch.randn((T, 3 * Hkv, d), generator=g) * torch.linspace(0.1, 30, T)[:, None, None]
    dev, freqs = x.to(cuda()), lr.RopeFreqs(d)
    caches = []
    for steps in ([T], [1, 50, 3, 20, 29, 25]):
        cache, at = Cache(1, Hkv, d, T, block, 0, 1), 0
        for m in steps:
            _, status = append(cache, dev[at:at + m], Hkv, torch.tensor([0, m], dtype=torch.int32),
                               torch.tensor([at], dtype=torch.int32), freqs)
            assert status == 0
            at += m
        caches.append([t.cpu() for t in cache.dev])
    for which in range(2):
        a, b = (c[which].double() for c in caches)
        ea, eb = (c[2 + which] for c in caches)
        assert torch.equal(ea, eb)
        normal = a.abs() >= 2.0 ** -6
        assert torch.equal(a[normal], b[normal]) and bool((a - b).abs().max() <= 2.0 ** -9)


def test_append_special_values():
    """Zeros, infinities, NaN: the scale is the finite values'; infinities saturate, NaN stays."""
    Hkv, d = 1, 64
    x = torch.zeros((48, 3, d))
    x[16:32] = torch.randn((16, 3, d), generator=torch.Generator().manual_seed(1))
    x[20, 2, 3], x[21, 2, 4], x[22, 2, 5] = math.inf, -math.inf, math.nan
    x[32:] = math.nan
    cache = Cache(1, Hkv, d, 48, 16, 0, 1)
    _, status = append(cache, x.to(cuda()), 1, torch.tensor([0, 48], dtype=torch.int32), torch.tensor([0], dtype=torch.int32),
                       lr.RopeFreqs(d))
    assert status == 0
    V, Vs = cache.dev[1].cpu()[0, 0].double(), cache.dev[3].cpu()[0, 0].double() - 127
    v = x[:, 2].double()
    assert bool((V[:16] == 0).all()) and Vs[0] == -60 and Vs[2] == -60
    assert bool(torch.isnan(V[32:]).all())
    fine = torch.isfinite(v[16:32])
    assert Vs[1] == exponent(v[16:32][fine].abs().max())
    want = to_e4m3(v[16:32] / 2.0 ** Vs[1])
    assert torch.equal(V[16:32][fine], want[fine])
    assert V[20, 3] == 448 and V[21, 4] == -448 and bool(torch.isnan(V[22, 5]))


def test_append_without_queries_at_given_positions():
    g = torch.Generator().manual_seed(2)
    T, Hkv, d = 40, 2, 128
    x = torch.randn((T, 2 * Hkv, d), generator=g)
    cache = Cache(2, Hkv, d, 64, 16, 16, 3)
    before = [t.cpu().clone() for t in cache.dev]
    pos = torch.randint(0, 100000, (T,), generator=g, dtype=torch.int32)
    out, status = append(cache, x.to(cuda()), 0, torch.tensor([0, 30, 40], dtype=torch.int32),
                         torch.tensor([3, 17], dtype=torch.int32), lr.RopeFreqs(d), pos=pos.to(cuda()), queries=False)
    assert out is None and status == 0
    k, lk = rotate64(x[:, :Hkv].double(), pos.numpy(), freqs64(d), False)
    check_cache(cache, "K", k, ROPE * lk, [30, 10], [3, 17], before)


def test_append_reports_what_does_not_fit():
    """Offsets that run backwards, a chunk beyond the capacity, a page that does not exist: those rows alone are skipped."""
    d, Hkv = 64, 1
    x = torch.randn((20, 3, d), generator=torch.Generator().manual_seed(4))
    freqs = lr.RopeFreqs(d)

    def case(cu, kv, change=None, page=16, B=2, cap=32):
        cache = Cache(B, Hkv, d, cap, 16, page, 9)
        if change:
            cache.dev_table[0][change] = cache.codes[0].shape[0]
        before = [t.cpu().clone() for t in cache.dev]
        _, status = append(cache, x.to(cuda()), 1, torch.tensor(cu, dtype=torch.int32), torch.tensor(kv, dtype=torch.int32), freqs)
        return cache, before, status

    v = x[:, 2:].double()
    none = torch.zeros_like(v)
    cache, before, status = case([0, 8, 4], [3, 0])
    assert status == lr.ST_BAD_LENGTH
    check_cache(cache, "V", v, none, [8, 0], [3, 0], before)
    cache, before, status = case([0, 8, 21], [3, 0])
    assert status == lr.ST_BAD_LENGTH
    check_cache(cache, "V", v, none, [8, 0], [3, 0], before)
    cache, before, status = case([0, 10, 20], [3, 27])
    assert status == lr.ST_KV_OVERFLOW
    check_cache(cache, "V", v, none, [10, 5], [3, 27], before)
    cache, before, status = case([0, 10, 20], [-1, 32])
    assert status == lr.ST_KV_OVERFLOW
    check_cache(cache, "V", v, none, [0, 0], [0, 0], before)
    cache, before, status = case([0, 10, 20], [12, 5], change=(0, 1))
    assert status == lr.ST_BAD_PAGE
    check_cache(cache, "V", torch.cat([v[:4], v[10:]]), none[:14], [4, 10], [12, 5], before)


@pytest.mark.parametrize("d,Hkv,block,page", [(64, 2, 16, 0), (128, 1, 64, 64), (128, 8, 32, 96), (64, 3, 16, 16)])
def test_read_back(d, Hkv, block, page):
    n, start = [5, 0, 130, 1, 64], [3, 7, 0, 127, 64]
    cache = Cache(len(n), Hkv, d, 200, block, page, 7)
    cu = torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=torch.int32)
    ws = lr.ChunkWorkspace(1, 1, 1, 1, 64)
    T = sum(n) + 4  # rows of no sequence behind the last
    out = [torch.full((T, Hkv, d), 7.0, dtype=torch.bfloat16, device=cuda()) for _ in "KV"]
    fn = lr.libraspec_kv_read_q8_paged if page else lr.libraspec_kv_read_q8
    got = fn(*cache.dev, *cache.dev_table, cu.to(cuda()), torch.tensor(start, dtype=torch.int32, device=cuda()), T, ws, K=out[0],
             V=out[1])
    assert got[0] is out[0] and lr.libraspec_get_status(ws) == 0
    for i in range(2):
        y = got[i].double().cpu()
        want = torch.cat([cache.rows(cache.codes[i], cache.exps[i], b, s, s + m)[0] for b, (s, m) in enumerate(zip(start, n))])
        assert torch.equal(y[:sum(n)], want) and bool((y[sum(n):] == 7).all())


def test_read_back_every_code_and_exponent():
    """All 256 codes under exponents over the whole range, those beyond it read as its ends."""
    d = 64
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).view(4, d).repeat(4, 1)  # [16, 64]
    exps = torch.tensor([0, 60, 67, 100, 127, 150, 187, 188, 254, 255], dtype=torch.uint8)
    B = len(exps)
    K8 = codes.expand(B, 1, 16, d).contiguous()
    s = exps.view(B, 1, 1)
    dev = [t.to(cuda()) for t in (K8, K8, s, s)]
    cu = torch.arange(0, 16 * B + 1, 16, dtype=torch.int32, device=cuda())
    K, V = lr.libraspec_kv_read_q8(*dev, cu, torch.zeros(B, dtype=torch.int32, device=cuda()), 16 * B, lr.ChunkWorkspace(1, 1, 1, 1, 64))
    want = codes.double()[None] * torch.exp2(exps.double().clamp(67, 187) - 127)[:, None, None]
    for y in (K, V):
        assert torch.equal(torch.nan_to_num(y.double().cpu().view(B, 16, d), nan=123.0), torch.nan_to_num(want, nan=123.0))


def test_read_reports_what_it_cannot_read():
    cache = Cache(3, 1, 64, 32, 16, 16, 2)
    cache.dev_table[0][1, 0] = -1
    ws = lr.ChunkWorkspace(1, 1, 1, 1, 64)

    def read(cu, start):
        out = [torch.full((20, 1, 64), 7.0, dtype=torch.bfloat16, device=cuda()) for _ in "KV"]
        lr.libraspec_kv_read_q8_paged(*cache.dev, *cache.dev_table, torch.tensor(cu, dtype=torch.int32, device=cuda()),
                                      torch.tensor(start, dtype=torch.int32, device=cuda()), 20, ws, K=out[0], V=out[1])
        return out[0].double().cpu(), lr.libraspec_get_status(ws)

    def rows(b, a, e):
        return cache.rows(cache.codes[0], cache.exps[0], b, a, e)[0]

    y, status = read([0, 4, 8, 12], [0, 0, 28])
    assert status == lr.ST_BAD_PAGE
    assert torch.equal(y[:4], rows(0, 0, 4)) and bool((y[4:8] == 7).all()) and torch.equal(y[8:12], rows(2, 28, 32))
    y, status = read([0, 4, 4, 12], [0, 0, 28])
    assert status == lr.ST_KV_OVERFLOW and torch.equal(y[4:8], rows(2, 28, 32)) and bool((y[8:] == 7).all())
    y, status = read([0, 4, 2, 25], [-1, 0, 0])
    assert status == lr.ST_BAD_LENGTH | lr.ST_KV_OVERFLOW and bool((y == 7).all())


def test_append_and_read_as_a_graph():
    """Captured, replayed on other inputs in the same buffers: what eager calls give."""
    g = torch.Generator().manual_seed(8)
    B, Hkv, d = 3, 2, 64
    x = torch.randn((2, 30, 3 * Hkv, d), generator=g).to(cuda())
    cu, kv = torch.tensor([0, 10, 11, 30], dtype=torch.int32, device=cuda()), torch.tensor([5, 31, 64], dtype=torch.int32, device=cuda())
    freqs, ws = lr.RopeFreqs(d), lr.ChunkWorkspace(1, 1, 1, 1, 64)
    eager, cache = Cache(B, Hkv, d, 96, 32, 32, 4), Cache(B, Hkv, d, 96, 32, 32, 4)

    def step(c, qkv):
        q = lr.libraspec_rope_append_q8_paged(qkv[:, :Hkv], qkv[:, Hkv:2 * Hkv], qkv[:, 2 * Hkv:], *c.dev, *c.dev_table, cu, kv,
                                              freqs, ws)
        return (q, *lr.libraspec_kv_read_q8_paged(*c.dev, *c.dev_table, cu, kv, 30, ws))

    want = [[t.clone() for t in step(eager, x[i])] for i in range(2)]
    buf = x[0].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = step(cache, buf)
    for i in range(2):
        buf.copy_(x[i])
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(out, want[i]))
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(cache.dev, eager.dev))


@pytest.mark.parametrize("n", [[2, 1], [40, 9]])
def test_append_leaves_rows_of_no_sequence_alone(n):
    d, Hq, Hkv = 64, 3, 1
    T = sum(n) + 5
    x = torch.randn((T, Hq + 2 * Hkv, d), generator=torch.Generator().manual_seed(4)).to(cuda())
    cache = Cache(2, Hkv, d, 64, 16, 16, 9)
    cu, kv = torch.tensor([0, n[0], sum(n)], dtype=torch.int32, device=cuda()), torch.tensor([3, 16], dtype=torch.int32, device=cuda())
    Qo = torch.full((T, Hq, d), 7.0, dtype=torch.bfloat16, device=cuda())
    ws = lr.ChunkWorkspace(1, 1, 1, 1, 64)
    lr.libraspec_rope_append_q8_paged(x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], *cache.dev, *cache.dev_table, cu, kv,
                                      lr.RopeFreqs(d), ws, Qo=Qo)
    assert lr.libraspec_get_status(ws) == 0
    assert bool((Qo[sum(n):] == 7).all()) and not bool((Qo[:sum(n)] == 7).all(-1).any())


@pytest.mark.parametrize("B", [3, 40])
def test_append_of_ranges_that_overlap(B):
    """Beside offsets that decrease the ranges of others may overlap: reported; a sequence before them holds what it should."""
    d, Hkv, T = 64, 1, 60
    x = torch.randn((T, 3, d), generator=torch.Generator().manual_seed(4))
    cache = Cache(B, Hkv, d, 80, 16, 16, 9)
    before = [t.cpu().clone() for t in cache.dev]
    cu = [0, 20] + [0, T] * B
    cu, kv = torch.tensor(cu[:B + 1], dtype=torch.int32), torch.zeros(B, dtype=torch.int32)
    _, status = append(cache, x.to(cuda()), 1, cu, kv, lr.RopeFreqs(d))
    assert status == lr.ST_BAD_LENGTH
    got, _ = cache.rows(cache.dev[1].cpu(), cache.dev[3].cpu(), 0, 0, 20)
    v = x[:20, 2:].double()
    assert bool(((got - v).abs() <= 2.0 ** -4 * v.abs() + 2.0 ** -10).all())


def test_empty_calls():
    d = 64
    cache = Cache(2, 1, d, 32, 16, 16, 9)
    before = [t.cpu().clone() for t in cache.dev]
    x = torch.zeros((0, 3, d), device=cuda())
    cu, kv = torch.zeros(3, dtype=torch.int32), torch.tensor([3, 0], dtype=torch.int32)
    out, status = append(cache, x, 1, cu, kv, lr.RopeFreqs(d))
    assert out.shape == (0, 1, d) and status == 0
    ws = lr.ChunkWorkspace(1, 1, 1, 1, 64)
    K, V = lr.libraspec_kv_read_q8_paged(*cache.dev, *cache.dev_table, cu.to(cuda()), kv.to(cuda()), 0, ws)
    assert K.shape == V.shape == (0, 1, d)
    one = torch.ones(d, device=cuda())
    y = lr.libraspec_qk_norm_rope(x, 1, lr.QkNorm(one, one), torch.zeros(0, dtype=torch.int32, device=cuda()), lr.RopeFreqs(d))
    assert y.shape == x.shape
    assert all(torch.equal(a.cpu().view(torch.uint8), b.view(torch.uint8)) for a, b in zip(cache.dev, before))
