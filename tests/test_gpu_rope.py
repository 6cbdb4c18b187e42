"""GPU: rotary positions (libraspec_rope) and the append of a ragged chunk with the rotation on the way
(libraspec_rope_append[_paged]) against the definition in 64 bits.

Tolerances, from the arithmetic: the angle is known to 2^-24 of a turn (3.8e-7 rad), sine and cosine to 2 ulp, the two
products and their sum round once each in binary32: below 4e-6 of the pair's length. A bf16 result adds half a unit of
8 significant bits, 2^-8 of the value.
"""
import math

import numpy as np
import pytest
import torch

from helpers import cuda
from paper_2608_08721_gb300 import binding as lr

pytestmark = pytest.mark.gpu


def freqs64(rot, theta=10000.0, scaling="none", factor=1.0, original_len=0.0, low=1.0, high=32.0):
    if scaling == "ntk":
        theta = theta * factor ** (rot / (rot - 2))
    f = np.array([theta ** (-2.0 * i / rot) for i in range(rot // 2)])
    if scaling == "linear":
        f = f / factor
    if scaling == "parts":
        k = np.clip((original_len * f / (2 * math.pi) - low) / (high - low), 0, 1)
        f = (1 - k) * f / factor + k * f
    return f


def rotate64(x, pos, f, inter, magnitude=1.0, inverse=False):
    """x [T, H, d] float64 (CPU), pos [T]; returns (rotated, length of each element's pair)."""
    half = len(f)
    a = torch.from_numpy(np.asarray(pos, np.float64)[:, None] * f)[:, None]
    c, s = torch.cos(a), torch.sin(a) * (-1.0 if inverse else 1.0)
    i0 = torch.arange(half) * 2 if inter else torch.arange(half)
    i1 = i0 + 1 if inter else i0 + half
    y, r = x.clone(), torch.zeros_like(x)
    y[..., i0] = magnitude * (x[..., i0] * c - x[..., i1] * s)
    y[..., i1] = magnitude * (x[..., i0] * s + x[..., i1] * c)
    r[..., i0] = r[..., i1] = magnitude * torch.hypot(x[..., i0], x[..., i1])
    return y, r


def assert_rotated(got, want, length, bf16):
    bound = 4e-6 * length + (2.0 ** -8 * 1.001 * want.abs() if bf16 else 0.0)
    err = (got.double().cpu() - want).abs()
    assert bool((err <= bound).all()), "max %.3e over the bound by %.3e" % (err.max(), (err - bound).max())


@pytest.mark.parametrize("d,rot,H,T", [(128, 128, 32, 64), (64, 64, 8, 1), (128, 64, 7, 33), (128, 24, 3, 19),
                                       (64, 58, 2, 5), (128, 2, 1, 3), (256, 256, 5, 9), (36, 20, 3, 11)])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rope(d, rot, H, T, inter, dtype):
    g = torch.Generator().manual_seed(d * rot + H)
    x = torch.randn((T, H, d), generator=g).to(dtype)
    pos = torch.randint(0, 131072, (T,), generator=g, dtype=torch.int32)
    pos[0] = 0
    y = lr.libraspec_rope(x.to(cuda()), pos.to(cuda()), lr.RopeFreqs(rot), interleaved=inter)
    want, length = rotate64(x.double(), pos.numpy(), freqs64(rot), inter)
    assert_rotated(y, want, length, dtype == torch.bfloat16)
    assert torch.equal(y[..., rot:].cpu(), x[..., rot:])


@pytest.mark.parametrize("rule", [dict(scaling="linear", factor=8.0), dict(scaling="ntk", factor=4.0),
                                  dict(scaling="parts", factor=4.0, original_len=8192.0, low=1.0, high=4.0),
                                  dict(scaling="parts", factor=16.0, original_len=4096.0)])
def test_rope_scaled_frequencies_and_magnitude(rule):
    g = torch.Generator().manual_seed(5)
    x = torch.randn((40, 4, 64), generator=g)
    pos = torch.randint(0, 131072, (40,), generator=g, dtype=torch.int32)
    fr = lr.RopeFreqs(64, theta=500000.0, magnitude=1.25, **rule)
    y = lr.libraspec_rope(x.to(cuda()), pos.to(cuda()), fr)
    want, length = rotate64(x.double(), pos.numpy(), freqs64(64, 500000.0, **rule), False, 1.25)
    assert_rotated(y, want, length, False)


def test_rope_positions_beyond_24_bits_and_negative():
    pos = torch.tensor([2**24 + 1, 2**31 - 1, 2**30 + 12345, -1, -70000, -(2**31)], dtype=torch.int32)
    x = torch.randn((6, 2, 128), generator=torch.Generator().manual_seed(1))
    y = lr.libraspec_rope(x.to(cuda()), pos.to(cuda()), lr.RopeFreqs(128))
    # (the frequencies as two floats hold 48 bits: at 2^31 the first pair's angle is known to 2^-18 turns = 2.4e-5 rad)
    want, length = rotate64(x.double(), pos.numpy(), freqs64(128), False)
    assert bool(((y.double().cpu() - want).abs() <= 3e-5 * length).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("offset", [0, 1])
def test_rope_strided_in_place_and_unaligned(dtype, inter, offset):
    """The keys' part of a wider projection, rotated in place: the rest of the row stays; also at an odd offset."""
    g = torch.Generator().manual_seed(3)
    T, H, d, width = 21, 4, 64, 11 * 64 + 3
    buf = torch.randn((T, width), generator=g).to(dtype)
    dev = buf.to(cuda())
    view = dev[:, 128 + offset:128 + offset + H * d].unflatten(1, (H, d))
    x = buf[:, 128 + offset:128 + offset + H * d].unflatten(1, (H, d)).double()
    pos = torch.arange(7, 7 + T, dtype=torch.int32)
    out = lr.libraspec_rope(view, pos.to(cuda()), lr.RopeFreqs(d), interleaved=inter, Y=view)
    assert out is view
    want, length = rotate64(x, pos.numpy(), freqs64(d), inter)
    assert_rotated(view, want, length, dtype == torch.bfloat16)
    same = torch.ones(width, dtype=torch.bool)
    same[128 + offset:128 + offset + H * d] = False
    assert torch.equal(dev.cpu()[:, same], buf[:, same])


@pytest.mark.parametrize("inter", [False, True])
def test_rope_inverse_is_the_gradient(inter):
    """y = R x: the gradient of sum(w y) is R^T w, by the formula and by differences of the forward pass."""
    g = torch.Generator().manual_seed(9)
    T, H, d, rot = 5, 2, 64, 32
    x, w = torch.randn((T, H, d), generator=g), torch.randn((T, H, d), generator=g)
    pos = torch.tensor([0, 1, 77, 4096, 131071], dtype=torch.int32)
    fr = lr.RopeFreqs(rot, magnitude=1.5)
    grad = lr.libraspec_rope(w.to(cuda()), pos.to(cuda()), fr, interleaved=inter, inverse=True)
    want, length = rotate64(w.double(), pos.numpy(), freqs64(rot), inter, 1.5, inverse=True)
    assert_rotated(grad, want, length, False)
    for k in range(d):  # the map is linear: a step of 1 along element k has no error but rounding
        step = torch.zeros_like(x)
        step[..., k] = 1.0
        diff = (lr.libraspec_rope((x + step).to(cuda()), pos.to(cuda()), fr, interleaved=inter).double()
                - lr.libraspec_rope(x.to(cuda()), pos.to(cuda()), fr, interleaved=inter).double()).cpu()
        dot = (diff * w.double()).sum(dim=-1)
        # two results of pairs of length below 8, each off by 4e-6 of it, times the two weights of the pair
        assert bool(((dot - grad[..., k].double().cpu()).abs() <= 2 * 8 * 4e-6 * 2 * w.abs().max()).all())


def _chunk(n, kv, Hq, Hkv, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    T = int(sum(n))
    qkv = torch.randn((T, Hq + 2 * Hkv, d), generator=g).to(dtype)
    cu = torch.from_numpy(np.concatenate([[0], np.cumsum(n)]).astype(np.int32))
    return qkv, cu, torch.tensor(kv, dtype=torch.int32), g


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("Hq,Hkv,d,rot,inter,page", [(32, 8, 128, 128, False, 0), (28, 4, 128, 64, True, 16),
                                                    (8, 2, 64, 24, False, 128), (8, 8, 64, 58, True, 20),
                                                    (16, 2, 128, 122, False, 256)])
def test_rope_append(dtype, Hq, Hkv, d, rot, inter, page):
    n, kv = [1, 37, 0, 5, 130], [100, 0, 50, 299, 15]
    qkv, cu, kvl, g = _chunk(n, kv, Hq, Hkv, d, dtype, Hq + page)
    B, S = len(n), 320
    fr = lr.RopeFreqs(rot, theta=500000.0)
    table = None
    if page:
        per = (S + page - 1) // page
        table = torch.randperm(B * per + 2, generator=g)[:B * per].view(B, per).to(torch.int32)
        shape = (B * per + 2, Hkv, page, d)
    else:
        shape = (B, Hkv, S, d)
    Kc, Vc = (torch.randn(shape, generator=g).to(torch.bfloat16) for _ in range(2))
    wantK, wantV = Kc.double(), Vc.double()
    Kd, Vd = Kc.to(cuda()), Vc.to(cuda())
    dev = qkv.to(cuda())
    q, k, v = dev[:, :Hq], dev[:, Hq:Hq + Hkv], dev[:, Hq + Hkv:]
    ws = lr.ChunkWorkspace(1, 1, 1, 1, 64)
    if page:
        Qo = lr.libraspec_rope_append_paged(q, k, v, Kd, Vd, table.to(cuda()), cu.to(cuda()), kvl.to(cuda()), fr, ws,
                                            interleaved=inter)
    else:
        Qo = lr.libraspec_rope_append(q, k, v, Kd, Vd, cu.to(cuda()), kvl.to(cuda()), fr, ws, interleaved=inter)
    torch.cuda.synchronize()
    assert lr.libraspec_get_status(ws) == 0
    pos = np.concatenate([np.arange(c, c + m) for m, c in zip(n, kv)])
    x = qkv.double()
    f = freqs64(rot, 500000.0)
    want, length = rotate64(x[:, :Hq], pos, f, inter)
    assert_rotated(Qo, want, length, True)
    k64, kl = rotate64(x[:, Hq:Hq + Hkv], pos, f, inter)
    bound = torch.zeros_like(wantK)
    at = 0
    for b in range(B):
        for j in range(n[b]):
            s = kv[b] + j
            i = (int(table[b, s // page]), slice(None), s % page) if page else (b, slice(None), s)
            wantK[i], wantV[i] = k64[at], qkv[at, Hq + Hkv:].to(torch.bfloat16).double()
            bound[i] = 4e-6 * kl[at] + 2.0 ** -8 * 1.001 * k64[at].abs()
            at += 1
    assert bool(((Kd.double().cpu() - wantK).abs() <= bound).all())  # (untouched rows: exactly)
    assert torch.equal(Vd.double().cpu(), wantV)


def test_rope_append_explicit_positions_and_no_queries():
    n, kv = [3, 2], [4, 0]
    qkv, cu, kvl, g = _chunk(n, kv, 0, 2, 64, torch.float32, 8)
    pos = torch.tensor([9, 0, 131071, 5, 6], dtype=torch.int32)
    Kd, Vd = (torch.zeros((2, 2, 8, 64), dtype=torch.bfloat16, device=cuda()) for _ in range(2))
    dev = qkv.to(cuda())
    ws = lr.ChunkWorkspace(1, 1, 1, 1, 64)
    assert lr.libraspec_rope_append(None, dev[:, :2], dev[:, 2:], Kd, Vd, cu.to(cuda()), kvl.to(cuda()),
                                    lr.RopeFreqs(64), ws, pos=pos.to(cuda())) is None
    want, length = rotate64(qkv[:, :2].double(), pos.numpy(), freqs64(64), False)
    assert_rotated(torch.cat([Kd[0, :, 4:7].transpose(0, 1), Kd[1, :, :2].transpose(0, 1)]), want, length, True)
    assert torch.equal(Vd[0, :, 4:7].transpose(0, 1).cpu(), qkv[:3, 2:].to(torch.bfloat16))
    assert lr.libraspec_get_status(ws) == 0


def test_rope_append_violations_set_status_and_write_nothing_else():
    g = torch.Generator().manual_seed(2)
    Hkv, d, page = 2, 64, 16
    fr, ws = lr.RopeFreqs(d), lr.ChunkWorkspace(1, 1, 1, 1, 64)
    x = torch.randn((6, 4 + 2 * Hkv, d), generator=g).to(torch.bfloat16).to(cuda())
    q, k, v = x[:, :4], x[:, 4:6], x[:, 6:]
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device=cuda())  # noqa: E731
    want, length = rotate64(q.double().cpu(), np.array([14, 15, 16, 3, 4, 5]), freqs64(d), False)
    # dense, capacity 16: the third token of sequence 0 does not fit; its query is rotated all the same
    Kd, Vd = (torch.zeros((2, Hkv, 16, d), dtype=torch.bfloat16, device=cuda()) for _ in range(2))
    Qo = lr.libraspec_rope_append(q, k, v, Kd, Vd, i32(0, 3, 6), i32(14, 3), fr, ws)
    assert lr.libraspec_get_status(ws) == lr.ST_KV_OVERFLOW
    assert_rotated(Qo, want, length, True)
    assert torch.equal(Vd[0, :, 14:16].transpose(0, 1), v[:2]) and torch.equal(Vd[1, :, 3:6].transpose(0, 1), v[3:])
    assert int((Vd != 0).any(dim=-1).sum()) == 5 * Hkv
    # a negative length, and a page outside the pool
    Kp, Vp = (torch.zeros((3, Hkv, page, d), dtype=torch.bfloat16, device=cuda()) for _ in range(2))
    table = torch.tensor([[0, 3], [1, -1]], dtype=torch.int32, device=cuda())
    lr.libraspec_rope_append_paged(q, k, v, Kp, Vp, table, i32(0, 3, 6), i32(14, -1), fr, ws)
    assert lr.libraspec_get_status(ws) == lr.ST_KV_OVERFLOW | lr.ST_BAD_PAGE
    assert torch.equal(Vp[0, :, 14:16].transpose(0, 1), v[:2]) and int((Vp != 0).any(dim=-1).sum()) == 2 * Hkv
    # offsets beyond the rows
    Qo = torch.zeros_like(q).contiguous()
    lr.libraspec_rope_append_paged(q, k, v, Kp, Vp, table, i32(0, 3, 9), i32(0, 0), fr, ws, Qo=Qo)
    assert lr.libraspec_get_status(ws) == lr.ST_BAD_LENGTH
    # rows of no sequence are left alone
    Qo.zero_()
    lr.libraspec_rope_append_paged(q, k, v, Kp, Vp, table, i32(1, 1, 2), i32(0, 0), fr, ws, Qo=Qo)
    assert lr.libraspec_get_status(ws) == 0 and (Qo != 0).any(-1).any(-1).tolist() == [False, True] + [False] * 4


def test_rope_append_many_sequences_on_another_stream():
    """More sequences than a CTA has threads, each with a token or none, on a stream of its own."""
    B, Hkv, d = 1500, 1, 64
    r = np.random.default_rng(4)
    n, kv = r.integers(0, 2, B).tolist(), r.integers(0, 60, B).tolist()
    qkv, cu, kvl, g = _chunk(n, kv, 1, Hkv, d, torch.bfloat16, 4)
    s = torch.cuda.Stream()
    dev, cud, kvd = qkv.to(cuda()), cu.to(cuda()), kvl.to(cuda())
    Kd, Vd = (torch.zeros((B, Hkv, 64, d), dtype=torch.bfloat16, device=cuda()) for _ in range(2))
    fr, ws = lr.RopeFreqs(d), lr.ChunkWorkspace(1, 1, 1, 1, 64)
    torch.cuda.synchronize()
    lr.libraspec_rope_append(dev[:, :1], dev[:, 1:2], dev[:, 2:], Kd, Vd, cud, kvd, fr, ws, stream=s)
    s.synchronize()
    seq = np.repeat(np.arange(B), n)
    pos = np.asarray(kv)[seq]
    want, length = rotate64(qkv[:, 1:2].double(), pos, freqs64(d), False)
    assert_rotated(Kd[seq, :, pos], want, length, True)
    assert torch.equal(Vd[seq, :, pos].cpu(), qkv[:, 2:])
    assert int((Vd != 0).any(-1).sum()) == len(seq) and lr.libraspec_get_status(ws) == 0


def _append_case(cu, B, dtype=torch.float32, T=6, S=16):
    """An append of T tokens into caches of B sequences (their lengths 2, 3, ...) under the offsets `cu`."""
    Hq, Hkv, d = 2, 2, 64
    x = torch.randn((T, Hq + 2 * Hkv, d), generator=torch.Generator().manual_seed(12)).to(dtype).to(cuda())
    Kd, Vd = (torch.zeros((B, Hkv, S, d), dtype=torch.bfloat16, device=cuda()) for _ in range(2))
    Qo = torch.zeros((T, Hq, d), dtype=torch.bfloat16, device=cuda())
    kvl = torch.arange(2, 2 + B, dtype=torch.int32, device=cuda())
    ws = lr.ChunkWorkspace(1, 1, 1, 1, d)
    lr.libraspec_rope_append(x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], Kd, Vd,
                             torch.tensor(cu, dtype=torch.int32, device=cuda()), kvl, lr.RopeFreqs(d), ws, Qo=Qo)
    return x.cpu(), Qo, Kd, Vd, lr.libraspec_get_status(ws)


@pytest.mark.parametrize("cu,good", [([-1, 2, 6], [1]), ([0, 3, 7], [0]), ([2, 1, 4], [1]),
                                     ([-(2**31), 2, 6], [1]), ([-(2**31) + 3, 6], []), ([0, 2**31 - 1, 6], [])])
def test_rope_append_skips_sequences_of_bad_offsets(cu, good):
    """Offsets below 0, past the rows, or running backwards: the status, and nothing of that sequence written, also
    where an index counted from such an offset would not fit 32 bits."""
    x, Qo, Kd, Vd, status = _append_case(cu, len(cu) - 1)
    assert status == lr.ST_BAD_LENGTH
    touched = torch.zeros(6, dtype=torch.bool)
    rows = torch.zeros((len(cu) - 1, 16), dtype=torch.bool)
    for b in good:
        n = cu[b + 1] - cu[b]
        touched[cu[b]:cu[b + 1]] = True
        rows[b, 2 + b:2 + b + n] = True
        want, length = rotate64(x[cu[b]:cu[b + 1], 2:4].double(), np.arange(2 + b, 2 + b + n), freqs64(64), False)
        assert_rotated(Kd[b, :, 2 + b:2 + b + n].transpose(0, 1), want, length, True)
    assert (Qo != 0).any(-1).any(-1).cpu().tolist() == touched.tolist()
    for c in (Kd, Vd):
        assert torch.equal((c != 0).any(-1).all(1).cpu(), rows) and torch.equal((c != 0).any(-1).any(1).cpu(), rows)


@pytest.mark.parametrize("T,B", [(6, 3), (3000, 3), (6, 1200)])
def test_rope_append_gives_a_row_of_two_sequences_to_the_first(T, B):
    """Offsets that decrease, and ranges on either side of it that overlap: each token has one row of the cache, and the
    position that belongs to it. One token a CTA and two; the second sequence looked up by another thread, and by the
    same one later."""
    cu = [0] * (B + 1)
    later = B - 1
    cu[1:later] = [4 * T // 6] * (later - 1)
    cu[later], cu[B] = T // 2, T   # sequence 0: [0, 4 T / 6), the one before the last runs backwards, the last: [T / 2, T)
    x, Qo, Kd, Vd, status = _append_case(cu, B, T=T, S=T + B + 2)
    assert status == lr.ST_BAD_LENGTH
    first = cu[1]
    for b, lo, hi in ((0, 0, first), (later, first, T)):
        pos = np.arange(lo, hi) - cu[b] + 2 + b
        want, length = rotate64(x[lo:hi].double(), pos, freqs64(64), False)
        assert_rotated(Qo[lo:hi], want[:, :2], length[:, :2], True)
        assert_rotated(Kd[b, :, pos].transpose(0, 1), want[:, 2:4], length[:, 2:4], True)
        assert torch.equal(Vd[b, :, pos].transpose(0, 1).cpu(), x[lo:hi, 4:].to(torch.bfloat16))
    assert int((Vd != 0).any(-1).sum()) == 2 * T


def test_host_memory_is_refused():
    """Frequencies and workspaces that were made on the host do not reach a kernel."""
    d = 64
    X = torch.zeros((4, 4, d), device=cuda(), dtype=torch.bfloat16)
    pos = torch.zeros(4, dtype=torch.int32, device=cuda())
    cu, kvl = torch.tensor([0, 4], dtype=torch.int32, device=cuda()), torch.zeros(1, dtype=torch.int32, device=cuda())
    Kd, Vd = (torch.zeros((1, 1, 8, d), dtype=torch.bfloat16, device=cuda()) for _ in range(2))
    fr, ws = lr.RopeFreqs(d), lr.ChunkWorkspace(4, 1, 2, 1, d)
    host_fr, host_ws = lr.RopeFreqs(d, device="cpu"), lr.ChunkWorkspace(4, 1, 2, 1, d, device="cpu")
    q, k, v = X[:, :2], X[:, 2:3], X[:, 3:]
    for call in (lambda: lr.libraspec_rope(X, pos, host_fr),
                 lambda: lr.libraspec_rope_append(q, k, v, Kd, Vd, cu, kvl, host_fr, ws),
                 lambda: lr.libraspec_rope_append(q, k, v, Kd, Vd, cu, kvl, fr, host_ws),
                 lambda: lr.libraspec_chunk_attn(q.contiguous(), Kd, Vd, cu, kvl, host_ws)):
        with pytest.raises(ValueError):
            call()
    torch.cuda.synchronize()
    assert int((Kd != 0).sum()) == 0 and lr.libraspec_get_status(ws) == 0
