"""The prompt calls' refusals (no GPU needed: nothing is enqueued) and the rotary frequencies."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2608_08721_gb300 import binding as lr

P = ctypes.c_void_p
FAKE = P(0x10000)  # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    from paper_2608_08721_gb300 import build

    build.build()
    return lr.load()


@pytest.mark.parametrize("rule", [dict(), dict(scaling="linear", factor=8.0), dict(scaling="ntk", factor=4.0),
                                  dict(scaling="parts", factor=4.0, original_len=8192.0, low=1.0, high=4.0)])
def test_frequencies_in_turns(lib, rule):
    """Two floats hold 48 bits of the frequency (theta^x itself is good to a few ulp of 64 bits)."""
    rot, theta = 128, 500000.0
    got = lr.RopeFreqs(rot, theta=theta, device="cpu", **rule).turns.double().numpy()
    s = rule.get("factor", 1.0)
    base = theta * s ** (rot / (rot - 2.0)) if rule.get("scaling") == "ntk" else theta
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot)
        if rule.get("scaling") == "linear":
            f /= s
        if rule.get("scaling") == "parts":
            turns = 8192.0 * f / (2 * math.pi)
            k = 0.0 if turns <= 1 else 1.0 if turns >= 4 else (turns - 1) / 3
            f = (1 - k) * f / s + k * f
        assert abs(got[i].sum() * 2 * math.pi - f) <= 2.0 ** -46 * f
        assert got[i, 0] == np.float32(got[i].sum())


def test_frequencies_refuse(lib):
    out = torch.empty((256, 2))
    f = lib.libraspec_rope_frequencies
    ok = (64, 10000.0, 0, 1.0, 1.0, 32.0, 0.0, out.data_ptr())
    assert f(*ok) == lr.OK
    for i, v, rc in [(0, 63, lr.EINVAL), (0, 0, lr.EINVAL), (0, 514, lr.EINVAL), (1, 0.0, lr.EINVAL),
                     (1, math.nan, lr.EINVAL), (1, math.inf, lr.EINVAL), (2, 4, lr.EUNSUPPORTED),
                     (2, -1, lr.EUNSUPPORTED), (7, None, lr.EINVAL)]:
        a = list(ok)
        a[i] = v
        assert f(*a) == rc, (i, v)
    assert f(64, 1e4, 1, 0.0, 0, 0, 0, out.data_ptr()) == lr.EINVAL           # no factor
    assert f(2, 1e4, 2, 4.0, 0, 0, 0, out.data_ptr()) == lr.EINVAL            # the exponent rot / (rot - 2)
    assert f(64, 1e4, 3, 4.0, 2.0, 2.0, 8192.0, out.data_ptr()) == lr.EINVAL  # an empty ramp
    assert f(64, 1e4, 3, 4.0, 1.0, 2.0, 0.0, out.data_ptr()) == lr.EINVAL
    with pytest.raises(ValueError, match="scaling"):
        lr.RopeFreqs(64, scaling="other", device="cpu")
    with pytest.raises(lr.LibraspecError):
        lr.RopeFreqs(63, device="cpu")


def test_rope_refuses(lib):
    def call(X=FAKE, xs=512, pos=FAKE, turns=FAKE, T=4, H=8, d=64, rot=64, Y=FAKE, ys=512, fn="libraspec_rope"):
        return getattr(lib, fn)(X, xs, pos, turns, 1.0, T, H, d, rot, 0, 0, Y, ys, None)

    for kw in (dict(X=None), dict(pos=None), dict(turns=None), dict(Y=None), dict(xs=511), dict(ys=511), dict(T=-1),
               dict(H=0), dict(d=63, rot=62), dict(rot=63), dict(rot=66), dict(rot=0), dict(X=P(0x10002)),
               dict(pos=P(0x10002)), dict(turns=P(0x10004)), dict(xs=600)):  # (the last: in place, another stride)
        assert call(**kw) == lr.EINVAL, kw
    assert call(X=P(0x10001), fn="libraspec_rope_bf16") == lr.EINVAL
    assert call(T=0, X=None, Y=None) == lr.OK


@pytest.mark.parametrize("kind", ["", "_bf16"])
def test_append_refuses(lib, kind):
    def dense(Q=FAKE, K=FAKE, V=FAKE, cu=FAKE, kv=FAKE, turns=FAKE, T=4, B=2, Hq=8, Hkv=2, d=64, rot=64, Qo=FAKE,
              Kc=FAKE, Vc=FAKE, S=64, ws=FAKE, wb=256, qs=512, ks=128):
        return getattr(lib, "libraspec_rope_append" + kind)(Q, qs, K, ks, V, 128, cu, kv, None, turns, 1.0, T, B, Hq, Hkv,
                                                            d, rot, 0, Qo, Kc, Vc, S, ws, wb, None)

    assert dense(d=96, rot=96) == lr.EUNSUPPORTED
    for kw in (dict(K=None), dict(V=None), dict(Q=None), dict(Qo=None), dict(cu=None), dict(kv=None), dict(turns=None),
               dict(Kc=None), dict(Vc=P(0x10008)), dict(ws=None), dict(wb=255), dict(ws=P(0x10010)), dict(T=-1), dict(B=-1),
               dict(B=5000), dict(Hkv=0), dict(qs=511), dict(ks=127), dict(S=0), dict(rot=65)):
        assert dense(**kw) == lr.EINVAL, kw
    assert dense(T=0, K=None) == lr.OK and dense(B=0, K=None) == lr.OK

    def paged(table=FAKE, mp=4, ps=16, np_=9):
        return getattr(lib, "libraspec_rope_append_paged" + kind)(FAKE, 512, FAKE, 128, FAKE, 128, FAKE, FAKE, None, FAKE,
                                                                  1.0, 4, 2, 8, 2, 64, 64, 0, FAKE, FAKE, None, table, mp,
                                                                  ps, np_, FAKE, 256, None)

    for kw in (dict(), dict(table=None), dict(mp=0), dict(ps=0), dict(np_=0), dict(mp=1 << 20, ps=1 << 12)):
        assert paged(**kw) == lr.EINVAL, kw  # (the first: no value pool)


def test_chunk_attn_refuses(lib):
    big = 1 << 40

    def dense(Q=FAKE, K=FAKE, V=FAKE, cu=FAKE, kv=FAKE, T=4, B=2, Hq=8, Hkv=2, d=64, S=64, scale=0.125, opts=None, O=FAKE,
              lse=None, ws=FAKE, wb=big):
        return lib.libraspec_chunk_attn(Q, K, V, cu, kv, T, B, Hq, Hkv, d, S, scale, opts, O, lse, ws, wb, None)

    def opts(cap=0.0, window=0, slopes=None, first=None, prefix=None):
        return ctypes.byref(lr._ScoreOpts(cap, window, slopes, first, prefix))

    assert dense(d=96) == lr.EUNSUPPORTED
    for kw in (dict(Q=None), dict(K=None), dict(V=None), dict(cu=None), dict(kv=None), dict(O=None), dict(T=-1), dict(B=-1),
               dict(B=4097), dict(Hq=7), dict(Hkv=0), dict(Hq=258, Hkv=2), dict(S=0), dict(scale=0.0), dict(scale=math.nan),
               dict(scale=math.inf), dict(Q=P(0x10008)), dict(K=P(0x10008)), dict(O=P(0x10008)), dict(lse=P(0x10002)),
               dict(ws=None), dict(ws=P(0x10010)), dict(wb=1 << 16), dict(opts=opts(cap=-1.0)),
               dict(opts=opts(cap=math.nan)), dict(opts=opts(window=-1)), dict(opts=opts(first=0x10001)),
               dict(opts=opts(slopes=0x10002)), dict(opts=opts(prefix=0x10003))):
        assert dense(**kw) == lr.EINVAL, kw
    assert dense(T=0, Q=None) == lr.OK and dense(B=0, Q=None) == lr.OK

    def paged(table=FAKE, mp=4, ps=16, np_=9):
        return lib.libraspec_chunk_attn_paged(FAKE, FAKE, FAKE, table, mp, ps, np_, FAKE, FAKE, 4, 2, 8, 2, 64, 0.125,
                                              None, FAKE, None, None, 0, None)

    assert paged(ps=24) == lr.EUNSUPPORTED
    for kw in (dict(), dict(table=None), dict(mp=0), dict(ps=0), dict(np_=0), dict(mp=1 << 20, ps=1 << 12)):
        assert paged(**kw) == lr.EINVAL, kw  # (the first: no workspace)


def test_chunk_workspace_size(lib):
    f = lib.libraspec_chunk_workspace_size
    s = f(8192, 64, 32, 8, 128)
    assert s > 0 and s % 256 == 0 and 0 < f(1, 1, 8, 2, 64) < s
    assert f(-1, 1, 8, 2, 64) == f(1, 4097, 8, 2, 64) == f(1, 1, 7, 2, 64) == f(1, 1, 8, 2, 96) == 0


def test_binding_names_what_is_wrong():
    x = torch.zeros((4, 8, 64))
    with pytest.raises(TypeError, match="^Q must be"):
        lr.libraspec_chunk_attn(x, x, x, x, x, None)
    with pytest.raises(ValueError, match="^X must be on a CUDA device"):
        lr.libraspec_rope(x, x, None)
    with pytest.raises(TypeError, match="^K must be"):
        lr.libraspec_rope_append(None, x.half(), x, x, x, x, x, None, None)


def test_frequencies_that_no_float_holds_are_refused(lib):
    out = torch.empty((32, 2))
    f = lib.libraspec_rope_frequencies
    assert f(64, 1e-30, 0, 1.0, 1.0, 32.0, 0.0, out.data_ptr()) == lr.OK and bool(torch.isfinite(out).all())
    assert f(64, 1e-300, 0, 1.0, 1.0, 32.0, 0.0, out.data_ptr()) == lr.EINVAL
    assert f(64, 10000.0, 1, 1e-300, 1.0, 32.0, 0.0, out.data_ptr()) == lr.EINVAL
