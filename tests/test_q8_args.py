"""Refusals of the calls around the cache in 8 bits and of the norm with rotation (no GPU needed: nothing is enqueued)."""
import ctypes
import math

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


@pytest.mark.parametrize("kind", ["", "_bf16"])
def test_norm_rope_refuses(lib, kind):
    def call(X=FAKE, xs=640, pos=FAKE, turns=FAKE, wq=FAKE, wk=FAKE, eps=1e-6, T=4, Hq=8, Hk=2, d=64, rot=64, Y=FAKE, ys=640):
        return getattr(lib, "libraspec_qk_norm_rope" + kind)(X, xs, pos, turns, 1.0, wq, wk, eps, T, Hq, Hk, d, rot, 0, Y, ys,
                                                             None)

    for kw in (dict(X=None), dict(pos=None), dict(turns=None), dict(Y=None), dict(wq=None), dict(wk=None), dict(xs=639),
               dict(ys=639), dict(T=-1), dict(Hq=0, Hk=0), dict(Hq=-1), dict(Hk=-1), dict(Hq=1 << 21), dict(d=63, rot=62),
               dict(d=514, rot=64, xs=5140, ys=5140), dict(rot=63), dict(rot=66), dict(rot=0), dict(X=P(0x10001)),
               dict(pos=P(0x10002)), dict(turns=P(0x10004)), dict(wq=P(0x10002)), dict(wk=P(0x10001)), dict(eps=-1e-9),
               dict(eps=math.nan), dict(eps=math.inf), dict(xs=700)):  # (the last: in place, another stride)
        assert call(**kw) == lr.EINVAL, kw
    assert call(T=0, X=None, Y=None) == lr.OK


@pytest.mark.parametrize("kind", ["", "_bf16"])
def test_append_refuses(lib, kind):
    def dense(Q=FAKE, K=FAKE, V=FAKE, cu=FAKE, kv=FAKE, turns=FAKE, wq=None, wk=None, eps=0.0, T=4, B=2, Hq=8, Hkv=2, d=64,
              rot=64, Qo=FAKE, K8=FAKE, V8=FAKE, Ks=FAKE, Vs=FAKE, S=64, block=16, ws=FAKE, wb=256, qs=512, ks=128):
        return getattr(lib, "libraspec_rope_append_q8" + kind)(
            Q, qs, K, ks, V, 128, cu, kv, None, turns, 1.0, wq, wk, eps, T, B, Hq, Hkv, d, rot, 0, Qo, K8, V8, Ks, Vs, S, block,
            ws, wb, None)

    for kw in (dict(d=96, rot=96), dict(block=8), dict(block=48), dict(block=0), dict(block=128)):
        assert dense(**kw) == lr.EUNSUPPORTED, kw
    for kw in (dict(K=None), dict(V=None), dict(Q=None), dict(Qo=None), dict(cu=None), dict(kv=None), dict(turns=None),
               dict(K8=None), dict(V8=P(0x10008)), dict(Ks=None), dict(Vs=None), dict(ws=None), dict(wb=255),
               dict(ws=P(0x10010)), dict(T=-1), dict(B=-1), dict(B=5000), dict(Hkv=0), dict(qs=511), dict(ks=127), dict(S=0),
               dict(S=72), dict(rot=65), dict(wq=FAKE), dict(wk=FAKE), dict(wq=P(0x10002), wk=FAKE), dict(eps=-1.0),
               dict(wq=FAKE, wk=FAKE, eps=math.nan)):
        assert dense(**kw) == lr.EINVAL, kw
    assert dense(T=0, K=None) == lr.OK and dense(B=0, K=None) == lr.OK

    def paged(table=FAKE, mp=4, ps=32, np_=9, block=16, V8=None):
        return getattr(lib, "libraspec_rope_append_q8_paged" + kind)(
            FAKE, 512, FAKE, 128, FAKE, 128, FAKE, FAKE, None, FAKE, 1.0, None, None, 0.0, 4, 2, 8, 2, 64, 64, 0, FAKE, FAKE, V8,
            FAKE, FAKE, table, mp, ps, np_, block, FAKE, 256, None)

    for kw in (dict(), dict(V8=FAKE, table=None), dict(V8=FAKE, mp=0), dict(V8=FAKE, ps=0), dict(V8=FAKE, np_=0),
               dict(V8=FAKE, ps=48, block=32), dict(V8=FAKE, mp=1 << 20, ps=1 << 12)):
        assert paged(**kw) == lr.EINVAL, kw  # (the first: no value codes)


def test_read_refuses(lib):
    def dense(K8=FAKE, V8=FAKE, Ks=FAKE, Vs=FAKE, cu=FAKE, start=FAKE, T=4, B=2, Hkv=2, d=64, S=64, block=16, K=FAKE, V=FAKE,
              ws=FAKE, wb=256):
        return lib.libraspec_kv_read_q8(K8, V8, Ks, Vs, cu, start, T, B, Hkv, d, S, block, K, V, ws, wb, None)

    for kw in (dict(d=96), dict(block=20)):
        assert dense(**kw) == lr.EUNSUPPORTED, kw
    for kw in (dict(K8=None), dict(V8=P(0x10004)), dict(Ks=None), dict(Vs=None), dict(cu=None), dict(start=None),
               dict(K=None), dict(V=P(0x10008)), dict(T=-1), dict(B=4097), dict(Hkv=0), dict(S=40), dict(ws=None),
               dict(wb=16)):
        assert dense(**kw) == lr.EINVAL, kw
    assert dense(T=0, K8=None) == lr.OK and dense(B=0, K8=None) == lr.OK

    def paged(table=FAKE, mp=4, ps=32, np_=9, block=16, K=None):
        return lib.libraspec_kv_read_q8_paged(FAKE, FAKE, FAKE, FAKE, table, mp, ps, np_, FAKE, FAKE, 4, 2, 2, 64, block, K,
                                              FAKE, FAKE, 256, None)

    for kw in (dict(), dict(K=FAKE, table=None), dict(K=FAKE, mp=0), dict(K=FAKE, ps=48, block=32), dict(K=FAKE, np_=0)):
        assert paged(**kw) == lr.EINVAL, kw


def test_binding_names_what_is_wrong():
    x = torch.zeros((4, 8, 64))
    with pytest.raises(ValueError, match="^q_weight must be on a CUDA device"):
        lr.QkNorm(torch.ones(64), torch.ones(64))
    with pytest.raises(TypeError, match="^k_weight|^q_weight"):
        lr.QkNorm(torch.ones(64).half(), torch.ones(64))
    with pytest.raises(ValueError, match="^X must be on a CUDA device"):
        lr.libraspec_qk_norm_rope(x, 4, None, x, None)
    with pytest.raises(TypeError, match="^K must be"):
        lr.libraspec_rope_append_q8(None, x.half(), x, x, x, x, x, x, x, None, None)
    with pytest.raises(TypeError, match="^start must be|^kv_len must be"):
        lr.libraspec_kv_read_q8(x, x, x, x, x, x, 4, None)
