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


def _opts(cap=0.0, window=0, slopes=None, first=None, prefix=None):
    return ctypes.byref(lr._ScoreOpts(cap, window, slopes, first, prefix))


def test_chunk_attn_q8_refuses(lib):
    big = 1 << 40

    def dense(Q=FAKE, K8=FAKE, V8=FAKE, Ks=FAKE, Vs=FAKE, cu=FAKE, kv=FAKE, T=4, B=2, Hq=8, Hkv=2, d=64, S=64, block=16,
              scale=0.125, opts=None, sinks=0, O=FAKE, lse=None, ws=FAKE, wb=big):
        return lib.libraspec_chunk_attn_q8(Q, K8, V8, Ks, Vs, cu, kv, T, B, Hq, Hkv, d, S, block, scale, opts, sinks, O, lse, ws,
                                           wb, None)

    for kw in (dict(d=96), dict(block=8), dict(block=48)):
        assert dense(**kw) == lr.EUNSUPPORTED, kw
    for kw in (dict(Q=None), dict(K8=None), dict(V8=None), dict(Ks=None), dict(Vs=None), dict(cu=None), dict(kv=None),
               dict(O=None), dict(T=-1), dict(B=-1), dict(B=4097), dict(Hq=7), dict(Hkv=0), dict(Hq=258, Hkv=2), dict(S=0),
               dict(S=72), dict(scale=0.0), dict(scale=math.inf), dict(Q=P(0x10008)), dict(K8=P(0x10008)), dict(O=P(0x10008)),
               dict(ws=None), dict(ws=P(0x10010)), dict(wb=1 << 16), dict(opts=_opts(cap=-1.0)), dict(opts=_opts(window=-1)),
               dict(sinks=-1), dict(sinks=(1 << 20) + 1, opts=_opts(window=5)), dict(sinks=1, opts=_opts(window=5, first=0x10000)),
               dict(opts=_opts(first=0x10001))):
        assert dense(**kw) == lr.EINVAL, kw
    assert dense(T=0, Q=None) == lr.OK and dense(B=0, Q=None) == lr.OK

    def paged(table=FAKE, mp=4, ps=32, np_=9, block=16):
        return lib.libraspec_chunk_attn_q8_paged(FAKE, FAKE, FAKE, FAKE, FAKE, table, mp, ps, np_, FAKE, FAKE, 4, 2, 8, 2, 64,
                                                 block, 0.125, None, 0, FAKE, None, None, 0, None)

    for kw in (dict(), dict(table=None), dict(mp=0), dict(ps=0), dict(ps=48, block=32), dict(ps=24), dict(np_=0),
               dict(mp=1 << 20, ps=1 << 12)):
        assert paged(**kw) == lr.EINVAL, kw  # (the first: no workspace)


def test_sink_attn_refuses(lib):
    def dense(K=FAKE, S=64, opts=None, sinks=4, ws=FAKE, wb=1 << 40, d=64):
        return lib.libraspec_sink_attn(FAKE, K, FAKE, FAKE, FAKE, 4, 2, 8, 2, d, S, 0.125, opts, sinks, FAKE, None, ws, wb, None)

    assert dense(d=96) == lr.EUNSUPPORTED
    for kw in (dict(K=None), dict(S=0), dict(sinks=-1), dict(sinks=(1 << 20) + 1), dict(opts=_opts(window=5, first=0x10000)),
               dict(ws=None), dict(wb=1 << 10), dict(opts=_opts(window=-2))):
        assert dense(**kw) == lr.EINVAL, kw
    assert lib.libraspec_sink_attn_paged(FAKE, FAKE, FAKE, FAKE, 4, 24, 9, FAKE, FAKE, 4, 2, 8, 2, 64, 0.125, None, 4, FAKE, None,
                                         FAKE, 1 << 40, None) == lr.EUNSUPPORTED


def test_limits_match_the_header():
    import os
    import re

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    header = open(os.path.join(root, "include", "libraspec.h")).read()
    call = open(os.path.join(root, "paper_2608_08721_gb300", "csrc", "chunk_call.h")).read()
    shift = re.search(r"LIBRASPEC_MAX_SINKS \(1 << (\d+)\)", header).group(1)
    assert re.search(r"kChunkMaxSinks = 1 << (\d+);", call).group(1) == shift


@pytest.mark.gpu
def test_binding_names_what_is_wrong_with_a_cache():
    dev = torch.device("cuda", 0)
    codes, exps = torch.zeros((2, 1, 64, 64), dtype=torch.float8_e4m3fn, device=dev), torch.zeros((2, 1, 4), dtype=torch.uint8, device=dev)
    table = torch.zeros((2, 1), dtype=torch.int32, device=dev)
    check = lr._check_caches_q8
    assert check(codes, codes, exps, exps, None, 2) == (1, 64, 64, 0, 0, 0, 16)
    assert check(codes, codes, exps, exps, table, 2) == (1, 64, 0, 1, 64, 2, 16)
    for args, error, match in (((codes.view(torch.uint8), codes, exps, exps, None, 2), TypeError, "^K8 must be"),
                               ((codes[0], codes, exps, exps, None, 2), ValueError, "^K8 must be"),
                               ((codes, codes[:1], exps, exps, None, 2), ValueError, "^V8 must have"),
                               ((codes, codes.transpose(2, 3), exps, exps, None, 2), ValueError, "^V8 must be contiguous"),
                               ((codes, codes, exps.float(), exps, None, 2), TypeError, "^Ks must be"),
                               ((codes, codes, exps, exps.cpu(), None, 2), ValueError, "^Vs must be on"),
                               ((codes, codes, exps[:, :, :0], exps[:, :, :0], None, 2), ValueError, "^Ks must be"),
                               ((codes, codes, exps[:, :, :3].contiguous(), exps[:, :, :3].contiguous(), None, 2), ValueError, "^Ks must be"),
                               ((codes, codes, exps, exps, None, 3), ValueError, "^K8 must be"),
                               ((codes, codes, exps, exps, table[0], 2), ValueError, "^block_table must be"),
                               ((codes, codes, exps, exps, table.long(), 2), TypeError, "^block_table must be"),
                               ((None, codes, exps, exps, None, 2), TypeError, "^K8 must be")):
        with pytest.raises(error, match=match):
            check(*args)
    norm = lr.QkNorm(torch.ones(64, device=dev), torch.ones(64, device=dev))
    x, pos = torch.zeros((3, 2, 128), device=dev), torch.zeros(3, dtype=torch.int32, device=dev)
    with pytest.raises(ValueError, match="^norm: weights of 64"):
        lr.libraspec_qk_norm_rope(x, 1, norm, pos, lr.RopeFreqs(128))
    with pytest.raises(ValueError, match="^n_q must lie"):
        lr.libraspec_qk_norm_rope(x[..., :64].contiguous(), 3, norm, pos, lr.RopeFreqs(64))


@pytest.mark.gpu
def test_tensors_of_another_device_are_refused(monkeypatch):
    """A call launches on the current device; with tensors of another it is refused, before anything is enqueued."""
    from helpers import cuda

    d, Hq, Hkv, B, S, T = 64, 4, 2, 1, 64, 2
    z = dict(device=cuda())
    X, pos = torch.zeros((T, Hq + 2 * Hkv, d), **z), torch.zeros(T, dtype=torch.int32, **z)
    K8, V8 = [torch.zeros((B, Hkv, S, d), dtype=torch.uint8, **z).view(torch.float8_e4m3fn) for _ in "KV"]
    Ks, Vs = [torch.zeros((B, Hkv, S // 16), dtype=torch.uint8, **z) for _ in "KV"]
    Kc, Vc = [torch.zeros((B, Hkv, S, d), dtype=torch.bfloat16, **z) for _ in "KV"]
    cu, kv = torch.tensor([0, T], dtype=torch.int32, **z), torch.zeros(B, dtype=torch.int32, **z)
    one, Q = torch.ones(d, **z), torch.zeros((T, Hq, d), dtype=torch.bfloat16, **z)
    norm, freqs, ws = lr.QkNorm(one, one), lr.RopeFreqs(d), lr.ChunkWorkspace(T, B, Hq, Hkv, d)
    calls = [lambda: lr.libraspec_qk_norm_rope(X, Hq, norm, pos, freqs),
             lambda: lr.libraspec_rope_append_q8(X[:, :Hq], X[:, Hq:Hq + Hkv], X[:, Hq + Hkv:], K8, V8, Ks, Vs, cu, kv, freqs,
                                                 ws, norm=norm),
             lambda: lr.libraspec_kv_read_q8(K8, V8, Ks, Vs, cu, kv, T, ws),
             lambda: lr.libraspec_chunk_attn_q8(Q, K8, V8, Ks, Vs, cu, kv, ws),
             lambda: lr.libraspec_sink_attn(Q, Kc, Vc, cu, kv, ws, window=8, sinks=1)]
    for call in calls:
        call()
    torch.cuda.synchronize()
    assert lr.libraspec_get_status(ws) == 0
    monkeypatch.setattr(torch.cuda, "current_device", lambda: cuda().index + 1)
    for call in calls:
        with pytest.raises(ValueError, match="current device"):
            call()
