"""The chunk calls' workspace: those over a bf16 cache do without what only those over a cache in 8 bits need."""
import ctypes

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


def test_sizes(lib):
    both, bf16 = lib.libraspec_chunk_workspace_size, lib.libraspec_chunk_workspace_size_bf16
    for T, B, Hq, Hkv, d in ((8192, 64, 32, 8, 128), (1, 1, 8, 2, 64), (300, 4096, 16, 1, 64), (0, 0, 1, 1, 128)):
        a, b = both(T, B, Hq, Hkv, d), bf16(T, B, Hq, Hkv, d)
        assert a % 256 == b % 256 == 0 and 0 < b
        assert T * Hq * (2 * d + 1) <= a - b < T * Hq * (2 * d + 1) + 512
    assert bf16(-1, 1, 8, 2, 64) == bf16(1, 4097, 8, 2, 64) == bf16(1, 1, 7, 2, 64) == bf16(1, 1, 8, 2, 96) == 0


def test_what_is_too_small_is_refused(lib):
    T, B, Hq, Hkv, d = 300, 2, 8, 2, 64
    big, small = lib.libraspec_chunk_workspace_size(T, B, Hq, Hkv, d), lib.libraspec_chunk_workspace_size_bf16(T, B, Hq, Hkv, d)
    sizes = (T, B, Hq, Hkv, d, 64)
    for n in (big - 1, small):
        assert lib.libraspec_chunk_attn_q8(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, *sizes, 16, 0.125, None, 0, FAKE, None, FAKE,
                                           n, None) == lr.EINVAL
    assert lib.libraspec_chunk_attn(FAKE, FAKE, FAKE, FAKE, FAKE, *sizes, 0.125, None, FAKE, None, FAKE, small - 1, None) == lr.EINVAL
    assert lib.libraspec_sink_attn(FAKE, FAKE, FAKE, FAKE, FAKE, *sizes, 0.125, None, 4, FAKE, None, FAKE, small - 1,
                                   None) == lr.EINVAL


@pytest.mark.gpu
def test_calls_over_a_bf16_cache_take_the_smaller_one():
    from helpers import cuda

    T, B, Hq, Hkv, d, S = 300, 3, 8, 2, 64, 2048
    g = torch.Generator(device=cuda()).manual_seed(1)
    Q = torch.randn((T, Hq, d), generator=g, device=cuda()).to(torch.bfloat16)
    Kc, Vc = (torch.randn((B, Hkv, S, d), generator=g, device=cuda()).to(torch.bfloat16) for _ in "KV")
    cu = torch.tensor([0, 200, 201, T], dtype=torch.int32, device=cuda())
    kv = torch.tensor([100, 2000, 700], dtype=torch.int32, device=cuda())
    sizes = (T, B, Hq, Hkv, d)
    small, big = lr.ChunkWorkspace(*sizes, q8=False), lr.ChunkWorkspace(*sizes)
    assert small.nbytes + T * Hq * (2 * d + 1) <= big.nbytes
    # nothing behind its end is written: the larger one's rest keeps its bytes
    big.buf[small.nbytes:] = 0xa5
    for opts in (dict(), dict(window=90)):
        a, b = (lr.libraspec_chunk_attn(Q, Kc, Vc, cu, kv, ws, **opts)[0] for ws in (small, big))
        assert torch.equal(a, b)
    a, b = (lr.libraspec_sink_attn(Q, Kc, Vc, cu, kv, ws, window=90, sinks=4)[0] for ws in (small, big))
    assert torch.equal(a, b) and bool((big.buf[small.nbytes:] == 0xa5).all())
    assert lr.libraspec_get_status(small) == lr.libraspec_get_status(big) == 0
    K8, V8 = (torch.zeros((B, Hkv, S, d), dtype=torch.uint8, device=cuda()).view(torch.float8_e4m3fn) for _ in "KV")
    Ks, Vs = (torch.zeros((B, Hkv, S // 16), dtype=torch.uint8, device=cuda()) for _ in "KV")
    with pytest.raises(lr.LibraspecError, match="invalid argument"):
        lr.libraspec_chunk_attn_q8(Q, K8, V8, Ks, Vs, cu, kv, small)
