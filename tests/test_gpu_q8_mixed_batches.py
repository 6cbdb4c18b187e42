"""GPU: a prompt's chunk among sequences without new tokens, over a cache in 8 bits: the call has fewer new tokens than
sequences, as a decode step has, and is none."""
import pytest
import torch

from helpers import cuda
from paper_2608_08721_gb300 import binding as lr

pytestmark = pytest.mark.gpu


def chunk(B, T, kv, Hq, Hkv, d, page=64, block=32):
    """T new tokens of the last of B sequences; returns a call and its workspace."""
    g = torch.Generator(device=cuda()).manual_seed(3)
    pages = (kv + T + page - 1) // page
    codes = [(torch.randn((pages, Hkv, page, d), generator=g, device=cuda()) * 50).to(torch.float8_e4m3fn) for _ in "KV"]
    exps = [torch.full((pages, Hkv, page // block), 121, dtype=torch.uint8, device=cuda()) for _ in "KV"]
    table = torch.zeros((B, pages), dtype=torch.int32, device=cuda())
    table[B - 1] = torch.arange(pages, dtype=torch.int32)
    cu = torch.zeros(B + 1, dtype=torch.int32, device=cuda())
    cu[B] = T
    kvl = torch.full((B,), 5, dtype=torch.int32, device=cuda())
    kvl[B - 1] = kv
    Q = torch.randn((T, Hq, d), generator=g, device=cuda()).to(torch.bfloat16)
    ws = lr.ChunkWorkspace(T, B, Hq, Hkv, d)
    return lambda: lr.libraspec_chunk_attn_q8_paged(Q, *codes, *exps, table, cu, kvl, ws, want_lse=True), ws


def ms(call):
    for _ in range(3):
        call()
    times = []
    for _ in range(5):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        call()
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b))
    return min(times)


def test_a_chunk_among_idle_sequences():
    """4096 new tokens of one sequence of 4096 (16384 rows for each head of the cache): the results of the chunk by itself,
    in less than three times its time. (Read for 8 rows at a time its keys would take some thirty times as many loads.)"""
    alone, ws1 = chunk(1, 4096, 2000, 8, 2, 128)
    among, ws2 = chunk(4096, 4096, 2000, 8, 2, 128)
    (O1, lse1), (O2, lse2) = alone(), among()
    assert lr.libraspec_get_status(ws1) == lr.libraspec_get_status(ws2) == 0
    # (its blocks may be cut elsewhere)
    assert bool(((O1.float() - O2.float()).abs() <= 2.0 ** -6 * O1.float().abs() + 1e-3).all())
    assert bool(((lse1 - lse2).abs() <= 1e-3).all())
    assert ms(among) < 3 * ms(alone)
