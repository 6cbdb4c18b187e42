"""GPU: steps through a paged cache in 8 bits with normed heads and sinks, as a server runs them (PagedSequences): norm,
rotation, append, attention and read-back one after the other."""
import numpy as np
import pytest
import torch

from helpers import cuda
from paper_2608_08721_gb300 import binding as lr
from paper_2608_08721_gb300 import prefill
from test_gpu_chunk_q8 import attend64
from test_gpu_rope import freqs64, rotate64
from test_gpu_rope_q8 import norm64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,d,block", [(32, 8, 128, 16), (8, 2, 64, 64)])
def test_prompts_decode_and_verify_in_8_bits(Hq, Hkv, d, block):
    """Against a cache of 16 bits: a key or value is off by 2^-4 of itself at most, in norm by less; two independent such
    errors move a result by 2^-4 x sqrt(2) of it in norm at most where the scores are small (normed heads). Against the
    verify attention of the same values: P in bf16 there, 2^-8, and both results' roundings, 2 x 2^-8."""
    r = prefill.run_q8(prompts=(300, 1, 129), chunk=100, decode=2, K=5, Hq=Hq, Hkv=Hkv, d=d, block=block, window=64)
    assert 0 < r["rel_to_16_bits"] <= 2.0 ** -4 * 2 ** 0.5
    assert r["verify_rel_diff"] <= 3 * 2.0 ** -8


@pytest.mark.parametrize("block", [0, 16])
def test_steps_against_the_definitions(block):
    """Three steps (chunks, then a token each) of a sequence pair; the attention against 64 bits on the values that the cache
    holds, with a window and sinks; the cache itself within half a step of e4m3 (or bf16) of what it should hold."""
    B, Hq, Hkv, d, window, sinks = 2, 4, 2, 64, 30, 5
    g = torch.Generator().manual_seed(3)
    wq, wk = 1.0 + 0.3 * torch.randn((2, d), generator=g)
    norm = lr.QkNorm(wq.to(cuda()), wk.to(cuda()), 1e-5)
    seqs = prefill.PagedSequences(1, B, 100, Hq, Hkv, d, lr.RopeFreqs(d), 80, page_size=16, block=block, norm=norm)
    keys = [torch.zeros((Hkv, 0, d), dtype=torch.float64) for _ in range(B)]
    kv = [0, 0]
    for n in ([37, 5], [20, 60], [1, 1]):
        x = torch.randn((sum(n), Hq + 2 * Hkv, d), generator=g).to(torch.bfloat16)
        step = seqs.begin(n)
        lse = torch.empty((sum(n), Hq), device=cuda())
        O = seqs.layer(0, x.to(cuda()), step, lse=lse, window=window, sinks=sinks).double().cpu()
        seqs.end(step)
        pos = torch.cat([torch.arange(a, a + m) for a, m in zip(kv, n)]).numpy()
        q, _ = rotate64(norm64(x[:, :Hq].double(), wq.double(), 1e-5), pos, freqs64(d), False)
        k, _ = rotate64(norm64(x[:, Hq:Hq + Hkv].double(), wk.double(), 1e-5), pos, freqs64(d), False)
        at = 0
        for b in range(B):
            keys[b] = torch.cat([keys[b], k[at:at + n[b]].transpose(0, 1)], 1)
            at += n[b]
        kv = [a + m for a, m in zip(kv, n)]
        pools = seqs.unpacked(0)
        held = [[pools[p].cpu()[seqs.block_table[b].cpu().long()].transpose(0, 1).reshape(Hkv, -1, d)[:, :kv[b]].double()
                 for b in range(B)] for p in ("Kp", "Vp")]
        for b in range(B):
            # half a step of e4m3 (2^-4 of the value, 2^-10 of a scale of 2^-7 of the largest at least), and as much again
            # where a scale grew later; of bf16: the normed and rotated value rounded twice, 2^-8 each
            off = (held[0][b] - keys[b]).abs()
            bound = keys[b].abs() * (2.0 ** -3 if block else 2.0 ** -7) + (2.0 ** -15 * keys[b].abs().max() if block else 1e-5)
            assert bool((off <= bound).all())
        was = [a - m for a, m in zip(kv, n)]
        qb = q.to(torch.bfloat16).double()
        want, A, want_lse, top, mag = attend64(qb, held[0], held[1], n, was, d ** -0.5, window=window, sinks=sinks)
        # (a query element that lies at the middle of two bf16 numbers may round the other way: 2^-8 of it, below 2^-8 of
        # a score's magnitudes)
        delta = 2.0 ** -12 + (2.0 ** -8 + 2.0 ** -17) * mag
        bound = (2.0 ** -8 * 1.01 + 2 * delta) * A + 2.0 ** -8 * 1.01 * want.abs()
        assert bool(((O - want).abs() <= bound).all())
        assert bool(((lse.double().cpu() - want_lse).abs() <= delta + 1e-5 * want_lse.abs()).all())
    seqs.check()
    assert seqs.lengths == kv == seqs.kv_len.tolist()


def test_a_layer_on_another_stream():
    """The steps on a side stream give the same as on the current one."""
    B, Hq, Hkv, d = 2, 4, 2, 64
    g = torch.Generator().manual_seed(1)
    freqs = lr.RopeFreqs(d)
    xs = [torch.randn((B * n, Hq + 2 * Hkv, d), generator=g).to(torch.bfloat16).to(cuda()) for n in (40, 1, 1)]
    outs = []
    for stream in (None, torch.cuda.Stream()):
        seqs = prefill.PagedSequences(1, B, 64, Hq, Hkv, d, freqs, 80, page_size=32, block=32)
        got = []
        for x in xs:
            step = seqs.begin([x.shape[0] // B] * B)
            got.append(seqs.layer(0, x, step, stream=stream, window=20, sinks=2).clone())
            seqs.end(step)
        seqs.check()
        outs.append(got)
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_blocks_that_pages_do_not_hold_are_refused():
    with pytest.raises(ValueError, match="whole blocks"):
        prefill.PagedSequences(1, 1, 32, 4, 2, 64, lr.RopeFreqs(64), 8, page_size=16, block=32)
