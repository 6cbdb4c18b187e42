"""GPU: prompts through the paged cache in chunks, decoded from, and verified (paper_2608_08721_gb300.prefill)."""
import pytest
import torch

from helpers import cuda
from paper_2608_08721_gb300 import binding as lr
from paper_2608_08721_gb300 import prefill
from test_gpu_chunk_attn import assert_close, attend64
from test_gpu_rope import freqs64, rotate64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,d", [(32, 8, 128), (8, 2, 64)])
def test_chunks_decode_and_verify(Hq, Hkv, d):
    """The cache is the same in chunks as at once, and two kernels agree on the drafted block: each rounds its
    probabilities to 8 bits and its result, 2 x (2^-8 + 2^-8) apart at most, and far less in norm."""
    r = prefill.run(prompts=(300, 1, 129), chunk=100, decode=2, K=5, n_layers=2, Hq=Hq, Hkv=Hkv, d=d)
    assert r["chunks"] == 3 and r["cache_equal"] and r["decoded"] == 3
    assert r["verify_rel_diff"] <= 2.0 ** -7


def test_a_step_against_the_definitions():
    """Rotation, append and attention of two steps, the second over the first, with a window and capped scores."""
    B, Hq, Hkv, d = 2, 4, 2, 64
    g = torch.Generator().manual_seed(3)
    fr = lr.RopeFreqs(d)
    seqs = prefill.PagedSequences(1, B, 100, Hq, Hkv, d, fr, 80, page_size=16)
    chunks = [[37, 5], [20, 60]]
    rows = [torch.randn((sum(n), Hq + 2 * Hkv, d), generator=g) for n in chunks]
    keys, values = [[] for _ in range(B)], [[] for _ in range(B)]
    kv = [0, 0]
    for n, x in zip(chunks, rows):
        step = seqs.begin(n)
        lse = torch.empty((sum(n), Hq), device=cuda())
        O = seqs.layer(0, x.to(cuda()), step, lse=lse, window=30, softcap=5.0)
        seqs.end(step)
        pos = torch.cat([torch.arange(kv[b], kv[b] + n[b]) for b in range(B)]).numpy()
        q, _ = rotate64(x[:, :Hq].double(), pos, freqs64(d), False)
        k, _ = rotate64(x[:, Hq:Hq + Hkv].double(), pos, freqs64(d), False)
        at = 0
        for b in range(B):
            keys[b].append(k[at:at + n[b]].transpose(0, 1).to(torch.bfloat16).double())
            values[b].append(x[at:at + n[b], Hq + Hkv:].transpose(0, 1).to(torch.bfloat16).double())
            at += n[b]
        want = attend64(q.to(torch.bfloat16).double(), [torch.cat(t, 1) for t in keys], [torch.cat(t, 1) for t in values],
                        n, kv, d ** -0.5, window=30, softcap=5.0)
        # (a rotated value that lies at the middle of two bf16 numbers may round the other way: 2^-8 of a query or key
        # element, below 2^-8 of a score in a sum of 64)
        assert_close(O, lse, *want, q_scale=16.0)
        kv = [a + m for a, m in zip(kv, n)]
    seqs.check()
    assert seqs.lengths == kv == seqs.kv_len.tolist()


def test_begin_refuses():
    seqs = prefill.PagedSequences(1, 2, 32, 4, 2, 64, lr.RopeFreqs(64), 40, page_size=16)
    for n in ([1], [-1, 1], [20, 21], [33, 0]):
        with pytest.raises(ValueError):
            seqs.begin(n)


def test_layers_on_another_stream_keep_the_order_of_the_steps():
    """Steps on a side stream that lags behind give what they give on the current one: lengths advance behind the
    layers that read them, and what a layer drops is not handed out while the stream still works on it."""
    B, Hq, Hkv, d, layers = 3, 8, 2, 64, 2
    steps = [[120, 3, 60], [1, 1, 1], [40, 64, 0], [1, 1, 1]]
    g = torch.Generator(device=cuda()).manual_seed(8)
    rows = [torch.randn((layers, sum(n), Hq + 2 * Hkv, d), generator=g, device=cuda(), dtype=torch.bfloat16)
            for n in steps]

    def go(stream):
        seqs = prefill.PagedSequences(layers, B, 200, Hq, Hkv, d, lr.RopeFreqs(d), 200, page_size=16)
        for pool in seqs.pools:
            for p in pool.values():
                p.zero_()
        out = []
        for n, x in zip(steps, rows):
            step = seqs.begin(n)
            for l in range(layers):
                if stream is not None:
                    with torch.cuda.stream(stream):
                        torch.cuda._sleep(2_000_000)  # about a millisecond
                qkv = x[l].clone()  # (from the current stream, and dropped after the layer)
                O = seqs.layer(l, qkv, step, stream=stream)
                del qkv
                scratch = [torch.full((sum(n), Hq, d), 9.0, device=cuda(), dtype=torch.bfloat16) for _ in range(4)]
                out.append(O.clone())
                del O, scratch
            seqs.end(step)
        torch.cuda.synchronize()
        seqs.check()
        return out, seqs

    want, a = go(None)
    got, b = go(torch.cuda.Stream())
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert a.lengths == b.lengths == b.kv_len.tolist()
    assert all(torch.equal(p[n], q[n]) for p, q in zip(a.pools, b.pools) for n in p)


def test_layer_refuses_rows_of_another_step():
    seqs = prefill.PagedSequences(1, 2, 32, 4, 2, 64, lr.RopeFreqs(64), 40, page_size=16)
    step = seqs.begin([3, 5])
    for shape in ((9, 8, 64), (7, 8, 64), (8, 9, 64), (8, 7, 64), (8, 8, 128), (8, 512)):
        with pytest.raises(ValueError):
            seqs.layer(0, torch.zeros(shape, device=cuda()), step)
