"""GPU: a call launches on the current device and takes pointers; any tensor of another device, weights, positions, lengths and
outputs among them, refuses it before anything is enqueued."""
import pytest
import torch

from helpers import cuda
from paper_2608_08721_gb300 import binding as lr

pytestmark = pytest.mark.gpu


def calls():
    d, Hq, Hkv, B, S, T = 64, 4, 2, 1, 64, 2
    z = dict(device=cuda())
    i32 = dict(dtype=torch.int32, **z)
    bf = dict(dtype=torch.bfloat16, **z)
    Q, K, V = (torch.zeros((T, h, d), **bf) for h in (Hq, Hkv, Hkv))
    pos, cu, kv = torch.zeros(T, **i32), torch.tensor([0, T], **i32), torch.zeros(B, **i32)
    K8, V8 = [torch.zeros((B, Hkv, S, d), dtype=torch.uint8, **z).view(torch.float8_e4m3fn) for _ in "KV"]
    Ks, Vs = [torch.zeros((B, Hkv, S // 16), dtype=torch.uint8, **z) for _ in "KV"]
    Kc, Vc = [torch.zeros((B, Hkv, S, d), **bf) for _ in "KV"]
    table, O, lse = torch.zeros((B, 1), **i32), torch.zeros((T, Hq, d), **bf), torch.zeros((T, Hq), **z)
    slopes, first, prefix = torch.zeros(Hq, **z), torch.zeros(T, **i32), torch.zeros(B, **i32)
    wq, wk = torch.ones(d, **z), torch.ones(d, **z)
    norm, freqs, ws = lr.QkNorm(wq, wk), lr.RopeFreqs(d), lr.ChunkWorkspace(T, B, Hq, Hkv, d)
    step, cache = dict(cu_new=cu, kv_len=kv), dict(K8=K8, V8=V8, Ks=Ks, Vs=Vs)
    rows = dict(K=torch.zeros((T, Hkv, d), **bf), V=torch.zeros((T, Hkv, d), **bf))
    X = torch.zeros((T, Hq + Hkv, d), **bf)
    own = [wq, wk, freqs.turns]
    return ws, [
        (lr.libraspec_qk_norm_rope, dict(X=X, n_q=Hq, norm=norm, pos=pos, freqs=freqs, Y=torch.zeros_like(X)), own),
        (lr.libraspec_rope_append_q8, dict(Q=Q, K=K, V=V, **cache, **step, freqs=freqs, ws=ws, norm=norm, pos=pos, Qo=O), own + [ws.buf]),
        (lr.libraspec_rope_append_q8_paged, dict(Q=Q, K=K, V=V, **cache, block_table=table, **step, freqs=freqs, ws=ws, Qo=O),
         [freqs.turns, ws.buf]),
        (lr.libraspec_kv_read_q8, dict(**cache, cu=cu, start=kv, T=T, ws=ws, **rows), [ws.buf]),
        (lr.libraspec_kv_read_q8_paged, dict(**cache, block_table=table, cu=cu, start=kv, T=T, ws=ws, **rows), [ws.buf]),
        (lr.libraspec_chunk_attn_q8, dict(Q=Q, **cache, **step, ws=ws, slopes=slopes, first_key=first, prefix_len=prefix, O=O,
                                          lse=lse), [ws.buf]),
        (lr.libraspec_chunk_attn_q8_paged, dict(Q=Q, **cache, block_table=table, **step, ws=ws, O=O, lse=lse), [ws.buf]),
        (lr.libraspec_sink_attn, dict(Q=Q, Kc=Kc, Vc=Vc, **step, ws=ws, window=8, sinks=1, slopes=slopes, prefix_len=prefix, O=O,
                                      lse=lse), [ws.buf]),
        (lr.libraspec_sink_attn_paged, dict(Q=Q, Kp=Kc, Vp=Vc, block_table=table, **step, ws=ws, window=8, sinks=1, O=O), [ws.buf]),
    ]


def test_every_tensor_of_a_call_is_looked_at(monkeypatch):
    """One tensor at a time is elsewhere (the library is told so; nothing is launched)."""
    ws, all_calls = calls()
    place = torch.Tensor.get_device
    monkeypatch.setattr(lr, "_several_devices", lambda: True)  # (with a single one nothing can be elsewhere)
    for fn, kw, held in all_calls:
        fn(**kw)
        tensors = [t for t in kw.values() if isinstance(t, torch.Tensor)] + held
        for t in tensors:
            at = t.data_ptr()
            with monkeypatch.context() as m:
                m.setattr(torch.Tensor, "get_device", lambda x: place(x) + (x.data_ptr() == at))
                with pytest.raises(ValueError, match="current device"):
                    fn(**kw)
        fn(**kw)
    torch.cuda.synchronize()
    assert lr.libraspec_get_status(ws) == 0
