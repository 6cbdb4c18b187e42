"""Performance cases of the calls around a KV cache held in 8 bits.

Five entry points of the public binding, on device-resident inputs: the norm of query and key heads with
the rotation in the same pass (``libraspec_qk_norm_rope``), the append of a ragged chunk to a cache of e4m3
codes with a scale for each block of tokens and kv head (``libraspec_rope_append_q8``), that cache read back
(``libraspec_kv_read_q8``), attention of a chunk over it (``libraspec_chunk_attn_q8``), and attention in a
sliding window whose first tokens stay visible (``libraspec_sink_attn``; ``sinks`` of the former). Dense
caches or pages behind block tables.

An 8-bit cache holds, for block i of ``block`` tokens of a kv head, codes c and the exponent of a power of
two: the values are c 2^e. A block written afresh takes e = floor(log2 max |x|) - 7 within [-60, 60]; one that
had tokens keeps the larger of the two, and its codes are rounded to the new scale where that grows.

Shapes are the repository's own workloads (GQA 8/2, 32/8, 28/4, 64/8, head dim 64 / 128, batch 1 to 64,
caches of 512 to 131072 keys) with chunks of 1 to 8192 new tokens; ``draw`` spreads over the ranges between
and around them. Lengths come from the case itself (``lens`` seeds them), so that the work of a case is known
from the case; every tensor's values come from the seed.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False  # set by the tools: the framework's operators instead of the plain forms

EPS = 1e-6  # of the norms


def listed():
    return [
        # one decode step's queries and keys of a batch of 64 sequences, side by side in the projection: latency
        dict(name="norm_decode", kind="norm", T=64, Hq=32, Hkv=8, d=128, rot=128, inter=False, f32=False,
             pos_hi=32768, scaling="none"),
        # a long prompt chunk from fp32 projections, interleaved pairs over half of the head, positions scaled by parts
        dict(name="norm_long_f32", kind="norm", T=8192, Hq=64, Hkv=8, d=128, rot=64, inter=True, f32=True,
             pos_hi=131072, scaling="parts"),
        # one decode step's token of 64 sequences into a paged cache (most within a block that has tokens), normed
        dict(name="append_decode", kind="append", B=64, n_lo=1, n_hi=1, kv_lo=512, kv_hi=4096, Hq=32, Hkv=8, d=128,
             rot=128, inter=False, f32=False, page=128, block=16, norm=True, scaling="none", lens=1),
        # 16 ragged prompt chunks, g = 7, linearly scaled positions, scales for 64 tokens
        dict(name="append_ragged", kind="append", B=16, n_lo=7, n_hi=2048, kv_lo=1, kv_hi=8192, Hq=28, Hkv=4, d=128,
             rot=128, inter=False, f32=False, page=256, block=64, norm=False, scaling="linear", lens=2),
        # four short sequences of small heads, dense: what a tree verification takes from an 8-bit cache
        dict(name="read_small", kind="read", B=4, n_lo=100, n_hi=600, kv_lo=0, kv_hi=0, Hkv=2, d=64, page=0, block=32,
             lens=3),
        # a whole serving batch's caches, paged, from the middle of a block on
        dict(name="read_batch", kind="read", B=16, n_lo=512, n_hi=32768, kv_lo=0, kv_hi=100, Hkv=8, d=128, page=64,
             block=16, lens=4),
        # the smallest attention: one token of one sequence over 512 keys, dense, head dim 64
        dict(name="q8_decode_small", kind="attn", q8=True, B=1, n_lo=1, n_hi=1, kv_lo=512, kv_hi=512, Hq=8, Hkv=2, d=64,
             page=0, block=16, cap=0.0, bias=False, window=0, sinks=0, docs=False, prefix=False, lse=False, lens=5),
        # a decode step of a full serving batch, log-uniform cache lengths, paged
        dict(name="q8_decode_batch", kind="attn", q8=True, B=64, n_lo=1, n_hi=1, kv_lo=512, kv_hi=32768, Hq=32, Hkv=8,
             d=128, page=128, block=16, cap=0.0, bias=False, window=0, sinks=0, docs=False, prefix=False, lse=False,
             lens=6),
        # a prompt of 8192 tokens at once
        dict(name="q8_prompt", kind="attn", q8=True, B=1, n_lo=8192, n_hi=8192, kv_lo=0, kv_hi=0, Hq=32, Hkv=8, d=128,
             page=256, block=64, cap=0.0, bias=False, window=0, sinks=0, docs=False, prefix=False, lse=False, lens=7),
        # chunks of unequal length beside decoding sequences in a window of 1024 keys with 4 sinks, g = 7, lse wanted
        dict(name="q8_sinks_mixed", kind="attn", q8=True, B=16, n_lo=1, n_hi=512, kv_lo=1024, kv_hi=16384, Hq=28, Hkv=4,
             d=128, page=64, block=32, cap=0.0, bias=False, window=1024, sinks=4, docs=False, prefix=False, lse=True,
             lens=8),
        # a decode step of 64 long streams in 16 bits: a window of 4096 keys and 4 sinks
        dict(name="sink_decode", kind="attn", q8=False, B=64, n_lo=1, n_hi=1, kv_lo=4096, kv_hi=32768, Hq=32, Hkv=8,
             d=128, page=128, block=0, cap=0.0, bias=False, window=4096, sinks=4, docs=False, prefix=False, lse=False,
             lens=9),
        # prompts of uneven length in 16 bits, capped scores, a window of 1024 keys and the first page of 128 as sinks
        dict(name="sink_prompt_capped", kind="attn", q8=False, B=4, n_lo=1000, n_hi=4000, kv_lo=1, kv_hi=4096, Hq=16,
             Hkv=4, d=128, page=64, block=0, cap=50.0, bias=False, window=1024, sinks=128, docs=False, prefix=False,
             lse=False, lens=10),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_SCALINGS = ["none", "linear", "ntk", "parts"]


def draw(rng):
    kind = rng.choice(["norm", "append", "append", "read", "attn", "attn", "attn", "attn"])
    d = rng.choice([64, 128, 128])
    Hq, Hkv = rng.choice([(8, 2), (16, 4), (32, 8), (28, 4), (64, 8), (8, 8), (16, 2), (32, 4)])
    block = rng.choice([16, 16, 32, 64])
    page = rng.choice([0, 0, block, 64, 128, 256])
    lens = rng.randrange(1 << 30)
    if kind in ("norm", "append"):
        base = dict(kind=kind, d=d, rot=rng.choice([d, d, d // 2, 24, d - 6]), inter=rng.random() < 0.5,
                    f32=rng.random() < 0.4, scaling=rng.choice(_SCALINGS), Hq=Hq, Hkv=Hkv)
        if kind == "norm":
            return dict(base, T=_log_int(rng, 1, 8192), pos_hi=_log_int(rng, 512, 131072))
        B = _log_int(rng, 1, 64)
        n_hi = _log_int(rng, 1, max(2, 8192 // B))
        kv_hi = _log_int(rng, 1, max(2, min(32768, 262144 // B)))
        return dict(base, B=B, n_lo=rng.choice([1, n_hi]), n_hi=n_hi, kv_lo=rng.choice([1, kv_hi]), kv_hi=kv_hi,
                    page=page, block=block, norm=rng.random() < 0.5, lens=lens)
    B = _log_int(rng, 1, 64)
    if kind == "read":
        n_hi = _log_int(rng, 1, max(2, min(32768, 262144 // B)))
        return dict(kind=kind, B=B, n_lo=rng.choice([1, n_hi, 0 if B > 7 else 1]), n_hi=n_hi, kv_lo=0, kv_hi=_log_int(rng, 1, 1000),
                    Hkv=Hkv, d=d, page=page, block=block, lens=lens)
    q8 = rng.random() < 0.7
    decode = rng.random() < 0.35
    n_hi = rng.choice([1, 1, 2, 5]) if decode else _log_int(rng, 1, max(2, min(8192 // B, int((2e9 / (B * Hq)) ** 0.5))))
    # no more scores than the prompt of 8192 tokens has, no more bytes than the decoding batch reads
    most = min(131072, 1_000_000_000 // (B * Hq * n_hi) - n_hi // 2, 1_100_000_000 // (B * Hkv * d * 4) - n_hi)
    kv_hi = _log_int(rng, 16, max(17, most))
    windowed = not q8 or rng.random() < 0.4
    sinks = rng.choice([1, 4, 16, _log_int(rng, 1, 1000)]) if windowed else 0
    return dict(kind="attn", q8=q8, B=B, n_lo=rng.choice([1, n_hi, (n_hi + 1) // 2]), n_hi=n_hi,
                kv_lo=rng.choice([kv_hi, max(1, kv_hi // 32), 0]), kv_hi=kv_hi, Hq=Hq, Hkv=Hkv, d=d, page=page,
                block=block if q8 else 0, cap=rng.choice([0.0, 0.0, 0.0, 30.0, 50.0]), bias=rng.random() < 0.15,
                window=_log_int(rng, 16, 8192) if windowed else 0, sinks=sinks,
                docs=not sinks and rng.random() < 0.2, prefix=rng.random() < 0.2, lse=rng.random() < 0.5, lens=lens)


# ---------------------------------------------------------------------------------------------- lengths
def _lengths(case):
    """(new tokens, cache length before them) of every sequence: log-uniform in [n_lo, n_hi] and [kv_lo, kv_hi]."""
    r = np.random.default_rng([case["lens"], 1])

    def spread(lo, hi):
        x = np.exp(r.uniform(math.log(lo + 1), math.log(hi + 1), case["B"])) - 1
        return np.clip(x.round(), lo, hi).astype(np.int32)

    return spread(case["n_lo"], case["n_hi"]), spread(case["kv_lo"], case["kv_hi"])


def _touched(case):
    """Of an append: first row and number of rows of the blocks that it writes to, of every sequence."""
    n, kv = _lengths(case)
    start = kv // case["block"] * case["block"]
    return start, kv + n - start


def _rows(n, kv):
    """Sequence and position of every packed row."""
    seq = np.repeat(np.arange(len(n)), n)
    start = np.concatenate([[0], np.cumsum(n)[:-1]])
    return seq, (np.arange(int(n.sum())) - start[seq] + kv[seq]).astype(np.int32)


def _first_keys(case, n, kv):
    """First key of each row's document: documents of 64 to 2048 tokens packed one after the other."""
    r = np.random.default_rng([case["lens"], 2])
    first = []
    for b in range(len(n)):
        total, edges, at = int(n[b] + kv[b]), [], 0
        while at < total:
            edges.append(at)
            at += int(np.exp(r.uniform(math.log(64), math.log(2048))))
        pos = np.arange(kv[b], total)
        first.append(np.array(edges)[np.searchsorted(edges, pos, side="right") - 1])
    return np.concatenate(first).astype(np.int32)


def _prefixes(case, n, kv):
    """Length of the part of each sequence that is seen in both directions: up to half of the new tokens."""
    r = np.random.default_rng([case["lens"], 3])
    return (kv + (n * r.uniform(0.0, 0.5, len(n))).astype(np.int64)).astype(np.int32)


def _seen(case):
    """Every packed row sees the keys [0, first) and [lo, hi), where first <= lo."""
    n, kv = _lengths(case)
    seq, pos = _rows(n, kv)
    lo, hi = np.zeros_like(pos), pos + 1
    if case["window"]:
        lo = np.maximum(lo, pos - case["window"] + 1)
    if case["docs"]:
        lo = np.maximum(lo, _first_keys(case, n, kv))
    if case["prefix"]:
        hi = np.maximum(hi, np.minimum(_prefixes(case, n, kv), n + kv)[seq])
    return np.minimum(case["sinks"], lo).astype(np.int64), lo.astype(np.int64), hi.astype(np.int64)


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _rope_rule(case):
    """Arguments of the rotation's frequencies: base 500000 and a fourfold longer context than the original 8192."""
    rule = {"theta": 500000.0, "scaling": case["scaling"]}
    if case["scaling"] != "none":
        rule["factor"] = 4.0
    if case["scaling"] == "parts":
        rule.update(original_len=8192.0, low=1.0, high=32.0, magnitude=0.1 * math.log(4.0) + 1.0)
    return rule


def _exponents(amax):
    """floor(log2 amax) - 7 within [-60, 60], of a block's largest magnitude."""
    e = torch.frexp(amax)[1].to(torch.int32) - 8
    return torch.where(amax > 0, e, -60).clamp_(-60, 60)


def _power(e):
    """2^e in 32 bits, of whole numbers in [-126, 127]."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _codes(x, e):
    """x 2^-e, rounded to e4m3."""
    return (x * _power(-e)).to(torch.float8_e4m3fn)


def _pool(case, g, planes, rows):
    """Keys or values [planes, Hkv, rows, d]: N(0, 1) times a magnitude of each plane's head. In 8 bits: (codes, exponent
    + 127 of each block)."""
    Hkv, d, block = case["Hkv"], case["d"], case["block"]
    x = torch.randn((planes, Hkv, rows, d), generator=g, dtype=torch.bfloat16, device="cuda")
    x *= torch.exp(0.4 * torch.randn((planes, Hkv, 1, 1), generator=g, device="cuda")).to(torch.bfloat16)
    if not block:
        return x
    e = _exponents(x.view(planes, Hkv, rows // block, block * d).abs().amax(dim=-1).float())
    codes = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device="cuda")
    step = max(1, (1 << 28) // (Hkv * rows * d))
    for i in range(0, planes, step):  # (fp32 copies of a part at a time)
        codes[i:i + step] = _codes(x[i:i + step].float(), e[i:i + step].repeat_interleave(block, dim=2)[..., None])
    return codes, (e + 127).to(torch.uint8)


def _caches(case, g, need):
    """Key and value cache, dense [B, Hkv, S, d] or pools of pages, and a shuffled block table."""
    B, page = case["B"], case["page"]
    if not page:
        unit = case["block"] or 1
        planes, rows, table = B, (need + 3 + unit - 1) // unit * unit, None
    else:
        per = (need + page - 1) // page
        planes, rows = B * per + 3, page
        table = torch.randperm(planes, generator=g, device="cuda")[:B * per].view(B, per).to(torch.int32)
    return _pool(case, g, planes, rows), _pool(case, g, planes, rows), table


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    kind, d, Hkv = case["kind"], case["d"], case["Hkv"]
    dt = torch.float32 if case.get("f32") else torch.bfloat16
    if kind == "norm":  # queries and keys side by side in a projection's output that holds the values too
        T, Hq = case["T"], case["Hq"]
        s["qkv"] = torch.randn((T, Hq + 2 * Hkv, d), generator=g, dtype=dt, device="cuda")
        s["pos"] = torch.randint(0, case["pos_hi"], (T,), generator=g, device="cuda").to(torch.int32)
    else:
        n, kv = _lengths(case)
        T = int(n.sum())
        seq, pos = _rows(n, kv)
        K, V, s["table"] = _caches(case, g, max(1, int((n + kv).max())))
        if case["block"]:
            (s["K"], s["Ks"]), (s["V"], s["Vs"]) = K, V
        else:
            s["K"], s["V"] = K, V
        s["cu_new"] = torch.from_numpy(np.concatenate([[0], np.cumsum(n)]).astype(np.int32)).cuda()
        s["kv_len"] = torch.from_numpy(kv).cuda()
        s["seq"], s["pos"] = torch.from_numpy(seq).cuda(), torch.from_numpy(pos).cuda()
        if kind == "append":  # the projections' output, queries, keys and values side by side
            s["qkv"] = torch.randn((T, case["Hq"] + 2 * Hkv, d), generator=g, dtype=dt, device="cuda")
            start, count = _touched(case)
            rseq, rpos = _rows(count, start)
            s["cu_read"] = torch.from_numpy(np.concatenate([[0], np.cumsum(count)]).astype(np.int32)).cuda()
            s["start"] = torch.from_numpy(start.astype(np.int32)).cuda()
            s["rseq"], s["rpos"] = torch.from_numpy(rseq).cuda(), torch.from_numpy(rpos).cuda()
            old = rpos < kv[rseq]
            s["oseq"], s["opos"] = torch.from_numpy(rseq[old]).cuda(), torch.from_numpy(rpos[old]).cuda()
            s["blocks"] = int(((kv + n + case["block"] - 1) // case["block"] - kv // case["block"]).max())
        elif kind == "attn":
            Hq = case["Hq"]
            s["Q"] = torch.randn((T, Hq, d), generator=g, dtype=dt, device="cuda")
            if case["cap"]:  # models that cap their scores have large ones
                s["Q"] *= 8.0
            s["n"], s["keys"] = n, int((n + kv).max())
            i = torch.arange(1, Hq + 1, device="cuda")
            s["slopes"] = torch.exp2(-8.0 * i / Hq).float() if case["bias"] else None
            s["first"] = torch.from_numpy(_first_keys(case, n, kv)).cuda() if case["docs"] else None
            s["prefix"] = torch.from_numpy(_prefixes(case, n, kv)).cuda() if case["prefix"] else None
    if kind in ("norm", "append"):
        rule = _rope_rule(case)
        s["freqs"] = torch.from_numpy(_frequencies(case["rot"], **{k: v for k, v in rule.items() if k != "magnitude"})).cuda()
        s["magnitude"] = rule.get("magnitude", 1.0)
        s["wq"], s["wk"] = (1.0 + 0.3 * torch.randn((2, d), generator=g, device="cuda")).unbind()
    if own:
        from paper_2608_08721_gb300 import binding as lr

        s["lr"] = lr
        if kind == "attn":
            s["ws"] = lr.ChunkWorkspace(s["Q"].shape[0], case["B"], case["Hq"], Hkv, d)
        else:
            s["ws"] = lr.ChunkWorkspace(1, 1, 1, 1, 64)
        if kind in ("norm", "append"):
            s["rope"] = lr.RopeFreqs(case["rot"], **_rope_rule(case))
            s["norm"] = lr.QkNorm(s["wq"], s["wk"], EPS)
    return s


# ------------------------------------------------------------------------------------------- plain forms
def _frequencies(rot, theta, scaling, factor=1.0, original_len=0.0, low=0.0, high=0.0):
    """Radians per position of each pair, in 64 bits."""
    if scaling == "ntk":
        theta = theta * factor ** (rot / (rot - 2))
    f = theta ** (-np.arange(0, rot, 2, dtype=np.float64) / rot)
    if scaling == "linear":
        f = f / factor
    if scaling == "parts":
        keep = np.clip((original_len * f / (2 * math.pi) - low) / (high - low), 0.0, 1.0)
        f = (1 - keep) * f / factor + keep * f
    return f


def _rotate(x, s):
    """x [T, H, d] in 32 bits, rotated. (The angle alone in 64 bits: in 32 a position of 131072 is off by 0.004 rad.)"""
    rot, inter = s["case"]["rot"], s["case"]["inter"]
    a = s["pos"].double()[:, None, None] * s["freqs"]
    a = torch.remainder(a, 2 * math.pi).float()
    cos, sin = torch.cos(a) * s["magnitude"], torch.sin(a) * s["magnitude"]
    r = x[..., :rot]
    x0, x1 = (r[..., 0::2], r[..., 1::2]) if inter else (r[..., :rot // 2], r[..., rot // 2:])
    y0, y1 = x0 * cos - x1 * sin, x0 * sin + x1 * cos
    y = torch.stack([y0, y1], dim=-1).flatten(-2) if inter else torch.cat([y0, y1], dim=-1)
    return torch.cat([y, x[..., rot:]], dim=-1)


def _normed(x, w):
    """x [T, H, d] in 32 bits over its heads' root mean squares, times w."""
    return x * torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + EPS) * w


def _plain_norm(s):
    Hq, Hkv = s["case"]["Hq"], s["case"]["Hkv"]
    x = s["qkv"][:, :Hq + Hkv].float()
    w = torch.cat([s["wq"].expand(Hq, -1), s["wk"].expand(Hkv, -1)])
    return {"Y": _rotate(_normed(x, w), s).to(s["qkv"].dtype)}


def _at(s, seq, pos):
    """Plane and row of keys in the cache."""
    page = s["case"]["page"]
    if not page:
        return seq, pos.long()
    return s["table"][seq, pos // page].long(), (pos % page).long()


def _values(codes, scales, plane, row, block):
    """Rows of an 8-bit cache in 32 bits, [rows, Hkv, d]."""
    return codes[plane, :, row].float() * _power(scales[plane, :, row // block].int() - 127)[..., None]


def _plain_write(s, x, codes, scales):
    """x [T, Hkv, d] in 32 bits into one of the caches."""
    c, (T, Hkv, d) = s["case"], x.shape
    B, block, NB = c["B"], c["block"], s["blocks"]
    first = s["kv_len"] // block  # block of each sequence's first new token
    i = s["pos"] // block - first[s["seq"]]
    padded = torch.zeros((B, NB * block, Hkv, d), device="cuda")
    padded[s["seq"], s["pos"] - first[s["seq"]] * block] = x.abs()
    e = _exponents(padded.view(B, NB, block, Hkv, d).amax(dim=(2, 4)))
    # a first block that has tokens
    has = s["kv_len"] % block > 0
    plane, row = _at(s, torch.arange(B, device="cuda"), torch.where(has, first * block, 0))
    before = scales[plane, :, row // block].int() - 127
    e[:, 0] = torch.where(has[:, None], torch.maximum(e[:, 0], before), e[:, 0])
    plane, row = _at(s, s["oseq"], s["opos"])
    y = _values(codes, scales, plane, row, block)
    codes[plane, :, row] = _codes(y, e[s["oseq"], 0][..., None])
    plane, row = _at(s, s["seq"], s["pos"])
    e = e[s["seq"], i]
    codes[plane, :, row] = _codes(x, e[..., None])
    scales[plane, :, row // block] = (e + 127).to(torch.uint8)


def _plain_append(s):
    c = s["case"]
    Hq, Hkv = c["Hq"], c["Hkv"]
    x = s["qkv"].float()
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    if c["norm"]:
        q, k = _normed(q, s["wq"]), _normed(k, s["wk"])
    _plain_write(s, _rotate(k, s), s["K"], s["Ks"])
    _plain_write(s, v, s["V"], s["Vs"])
    plane, row = _at(s, s["rseq"], s["rpos"])
    return {"Q": _rotate(q, s).to(torch.bfloat16),
            "K": _values(s["K"], s["Ks"], plane, row, c["block"]).to(torch.bfloat16),
            "V": _values(s["V"], s["Vs"], plane, row, c["block"]).to(torch.bfloat16)}


def _plain_read(s):
    plane, row = _at(s, s["seq"], s["pos"])
    return {x: _values(s[x], s[x + "s"], plane, row, s["case"]["block"]).to(torch.bfloat16) for x in "KV"}


def _plain_attn(s):
    c, B = s["case"], s["case"]["B"]
    Hq, Hkv, d, N, Tm = c["Hq"], c["Hkv"], c["d"], s["keys"], int(s["n"].max())
    g = Hq // Hkv
    n, kv, cu = (s["cu_new"][1:] - s["cu_new"][:-1]).long(), s["kv_len"].long(), s["cu_new"].long()
    t, key = torch.arange(Tm, device="cuda"), torch.arange(N, device="cuda")
    row = (cu[:-1, None] + t).clamp_(max=s["Q"].shape[0] - 1)  # [B, Tm], padded
    pos = kv[:, None] + t
    q = s["Q"][row].float().view(B, Tm, Hkv, g, d).permute(0, 2, 3, 1, 4)  # [B, Hkv, g, Tm, d]

    def cache(name):
        x = s[name]
        if c["q8"]:
            e = _power(s[name + "s"].int() - 127).repeat_interleave(c["block"], dim=2)
        if s["table"] is not None:
            at = s["table"].long()
            x = x[at].permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, d)
            if c["q8"]:
                e = e[at].permute(0, 2, 1, 3).reshape(B, Hkv, -1)
        x = x[:, :, :N].float()
        return x.mul_(e[:, :, :N, None]) if c["q8"] else x

    see = (key < (kv + n)[:, None])[:, None] & (t < n[:, None])[:, :, None]
    ahead = key <= pos[:, :, None]
    if s["prefix"] is not None:
        ahead |= key < s["prefix"][:, None, None]
    see &= ahead
    if c["window"]:
        see &= (key > pos[:, :, None] - c["window"]) | (key < c["sinks"])
    if s["first"] is not None:
        see &= key >= s["first"][row][:, :, None]
    x = torch.matmul(q.reshape(B, Hkv, g * Tm, d), cache("K").transpose(2, 3)).view(B, Hkv, g, Tm, N)
    x.mul_(d ** -0.5)
    if c["cap"]:
        x.div_(c["cap"]).tanh_().mul_(c["cap"])
    if s["slopes"] is not None:
        dist = (pos[:, :, None] - key).abs().float()
        x.sub_(s["slopes"].view(Hkv, g, 1, 1) * dist[:, None, None])
    x.masked_fill_(~see[:, None, None], -math.inf)
    m = x.amax(dim=-1, keepdim=True)
    x.sub_(torch.where(m == -math.inf, 0.0, m)).exp_()
    l = x.sum(dim=-1, keepdim=True)
    o = torch.matmul(x.view(B, Hkv, g * Tm, N), cache("V")).view(B, Hkv, g, Tm, d)
    o = torch.where(l > 0, o / l, 0.0)
    at = s["pos"] - s["kv_len"][s["seq"]]
    out = {"O": o.permute(0, 3, 1, 2, 4).reshape(B, Tm, Hq, d)[s["seq"], at].to(torch.bfloat16)}
    if c["lse"]:
        out["lse"] = (m + torch.log(l))[..., 0].permute(0, 3, 1, 2).reshape(B, Tm, Hq)[s["seq"], at]
    return out


def run(state):
    s = state
    c = s["case"]
    kind = c["kind"]
    if not own:
        return {"norm": _plain_norm, "append": _plain_append, "read": _plain_read, "attn": _plain_attn}[kind](s)
    lr = s["lr"]
    if kind == "norm":
        return {"Y": lr.libraspec_qk_norm_rope(s["qkv"][:, :c["Hq"] + c["Hkv"]], c["Hq"], s["norm"], s["pos"], s["rope"],
                                               interleaved=c["inter"])}
    if kind == "attn":
        opts = dict(softcap=c["cap"], slopes=s["slopes"], window=c["window"], sinks=c["sinks"], prefix_len=s["prefix"],
                    want_lse=c["lse"])
        caches = [s["K"], s["V"]]
        if c["q8"]:
            opts["first_key"] = s["first"]
            caches += [s["Ks"], s["Vs"]]
            fn = lr.libraspec_chunk_attn_q8 if s["table"] is None else lr.libraspec_chunk_attn_q8_paged
        else:
            fn = lr.libraspec_sink_attn if s["table"] is None else lr.libraspec_sink_attn_paged
        if s["table"] is not None:
            caches.append(s["table"])
        o, lse = fn(s["Q"], *caches, s["cu_new"], s["kv_len"], s["ws"], **opts)
        return {"O": o, "lse": lse} if c["lse"] else {"O": o}
    caches = [s["K"], s["V"], s["Ks"], s["Vs"]] + ([] if s["table"] is None else [s["table"]])
    read = lr.libraspec_kv_read_q8 if s["table"] is None else lr.libraspec_kv_read_q8_paged
    if kind == "read":
        k, v = read(*caches, s["cu_new"], s["kv_len"], s["seq"].numel(), s["ws"])
        return {"K": k, "V": v}
    Hq, Hkv = c["Hq"], c["Hkv"]
    q, k, v = s["qkv"][:, :Hq], s["qkv"][:, Hq:Hq + Hkv], s["qkv"][:, Hq + Hkv:]
    append = lr.libraspec_rope_append_q8 if s["table"] is None else lr.libraspec_rope_append_q8_paged
    q = append(q, k, v, *caches, s["cu_new"], s["kv_len"], s["rope"], s["ws"], norm=s["norm"] if c["norm"] else None,
               interleaved=c["inter"])
    # the values of what the touched blocks hold now
    k, v = read(*caches, s["cu_read"], s["start"], s["rseq"].numel(), s["ws"])
    return {"Q": q, "K": k, "V": v}


# ---------------------------------------------------------------------------------------------- the work
def work(case):
    eb, d, kind = 4 if case.get("f32") else 2, case["d"], case["kind"]
    if kind == "norm":
        heads = case["T"] * (case["Hq"] + case["Hkv"])
        return {"bytes": 2 * heads * d * eb + 4 * case["T"] + 8 * d, "flops": heads * (3.0 * case["rot"] + 4.0 * d)}
    n, kv = _lengths(case)
    T, Hkv = int(n.sum()), case["Hkv"]
    if kind == "read":
        return {"bytes": T * Hkv * d * 6 + T * Hkv * 2 // case["block"] + 8, "flops": 2.0 * T * Hkv * d}
    Hq = case["Hq"]
    if kind == "append":
        rows = int(_touched(case)[1].sum())
        return {"bytes": T * (Hq * (eb + 2) + 2 * Hkv * (eb + 1)) * d + rows * Hkv * d * 6,
                "flops": 3.0 * T * (Hq + Hkv) * case["rot"] + (4.0 * T * (Hq + Hkv) * d if case["norm"] else 0.0)}
    first, lo, hi = _seen(case)
    ends = np.concatenate([[0], np.cumsum(n)])
    keys = 0.0
    for a, e in zip(ends[:-1], ends[1:]):
        if e > a:
            keys += float(hi[a:e].max() - lo[a:e].min()) + min(float(first[a:e].max()), float(lo[a:e].min()))
    per_key = 2 * d + 2.0 / case["block"] if case["q8"] else 4 * d
    return {"bytes": keys * Hkv * per_key + T * Hq * (4 * d + (4 if case["lse"] else 0)),
            "flops": 4.0 * d * Hq * float((np.maximum(hi - lo, 0) + first).sum())}


# ------------------------------------------------------------------------------------- the same in 64 bits
def _exact_turn(x, pos, case):
    """x [T, H, d] in 64 bits: each pair as a complex number times m e^(i angle)."""
    rot, rule = case["rot"], _rope_rule(case)
    base, s = rule["theta"], rule.get("factor", 1.0)
    if rule["scaling"] == "ntk":
        base *= s ** (rot / (rot - 2.0))
    f = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if rule["scaling"] == "linear":
        f = [v / s for v in f]
    if rule["scaling"] == "parts":
        turns = [rule["original_len"] * v / (2 * math.pi) for v in f]
        share = [min(1.0, max(0.0, (t - rule["low"]) / (rule["high"] - rule["low"]))) for t in turns]
        f = [v * (k + (1 - k) / s) for v, k in zip(f, share)]
    angle = pos.double()[:, None] * torch.tensor(f, dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.full_like(angle, rule.get("magnitude", 1.0)), angle)[:, None]
    y = x.double().clone()
    half = rot // 2
    i0 = torch.arange(half, device="cuda") * 2 if case["inter"] else torch.arange(half, device="cuda")
    i1 = i0 + (1 if case["inter"] else half)
    z = torch.complex(y[..., i0].contiguous(), y[..., i1].contiguous()) * turn
    y[..., i0], y[..., i1] = z.real, z.imag
    return y


def _exact_norm(x, w):
    x = x.double()
    return x / torch.sqrt((x * x).sum(dim=-1, keepdim=True) / x.shape[-1] + EPS) * w.double()


def _to_e4m3(x):
    """x in 64 bits, rounded to three bits behind the leading one (the last of 2^-9), ties to even."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))).clamp_min(-6) - 3)
    return torch.round(x / step) * step


def _exact_write(case, s, x, name):
    """What the touched blocks of one cache hold after the append of x [T, Hkv, d]; rows packed."""
    block = case["block"]
    n, kv = _lengths(case)
    out, at = [], 0
    for b in range(case["B"]):
        a, e = int(kv[b]), int(kv[b] + n[b])
        for first in range(a // block * block, e, block):
            new = x[at + max(first, a) - a:at + min(first + block, e) - a]
            amax = new.abs().amax(dim=(0, 2))
            top = torch.floor(torch.log2(amax.clamp_min(2.0 ** -53))) - 7
            top = top.clamp(-60, 60)
            if first < a:  # tokens that it had
                rows = torch.arange(first, a, device="cuda")
                if case["page"]:
                    plane, row = int(s["table"][b, first // case["page"]]), rows % case["page"]
                else:
                    plane, row = b, rows
                had = s[name + "s"][plane, :, row[0] // block].double() - 127
                top = torch.maximum(top, had)
                codes = s[name][plane][:, row].double().transpose(0, 1)
                out.append(_to_e4m3(codes * torch.exp2(had - top)[:, None]) * torch.exp2(top)[:, None])
            out.append(_to_e4m3(new / torch.exp2(top)[:, None]) * torch.exp2(top)[:, None])
        at += int(n[b])
    return torch.cat(out)


def _exact_rows(case, s, name, b, kvh, total):
    """Keys or values [total, d] of a sequence's kv head in 64 bits."""
    page, block = case["page"], case["block"]
    if page:
        ids = s["table"][b].long()[:(total + page - 1) // page]
        x = s[name][ids, kvh].reshape(-1, case["d"])[:total].double()
        e = s[name + "s"][ids, kvh].reshape(-1) if block else None
    else:
        x = s[name][b, kvh, :total].double()
        e = s[name + "s"][b, kvh] if block else None
    if e is None:
        return x
    return x * torch.exp2(e.double() - 127)[torch.arange(total, device="cuda") // block][:, None]


def _exact_attn(case, s):
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    g = Hq // Hkv
    n, kv = _lengths(case)
    sink, lo, hi = _seen(case)
    O, lse, at = [], [], 0
    for b in range(case["B"]):
        nb, total = int(n[b]), int(n[b] + kv[b])
        pos = torch.arange(int(kv[b]), total, device="cuda").double()[:, None]
        key = torch.arange(total, device="cuda").double()
        zero, first, last = (torch.from_numpy(x[at:at + nb]).cuda()[:, None] for x in (sink, lo, hi))
        hidden = ((key < first) & (key >= zero)) | (key >= last)
        o = torch.zeros((nb, Hq, d), dtype=torch.float64, device="cuda")
        e = torch.zeros((nb, Hq), dtype=torch.float64, device="cuda")
        for h in range(Hq):
            if h % g == 0:
                k, v = (_exact_rows(case, s, name, b, h // g, total) for name in "KV")
            x = s["Q"][at:at + nb, h].double() @ k.T / math.sqrt(d)
            if case["cap"]:
                x = torch.tanh(x / case["cap"]) * case["cap"]
            if case["bias"]:
                x -= 2.0 ** (-8.0 * (h + 1) / Hq) * (pos - key).abs()
            x.masked_fill_(hidden, -math.inf)
            e[:, h] = torch.logsumexp(x, dim=-1)
            o[:, h] = torch.exp(x - e[:, h:h + 1].nan_to_num(neginf=0.0)) @ v
        O.append(o)
        lse.append(e)
        at += nb
    return torch.cat(O), torch.cat(lse)


def exact(case, seed):
    s = prepare(case, seed)
    kind, Hkv = case["kind"], case["Hkv"]
    if kind == "norm":
        x, Hq = s["qkv"], case["Hq"]
        y = torch.cat([_exact_norm(x[:, :Hq], s["wq"]), _exact_norm(x[:, Hq:Hq + Hkv], s["wk"])], dim=1)
        return {"Y": _exact_turn(y, s["pos"], case)}
    if kind == "append":
        Hq = case["Hq"]
        q, k, v = s["qkv"][:, :Hq].double(), s["qkv"][:, Hq:Hq + Hkv].double(), s["qkv"][:, Hq + Hkv:].double()
        if case["norm"]:
            q, k = _exact_norm(q, s["wq"]), _exact_norm(k, s["wk"])
        return {"Q": _exact_turn(q, s["pos"], case), "K": _exact_write(case, s, _exact_turn(k, s["pos"], case), "K"),
                "V": _exact_write(case, s, v, "V")}
    if kind == "read":
        n, kv = _lengths(case)
        out = {}
        for name in "KV":
            rows = [torch.stack([_exact_rows(case, s, name, b, h, int(kv[b] + n[b]))[int(kv[b]):] for h in range(Hkv)], 1)
                    for b in range(case["B"])]
            out[name] = torch.cat(rows)
        return out
    O, lse = _exact_attn(case, s)
    return {"O": O, "lse": lse} if case["lse"] else {"O": O}
