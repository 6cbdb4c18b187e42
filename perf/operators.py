"""Performance cases of the calls that bring a prompt into the KV cache and decode from it.

Three entry points of the public binding, on device-resident inputs: rotary positions
(``libraspec_rope``), the append of a ragged chunk of new tokens with the rotation on the way
(``libraspec_rope_append``), and attention of that chunk over the cache, dense or paged
(``libraspec_chunk_attn``, ``libraspec_chunk_attn_paged``), with capped scores, a distance bias, a
sliding window, a document mask and a prefix mask as options.

Shapes are the repository's own workloads (GQA 8/2, 32/8, 28/4, 64/8, head dim 64 / 128, batch 1 to 64,
caches of 512 to 131072 keys) with chunks of 1 to 8192 new tokens; ``draw`` spreads over the ranges
between and around them. Lengths come from the case itself (``lens`` seeds them), so that the work of a
case is known from the case; every tensor's values come from the seed.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False  # set by the tools: the framework's operators instead of the plain forms


def listed():
    return [
        # one decode step's queries of a batch of 64 sequences: latency
        dict(name="rope_decode", kind="rope", T=64, H=32, d=128, rot=128, inter=False, f32=False, inverse=False,
             pos_hi=32768, scaling="none"),
        # queries of a long prompt chunk, interleaved pairs over half of the head, positions scaled by parts, in fp32
        dict(name="rope_long_f32", kind="rope", T=8192, H=64, d=128, rot=64, inter=True, f32=True, inverse=False,
             pos_hi=131072, scaling="parts"),
        # one decode step's token of 64 sequences into a paged cache
        dict(name="append_decode", kind="append", B=64, n_lo=1, n_hi=1, kv_lo=512, kv_hi=4096, Hq=32, Hkv=8, d=128,
             rot=128, inter=False, f32=False, page=128, scaling="none", lens=1),
        # 16 ragged prompt chunks into a paged cache, linearly scaled positions, g = 7
        dict(name="append_ragged", kind="append", B=16, n_lo=7, n_hi=2048, kv_lo=1, kv_hi=8192, Hq=28, Hkv=4, d=128,
             rot=128, inter=False, f32=False, page=256, scaling="linear", lens=2),
        # a prompt of 8192 tokens from fp32 projections into a dense cache, interleaved, part of a head of 64
        dict(name="append_dense_f32", kind="append", B=2, n_lo=4095, n_hi=4097, kv_lo=1, kv_hi=64, Hq=32, Hkv=8, d=64,
             rot=32, inter=True, f32=True, page=0, scaling="ntk", lens=3),
        # the smallest attention: one token of one sequence over 512 keys, dense, head dim 64
        dict(name="attn_decode_small", kind="attn", B=1, n_lo=1, n_hi=1, kv_lo=512, kv_hi=512, Hq=8, Hkv=2, d=64,
             page=0, cap=0.0, bias=False, window=0, docs=False, prefix=False, lse=False, lens=4),
        # a decode step of a full serving batch, log-uniform cache lengths, paged
        dict(name="attn_decode_batch", kind="attn", B=64, n_lo=1, n_hi=1, kv_lo=512, kv_hi=32768, Hq=32, Hkv=8, d=128,
             page=128, cap=0.0, bias=False, window=0, docs=False, prefix=False, lse=False, lens=5),
        # chunks of unequal length beside decoding sequences, g = 7, log-sum-exp wanted
        dict(name="attn_mixed", kind="attn", B=16, n_lo=1, n_hi=512, kv_lo=1024, kv_hi=8192, Hq=28, Hkv=4, d=128,
             page=64, cap=0.0, bias=False, window=0, docs=False, prefix=False, lse=True, lens=6),
        # a whole prompt of 8192 tokens at once
        dict(name="attn_prompt", kind="attn", B=1, n_lo=8192, n_hi=8192, kv_lo=0, kv_hi=0, Hq=32, Hkv=8, d=128,
             page=256, cap=0.0, bias=False, window=0, docs=False, prefix=False, lse=False, lens=7),
        # a chunk of 1024 tokens at the end of a context of 128K keys
        dict(name="attn_long_chunk", kind="attn", B=1, n_lo=1024, n_hi=1024, kv_lo=130048, kv_hi=130048, Hq=64, Hkv=8,
             d=128, page=128, cap=0.0, bias=False, window=0, docs=False, prefix=False, lse=False, lens=8),
        # capped scores in a sliding window of 1024 keys over prompts of uneven length
        dict(name="attn_capped", kind="attn", B=4, n_lo=1000, n_hi=4000, kv_lo=1, kv_hi=4096, Hq=16, Hkv=4, d=128,
             page=64, cap=50.0, bias=False, window=1024, docs=False, prefix=False, lse=False, lens=9),
        # a distance bias over packed documents whose prompt is seen in both directions, head dim 64
        dict(name="attn_bias_docs", kind="attn", B=2, n_lo=2048, n_hi=4096, kv_lo=1, kv_hi=1024, Hq=16, Hkv=16, d=64,
             page=0, cap=0.0, bias=True, window=0, docs=True, prefix=True, lse=True, lens=10),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_SCALINGS = ["none", "linear", "ntk", "parts"]


def draw(rng):
    kind = rng.choice(["rope", "append", "attn", "attn", "attn"])
    d = rng.choice([64, 128, 128])
    Hq, Hkv = rng.choice([(8, 2), (16, 4), (32, 8), (28, 4), (64, 8), (8, 8), (16, 2), (32, 4)])
    if kind in ("rope", "append"):
        base = dict(kind=kind, d=d, rot=rng.choice([d, d, d // 2, 24, d - 6]), inter=rng.random() < 0.5,
                    f32=rng.random() < 0.4, scaling=rng.choice(_SCALINGS))
        if kind == "rope":
            return dict(base, T=_log_int(rng, 1, 8192), H=Hq, inverse=rng.random() < 0.3,
                        pos_hi=_log_int(rng, 512, 131072))
        B = _log_int(rng, 1, 64)
        n_hi = _log_int(rng, 1, max(2, 8192 // B))
        kv_hi = _log_int(rng, 1, max(2, min(32768, 262144 // B)))
        return dict(base, B=B, n_lo=rng.choice([1, n_hi]), n_hi=n_hi, kv_lo=rng.choice([1, kv_hi]), kv_hi=kv_hi, Hq=Hq,
                    Hkv=Hkv, page=rng.choice([0, 16, 32, 64, 128, 256]), lens=rng.randrange(1 << 30))
    B = _log_int(rng, 1, 64)
    decode = rng.random() < 0.35
    n_hi = rng.choice([1, 1, 2, 5]) if decode else _log_int(rng, 1, max(2, min(8192, 8192 // B)))
    # keys bounded so that the fp32 scores of the plain form take at most 12 GB and the batch's cache 4 GB
    most = min(131072, 3_000_000_000 // (B * Hq * n_hi) - n_hi, 4_000_000_000 // (B * Hkv * d * 4) - n_hi)
    kv_hi = _log_int(rng, 16, max(17, most))
    bias, cap = rng.random() < 0.2, rng.choice([0.0, 0.0, 0.0, 30.0, 50.0])
    return dict(kind=kind, B=B, n_lo=rng.choice([1, n_hi, (n_hi + 1) // 2]), n_hi=n_hi,
                kv_lo=rng.choice([kv_hi, max(1, kv_hi // 32), 0]), kv_hi=kv_hi, Hq=Hq, Hkv=Hkv, d=d,
                page=rng.choice([0, 0, 16, 32, 64, 128, 256]), cap=cap, bias=bias,
                window=_log_int(rng, 16, 8192) if rng.random() < 0.25 else 0, docs=rng.random() < 0.2,
                prefix=rng.random() < 0.2, lse=rng.random() < 0.5, lens=rng.randrange(1 << 30))


# ---------------------------------------------------------------------------------------------- lengths
def _lengths(case):
    """(new tokens, cache length before them) of every sequence: log-uniform in [n_lo, n_hi] and [kv_lo, kv_hi]."""
    r = np.random.default_rng([case["lens"], 1])

    def spread(lo, hi):
        x = np.exp(r.uniform(math.log(lo + 1), math.log(hi + 1), case["B"])) - 1
        return np.clip(x.round(), lo, hi).astype(np.int32)

    return spread(case["n_lo"], case["n_hi"]), spread(case["kv_lo"], case["kv_hi"])


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
    """First key seen and one past the last, of every packed row."""
    n, kv = _lengths(case)
    seq, pos = _rows(n, kv)
    lo, hi = np.zeros_like(pos), pos + 1
    if case["window"]:
        lo = np.maximum(lo, pos - case["window"] + 1)
    if case["docs"]:
        lo = np.maximum(lo, _first_keys(case, n, kv))
    if case["prefix"]:
        hi = np.maximum(hi, np.minimum(_prefixes(case, n, kv), n + kv)[seq])
    return seq, lo.astype(np.int64), hi.astype(np.int64)


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


def _caches(case, g, need):
    """Key and value cache of N(0, 1) bf16: dense [B, Hkv, S, d], or pools of pages and a shuffled block table."""
    B, Hkv, d, page = case["B"], case["Hkv"], case["d"], case["page"]
    if not page:
        shape, table = (B, Hkv, need + 3, d), None
    else:
        per = (need + page - 1) // page
        shape = (B * per + 3, Hkv, page, d)
        table = torch.randperm(B * per + 3, generator=g, device="cuda")[:B * per].view(B, per).to(torch.int32)
    K, V = (torch.randn(shape, generator=g, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    return K, V, table


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    dt = torch.float32 if case.get("f32") else torch.bfloat16
    if case["kind"] == "rope":
        s["X"] = torch.randn((case["T"], case["H"], case["d"]), generator=g, dtype=dt, device="cuda")
        s["pos"] = torch.randint(0, case["pos_hi"], (case["T"],), generator=g, device="cuda").to(torch.int32)
    else:
        n, kv = _lengths(case)
        T, Hq, Hkv, d = int(n.sum()), case["Hq"], case["Hkv"], case["d"]
        seq, pos = _rows(n, kv)
        s["K"], s["V"], s["table"] = _caches(case, g, int((n + kv).max()))
        s["cu_new"] = torch.from_numpy(np.concatenate([[0], np.cumsum(n)]).astype(np.int32)).cuda()
        s["kv_len"] = torch.from_numpy(kv).cuda()
        s["seq"], s["pos"] = torch.from_numpy(seq).cuda(), torch.from_numpy(pos).cuda()
        if case["kind"] == "append":  # the projections' output, queries, keys and values side by side
            s["qkv"] = torch.randn((T, Hq + 2 * Hkv, d), generator=g, dtype=dt, device="cuda")
        else:
            s["Q"] = torch.randn((T, Hq, d), generator=g, dtype=dt, device="cuda")
            if case["cap"]:  # models that cap their scores have large ones
                s["Q"] *= 8.0
            s["n"], s["keys"] = n, int((n + kv).max())
            i = torch.arange(1, Hq + 1, device="cuda")
            s["slopes"] = torch.exp2(-8.0 * i / Hq).float() if case["bias"] else None
            s["first"] = torch.from_numpy(_first_keys(case, n, kv)).cuda() if case["docs"] else None
            s["prefix"] = torch.from_numpy(_prefixes(case, n, kv)).cuda() if case["prefix"] else None
    if case["kind"] != "attn":
        rule = _rope_rule(case)
        s["freqs"] = torch.from_numpy(_frequencies(case["rot"], **{k: v for k, v in rule.items() if k != "magnitude"})).cuda()
        s["magnitude"] = rule.get("magnitude", 1.0)
    if own:
        from paper_2608_08721_gb300 import binding as lr

        s["lr"] = lr
        if case["kind"] == "attn":
            s["ws"] = lr.ChunkWorkspace(s["Q"].shape[0], case["B"], case["Hq"], case["Hkv"], case["d"])
        else:
            s["rope"] = lr.RopeFreqs(case["rot"], **_rope_rule(case))
            s["ws"] = lr.ChunkWorkspace(1, 1, 1, 1, case["d"])
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


def _rotate(x, pos, s, inter, rot, inverse=False):
    """x [T, H, d] in 32 bits, rotated. (The angle alone in 64 bits: in 32 a position of 131072 is off by 0.004 rad.)"""
    a = pos.double()[:, None, None] * s["freqs"]
    a = torch.remainder(a, 2 * math.pi).float()
    cos, sin = torch.cos(a) * s["magnitude"], torch.sin(a) * (-s["magnitude"] if inverse else s["magnitude"])
    r = x[..., :rot]
    x0, x1 = (r[..., 0::2], r[..., 1::2]) if inter else (r[..., :rot // 2], r[..., rot // 2:])
    y0, y1 = x0 * cos - x1 * sin, x0 * sin + x1 * cos
    y = torch.stack([y0, y1], dim=-1).flatten(-2) if inter else torch.cat([y0, y1], dim=-1)
    return torch.cat([y, x[..., rot:]], dim=-1)


def _plain_append(s):
    c = s["case"]
    Hq, Hkv = c["Hq"], c["Hkv"]
    qkv = s["qkv"].float()
    q = _rotate(qkv[:, :Hq], s["pos"], s, c["inter"], c["rot"])
    k = _rotate(qkv[:, Hq:Hq + Hkv], s["pos"], s, c["inter"], c["rot"])
    pos = s["pos"].long()
    if s["table"] is None:
        plane, row = s["seq"], pos
    else:
        plane, row = s["table"][s["seq"], pos // c["page"]].long(), pos % c["page"]
    s["K"][plane, :, row] = k.to(torch.bfloat16)
    s["V"][plane, :, row] = qkv[:, Hq + Hkv:].to(torch.bfloat16)
    return {"Q": q.to(torch.bfloat16), "K": s["K"], "V": s["V"]}


def _plain_attn(s):
    c, B = s["case"], s["case"]["B"]
    Hq, Hkv, d, N, Tm = c["Hq"], c["Hkv"], c["d"], s["keys"], int(s["n"].max())
    g = Hq // Hkv
    n, kv, cu = (s["cu_new"][1:] - s["cu_new"][:-1]).long(), s["kv_len"].long(), s["cu_new"].long()
    t, key = torch.arange(Tm, device="cuda"), torch.arange(N, device="cuda")
    row = (cu[:-1, None] + t).clamp_(max=s["Q"].shape[0] - 1)  # [B, Tm], padded
    pos = kv[:, None] + t
    q = s["Q"][row].float().view(B, Tm, Hkv, g, d).permute(0, 2, 3, 1, 4)  # [B, Hkv, g, Tm, d]

    def cache(x):
        if s["table"] is not None:
            x = x[s["table"].long()].permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, d)
        return x[:, :, :N].float()

    see = (key < (kv + n)[:, None])[:, None] & (t < n[:, None])[:, :, None]
    ahead = key <= pos[:, :, None]
    if s["prefix"] is not None:
        ahead |= key < s["prefix"][:, None, None]
    see &= ahead
    if c["window"]:
        see &= key > pos[:, :, None] - c["window"]
    if s["first"] is not None:
        see &= key >= s["first"][row][:, :, None]
    x = torch.matmul(q.reshape(B, Hkv, g * Tm, d), cache(s["K"]).transpose(2, 3)).view(B, Hkv, g, Tm, N)
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
    o = torch.matmul(x.view(B, Hkv, g * Tm, N), cache(s["V"])).view(B, Hkv, g, Tm, d)
    o = torch.where(l > 0, o / l, 0.0)
    out = {"O": o.permute(0, 3, 1, 2, 4).reshape(B, Tm, Hq, d)[s["seq"], s["pos"] - s["kv_len"][s["seq"]]].to(
        torch.bfloat16)}
    if c["lse"]:
        lse = (m + torch.log(l))[..., 0]
        out["lse"] = lse.permute(0, 3, 1, 2).reshape(B, Tm, Hq)[s["seq"], s["pos"] - s["kv_len"][s["seq"]]]
    return out


def run(state):
    s = state
    c = s["case"]
    if not own:
        if c["kind"] == "rope":
            return {"Y": _rotate(s["X"].float(), s["pos"], s, c["inter"], c["rot"], c["inverse"]).to(s["X"].dtype)}
        return _plain_append(s) if c["kind"] == "append" else _plain_attn(s)
    lr = s["lr"]
    if c["kind"] == "rope":
        return {"Y": lr.libraspec_rope(s["X"], s["pos"], s["rope"], interleaved=c["inter"], inverse=c["inverse"])}
    if c["kind"] == "append":
        Hq, Hkv = c["Hq"], c["Hkv"]
        q, k, v = s["qkv"][:, :Hq], s["qkv"][:, Hq:Hq + Hkv], s["qkv"][:, Hq + Hkv:]
        if s["table"] is None:
            q = lr.libraspec_rope_append(q, k, v, s["K"], s["V"], s["cu_new"], s["kv_len"], s["rope"], s["ws"],
                                         interleaved=c["inter"])
        else:
            q = lr.libraspec_rope_append_paged(q, k, v, s["K"], s["V"], s["table"], s["cu_new"], s["kv_len"], s["rope"],
                                               s["ws"], interleaved=c["inter"])
        return {"Q": q, "K": s["K"], "V": s["V"]}
    opts = dict(softcap=c["cap"], slopes=s["slopes"], window=c["window"], first_key=s["first"], prefix_len=s["prefix"],
                want_lse=c["lse"])
    if s["table"] is None:
        o, lse = lr.libraspec_chunk_attn(s["Q"], s["K"], s["V"], s["cu_new"], s["kv_len"], s["ws"], **opts)
    else:
        o, lse = lr.libraspec_chunk_attn_paged(s["Q"], s["K"], s["V"], s["table"], s["cu_new"], s["kv_len"], s["ws"],
                                               **opts)
    return {"O": o, "lse": lse} if c["lse"] else {"O": o}


# ---------------------------------------------------------------------------------------------- the work
def work(case):
    eb, d = 4 if case.get("f32") else 2, case["d"]
    if case["kind"] == "rope":
        x = case["T"] * case["H"] * d
        return {"bytes": 2 * x * eb + 4 * case["T"], "flops": 3.0 * case["T"] * case["H"] * case["rot"]}
    n, kv = _lengths(case)
    T, Hq, Hkv = int(n.sum()), case["Hq"], case["Hkv"]
    if case["kind"] == "append":
        return {"bytes": T * (Hq + 2 * Hkv) * d * (eb + 2), "flops": 3.0 * T * (Hq + Hkv) * case["rot"]}
    seq, lo, hi = _seen(case)
    ends = np.concatenate([[0], np.cumsum(n)])
    keys = sum(float(hi[a:e].max() - lo[a:e].min()) for a, e in zip(ends[:-1], ends[1:]))
    return {"bytes": keys * Hkv * d * 4 + T * Hq * (4 * d + (4 if case["lse"] else 0)),
            "flops": 4.0 * d * Hq * float(np.maximum(hi - lo, 0).sum())}


# ------------------------------------------------------------------------------------- the same in 64 bits
def _exact_turn(x, pos, case, back=False):
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
    turn = torch.polar(torch.full_like(angle, rule.get("magnitude", 1.0)), -angle if back else angle)[:, None]
    y = x.double().clone()
    half = rot // 2
    i0 = torch.arange(half, device="cuda") * 2 if case["inter"] else torch.arange(half, device="cuda")
    i1 = i0 + (1 if case["inter"] else half)
    z = torch.complex(y[..., i0].contiguous(), y[..., i1].contiguous()) * turn
    y[..., i0], y[..., i1] = z.real, z.imag
    return y


def _exact_attn(case, s):
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    g = Hq // Hkv
    n, kv = _lengths(case)
    _, lo, hi = _seen(case)
    O, lse, at = [], [], 0
    for b in range(case["B"]):
        nb, total = int(n[b]), int(n[b] + kv[b])
        pos = torch.arange(int(kv[b]), total, device="cuda").double()[:, None]
        key = torch.arange(total, device="cuda").double()
        first = torch.from_numpy(lo[at:at + nb]).cuda()[:, None]
        last = torch.from_numpy(hi[at:at + nb]).cuda()[:, None]
        hidden = (key < first) | (key >= last)
        o = torch.zeros((nb, Hq, d), dtype=torch.float64, device="cuda")
        e = torch.zeros((nb, Hq), dtype=torch.float64, device="cuda")
        for h in range(Hq):
            if case["page"]:
                ids = s["table"][b].long()
                k, v = (p[ids, h // g].reshape(-1, d)[:total].double() for p in (s["K"], s["V"]))
            else:
                k, v = (p[b, h // g, :total].double() for p in (s["K"], s["V"]))
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
    if case["kind"] == "rope":
        return {"Y": _exact_turn(s["X"], s["pos"], case, case["inverse"])}
    if case["kind"] == "append":
        Hq, Hkv = case["Hq"], case["Hkv"]
        x = s["qkv"].double()
        k, v = _exact_turn(x[:, Hq:Hq + Hkv], s["pos"], case), x[:, Hq + Hkv:]
        n, kv = _lengths(case)
        K, V = s["K"].double(), s["V"].double()
        at = 0
        for b in range(case["B"]):
            p = torch.arange(int(kv[b]), int(kv[b] + n[b]), device="cuda")
            rows = slice(at, at + int(n[b]))
            if case["page"]:
                ids = s["table"][b].long()[p // case["page"]]
                K[ids, :, p % case["page"]], V[ids, :, p % case["page"]] = k[rows], v[rows]
            else:
                K[b, :, p], V[b, :, p] = k[rows].transpose(0, 1), v[rows].transpose(0, 1)
            at += int(n[b])
        return {"Q": _exact_turn(x[:, :Hq], s["pos"], case), "K": K, "V": V}
    O, lse = _exact_attn(case, s)
    return {"O": O, "lse": lse} if case["lse"] else {"O": O}
