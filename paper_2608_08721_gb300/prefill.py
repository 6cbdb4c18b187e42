"""The prompt's way into a paged KV cache, and decoding from it, up to the verify round.

``PagedSequences`` owns what a serving loop keeps for a batch of sequences: every layer's page pools, the block
table, the sequences' lengths and the workspace. A step takes a ragged chunk of new tokens (a prompt, a part of one,
the one token of a decode step, or all of these side by side) through ``libraspec_rope_append_paged`` and
``libraspec_chunk_attn_paged``, layer by layer; the verify attention then reads the same pools. The cache may be held
in 8 bits (``libraspec_rope_append_q8_paged``, ``libraspec_chunk_attn_q8_paged``; a verified chain is then one more
chunk, and ``unpacked`` gives pools for the tree calls), query and key heads may be normed before they are rotated, and
a window may leave first tokens visible.

``python -m paper_2608_08721_gb300.prefill`` fills a cache with prompts of uneven length in chunks, decodes a few
tokens, verifies a drafted block on the result and prints what it compared; then the same in 8 bits with normed heads
and a window with sinks.
"""
from __future__ import annotations

from typing import List, Optional, Sequence

import torch

from . import binding


class Step:
    """One chunk of new tokens: how many each sequence has, their offsets in the packed rows and, with the sequences'
    lengths, the tokens' positions."""

    def __init__(self, n_new: Sequence[int], device, lengths: Optional[Sequence[int]] = None):
        self.n_new = [int(n) for n in n_new]
        offsets = [0]
        for n in self.n_new:
            offsets.append(offsets[-1] + n)
        self.T = offsets[-1]
        self.cu_new = torch.tensor(offsets, dtype=torch.int32).to(device)
        self.n_dev = torch.tensor(self.n_new, dtype=torch.int32).to(device)
        if lengths is not None:
            self.pos = torch.cat([torch.arange(a, a + n, dtype=torch.int32) for a, n in zip(lengths, self.n_new)]).to(device)


class PagedSequences:
    def __init__(self, n_layers: int, B: int, capacity: int, Hq: int, Hkv: int, head_dim: int,
                 freqs: binding.RopeFreqs, max_new: int, page_size: int = 64, interleaved: bool = False, device=None,
                 block: int = 0, norm: Optional[binding.QkNorm] = None):
        """capacity: keys per sequence; max_new: new tokens of a step, over all sequences, at most; block: tokens that
        share a scale in a cache of 8 bits (16, 32 or 64, a divisor of page_size; 0: a cache of bf16); norm: weights of
        the norm of query and key heads."""
        self.device = torch.device("cuda") if device is None else torch.device(device)
        self.B, self.Hq, self.Hkv, self.d, self.page_size = B, Hq, Hkv, head_dim, page_size
        self.freqs, self.interleaved, self.max_new = freqs, interleaved, max_new
        per = (capacity + page_size - 1) // page_size
        self.capacity = per * page_size
        bf = dict(dtype=torch.bfloat16, device=self.device)
        shape = (B * per, Hkv, page_size, head_dim)
        if block and page_size % block:
            raise ValueError("pages of %d keys do not hold whole blocks of %d" % (page_size, block))
        self.block, self.norm = block, norm
        if block:
            q8, u8 = (dict(dtype=t, device=self.device) for t in (torch.float8_e4m3fn, torch.uint8))
            exps = (B * per, Hkv, page_size // block)
            self.pools = [{"K8": torch.empty(shape, **q8), "V8": torch.empty(shape, **q8), "Ks": torch.empty(exps, **u8),
                           "Vs": torch.empty(exps, **u8)} for _ in range(n_layers)]
        else:
            self.pools = [{"Kp": torch.empty(shape, **bf), "Vp": torch.empty(shape, **bf)} for _ in range(n_layers)]
        # what is rotated already is appended by a rotation by nothing: of one pair, at position 0
        self.still = binding.RopeFreqs(2, device=self.device)
        self.no_pos = torch.zeros(max_new, dtype=torch.int32, device=self.device)
        self.block_table = torch.arange(B * per, dtype=torch.int32, device=self.device).view(B, per)
        self.lengths: List[int] = [0] * B
        self.kv_len = torch.zeros(B, dtype=torch.int32, device=self.device)
        self.ws = binding.ChunkWorkspace(max_new, B, Hq, Hkv, head_dim, device=self.device, q8=bool(block))

    def begin(self, n_new: Sequence[int]) -> Step:
        """A step of n_new[b] tokens for each sequence (0: none)."""
        if len(n_new) != self.B or min(n_new) < 0 or sum(n_new) > self.max_new:
            raise ValueError("n_new: a count for each of the %d sequences, %d tokens in all at most" % (self.B, self.max_new))
        for b, n in enumerate(n_new):
            if self.lengths[b] + n > self.capacity:
                raise ValueError("sequence %d: %d + %d keys do not fit %d" % (b, self.lengths[b], n, self.capacity))
        return Step(n_new, self.device, None if self.norm is None else self.lengths)

    def layer(self, l: int, qkv: torch.Tensor, step: Step, lse: Optional[torch.Tensor] = None, stream=None, **options):
        """Layer l of the step: qkv [T, Hq + 2 Hkv, d] (f32 or bf16, the projections' output) is rotated and appended,
        and its queries attend to the cache. options: libraspec_chunk_attn's (softcap, slopes, window, first_key,
        prefix_len, softmax_scale; None: not given) and sinks (first tokens that the window leaves visible; not with
        first_key). Returns O [T, Hq, d] bf16.

        On a stream other than the current one the layer runs behind what the current stream holds, and what the
        current stream gets next (the advance of the lengths in ``end`` among it) runs behind the layer."""
        if stream is None:
            return self._layer(l, qkv, step, lse, options)
        here = torch.cuda.current_stream()
        stream.wait_stream(here)
        with torch.cuda.stream(stream):  # (the rotated queries and O are the stream's own memory)
            O = self._layer(l, qkv, step, lse, options)
        here.wait_stream(stream)
        O.record_stream(here)
        return O

    def _layer(self, l, qkv, step, lse, options):
        Hq, Hkv, pool = self.Hq, self.Hkv, self.pools[l]
        if qkv.shape != (step.T, Hq + 2 * Hkv, self.d):  # (rows of no sequence would come back unwritten)
            raise ValueError("qkv must be [%d, %d, %d], got %s" % (step.T, Hq + 2 * Hkv, self.d, tuple(qkv.shape)))
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        options = {key: x for key, x in options.items() if x is not None}
        sinks = options.pop("sinks", 0)
        if sinks and "first_key" in options:
            raise ValueError("sinks and first_key exclude each other")
        if self.block:
            cache = (pool["K8"], pool["V8"], pool["Ks"], pool["Vs"], self.block_table, step.cu_new, self.kv_len)
            q = binding.libraspec_rope_append_q8_paged(q, k, v, *cache, self.freqs, self.ws, norm=self.norm,
                                                       interleaved=self.interleaved)
            return binding.libraspec_chunk_attn_q8_paged(q, *cache, self.ws, lse=lse, sinks=sinks, **options)[0]
        freqs, pos = self.freqs, None
        if self.norm is not None:
            qk = binding.libraspec_qk_norm_rope(qkv[:, :Hq + Hkv], Hq, self.norm, step.pos, freqs,
                                                interleaved=self.interleaved)
            q, k, freqs, pos = qk[:, :Hq], qk[:, Hq:], self.still, self.no_pos[:step.T]
        q = binding.libraspec_rope_append_paged(q, k, v, pool["Kp"], pool["Vp"], self.block_table, step.cu_new,
                                                self.kv_len, freqs, self.ws, pos=pos, interleaved=self.interleaved)
        attend = binding.libraspec_chunk_attn_paged
        if sinks:
            attend = binding.libraspec_sink_attn_paged
            options = {"window": 0, **options, "sinks": sinks}
        return attend(q, pool["Kp"], pool["Vp"], self.block_table, step.cu_new, self.kv_len, self.ws, lse=lse, **options)[0]

    def unpacked(self, l: int, extra: int = 0) -> dict:
        """Layer l of a cache in 8 bits as bf16 pools {"Kp", "Vp"} under the same block table, for the verify calls: each
        sequence's keys, and ``extra`` more that were appended behind them. (Exact: a scale is a power of two.)"""
        if not self.block:
            return self.pools[l]
        n = [a + extra for a in self.lengths]
        whole, pool = Step(n, self.device), self.pools[l]
        start = torch.zeros_like(self.kv_len)
        K, V = binding.libraspec_kv_read_q8_paged(pool["K8"], pool["V8"], pool["Ks"], pool["Vs"], self.block_table,
                                                  whole.cu_new, start, whole.T, self.ws)
        out = {k: torch.empty(pool["K8"].shape, dtype=torch.bfloat16, device=self.device) for k in ("Kp", "Vp")}
        binding.libraspec_rope_append_paged(None, K, V, out["Kp"], out["Vp"], self.block_table, whole.cu_new, start, self.still,
                                            self.ws, pos=torch.zeros(whole.T, dtype=torch.int32, device=self.device))
        return out

    def end(self, step: Step) -> None:
        """Every layer has had the step: its tokens count as the sequences' own."""
        self.kv_len += step.n_dev
        self.lengths = [a + n for a, n in zip(self.lengths, step.n_new)]

    def check(self) -> None:
        """Raises if a kernel reported a violation (synchronises)."""
        status = binding.libraspec_get_status(self.ws)
        if status:
            raise RuntimeError("device reported a violation: 0x%x" % status)


def run(prompts=(700, 3, 129, 1500), chunk=256, decode=3, K=7, n_layers=2, Hq=32, Hkv=8, d=128, seed=0) -> dict:
    """Prompts in chunks of at most ``chunk`` tokens each, ``decode`` tokens one at a time, then the verification of K
    drafted tokens by the verify attention and, for comparison, as one more chunk. Random projections."""
    device = torch.device("cuda")
    g = torch.Generator(device=device).manual_seed(seed)
    B = len(prompts)
    total = [p + decode + K + 1 for p in prompts]
    qkv = [[torch.randn((t, Hq + 2 * Hkv, d), generator=g, dtype=torch.bfloat16, device=device) for t in total]
           for _ in range(n_layers)]
    freqs = binding.RopeFreqs(d, theta=500000.0, device=device)

    def feed(seqs, n_new):
        step = seqs.begin(n_new)
        rows = [torch.cat([qkv[l][b][seqs.lengths[b]:seqs.lengths[b] + n_new[b]] for b in range(B)])
                for l in range(n_layers)]
        out = [seqs.layer(l, rows[l], step) for l in range(n_layers)]
        seqs.end(step)
        return out

    def fresh(max_new):
        return PagedSequences(n_layers, B, max(total), Hq, Hkv, d, freqs, max_new)

    whole = fresh(sum(total))
    feed(whole, list(prompts))
    seqs = fresh(max(B * chunk, B * (K + 1)))
    steps = 0
    while any(a < p for a, p in zip(seqs.lengths, prompts)):
        last = feed(seqs, [min(chunk, p - a) for a, p in zip(seqs.lengths, prompts)])
        steps += 1
    same = all(torch.equal(a[n][seqs.block_table[b].long()].transpose(0, 1).reshape(Hkv, -1, d)[:, :prompts[b]],
                           w[n][whole.block_table[b].long()].transpose(0, 1).reshape(Hkv, -1, d)[:, :prompts[b]])
               for a, w in zip(seqs.pools, whole.pools) for n in ("Kp", "Vp") for b in range(B))
    for _ in range(decode):
        last = feed(seqs, [1] * B)
    # the drafted block: its keys appended beyond the cache (the lengths stay), the verify attention over it
    kv = seqs.kv_len.clone()
    step = seqs.begin([K + 1] * B)
    rows = [torch.cat([qkv[l][b][seqs.lengths[b]:] for b in range(B)]) for l in range(n_layers)]
    chunk_out = [seqs.layer(l, rows[l], step) for l in range(n_layers)]
    pos = torch.cat([torch.arange(a, a + K + 1) for a in seqs.lengths]).to(torch.int32).to(device)
    layers = [{"Q": binding.libraspec_rope(rows[l][:, :Hq], pos, freqs).view(B, K + 1, Hq, d), **seqs.pools[l]}
              for l in range(n_layers)]
    vws = binding.Workspace(B, K, 1, Hq, Hkv, d, seqs.capacity, device=device)
    L = torch.full((B,), K, dtype=torch.int32, device=device)
    verify, _ = binding.libraspec_verify_attn_paged_layers(layers, seqs.block_table, kv, L, vws)
    seqs.check()
    whole.check()
    if binding.libraspec_get_status(vws):
        raise RuntimeError("device reported a violation (verify)")
    diff = max(float((a.view(B, K + 1, Hq, d).float() - b.float()).norm() / b.float().norm())
               for a, b in zip(chunk_out, verify))
    return {"chunks": steps, "cache_equal": same, "verify_rel_diff": diff, "decoded": last[0].shape[0]}


def run_q8(prompts=(700, 3, 129, 1500), chunk=256, decode=3, K=7, Hq=32, Hkv=8, d=128, block=16, window=512, sinks=4,
           seed=0) -> dict:
    """One layer with normed heads, a window and sinks over a cache in 8 bits: prompts in chunks, ``decode`` tokens one at
    a time, then K + 1 tokens as one chunk, and by the verify attention (no window) over the unpacked cache."""
    device = torch.device("cuda")
    g = torch.Generator(device=device).manual_seed(seed)
    B, total = len(prompts), [p + decode + K + 1 for p in prompts]
    qkv = [torch.randn((t, Hq + 2 * Hkv, d), generator=g, dtype=torch.bfloat16, device=device) for t in total]
    freqs = binding.RopeFreqs(d, theta=500000.0, device=device)
    norm = binding.QkNorm(*(1.0 + 0.2 * torch.randn((2, d), generator=g, device=device)).unbind())
    max_new = max(B * chunk, sum(total))
    both = [PagedSequences(1, B, max(total), Hq, Hkv, d, freqs, max_new, block=b, norm=norm, device=device)
            for b in (block, 0)]

    def feed(n_new, **options):
        out = []
        for seqs in both:
            step = seqs.begin(n_new)
            rows = torch.cat([x[a:a + n] for x, a, n in zip(qkv, seqs.lengths, n_new)])
            out.append(seqs.layer(0, rows, step, **options))
        return step, rows, out

    def rel(a, b):
        return float((a.float() - b.float()).norm() / b.float().norm())

    def advance(step):
        for seqs in both:
            seqs.end(step)

    worst = 0.0
    while any(a < p for a, p in zip(both[0].lengths, prompts)):
        step, _, (O8, O16) = feed([min(chunk, p - a) for a, p in zip(both[0].lengths, prompts)], window=window, sinks=sinks)
        worst = max(worst, rel(O8, O16))
        advance(step)
    for _ in range(decode):
        step, _, (O8, O16) = feed([1] * B, window=window, sinks=sinks)
        worst = max(worst, rel(O8, O16))
        advance(step)
    seqs = both[0]
    step, rows, (O8, _) = feed([K + 1] * B)
    Q = binding.libraspec_qk_norm_rope(rows[:, :Hq], Hq, norm, step.pos, freqs).view(B, K + 1, Hq, d)
    vws = binding.Workspace(B, K, 1, Hq, Hkv, d, seqs.capacity, device=device)
    L = torch.full((B,), K, dtype=torch.int32, device=device)
    verify, _ = binding.libraspec_verify_attn_paged_layers([{"Q": Q, **seqs.unpacked(0, K + 1)}], seqs.block_table, seqs.kv_len,
                                                           L, vws)
    for s in both:
        s.check()
    if binding.libraspec_get_status(vws):
        raise RuntimeError("device reported a violation (verify)")
    return {"rel_to_16_bits": worst, "verify_rel_diff": rel(O8.view(B, K + 1, Hq, d), verify[0])}


def main() -> None:
    r = run()
    print("prompts in %d chunks; the cache of one whole step: %s; verify attention against the chunk's: %.1e apart" % (
        r["chunks"], "equal" if r["cache_equal"] else "DIFFERENT", r["verify_rel_diff"]))
    r = run_q8()
    print("in 8 bits, with normed heads, a window and sinks: %.1e from the 16-bit cache's; verify attention of the unpacked "
          "cache against the chunk's: %.1e apart" % (r["rel_to_16_bits"], r["verify_rel_diff"]))


if __name__ == "__main__":
    main()
