"""Thin ctypes binding of libraspec.so (include/libraspec.h).

Functions carry the C names and take torch tensors; they only check and
marshal arguments (dtype, device, contiguity, shapes) and pass the current
CUDA stream. Every step of the verify round runs in the library's kernels.
A missing or unloadable library raises; there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libraspec.so")

OK, EINVAL, EUNSUPPORTED, ECUDA, EDEVICE = 0, -1, -2, -3, -4
ST_BAD_LENGTH, ST_BAD_COST, ST_KV_OVERFLOW, ST_BAD_TOKEN, ST_TIMEOUT, ST_MISSING_INPUT = 1, 2, 4, 8, 16, 32
ST_BAD_PAGE, ST_BAD_TREE = 0x40, 0x80
MAX_K = 64
MAX_TREE_NODES = 512

# Every entry point declared in include/libraspec.h, with its ctypes signature.
_P, _I, _U32, _U64, _F, _SZ = (ctypes.c_void_p, ctypes.c_int, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_float,
                               ctypes.c_size_t)
_I64, _D = ctypes.c_int64, ctypes.c_double
_Q8_HEAD = [_P, _I64] * 3 + [_P] * 4 + [_F, _P, _P, _F] + [_I] * 7 + [_P] * 5  # of the appends to a cache in 8 bits
SIGNATURES = {
    "libraspec_version": (ctypes.c_char_p, []),
    "libraspec_status_string": (ctypes.c_char_p, [_I]),
    "libraspec_workspace_size": (_SZ, [_I, _I, _I, _I, _I, _I, _I]),
    "libraspec_workspace_init": (_I, [_P, _SZ, _P]),
    "libraspec_get_status": (_I, [_P, _P, _P]),
    "libraspec_selftest_wait": (_I, [_P, _U64, _P, _P, _SZ, _P]),
    "libraspec_confidence": (_I, [_P, _P, _P, _I, _I, _I, _P, _P, _P, _SZ, _P]),
    "libraspec_confidence_bf16": (_I, [_P, _P, _P, _I, _I, _I, _P, _P, _P, _SZ, _P]),
    "libraspec_confidence_noalloc": (_I, [_P, _P, _P, _I, _I, _I, _P, _P, _P, _P]),
    "libraspec_confidence_select": (_I, [_P, _P, _P, _P, _I, _I, _I, _P, _P, _P, _P, _SZ, _P]),
    "libraspec_confidence_select_bf16": (_I, [_P, _P, _P, _P, _I, _I, _I, _P, _P, _P, _P, _SZ, _P]),
    "libraspec_select_lengths": (_I, [_P, _P, _I, _I, _P, _P, _SZ, _P]),
    "libraspec_select_alpha": (_I, [_P, _I, _I, _I, _F, _P, _P, _P]),
    "libraspec_verify_attn": (_I, [_P, _P, _P, _P, _P, _I, _I, _I, _I, _I, _I, _F, _P, _P, _P, _SZ, _P]),
    "libraspec_verify_attn_layers": (_I, [_P, _P, _P, _I, _P, _P, _I, _I, _I, _I, _I, _I, _F, _P, _P, _P, _SZ, _P]),
    "libraspec_verify_attn_paged_layers": (_I, [_P, _P, _P, _I, _P, _I, _I, _I, _P, _P, _I, _I, _I, _I, _I, _F, _P, _P,
                                                _P, _SZ, _P]),
    "libraspec_verify_attn_tree_layers": (_I, [_P, _P, _P, _I, _P, _P, _P, _I, _I, _I, _I, _I, _I, _F, _P, _P, _P,
                                               _SZ, _P]),
    "libraspec_verify_attn_tree_paged_layers": (_I, [_P, _P, _P, _I, _P, _P, _I, _I, _I, _P, _P, _I, _I, _I, _I, _I,
                                                     _F, _P, _P, _P, _SZ, _P]),
    "libraspec_accept_tree_greedy": (_I, [_P, _P, _P, _P, _I, _I, _I, _P, _P, _P, _P, _SZ, _P]),
    "libraspec_accept_tree_greedy_bf16": (_I, [_P, _P, _P, _P, _I, _I, _I, _P, _P, _P, _P, _SZ, _P]),
    "libraspec_accept_tree": (_I, [_P, _P, _P, _P, _P, _I, _I, _I, _U64, _U64, _U32, _P, _P, _P, _P, _SZ, _P]),
    "libraspec_accept_tree_bf16": (_I, [_P, _P, _P, _P, _P, _I, _I, _I, _U64, _U64, _U32, _P, _P, _P, _P, _SZ,
                                        _P]),
    "libraspec_verify_round_staged": (_I, [_P] * 18 + [_I, _P] + [_I] * 7 + [_F, _U64, _U64, _U32] + [_P] * 6 +
                                      [_SZ, _P]),
    "libraspec_verify_round_staged_bf16": (_I, [_P] * 18 + [_I, _P] + [_I] * 7 + [_F, _U64, _U64, _U32] + [_P] * 6 +
                                           [_SZ, _P]),
    "libraspec_lm_head_workspace_size": (_SZ, [_I, _I]),
    "libraspec_lm_head_stats": (_I, [_P, _P, _P, _I, _P, _I, _I, _I, _P, _P, _P, _P, _SZ, _P]),
    "libraspec_kv_append": (_I, [_P, _P, _P, _I, _P, _I, _I, _I, _I, _I, _P, _SZ, _P]),
    "libraspec_kv_append_paged": (_I, [_P, _P, _P, _I, _P, _I, _I, _I, _P, _I, _I, _I, _I, _P, _SZ, _P]),
    "libraspec_rope_frequencies": (_I, [_I, _D, _I, _D, _D, _D, _D, _P]),
    "libraspec_rope": (_I, [_P, _I64, _P, _P, _F] + [_I] * 6 + [_P, _I64, _P]),
    "libraspec_rope_bf16": (_I, [_P, _I64, _P, _P, _F] + [_I] * 6 + [_P, _I64, _P]),
    "libraspec_rope_append": (_I, [_P, _I64] * 3 + [_P] * 4 + [_F] + [_I] * 7 + [_P] * 3 + [_I, _P, _SZ, _P]),
    "libraspec_rope_append_bf16": (_I, [_P, _I64] * 3 + [_P] * 4 + [_F] + [_I] * 7 + [_P] * 3 + [_I, _P, _SZ, _P]),
    "libraspec_rope_append_paged": (_I, [_P, _I64] * 3 + [_P] * 4 + [_F] + [_I] * 7 + [_P] * 4 + [_I] * 3 +
                                    [_P, _SZ, _P]),
    "libraspec_rope_append_paged_bf16": (_I, [_P, _I64] * 3 + [_P] * 4 + [_F] + [_I] * 7 + [_P] * 4 + [_I] * 3 +
                                         [_P, _SZ, _P]),
    "libraspec_qk_norm_rope": (_I, [_P, _I64, _P, _P, _F, _P, _P, _F] + [_I] * 6 + [_P, _I64, _P]),
    "libraspec_qk_norm_rope_bf16": (_I, [_P, _I64, _P, _P, _F, _P, _P, _F] + [_I] * 6 + [_P, _I64, _P]),
    "libraspec_rope_append_q8": (_I, _Q8_HEAD + [_I, _I, _P, _SZ, _P]),
    "libraspec_rope_append_q8_bf16": (_I, _Q8_HEAD + [_I, _I, _P, _SZ, _P]),
    "libraspec_rope_append_q8_paged": (_I, _Q8_HEAD + [_P, _I, _I, _I, _I, _P, _SZ, _P]),
    "libraspec_rope_append_q8_paged_bf16": (_I, _Q8_HEAD + [_P, _I, _I, _I, _I, _P, _SZ, _P]),
    "libraspec_kv_read_q8": (_I, [_P] * 6 + [_I] * 6 + [_P, _P, _P, _SZ, _P]),
    "libraspec_kv_read_q8_paged": (_I, [_P] * 5 + [_I] * 3 + [_P] * 2 + [_I] * 5 + [_P, _P, _P, _SZ, _P]),
    "libraspec_chunk_workspace_size": (_SZ, [_I] * 5),
    "libraspec_chunk_workspace_size_bf16": (_SZ, [_I] * 5),
    "libraspec_chunk_attn": (_I, [_P] * 5 + [_I] * 6 + [_F] + [_P] * 4 + [_SZ, _P]),
    "libraspec_chunk_attn_paged": (_I, [_P] * 4 + [_I] * 3 + [_P] * 2 + [_I] * 5 + [_F] + [_P] * 4 + [_SZ, _P]),
    "libraspec_sink_attn": (_I, [_P] * 5 + [_I] * 6 + [_F, _P, _I] + [_P] * 3 + [_SZ, _P]),
    "libraspec_sink_attn_paged": (_I, [_P] * 4 + [_I] * 3 + [_P] * 2 + [_I] * 5 + [_F, _P, _I] + [_P] * 3 + [_SZ, _P]),
    "libraspec_chunk_attn_q8": (_I, [_P] * 7 + [_I] * 7 + [_F, _P, _I] + [_P] * 3 + [_SZ, _P]),
    "libraspec_chunk_attn_q8_paged": (_I, [_P] * 6 + [_I] * 3 + [_P] * 2 + [_I] * 6 + [_F, _P, _I] + [_P] * 3 + [_SZ, _P]),
    "libraspec_accept": (_I, [_P, _P, _P, _P, _P, _P, _P, _I, _I, _I, _U64, _U64, _U32, _P, _P, _P, _SZ, _P]),
    "libraspec_accept_bf16": (_I, [_P, _P, _P, _P, _P, _P, _P, _I, _I, _I, _U64, _U64, _U32, _P, _P, _P, _SZ, _P]),
    "libraspec_verify_round": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _I, _P, _I, _I, _I, _I, _I, _I, _I,
                                    _F, _U64, _U64, _U32, _P, _P, _P, _P, _P, _P, _SZ, _P]),
    "libraspec_verify_round_bf16": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _I, _P, _I, _I, _I, _I, _I, _I,
                                         _I, _F, _U64, _U64, _U32, _P, _P, _P, _P, _P, _P, _SZ, _P]),
}

_lib = None


class LibraspecError(RuntimeError):
    def __init__(self, what: str, status: int):
        super().__init__("%s failed: %s (%d)" % (what, _status_name(status), status))
        self.status = status


def _status_name(status: int) -> str:
    return {OK: "ok", EINVAL: "invalid argument", EUNSUPPORTED: "unsupported shape", ECUDA: "CUDA error",
            EDEVICE: "device-reported violation"}.get(status, "unknown")


def load() -> ctypes.CDLL:
    """Load libraspec.so (built by build.py); raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("libraspec.so is not built (%s); run `python -m paper_2608_08721_gb300.build` or "
                           "__graft_entry__.build()" % LIB_PATH)
    lib = ctypes.CDLL(LIB_PATH)
    for name, (res, args) in SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def _check(rc: int, what: str) -> None:
    if rc != OK:
        raise LibraspecError(what, rc)


# The current stream's handle without making a Stream object (3.0 us -> 0.5); not a public function of torch.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream: Optional[torch.cuda.Stream]) -> int:
    """The handle of the stream, or of the current one."""
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _req_dev_or_pinned(t: torch.Tensor, dtype, name: str, shape=None) -> torch.Tensor:
    """_req, or the same checks on a pinned host tensor (read in place by the kernels)."""
    if isinstance(t, torch.Tensor) and not t.is_cuda:
        if not t.is_pinned():
            raise ValueError("%s must be on a CUDA device or in pinned host memory" % name)
        if t.dtype != dtype or not t.is_contiguous() or (shape is not None and tuple(t.shape) != tuple(shape)):
            raise ValueError("%s: dtype %s, contiguous, shape %s required" % (name, dtype, shape))
        return t
    return _req(t, dtype, name, shape)


def _req(t: torch.Tensor, dtype, name: str, shape=None) -> torch.Tensor:
    # every condition at once; what fails is named below (a list of sizes, unequal to a torch.Size, passes there)
    if (isinstance(t, torch.Tensor) and t.dtype == dtype and t.is_cuda and t.is_contiguous()
            and (shape is None or t.shape == shape)):
        return t
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch tensor" % name)
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if not t.is_cuda:
        raise ValueError("%s must be on a CUDA device" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    return t


class Workspace:
    """Device scratch for one round's shapes (a zero-filled torch buffer)."""

    def __init__(self, B, K, V, Hq=1, Hkv=1, head_dim=64, S_cap=1, device=None):
        lib = load()
        self.nbytes = int(lib.libraspec_workspace_size(B, K, V, Hq, Hkv, head_dim, S_cap))
        if self.nbytes == 0:
            raise ValueError("invalid workspace shapes")
        dev = torch.device("cuda") if device is None else torch.device(device)
        self.buf = torch.zeros(self.nbytes, dtype=torch.uint8, device=dev)
        if self.buf.data_ptr() % 256:
            raise RuntimeError("workspace allocation is not 256-byte aligned")
        self.shapes = (B, K, V, Hq, Hkv, head_dim, S_cap)

    @property
    def ptr(self) -> int:
        return self.buf.data_ptr()


def libraspec_version() -> str:
    return load().libraspec_version().decode()


def libraspec_workspace_size(B, K, V, Hq, Hkv, head_dim, S_cap) -> int:
    return int(load().libraspec_workspace_size(B, K, V, Hq, Hkv, head_dim, S_cap))


def libraspec_get_status(ws: Workspace, stream=None) -> int:
    out = ctypes.c_int32(0)
    rc = load().libraspec_get_status(ctypes.c_void_p(ws.ptr), _stream(stream), ctypes.byref(out))
    if rc not in (OK, EDEVICE):
        _check(rc, "libraspec_get_status")
    return int(out.value)


def libraspec_selftest_wait(flag, limit_ns: int, ws: Workspace, observed=None, stream=None) -> torch.Tensor:
    """The library's bounded wait on the device word ``flag`` (uint32 stored as int32 [1]) with a limit of
    limit_ns; returns ``observed`` (int32 [1] on the device): 1 if the flag was seen, 0 if the wait gave up
    (LIBRASPEC_ST_TIMEOUT is then set in the workspace's status)."""
    _req(flag, torch.int32, "flag", (1,))
    observed = torch.empty((1,), dtype=torch.int32, device=flag.device) if observed is None else _req(
        observed, torch.int32, "observed", (1,))
    rc = load().libraspec_selftest_wait(_ptr(flag), int(limit_ns), _ptr(observed), ws.ptr, ws.nbytes,
                                        _stream(stream))
    _check(rc, "libraspec_selftest_wait")
    return observed


def libraspec_confidence(draft_logits, draft_tokens, temperature, ws: Workspace, conf=None, dstat=None,
                         stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    B, K, V = draft_logits.shape
    bf16 = draft_logits.dtype == torch.bfloat16  # libraspec_confidence_bf16
    _req(draft_logits, torch.bfloat16 if bf16 else torch.float32, "draft_logits")
    _req(draft_tokens, torch.int32, "draft_tokens", (B, K))
    _req(temperature, torch.float32, "temperature", (B,))
    dev = draft_logits.device
    conf = torch.empty((B, K), dtype=torch.float32, device=dev) if conf is None else _req(conf, torch.float32,
                                                                                          "conf", (B, K))
    dstat = torch.empty((B, K, 2), dtype=torch.float32, device=dev) if dstat is None else _req(
        dstat, torch.float32, "dstat", (B, K, 2))
    name = "libraspec_confidence_bf16" if bf16 else "libraspec_confidence"
    rc = getattr(load(), name)(_ptr(draft_logits), _ptr(draft_tokens), _ptr(temperature), B, K, V, _ptr(conf),
                               _ptr(dstat), ws.ptr, ws.nbytes, _stream(stream))
    _check(rc, name)
    return conf, dstat


NOALLOC_MAX_ROWS = 4096


def libraspec_confidence_noalloc(draft_logits, draft_tokens, temperature, conf, dstat=None, status=None,
                                 stream=None) -> None:
    """libraspec_confidence with the library's static scratch instead of a
    workspace. Allocates nothing: the outputs (conf [B,K], optional dstat
    [B,K,2], optional status [1] int32) are caller tensors."""
    B, K, V = draft_logits.shape
    _req(draft_logits, torch.float32, "draft_logits")
    _req(draft_tokens, torch.int32, "draft_tokens", (B, K))
    _req(temperature, torch.float32, "temperature", (B,))
    _req(conf, torch.float32, "conf", (B, K))
    if dstat is not None:
        _req(dstat, torch.float32, "dstat", (B, K, 2))
    if status is not None:
        _req(status, torch.int32, "status", (1,))
    if B * K > NOALLOC_MAX_ROWS:
        raise ValueError("libraspec_confidence_noalloc: B*K = %d drafter rows exceeds the static scratch limit "
                         "of %d rows; use libraspec_confidence with a workspace" % (B * K, NOALLOC_MAX_ROWS))
    rc = load().libraspec_confidence_noalloc(_ptr(draft_logits), _ptr(draft_tokens), _ptr(temperature), B, K, V,
                                             _ptr(conf), _ptr(dstat), _ptr(status), _stream(stream))
    _check(rc, "libraspec_confidence_noalloc")


def libraspec_confidence_select(draft_logits, draft_tokens, temperature, cost_table, ws: Workspace, conf=None,
                                dstat=None, L=None, stream=None):
    """Confidence and the Thm. 4 selection in one launch: (conf [B,K], dstat [B,K,2], L [B])."""
    B, K, V = draft_logits.shape
    bf16 = draft_logits.dtype == torch.bfloat16
    _req(draft_logits, torch.bfloat16 if bf16 else torch.float32, "draft_logits")
    _req(draft_tokens, torch.int32, "draft_tokens", (B, K))
    _req(temperature, torch.float32, "temperature", (B,))
    _req(cost_table, torch.float32, "cost_table", (K + 1,))
    dev = draft_logits.device
    conf = torch.empty((B, K), dtype=torch.float32, device=dev) if conf is None else conf
    dstat = torch.empty((B, K, 2), dtype=torch.float32, device=dev) if dstat is None else dstat
    L = torch.empty((B,), dtype=torch.int32, device=dev) if L is None else L
    name = "libraspec_confidence_select_bf16" if bf16 else "libraspec_confidence_select"
    rc = getattr(load(), name)(_ptr(draft_logits), _ptr(draft_tokens), _ptr(temperature), _ptr(cost_table), B, K, V,
                               _ptr(conf), _ptr(dstat), _ptr(L), ws.ptr, ws.nbytes, _stream(stream))
    _check(rc, name)
    return conf, dstat, L


def libraspec_select_lengths(conf, cost_table, ws: Workspace, L=None, stream=None) -> torch.Tensor:
    B, K = conf.shape
    _req(conf, torch.float32, "conf")
    _req(cost_table, torch.float32, "cost_table", (K + 1,))
    L = torch.empty((B,), dtype=torch.int32, device=conf.device) if L is None else _req(L, torch.int32, "L", (B,))
    rc = load().libraspec_select_lengths(_ptr(conf), _ptr(cost_table), B, K, _ptr(L), ws.ptr, ws.nbytes,
                                         _stream(stream))
    _check(rc, "libraspec_select_lengths")
    return L


def libraspec_select_alpha(conf, block_size: int, alpha: float, L=None, n_blocks=None, stream=None):
    """Algorithm 1's alpha-mode search: L[B] and blocks drafted[B] (int32, device)."""
    B, K = conf.shape
    _req(conf, torch.float32, "conf")
    L = torch.empty((B,), dtype=torch.int32, device=conf.device) if L is None else _req(L, torch.int32, "L", (B,))
    if n_blocks is None:
        n_blocks = torch.empty((B,), dtype=torch.int32, device=conf.device)
    else:
        _req(n_blocks, torch.int32, "n_blocks", (B,))
    rc = load().libraspec_select_alpha(_ptr(conf), B, K, int(block_size), float(alpha), _ptr(L), _ptr(n_blocks),
                                       _stream(stream))
    _check(rc, "libraspec_select_alpha")
    return L, n_blocks


def libraspec_verify_attn(Q, Kc, Vc, kv_len, L, ws: Workspace, softmax_scale=None, O=None, lse=None,
                          want_lse=False, stream=None):
    B, K1, Hq, D = Q.shape
    _, Hkv, S_cap, D2 = Kc.shape
    _req(Q, torch.bfloat16, "Q")
    _req(Kc, torch.bfloat16, "Kc", (B, Hkv, S_cap, D))
    _req(Vc, torch.bfloat16, "Vc", (B, Hkv, S_cap, D))
    _req(kv_len, torch.int32, "kv_len", (B,))
    _req(L, torch.int32, "L", (B,))
    if softmax_scale is None:
        softmax_scale = D ** -0.5
    O = torch.empty_like(Q) if O is None else _req(O, torch.bfloat16, "O", Q.shape)
    if want_lse and lse is None:
        lse = torch.empty((B, K1, Hq), dtype=torch.float32, device=Q.device)
    rc = load().libraspec_verify_attn(_ptr(Q), _ptr(Kc), _ptr(Vc), _ptr(kv_len), _ptr(L), B, K1 - 1, Hq, Hkv, D,
                                      S_cap, float(softmax_scale), _ptr(O), _ptr(lse), ws.ptr, ws.nbytes,
                                      _stream(stream))
    _check(rc, "libraspec_verify_attn")
    return O, lse


def libraspec_verify_attn_layers(layers, kv_len, L, ws: Workspace, softmax_scale=None, want_lse=False,
                                 stream=None):
    """layers: sequence of dicts with Q, Kc, Vc (and optionally O, lse). Returns (O list, lse list or None)."""
    return _attn_layers(layers, None, kv_len, L, ws, softmax_scale, want_lse, stream)


def libraspec_verify_attn_tree_layers(layers, parent, kv_len, L, ws: Workspace, softmax_scale=None, want_lse=False,
                                      stream=None):
    """Draft-tree verify attention; parent [B, K+1] int32 (parent[b, t] < t). As libraspec_verify_attn_layers."""
    return _attn_layers(layers, parent, kv_len, L, ws, softmax_scale, want_lse, stream)


def _check_parent(parent, B, K1):
    _req(parent, torch.int32, "parent", (B, K1))


def _attn_layers(layers, parent, kv_len, L, ws, softmax_scale, want_lse, stream):
    n = len(layers)
    if n == 0:
        return [], None
    B, K1, Hq, D = layers[0]["Q"].shape
    _, Hkv, S_cap, _ = layers[0]["Kc"].shape
    _check_layers(layers, "Kc", "Vc", (B, K1, Hq, D), (B, Hkv, S_cap, D))
    _req(kv_len, torch.int32, "kv_len", (B,))
    _req(L, torch.int32, "L", (B,))
    if parent is not None:
        _check_parent(parent, B, K1)
    if softmax_scale is None:
        softmax_scale = D ** -0.5
    outs = [lay.get("O") if lay.get("O") is not None else torch.empty_like(lay["Q"]) for lay in layers]
    lses = None
    if want_lse:
        lses = [lay.get("lse") if lay.get("lse") is not None else
                torch.empty((B, K1, Hq), dtype=torch.float32, device=layers[0]["Q"].device) for lay in layers]
    args = [_ptr_array([l["Q"] for l in layers]), _ptr_array([l["Kc"] for l in layers]),
            _ptr_array([l["Vc"] for l in layers]), n]
    name = "libraspec_verify_attn_layers"
    if parent is not None:
        args.append(_ptr(parent))
        name = "libraspec_verify_attn_tree_layers"
    rc = getattr(load(), name)(
        *args, _ptr(kv_len), _ptr(L), B, K1 - 1, Hq, Hkv, D, S_cap, float(softmax_scale), _ptr_array(outs),
        _ptr_array(lses) if lses is not None else None, ws.ptr, ws.nbytes, _stream(stream))
    _check(rc, name)
    return outs, lses


def libraspec_verify_attn_paged_layers(layers, block_table, kv_len, L, ws: Workspace, softmax_scale=None,
                                       want_lse=False, stream=None):
    """layers: dicts with Q [B,K+1,Hq,d] and page pools Kp, Vp [n_pages,Hkv,page_size,d] (optionally O,
    lse); block_table [B, max_pages] int32. Returns (O list, lse list or None)."""
    return _attn_paged_layers(layers, None, block_table, kv_len, L, ws, softmax_scale, want_lse, stream)


def libraspec_verify_attn_tree_paged_layers(layers, parent, block_table, kv_len, L, ws: Workspace,
                                            softmax_scale=None, want_lse=False, stream=None):
    """Draft-tree verify attention over a paged cache; parent [B, K+1] int32."""
    return _attn_paged_layers(layers, parent, block_table, kv_len, L, ws, softmax_scale, want_lse, stream)


def _attn_paged_layers(layers, parent, block_table, kv_len, L, ws, softmax_scale, want_lse, stream):
    n = len(layers)
    if n == 0:
        return [], None
    B, K1, Hq, D = layers[0]["Q"].shape
    n_pages, Hkv, page_size, _ = layers[0]["Kp"].shape
    _check_layers(layers, "Kp", "Vp", (B, K1, Hq, D), (n_pages, Hkv, page_size, D))
    _req(block_table, torch.int32, "block_table")
    if block_table.dim() != 2 or block_table.shape[0] != B:
        raise ValueError("block_table must be [B, max_pages]")
    max_pages = block_table.shape[1]
    _req(kv_len, torch.int32, "kv_len", (B,))
    _req(L, torch.int32, "L", (B,))
    if parent is not None:
        _check_parent(parent, B, K1)
    if softmax_scale is None:
        softmax_scale = D ** -0.5
    outs = [lay.get("O") if lay.get("O") is not None else torch.empty_like(lay["Q"]) for lay in layers]
    lses = None
    if want_lse:
        lses = [lay.get("lse") if lay.get("lse") is not None else
                torch.empty((B, K1, Hq), dtype=torch.float32, device=layers[0]["Q"].device) for lay in layers]
    args = [_ptr_array([l["Q"] for l in layers]), _ptr_array([l["Kp"] for l in layers]),
            _ptr_array([l["Vp"] for l in layers]), n]
    name = "libraspec_verify_attn_paged_layers"
    if parent is not None:
        args.append(_ptr(parent))
        name = "libraspec_verify_attn_tree_paged_layers"
    rc = getattr(load(), name)(
        *args, _ptr(block_table), max_pages, page_size, n_pages, _ptr(kv_len), _ptr(L), B, K1 - 1, Hq, Hkv, D,
        float(softmax_scale), _ptr_array(outs), _ptr_array(lses) if lses is not None else None, ws.ptr, ws.nbytes,
        _stream(stream))
    _check(rc, name)
    return outs, lses


def libraspec_accept(target_logits, draft_logits, draft_tokens, conf, dstat, L, temperature, seed: int,
                     ws: Workspace, round_offset: int = 0, seq_offset: int = 0, n_accepted=None, bonus_token=None,
                     stream=None):
    B, K1, V = target_logits.shape
    K = K1 - 1
    bf16 = target_logits.dtype == torch.bfloat16  # libraspec_accept_bf16: both logit tensors bf16
    ldt = torch.bfloat16 if bf16 else torch.float32
    _req(target_logits, ldt, "target_logits")
    _req(draft_logits, ldt, "draft_logits", (B, K, V))
    _req(draft_tokens, torch.int32, "draft_tokens", (B, K))
    if conf is not None:
        _req(conf, torch.float32, "conf", (B, K))
    if dstat is not None:
        _req(dstat, torch.float32, "dstat", (B, K, 2))
    _req(L, torch.int32, "L", (B,))
    _req(temperature, torch.float32, "temperature", (B,))
    dev = target_logits.device
    n_accepted = torch.empty((B,), dtype=torch.int32, device=dev) if n_accepted is None else n_accepted
    bonus_token = torch.empty((B,), dtype=torch.int32, device=dev) if bonus_token is None else bonus_token
    name = "libraspec_accept_bf16" if bf16 else "libraspec_accept"
    rc = getattr(load(), name)(_ptr(target_logits), _ptr(draft_logits), _ptr(draft_tokens), _ptr(conf), _ptr(dstat),
                               _ptr(L), _ptr(temperature), B, K, V, int(seed) & (2**64 - 1), int(round_offset),
                               int(seq_offset), _ptr(n_accepted), _ptr(bonus_token), ws.ptr, ws.nbytes,
                               _stream(stream))
    _check(rc, name)
    return n_accepted, bonus_token


def libraspec_accept_tree_greedy(target_logits, draft_tokens, parent, L, ws: Workspace, n_accepted=None,
                                 last_node=None, bonus_token=None, stream=None):
    """Greedy walk of a draft tree. Returns (n_accepted, last_node, bonus_token), int32 [B] each."""
    B, K1, V = target_logits.shape
    K = K1 - 1
    bf16 = target_logits.dtype == torch.bfloat16
    _req(target_logits, torch.bfloat16 if bf16 else torch.float32, "target_logits")
    _req(draft_tokens, torch.int32, "draft_tokens", (B, K))
    _check_parent(parent, B, K1)
    _req(L, torch.int32, "L", (B,))
    dev = target_logits.device
    n_accepted = torch.empty((B,), dtype=torch.int32, device=dev) if n_accepted is None else n_accepted
    last_node = torch.empty((B,), dtype=torch.int32, device=dev) if last_node is None else last_node
    bonus_token = torch.empty((B,), dtype=torch.int32, device=dev) if bonus_token is None else bonus_token
    name = "libraspec_accept_tree_greedy_bf16" if bf16 else "libraspec_accept_tree_greedy"
    rc = getattr(load(), name)(_ptr(target_logits), _ptr(draft_tokens), _ptr(parent), _ptr(L), B, K, V,
                               _ptr(n_accepted), _ptr(last_node), _ptr(bonus_token), ws.ptr, ws.nbytes,
                               _stream(stream))
    _check(rc, name)
    return n_accepted, last_node, bonus_token


def libraspec_accept_tree(target_logits, draft_tokens, parent, L, temperature, seed: int, ws: Workspace,
                          round_offset: int = 0, seq_offset: int = 0, n_accepted=None, last_node=None,
                          bonus_token=None, stream=None):
    """Walk of a draft tree drawing the target's token at each node (greedy where temperature is 0).
    Returns (n_accepted, last_node, bonus_token), int32 [B] each."""
    B, K1, V = target_logits.shape
    K = K1 - 1
    bf16 = target_logits.dtype == torch.bfloat16
    _req(target_logits, torch.bfloat16 if bf16 else torch.float32, "target_logits")
    _req(draft_tokens, torch.int32, "draft_tokens", (B, K))
    _check_parent(parent, B, K1)
    _req(L, torch.int32, "L", (B,))
    _req(temperature, torch.float32, "temperature", (B,))
    dev = target_logits.device
    n_accepted = torch.empty((B,), dtype=torch.int32, device=dev) if n_accepted is None else n_accepted
    last_node = torch.empty((B,), dtype=torch.int32, device=dev) if last_node is None else last_node
    bonus_token = torch.empty((B,), dtype=torch.int32, device=dev) if bonus_token is None else bonus_token
    name = "libraspec_accept_tree_bf16" if bf16 else "libraspec_accept_tree"
    rc = getattr(load(), name)(_ptr(target_logits), _ptr(draft_tokens), _ptr(parent), _ptr(L), _ptr(temperature), B,
                               K, V, int(seed) & (2**64 - 1), int(round_offset), int(seq_offset), _ptr(n_accepted),
                               _ptr(last_node), _ptr(bonus_token), ws.ptr, ws.nbytes, _stream(stream))
    _check(rc, name)
    return n_accepted, last_node, bonus_token


def libraspec_kv_append(kv_new, caches, kv_len, ws: Workspace, block_table=None, stream=None) -> None:
    """kv_new [n_layers, 2, B, Hkv, T, d] bf16; caches: per layer {"Kc", "Vc"} (dense [B,Hkv,S_cap,d]) or
    {"Kp", "Vp"} (page pools [n_pages,Hkv,page_size,d], with block_table [B, max_pages])."""
    n_layers, two, B, Hkv, T, d = kv_new.shape
    if two != 2 or len(caches) != n_layers:
        raise ValueError("kv_new must be [n_layers, 2, B, Hkv, T, d] with one cache per layer")
    _req(kv_new, torch.bfloat16, "kv_new")
    _req(kv_len, torch.int32, "kv_len", (B,))
    if block_table is None:
        S_cap = caches[0]["Kc"].shape[2] if n_layers else 1
        for i, c in enumerate(caches):
            _req(c["Kc"], torch.bfloat16, "Kc[%d]" % i, (B, Hkv, S_cap, d))
            _req(c["Vc"], torch.bfloat16, "Vc[%d]" % i, (B, Hkv, S_cap, d))
        rc = load().libraspec_kv_append(_ptr(kv_new), _ptr_array([c["Kc"] for c in caches]),
                                        _ptr_array([c["Vc"] for c in caches]), n_layers, _ptr(kv_len), B, T, Hkv,
                                        d, S_cap, ws.ptr, ws.nbytes, _stream(stream))
        _check(rc, "libraspec_kv_append")
        return
    _req(block_table, torch.int32, "block_table")
    n_pages, _, page_size, _ = caches[0]["Kp"].shape
    for i, c in enumerate(caches):
        _req(c["Kp"], torch.bfloat16, "Kp[%d]" % i, (n_pages, Hkv, page_size, d))
        _req(c["Vp"], torch.bfloat16, "Vp[%d]" % i, (n_pages, Hkv, page_size, d))
    rc = load().libraspec_kv_append_paged(_ptr(kv_new), _ptr_array([c["Kp"] for c in caches]),
                                          _ptr_array([c["Vp"] for c in caches]), n_layers, _ptr(block_table),
                                          block_table.shape[1], page_size, n_pages, _ptr(kv_len), B, T, Hkv, d,
                                          ws.ptr, ws.nbytes, _stream(stream))
    _check(rc, "libraspec_kv_append_paged")


class LmHeadWorkspace:
    """Device scratch of libraspec_lm_head_stats for M rows and a vocabulary of V."""

    def __init__(self, M, V, device=None):
        self.nbytes = int(load().libraspec_lm_head_workspace_size(M, V))
        if self.nbytes == 0:
            raise ValueError("invalid LM-head workspace shapes")
        dev = torch.device("cuda") if device is None else torch.device(device)
        self.buf = torch.zeros(self.nbytes, dtype=torch.uint8, device=dev)

    @property
    def ptr(self) -> int:
        return self.buf.data_ptr()


def libraspec_lm_head_stats(H, W, ws: "LmHeadWorkspace", temperature=None, rows_per_seq: int = 1, tokens=None,
                            row_stat=None, row_argmax=None, token_prob=None, stream=None):
    """Row statistics of H @ W^T without storing it: (row_stat [M,2], row_argmax [M], token_prob [M] or None)."""
    M, Dm = H.shape
    V = W.shape[0]
    _req(H, torch.bfloat16, "H")
    _req(W, torch.bfloat16, "W", (V, Dm))
    if temperature is not None:
        _req(temperature, torch.float32, "temperature")
        if temperature.numel() * rows_per_seq < M:
            raise ValueError("temperature needs one entry per sequence of rows_per_seq rows")
    if tokens is not None:
        _req(tokens, torch.int32, "tokens", (M,))
    dev = H.device
    row_stat = torch.empty((M, 2), dtype=torch.float32, device=dev) if row_stat is None else row_stat
    row_argmax = torch.empty((M,), dtype=torch.int32, device=dev) if row_argmax is None else row_argmax
    if tokens is not None and token_prob is None:
        token_prob = torch.empty((M,), dtype=torch.float32, device=dev)
    rc = load().libraspec_lm_head_stats(_ptr(H), _ptr(W), _ptr(temperature), int(rows_per_seq), _ptr(tokens), M, V,
                                        Dm, _ptr(row_stat), _ptr(row_argmax), _ptr(token_prob), ws.ptr, ws.nbytes,
                                        _stream(stream))
    _check(rc, "libraspec_lm_head_stats")
    return row_stat, row_argmax, token_prob


class RopeFreqs:
    """Frequencies of a rotation, made once per model: ``turns`` [rot_dim / 2, 2] f32 on the device (turns per
    position of each pair, as two floats) and ``magnitude``, the factor of the rotated pairs.

    scaling: "none", "linear" (f / factor), "ntk" (theta grows with factor) or "parts" (pairs of less than ``low``
    turns over ``original_len`` positions as "linear", of more than ``high`` unchanged, a ramp between)."""

    SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "parts": 3}

    def __init__(self, rot_dim: int, theta: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                 original_len: float = 0.0, low: float = 1.0, high: float = 32.0, magnitude: float = 1.0, device=None):
        if scaling not in self.SCALINGS:
            raise ValueError("scaling must be one of %s" % ", ".join(self.SCALINGS))
        host = torch.empty((max(0, rot_dim // 2), 2), dtype=torch.float32)
        rc = load().libraspec_rope_frequencies(int(rot_dim), float(theta), self.SCALINGS[scaling], float(factor),
                                               float(low), float(high), float(original_len), _ptr(host))
        _check(rc, "libraspec_rope_frequencies")
        self.rot_dim, self.magnitude = int(rot_dim), float(magnitude)
        self.turns = host.to(torch.device("cuda") if device is None else torch.device(device))
        self.turns_ptr = self.turns.data_ptr()


def _heads_stride(t: torch.Tensor, dtype, name: str, shape=None) -> int:
    """Checks [T, H, d] whose tokens' heads are contiguous (any stride from token to token, as in a slice of a wider
    projection); returns that stride."""
    # every condition at once; what fails is named below
    if isinstance(t, torch.Tensor) and t.dtype == dtype and t.is_cuda and t.dim() == 3:
        s0, s1, s2 = t.stride()
        T, H, d = t.shape
        if s2 == 1 and s1 == d and s0 >= H * d and (shape is None or t.shape == shape):
            return s0
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch tensor" % name)
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if not t.is_cuda:
        raise ValueError("%s must be on a CUDA device" % name)
    if t.dim() != 3 or (shape is not None and t.shape != shape):
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape) if shape else "[T, H, d]", tuple(t.shape)))
    T, H, d = t.shape  # (strides of dimensions of size 0 or 1 say nothing)
    if t.numel() and ((d > 1 and t.stride(2) != 1) or (H > 1 and t.stride(1) != d) or (T > 1 and t.stride(0) < H * d)):
        raise ValueError("%s: each token's heads must be contiguous" % name)
    return t.stride(0) if T > 1 and t.numel() else H * d


def _check_device(t: torch.Tensor, name: str) -> None:
    """Frequencies and workspaces may be made on the host; kernels take them on the device."""
    if not t.is_cuda:
        raise ValueError("%s must be on a CUDA device" % name)


_several = None


def _several_devices() -> bool:
    global _several
    if _several is None:
        _several = torch.cuda.device_count() > 1
    return _several


def _on_current(x: torch.Tensor, y: torch.Tensor, *others: Optional[torch.Tensor]) -> None:
    """Refuses a call with a tensor (of those given) of another device than the current one, where it would launch. Where
    there is but one device, two are asked: that the others are on a device at all has been checked. (To ask each of
    fourteen takes 2 to 3 us of a call's 20.)"""
    dev = torch.cuda.current_device()
    if x.get_device() != dev or y.get_device() != dev or (
            _several_devices() and any(t is not None and t.get_device() != dev for t in others)):
        raise ValueError("all tensors must be on the current device (%d), got %s" % (
            dev, ", ".join(sorted({str(t.device) for t in (x, y) + others if t is not None}))))


def _out(shape, dtype, device, stream) -> torch.Tensor:
    """An output of a call, made on the stream that it runs on: what the current stream has given back may still be in
    use there, where nothing orders the call's stream behind it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def libraspec_rope(X, pos, freqs: RopeFreqs, interleaved=False, inverse=False, Y=None, stream=None) -> torch.Tensor:
    """X [T, H, d] (f32 or bf16) rotated to the positions pos [T] int32; ``inverse`` rotates back (the gradient of X
    from that of Y). Y may be X (in place)."""
    bf16 = isinstance(X, torch.Tensor) and X.dtype == torch.bfloat16
    dt = torch.bfloat16 if bf16 else torch.float32
    xs = _heads_stride(X, dt, "X")
    shape = X.shape
    T, H, d = shape
    _req(pos, torch.int32, "pos", (T,))
    _check_device(freqs.turns, "freqs")
    if Y is None:
        Y = _out(shape, dt, X.device, stream)
        ys = H * d
    else:
        ys = _heads_stride(Y, dt, "Y", shape)
    lib = load()
    rc = (lib.libraspec_rope_bf16 if bf16 else lib.libraspec_rope)(
        X.data_ptr(), xs, pos.data_ptr(), freqs.turns_ptr, freqs.magnitude, T, H, d, freqs.rot_dim,
        1 if interleaved else 0, 1 if inverse else 0, Y.data_ptr(), ys, _stream(stream))
    if rc != OK:
        _check(rc, "libraspec_rope_bf16" if bf16 else "libraspec_rope")
    return Y


def libraspec_rope_append(Q, K, V, Kc, Vc, cu_new, kv_len, freqs: RopeFreqs, ws, pos=None, interleaved=False, Qo=None,
                          stream=None):
    """Rotates a ragged chunk's keys into the dense caches Kc, Vc [B, Hkv, S_cap, d] beside its values, and its queries
    into Qo [T, Hq, d] bf16 (Q None: keys and values alone). ws: any of the library's workspaces (its status word).
    Returns Qo."""
    return _rope_append(Q, K, V, Kc, Vc, None, cu_new, kv_len, freqs, ws, pos, interleaved, Qo, stream)


def libraspec_rope_append_paged(Q, K, V, Kp, Vp, block_table, cu_new, kv_len, freqs: RopeFreqs, ws, pos=None,
                                interleaved=False, Qo=None, stream=None):
    """libraspec_rope_append into page pools Kp, Vp [n_pages, Hkv, page_size, d] by block_table [B, max_pages]."""
    return _rope_append(Q, K, V, Kp, Vp, block_table, cu_new, kv_len, freqs, ws, pos, interleaved, Qo, stream)


def _check_new(cu_new, kv_len):
    """Offsets of the new tokens [B + 1] and cache lengths [B]; returns B."""
    _req(kv_len, torch.int32, "kv_len")
    if kv_len.dim() != 1:
        raise ValueError("kv_len must be [B]")
    B = kv_len.shape[0]
    _req(cu_new, torch.int32, "cu_new", (B + 1,))
    return B


def _check_caches(Kc, Vc, block_table, B, Hkv, d):
    """Dense caches, or pools and their table; returns (capacity, max_pages, page_size, n_pages)."""
    paged = block_table is not None
    _req(Kc, torch.bfloat16, "Kp" if paged else "Kc")
    shape = Kc.shape
    if len(shape) != 4 or shape[1] != Hkv or shape[3] != d or not (paged or shape[0] == B):
        raise ValueError("%s must be %s, got %s" % (("Kp", "[n_pages, %d, page_size, %d]" % (Hkv, d), tuple(shape)) if paged
                                                    else ("Kc", "[%d, %d, S_cap, %d]" % (B, Hkv, d), tuple(shape))))
    _req(Vc, torch.bfloat16, "Vp" if paged else "Vc", shape)
    if not paged:
        return shape[2], 0, 0, 0
    _req(block_table, torch.int32, "block_table")
    t = block_table.shape
    if len(t) != 2 or t[0] != B:
        raise ValueError("block_table must be [B, max_pages]")
    return 0, t[1], shape[2], shape[0]


def _rope_append(Q, K, V, Kc, Vc, block_table, cu_new, kv_len, freqs, ws, pos, interleaved, Qo, stream):
    bf16 = isinstance(K, torch.Tensor) and K.dtype == torch.bfloat16
    dt = torch.bfloat16 if bf16 else torch.float32
    ks = _heads_stride(K, dt, "K")
    shape = K.shape
    T, Hkv, d = shape
    vs = _heads_stride(V, dt, "V", shape)
    B = _check_new(cu_new, kv_len)
    S_cap, max_pages, page_size, n_pages = _check_caches(Kc, Vc, block_table, B, Hkv, d)
    if pos is not None:
        _req(pos, torch.int32, "pos", (T,))
    _check_device(freqs.turns, "freqs")
    _check_device(ws.buf, "the workspace")
    Hq = qs = 0
    if Q is not None:
        qs = _heads_stride(Q, dt, "Q")
        shape = Q.shape
        Hq = shape[1]
        if shape[0] != T or shape[2] != d:
            raise ValueError("Q must have shape [%d, Hq, %d], got %s" % (T, d, tuple(shape)))
        if Qo is None:
            Qo = _out(shape, torch.bfloat16, K.device, stream)
        else:
            _req(Qo, torch.bfloat16, "Qo", shape)
    elif Qo is not None:
        raise ValueError("Qo without Q")
    lib = load()
    name = "libraspec_rope_append" + ("" if block_table is None else "_paged") + ("_bf16" if bf16 else "")
    head = (_ptr(Q), qs, K.data_ptr(), ks, V.data_ptr(), vs, cu_new.data_ptr(), kv_len.data_ptr(), _ptr(pos),
            freqs.turns_ptr, freqs.magnitude, T, B, Hq, Hkv, d, freqs.rot_dim, 1 if interleaved else 0, _ptr(Qo),
            Kc.data_ptr(), Vc.data_ptr())
    if block_table is None:
        rc = getattr(lib, name)(*head, S_cap, ws.ptr, ws.nbytes, _stream(stream))
    else:
        rc = getattr(lib, name)(*head, block_table.data_ptr(), max_pages, page_size, n_pages, ws.ptr, ws.nbytes,
                                _stream(stream))
    if rc != OK:
        _check(rc, name)
    return Qo


class QkNorm:
    """Weights of the norm of query and key heads [d] (f32, on the device) and what is added to the mean square."""

    def __init__(self, q_weight: torch.Tensor, k_weight: torch.Tensor, eps: float = 1e-6):
        _req(q_weight, torch.float32, "q_weight")
        if q_weight.dim() != 1:
            raise ValueError("q_weight must be [d], got %s" % (tuple(q_weight.shape),))
        _req(k_weight, torch.float32, "k_weight", q_weight.shape)
        self.q_weight, self.k_weight, self.eps, self.d = q_weight, k_weight, float(eps), q_weight.shape[0]
        self.q_ptr, self.k_ptr = q_weight.data_ptr(), k_weight.data_ptr()


def _check_norm(norm, d) -> None:
    if norm.d != d:
        raise ValueError("norm: weights of %d elements for heads of %d" % (norm.d, d))


def libraspec_qk_norm_rope(X, n_q: int, norm: QkNorm, pos, freqs: RopeFreqs, interleaved=False, Y=None,
                           stream=None) -> torch.Tensor:
    """X [T, H, d] (f32 or bf16), queries and keys side by side: each head over its root mean square, times the weights
    of queries (the first n_q heads) or keys, then rotated to the positions pos [T] int32. Y may be X (in place)."""
    bf16 = isinstance(X, torch.Tensor) and X.dtype == torch.bfloat16
    dt = torch.bfloat16 if bf16 else torch.float32
    xs = _heads_stride(X, dt, "X")
    shape = X.shape
    T, H, d = shape
    if not 0 <= n_q <= H:
        raise ValueError("n_q must lie in [0, %d], got %s" % (H, n_q))
    _check_norm(norm, d)
    _req(pos, torch.int32, "pos", (T,))
    _check_device(freqs.turns, "freqs")
    if Y is None:
        Y = _out(shape, dt, X.device, stream)
        ys = H * d
    else:
        ys = _heads_stride(Y, dt, "Y", shape)
    _on_current(X, freqs.turns, pos, norm.q_weight, norm.k_weight, Y)
    lib = load()
    rc = (lib.libraspec_qk_norm_rope_bf16 if bf16 else lib.libraspec_qk_norm_rope)(
        X.data_ptr(), xs, pos.data_ptr(), freqs.turns_ptr, freqs.magnitude, norm.q_ptr, norm.k_ptr, norm.eps, T, n_q,
        H - n_q, d, freqs.rot_dim, 1 if interleaved else 0, Y.data_ptr(), ys, _stream(stream))
    if rc != OK:
        _check(rc, "libraspec_qk_norm_rope_bf16" if bf16 else "libraspec_qk_norm_rope")
    return Y


def _check_caches_q8(K8, V8, Ks, Vs, block_table, B):
    """Codes and exponents of a cache in 8 bits; returns (Hkv, d, capacity, max_pages, page_size, n_pages, block)."""
    paged = block_table is not None
    # every condition at once; what fails is named below
    try:
        planes, Hkv, rows, d = shape = K8.shape
        n = Ks.shape[2]
        fine = (K8.dtype == V8.dtype == torch.float8_e4m3fn and Ks.dtype == Vs.dtype == torch.uint8 and V8.shape == shape
                and Ks.shape == Vs.shape == (planes, Hkv, n) and n > 0 and rows % n == 0 and K8.is_cuda and V8.is_cuda
                and Ks.is_cuda and Vs.is_cuda and K8.is_contiguous() and V8.is_contiguous() and Ks.is_contiguous()
                and Vs.is_contiguous())
    except (AttributeError, IndexError, TypeError, ValueError):
        fine = False
    if not fine:
        _req(K8, torch.float8_e4m3fn, "K8")
        shape = K8.shape
        if len(shape) != 4:
            raise ValueError("K8 must be %s, got %s" % ("[n_pages, Hkv, page_size, d]" if paged else "[B, Hkv, S_cap, d]",
                                                        tuple(shape)))
        _req(V8, torch.float8_e4m3fn, "V8", shape)
        _req(Ks, torch.uint8, "Ks")
        _req(Vs, torch.uint8, "Vs", Ks.shape)
        raise ValueError("Ks must be [%d, %d, %s / block], got %s" % (shape[0], shape[1], shape[2], tuple(Ks.shape)))
    if not paged:
        if planes != B:
            raise ValueError("K8 must be [%d, Hkv, S_cap, d], got %s" % (B, tuple(shape)))
        return Hkv, d, rows, 0, 0, 0, rows // n
    _req(block_table, torch.int32, "block_table")
    t = block_table.shape
    if len(t) != 2 or t[0] != B:
        raise ValueError("block_table must be [B, max_pages]")
    return Hkv, d, 0, t[1], rows, planes, rows // n


def libraspec_rope_append_q8(Q, K, V, K8, V8, Ks, Vs, cu_new, kv_len, freqs: RopeFreqs, ws, norm: Optional[QkNorm] = None,
                             pos=None, interleaved=False, Qo=None, stream=None):
    """libraspec_rope_append into a cache in 8 bits: codes K8, V8 [B, Hkv, S_cap, d] float8_e4m3fn and exponents Ks, Vs
    [B, Hkv, S_cap / block] uint8 (e + 127; block 16, 32 or 64). ``norm``: query and key heads are normed first. ws: any
    of the library's workspaces (its status word). Returns Qo [T, Hq, d] bf16, or None without Q."""
    return _rope_append_q8(Q, K, V, K8, V8, Ks, Vs, None, cu_new, kv_len, freqs, ws, norm, pos, interleaved, Qo, stream)


def libraspec_rope_append_q8_paged(Q, K, V, K8, V8, Ks, Vs, block_table, cu_new, kv_len, freqs: RopeFreqs, ws,
                                   norm: Optional[QkNorm] = None, pos=None, interleaved=False, Qo=None, stream=None):
    """libraspec_rope_append_q8 into page pools K8, V8 [n_pages, Hkv, page_size, d] with exponents [n_pages, Hkv,
    page_size / block], by block_table [B, max_pages]."""
    return _rope_append_q8(Q, K, V, K8, V8, Ks, Vs, block_table, cu_new, kv_len, freqs, ws, norm, pos, interleaved, Qo,
                           stream)


def _rope_append_q8(Q, K, V, K8, V8, Ks, Vs, block_table, cu_new, kv_len, freqs, ws, norm, pos, interleaved, Qo, stream):
    bf16 = isinstance(K, torch.Tensor) and K.dtype == torch.bfloat16
    dt = torch.bfloat16 if bf16 else torch.float32
    ks = _heads_stride(K, dt, "K")
    shape = K.shape
    T, Hkv, d = shape
    vs = _heads_stride(V, dt, "V", shape)
    B = _check_new(cu_new, kv_len)
    h, dc, S_cap, max_pages, page_size, n_pages, block = _check_caches_q8(K8, V8, Ks, Vs, block_table, B)
    if h != Hkv or dc != d:
        raise ValueError("the cache has %d heads of %d, K %d of %d" % (h, dc, Hkv, d))
    if pos is not None:
        _req(pos, torch.int32, "pos", (T,))
    _check_device(freqs.turns, "freqs")
    _check_device(ws.buf, "the workspace")
    q_w = k_w = None
    eps = 0.0
    if norm is not None:
        _check_norm(norm, d)
        q_w, k_w, eps = norm.q_ptr, norm.k_ptr, norm.eps
    Hq = qs = 0
    if Q is not None:
        qs = _heads_stride(Q, dt, "Q")
        shape = Q.shape
        Hq = shape[1]
        if shape[0] != T or shape[2] != d:
            raise ValueError("Q must have shape [%d, Hq, %d], got %s" % (T, d, tuple(shape)))
        if Qo is None:
            Qo = _out(shape, torch.bfloat16, K.device, stream)
        else:
            _req(Qo, torch.bfloat16, "Qo", shape)
    elif Qo is not None:
        raise ValueError("Qo without Q")
    _on_current(K, K8, Q, V, V8, Ks, Vs, block_table, cu_new, kv_len, pos, freqs.turns, ws.buf, Qo,
                *(() if norm is None else (norm.q_weight, norm.k_weight)))
    lib = load()
    name = "libraspec_rope_append_q8" + ("" if block_table is None else "_paged") + ("_bf16" if bf16 else "")
    head = (_ptr(Q), qs, K.data_ptr(), ks, V.data_ptr(), vs, cu_new.data_ptr(), kv_len.data_ptr(), _ptr(pos),
            freqs.turns_ptr, freqs.magnitude, q_w, k_w, eps, T, B, Hq, Hkv, d, freqs.rot_dim, 1 if interleaved else 0,
            _ptr(Qo), K8.data_ptr(), V8.data_ptr(), Ks.data_ptr(), Vs.data_ptr())
    if block_table is None:
        rc = getattr(lib, name)(*head, S_cap, block, ws.ptr, ws.nbytes, _stream(stream))
    else:
        rc = getattr(lib, name)(*head, block_table.data_ptr(), max_pages, page_size, n_pages, block, ws.ptr, ws.nbytes,
                                _stream(stream))
    if rc != OK:
        _check(rc, name)
    return Qo


def libraspec_kv_read_q8(K8, V8, Ks, Vs, cu, start, T: int, ws, K=None, V=None, stream=None):
    """Keys start[b] .. start[b] + cu[b + 1] - cu[b] - 1 of every sequence of a dense cache in 8 bits, as packed bf16 rows
    (K, V) [T, Hkv, d]: row cu[b] + j is key start[b] + j. cu [B + 1], start [B] int32. Rows of no sequence, or that
    cannot be read, are left alone."""
    return _kv_read_q8(K8, V8, Ks, Vs, None, cu, start, T, ws, K, V, stream)


def libraspec_kv_read_q8_paged(K8, V8, Ks, Vs, block_table, cu, start, T: int, ws, K=None, V=None, stream=None):
    """libraspec_kv_read_q8 from page pools by block_table [B, max_pages]."""
    return _kv_read_q8(K8, V8, Ks, Vs, block_table, cu, start, T, ws, K, V, stream)


def _kv_read_q8(K8, V8, Ks, Vs, block_table, cu, start, T, ws, K, V, stream):
    B = _check_new(cu, start)
    Hkv, d, S_cap, max_pages, page_size, n_pages, block = _check_caches_q8(K8, V8, Ks, Vs, block_table, B)
    _check_device(ws.buf, "the workspace")
    T = int(T)
    if T < 0:
        raise ValueError("T must not be negative")
    shape = (T, Hkv, d)
    K = _out(shape, torch.bfloat16, K8.device, stream) if K is None else _req(K, torch.bfloat16, "K", shape)
    V = _out(shape, torch.bfloat16, K8.device, stream) if V is None else _req(V, torch.bfloat16, "V", shape)
    _on_current(K8, ws.buf, V8, Ks, Vs, block_table, cu, start, K, V)
    lib = load()
    tail = (cu.data_ptr(), start.data_ptr(), T, B, Hkv, d)
    head = (K8.data_ptr(), V8.data_ptr(), Ks.data_ptr(), Vs.data_ptr())
    end = (block, K.data_ptr(), V.data_ptr(), ws.ptr, ws.nbytes, _stream(stream))
    if block_table is None:
        rc = lib.libraspec_kv_read_q8(*head, *tail, S_cap, *end)
    else:
        rc = lib.libraspec_kv_read_q8_paged(*head, block_table.data_ptr(), max_pages, page_size, n_pages, *tail, *end)
    if rc != OK:
        _check(rc, "libraspec_kv_read_q8" + ("" if block_table is None else "_paged"))
    return K, V


class ChunkWorkspace:
    """Device scratch of the chunk calls, for up to T new tokens of B sequences; q8=False: of those over a bf16 cache alone
    (T Hq (2 d + 1) bytes less)."""

    def __init__(self, T, B, Hq, Hkv, head_dim, device=None, q8=True):
        lib = load()
        size = lib.libraspec_chunk_workspace_size if q8 else lib.libraspec_chunk_workspace_size_bf16
        self.nbytes = int(size(T, B, Hq, Hkv, head_dim))
        if self.nbytes == 0:
            raise ValueError("invalid chunk workspace shapes")
        dev = torch.device("cuda") if device is None else torch.device(device)
        self.buf = torch.zeros(self.nbytes, dtype=torch.uint8, device=dev)
        self.ptr = self.buf.data_ptr()


class _ScoreOpts(ctypes.Structure):
    _fields_ = [("softcap", _F), ("window", _I), ("slopes", _P), ("first_key", _P), ("prefix_len", _P)]


def libraspec_chunk_attn(Q, Kc, Vc, cu_new, kv_len, ws: ChunkWorkspace, softmax_scale=None, softcap: float = 0.0,
                         slopes=None, window: int = 0, first_key=None, prefix_len=None, O=None, lse=None,
                         want_lse=False, stream=None):
    """Attention of packed new tokens Q [T, Hq, d] over the dense caches Kc, Vc [B, Hkv, S_cap, d] that hold them
    already. Options: softcap (tanh cap of the scores), slopes [Hq] f32 (bias by distance), window (keys a row looks
    back, itself included), first_key [T] int32 (start of the row's document), prefix_len [B] int32 (keys that all
    rows see). Returns (O, lse or None)."""
    return _chunk_attn(Q, Kc, Vc, None, cu_new, kv_len, ws, softmax_scale, softcap, slopes, window, first_key,
                       prefix_len, O, lse, want_lse, stream)


def libraspec_chunk_attn_paged(Q, Kp, Vp, block_table, cu_new, kv_len, ws: ChunkWorkspace, softmax_scale=None,
                               softcap: float = 0.0, slopes=None, window: int = 0, first_key=None, prefix_len=None,
                               O=None, lse=None, want_lse=False, stream=None):
    """libraspec_chunk_attn over page pools Kp, Vp [n_pages, Hkv, page_size, d] (page_size a multiple of 16) by
    block_table [B, max_pages] int32."""
    return _chunk_attn(Q, Kp, Vp, block_table, cu_new, kv_len, ws, softmax_scale, softcap, slopes, window, first_key,
                       prefix_len, O, lse, want_lse, stream)


def libraspec_sink_attn(Q, Kc, Vc, cu_new, kv_len, ws: ChunkWorkspace, window: int, sinks: int, softmax_scale=None,
                        softcap: float = 0.0, slopes=None, prefix_len=None, O=None, lse=None, want_lse=False, stream=None):
    """libraspec_chunk_attn in a window whose first ``sinks`` tokens stay visible to every row. Returns (O, lse or None)."""
    return _chunk_attn(Q, Kc, Vc, None, cu_new, kv_len, ws, softmax_scale, softcap, slopes, window, None, prefix_len, O, lse,
                       want_lse, stream, "libraspec_sink_attn", sinks)


def libraspec_sink_attn_paged(Q, Kp, Vp, block_table, cu_new, kv_len, ws: ChunkWorkspace, window: int, sinks: int,
                              softmax_scale=None, softcap: float = 0.0, slopes=None, prefix_len=None, O=None, lse=None,
                              want_lse=False, stream=None):
    """libraspec_sink_attn over page pools Kp, Vp [n_pages, Hkv, page_size, d] by block_table [B, max_pages]."""
    return _chunk_attn(Q, Kp, Vp, block_table, cu_new, kv_len, ws, softmax_scale, softcap, slopes, window, None, prefix_len,
                       O, lse, want_lse, stream, "libraspec_sink_attn", sinks)


def libraspec_chunk_attn_q8(Q, K8, V8, Ks, Vs, cu_new, kv_len, ws: ChunkWorkspace, softmax_scale=None, softcap: float = 0.0,
                            slopes=None, window: int = 0, sinks: int = 0, first_key=None, prefix_len=None, O=None, lse=None,
                            want_lse=False, stream=None):
    """libraspec_chunk_attn over a cache in 8 bits (as libraspec_rope_append_q8 fills it): codes K8, V8 [B, Hkv, S_cap, d]
    float8_e4m3fn and exponents Ks, Vs [B, Hkv, S_cap / block] uint8; sinks: first tokens that the window leaves visible
    (not with first_key). Returns (O, lse or None)."""
    return _chunk_attn(Q, K8, V8, None, cu_new, kv_len, ws, softmax_scale, softcap, slopes, window, first_key, prefix_len, O,
                       lse, want_lse, stream, "libraspec_chunk_attn_q8", sinks, Ks, Vs)


def libraspec_chunk_attn_q8_paged(Q, K8, V8, Ks, Vs, block_table, cu_new, kv_len, ws: ChunkWorkspace, softmax_scale=None,
                                  softcap: float = 0.0, slopes=None, window: int = 0, sinks: int = 0, first_key=None,
                                  prefix_len=None, O=None, lse=None, want_lse=False, stream=None):
    """libraspec_chunk_attn_q8 over page pools K8, V8 [n_pages, Hkv, page_size, d] with exponents [n_pages, Hkv,
    page_size / block], by block_table [B, max_pages]."""
    return _chunk_attn(Q, K8, V8, block_table, cu_new, kv_len, ws, softmax_scale, softcap, slopes, window, first_key,
                       prefix_len, O, lse, want_lse, stream, "libraspec_chunk_attn_q8", sinks, Ks, Vs)


def _chunk_attn(Q, Kc, Vc, block_table, cu_new, kv_len, ws, softmax_scale, softcap, slopes, window, first_key,
                prefix_len, O, lse, want_lse, stream, name="libraspec_chunk_attn", sinks=None, Ks=None, Vs=None):
    _req(Q, torch.bfloat16, "Q")
    shape = Q.shape
    if len(shape) != 3:
        raise ValueError("Q must be [T, Hq, d]")
    T, Hq, d = shape
    B = _check_new(cu_new, kv_len)
    block = ()
    if Ks is None:
        Hkv = Kc.shape[1] if isinstance(Kc, torch.Tensor) and Kc.dim() == 4 else 0
        S_cap, max_pages, page_size, n_pages = _check_caches(Kc, Vc, block_table, B, Hkv, d)
        caches = (Kc.data_ptr(), Vc.data_ptr())
    else:
        Hkv, dc, S_cap, max_pages, page_size, n_pages, block = _check_caches_q8(Kc, Vc, Ks, Vs, block_table, B)
        if dc != d:
            raise ValueError("the cache has heads of %d, Q of %d" % (dc, d))
        caches = (Kc.data_ptr(), Vc.data_ptr(), Ks.data_ptr(), Vs.data_ptr())
        block = (block,)
    _check_device(ws.buf, "the workspace")
    opts = None
    if softcap or slopes is not None or window or first_key is not None or prefix_len is not None:
        if slopes is not None:
            _req(slopes, torch.float32, "slopes", (Hq,))
        if first_key is not None:
            _req(first_key, torch.int32, "first_key", (T,))
        if prefix_len is not None:
            _req(prefix_len, torch.int32, "prefix_len", (B,))
        opts = ctypes.byref(_ScoreOpts(float(softcap), int(window), _ptr(slopes), _ptr(first_key), _ptr(prefix_len)))
    if O is None:
        O = _out(shape, torch.bfloat16, Q.device, stream)
    else:
        _req(O, torch.bfloat16, "O", shape)
    if lse is not None:
        _req(lse, torch.float32, "lse", (T, Hq))
    elif want_lse:
        lse = _out((T, Hq), torch.float32, Q.device, stream)
    if sinks is not None:
        _on_current(Q, Kc, Vc, Ks, Vs, block_table, cu_new, kv_len, ws.buf, slopes, first_key, prefix_len, O, lse)
    tail = (d ** -0.5 if softmax_scale is None else float(softmax_scale), opts,
            *(() if sinks is None else (int(sinks),)), O.data_ptr(), _ptr(lse), ws.ptr, ws.nbytes, _stream(stream))
    if block_table is None:
        rc = getattr(load(), name)(Q.data_ptr(), *caches, cu_new.data_ptr(), kv_len.data_ptr(), T, B, Hq, Hkv, d, S_cap,
                                   *block, *tail)
    else:
        name += "_paged"
        rc = getattr(load(), name)(Q.data_ptr(), *caches, block_table.data_ptr(), max_pages, page_size, n_pages,
                                   cu_new.data_ptr(), kv_len.data_ptr(), T, B, Hq, Hkv, d, *block, *tail)
    if rc != OK:
        _check(rc, name)
    return O, lse


def _ptr_array(tensors: Sequence[Optional[torch.Tensor]]):
    return (ctypes.c_void_p * max(1, len(tensors)))(*[None if t is None else t.data_ptr() for t in tensors])


def _check_layers(layers, k: str, v: str, q_shape, kv_shape) -> None:
    """Q and the caches (dict keys k and v) of every layer."""
    for i, lay in enumerate(layers):
        for key, shape in (("Q", q_shape), (k, kv_shape), (v, kv_shape)):
            t = lay[key]
            if not (isinstance(t, torch.Tensor) and t.dtype == torch.bfloat16 and t.is_cuda and t.is_contiguous()
                    and t.shape == shape):
                _req(t, torch.bfloat16, "%s[%d]" % (key, i), shape)


class RoundOutputs:
    def __init__(self, conf, dstat, L, n_accepted, bonus_token, O, lse):
        self.conf, self.dstat, self.L = conf, dstat, L
        self.n_accepted, self.bonus_token = n_accepted, bonus_token
        self.O, self.lse = O, lse


def libraspec_verify_round(draft_logits, draft_tokens, temperature, cost_table, target_logits, layers, kv_len,
                           seed: int, ws: Workspace, round_offset: int = 0, seq_offset: int = 0,
                           softmax_scale=None, outputs: Optional[RoundOutputs] = None, want_lse=False,
                           stream=None) -> RoundOutputs:
    """layers: sequence of dicts with Q, Kc, Vc (and optionally O)."""
    B, K, V = draft_logits.shape
    bf16 = draft_logits.dtype == torch.bfloat16  # libraspec_verify_round_bf16: both logit tensors bf16
    ldt = torch.bfloat16 if bf16 else torch.float32
    _req(draft_logits, ldt, "draft_logits")
    _req(target_logits, ldt, "target_logits", (B, K + 1, V))
    _req(draft_tokens, torch.int32, "draft_tokens", (B, K))
    _req(temperature, torch.float32, "temperature", (B,))
    _req(cost_table, torch.float32, "cost_table", (K + 1,))
    _req(kv_len, torch.int32, "kv_len", (B,))
    n_layers = len(layers)
    Hq, D = (layers[0]["Q"].shape[2], layers[0]["Q"].shape[3]) if n_layers else (1, 64)
    Hkv, S_cap = (layers[0]["Kc"].shape[1], layers[0]["Kc"].shape[2]) if n_layers else (1, 1)
    _check_layers(layers, "Kc", "Vc", (B, K + 1, Hq, D), (B, Hkv, S_cap, D))
    dev = draft_logits.device
    if outputs is None:
        outputs = RoundOutputs(
            torch.empty((B, K), dtype=torch.float32, device=dev), torch.empty((B, K, 2), dtype=torch.float32, device=dev),
            torch.empty((B,), dtype=torch.int32, device=dev), torch.empty((B,), dtype=torch.int32, device=dev),
            torch.empty((B,), dtype=torch.int32, device=dev),
            [lay.get("O") if lay.get("O") is not None else torch.empty_like(lay["Q"]) for lay in layers],
            [torch.empty((B, K + 1, Hq), dtype=torch.float32, device=dev) for _ in layers] if want_lse else None)
    if softmax_scale is None:
        softmax_scale = D ** -0.5
    qa = _ptr_array([lay["Q"] for lay in layers])
    ka = _ptr_array([lay["Kc"] for lay in layers])
    va = _ptr_array([lay["Vc"] for lay in layers])
    oa = _ptr_array(outputs.O)
    la = _ptr_array(outputs.lse) if outputs.lse is not None else None
    name = "libraspec_verify_round_bf16" if bf16 else "libraspec_verify_round"
    rc = getattr(load(), name)(
        _ptr(draft_logits), _ptr(draft_tokens), _ptr(temperature), _ptr(cost_table), _ptr(target_logits), qa, ka, va,
        oa, la, n_layers, _ptr(kv_len), B, K, V, Hq, Hkv, D, S_cap, float(softmax_scale), int(seed) & (2**64 - 1),
        int(round_offset), int(seq_offset), _ptr(outputs.conf), _ptr(outputs.dstat), _ptr(outputs.L),
        _ptr(outputs.n_accepted), _ptr(outputs.bonus_token), ws.ptr, ws.nbytes, _stream(stream))
    _check(rc, name)
    return outputs


class StagedRound:
    """Marshalled arguments of libraspec_verify_round_staged for fixed buffers: built (and checked)
    once, then each call enqueues one round.

    host_parts / dev_parts: three (pinned host, device) uint8 tensors, the drafter part, the layers
    part and the target part; the typed inputs (draft_logits ... target_logits, each layer's Q,
    kv_new) are device tensors inside dev_parts; layers: per layer {"Q", "Kc", "Vc"};
    outputs: RoundOutputs; n_host / bonus_host: pinned int32 [B] tensors."""

    def __init__(self, host_parts, dev_parts, kv_new, n_host, bonus_host, draft_logits, draft_tokens, temperature,
                 cost_table, target_logits, layers, kv_len, outputs: "RoundOutputs", ws: Workspace,
                 rng_host, rng_dev, softmax_scale=None, copy_stream=None, copy_parts=(True, True, True)):
        """copy_parts[i] False: part i is not copied; its typed inputs (and kv_new / rng_dev when they
        lie in it) are then pinned host tensors that the kernels read in place (a pinned allocation's
        address is valid on the device under unified addressing)."""
        B, K, V = draft_logits.shape
        bf16 = draft_logits.dtype == torch.bfloat16
        ldt = torch.bfloat16 if bf16 else torch.float32
        req = _req_dev_or_pinned
        req(draft_logits, ldt, "draft_logits")
        req(target_logits, ldt, "target_logits", (B, K + 1, V))
        req(draft_tokens, torch.int32, "draft_tokens", (B, K))
        req(temperature, torch.float32, "temperature", (B,))
        req(cost_table, torch.float32, "cost_table", (K + 1,))
        _req(kv_len, torch.int32, "kv_len", (B,))
        n_layers = len(layers)
        Hq, D = layers[0]["Q"].shape[2], layers[0]["Q"].shape[3]
        Hkv, S_cap = layers[0]["Kc"].shape[1], layers[0]["Kc"].shape[2]
        _check_layers(layers, "Kc", "Vc", (B, K + 1, Hq, D), (B, Hkv, S_cap, D))
        req(kv_new, torch.bfloat16, "kv_new", (n_layers, 2, B, Hkv, K + 1, D))
        if len(host_parts) != 3 or len(dev_parts) != 3:
            raise ValueError("three host and three device parts")
        for h, d in zip(host_parts, dev_parts):
            if not h.is_pinned() or h.numel() != d.numel() or not d.is_cuda:
                raise ValueError("each part: a pinned host tensor and a device tensor of the same size")
        req(rng_dev, torch.int64, "rng_dev", (3,))
        if (not isinstance(rng_host, torch.Tensor) or rng_host.dtype != torch.int64 or rng_host.numel() != 3
                or not rng_host.is_pinned()):
            raise ValueError("rng_host must be 3 int64 of pinned host memory inside host part 2")
        if softmax_scale is None:
            softmax_scale = D ** -0.5
        self._keep = (host_parts, dev_parts, layers, outputs, n_host, bonus_host, rng_host, rng_dev)
        self._hp = (ctypes.c_void_p * 3)(*[h.data_ptr() for h in host_parts])
        self._dp = (ctypes.c_void_p * 3)(*[d.data_ptr() for d in dev_parts])
        self._nb = (ctypes.c_size_t * 3)(*[h.numel() * h.element_size() if c else 0
                                           for h, c in zip(host_parts, copy_parts)])
        self._copy = copy_stream if copy_stream is not None else torch.cuda.Stream(device=kv_len.device)
        self._qa = _ptr_array([l["Q"] for l in layers])
        self._ka = _ptr_array([l["Kc"] for l in layers])
        self._va = _ptr_array([l["Vc"] for l in layers])
        self._oa = _ptr_array(outputs.O)
        self._name = "libraspec_verify_round_staged_bf16" if bf16 else "libraspec_verify_round_staged"
        self._fn = getattr(load(), self._name)
        self._pre = (self._hp, self._dp, self._nb, ctypes.c_void_p(self._copy.cuda_stream), _ptr(kv_new),
                     _ptr(rng_host), _ptr(rng_dev), _ptr(n_host), _ptr(bonus_host), _ptr(draft_logits), _ptr(draft_tokens), _ptr(temperature),
                     _ptr(cost_table), _ptr(target_logits), self._qa, self._ka, self._va, self._oa, n_layers,
                     _ptr(kv_len), B, K, V, Hq, Hkv, D, S_cap, float(softmax_scale))
        self._post = (_ptr(outputs.conf), _ptr(outputs.dstat), _ptr(outputs.L), _ptr(outputs.n_accepted),
                      _ptr(outputs.bonus_token), ws.ptr, ws.nbytes)

    def __call__(self, seed: int, round_offset: int = 0, seq_offset: int = 0, stream=None) -> None:
        rc = self._fn(*self._pre, int(seed) & (2**64 - 1), int(round_offset), int(seq_offset), *self._post,
                      _stream(stream))
        _check(rc, self._name)


def libraspec_verify_round_staged(host_parts, dev_parts, kv_new, n_host, bonus_host, draft_logits, draft_tokens,
                                  temperature, cost_table, target_logits, layers, kv_len, outputs, ws, rng_host,
                                  rng_dev, seed: int, round_offset: int = 0, seq_offset: int = 0, softmax_scale=None,
                                  copy_stream=None, stream=None) -> None:
    """One staged round (see StagedRound); returns after enqueuing."""
    StagedRound(host_parts, dev_parts, kv_new, n_host, bonus_host, draft_logits, draft_tokens, temperature,
                cost_table, target_logits, layers, kv_len, outputs, ws, rng_host, rng_dev, softmax_scale,
                copy_stream)(
        seed, round_offset, seq_offset, stream)

