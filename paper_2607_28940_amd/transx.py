"""Python binding of libtransx.so (the TransX serving path on MI355X).

Argument marshalling only: every step of the path runs in the library's HIP
kernels. PyTorch provides device memory (weights, the page pool, workspaces,
inputs, outputs) and the stream; the functions mirror the C ABI of
include/transx.h (kv_cache_build, kv_cache_append, score_candidates, and the
training operators tx_rel_attn_*, tx_event_attn_*, tx_preference_*).
If the library has not been built, loading fails loudly: there is no
fallback implementation.
"""
from __future__ import annotations

import ctypes
import os
import re
from typing import List, Optional, Sequence

import numpy as np

from .inputs import ModelConfig

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtransx.so")
HEADER = os.path.join(os.path.dirname(_HERE), "include", "transx.h")

TX_OK, TX_E_INVALID, TX_E_NOMEM, TX_E_NOCACHE, TX_E_HIP, TX_E_UNSUPPORTED = 0, -1, -2, -3, -4, -5
TX_F32, TX_BF16 = 0, 1
TX_OP_BUILD, TX_OP_APPEND, TX_OP_SCORE = 0, 1, 2
PAGE_TOKENS = 64
STATUS_NAMES = {0: "TX_OK", -1: "TX_E_INVALID", -2: "TX_E_NOMEM", -3: "TX_E_NOCACHE", -4: "TX_E_HIP",
                -5: "TX_E_UNSUPPORTED"}


class TxError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{STATUS_NAMES.get(code, code)}: {msg}")
        self.code = code


class Config(ctypes.Structure):
    _fields_ = [("d_model", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("d_ffn", ctypes.c_int32),
                ("n_enc_layers", ctypes.c_int32), ("n_dec_layers", ctypes.c_int32),
                ("rel_pos_buckets", ctypes.c_int32), ("ln_eps", ctypes.c_float), ("dtype", ctypes.c_int32),
                ("l_local", ctypes.c_int32), ("global_pool", ctypes.c_int32), ("n_actions", ctypes.c_int32)]

    @classmethod
    def of(cls, m: ModelConfig) -> "Config":
        return cls(m.d_model, m.n_heads, m.d_ffn, m.n_enc_layers, m.n_dec_layers, m.rel_pos_buckets,
                   float(m.ln_eps), TX_BF16 if m.dtype == "bf16" else TX_F32, int(m.l_local),
                   int(bool(m.global_pool)), int(m.n_actions))


class AttnConfig(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("d_head", ctypes.c_int32), ("rel_pos_buckets", ctypes.c_int32), ("scale", ctypes.c_float)]


class Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("row_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class PreferenceConfig(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("n_actions", ctypes.c_int32), ("beta", ctypes.c_float),
                ("smoothing", ctypes.c_float)]


_lib = None
VP = ctypes.c_void_p
I32P = ctypes.POINTER(ctypes.c_int32)
I64P = ctypes.POINTER(ctypes.c_int64)
CFGP = ctypes.POINTER(Config)
ACFGP = ctypes.POINTER(AttnConfig)
PCFGP = ctypes.POINTER(PreferenceConfig)
ROWSP = ctypes.POINTER(Rows)

_SIGS = {
    "tx_last_error": (ctypes.c_char_p, []),
    "tx_num_weights": (ctypes.c_int32, [CFGP]),
    "tx_model_repack_bytes": (ctypes.c_size_t, [CFGP]),
    "tx_model_create": (ctypes.c_int, [CFGP, VP, ctypes.c_size_t, ctypes.c_uint64, ctypes.POINTER(VP)]),
    "tx_model_set_weights": (ctypes.c_int, [VP, ctypes.POINTER(VP), ctypes.c_int32, VP]),
    "tx_model_destroy": (None, [VP]),
    "tx_kv_page_bytes": (ctypes.c_size_t, [CFGP]),
    "tx_kv_pool_bytes": (ctypes.c_size_t, [CFGP, ctypes.c_int64, ctypes.c_int32, ctypes.c_int64]),
    "tx_kv_cache_create": (ctypes.c_int, [VP, VP, ctypes.c_size_t, ctypes.c_int64, ctypes.c_int32, ctypes.c_int64,
                                          ctypes.POINTER(VP)]),
    "tx_kv_cache_destroy": (None, [VP]),
    "tx_kv_cache_release": (ctypes.c_int, [VP, ctypes.c_int32, I32P]),
    "tx_kv_cache_length": (ctypes.c_int, [VP, ctypes.c_int32, I64P]),
    "tx_kv_cache_free_pages": (ctypes.c_int64, [VP]),
    "tx_kv_cache_model_id": (ctypes.c_uint64, [VP]),
    "tx_kv_cache_export": (ctypes.c_int, [VP, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, VP, VP]),
    "tx_workspace_bytes": (ctypes.c_size_t, [VP, ctypes.c_int32, ctypes.c_int32, I64P, I64P]),
    "tx_workspace_min_bytes": (ctypes.c_size_t, [VP, ctypes.c_int32, ctypes.c_int32, I64P, I64P]),
    "kv_cache_build": (ctypes.c_int, [VP, ctypes.c_int32, I32P, VP, I64P, VP, ctypes.c_size_t, VP]),
    "kv_cache_append": (ctypes.c_int, [VP, ctypes.c_int32, I32P, VP, I64P, VP, ctypes.c_size_t, VP]),
    "score_candidates": (ctypes.c_int, [VP, ctypes.c_int32, I32P, VP, I64P, VP, I64P, VP, VP, ctypes.c_size_t, VP]),
    "score_candidates_static": (ctypes.c_int, [VP, ctypes.c_int32, I32P, VP, I64P, VP, I64P, VP, VP]),
    "score_events": (ctypes.c_int, [VP, ctypes.c_int32, I32P, I64P, VP, I64P, VP, I64P, VP, VP, ctypes.c_size_t, VP]),
    "tx_rel_attn_workspace_bytes": (ctypes.c_size_t, [ACFGP, ctypes.c_int32, ctypes.c_int32, VP]),
    "tx_rel_attn_forward": (ctypes.c_int, [ACFGP, ctypes.c_int32, VP, ROWSP, ROWSP, ROWSP, VP, ROWSP, VP,
                                           ctypes.c_int64, VP, ctypes.c_size_t, VP]),
    "tx_rel_attn_backward": (ctypes.c_int, [ACFGP, ctypes.c_int32, VP, ROWSP, ROWSP, ROWSP, VP, ROWSP, VP,
                                            ctypes.c_int64, ROWSP, ROWSP, ROWSP, ROWSP, VP, VP, ctypes.c_size_t, VP]),
    "tx_event_attn_workspace_bytes": (ctypes.c_size_t, [ACFGP, ctypes.c_int32, ctypes.c_int32, VP, VP, VP, VP]),
    "tx_event_attn_forward": (ctypes.c_int, [ACFGP, ctypes.c_int32, VP, VP, VP, VP, ROWSP, ROWSP, ROWSP,
                                             ROWSP, VP, ctypes.c_int64, VP, ctypes.c_size_t, VP]),
    "tx_event_attn_backward": (ctypes.c_int, [ACFGP, ctypes.c_int32, VP, VP, VP, VP, ROWSP, ROWSP, ROWSP,
                                              ROWSP, VP, ctypes.c_int64, ROWSP, ROWSP, ROWSP, ROWSP, VP,
                                              ctypes.c_size_t, VP]),
    "tx_preference_workspace_bytes": (ctypes.c_size_t, [PCFGP, ctypes.c_int32, VP]),
    "tx_preference_forward": (ctypes.c_int, [PCFGP, ctypes.c_int32, VP, VP, ctypes.c_int64, VP, VP, VP, VP, VP, VP,
                                             ctypes.c_size_t, VP]),
    "tx_preference_backward": (ctypes.c_int, [PCFGP, ctypes.c_int32, VP, VP, ctypes.c_int64, VP, VP, VP, VP, VP, VP,
                                              ctypes.c_int64, VP, ctypes.c_size_t, VP]),
    "tx_profile_enable": (ctypes.c_int, [ctypes.c_int32]),
    "tx_profile_select": (ctypes.c_int, [ctypes.c_uint64]),
    "tx_profile_classes": (ctypes.c_int32, []),
    "tx_profile_class_name": (ctypes.c_char_p, [ctypes.c_int32]),
    "tx_profile_read": (ctypes.c_int, [ctypes.POINTER(ctypes.c_double), I64P, ctypes.POINTER(ctypes.c_double),
                                       ctypes.POINTER(ctypes.c_double)]),
}


def header_functions() -> List[str]:
    """Names of the functions include/transx.h declares."""
    text = open(HEADER).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    text = re.sub(r"^\s*#.*$", "", text, flags=re.M)  # preprocessor lines (macros)
    return sorted(set(re.findall(r"\b([A-Za-z_][A-Za-z0-9_]*)\s*\(", text)) -
                  {"if", "defined", "sizeof", "TRANSX_H"})


def lib():
    """Load libtransx.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build the HIP library first "
                               "(python -c 'import __graft_entry__ as g; g.build()')")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGS.items():
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _lib = L
    return _lib


def check(code: int):
    if code != TX_OK:
        msg = lib().tx_last_error().decode(errors="replace")
        raise TxError(code, msg)


def _i64(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a, dtype=np.int64))


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


def _p(a: np.ndarray, t):
    return a.ctypes.data_as(t)


def _stream(stream) -> int:
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return int(s.cuda_stream)


def _torch_dtype(m: ModelConfig):
    import torch
    return torch.bfloat16 if m.dtype == "bf16" else torch.float32


class Model:
    """Model config + repacked device weights (owns the repack buffer)."""

    def __init__(self, mc: ModelConfig, weights: Sequence, model_id: int = 1, device: str = "cuda", stream=None):
        import torch
        self.mc = mc
        self.cfg = Config.of(mc)
        L = lib()
        nbytes = L.tx_model_repack_bytes(ctypes.byref(self.cfg))
        if nbytes == 0:
            raise TxError(TX_E_INVALID, "unsupported model config")
        self.repack = torch.empty(nbytes, dtype=torch.uint8, device=device)
        h = VP()
        check(L.tx_model_create(ctypes.byref(self.cfg), VP(self.repack.data_ptr()), nbytes, model_id,
                                ctypes.byref(h)))
        self.handle = h
        dt = _torch_dtype(mc)
        src = [torch.as_tensor(np.asarray(w, dtype=np.float32)).to(dt).to(device).contiguous() for w in weights]
        ptrs = (VP * len(src))(*[VP(t.data_ptr()) if t.numel() else VP() for t in src])
        check(L.tx_model_set_weights(self.handle, ptrs, len(src), VP(_stream(stream))))
        (stream or torch.cuda.current_stream()).synchronize()  # sources may go now
        self.model_id = model_id

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.tx_model_destroy(self.handle)
            self.handle = None


class KVCache:
    """Paged per-request cache in a torch-owned device pool, plus a growable
    torch workspace reused across calls."""

    def __init__(self, model: Model, n_pages: int, max_requests: int, max_tokens: int, device: str = "cuda",
                 fill_byte: Optional[int] = None):
        import torch
        self.model = model
        L = lib()
        nbytes = L.tx_kv_pool_bytes(ctypes.byref(model.cfg), n_pages, max_requests, max_tokens)
        if nbytes == 0:
            raise TxError(TX_E_INVALID, "bad pool geometry")
        self.pool = torch.empty(nbytes, dtype=torch.uint8, device=device)
        if fill_byte is not None:
            self.pool.fill_(fill_byte)
        h = VP()
        check(L.tx_kv_cache_create(model.handle, VP(self.pool.data_ptr()), nbytes, n_pages, max_requests,
                                   max_tokens, ctypes.byref(h)))
        self.handle = h
        self.ws = None
        self.device = device

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.tx_kv_cache_destroy(self.handle)
            self.handle = None

    # ---------------------------------------------------------------- helpers
    def workspace(self, nbytes: int):
        import torch
        if self.ws is None or self.ws.numel() < nbytes:
            self.ws = None
            self.ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=self.device)
        return self.ws

    def workspace_bytes(self, op: int, n: int, a, b=None) -> int:
        a = _i64(a)
        bp = _p(_i64(b), I64P) if b is not None else None
        return int(lib().tx_workspace_bytes(self.handle, op, n, _p(a, I64P), bp))

    def workspace_min_bytes(self, op: int, n: int, a, b=None) -> int:
        a = _i64(a)
        bp = _p(_i64(b), I64P) if b is not None else None
        return int(lib().tx_workspace_min_bytes(self.handle, op, n, _p(a, I64P), bp))

    def _ws_for(self, op, n, a, b, ws_limit):
        need = self.workspace_bytes(op, n, a, b)
        if ws_limit is not None:
            need = min(need, max(int(ws_limit), self.workspace_min_bytes(op, n, a, b)))
        ws = self.workspace(need)
        return ws, need

    # ---------------------------------------------------------------- the path
    def build(self, req_ids, behavior, offsets, stream=None, ws_limit: Optional[int] = None):
        ids, off = _i32(req_ids), _i64(offsets)
        ws, n = self._ws_for(TX_OP_BUILD, len(ids), off, None, ws_limit)
        check(lib().kv_cache_build(self.handle, len(ids), _p(ids, I32P), VP(behavior.data_ptr()), _p(off, I64P),
                                   VP(ws.data_ptr()), n, VP(_stream(stream))))

    def append(self, req_ids, events, offsets, stream=None, ws_limit: Optional[int] = None):
        ids, off = _i32(req_ids), _i64(offsets)
        ws, n = self._ws_for(TX_OP_APPEND, len(ids), off, None, ws_limit)
        check(lib().kv_cache_append(self.handle, len(ids), _p(ids, I32P), VP(events.data_ptr()), _p(off, I64P),
                                    VP(ws.data_ptr()), n, VP(_stream(stream))))

    def score(self, req_ids, serving, serving_offsets, candidates, candidate_offsets, out=None, stream=None,
              ws_limit: Optional[int] = None):
        import torch
        ids, so, co = _i32(req_ids), _i64(serving_offsets), _i64(candidate_offsets)
        if out is None:
            n = int(co[-1]) if len(co) else 0
            k = self.model.mc.n_actions
            out = torch.empty((n, k) if k else n, dtype=torch.float32, device=self.device)
        ws, n = self._ws_for(TX_OP_SCORE, len(ids), so, co, ws_limit)
        check(lib().score_candidates(self.handle, len(ids), _p(ids, I32P), VP(serving.data_ptr()), _p(so, I64P),
                                     VP(candidates.data_ptr()), _p(co, I64P), VP(out.data_ptr()), VP(ws.data_ptr()),
                                     n, VP(_stream(stream))))
        return out

    def score_static(self, req_ids, serving, serving_offsets, candidates, candidate_offsets, out=None, stream=None):
        """score_candidates_static: no workspace argument, nothing allocated by
        the library (its fixed device array serves as the workspace)."""
        import torch
        ids, so, co = _i32(req_ids), _i64(serving_offsets), _i64(candidate_offsets)
        if out is None:
            n = int(co[-1]) if len(co) else 0
            k = self.model.mc.n_actions
            out = torch.empty((n, k) if k else n, dtype=torch.float32, device=self.device)
        check(lib().score_candidates_static(self.handle, len(ids), _p(ids, I32P), VP(serving.data_ptr()),
                                            _p(so, I64P), VP(candidates.data_ptr()), _p(co, I64P),
                                            VP(out.data_ptr()), VP(_stream(stream))))
        return out

    def score_events(self, req_ids, prefix_len, serving, serving_offsets, candidates, candidate_offsets, out=None,
                     stream=None, ws_limit: Optional[int] = None):
        """Event-sliced decoding: event e decodes against the first
        prefix_len[e] cached tokens of request req_ids[e] (ids may repeat)."""
        import torch
        ids, pre, so, co = _i32(req_ids), _i64(prefix_len), _i64(serving_offsets), _i64(candidate_offsets)
        if out is None:
            n = int(co[-1]) if len(co) else 0
            k = self.model.mc.n_actions
            out = torch.empty((n, k) if k else n, dtype=torch.float32, device=self.device)
        ws, n = self._ws_for(TX_OP_SCORE, len(ids), so, co, ws_limit)
        check(lib().score_events(self.handle, len(ids), _p(ids, I32P), _p(pre, I64P), VP(serving.data_ptr()),
                                 _p(so, I64P), VP(candidates.data_ptr()), _p(co, I64P), VP(out.data_ptr()),
                                 VP(ws.data_ptr()), n, VP(_stream(stream))))
        return out

    def release(self, req_ids):
        ids = _i32(req_ids)
        check(lib().tx_kv_cache_release(self.handle, len(ids), _p(ids, I32P)))

    def length(self, req_id: int) -> int:
        v = ctypes.c_int64()
        check(lib().tx_kv_cache_length(self.handle, req_id, ctypes.byref(v)))
        return v.value

    def free_pages(self) -> int:
        return int(lib().tx_kv_cache_free_pages(self.handle))

    def model_id(self) -> int:
        return int(lib().tx_kv_cache_model_id(self.handle))

    def export(self, req_id: int, part: int, layer: int, stream=None):
        """Cached tensor of a request as a dense [len, d] device tensor.
        part: 0 encoder K, 1 encoder V, 2 cross K, 3 cross V; 4 and 5 the
        global token's cross K and V (one row) of a model with global pooling."""
        import torch
        n = 1 if part >= 4 else self.length(req_id)
        out = torch.empty((max(n, 0), self.model.mc.d_model), dtype=_torch_dtype(self.model.mc), device=self.device)
        check(lib().tx_kv_cache_export(self.handle, req_id, part, layer, VP(out.data_ptr()), VP(_stream(stream))))
        return out


# ----------------------------------------------------------------- training
# Operators of a training step. Tensors are torch tensors on one GPU, host
# offsets anything numpy takes. A call runs on `stream` (default: the current
# stream of the tensors' device), which has to be ordered after the work that
# makes its inputs; outputs it allocates belong to that stream. Workspaces come
# from torch's allocator, one per call, so calls may be captured into graphs.

def _invalid(msg: str):
    raise TxError(TX_E_INVALID, msg)


class _On:
    """The tensors' device and the call's stream, current for the call."""

    def __init__(self, names: str, tensors, stream):
        import torch
        dev = None
        for i, t in enumerate(tensors):
            if t is None:
                continue
            if not (isinstance(t, torch.Tensor) and t.is_cuda):
                _invalid(f"{names.split()[i]} is not a GPU tensor")
            if dev is None:
                dev = t.device
            elif t.device != dev:
                _invalid(f"{names.split()[i]} is on {t.device}, other tensors are on {dev}")
        if stream is not None and stream.device != dev:
            _invalid(f"the stream belongs to {stream.device}, the tensors are on {dev}")
        self.dev, self.ctx = dev, None
        if stream is not None:
            self.ctx = torch.cuda.stream(stream)
        elif dev.index != torch.cuda.current_device():
            self.ctx = torch.cuda.device(dev)
        self.empty, self.uint8 = torch.empty, torch.uint8
        self.current = torch.cuda.current_stream

    def __enter__(self):
        if self.ctx is not None:
            self.ctx.__enter__()
        self.stream = self.current(self.dev).cuda_stream
        return self

    def __exit__(self, *exc):
        if self.ctx is not None:
            self.ctx.__exit__(*exc)

    def workspace(self, nbytes: int):
        # (0: the size function refused the arguments, and the call will say why)
        return self.empty(max(nbytes, 256), dtype=self.uint8, device=self.dev)


def _heads(t, name: str, dtype, shape=None) -> Rows:
    """[rows, heads, d_head] tensor, features contiguous, as the C ABI takes it."""
    if t.dim() != 3:
        _invalid(f"{name} must be [rows, heads, d_head]")
    if t.dtype != dtype:
        _invalid(f"{name} is {t.dtype}, q is {dtype}")
    n, h, d = t.shape
    if shape is not None and (n, h, d) != tuple(shape):
        _invalid(f"{name} is {(n, h, d)}, expected {tuple(shape)}")
    row, head, one = t.stride()
    if one != 1 and d > 1 and n * h:
        _invalid(f"{name}: features of a head must be contiguous")
    # (torch leaves the stride of a single row or head to chance)
    return Rows(t.data_ptr(), row if n > 1 else h * d, head if h > 1 else d)


def _plain(t, name: str, dtype, shape) -> int:
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        _invalid(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)}")
    return t.data_ptr()


def _dtype_of(t, name: str) -> int:
    import torch
    if t.dtype == torch.bfloat16:
        return TX_BF16
    if t.dtype == torch.float32:
        return TX_F32
    return _invalid(f"{name} is {t.dtype}: bfloat16 or float32")


def _attn_config(q, k, rel, scale) -> AttnConfig:
    if q.dim() != 3 or k.dim() != 3 or q.shape[2] != k.shape[2]:
        _invalid("q and k must be [rows, heads, d_head] of one d_head")
    R = 0
    if rel is not None:
        if rel.dim() != 2 or rel.shape[0] != q.shape[1] or not rel.is_contiguous() or rel.dtype != q.dtype:
            _invalid("rel must be a contiguous [heads, buckets] tensor of q's type")
        R = rel.shape[1]
    if scale is not None and not scale > 0:
        _invalid("scale must be positive")
    return AttnConfig(_dtype_of(q, "q"), q.shape[1], k.shape[1], q.shape[2], R, 0.0 if scale is None else float(scale))


def _offsets(a, name: str, n: Optional[int] = None) -> np.ndarray:
    a = _i64(a)
    if a.ndim != 1 or len(a) < 1 or (n is not None and len(a) != n):
        _invalid(f"{name} must be a vector of {n if n is not None else 'at least 1'} entries")
    return a


def _at(a: np.ndarray) -> int:
    return a.__array_interface__["data"][0]


def _covers(rows: int, off: np.ndarray, name: str) -> bool:
    """Whether the offsets take every row; refuses offsets past the last."""
    if off[-1] > rows:
        _invalid(f"{name} offsets reach row {int(off[-1])} of {rows}")
    return bool(off[0] == 0 and off[-1] == rows)


def _new_like(t, rows_used: bool):
    """Output of t's shape, head by head in a row; zeros when some rows belong to no group."""
    import torch
    return (torch.empty if rows_used else torch.zeros)(t.shape, dtype=t.dtype, device=t.device)


def _new_lse(H: int, M: int, full: bool, dev):
    import torch
    return torch.empty((H, M), dtype=torch.float32, device=dev) if full else \
        torch.full((H, M), -float("inf"), dtype=torch.float32, device=dev)


def _f32():
    import torch
    return torch.float32


def rel_attention(q, k, v, rel, offsets, scale: Optional[float] = None, out=None, lse=None, stream=None):
    """Causal self-attention of packed sequences with the encoder's learned
    relative position bias (tx_rel_attn_forward). q [rows, heads, d_head], k and
    v [rows, kv heads, d_head], rel [heads, buckets] or None. Returns out like q
    and lse fp32 [heads, rows]; rows outside the offsets keep what `out` and
    `lse` held (0 and -inf where this call makes them)."""
    off = _offsets(offsets, "sequence offsets")
    with _On("q k v rel out lse", (q, k, v, rel, out, lse), stream) as on:
        cfg = _attn_config(q, k, rel, scale)
        M, H, dt = q.shape[0], q.shape[1], q.dtype
        whole, kv = _covers(M, off, "sequence"), (M, k.shape[1], k.shape[2])
        out = _new_like(q, whole) if out is None else out
        lse = _new_lse(H, M, whole, on.dev) if lse is None else lse
        L, n, op = lib(), len(off) - 1, _at(off)
        ws = on.workspace(L.tx_rel_attn_workspace_bytes(cfg, 0, n, op))
        check(L.tx_rel_attn_forward(cfg, n, op, _heads(q, "q", dt), _heads(k, "k", dt, kv), _heads(v, "v", dt, kv),
                                    rel.data_ptr() if rel is not None else None, _heads(out, "out", dt, q.shape),
                                    _plain(lse, "lse", _f32(), (H, M)), M, ws.data_ptr(), ws.numel(), on.stream))
    return out, lse


def rel_attention_backward(dout, q, k, v, rel, out, lse, offsets, scale: Optional[float] = None, dq=None, dk=None,
                           dv=None, drel=None, stream=None):
    """Gradients of rel_attention for dout, given its inputs and outputs
    (tx_rel_attn_backward): dq, dk, dv and drel (None without a bias)."""
    off = _offsets(offsets, "sequence offsets")
    with _On("q k v rel out lse dout dq dk dv drel", (q, k, v, rel, out, lse, dout, dq, dk, dv, drel), stream) as on:
        cfg = _attn_config(q, k, rel, scale)
        M, H, dt = q.shape[0], q.shape[1], q.dtype
        whole, kv = _covers(M, off, "sequence"), (M, k.shape[1], k.shape[2])
        dq = _new_like(q, whole) if dq is None else dq
        dk = _new_like(k, whole) if dk is None else dk
        dv = _new_like(v, whole) if dv is None else dv
        rel_at = drel_at = None
        if rel is not None:
            drel = _new_like(rel, True) if drel is None else drel
            rel_at, drel_at = rel.data_ptr(), _plain(drel, "drel", dt, rel.shape)
        L, n, op = lib(), len(off) - 1, _at(off)
        ws = on.workspace(L.tx_rel_attn_workspace_bytes(cfg, 1, n, op))
        check(L.tx_rel_attn_backward(cfg, n, op, _heads(q, "q", dt), _heads(k, "k", dt, kv), _heads(v, "v", dt, kv),
                                     rel_at, _heads(out, "out", dt, q.shape), _plain(lse, "lse", _f32(), (H, M)), M,
                                     _heads(dout, "dout", dt, q.shape), _heads(dq, "dq", dt, q.shape),
                                     _heads(dk, "dk", dt, kv), _heads(dv, "dv", dt, kv), drel_at, ws.data_ptr(),
                                     ws.numel(), on.stream))
    return dq, dk, dv, (drel if rel is not None else None)


def _event_args(key_offsets, event_offsets, query_offsets, prefix_len):
    ko = _offsets(key_offsets, "key offsets")
    eo = _offsets(event_offsets, "event offsets", len(ko))
    if eo[0] != 0 or (eo[1:] < eo[:-1]).any():
        _invalid("event offsets must start at 0 and not decrease")
    qo = _offsets(query_offsets, "query offsets", int(eo[-1]) + 1)
    pre = _i64(prefix_len)
    if pre.ndim != 1 or len(pre) != int(eo[-1]):
        _invalid(f"prefix lengths must be a vector of {int(eo[-1])} entries")
    return ko, eo, qo, pre


def event_attention(q, k, v, key_offsets, event_offsets, query_offsets, prefix_len, scale: Optional[float] = None,
                    out=None, lse=None, stream=None):
    """Cross-attention of event-sliced decoding (tx_event_attn_forward): the
    query rows of event e see the first prefix_len[e] key rows of their user. q
    [query rows, heads, d_head], k and v [key rows, kv heads, d_head]. Returns
    out like q and lse fp32 [heads, query rows]."""
    where = _event_args(key_offsets, event_offsets, query_offsets, prefix_len)
    with _On("q k v out lse", (q, k, v, out, lse), stream) as on:
        cfg = _attn_config(q, k, None, scale)
        M, H, dt = q.shape[0], q.shape[1], q.dtype
        whole = _covers(M, where[2], "query")
        _covers(k.shape[0], where[0], "key")
        out = _new_like(q, whole) if out is None else out
        lse = _new_lse(H, M, whole, on.dev) if lse is None else lse
        L, n, wp = lib(), len(where[0]) - 1, [_at(x) for x in where]
        ws = on.workspace(L.tx_event_attn_workspace_bytes(cfg, 0, n, *wp))
        check(L.tx_event_attn_forward(cfg, n, *wp, _heads(q, "q", dt), _heads(k, "k", dt), _heads(v, "v", dt, k.shape),
                                      _heads(out, "out", dt, q.shape), _plain(lse, "lse", _f32(), (H, M)), M,
                                      ws.data_ptr(), ws.numel(), on.stream))
    return out, lse


def event_attention_backward(dout, q, k, v, out, lse, key_offsets, event_offsets, query_offsets, prefix_len,
                             scale: Optional[float] = None, dq=None, dk=None, dv=None, stream=None):
    """Gradients of event_attention for dout, given its inputs and outputs
    (tx_event_attn_backward): dq, dk, dv."""
    where = _event_args(key_offsets, event_offsets, query_offsets, prefix_len)
    with _On("q k v out lse dout dq dk dv", (q, k, v, out, lse, dout, dq, dk, dv), stream) as on:
        cfg = _attn_config(q, k, None, scale)
        M, H, dt = q.shape[0], q.shape[1], q.dtype
        whole, whole_k = _covers(M, where[2], "query"), _covers(k.shape[0], where[0], "key")
        dq = _new_like(q, whole) if dq is None else dq
        dk = _new_like(k, whole_k) if dk is None else dk
        dv = _new_like(v, whole_k) if dv is None else dv
        L, n, wp = lib(), len(where[0]) - 1, [_at(x) for x in where]
        ws = on.workspace(L.tx_event_attn_workspace_bytes(cfg, 1, n, *wp))
        check(L.tx_event_attn_backward(cfg, n, *wp, _heads(q, "q", dt), _heads(k, "k", dt), _heads(v, "v", dt, k.shape),
                                       _heads(out, "out", dt, q.shape), _plain(lse, "lse", _f32(), (H, M)), M,
                                       _heads(dout, "dout", dt, q.shape), _heads(dq, "dq", dt, q.shape),
                                       _heads(dk, "dk", dt, k.shape), _heads(dv, "dv", dt, k.shape), ws.data_ptr(),
                                       ws.numel(), on.stream))
    return dq, dk, dv


def _pref_args(logits, actions, offsets, beta, smoothing):
    import torch
    off = _offsets(offsets, "answer offsets")
    if len(off) % 2 == 0:
        _invalid("answer offsets must hold two answers per pair")
    if logits.dim() not in (1, 2) or (logits.dim() == 2 and logits.shape[1] > 1 and logits.stride(1) != 1):
        _invalid("logits must be [rows] or [rows, actions] with contiguous actions")
    if actions.dtype != torch.int32 or tuple(actions.shape) != (logits.shape[0],) or not actions.is_contiguous():
        _invalid("actions must be a contiguous int32 tensor with an entry per row")
    if logits.dim() == 2 and logits.shape[1] < 2:
        _invalid("logits need two actions or more (or [rows] for the scalar head)")
    whole = _covers(logits.shape[0], off, "answer")
    k = 1 if logits.dim() == 1 else logits.shape[1]
    return off, PreferenceConfig(_dtype_of(logits, "logits"), k, float(beta), float(smoothing)), whole


def _row_stride(t) -> int:
    return t.stride(0) if t.shape[0] > 1 else 1 if t.dim() == 1 else t.shape[1]


def preference_loss(logits, actions, offsets, ref_logp=None, beta: float = 0.1, smoothing: float = 0.0, stream=None):
    """Preference loss of paired answers (tx_preference_forward). logits [rows]
    (scalar head) or [rows, actions], actions int32 [rows], offsets of the answers
    (2p preferred, 2p + 1 not), ref_logp fp32 [answers] or None. Returns loss
    fp32 [pairs], logp fp32 [answers] and row_lse fp32 [rows] (for the backward)."""
    import torch
    f32 = torch.float32
    with _On("logits actions ref_logp", (logits, actions, ref_logp), stream) as on:
        off, cfg, _ = _pref_args(logits, actions, offsets, beta, smoothing)
        P = len(off) // 2
        ref = _plain(ref_logp, "ref_logp", f32, (2 * P,)) if ref_logp is not None else None
        loss, logp, row_lse = (torch.empty(n, dtype=f32, device=on.dev) for n in (P, 2 * P, logits.shape[0]))
        L, op = lib(), _at(off)
        ws = on.workspace(L.tx_preference_workspace_bytes(cfg, P, op))
        check(L.tx_preference_forward(cfg, P, op, logits.data_ptr(), _row_stride(logits), actions.data_ptr(), ref,
                                      loss.data_ptr(), logp.data_ptr(), row_lse.data_ptr(), ws.data_ptr(), ws.numel(),
                                      on.stream))
    return loss, logp, row_lse


def preference_loss_backward(dloss, logits, actions, offsets, ref_logp, logp, row_lse, beta: float = 0.1,
                             smoothing: float = 0.0, dlogits=None, stream=None):
    """d_logits of preference_loss for dloss fp32 [pairs] (tx_preference_backward);
    rows outside the offsets keep what `dlogits` held (0 where this call makes it)."""
    with _On("logits actions ref_logp logp row_lse dloss dlogits",
             (logits, actions, ref_logp, logp, row_lse, dloss, dlogits), stream) as on:
        off, cfg, whole = _pref_args(logits, actions, offsets, beta, smoothing)
        P, M, f32 = len(off) // 2, logits.shape[0], _f32()
        ref = _plain(ref_logp, "ref_logp", f32, (2 * P,)) if ref_logp is not None else None
        if dlogits is None:
            dlogits = _new_like(logits, whole)
        if dlogits.dtype != logits.dtype or dlogits.shape != logits.shape or \
                (dlogits.dim() == 2 and dlogits.stride(1) != 1):
            _invalid("dlogits must be like logits, actions contiguous")
        L, op = lib(), _at(off)
        ws = on.workspace(L.tx_preference_workspace_bytes(cfg, P, op))
        check(L.tx_preference_backward(cfg, P, op, logits.data_ptr(), _row_stride(logits), actions.data_ptr(), ref,
                                       _plain(logp, "logp", f32, (2 * P,)), _plain(row_lse, "row_lse", f32, (M,)),
                                       _plain(dloss, "dloss", f32, (P,)), dlogits.data_ptr(), _row_stride(dlogits),
                                       ws.data_ptr(), ws.numel(), on.stream))
    return dlogits


def profile_enable(on: bool = True):
    check(lib().tx_profile_enable(1 if on else 0))


def profile_select(classes) -> None:
    """Record only the named kernel classes (until profile_enable)."""
    L = lib()
    names = [L.tx_profile_class_name(i).decode() for i in range(L.tx_profile_classes())]
    mask = 0
    for c in classes:
        mask |= 1 << names.index(c)
    check(L.tx_profile_select(mask))


def profile_read() -> dict:
    """{class name: {"ms": total, "launches": n, "flops": F, "bytes": B}} for
    classes with at least one recorded launch."""
    L = lib()
    k = L.tx_profile_classes()
    ms, fl, by = (np.zeros(k) for _ in range(3))
    n = np.zeros(k, dtype=np.int64)
    D = ctypes.POINTER(ctypes.c_double)
    check(L.tx_profile_read(_p(ms, D), _p(n, I64P), _p(fl, D), _p(by, D)))
    return {L.tx_profile_class_name(i).decode(): {"ms": float(ms[i]), "launches": int(n[i]), "flops": float(fl[i]),
                                                  "bytes": float(by[i])} for i in range(k) if n[i] > 0}


def to_device(x: np.ndarray, mc: ModelConfig, device: str = "cuda"):
    """Host float32 array holding stored values -> device tensor of the model dtype."""
    import torch
    return torch.as_tensor(np.ascontiguousarray(x, dtype=np.float32)).to(_torch_dtype(mc)).to(device)
