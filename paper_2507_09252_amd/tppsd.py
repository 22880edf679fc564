"""Python binding of libtppsd (the C ABI declared in include/tppsd.h).

Argument marshalling only: every step of the sampler runs in the HIP library.
torch provides device memory and the stream (its current HIP stream); torch
must be imported before the library is loaded so both use the same HIP
runtime. If the library has not been built, loading fails loudly: there is no
fallback.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import POINTER, c_char_p, c_double, c_int, c_int32, c_int64, c_size_t, c_uint, c_uint32, c_uint64, c_void_p
from typing import Dict, Optional

import numpy as np
import torch  # noqa: F401  (loads torch's HIP runtime first)

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libtppsd.so")

TPPSD_OK = 0
PREC = {"fp32": 0, "bf16": 1}
FLAG_BONUS, FLAG_CACHE8 = 1, 2
STATUS_CAPACITY, STATUS_NONFINITE, STATUS_AR_CAP = 1, 2, 4
STATUS_PAGES, STATUS_SEQUENCE, STATUS_OPEN = 8, 16, 32
CACHE_BLOCK, CACHE_RING = 64, 128

ERRORS = {1: "TPPSD_E_ARG", 2: "TPPSD_E_CONFIG", 3: "TPPSD_E_WORKSPACE", 4: "TPPSD_E_ORDER", 5: "TPPSD_E_HIP"}

# every symbol the header declares
EXPORTS = [
    "tppsd_weights_bytes", "tppsd_weights_entry", "tppsd_model_create", "tppsd_model_destroy",
    "tppsd_state_bytes", "tppsd_state_create", "tppsd_state_destroy", "tppsd_prefill", "tppsd_draft",
    "tppsd_verify", "tppsd_accept", "tppsd_sample_ar", "tppsd_sample_sd", "tppsd_read_events",
    "tppsd_state_status", "tppsd_timing_enable", "tppsd_timing_read", "tppsd_last_error",
    "tppsd_poisson_fit", "tppsd_draft_poisson", "tppsd_sample_sd_poisson", "tppsd_prefill_window",
    "tppsd_read_loglik", "tppsd_verify_noalloc",
    "tppsd_cache_bytes", "tppsd_cache_entry", "tppsd_cache_create", "tppsd_cache_destroy", "tppsd_cache_reset",
    "tppsd_cache_begin", "tppsd_cache_append", "tppsd_cache_attend", "tppsd_cache_commit", "tppsd_cache_truncate",
    "tppsd_cache_fork", "tppsd_cache_copy", "tppsd_cache_read", "tppsd_cache_status",
    "tppsd_state_bytes_flags", "tppsd_state_fork",
]


class TppsdError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"{ERRORS.get(code, code)}: {msg}")
        self.code = code


TIME_KERNELS = 1   # TPPSD_TIME_KERNELS
TIME_PHASES = 2    # TPPSD_TIME_PHASES


class TimingC(ctypes.Structure):
    _fields_ = [("attn_ms", c_double), ("attn_launches", c_int64), ("gemm_ms", c_double),
                ("gemm_launches", c_int64), ("gemm_flop", c_double), ("draft_ms", c_double),
                ("verify_ms", c_double), ("accept_ms", c_double), ("rounds", c_int64),
                ("draft_kernel_ms", c_double), ("draft_kernel_launches", c_int64),
                ("draft_attn_ms", c_double), ("draft_attn_launches", c_int64),
                ("draft_rows_ms", c_double), ("draft_rows_launches", c_int64)]


ENCODER = {"thp": 0, "attnhp": 1}   # TPPSD_ENC_*


class ModelCfgC(ctypes.Structure):
    _fields_ = [(n, c_int32) for n in ("n_layers", "d_model", "n_heads", "d_ffn", "n_mix", "n_types", "prec",
                                       "encoder")] + [("time_m", ctypes.c_float), ("time_M", ctypes.c_float)]


class DraftBufC(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in ("tau", "t", "k", "logg", "logf", "mix", "logtype", "rate")]


class VerifyBufC(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in ("logg", "logf", "mix", "logtype")]


class AcceptBufC(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in ("L", "n_new", "k_new", "t_new", "tau_new", "ar_iter", "flags")]


class CacheCfgC(ctypes.Structure):
    _fields_ = [(n, c_int32) for n in ("n_layers", "n_heads", "n_kv_heads", "d_head", "prec", "max_seqs", "max_events",
                                       "n_pages")]


class CacheRowsC(ctypes.Structure):
    _fields_ = [(n, c_void_p) for n in ("q", "k", "v", "o")] + [(n, c_int64) for n in ("ldq", "ldk", "ldv", "ldo")]


_lib = None


def lib():
    """Load libtppsd.so (built in-tree); raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is not built; run __graft_entry__.build() "
                           "(python paper_2507_09252_amd/build.py)")
    L = ctypes.CDLL(LIB_PATH)
    P = POINTER
    sig = {
        "tppsd_weights_bytes": (c_int, [P(ModelCfgC), P(c_size_t)]),
        "tppsd_weights_entry": (c_int, [P(ModelCfgC), c_int, P(c_char_p), P(c_size_t), P(c_int64), P(c_int64), P(c_int)]),
        "tppsd_model_create": (c_int, [P(ModelCfgC), c_void_p, P(c_void_p)]),
        "tppsd_model_destroy": (None, [c_void_p]),
        "tppsd_state_bytes": (c_int, [c_void_p, c_void_p, c_int, c_int, c_int, P(c_size_t)]),
        "tppsd_state_create": (c_int, [c_void_p, c_void_p, c_int, c_int, c_int, c_uint64, c_uint, c_void_p,
                                       c_size_t, P(c_void_p)]),
        "tppsd_state_destroy": (None, [c_void_p]),
        "tppsd_prefill": (c_int, [c_void_p, c_void_p, c_void_p, c_int, c_int, c_void_p]),
        "tppsd_draft": (c_int, [c_void_p, c_int, P(DraftBufC), c_void_p]),
        "tppsd_verify": (c_int, [c_void_p, c_int, P(DraftBufC), P(VerifyBufC), c_void_p]),
        "tppsd_verify_noalloc": (c_int, [c_void_p, c_int, P(DraftBufC), P(VerifyBufC), c_void_p]),
        "tppsd_accept": (c_int, [c_void_p, c_int, P(DraftBufC), P(VerifyBufC), c_void_p, P(AcceptBufC), c_void_p]),
        "tppsd_sample_ar": (c_int, [c_void_p, c_int, c_void_p, c_void_p, c_void_p]),
        "tppsd_sample_sd": (c_int, [c_void_p, c_int, c_int, P(c_int), c_void_p]),
        "tppsd_read_events": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]),
        "tppsd_state_status": (c_int, [c_void_p, c_void_p, P(c_uint32), P(c_int32), P(c_int64), P(c_int64), P(c_int64)]),
        "tppsd_timing_enable": (c_int, [c_void_p, c_int]),
        "tppsd_timing_read": (c_int, [c_void_p, P(TimingC)]),
        "tppsd_last_error": (c_char_p, []),
        "tppsd_poisson_fit": (c_int, [c_void_p, c_void_p, c_int, c_int, c_int, c_void_p, c_void_p]),
        "tppsd_draft_poisson": (c_int, [c_void_p, c_int, c_void_p, P(DraftBufC), c_void_p]),
        "tppsd_sample_sd_poisson": (c_int, [c_void_p, c_int, c_void_p, c_int, P(c_int), c_void_p]),
        "tppsd_prefill_window": (c_int, [c_void_p, c_void_p, c_void_p, c_int, c_int, c_void_p, c_void_p]),
        "tppsd_read_loglik": (c_int, [c_void_p, c_void_p, c_void_p]),
        "tppsd_state_bytes_flags": (c_int, [c_void_p, c_void_p, c_int, c_int, c_int, c_uint, P(c_size_t)]),
        "tppsd_state_fork": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p]),
        "tppsd_cache_bytes": (c_int, [P(CacheCfgC), P(c_size_t)]),
        "tppsd_cache_entry": (c_int, [P(CacheCfgC), c_int, P(c_char_p), P(c_size_t)]),
        "tppsd_cache_create": (c_int, [P(CacheCfgC), c_void_p, c_size_t, P(c_void_p)]),
        "tppsd_cache_destroy": (None, [c_void_p]),
        "tppsd_cache_reset": (c_int, [c_void_p, c_void_p]),
        "tppsd_cache_begin": (c_int, [c_void_p, c_int, c_int, c_void_p, c_void_p, c_void_p]),
        "tppsd_cache_append": (c_int, [c_void_p, c_int, P(CacheRowsC), c_void_p]),
        "tppsd_cache_attend": (c_int, [c_void_p, c_int, P(CacheRowsC), ctypes.c_float, c_int, c_void_p]),
        "tppsd_cache_commit": (c_int, [c_void_p, c_void_p, c_void_p]),
        "tppsd_cache_truncate": (c_int, [c_void_p, c_int, c_void_p, c_void_p, c_void_p]),
        "tppsd_cache_fork": (c_int, [c_void_p, c_int, c_void_p, c_void_p, c_void_p]),
        "tppsd_cache_copy": (c_int, [c_void_p, c_void_p, c_int, c_void_p, c_void_p, c_void_p]),
        "tppsd_cache_read": (c_int, [c_void_p, c_int, c_int, c_void_p, c_void_p, c_int, c_void_p, c_void_p,
                                     c_void_p]),
        "tppsd_cache_status": (c_int, [c_void_p, c_void_p, P(c_uint32)]),
    }
    for name, (res, args) in sig.items():
        f = getattr(L, name)
        f.restype = res
        f.argtypes = args
    _lib = L
    return L


def _check(rc):
    if rc != TPPSD_OK:
        raise TppsdError(rc, lib().tppsd_last_error().decode())


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else c_void_p(t.data_ptr())


def _stream():
    return c_void_p(torch.cuda.current_stream().cuda_stream)


def cfg_c(cfg) -> ModelCfgC:
    return ModelCfgC(cfg.n_layers, cfg.d_model, cfg.n_heads, cfg.d_ffn, cfg.n_mix, cfg.n_types, PREC[cfg.prec],
                     ENCODER[getattr(cfg, "encoder", "thp")], float(getattr(cfg, "time_m", 1.0)),
                     float(getattr(cfg, "time_M", 100.0)))


# ---------------------------------------------------------------------------
# weights
# ---------------------------------------------------------------------------

def tppsd_weights_bytes(cfg) -> int:
    n = c_size_t()
    _check(lib().tppsd_weights_bytes(ctypes.byref(cfg_c(cfg)), ctypes.byref(n)))
    return n.value


def weights_layout(cfg):
    """[(name, offset, rows, cols, is_bf16)] of the packed layout, from the library."""
    out, i = [], 0
    c = cfg_c(cfg)
    L = lib()
    while True:
        name, off, r, cl, bf = c_char_p(), c_size_t(), c_int64(), c_int64(), c_int()
        rc = L.tppsd_weights_entry(ctypes.byref(c), i, ctypes.byref(name), ctypes.byref(off), ctypes.byref(r),
                                   ctypes.byref(cl), ctypes.byref(bf))
        if rc != TPPSD_OK:
            break
        out.append((name.value.decode(), off.value, r.value, cl.value, bf.value))
        i += 1
    return out


def pack_weights(cfg, weights: Dict[str, np.ndarray], device="cuda") -> torch.Tensor:
    """Packs named parameters into the library's device layout (a uint8 tensor)."""
    total = tppsd_weights_bytes(cfg)
    buf = torch.zeros(total, dtype=torch.uint8)
    for name, off, r, cl, bf in weights_layout(cfg):
        a = np.asarray(weights[name], dtype=np.float32).reshape(r * cl)
        t = torch.from_numpy(a.copy())
        if bf:
            t = t.to(torch.bfloat16)
        raw = t.view(torch.uint8)
        buf[off:off + raw.numel()] = raw
    return buf.to(device)


class Model:
    """tppsd_model handle over packed device weights (kept alive here)."""

    def __init__(self, cfg, weights: Dict[str, np.ndarray], device="cuda"):
        self.cfg = cfg
        self.wbuf = pack_weights(cfg, weights, device)
        h = c_void_p()
        _check(lib().tppsd_model_create(ctypes.byref(cfg_c(cfg)), _ptr(self.wbuf), ctypes.byref(h)))
        self.handle = h

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.tppsd_model_destroy(self.handle)
            self.handle = None


def tppsd_poisson_fit(t: torch.Tensor, k: torch.Tensor, K: int) -> torch.Tensor:
    """Homogeneous-Poisson draft parameters [1 + K] (rate, log p) fitted on the
    device from sequences t/k [B, n0]."""
    t = t.to(torch.float32).contiguous()
    k = k.to(torch.int32).contiguous()
    params = torch.empty(1 + K, dtype=torch.float32, device=t.device)
    _check(lib().tppsd_poisson_fit(_ptr(t), _ptr(k), t.shape[0], t.shape[1], K, _ptr(params), _stream()))
    return params


# ---------------------------------------------------------------------------
# round buffers
# ---------------------------------------------------------------------------

class DraftBuffers:
    """Draft record; poisson=True makes the record of a homogeneous-Poisson
    draft (a rate array, no mixture)."""

    def __init__(self, B, max_gamma, M, K, device="cuda", poisson=False):
        f = dict(dtype=torch.float32, device=device)
        self.tau = torch.zeros(B, max_gamma, **f)
        self.t = torch.zeros(B, max_gamma, **f)
        self.k = torch.zeros(B, max_gamma, dtype=torch.int32, device=device)
        self.logg = torch.zeros(B, max_gamma, **f)
        self.logf = torch.zeros(B, max_gamma, **f)
        self.mix = None if poisson else torch.zeros(B, max_gamma, 3, M, **f)
        self.logtype = torch.zeros(B, max_gamma, K, **f)
        self.rate = torch.zeros(B, **f) if poisson else None

    def c(self):
        return DraftBufC(*(None if t is None else t.data_ptr()
                           for t in (self.tau, self.t, self.k, self.logg, self.logf, self.mix, self.logtype,
                                     self.rate)))


class VerifyBuffers:
    def __init__(self, B, max_gamma, M, K, device="cuda"):
        f = dict(dtype=torch.float32, device=device)
        self.logg = torch.zeros(B, max_gamma, **f)
        self.logf = torch.zeros(B, max_gamma, **f)
        self.mix = torch.zeros(B, max_gamma + 1, 3, M, **f)
        self.logtype = torch.zeros(B, max_gamma + 1, K, **f)

    def c(self):
        return VerifyBufC(*(t.data_ptr() for t in (self.logg, self.logf, self.mix, self.logtype)))


class AcceptBuffers:
    def __init__(self, B, max_gamma, device="cuda"):
        i = dict(dtype=torch.int32, device=device)
        self.L = torch.zeros(B, **i)
        self.n_new = torch.zeros(B, **i)
        self.k_new = torch.zeros(B, max_gamma + 1, **i)
        self.t_new = torch.zeros(B, max_gamma + 1, dtype=torch.float32, device=device)
        self.tau_new = torch.zeros(B, max_gamma + 1, dtype=torch.float32, device=device)
        self.ar_iter = torch.zeros(B, **i)
        self.flags = torch.zeros(B, dtype=torch.uint8, device=device)

    def c(self):
        return AcceptBufC(*(t.data_ptr() for t in (self.L, self.n_new, self.k_new, self.t_new, self.tau_new,
                                                    self.ar_iter, self.flags)))


# ---------------------------------------------------------------------------
# sampler state
# ---------------------------------------------------------------------------

class State:
    """tppsd_state over a torch-allocated workspace; methods map 1:1 to the C ABI.
    cache8: the target's keys and values in an 8-bit paged cache (TPPSD_FLAG_CACHE8)."""

    def __init__(self, target: Model, draft: Optional[Model], B: int, max_events: int, max_gamma: int,
                 seed: int = 0, bonus: bool = True, device="cuda", cache8: bool = False):
        self.target, self.draft = target, draft
        self.B, self.max_events, self.max_gamma = B, max_events, max_gamma
        n = c_size_t()
        dh = draft.handle if draft is not None else None
        flags = (FLAG_BONUS if bonus else 0) | (FLAG_CACHE8 if cache8 else 0)
        _check(lib().tppsd_state_bytes_flags(target.handle, dh, B, max_events, max_gamma, flags, ctypes.byref(n)))
        self.ws = torch.empty(n.value, dtype=torch.uint8, device=device)
        h = c_void_p()
        _check(lib().tppsd_state_create(target.handle, dh, B, max_events, max_gamma, c_uint64(seed),
                                        flags, _ptr(self.ws), n.value, ctypes.byref(h)))
        self.handle = h

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.tppsd_state_destroy(self.handle)
            self.handle = None

    def tppsd_prefill(self, t: torch.Tensor, k: torch.Tensor, n_gen: int, t_end: Optional[torch.Tensor] = None):
        """t_end [B] (optional): per-sequence end time (tppsd_prefill_window)."""
        t = t.contiguous()
        k = k.to(torch.int32).contiguous()
        self._hist = (t, k)
        if t_end is None:
            _check(lib().tppsd_prefill(self.handle, _ptr(t), _ptr(k), t.shape[1], n_gen, _stream()))
        else:
            t_end = t_end.to(torch.float32).contiguous()
            self._t_end = t_end
            _check(lib().tppsd_prefill_window(self.handle, _ptr(t), _ptr(k), t.shape[1], n_gen, _ptr(t_end),
                                              _stream()))

    def tppsd_state_fork(self, source: "State", parent: torch.Tensor):
        """Sequence b becomes a copy of source's sequence parent[b] (source may be self)."""
        parent = parent.to(torch.int32).contiguous()
        if parent.numel() != self.B or parent.device != self.ws.device:
            raise TppsdError(1, f"parent must hold {self.B} sequences on {self.ws.device}")
        if source.ws.device != self.ws.device:
            raise TppsdError(1, "states lie on different devices")
        self._parent = parent
        _check(lib().tppsd_state_fork(self.handle, source.handle, _ptr(parent), _stream()))

    def tppsd_draft(self, gamma: int, out: DraftBuffers):
        _check(lib().tppsd_draft(self.handle, gamma, ctypes.byref(out.c()), _stream()))

    def tppsd_draft_poisson(self, gamma: int, params: torch.Tensor, out: DraftBuffers):
        _check(lib().tppsd_draft_poisson(self.handle, gamma, _ptr(params), ctypes.byref(out.c()), _stream()))

    def tppsd_verify(self, gamma: int, drafts: DraftBuffers, out: VerifyBuffers):
        _check(lib().tppsd_verify(self.handle, gamma, ctypes.byref(drafts.c()), ctypes.byref(out.c()), _stream()))

    def tppsd_verify_noalloc(self, gamma: int, drafts: DraftBuffers, out: VerifyBuffers):
        _check(lib().tppsd_verify_noalloc(self.handle, gamma, ctypes.byref(drafts.c()), ctypes.byref(out.c()),
                                          _stream()))

    def tppsd_accept(self, gamma: int, drafts: DraftBuffers, verify: VerifyBuffers, out: AcceptBuffers,
                     uniforms: Optional[torch.Tensor] = None):
        _check(lib().tppsd_accept(self.handle, gamma, ctypes.byref(drafts.c()), ctypes.byref(verify.c()),
                                  _ptr(uniforms), ctypes.byref(out.c()), _stream()))

    def tppsd_sample_ar(self, n_events: int, t_out: Optional[torch.Tensor] = None,
                        k_out: Optional[torch.Tensor] = None):
        _check(lib().tppsd_sample_ar(self.handle, n_events, _ptr(t_out), _ptr(k_out), _stream()))

    def tppsd_sample_sd(self, gamma: int, max_rounds: int = 1 << 30) -> int:
        r = c_int()
        _check(lib().tppsd_sample_sd(self.handle, gamma, max_rounds, ctypes.byref(r), _stream()))
        return r.value

    def tppsd_sample_sd_poisson(self, gamma: int, params: torch.Tensor, max_rounds: int = 1 << 30) -> int:
        r = c_int()
        _check(lib().tppsd_sample_sd_poisson(self.handle, gamma, _ptr(params), max_rounds, ctypes.byref(r),
                                             _stream()))
        return r.value

    def tppsd_read_events(self):
        t = torch.empty(self.B, self.max_events, dtype=torch.float32, device=self.ws.device)
        k = torch.empty(self.B, self.max_events, dtype=torch.int32, device=self.ws.device)
        n = torch.empty(self.B, dtype=torch.int32, device=self.ws.device)
        _check(lib().tppsd_read_events(self.handle, _ptr(t), _ptr(k), _ptr(n), _stream()))
        return t, k, n

    def tppsd_read_loglik(self) -> torch.Tensor:
        ll = torch.empty(self.B, dtype=torch.float64, device=self.ws.device)
        _check(lib().tppsd_read_loglik(self.handle, _ptr(ll), _stream()))
        return ll

    def tppsd_state_status(self):
        bits, nd, acc, dr, ar = c_uint32(), c_int32(), c_int64(), c_int64(), c_int64()
        _check(lib().tppsd_state_status(self.handle, _stream(), ctypes.byref(bits), ctypes.byref(nd),
                                        ctypes.byref(acc), ctypes.byref(dr), ctypes.byref(ar)))
        return dict(bits=bits.value, n_done=nd.value, accepted=acc.value, drafted=dr.value, ar_candidates=ar.value)

    def tppsd_timing_enable(self, modes: int):
        """modes: 0 (off), TIME_KERNELS or TIME_PHASES."""
        _check(lib().tppsd_timing_enable(self.handle, int(modes)))

    def tppsd_timing_read(self):
        t = TimingC()
        _check(lib().tppsd_timing_read(self.handle, ctypes.byref(t)))
        return {name: getattr(t, name) for name, _ in TimingC._fields_}


# ---------------------------------------------------------------------------
# 8-bit paged cache
# ---------------------------------------------------------------------------

class Cache:
    """tppsd_cache over a torch-allocated workspace, emptied; methods map 1:1 to
    the C ABI. Rows are tensors [B, n_new, heads, d_head] whose heads are
    contiguous ([d_head] elements each) and whose rows of the batch are n_new
    positions apart (a slice of a fused projection's output is taken as it is).
    Index tensors are int32 on the cache's device.

    pages, scales, tails, table, lens, refs: views of the cache's arrays."""

    def __init__(self, n_layers: int, n_heads: int, n_kv_heads: int, d_head: int, prec: str, max_seqs: int,
                 max_events: int, n_pages: int = 0, device="cuda"):
        self.n_layers, self.n_heads, self.n_kv_heads, self.d_head = n_layers, n_heads, n_kv_heads, d_head
        self.max_seqs, self.max_events = max_seqs, max_events
        self.dtype = torch.bfloat16 if prec == "bf16" else torch.float32
        cfg = CacheCfgC(n_layers, n_heads, n_kv_heads, d_head, PREC[prec], max_seqs, max_events, n_pages)
        n = c_size_t()
        _check(lib().tppsd_cache_bytes(ctypes.byref(cfg), ctypes.byref(n)))
        self.ws = torch.zeros(n.value, dtype=torch.uint8, device=device)
        h = c_void_p()
        _check(lib().tppsd_cache_create(ctypes.byref(cfg), _ptr(self.ws), n.value, ctypes.byref(h)))
        self.handle, self._dev = h, self.ws.get_device()
        np_ = (max_events + CACHE_BLOCK - 1) // CACHE_BLOCK
        self.n_pages = n_pages or np_ * max_seqs
        L, S, KV, dh, N = n_layers, max_seqs, n_kv_heads, d_head, self.n_pages
        shapes = {"pages": (torch.uint8, (L, N, KV, 2 * CACHE_BLOCK * dh)), "scales": (torch.float32, (L, N, KV, 2)),
                  "tails": (self.dtype, (L, S, KV, 2, CACHE_RING, dh)), "table": (torch.int32, (S, np_)),
                  "lens": (torch.int32, (S,)), "refs": (torch.int32, (N,))}
        for i in range(len(shapes)):
            name, off = c_char_p(), c_size_t()
            _check(lib().tppsd_cache_entry(ctypes.byref(cfg), i, ctypes.byref(name), ctypes.byref(off)))
            dt, shape = shapes[name.value.decode()]
            size = int(np.prod(shape)) * torch.empty(0, dtype=dt).element_size()
            setattr(self, name.value.decode(), self.ws[off.value:off.value + size].view(dt).view(shape))
        self.tppsd_cache_reset()

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.tppsd_cache_destroy(self.handle)
            self.handle = None

    # (decoding loops call these once per layer and step: plain integers go to
    # the library, and a tensor's properties are looked at once)
    def _call(self, fn, *args):
        """The entry point on this cache's device and that device's current stream."""
        dev = self._dev
        if dev == torch.cuda.current_device():
            _check(fn(self.handle, *args, torch.cuda.current_stream(dev).cuda_stream))
        else:
            with torch.cuda.device(dev):
                _check(fn(self.handle, *args, torch.cuda.current_stream(dev).cuda_stream))

    def _ints(self, t, n=None, what="index"):
        """Address of an index vector (None: NULL)."""
        if t is None:
            return None
        if t.dtype is not torch.int32 or t.get_device() != self._dev or t.dim() != 1 or not t.is_contiguous():
            raise TppsdError(1, f"{what} must be a contiguous int32 vector on {self.ws.device}")
        if n is not None and t.numel() != n:
            raise TppsdError(1, f"{what} has {t.numel()} elements, needs {n}")
        return t.data_ptr()

    def _row(self, t, heads, what):
        """Address and row stride of rows [B, n_new, heads, d_head]."""
        B, P = self._plan
        dh = self.d_head
        if t.dtype is not self.dtype or t.get_device() != self._dev or t.shape != (B, P, heads, dh):
            raise TppsdError(1, f"{what} must be {self.dtype} [{B}, {P}, {heads}, {dh}] on {self.ws.device}")
        if t.is_contiguous():
            return t.data_ptr(), heads * dh
        sb, sp, sh, sd = t.stride()
        ld = sp if P > 1 else (sb if B > 1 else heads * dh)
        if sd != 1 or (heads > 1 and sh != dh) or (B > 1 and sb != P * ld):
            raise TppsdError(1, f"{what}: heads must be contiguous and rows evenly spaced")
        return t.data_ptr(), ld

    def tppsd_cache_reset(self):
        self._call(_lib.tppsd_cache_reset)
        self._plan = None

    def tppsd_cache_begin(self, n_new: int, seqs: Optional[torch.Tensor] = None,
                          counts: Optional[torch.Tensor] = None, batch: Optional[int] = None):
        """batch: rows of the call (default: as many as seqs or counts has, or every sequence)."""
        if batch is None:
            batch = seqs.numel() if seqs is not None else counts.numel() if counts is not None else self.max_seqs
        self._call(_lib.tppsd_cache_begin, batch, n_new, self._ints(seqs, batch, "seqs"),
                   self._ints(counts, batch, "counts"))
        self._plan = (batch, n_new)

    def _planned(self):
        if self._plan is None:
            raise TppsdError(4, "call tppsd_cache_begin first")

    def tppsd_cache_append(self, layer: int, k: torch.Tensor, v: torch.Tensor):
        self._planned()
        (kp, ldk), (vp, ldv) = self._row(k, self.n_kv_heads, "k"), self._row(v, self.n_kv_heads, "v")
        r = CacheRowsC(None, kp, vp, None, 0, ldk, ldv, 0)
        self._call(_lib.tppsd_cache_append, layer, ctypes.byref(r))

    def tppsd_cache_attend(self, layer: int, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                           out: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                           sink: bool = False) -> torch.Tensor:
        """scale: default 1 / sqrt(d_head); out: default a new tensor, zero where rows are left out."""
        self._planned()
        if out is None:
            out = torch.zeros(q.shape, dtype=q.dtype, device=q.device)
        (qp, ldq), (op, ldo) = self._row(q, self.n_heads, "q"), self._row(out, self.n_heads, "out")
        (kp, ldk), (vp, ldv) = self._row(k, self.n_kv_heads, "k"), self._row(v, self.n_kv_heads, "v")
        r = CacheRowsC(qp, kp, vp, op, ldq, ldk, ldv, ldo)
        self._call(_lib.tppsd_cache_attend, layer, ctypes.byref(r),
                   self.d_head ** -0.5 if scale is None else scale, int(sink))
        return out

    def tppsd_cache_commit(self, accept: Optional[torch.Tensor] = None):
        self._planned()
        self._call(_lib.tppsd_cache_commit, self._ints(accept, self._plan[0], "accept"))
        self._plan = None

    def tppsd_cache_truncate(self, seqs: torch.Tensor, lens: Optional[torch.Tensor] = None):
        n = seqs.numel()
        self._call(_lib.tppsd_cache_truncate, n, self._ints(seqs, n, "seqs"), self._ints(lens, n, "lens"))
        self._plan = None

    def tppsd_cache_fork(self, src: torch.Tensor, dst: torch.Tensor):
        n = src.numel()
        self._call(_lib.tppsd_cache_fork, n, self._ints(src, n, "src"), self._ints(dst, n, "dst"))
        self._plan = None

    def tppsd_cache_copy(self, source: "Cache", src: torch.Tensor, dst: torch.Tensor):
        """Sequences src of the cache `source` into this cache's sequences dst."""
        n = src.numel()
        if source.ws.device != self.ws.device:
            raise TppsdError(1, "caches lie on different devices")
        self._call(_lib.tppsd_cache_copy, source.handle, n, self._ints(src, n, "src"), self._ints(dst, n, "dst"))
        self._plan = None

    def tppsd_cache_read(self, layer: int, first: Optional[torch.Tensor], count: int,
                         k: Optional[torch.Tensor] = None, v: Optional[torch.Tensor] = None,
                         seqs: Optional[torch.Tensor] = None):
        """(k, v) [n, count, n_kv_heads, d_head] of positions first .. first + count - 1 (default 0)."""
        n = seqs.numel() if seqs is not None else first.numel() if first is not None else self.max_seqs
        shape = (n, count, self.n_kv_heads, self.d_head)
        if k is None:
            k = torch.zeros(shape, dtype=self.dtype, device=self.ws.device)
        if v is None:
            v = torch.zeros(shape, dtype=self.dtype, device=self.ws.device)
        for t in (k, v):
            if t.shape != shape or t.dtype is not self.dtype or t.get_device() != self._dev or not t.is_contiguous():
                raise TppsdError(1, f"outputs must be contiguous {self.dtype} {list(shape)}")
        self._call(_lib.tppsd_cache_read, layer, n, self._ints(seqs, n, "seqs"), self._ints(first, n, "first"), count,
                   k.data_ptr(), v.data_ptr())
        return k, v

    def tppsd_cache_status(self) -> int:
        bits = c_uint32()
        with torch.cuda.device(self.ws.device):
            _check(lib().tppsd_cache_status(self.handle, _stream(), ctypes.byref(bits)))
        return bits.value
