"""ctypes binding of librouterelay.so (C ABI in include/routerelay.h).

Argument marshalling only: every step of the path runs in the library's HIP
kernels.  Tensors are torch device tensors that supply ``data_ptr()``; the
stream is torch's current stream unless one is given.  Importing this module
loads the library and raises ImportError if it has not been built.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "librouterelay.so")

RR_OK, RR_ERR_INVALID, RR_ERR_OOM, RR_ERR_HIP, RR_ERR_STATE, RR_ERR_UNSUPPORTED = 0, -1, -2, -3, -4, -5
RR_F32, RR_BF16, RR_E4M3 = 0, 1, 2
RR_OPT_SPLIT_RELAY, RR_OPT_ONE_PASS_RELAY = 1, 2

EXPORTED = (
    "rr_ledger_create", "rr_ledger_destroy", "rr_anchor_route", "rr_relay_layer", "rr_full_route",
    "rr_ledger_routes", "rr_ledger_export", "rr_ledger_import", "rr_ledger_relay_stats",
    "rr_ledger_index_bytes", "rr_status_string", "rr_last_error", "rr_profile_start",
    "rr_profile_stop", "rr_unconverged_rows", "rr_set_sweep_cap", "rr_relay_layer_static",
    "rr_pool_chunks", "rr_expand_tokens", "rr_sparse_attention", "rr_cache_append",
    "rr_paged_workspace_bytes", "rr_paged_attention", "rr_prefix_attention", "rr_cache_append_axes", "rr_rotate",
    "rr_cache_fork", "rr_pages_workspace_bytes", "rr_cache_resize", "rr_cache_compact", "rr_verify_workspace_bytes",
    "rr_verify_drafts",
)
KERNEL_KINDS = ("full", "anchor", "reroute", "rescore", "relay", "pool", "expand", "attention", "append",
                "paged", "join", "rotate", "verify", "pages", "copy")


class RRError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{msg} (status {status})")
        self.status = status


_MOST = 2 ** 31 - 1


def _fits(*sizes):
    """Numbers that the library takes in 32 bits, to which ctypes would cut others
    without a word.  (Where only a tensor's sizes can be large, and time counts, a
    call tests them itself: their bits together, as none is below 0.)"""
    for n in sizes:
        if not -_MOST - 1 <= n <= _MOST:
            raise ValueError(f"{n} does not fit 32 bits")


class _Config(ctypes.Structure):
    _fields_ = [
        ("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("n_q", ctypes.c_int32),
        ("n_k", ctypes.c_int32), ("d", ctypes.c_int32), ("k", ctypes.c_int32), ("m", ctypes.c_int32),
        ("r", ctypes.c_int32), ("dtype", ctypes.c_int32), ("causal", ctypes.c_int32),
        ("gamma", ctypes.c_float), ("options", ctypes.c_uint32), ("seed", ctypes.c_uint64),
        ("n_sink", ctypes.c_int32), ("n_recent", ctypes.c_int32), ("min_reuse", ctypes.c_int32),
        ("reserved", ctypes.c_int32), ("gamma_rows", ctypes.c_void_p), ("k_rows", ctypes.c_void_p),
    ]


class _AttnConfig(ctypes.Structure):
    _fields_ = [
        ("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("n_tokens", ctypes.c_int32),
        ("d", ctypes.c_int32), ("chunk", ctypes.c_int32), ("k", ctypes.c_int32), ("causal", ctypes.c_int32),
        ("dtype", ctypes.c_int32), ("scale", ctypes.c_float), ("reserved", ctypes.c_int32),
    ]


class _AppendConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "n_heads", "n_kv_heads", "d", "page", "n_pages", "max_pages", "n_seqs", "n_tokens", "rot", "interleaved", "dtype",
        "cache_dtype")] + [("ldq", ctypes.c_int64), ("ldk", ctypes.c_int64), ("ldv", ctypes.c_int64),
                           ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p)]


class _PagedConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "n_heads", "n_kv_heads", "d", "page", "n_pages", "max_pages", "n_seqs", "n_q", "k", "n_sink", "n_recent",
        "n_prefix", "dtype", "cache_dtype")] + [("scale", ctypes.c_float), ("reserved", ctypes.c_int32),
                                                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p)]


class _Axes(ctypes.Structure):
    _fields_ = [("positions", ctypes.c_void_p), ("axis", ctypes.c_void_p), ("n_axes", ctypes.c_int32),
                ("real", ctypes.c_int32)]


class _RotateConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_heads", "n_tokens", "d", "rot", "interleaved", "inverse", "dtype",
                                              "reserved")] + \
               [(n, ctypes.c_int64) for n in ("x_token", "x_head", "y_token", "y_head")]


class _PagesConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_kv_heads", "d", "page", "n_pages", "cache_dtype", "n_pools", "max_pages",
                                              "n_seqs", "n_new", "reserved")]


class _VerifyConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_seqs", "n_drafts", "vocab", "dtype")] + \
               [(n, ctypes.c_int64) for n in ("p_seq", "p_row", "q_seq", "q_row")]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built: run `python -m paper_2609_07306_amd.build`")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, cfgp = ctypes.c_void_p, ctypes.c_int32, ctypes.POINTER(_Config)
    sig = {
        "rr_ledger_create": (ctypes.c_int, [cfgp, ctypes.POINTER(vp)]),
        "rr_ledger_destroy": (ctypes.c_int, [vp]),
        "rr_anchor_route": (ctypes.c_int, [vp, i32, vp, vp, vp, vp, vp]),
        "rr_relay_layer": (ctypes.c_int, [vp, i32, vp, vp, vp, vp, vp, vp, vp]),
        "rr_full_route": (ctypes.c_int, [cfgp, vp, vp, vp, vp, vp, vp]),
        "rr_ledger_routes": (vp, [vp]),
        "rr_ledger_export": (ctypes.c_int, [vp, vp, vp, vp, vp, vp]),
        "rr_ledger_import": (ctypes.c_int, [vp, i32, vp, vp, vp, vp, vp]),
        "rr_ledger_relay_stats": (ctypes.c_int, [vp, vp, vp, vp, vp]),
        "rr_ledger_index_bytes": (ctypes.c_size_t, [cfgp]),
        "rr_status_string": (ctypes.c_char_p, [ctypes.c_int]),
        "rr_last_error": (ctypes.c_char_p, []),
        "rr_profile_start": (ctypes.c_int, []),
        "rr_profile_stop": (ctypes.c_int, [vp, vp, i32]),
        "rr_unconverged_rows": (ctypes.c_int, [ctypes.POINTER(ctypes.c_uint64)]),
        "rr_set_sweep_cap": (ctypes.c_int, [i32]),
        "rr_relay_layer_static": (ctypes.c_int, [cfgp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]),
        "rr_pool_chunks": (ctypes.c_int, [vp, i32, i32, i32, i32, i32, vp, vp]),
        "rr_expand_tokens": (ctypes.c_int, [vp, ctypes.c_int64, i32, i32, i32, vp, vp]),
        "rr_sparse_attention": (ctypes.c_int, [ctypes.POINTER(_AttnConfig), vp, vp, vp, vp, vp, vp]),
        "rr_cache_append": (ctypes.c_int, [ctypes.POINTER(_AppendConfig)] + [vp] * 11),
        "rr_paged_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(_PagedConfig)]),
        "rr_paged_attention": (ctypes.c_int, [ctypes.POINTER(_PagedConfig)] + [vp] * 9 + [ctypes.c_size_t, vp]),
        "rr_prefix_attention": (ctypes.c_int, [ctypes.POINTER(_PagedConfig)] + [vp] * 9 + [ctypes.c_size_t, vp]),
        "rr_cache_append_axes": (ctypes.c_int, [ctypes.POINTER(_AppendConfig)] + [vp] * 7 + [ctypes.POINTER(_Axes)] + [vp] * 4),
        "rr_rotate": (ctypes.c_int, [ctypes.POINTER(_RotateConfig), vp, vp, ctypes.POINTER(_Axes), vp, vp]),
        "rr_cache_fork": (ctypes.c_int, [i32] * 3 + [vp] * 5),
        "rr_pages_workspace_bytes": (ctypes.c_size_t, [i32]),
        "rr_cache_resize": (ctypes.c_int, [ctypes.POINTER(_PagesConfig)] + [vp] * 7 + [ctypes.c_size_t, vp]),
        "rr_cache_compact": (ctypes.c_int, [ctypes.POINTER(_PagesConfig)] + [vp] * 6 + [ctypes.c_size_t, vp]),
        "rr_verify_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(_VerifyConfig)]),
        "rr_verify_drafts": (ctypes.c_int, [ctypes.POINTER(_VerifyConfig)] + [vp] * 9 + [ctypes.c_size_t, vp]),
    }
    for name, (res, args) in sig.items():
        f = getattr(lib, name)
        f.restype = res
        f.argtypes = args
    return lib


lib = _load()


def _check(status: int):
    if status != RR_OK:
        raise RRError(status, lib.rr_last_error().decode())


_RELAY_OPTIONS = {"auto": 0, "split": RR_OPT_SPLIT_RELAY, "one_pass": RR_OPT_ONE_PASS_RELAY}


@dataclass(frozen=True)
class Config:
    """Shape and rule parameters (rr_config)."""
    n_heads: int
    n_kv_heads: int
    n_q: int
    n_k: int
    d: int
    k: int
    m: int = 0
    r: int = 0
    dtype: str = "f32"  # "f32" | "bf16"
    causal: bool = False
    gamma: float = 0.0
    seed: int = 0
    relay: str = "auto"  # relay schedule: "auto" | "one_pass" | "split" (rr_option)
    n_sink: int = 0      # mandatory sentinels: sink chunks ...
    n_recent: int = 0    # ... and recent chunks
    min_reuse: int = 0   # minimum reuse horizon (layers)
    gamma_rows: object = None  # per-row guard margins: float32 device tensor [rows], or None
    k_rows: object = None      # per-row route widths in [1, k]: int32 device tensor [rows], or None

    @property
    def rows(self) -> int:
        return self.n_heads * self.n_q

    @property
    def sent_width(self) -> int:
        return self.m + self.r + self.n_sink + self.n_recent

    def c(self) -> _Config:
        sizes = (self.n_heads, self.n_kv_heads, self.n_q, self.n_k, self.d, self.k, self.m, self.r, self.n_sink,
                 self.n_recent, self.min_reuse)
        if min(sizes) < 0 or max(sizes) > _MOST:
            _fits(*sizes)
        g = None
        if self.gamma_rows is not None:
            t = self.gamma_rows
            if t.dtype != torch.float32 or tuple(t.shape) != (self.rows,):
                raise ValueError("gamma_rows must be a float32 tensor with one entry per row")
            g = _ptr(t)
        kr = None
        if self.k_rows is not None:
            t = self.k_rows
            if t.dtype != torch.int32 or tuple(t.shape) != (self.rows,):
                raise ValueError("k_rows must be an int32 tensor with one entry per row")
            kr = _ptr(t)
        return _Config(self.n_heads, self.n_kv_heads, self.n_q, self.n_k, self.d, self.k, self.m,
                       self.r, RR_BF16 if self.dtype == "bf16" else RR_F32, int(self.causal),
                       float(self.gamma), _RELAY_OPTIONS[self.relay],
                       int(self.seed) & 0xFFFFFFFFFFFFFFFF, int(self.n_sink), int(self.n_recent),
                       int(self.min_reuse), 0, g, kr)

    @staticmethod
    def of(w) -> "Config":
        """From a synth.Workload."""
        return Config(w.n_heads, w.n_kv_heads, w.n, w.nk, w.d, w.k, w.m, w.r, w.dtype, w.causal,
                      w.gamma, w.seed, n_sink=w.n_sink, n_recent=w.n_recent, min_reuse=w.min_reuse)


def _ptr(t):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("tensor must be on the GPU")
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _inputs(cfg: Config, Q, K):
    want = torch.bfloat16 if cfg.dtype == "bf16" else torch.float32
    if Q.dtype != want or K.dtype != want:
        raise TypeError(f"Qc/Kc must be {want}")
    if tuple(Q.shape) != (cfg.n_heads, cfg.n_q, cfg.d) or tuple(K.shape) != (cfg.n_kv_heads, cfg.n_k, cfg.d):
        raise ValueError(f"shapes {tuple(Q.shape)}, {tuple(K.shape)} do not match the config")
    return _ptr(Q), _ptr(K)


def _out(t, shape, dtype):
    if t is None:
        return None
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype:
        raise ValueError(f"output must be {dtype} of shape {shape}")
    return _ptr(t)


def profile_start():
    """Start bracketing every library kernel launch with HIP events."""
    _check(lib.rr_profile_start())


def profile_stop():
    """Stop profiling; returns {kind: (total_ms, launches)}."""
    ms = (ctypes.c_double * len(KERNEL_KINDS))()
    n = (ctypes.c_int64 * len(KERNEL_KINDS))()
    _check(lib.rr_profile_stop(ms, n, len(KERNEL_KINDS)))
    return {k: (ms[i], n[i]) for i, k in enumerate(KERNEL_KINDS)}


def unconverged_rows() -> int:
    """Rows (on the current device, since load) whose selection stopped at the sweep cap."""
    c = ctypes.c_uint64()
    _check(lib.rr_unconverged_rows(ctypes.byref(c)))
    return int(c.value)


def set_sweep_cap(cap: int):
    """Test hook: collection sweeps allowed per route tile (0: default)."""
    _fits(cap)
    _check(lib.rr_set_sweep_cap(int(cap)))


def index_bytes(cfg: Config) -> int:
    return int(lib.rr_ledger_index_bytes(ctypes.byref(cfg.c())))


def full_route(cfg: Config, Q, K, routes, scores=None, pairs=None, stream=None):
    """rr_full_route: every row's top-k (Eq. (1)-(2)) into ``routes`` [rows, k] int32."""
    q, k = _inputs(cfg, Q, K)
    _check(lib.rr_full_route(ctypes.byref(cfg.c()), q, k, _out(routes, (cfg.rows, cfg.k), torch.int32),
                             _out(scores, (cfg.rows, cfg.k), torch.float32),
                             _out(pairs, (1,), torch.int64), _stream(stream)))


def relay_static(cfg: Config, layer: int, Q, K, ledger, routes=None, mask=None, pairs=None, n_rerouted=None,
                 stream=None):
    """rr_relay_layer_static: a relay layer on a caller-owned ledger (a dict of
    int32 device tensors as Ledger.export returns), updated in place; the
    library allocates nothing."""
    _fits(layer)
    q, k = _inputs(cfg, Q, K)
    c = cfg
    _check(lib.rr_relay_layer_static(
        ctypes.byref(cfg.c()), layer, q, k, _out(ledger["routes"], (c.rows, c.k), torch.int32),
        _out(ledger["sent"], (c.rows, c.sent_width), torch.int32) if c.sent_width else None,
        _out(ledger["build"], (c.rows,), torch.int32), _out(ledger["age"], (c.rows,), torch.int32),
        _out(routes, (c.rows, c.k), torch.int32), _out(mask, (c.rows,), torch.uint8),
        _out(pairs, (1,), torch.int64), _out(n_rerouted, (1,), torch.int32), _stream(stream)))


class Ledger:
    """rr_ledger: the per-row route ledger on the current device."""

    def __init__(self, cfg: Config):
        self.cfg = cfg
        h = ctypes.c_void_p()
        _check(lib.rr_ledger_create(ctypes.byref(cfg.c()), ctypes.byref(h)))
        self._h = h

    def close(self):
        if getattr(self, "_h", None) and self._h.value:
            lib.rr_ledger_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    @property
    def handle(self):
        return self._h

    def anchor(self, layer: int, Q, K, routes=None, pairs=None, stream=None):
        _fits(layer)
        q, k = _inputs(self.cfg, Q, K)
        c = self.cfg
        _check(lib.rr_anchor_route(self._h, layer, q, k, _out(routes, (c.rows, c.k), torch.int32),
                                   _out(pairs, (1,), torch.int64), _stream(stream)))

    def relay(self, layer: int, Q, K, routes=None, mask=None, pairs=None, n_rerouted=None, stream=None):
        _fits(layer)
        q, k = _inputs(self.cfg, Q, K)
        c = self.cfg
        _check(lib.rr_relay_layer(self._h, layer, q, k, _out(routes, (c.rows, c.k), torch.int32),
                                  _out(mask, (c.rows,), torch.uint8), _out(pairs, (1,), torch.int64),
                                  _out(n_rerouted, (1,), torch.int32), _stream(stream)))

    def routes_ptr(self) -> int:
        return int(lib.rr_ledger_routes(self._h) or 0)

    def export(self, stream=None):
        """Copies of the ledger state: dict of int32 device tensors."""
        c = self.cfg
        dev = torch.device("cuda", torch.cuda.current_device())
        out = {
            "routes": torch.empty((c.rows, c.k), dtype=torch.int32, device=dev),
            "sent": torch.empty((c.rows, c.sent_width), dtype=torch.int32, device=dev),
            "build": torch.empty((c.rows,), dtype=torch.int32, device=dev),
            "age": torch.empty((c.rows,), dtype=torch.int32, device=dev),
        }
        _check(lib.rr_ledger_export(self._h, _ptr(out["routes"]), _ptr(out["sent"]) if c.sent_width else None,
                                    _ptr(out["build"]), _ptr(out["age"]), _stream(stream)))
        return out

    def import_(self, layer: int, routes, sent, build, age, stream=None):
        _fits(layer)
        c = self.cfg
        _check(lib.rr_ledger_import(self._h, layer, _out(routes, (c.rows, c.k), torch.int32),
                                    _out(sent, (c.rows, c.sent_width), torch.int32) if c.sent_width else None,
                                    _out(build, (c.rows,), torch.int32), _out(age, (c.rows,), torch.int32),
                                    _stream(stream)))

    def relay_stats(self, stream=None):
        c = self.cfg
        dev = torch.device("cuda", torch.cuda.current_device())
        alpha = torch.empty(c.rows, dtype=torch.float32, device=dev)
        beta = torch.empty(c.rows, dtype=torch.float32, device=dev)
        ids = torch.empty(c.rows, dtype=torch.int32, device=dev)
        _check(lib.rr_ledger_relay_stats(self._h, _ptr(alpha), _ptr(beta), _ptr(ids), _stream(stream)))
        return alpha, beta, ids


def to_device(x_dev, dtype: str, device="cuda"):
    """numpy array from synth (binary32 values or bf16 bits) -> torch device tensor."""
    import numpy as np
    if dtype == "bf16":
        t = torch.from_numpy(np.ascontiguousarray(x_dev).view(np.int16)).view(torch.bfloat16)
    else:
        t = torch.from_numpy(np.ascontiguousarray(x_dev, dtype=np.float32))
    return t.to(device)


# ------------------------------------------------- either side of the path

def n_chunks(n_tokens: int, chunk: int) -> int:
    return -(-n_tokens // chunk)


def pool_chunks(X, chunk: int, out=None, stream=None):
    """rr_pool_chunks: X [H, n_tokens, d] (float32 or bfloat16 device tensor)
    -> [H, n_chunks, d] chunk means of the same dtype."""
    if X.dim() != 3 or X.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("X must be a [H, n_tokens, d] float32 or bfloat16 tensor")
    H, n, d = X.shape
    _fits(H, n, d, chunk)
    shape = (H, n_chunks(n, chunk), d)
    if out is None:
        out = torch.empty(shape, dtype=X.dtype, device=X.device)
    dt = RR_BF16 if X.dtype == torch.bfloat16 else RR_F32
    _check(lib.rr_pool_chunks(_ptr(X), H, n, d, chunk, dt, _out(out, shape, X.dtype), _stream(stream)))
    return out


def expand_tokens(routes, chunk: int, n_tokens: int, out=None, stream=None):
    """rr_expand_tokens: routes [rows, k] int32 -> token ids [rows, k*chunk]."""
    if routes.dim() != 2 or routes.dtype != torch.int32:
        raise TypeError("routes must be a [rows, k] int32 tensor")
    rows, k = routes.shape
    _fits(k, chunk, n_tokens)
    shape = (rows, k * chunk)
    if out is None:
        out = torch.empty(shape, dtype=torch.int32, device=routes.device)
    _check(lib.rr_expand_tokens(_ptr(routes), rows, k, chunk, n_tokens, _out(out, shape, torch.int32),
                                _stream(stream)))
    return out


def sparse_attention(Q, K, V, routes, chunk: int, causal: bool, scale: float = 0.0, out=None, stream=None):
    """rr_sparse_attention: Q [H, n, d], K and V [H_kv, n, d] bfloat16,
    routes [H * n_chunks, k] int32 -> O [H, n, d] bfloat16."""
    for t in (Q, K, V):
        if t.dim() != 3 or t.dtype != torch.bfloat16:
            raise TypeError("Q, K and V must be 3-d bfloat16 tensors")
    H, n, d = Q.shape
    Hkv = K.shape[0]
    if tuple(K.shape) != (Hkv, n, d) or tuple(V.shape) != (Hkv, n, d):
        raise ValueError("K and V must be [H_kv, n_tokens, d]")
    _fits(H, Hkv, n, d, chunk, *routes.shape[1:])
    nc = n_chunks(n, chunk)
    if routes.dim() != 2 or routes.dtype != torch.int32 or routes.shape[0] != H * nc:
        raise ValueError("routes must be [H * n_chunks, k] int32")
    if out is None:
        out = torch.empty_like(Q)
    cfg = _AttnConfig(H, Hkv, n, d, chunk, routes.shape[1], int(causal), RR_BF16, float(scale), 0)
    _check(lib.rr_sparse_attention(ctypes.byref(cfg), _ptr(Q), _ptr(K), _ptr(V), _ptr(routes),
                                   _out(out, (H, n, d), torch.bfloat16), _stream(stream)))
    return out



# -------------------------------------------------------- the paged cache

_E4M3 = torch.float8_e4m3fn
# (the address alone: a torch.cuda.Stream object costs as much as a launch's checks)
_current_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch.cuda.current_device
_append, _paged, _prefix = lib.rr_cache_append, lib.rr_paged_attention, lib.rr_prefix_attention
_append_axes, _rotate, _verify = lib.rr_cache_append_axes, lib.rr_rotate, lib.rr_verify_drafts
_fork, _resize, _compact = lib.rr_cache_fork, lib.rr_cache_resize, lib.rr_cache_compact
_DTYPES = {torch.float32: RR_F32, torch.bfloat16: RR_BF16, _E4M3: RR_E4M3}


def _device_of(tensors):
    """The device index of the tensors of a call (None among them: not given);
    they have to share one."""
    dev = tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"tensors on {tensors[0].device} and {t.device}: a call takes one device's")
    if dev < 0:
        raise ValueError("tensor must be on the GPU")
    return dev


def _launch(dev, stream, call, *args):
    """call(*args, stream) with device `dev` current, on the given stream or the
    device's current one."""
    if stream is None:
        s = _current_stream(dev)
    elif stream.device_index != dev:
        raise ValueError(f"the stream is of {stream.device}, the tensors are on cuda:{dev}")
    else:
        s = stream.cuda_stream
    if _current_device() == dev:
        status = call(*args, s)
    else:
        with torch.cuda.device(dev):
            status = call(*args, s)
    if status:
        _check(status)


def _empty(shape, dtype, like, stream, zeros=False):
    """Memory for a call on the given stream (None: the current one), of that
    stream's own: freed, only what the stream does later can take it."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return _empty(shape, dtype, like, None, zeros)
    return (like.new_zeros if zeros else like.new_empty)(shape, dtype=dtype)


def _of(name, t, shape, dtype):
    if t.dtype != dtype or t.shape != shape:
        raise ValueError(f"{name} must be {dtype} of shape {list(shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _lists(page_table, lengths):
    """The addresses of page_table [B, max_pages] and lengths [B], and their sizes."""
    shape = page_table.shape
    if len(shape) != 2:
        raise ValueError("page_table must be [B, max_pages]")
    B, most = shape
    if page_table.dtype != torch.int32 or lengths.dtype != torch.int32 or lengths.shape != (B,):
        raise ValueError(f"page_table [B, max_pages] and lengths [B] must be int32: got {page_table.dtype} of shape "
                         f"{list(page_table.shape)}, {lengths.dtype} of shape {list(lengths.shape)}")
    if not (page_table.is_contiguous() and lengths.is_contiguous()):
        raise ValueError("page_table and lengths must be contiguous")
    return page_table.data_ptr(), lengths.data_ptr(), B, most


def _cache_of(K_cache, V_cache, dtype, k_scale, v_scale):
    """The pools' shape, type and addresses, and the scales' addresses."""
    kind, shape = K_cache.dtype, K_cache.shape
    if len(shape) != 4 or kind not in _DTYPES or V_cache.dtype != kind:
        raise TypeError("K_cache and V_cache must be [n_pages, H_kv, page, d] tensors of one type of "
                        "float32, bfloat16 and float8_e4m3fn")
    if V_cache.shape != shape:
        raise ValueError("K_cache and V_cache must have one shape")
    if kind != dtype and not (dtype == torch.bfloat16 and kind == _E4M3):
        raise TypeError("the cache must have the queries' type, or float8_e4m3fn with bfloat16")
    if (k_scale is not None) != (kind == _E4M3) or (v_scale is not None) != (kind == _E4M3):
        raise ValueError("k_scale and v_scale are given for float8_e4m3fn caches, and for them only")
    if not (K_cache.is_contiguous() and V_cache.is_contiguous()):
        raise ValueError("K_cache and V_cache must be contiguous")
    ks = vs = None
    if k_scale is not None:
        heads = (shape[1],)
        ks, vs = _of("k_scale", k_scale, heads, torch.float32), _of("v_scale", v_scale, heads, torch.float32)
    return shape, _DTYPES[kind], K_cache.data_ptr(), V_cache.data_ptr(), ks, vs


def _rows_of(name, t, shape, dtype):
    """Elements between one token's rows and the next one's: the rows of a token
    lie together, tokens may lie apart (views of a fused projection)."""
    if t.shape != shape or t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype} of shape {list(shape)}")
    n, heads, d = shape
    token, head, one = t.stride()
    if (d > 1 and one != 1) or (heads > 1 and head != d):
        raise ValueError(f"{name}: the rows of a token must be contiguous")
    return token if n > 1 else heads * d


def _axes_of(positions, axis, rot, n):
    """rr_axes of positions [n_axes, n] (or [n]) int32 or float32 and axis [rot / 2] int32."""
    kind = positions.dtype
    if kind != torch.int32 and kind != torch.float32:
        raise TypeError("positions must be int32 or float32")
    shape = positions.shape
    if not shape or shape[-1] != n or len(shape) > 2 or (len(shape) == 2 and not shape[0]):
        raise ValueError(f"positions must be [n_axes, {n}]: got {list(shape)}")
    if not positions.is_contiguous():
        raise ValueError("positions must be contiguous")
    if shape[0] > _MOST:
        _fits(shape[0])
    return _Axes(positions.data_ptr(), None if axis is None else _of("axis", axis, (rot // 2,), torch.int32),
                 shape[0] if len(shape) == 2 else 1, 1 if kind == torch.float32 else 0)


def cache_append(K, V, K_cache, V_cache, page_table, lengths, seq_start=None, freqs=None, interleaved=False, Q=None,
                 Q_out=None, k_scale=None, v_scale=None, stream=None, positions=None, axis=None):
    """rr_cache_append: new tokens' keys and values K, V [n_tokens, H_kv, d]
    into the pages of their sequences (K_cache, V_cache [n_pages, H_kv, page,
    d], page_table [B, max_pages] and lengths [B] int32, the new tokens counted
    in; seq_start [B + 1] int32, None: n_tokens / B each).  With freqs [rot / 2]
    float64 the first rot features of keys are rotated by position, and of
    queries Q [n_tokens, H, d] (returned, in Q_out if given).  K, V and Q may
    be views whose tokens lie apart.  positions [n_axes, n_tokens] int32 or
    float32: rotated by these, frequency j by those of axis[j] (axis [rot / 2]
    int32, None: the first), not by place in the sequence (rr_cache_append_axes)."""
    kind, shape = K.dtype, K.shape
    if len(shape) != 3 or kind not in (torch.float32, torch.bfloat16):
        raise TypeError("K must be a [n_tokens, H_kv, d] float32 or bfloat16 tensor")
    (n_pages, Hkv, page, d), cache, kc, vc, ks, vs = _cache_of(K_cache, V_cache, kind, k_scale, v_scale)
    if positions is None:
        dev = _device_of((K, V, K_cache, V_cache, page_table, lengths, seq_start, freqs, Q, Q_out, k_scale, v_scale))
    else:
        dev = _device_of((K, V, K_cache, V_cache, page_table, lengths, seq_start, freqs, Q, Q_out, k_scale, v_scale, positions,
                          axis))
    n = shape[0]
    rows = (n, Hkv, d)
    ldk, ldv = _rows_of("K", K, rows, kind), _rows_of("V", V, rows, kind)
    table, lens, B, most = _lists(page_table, lengths)
    H = ldq = rot = 0
    f = q = out = start = None
    if freqs is not None:
        half = freqs.numel()
        rot = 2 * half
        f = _of("freqs", freqs, (half,), torch.float64)
    if seq_start is not None:
        start = _of("seq_start", seq_start, (B + 1,), torch.int32)
    if Q is not None:
        heads = Q.shape
        if len(heads) != 3:
            raise TypeError("Q must be a [n_tokens, H, d] tensor")
        H = heads[1]
        rows = (n, H, d)
        ldq = _rows_of("Q", Q, rows, kind)
        if Q_out is None:
            Q_out = _empty(rows, kind, Q, stream)
        q, out = Q.data_ptr(), _of("Q_out", Q_out, rows, kind)
    elif Q_out is not None:
        raise ValueError("Q_out without Q")
    if n | n_pages | Hkv | page | d | B | most | H | rot > _MOST:
        _fits(n, n_pages, Hkv, page, d, B, most, H, rot)
    cfg = _AppendConfig(H, Hkv, d, page, n_pages, most, B, n, rot, 1 if interleaved else 0, _DTYPES[kind], cache, ldq, ldk,
                        ldv, ks, vs)
    if positions is None:
        if axis is not None:
            raise ValueError("axis without positions")
        _launch(dev, stream, _append, cfg, K.data_ptr(), V.data_ptr(), q, start, lens, table, f if rot else None, kc, vc, out)
        return Q_out
    if freqs is None:
        raise ValueError("positions without freqs")
    axes = _axes_of(positions, axis, rot, n)
    _launch(dev, stream, _append_axes, cfg, K.data_ptr(), V.data_ptr(), q, start, lens, table, f if rot else None, axes, kc, vc,
            out)
    return Q_out


def _strides(name, t, tokens):
    """Elements between the rows of tokens and of heads of t, tokens in dimension `tokens`."""
    s = t.stride()
    if t.shape[2] > 1 and s[2] != 1:
        raise ValueError(f"{name}: rows must be contiguous")
    return s[tokens], s[1 - tokens]


def rotate(X, positions, freqs, axis=None, tokens=0, interleaved=False, inverse=False, out=None, stream=None):
    """rr_rotate: the first rot features of every row of X rotated by position, as
    cache_append does: X [n_tokens, H, d] (tokens=0) or [H, n_tokens, d]
    (tokens=1) float32 or bfloat16, rows contiguous, positions [n_axes, n_tokens]
    int32 or float32, freqs [rot / 2] float64, axis as in cache_append.
    inverse=True: back (the gradient too).  out: X itself or another tensor."""
    kind, shape = X.dtype, X.shape
    if len(shape) != 3 or kind not in (torch.float32, torch.bfloat16):
        raise TypeError("X must be a 3-d float32 or bfloat16 tensor")
    if tokens not in (0, 1):
        raise ValueError("tokens must be 0 or 1")
    dev = _device_of((X, positions, freqs, axis, out))
    n, half = shape[tokens], freqs.numel()
    rot = 2 * half
    f = _of("freqs", freqs, (half,), torch.float64)
    axes = _axes_of(positions, axis, rot, n)
    if out is None:
        out = _empty(shape, kind, X, stream)
    elif out.shape != shape or out.dtype != kind:
        raise ValueError(f"out must be {kind} of shape {list(shape)}")
    H, d = shape[1 - tokens], shape[2]
    if n | H | d | rot > _MOST:
        _fits(n, H, d, rot)
    cfg = _RotateConfig(H, n, d, rot, 1 if interleaved else 0, 1 if inverse else 0, _DTYPES[kind], 0,
                        *_strides("X", X, tokens), *_strides("out", out, tokens))
    _launch(dev, stream, _rotate, cfg, X.data_ptr(), f, axes, out.data_ptr())
    return out


def _paged_config(Q, K_cache, V_cache, page_table, routes, n_sink, n_recent, n_prefix, scale, k_scale, v_scale, lengths):
    """The call's configuration, and the addresses of the pools, the page table and
    the lengths."""
    if Q.dim() != 4 or Q.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("Q must be a [B, n_q, H, d] float32 or bfloat16 tensor")
    (n_pages, Hkv, page, d), cache, kc, vc, ks, vs = _cache_of(K_cache, V_cache, Q.dtype, k_scale, v_scale)
    B, nq, H, dq = Q.shape
    if dq != d:
        raise ValueError(f"Q has rows of {dq} features, the cache of {d}")
    table, lens, rows, most = _lists(page_table, lengths)
    if rows != B:
        raise ValueError("page_table must be [B, max_pages]")
    k = 0
    if routes is not None:
        if routes.dim() != 2 or routes.shape[0] != B * H * nq:
            raise ValueError("routes must be [B * H * n_q, k]")
        k = routes.shape[1]
        if k == n_sink == n_recent == 0:
            k = 1  # (a slot that names no page, _some_routes: the library takes k = 0 alone for no routes)
    if not 0 <= n_sink | n_recent | n_prefix <= _MOST:
        _fits(n_sink, n_recent, n_prefix)
    if n_pages | Hkv | page | d | B | most | nq | H | k > _MOST:
        _fits(n_pages, Hkv, page, d, B, most, nq, H, k)
    cfg = _PagedConfig(H, Hkv, d, page, n_pages, most, B, nq, k, n_sink, n_recent, n_prefix, _DTYPES[Q.dtype], cache, scale, 0,
                       ks, vs)
    return cfg, kc, vc, table, lens


def _some_routes(routes, n_sink, n_recent, stream):
    """The routes that the library takes: none where there are no slots but other
    pages, and a slot without a page where a row has nothing to see."""
    if routes.shape[1]:
        return routes
    if n_sink or n_recent:
        return None
    with torch.cuda.stream(stream):
        return torch.full((routes.shape[0], 1), -1, dtype=torch.int32, device=routes.device)


def _workspace_bytes(cfg):
    n = lib.rr_paged_workspace_bytes(cfg)
    if n == 0:
        # the status is that of a call, which refuses the config before it looks
        # at a pointer (and would refuse these, were it not for the config)
        call, third = (_prefix, 1) if cfg.n_prefix else (_paged, 1 if cfg.k else None)
        _check(call(cfg, None, None, None, None, None, third, None, None, None, 0, None))
    return n


def paged_workspace(Q, K_cache, page_table, routes=None, n_sink=0, n_recent=0, n_prefix=0):
    """A workspace (uint8 device tensor, zeros) for paged_attention and
    prefix_attention calls of these shapes, one after the other in any order
    (the largest of several shapes' serves them all).  Calls that may run at
    the same time, captured graphs that are replayed side by side among them,
    need one each."""
    scale, lengths = None, torch.empty(len(page_table), dtype=torch.int32, device=page_table.device)
    if K_cache.dtype == _E4M3 and K_cache.dim() == 4:  # (values play no part)
        scale = torch.empty(K_cache.shape[1], dtype=torch.float32, device=K_cache.device)
    cfg = _paged_config(Q, K_cache, K_cache, page_table, routes, n_sink, n_recent, n_prefix, 0.0, scale, scale, lengths)[0]
    return torch.zeros(_workspace_bytes(cfg), dtype=torch.uint8, device=Q.device)


def _paged_call(call, config, dev, Q, third, out, lse, workspace, stream):
    cfg, kc, vc, table, lens = config
    if out is None:
        out = _empty(Q.shape, Q.dtype, Q, stream)
    elif out.shape != Q.shape or out.dtype != Q.dtype:
        raise ValueError(f"out must be {Q.dtype} of shape {list(Q.shape)}")
    if workspace is None:
        workspace = _empty((_workspace_bytes(cfg),), torch.uint8, Q, stream, zeros=True)
    elif workspace.dtype != torch.uint8 or workspace.dim() != 1:
        raise ValueError("workspace must be a one-dimensional uint8 tensor")
    if not (Q.is_contiguous() and out.is_contiguous() and workspace.is_contiguous()):
        raise ValueError("Q, out and workspace must be contiguous")
    _launch(dev, stream, call, cfg, Q.data_ptr(), kc, vc, table, lens, third, out.data_ptr(),
            None if lse is None else _of("lse", lse, Q.shape[:3], torch.float32), workspace.data_ptr(), workspace.numel())
    return out


def paged_attention(Q, K_cache, V_cache, page_table, lengths, routes=None, n_sink=0, n_recent=0, scale=0.0, k_scale=None,
                    v_scale=None, out=None, lse=None, workspace=None, stream=None):
    """rr_paged_attention: the newest n_q tokens' queries Q [B, n_q, H, d] over
    their sequences' caches (as in cache_append) -> O [B, n_q, H, d].  routes
    [B * H * n_q, k] int32 page indices: each query over those pages, its first
    n_sink and its last n_recent ones (k = 0: over these alone, zeros where there
    are none; as without routes where n_sink or n_recent is set).  lse: optional
    float32 output [B, n_q, H].  workspace: paged_workspace(...), or None for one
    of this call's own."""
    config = _paged_config(Q, K_cache, V_cache, page_table, routes, n_sink, n_recent, 0, scale, k_scale, v_scale, lengths)
    dev = _device_of((Q, K_cache, V_cache, page_table, lengths, routes, k_scale, v_scale, out, lse, workspace))
    third = None
    if routes is not None:
        _of("routes", routes, routes.shape, torch.int32)
        routes = _some_routes(routes, n_sink, n_recent, stream)  # (held to the end of the call)
        third = None if routes is None else routes.data_ptr()
    return _paged_call(_paged, config, dev, Q, third, out, lse, workspace, stream)


def prefix_attention(Q, K_cache, V_cache, page_table, lengths, prefix_pages, n_prefix, scale=0.0, k_scale=None,
                     v_scale=None, out=None, lse=None, workspace=None, stream=None):
    """rr_prefix_attention: paged_attention (without routes) for sequences that
    begin with the same n_prefix tokens, which are read for many of them at once from
    prefix_pages [ceil(n_prefix / page)] int32."""
    config = _paged_config(Q, K_cache, V_cache, page_table, None, 0, 0, n_prefix, scale, k_scale, v_scale, lengths)
    dev = _device_of((Q, K_cache, V_cache, page_table, lengths, prefix_pages, k_scale, v_scale, out, lse, workspace))
    third = _of("prefix_pages", prefix_pages, (n_chunks(n_prefix, max(K_cache.shape[2], 1)),), torch.int32)
    return _paged_call(_prefix, config, dev, Q, third, out, lse, workspace, stream)


# ------------------------------------------- which pages sequences hold

class Pools:
    """The pools of all layers that one page table serves, for cache_resize and
    cache_compact: K_caches and V_caches, tensors or lists of them (one a layer)
    of one shape [n_pages, H_kv, page, d] and type."""

    def __init__(self, K_caches, V_caches):
        one = isinstance(K_caches, torch.Tensor)
        self.tensors = [K_caches, V_caches] if one else [*K_caches, *V_caches]
        if not self.tensors or not one and len(K_caches) != len(V_caches):
            raise ValueError("K_caches and V_caches must be as many")
        first = self.tensors[0]
        self.shape, self.dtype = first.shape, first.dtype
        for t in self.tensors:
            if t.dim() != 4 or t.dtype not in _DTYPES:
                raise TypeError("caches must be [n_pages, H_kv, page, d] tensors of float32, bfloat16 or float8_e4m3fn")
            if t.shape != self.shape or t.dtype != self.dtype:
                raise ValueError("caches must have one shape and one type")
            if not t.is_contiguous():
                raise ValueError("caches must be contiguous")
        _fits(len(self.tensors), *self.shape)
        self.dev = _device_of(self.tensors)
        self._addresses = (ctypes.c_void_p * len(self.tensors))(*(t.data_ptr() for t in self.tensors))

    def _config(self, max_pages, n_seqs, n_new=0):
        n_pages, Hkv, page, d = self.shape
        return _PagesConfig(Hkv, d, page, n_pages, _DTYPES[self.dtype], len(self.tensors), max_pages, n_seqs, n_new, 0)


def pages_workspace(pools):
    """A workspace (uint8 device tensor, zeros) for cache_resize and cache_compact
    calls on these pools, one after the other.  Calls that may run at the same time,
    captured graphs that are replayed side by side among them, need one each."""
    n = lib.rr_pages_workspace_bytes(pools.shape[0])
    if n == 0:
        _check(RR_ERR_INVALID)
    return torch.zeros(n, dtype=torch.uint8, device=pools.tensors[0].device)


def _on(stream, make):
    """make() with the given stream current (None: as it is)."""
    if stream is None:
        return make()
    with torch.cuda.stream(stream):
        return make()


def _workspace(workspace):
    """A workspace's address and bytes."""
    if workspace.dtype != torch.uint8 or workspace.dim() != 1 or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous one-dimensional uint8 tensor")
    return workspace.data_ptr(), workspace.numel()


def _refs(refs, n_pages):
    return _of("refs", refs, (n_pages,), torch.int32)


def cache_fork(page_table, lengths, refs, parent, stream=None):
    """rr_cache_fork: row b of page_table [B, max_pages] and lengths[b] become
    what row parent[b] was (parent [B] int32; b itself: as it is; outside [0, B):
    empty), and refs [n_pages] counts who holds each page.  In place."""
    dev = _device_of((page_table, lengths, refs, parent))
    table, lens, B, most = _lists(page_table, lengths)
    if refs.dim() != 1:
        raise ValueError("refs must be [n_pages]")
    n_pages = refs.shape[0]
    if n_pages | B | most > _MOST:
        _fits(n_pages, B, most)
    _launch(dev, stream, _fork, B, most, n_pages, _of("parent", parent, (B,), torch.int32), table, lens, _refs(refs, n_pages))


def cache_resize(pools, page_table, lengths, refs, new_tokens, missing=None, workspace=None, stream=None):
    """rr_cache_resize: page_table [B, max_pages] follows lengths [B], new tokens
    counted in: pages past the end are freed, the entries of the new_tokens (an
    int, or [B] int32) newest get pages, copies of those that others hold too.
    refs [n_pages] counts who holds each page.  In place; returns missing [B]
    int32, the entries for which no page was free.  workspace:
    pages_workspace(pools), or None for one of this call's own."""
    many = isinstance(new_tokens, torch.Tensor)
    dev = _device_of((pools.tensors[0], page_table, lengths, refs, new_tokens if many else None, missing, workspace))
    table, lens, B, most = _lists(page_table, lengths)
    new = None
    if many:
        new = _of("new_tokens", new_tokens, (B,), torch.int32)
        _fits(B, most)
    elif not 0 <= new_tokens <= _MOST or B | most > _MOST:
        _fits(new_tokens, B, most)
    r = _refs(refs, pools.shape[0])
    if missing is None:
        missing = _empty((B,), torch.int32, page_table, stream)
    out = _of("missing", missing, (B,), torch.int32)
    if workspace is None:
        workspace = _on(stream, lambda: pages_workspace(pools))
    _launch(dev, stream, _resize, pools._config(most, B, 0 if many else new_tokens), pools._addresses, new, lens, table, r, out,
            *_workspace(workspace))
    return missing


def cache_compact(pools, page_table, refs, new_ids=None, n_used=None, workspace=None, stream=None):
    """rr_cache_compact: the n used pages (refs not 0) become pages 0 .. n - 1 of
    all pools, page_table [B, max_pages] and refs [n_pages] follow, in place.
    Returns (new_ids [n_pages] int32: where each page's tokens are now, -1 for a
    free one; n_used [1] int32: n).  workspace: as in cache_resize."""
    dev = _device_of((pools.tensors[0], page_table, refs, new_ids, n_used, workspace))
    if page_table.dim() != 2:
        raise ValueError("page_table must be [B, max_pages]")
    B, most = page_table.shape
    if B | most > _MOST:
        _fits(B, most)
    table = _of("page_table", page_table, (B, most), torch.int32)
    n_pages = pools.shape[0]
    r = _refs(refs, n_pages)
    if new_ids is None:
        new_ids = _empty((n_pages,), torch.int32, page_table, stream)
    if n_used is None:
        n_used = _empty((1,), torch.int32, page_table, stream)
    ids, used = _of("new_ids", new_ids, (n_pages,), torch.int32), _of("n_used", n_used, (1,), torch.int32)
    if workspace is None:
        workspace = _on(stream, lambda: pages_workspace(pools))
    _launch(dev, stream, _compact, pools._config(most, B), pools._addresses, table, r, ids, used, *_workspace(workspace))
    return new_ids, n_used


# --------------------------------------------------------- drafted tokens

def _verify_config(P, n_drafts, Q=None):
    """The configuration of P [B, n_drafts + 1, V] and Q [B, n_drafts, V], whose rows
    are contiguous but may lie apart (views of padded ones)."""
    kind, shape = P.dtype, P.shape
    if len(shape) != 3 or kind not in (torch.float32, torch.bfloat16):
        raise TypeError("P must be a [B, n_drafts + 1, V] float32 or bfloat16 tensor")
    B, rows, V = shape
    if rows != n_drafts + 1:
        raise ValueError(f"P has {rows} rows a sequence, one more than the {n_drafts} drafts is wanted")
    p_seq, p_row, one = P.stride()
    q_seq = q_row = 0
    if Q is not None:
        if Q.dtype != kind or Q.shape != (B, n_drafts, V):
            raise ValueError(f"draft_probs must be {kind} of shape {[B, n_drafts, V]}")
        q_seq, q_row, q_one = Q.stride()
        if q_one != 1 and V > 1:
            raise ValueError("draft_probs: rows must be contiguous")
    if one != 1 and V > 1:
        raise ValueError("P: rows must be contiguous")
    if B | n_drafts | V > _MOST:
        _fits(B, n_drafts, V)
    return _VerifyConfig(B, n_drafts, V, _DTYPES[kind], p_seq, p_row, q_seq, q_row)


def verify_workspace(P):
    """A workspace (uint8 device tensor, zeros) for verify_drafts calls of P's
    shape, one after the other (the largest of several shapes' serves them all).
    Calls that may run at the same time, captured graphs that are replayed side by
    side among them, need one each."""
    n = lib.rr_verify_workspace_bytes(_verify_config(P, P.shape[1] - 1))
    if n == 0:
        status = _verify(_verify_config(P, P.shape[1] - 1), None, None, None, None, None, None, None, None, None, 0, None)
        _check(status)
    return torch.zeros(n, dtype=torch.uint8, device=P.device)


def verify_drafts(P, drafts, uniforms, draft_probs=None, n_drafts=None, lengths=None, accepted=None, tokens=None,
                  workspace=None, stream=None):
    """rr_verify_drafts: drafts [B, n] int32 against the target's probabilities P
    [B, n + 1, V] (float32 or bfloat16) and those that they were drawn with,
    draft_probs [B, n, V] of the same type (None: not drawn), by uniforms [B, n +
    1] float32; n_drafts [B] int32: how many count.  lengths [B] int32 loses the
    drafts that were not taken, in place.  Returns (accepted [B], tokens [B, n +
    1]) int32: how many were taken; they, the token drawn after them, then -1.
    P and draft_probs may be views whose rows lie apart.  workspace:
    verify_workspace(P), or None for one of this call's own."""
    shape = drafts.shape
    if len(shape) != 2:
        raise ValueError("drafts must be [B, n_drafts]")
    B, n = shape
    dev = _device_of((P, drafts, uniforms, draft_probs, n_drafts, lengths, accepted, tokens, workspace))
    cfg = _verify_config(P, n, draft_probs)
    i32 = torch.int32
    d, u = _of("drafts", drafts, (cfg.n_seqs, n), i32), _of("uniforms", uniforms, (B, n + 1), torch.float32)
    count = None if n_drafts is None else _of("n_drafts", n_drafts, (B,), i32)
    lens = None if lengths is None else _of("lengths", lengths, (B,), i32)
    if accepted is None:
        accepted = _empty((B,), i32, drafts, stream)
        took = accepted.data_ptr()
    else:
        took = _of("accepted", accepted, (B,), i32)
    if tokens is None:
        tokens = _empty((B, n + 1), i32, drafts, stream)
        out = tokens.data_ptr()
    else:
        out = _of("tokens", tokens, (B, n + 1), i32)
    if workspace is None:
        workspace = _on(stream, lambda: verify_workspace(P))
    _launch(dev, stream, _verify, cfg, P.data_ptr(), None if draft_probs is None else draft_probs.data_ptr(), d, count, u, lens,
            took, out, *_workspace(workspace))
    return accepted, tokens
