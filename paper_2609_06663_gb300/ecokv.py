"""ctypes binding of libecokv.so: the C ABI of include/ecokv.h and
include/ecokv_decode.h under the same names, plus small helpers that allocate
outputs with torch.  Argument marshalling only: every step of the eviction pass
and of the decode step runs in the library's CUDA kernels, and there is no
fallback.  Importing this module does not load the
library; the first call does, and raises if it is missing.
"""
from __future__ import annotations

import contextlib
import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libecokv.so")

ECOKV_F32, ECOKV_BF16 = 0, 1
ECOKV_FLAG_SC_MIXKV_SIGN = 0x1
ECOKV_FLAG_LAMBDA_OVERRIDE = 0x2
ECOKV_FLAG_VNORM_IMP = 0x4
ECOKV_FLAG_CENTROID_NONWIN = 0x8
ECOKV_FLAG_WINSOR_1 = 0x10
ECOKV_FLAG_WINSOR_5 = 0x20
ECOKV_FLAG_MAD = 0x40
ECOKV_FLAG_FORCE_SIMT = 0x100
ECOKV_FLAG_TEST_STALL = 0x80000000
ECOKV_NOALLOC_SCRATCH_BYTES = 16 << 20   # fixed scratch of ecokv_evict_noalloc, per device
ECOKV_OK, ECOKV_ERR_INVALID_ARG, ECOKV_ERR_UNSUPPORTED, ECOKV_ERR_WORKSPACE = 0, 1, 2, 3
ECOKV_ERR_CUDA, ECOKV_ERR_TIMEOUT, ECOKV_ERR_DEVICE_INDEX = 4, 5, 6

STATUS = {0: "ECOKV_OK", 1: "ECOKV_ERR_INVALID_ARG", 2: "ECOKV_ERR_UNSUPPORTED", 3: "ECOKV_ERR_WORKSPACE",
          4: "ECOKV_ERR_CUDA", 5: "ECOKV_ERR_TIMEOUT", 6: "ECOKV_ERR_DEVICE_INDEX"}

EXPORTS = ("ecokv_params_default", "ecokv_check_params", "ecokv_workspace_size", "ecokv_score",
           "ecokv_select", "ecokv_compact", "ecokv_evict", "ecokv_device_status", "ecokv_status_string",
           "ecokv_evict_noalloc", "ecokv_set_stage_events", "ecokv_workspace_size_host", "ecokv_evict_host",
           "ecokv_evict_adaptive", "ecokv_evict_layered", "ecokv_pyramid_budgets",
           "ecokv_rotary_init", "ecokv_rotary_set", "ecokv_rotary_sections", "ecokv_rotate", "ecokv_append",
           "ecokv_attend_workspace_size", "ecokv_attend")
ROTARY_LAYOUT = {"half": 0, "interleaved": 1}
ROTARY_SCALING = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}
HEAD_DIM = 128


class EcokvError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {STATUS.get(code, code)} ({ecokv_status_string(code)})")


class ecokv_params(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("h_kv", ctypes.c_int32), ("h_q", ctypes.c_int32),
                ("n", ctypes.c_int32), ("d", ctypes.c_int32), ("window", ctypes.c_int32),
                ("budget", ctypes.c_int32), ("pool_kernel", ctypes.c_int32),
                ("alpha", ctypes.c_float), ("beta", ctypes.c_float), ("tau", ctypes.c_float),
                ("eps", ctypes.c_float), ("flags", ctypes.c_uint32), ("lambda_override", ctypes.c_float),
                ("sched_wave", ctypes.c_int32), ("sched_lag", ctypes.c_int32), ("timeout_us", ctypes.c_uint32)]

    def as_dict(self) -> dict:
        return {f: getattr(self, f) for f, _ in self._fields_}


_lib = None
_P = ctypes.POINTER(ecokv_params)
_vp, _sz = ctypes.c_void_p, ctypes.c_size_t
_i32, _i64 = ctypes.c_int32, ctypes.c_int64


class ecokv_rotary(ctypes.Structure):
    _fields_ = [("rot_dim", _i32), ("layout", _i32), ("axes", _i32), ("magnitude", ctypes.c_float),
                ("turns", ctypes.c_uint64 * 64), ("axis", ctypes.c_uint8 * 64)]


class ecokv_rows(ctypes.Structure):
    _fields_ = [("x", _vp), ("y", _vp), ("x_token", _i64), ("x_head", _i64), ("y_token", _i64), ("y_head", _i64),
                ("norm", _vp), ("heads", _i32)]


class ecokv_pages(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("page_stride", _i64), ("head_stride", _i64), ("slot_stride", _i64),
                ("n_pages", _i32), ("page_size", _i32), ("table", _vp), ("table_stride", _i32), ("lengths", _vp)]


class ecokv_prefix(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("head_stride", _i64), ("row_stride", _i64), ("rows", _i32),
                ("head_off", _vp)]


class ecokv_attend_params(ctypes.Structure):
    _fields_ = [("h_q", _i32), ("h_kv", _i32), ("d", _i32), ("tokens", _i32), ("batch", _i32),
                ("scale", ctypes.c_float), ("q_token", _i64), ("q_head", _i64), ("out_token", _i64),
                ("out_head", _i64), ("flags", ctypes.c_uint32), ("timeout_us", ctypes.c_uint32)]


def lib() -> ctypes.CDLL:
    """Load libecokv.so once (RuntimeError if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"libecokv.so not found at {LIB_PATH}; build it with "
                               "`python -m paper_2609_06663_gb300.build` (no CPU fallback exists)")
        L = ctypes.CDLL(LIB_PATH)
        L.ecokv_params_default.argtypes = [_P]
        L.ecokv_params_default.restype = None
        L.ecokv_check_params.argtypes = [_P]
        L.ecokv_check_params.restype = ctypes.c_int
        L.ecokv_workspace_size.argtypes = [_P]
        L.ecokv_workspace_size.restype = _sz
        L.ecokv_score.argtypes = [_P, ctypes.c_int, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
        L.ecokv_score.restype = ctypes.c_int
        L.ecokv_select.argtypes = [_P, _vp, _vp, _vp, _sz, _vp]
        L.ecokv_select.restype = ctypes.c_int
        L.ecokv_compact.argtypes = [_P, ctypes.c_int, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
        L.ecokv_compact.restype = ctypes.c_int
        L.ecokv_evict.argtypes = [_P, ctypes.c_int, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
        L.ecokv_evict.restype = ctypes.c_int
        L.ecokv_evict_noalloc.argtypes = [_P, ctypes.c_int, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]
        L.ecokv_evict_noalloc.restype = ctypes.c_int
        L.ecokv_workspace_size_host.argtypes = [_P, ctypes.c_int]
        L.ecokv_workspace_size_host.restype = _sz
        L.ecokv_evict_host.argtypes = [_P, ctypes.c_int, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
        L.ecokv_evict_host.restype = ctypes.c_int
        L.ecokv_evict_adaptive.argtypes = [_P, ctypes.c_int, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
        L.ecokv_evict_adaptive.restype = ctypes.c_int
        L.ecokv_evict_layered.argtypes = [_P, ctypes.c_int, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz,
                                          _vp]
        L.ecokv_evict_layered.restype = ctypes.c_int
        L.ecokv_pyramid_budgets.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_float, _vp]
        L.ecokv_pyramid_budgets.restype = ctypes.c_int
        L.ecokv_set_stage_events.argtypes = [ctypes.POINTER(_vp), ctypes.c_int]
        L.ecokv_set_stage_events.restype = ctypes.c_int
        f32, rows = ctypes.c_float, ctypes.POINTER(ecokv_rows)
        L.ecokv_rotary_init.argtypes = [ctypes.POINTER(ecokv_rotary), _i32, _i32, ctypes.c_double, _i32,
                                        ctypes.c_double, _i32]
        L.ecokv_rotary_init.restype = ctypes.c_int
        L.ecokv_rotary_set.argtypes = [ctypes.POINTER(ecokv_rotary), _i32, _i32, _vp, f32]
        L.ecokv_rotary_set.restype = ctypes.c_int
        L.ecokv_rotary_sections.argtypes = [ctypes.POINTER(ecokv_rotary), _vp, _i32]
        L.ecokv_rotary_sections.restype = ctypes.c_int
        L.ecokv_rotate.argtypes = [ctypes.POINTER(ecokv_rotary), ctypes.c_int, rows, rows, _vp, _i32, f32, _vp]
        L.ecokv_rotate.restype = ctypes.c_int
        L.ecokv_append.argtypes = [ctypes.POINTER(ecokv_rotary), ctypes.c_int, rows, rows, rows,
                                   ctypes.POINTER(ecokv_pages), _vp, _vp, _i32, _i32, f32, _vp, _sz, _vp]
        L.ecokv_append.restype = ctypes.c_int
        L.ecokv_attend_workspace_size.argtypes = [_i32, _i32, _i32, _i32, ctypes.c_int]
        L.ecokv_attend_workspace_size.restype = _sz
        L.ecokv_attend.argtypes = [ctypes.POINTER(ecokv_attend_params), ctypes.c_int, _vp,
                                   ctypes.POINTER(ecokv_prefix), ctypes.POINTER(ecokv_pages), _vp, _vp, _vp, _vp,
                                   _sz, _vp]
        L.ecokv_attend.restype = ctypes.c_int
        L.ecokv_device_status.argtypes = [_vp, _vp]
        L.ecokv_device_status.restype = ctypes.c_int
        L.ecokv_status_string.argtypes = [ctypes.c_int]
        L.ecokv_status_string.restype = ctypes.c_char_p
        _lib = L
    return _lib


def _ptr(x) -> int | None:
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _stream(s) -> int | None:
    if s is None:
        return None
    if isinstance(s, int):
        return s
    return s.cuda_stream


def _check(code: int, where: str) -> None:
    if code != 0:
        raise EcokvError(code, where)


# ---------------------------------------------------------------- C ABI, same names
def ecokv_params_default() -> ecokv_params:
    p = ecokv_params()
    lib().ecokv_params_default(ctypes.byref(p))
    return p


def ecokv_check_params(p: ecokv_params) -> int:
    return lib().ecokv_check_params(ctypes.byref(p))


def ecokv_workspace_size(p: ecokv_params) -> int:
    return lib().ecokv_workspace_size(ctypes.byref(p))


def ecokv_status_string(code: int) -> str:
    return lib().ecokv_status_string(code).decode()


def ecokv_score(p, dtype, K, Qwin, S, lam, dbg, ws, ws_bytes, stream=None) -> int:
    return lib().ecokv_score(ctypes.byref(p), dtype, _ptr(K), _ptr(Qwin), _ptr(S), _ptr(lam), _ptr(dbg),
                             _ptr(ws), ws_bytes, _stream(stream))


def ecokv_select(p, S, idx, ws=None, ws_bytes=0, stream=None) -> int:
    return lib().ecokv_select(ctypes.byref(p), _ptr(S), _ptr(idx), _ptr(ws), ws_bytes, _stream(stream))


def ecokv_compact(p, dtype, K, V, idx, K_out, V_out, ws=None, ws_bytes=0, stream=None) -> int:
    return lib().ecokv_compact(ctypes.byref(p), dtype, _ptr(K), _ptr(V), _ptr(idx), _ptr(K_out), _ptr(V_out),
                               _ptr(ws), ws_bytes, _stream(stream))


def ecokv_evict(p, dtype, K, V, Qwin, idx, K_out, V_out, S, lam, ws, ws_bytes, stream=None) -> int:
    return lib().ecokv_evict(ctypes.byref(p), dtype, _ptr(K), _ptr(V), _ptr(Qwin), _ptr(idx), _ptr(K_out),
                             _ptr(V_out), _ptr(S), _ptr(lam), _ptr(ws), ws_bytes, _stream(stream))


def ecokv_evict_adaptive(p, dtype, K, V, Qwin, idx, head_off, K_out, V_out, lam, ws, ws_bytes, stream=None) -> int:
    return lib().ecokv_evict_adaptive(ctypes.byref(p), dtype, _ptr(K), _ptr(V), _ptr(Qwin), _ptr(idx),
                                      _ptr(head_off), _ptr(K_out), _ptr(V_out), _ptr(lam), _ptr(ws), ws_bytes,
                                      _stream(stream))


def ecokv_evict_layered(p, dtype, K, V, Qwin, layer_budget, idx, K_out, V_out, S, lam, ws, ws_bytes,
                        stream=None) -> int:
    return lib().ecokv_evict_layered(ctypes.byref(p), dtype, _ptr(K), _ptr(V), _ptr(Qwin), _ptr(layer_budget),
                                     _ptr(idx), _ptr(K_out), _ptr(V_out), _ptr(S), _ptr(lam), _ptr(ws), ws_bytes,
                                     _stream(stream))


def pyramid_budgets(n_layers: int, budget: int, window: int, beta: float) -> list:
    """PyramidKV's per-layer budgets from the library (host computation)."""
    out = (ctypes.c_int32 * n_layers)()
    _check(lib().ecokv_pyramid_budgets(n_layers, budget, window, beta, ctypes.addressof(out)), "ecokv_pyramid_budgets")
    return list(out)


def ecokv_workspace_size_host(p, dtype) -> int:
    return lib().ecokv_workspace_size_host(ctypes.byref(p), dtype)


def ecokv_evict_host(p, dtype, K, V, Qwin, idx, K_out, V_out, lam, ws, ws_bytes, stream=None) -> int:
    return lib().ecokv_evict_host(ctypes.byref(p), dtype, _ptr(K), _ptr(V), _ptr(Qwin), _ptr(idx), _ptr(K_out),
                                  _ptr(V_out), _ptr(lam), _ptr(ws), ws_bytes, _stream(stream))


def ecokv_evict_noalloc(p, dtype, K, V, Qwin, idx, K_out, V_out, S, lam, dev_status, stream=None) -> int:
    return lib().ecokv_evict_noalloc(ctypes.byref(p), dtype, _ptr(K), _ptr(V), _ptr(Qwin), _ptr(idx),
                                     _ptr(K_out), _ptr(V_out), _ptr(S), _ptr(lam), _ptr(dev_status),
                                     _stream(stream))


def ecokv_set_stage_events(events) -> int:
    """events: None (hook off) or 4 torch.cuda.Event objects (or raw handles)."""
    if events is None:
        return lib().ecokv_set_stage_events(None, 0)
    hs = [e.cuda_event if hasattr(e, "cuda_event") else int(e) for e in events]
    arr = (_vp * len(hs))(*hs)
    return lib().ecokv_set_stage_events(arr, len(hs))


def ecokv_rotary_init(r, rot_dim, layout, base, scaling=0, factor=1.0, original=0) -> int:
    return lib().ecokv_rotary_init(r, rot_dim, layout, base, scaling, factor, original)


def ecokv_rotary_set(r, rot_dim, layout, inv_freq, magnitude=1.0) -> int:
    """inv_freq: rot_dim / 2 radians a position, or None."""
    f = None if inv_freq is None else (ctypes.c_double * len(inv_freq))(*inv_freq)
    return lib().ecokv_rotary_set(r, rot_dim, layout, f, magnitude)


def ecokv_rotary_sections(r, counts) -> int:
    return lib().ecokv_rotary_sections(r, (_i32 * len(counts))(*counts), len(counts))


def ecokv_rotate(r, dtype, q, k, positions, tokens, eps, stream=None) -> int:
    return lib().ecokv_rotate(r, dtype, q, k, _ptr(positions), tokens, eps, _stream(stream))


def ecokv_append(r, dtype, q, k, v, cache, positions, starts, tokens, batch, eps, ws=None, ws_bytes=0,
                 stream=None) -> int:
    return lib().ecokv_append(r, dtype, q, k, v, cache, _ptr(positions), _ptr(starts), tokens, batch, eps, _ptr(ws),
                              ws_bytes, _stream(stream))


def ecokv_attend_workspace_size(tokens, batch, h_q, h_kv, dtype) -> int:
    return lib().ecokv_attend_workspace_size(tokens, batch, h_q, h_kv, dtype)


def ecokv_attend(p, dtype, q, prefix, cache, starts, out, lse, ws, ws_bytes, stream=None) -> int:
    return lib().ecokv_attend(p, dtype, _ptr(q), prefix, cache, _ptr(starts), _ptr(out), _ptr(lse), _ptr(ws),
                              ws_bytes, _stream(stream))


def ecokv_device_status(ws, stream=None) -> int:
    return lib().ecokv_device_status(_ptr(ws), _stream(stream))


# ---------------------------------------------------------------- torch helpers
def make_params(*, n_layers, h_kv, h_q, n, d=128, window, budget, pool_kernel=5, alpha=0.8, beta=0.6,
                tau=0.0, eps=1e-6, flags=0, lambda_override=0.0, sched_wave=0, sched_lag=0,
                timeout_us=0) -> ecokv_params:
    p = ecokv_params()
    for k, v in dict(n_layers=n_layers, h_kv=h_kv, h_q=h_q, n=n, d=d, window=window, budget=budget,
                     pool_kernel=pool_kernel, alpha=alpha, beta=beta, tau=tau, eps=eps, flags=flags,
                     lambda_override=lambda_override, sched_wave=sched_wave, sched_lag=sched_lag,
                     timeout_us=timeout_us).items():
        setattr(p, k, v)
    return p


def dtype_code(t) -> int:
    import torch
    if t.dtype == torch.float32:
        return ECOKV_F32
    if t.dtype == torch.bfloat16:
        return ECOKV_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def alloc_workspace(p: ecokv_params, device="cuda"):
    import torch
    nbytes = ecokv_workspace_size(p)
    if nbytes == 0:
        _check(ecokv_check_params(p) or 1, "ecokv_workspace_size")
    ws = torch.zeros(nbytes, dtype=torch.uint8, device=device)
    return ws


_get_device = None


def _current(dev):
    """The library launches on the current device: dev is to be that one."""
    global _get_device
    if _get_device is None:
        import torch
        _get_device = torch._C._cuda_getDevice
    if dev != _get_device():
        raise ValueError(f"tensors on cuda:{dev}, while cuda:{_get_device()} is the current device")


# A call runs on `stream` (a torch.cuda.Stream or a raw handle), by default on
# torch's current one.  Tensors that are not given are allocated by the helper on
# that stream; those that are given the caller has ordered with it.
@contextlib.contextmanager
def _running(stream, device):
    """A call on `stream`, which is current within: what is allocated there belongs
    to it (a fill, and whoever had the memory before, come ahead of the call's
    kernels; memory that is given back is not used again ahead of them).  Yields the
    stream's raw handle and keep(), which keeps a tensor's memory until the caller's
    current stream is done with it too."""
    import torch
    if device != "cuda":
        _current(device.index)
    caller = torch.cuda.current_stream(device)
    if stream is None:
        yield caller.cuda_stream, lambda x: x
        return
    if isinstance(stream, int):  # (0 and 1: the legacy default stream, which is torch's default one)
        stream = torch.cuda.default_stream(device) if stream in (0, 1) else \
            torch.cuda.ExternalStream(stream, device=device)

    def keep(x):
        x.record_stream(caller)
        return x

    with torch.cuda.stream(stream):
        yield stream.cuda_stream, keep


def score(p, K, Qwin, ws=None, dbg=False, stream=None):
    """Run ecokv_score; returns (S [L,H,N-W], lambda [L,H], dbg or None)."""
    import torch
    with _running(stream, K.device) as (on, keep):
        ws = alloc_workspace(p, K.device) if ws is None else ws
        S = keep(torch.empty(p.n_layers, p.h_kv, p.n - p.window, dtype=torch.float32, device=K.device))
        lam = keep(torch.empty(p.n_layers, p.h_kv, dtype=torch.float32, device=K.device))
        D = keep(torch.empty(p.n_layers, p.h_kv, 5, p.n - p.window, dtype=torch.float32, device=K.device)) \
            if dbg else None
        _check(ecokv_score(p, dtype_code(K), K, Qwin, S, lam, D, ws, ws.numel(), on), "ecokv_score")
        return S, lam, D


def select(p, S, stream=None):
    import torch
    with _running(stream, S.device) as (on, keep):
        idx = keep(torch.empty(p.n_layers, p.h_kv, min(p.budget, p.n), dtype=torch.int32, device=S.device))
        _check(ecokv_select(p, S, idx, None, 0, on), "ecokv_select")
        return idx


def compact(p, K, V, idx, ws=None, stream=None):
    import torch
    with _running(stream, K.device) as (on, keep):
        n_keep = min(p.budget, p.n)
        Ko = keep(torch.empty(p.n_layers, p.h_kv, n_keep, p.d, dtype=K.dtype, device=K.device))
        Vo = keep(torch.empty_like(Ko))
        _check(ecokv_compact(p, dtype_code(K), K, V, idx, Ko, Vo, ws, 0 if ws is None else ws.numel(), on),
               "ecokv_compact")
        return Ko, Vo


def evict(p, K, V, Qwin, ws=None, want_scores=False, stream=None):
    """Run ecokv_evict; returns (idx, K_out, V_out, S or None, lambda)."""
    import torch
    with _running(stream, K.device) as (on, keep):
        ws = alloc_workspace(p, K.device) if ws is None else ws
        n_keep = min(p.budget, p.n)
        idx = keep(torch.empty(p.n_layers, p.h_kv, n_keep, dtype=torch.int32, device=K.device))
        Ko = keep(torch.empty(p.n_layers, p.h_kv, n_keep, p.d, dtype=K.dtype, device=K.device))
        Vo = keep(torch.empty_like(Ko))
        S = keep(torch.empty(p.n_layers, p.h_kv, p.n - p.window, dtype=torch.float32, device=K.device)) \
            if want_scores else None
        lam = keep(torch.empty(p.n_layers, p.h_kv, dtype=torch.float32, device=K.device))
        _check(ecokv_evict(p, dtype_code(K), K, V, Qwin, idx, Ko, Vo, S, lam, ws, ws.numel(), on),
               "ecokv_evict")
        return idx, Ko, Vo, S, lam


def evict_adaptive(p, K, V, Qwin, ws=None, stream=None):
    """Run ecokv_evict_adaptive (layer-wide budget); returns (idx [L][h_kv*B],
    head_off [L][h_kv+1], K_out, V_out [L][h_kv*B][d], lambda)."""
    import torch
    with _running(stream, K.device) as (on, keep):
        ws = alloc_workspace(p, K.device) if ws is None else ws
        rows = p.h_kv * min(p.budget, p.n)
        idx = keep(torch.empty(p.n_layers, rows, dtype=torch.int32, device=K.device))
        off = keep(torch.empty(p.n_layers, p.h_kv + 1, dtype=torch.int32, device=K.device))
        Ko = keep(torch.empty(p.n_layers, rows, p.d, dtype=K.dtype, device=K.device))
        Vo = keep(torch.empty_like(Ko))
        lam = keep(torch.empty(p.n_layers, p.h_kv, dtype=torch.float32, device=K.device))
        _check(ecokv_evict_adaptive(p, dtype_code(K), K, V, Qwin, idx, off, Ko, Vo, lam, ws, ws.numel(), on),
               "ecokv_evict_adaptive")
        return idx, off, Ko, Vo, lam


def evict_layered(p, K, V, Qwin, budgets, ws=None, want_scores=False, stream=None):
    """Run ecokv_evict_layered with budgets[l] for layer l (p.budget is the
    per-head stride, at least max(budgets)); returns as evict()."""
    import torch
    with _running(stream, K.device) as (on, keep):
        ws = alloc_workspace(p, K.device) if ws is None else ws
        n_keep = min(p.budget, p.n)
        lb = torch.tensor(list(budgets), dtype=torch.int32)
        idx = keep(torch.empty(p.n_layers, p.h_kv, n_keep, dtype=torch.int32, device=K.device))
        Ko = keep(torch.zeros(p.n_layers, p.h_kv, n_keep, p.d, dtype=K.dtype, device=K.device))
        Vo = keep(torch.zeros_like(Ko))
        S = keep(torch.empty(p.n_layers, p.h_kv, p.n - p.window, dtype=torch.float32, device=K.device)) \
            if want_scores else None
        lam = keep(torch.empty(p.n_layers, p.h_kv, dtype=torch.float32, device=K.device))
        _check(ecokv_evict_layered(p, dtype_code(K), K, V, Qwin, lb.data_ptr(), idx, Ko, Vo, S, lam, ws, ws.numel(),
                                   on), "ecokv_evict_layered")
        return idx, Ko, Vo, S, lam


def alloc_workspace_host(p, dtype, device="cuda"):
    """Device workspace for ecokv_evict_host (uint8 tensor)."""
    import torch
    n = ecokv_workspace_size_host(p, dtype)
    if n == 0:
        raise EcokvError(ECOKV_ERR_INVALID_ARG, "ecokv_workspace_size_host")
    return torch.empty(n, dtype=torch.uint8, device=device)


def evict_host(p, K, V, Qwin, ws=None, stream=None):
    """Run ecokv_evict_host on pinned host tensors; returns pinned host
    (idx, K_out, V_out, lambda), valid once the stream has been synchronised."""
    import torch
    with _running(stream, "cuda") as (on, _):
        dt = dtype_code(K)
        ws = alloc_workspace_host(p, dt) if ws is None else ws
        n_keep = min(p.budget, p.n)
        idx = torch.empty(p.n_layers, p.h_kv, n_keep, dtype=torch.int32).pin_memory()
        Ko = torch.empty(p.n_layers, p.h_kv, n_keep, p.d, dtype=K.dtype).pin_memory()
        Vo = torch.empty(p.n_layers, p.h_kv, n_keep, p.d, dtype=K.dtype).pin_memory()
        lam = torch.empty(p.n_layers, p.h_kv, dtype=torch.float32).pin_memory()
        _check(ecokv_evict_host(p, dt, K, V, Qwin, idx, Ko, Vo, lam, ws, ws.numel(), on), "ecokv_evict_host")
        return idx, Ko, Vo, lam


def evict_noalloc(p, K, V, Qwin, want_scores=False, stream=None):
    """Run ecokv_evict_noalloc (library-held scratch, no workspace argument);
    returns (idx, K_out, V_out, S or None, lambda, device status code)."""
    import torch
    with _running(stream, K.device) as (on, keep):
        n_keep = min(p.budget, p.n)
        idx = keep(torch.empty(p.n_layers, p.h_kv, n_keep, dtype=torch.int32, device=K.device))
        Ko = keep(torch.empty(p.n_layers, p.h_kv, n_keep, p.d, dtype=K.dtype, device=K.device))
        Vo = keep(torch.empty_like(Ko))
        S = keep(torch.empty(p.n_layers, p.h_kv, p.n - p.window, dtype=torch.float32, device=K.device)) \
            if want_scores else None
        lam = keep(torch.empty(p.n_layers, p.h_kv, dtype=torch.float32, device=K.device))
        code = keep(torch.full((1,), -1, dtype=torch.int32, device=K.device))
        _check(ecokv_evict_noalloc(p, dtype_code(K), K, V, Qwin, idx, Ko, Vo, S, lam, code, on),
               "ecokv_evict_noalloc")
        return idx, Ko, Vo, S, lam, int(code.item())


# ---------------------------------------------------------------- the decode step
def rotary(rot_dim=HEAD_DIM, base=10000.0, layout="half", scaling="none", factor=1.0, original=0, sections=None,
           inv_freq=None, magnitude=1.0) -> ecokv_rotary:
    """Rotary positions of a model, kept for its calls.  scaling: "none",
    "linear", "ntk" or "yarn" (the last needs `original`); inv_freq: the caller's
    own frequencies (with `magnitude`) in place of base and scaling; sections:
    pairs each position axis turns (time, height, width ...), default one axis."""
    r = ecokv_rotary()
    lay = ROTARY_LAYOUT[layout]
    if inv_freq is not None:
        inv_freq = [float(f) for f in inv_freq]
        if len(inv_freq) != rot_dim // 2:
            raise ValueError(f"{len(inv_freq)} frequencies for {rot_dim // 2} pairs")
        _check(ecokv_rotary_set(r, rot_dim, lay, inv_freq, magnitude), "ecokv_rotary_set")
    else:
        _check(ecokv_rotary_init(r, rot_dim, lay, base, ROTARY_SCALING[scaling], factor, original),
               "ecokv_rotary_init")
    if sections is not None:
        _check(ecokv_rotary_sections(r, sections), "ecokv_rotary_sections")
    return r


def _dtype(t, *others):
    """Their common dtype's code and CUDA device."""
    dt, dev = t.dtype, t.get_device()
    if dev < 0:
        raise ValueError("CUDA tensors are wanted")
    for x in others:
        if x is not None and (x.dtype is not dt or x.get_device() != dev):
            raise TypeError(f"{x.dtype} on {x.device} next to {dt} on {t.device}")
    code = _codes.get(dt)
    if code is None:
        code = _codes[dt] = dtype_code(t)
    return code, dev


_codes = {}  # torch dtype -> code


_int32 = None


def _ints(x, shape, what, dev):
    global _int32
    if x is None:
        return None
    if _int32 is None:
        import torch
        _int32 = torch.int32
    if x.dtype is not _int32 or x.get_device() != dev or not x.is_contiguous() or (shape and x.shape != shape):
        of = f" of shape {shape}" if shape else ""
        raise ValueError(f"{what}: a contiguous int32 tensor{of} on cuda:{dev} is wanted")
    return x.data_ptr()


def _strides(x):
    """Strides in elements; one that is never taken (an axis of one or none) counts as a row."""
    return tuple(s if n > 1 else HEAD_DIM for n, s in zip(x.shape[:-1], x.stride())) + x.stride()[-1:]


def _heads(x, what):
    """Rows [tokens, heads, d]: (tokens, heads, their two strides)."""
    n, s = x.shape, x.stride()
    if len(n) != 3 or n[2] != HEAD_DIM or s[2] != 1:
        raise ValueError(f"{what}: rows [tokens, heads, {HEAD_DIM}] with the last axis contiguous are wanted")
    tokens, heads, _ = n
    # (a stride that is never taken counts as a row)
    return tokens, heads, s[0] if tokens > 1 else HEAD_DIM, s[1] if heads > 1 else HEAD_DIM


def _rows(x, y, norm, what):
    n, s = x.shape, x.stride()
    if len(n) != 3 or n[2] != HEAD_DIM or s[2] != 1:
        _heads(x, what)  # (raises)
    tokens, heads, _ = n
    if norm is not None:
        if norm.numel() != HEAD_DIM or not norm.is_contiguous():
            raise ValueError(f"{what}: contiguous norm weights [{HEAD_DIM}] are wanted")
        norm = norm.data_ptr()
    at, t = None, (0, 0)
    if y is not None:
        if y.shape != n:
            raise ValueError(f"{what}: the output has another shape")
        at, t = y.data_ptr(), y.stride()
        if t[2] != 1:
            _heads(y, what)
    if tokens > 1 and heads > 1:
        return ecokv_rows(x.data_ptr(), at, s[0], s[1], t[0], t[1], norm, heads)
    # (a stride that is never taken counts as a row)
    many, two = tokens > 1, heads > 1
    return ecokv_rows(x.data_ptr(), at, s[0] if many else HEAD_DIM, s[1] if two else HEAD_DIM,
                      t[0] if many else HEAD_DIM, t[1] if two else HEAD_DIM, norm, heads)


_raw_stream = None


def _on(stream, dev):
    """The raw stream to launch on."""
    if _get_device is None or dev != _get_device():
        _current(dev)
    if stream is None:
        global _raw_stream
        if _raw_stream is None:
            import torch
            # (torch.cuda.current_stream builds an object: 2 us of a call of 8)
            _raw_stream = torch._C._cuda_getCurrentRawStream
        return _raw_stream(dev)
    return stream if isinstance(stream, int) else stream.cuda_stream


def _made(stream, t, make):
    """What make() allocates for a call on `stream`, beside the tensor t."""
    if stream is None:
        return make()
    with _running(stream, t.device) as (_, keep):
        return keep(make())


def _like(x, stream):
    return _made(stream, x, lambda: x.new_empty(x.shape))


def rotate(rot, positions, q, k=None, q_norm=None, k_norm=None, eps=1e-6, q_out=None, k_out=None, stream=None):
    """Run ecokv_rotate: norm (where weights are given) and rotary positions of
    q and k [tokens, heads, 128].  rot: from rotary(), None for the norms alone;
    positions int32 [axes, tokens] (or [tokens]).  Outputs may have any strides
    (k_out a view of the [heads, tokens, 128] that the eviction pass reads) or be
    the inputs.  Returns (q_out, k_out)."""
    if q_out is None:
        q_out = _like(q, stream)
    if k is not None and k_out is None:
        k_out = _like(k, stream)
    dt, dev = _dtype(q, k, q_norm, k_norm, q_out, k_out)
    tokens = q.shape[0]
    if k is not None and k.shape[0] != tokens:
        raise ValueError("q and k have different numbers of tokens")
    pos = _positions(rot, positions, tokens, dev)
    _check((_lib or lib()).ecokv_rotate(rot, dt, _rows(q, q_out, q_norm, "q"),
                              None if k is None else _rows(k, k_out, k_norm, "k"), pos, tokens, eps,
                              _on(stream, dev)), "ecokv_rotate")
    return q_out, k_out


def _positions(rot, positions, tokens, dev):
    if rot is None:
        return None
    if positions is None:
        raise ValueError("positions are wanted")
    n, axes = positions.shape, rot.axes
    if n[-1] != tokens or (n[0] != axes or len(n) != 2) and (len(n) != 1 or axes != 1):
        raise ValueError(f"positions: [{axes}, {tokens}] is wanted")
    return _ints(positions, None, "positions", dev)


class _Handle:
    """What the library was given the address of stays: a tensor in its place would not be read."""

    def __setattr__(self, name, x):
        if self.__dict__.get(name, x) is not x:
            raise AttributeError(f"{name}: write into the tensor, or make a new {type(self).__name__}")
        self.__dict__[name] = x


class PagedCache(_Handle):
    """A paged cache: k_pages, v_pages [n_pages, h_kv, page_size, 128] (views of
    any strides, the same for both, the last axis contiguous), table int32
    [batch, pages a sequence], lengths int32 [batch].  Holds its tensors; table and
    lengths are read on the device by every call, and written in place between them."""

    def __init__(self, k_pages, v_pages, table, lengths):
        _, dev = _dtype(k_pages, v_pages)
        s = _strides(k_pages)
        if k_pages.dim() != 4 or k_pages.shape[3] != HEAD_DIM or s[3] != 1:
            raise ValueError(f"pages [n_pages, h_kv, page_size, {HEAD_DIM}] with the last axis contiguous are wanted")
        if v_pages.shape != k_pages.shape or _strides(v_pages) != s:
            raise ValueError("k_pages and v_pages have different shapes or strides")
        if table.dim() != 2 or tuple(lengths.shape) != (table.shape[0],):
            raise ValueError("table [batch, pages a sequence] and lengths [batch] are wanted")
        self.k_pages, self.v_pages, self.table, self.lengths = k_pages, v_pages, table, lengths
        self.batch, self.h_kv = table.shape[0], k_pages.shape[1]
        self.c = ecokv_pages(k_pages.data_ptr(), v_pages.data_ptr(), s[0], s[1], s[2], k_pages.shape[0],
                             k_pages.shape[2], _ints(table, None, "table", dev), table.shape[1],
                             _ints(lengths, None, "lengths", dev))


class Prefix(_Handle):
    """The shared prefix of one layer: k, v [h_kv, rows, 128] as evict() returns a
    layer, or [rows, 128] with head_off int32 [h_kv + 1] as evict_adaptive() does."""

    def __init__(self, k, v, head_off=None):
        _, dev = _dtype(k, v)
        s = _strides(k)
        if k.dim() != (3 if head_off is None else 2) or k.shape[-1] != HEAD_DIM or s[-1] != 1:
            raise ValueError(f"prefix: [h_kv, rows, {HEAD_DIM}], or [rows, {HEAD_DIM}] with head_off, is wanted")
        if v.shape != k.shape or _strides(v) != s:
            raise ValueError("k and v have different shapes or strides")
        self.k, self.v, self.head_off = k, v, head_off
        self.h_kv = k.shape[0] if head_off is None else head_off.shape[0] - 1
        self.c = ecokv_prefix(k.data_ptr(), v.data_ptr(), s[0] if head_off is None else 0, s[-2], k.shape[-2],
                              _ints(head_off, None, "head_off", dev))


def append(cache, k, v, starts=None, rotary=None, positions=None, q=None, q_norm=None, k_norm=None, eps=1e-6,
           q_out=None, ws=None, stream=None):
    """Run ecokv_append: k (normed, rotated) and v [tokens, h_kv, 128] into the
    cache's slots, q (normed, rotated) to q_out, which is returned.  starts int32
    [batch + 1]: None = one token a sequence.  ws: a workspace whose status word
    takes device-side errors."""
    if q is not None and q_out is None:
        q_out = _like(q, stream)
    dt, dev = _dtype(k, v, cache.k_pages, q, q_norm, k_norm, q_out)
    tokens = k.shape[0]
    if v.shape != k.shape or k.shape[1] != cache.h_kv or (q is not None and q.shape[0] != tokens):
        raise ValueError("k, v and q do not fit together or the cache")
    if ws is not None and ws.get_device() != dev:
        raise ValueError(f"the workspace is on {ws.device}, the tensors on cuda:{dev}")
    _check((_lib or lib()).ecokv_append(rotary, dt, None if q is None else _rows(q, q_out, q_norm, "q"),
                              _rows(k, None, k_norm, "k"), _rows(v, None, None, "v"), cache.c,
                              _positions(rotary, positions, tokens, dev),
                              _ints(starts, (cache.batch + 1,), "starts", dev), tokens, cache.batch, eps, _ptr(ws),
                              0 if ws is None else ws.numel(), _on(stream, dev)),
           "ecokv_append")
    return q_out


def alloc_attend_workspace(tokens, batch, h_q, h_kv, dtype, device="cuda"):
    """Workspace of attend() for up to `tokens` tokens of `batch` sequences (dtype: torch's)."""
    import torch
    n = ecokv_attend_workspace_size(tokens, batch, h_q, h_kv, ECOKV_F32 if dtype == torch.float32 else ECOKV_BF16)
    if n == 0:
        raise EcokvError(ECOKV_ERR_INVALID_ARG, "ecokv_attend_workspace_size")
    return torch.zeros(n, dtype=torch.uint8, device=device)


def attend(q, prefix, cache, starts=None, scale=0.0, out=None, lse=None, ws=None, flags=0, timeout_us=0, stream=None):
    """Run ecokv_attend: q [tokens, h_q, 128] over prefix (a Prefix or None) and
    cache (a PagedCache or None); returns out [tokens, h_q, 128].  starts int32
    [batch + 1]: None = one token a sequence.  lse: float32 [tokens, h_q] to fill."""
    if out is None:
        out = _like(q, stream)
    if prefix is None and cache is None:
        raise ValueError("a prefix or a cache is wanted")
    dt, dev = _dtype(q, out, None if prefix is None else prefix.k, None if cache is None else cache.k_pages)
    tokens, h_q, qt, qh = _heads(q, "q")
    to, ho, ot, oh = _heads(out, "out")
    h_kv = prefix.h_kv if cache is None else cache.h_kv
    if to != tokens or ho != h_q or (prefix is not None and prefix.h_kv != h_kv):
        raise ValueError("out or the prefix does not fit")
    batch = 1 if cache is None else cache.batch
    if lse is not None and (str(lse.dtype) != "torch.float32" or tuple(lse.shape) != (tokens, h_q) or
                            not lse.is_contiguous() or lse.get_device() != dev):
        raise ValueError(f"lse: a contiguous float32 [tokens, h_q] tensor on cuda:{dev} is wanted")
    if ws is None:
        ws = _made(stream, q, lambda: alloc_attend_workspace(tokens, batch, h_q, h_kv, q.dtype, q.device))
    if ws.get_device() != dev:
        raise ValueError(f"the workspace is on {ws.device}, the tensors on cuda:{dev}")
    p = ecokv_attend_params(h_q, h_kv, HEAD_DIM, tokens, batch, scale, qt, qh, ot, oh, flags, timeout_us)
    _check((_lib or lib()).ecokv_attend(p, dt, q.data_ptr(), None if prefix is None else prefix.c,
                              None if cache is None else cache.c,
                              None if cache is None else _ints(starts, (batch + 1,), "starts", dev), out.data_ptr(),
                              _ptr(lse), ws.data_ptr(), ws.numel(), _on(stream, dev)), "ecokv_attend")
    return out
