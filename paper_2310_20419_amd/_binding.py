"""ctypes marshalling for librnnd.so -- same names as the C entry points, no arithmetic."""
from __future__ import annotations

import ctypes
import os
import re

RNND_U8, RNND_F32, RNND_F16, RNND_BF16 = 0, 1, 2, 3
RNND_L2SQ = 0
RNND_MAX_R = 128
RNND_MAX_ROUNDS = 256

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = os.path.join(_HERE, "librnnd.so")
_HEADER = os.path.join(os.path.dirname(_HERE), "include", "rnnd.h")


class RnndError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("rnnd status %d: %s" % (status, message))
        self.status = status


class Stats(ctypes.Structure):
    _fields_ = [
        ("rounds", ctypes.c_int32),
        ("reverse_calls", ctypes.c_int32),
        ("kernel_variant", ctypes.c_int32),
        ("group_scans", ctypes.c_int32),
        ("total_ms", ctypes.c_float),
        ("init_ms", ctypes.c_float),
        ("round_ms", ctypes.c_float * RNND_MAX_ROUNDS),
        ("scan_ms", ctypes.c_float * RNND_MAX_ROUNDS),
        ("reverse_ms", ctypes.c_float * RNND_MAX_ROUNDS),
        ("init_evals", ctypes.c_int64),
        ("active", ctypes.c_int64 * RNND_MAX_ROUNDS),
        ("proposals", ctypes.c_int64 * RNND_MAX_ROUNDS),
        ("algo_evals", ctypes.c_int64 * RNND_MAX_ROUNDS),
        ("exec_evals", ctypes.c_int64 * RNND_MAX_ROUNDS),
        ("gathered_rows", ctypes.c_int64 * RNND_MAX_ROUNDS),
        ("dropped", ctypes.c_int64 * RNND_MAX_ROUNDS),
    ]

    def as_dict(self) -> dict:
        n = min(self.rounds, RNND_MAX_ROUNDS)
        return {
            "rounds": self.rounds, "reverse_calls": self.reverse_calls,
            "kernel_variant": self.kernel_variant, "group_scans": self.group_scans,
            "total_ms": self.total_ms, "init_ms": self.init_ms,
            "round_ms": list(self.round_ms[:n]), "scan_ms": list(self.scan_ms[:n]),
            "reverse_ms": list(self.reverse_ms[:max(0, self.reverse_calls)]),
            "init_evals": self.init_evals, "active": list(self.active[:n]),
            "proposals": list(self.proposals[:n]), "algo_evals": list(self.algo_evals[:n]),
            "exec_evals": list(self.exec_evals[:n]), "gathered_rows": list(self.gathered_rows[:n]),
            "dropped": list(self.dropped[:n]),
        }


class AdamwTensor(ctypes.Structure):
    """rnnd_adamw_tensor."""
    _fields_ = [
        ("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("m", ctypes.c_void_p), ("v", ctypes.c_void_p),
        ("m_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p), ("copy", ctypes.c_void_p),
        ("n", ctypes.c_int64), ("counter", ctypes.c_uint64),
        ("grad_dtype", ctypes.c_int32), ("copy_dtype", ctypes.c_int32), ("state_bits", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
    ]


def lib_path() -> str:
    return _LIB


def exported_symbols() -> list:
    """Function names include/rnnd.h declares."""
    text = open(_HEADER).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(rnnd_[a-z_]+)\s*\(", text)))


_lib = None


def load_library():
    """Loads the in-tree librnnd.so; fails loudly if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB):
            raise RnndError(-6, "librnnd.so is not built (run `python -m paper_2310_20419_amd.build`); "
                                "there is no CPU fallback")
        # PyTorch owns the device memory and streams handed to the library, so both must share one
        # HIP runtime: import torch first, so that librnnd.so binds to the runtime torch has loaded.
        import torch  # noqa: F401
        L = ctypes.CDLL(_LIB)
        c = ctypes
        vp, i64, i32, u64 = c.c_void_p, c.c_int64, c.c_int32, c.c_uint64
        L.rnnd_build.argtypes = [vp, i64, i32, c.c_int, c.c_int, i32, i32, i32, i32, u64, vp, vp, vp]
        L.rnnd_build_ex.argtypes = [vp, i64, i32, c.c_int, c.c_int, i32, i32, i32, i32, u64, vp, vp, vp,
                                    c.POINTER(Stats), vp]
        L.rnnd_build_wide.argtypes = [vp, i64, i32, c.c_int, c.c_int, i32, i32, i32, i32, i32, u64, vp, vp, vp,
                                      c.POINTER(Stats), vp]
        L.rnnd_build_blocks.argtypes = [vp, i64, i32, c.c_int, c.c_int, i32, i32, i32, i32, u64, i64, vp, vp, vp,
                                        c.POINTER(Stats), vp]
        L.rnnd_update_neighbors_blocks.argtypes = [vp, i64, i32, c.c_int, c.c_int, i32, vp, vp, i32, i64,
                                                   c.POINTER(Stats), vp]
        L.rnnd_workspace_bytes.argtypes = [i64, i32, c.c_int, i32, i64, c.POINTER(c.c_size_t)]
        L.rnnd_build_static.argtypes = L.rnnd_build.argtypes
        L.rnnd_release_workspace.argtypes = []
        L.rnnd_set_workspace_poison.argtypes = [c.c_int]
        L.rnnd_random_graph.argtypes = [vp, i64, i32, c.c_int, c.c_int, i32, i32, u64, vp, vp, vp]
        L.rnnd_update_neighbors.argtypes = [vp, i64, i32, c.c_int, c.c_int, i32, vp, vp, i32,
                                            c.POINTER(Stats), vp]
        L.rnnd_add_reverse_edges.argtypes = [i64, i32, vp, vp, vp]
        L.rnnd_add_reverse_edges_wide.argtypes = [i64, i32, i32, vp, vp, vp]
        L.rnnd_export_graph.argtypes = [i64, i32, vp, vp, vp, vp, vp]
        L.rnnd_search.argtypes = [vp, i64, i32, c.c_int, c.c_int, vp, vp, i32, vp, i64, i32, i32, i32, c.c_uint64,
                                  vp, vp, c.POINTER(c.c_int64), vp]
        L.rnnd_probe_gather.argtypes = [vp, i64, i64, i64, u64, c.POINTER(c.c_double), vp]
        L.rnnd_probe_gather_map.argtypes = [vp, i64, i64, i64, c.c_int, u64, c.POINTER(c.c_double), vp]
        L.rnnd_set_kernel_variant.argtypes = [c.c_int]
        L.rnnd_set_transpose_path.argtypes = [c.c_int]
        L.rnnd_set_scan_launches.argtypes = [c.c_int]
        L.rnnd_set_event_timing.argtypes = [c.c_int]
        sz, f32, f64 = c.c_size_t, c.c_float, c.c_double
        L.rnnd_embed.argtypes = [vp, i64, i32, c.c_int, vp, i64, f32, vp, c.c_int, vp]
        L.rnnd_embed_grad.argtypes = [vp, c.c_int, vp, i64, i32, f32, i64, vp, c.c_int, c.c_int, vp, sz, vp]
        L.rnnd_embed_grad_workspace.argtypes = [i64, i32, i64, c.POINTER(sz)]
        L.rnnd_contrast.argtypes = [vp, i64, vp, i64, i32, c.c_int, c.c_int, vp, vp, vp, vp, vp, f32, vp, vp, vp, vp, sz, vp]
        L.rnnd_contrast_workspace.argtypes = [i64, i64, i32, c.c_int, c.c_int, c.POINTER(sz)]
        L.rnnd_distill.argtypes = [vp, i64, vp, i64, i32, c.c_int, c.c_int, vp, vp, i32, c.c_int, vp, vp, vp, vp, f32, vp, vp, vp, vp, sz, vp]
        L.rnnd_distill_workspace.argtypes = [i64, i64, i32, c.c_int, i32, c.c_int, c.POINTER(sz)]
        L.rnnd_logprob.argtypes = [vp, i64, vp, i64, i32, c.c_int, c.c_int, vp, vp, vp, vp, f32, i32, vp, vp, vp, vp, vp, sz, vp]
        L.rnnd_logprob_workspace.argtypes = [i64, i64, i32, c.c_int, i32, c.POINTER(sz)]
        L.rnnd_adamw.argtypes = [c.POINTER(AdamwTensor), i32, i64, f64, f64, f64, f64, f64, f64, u64, vp]
        L.rnnd_strerror.argtypes = [c.c_int]
        L.rnnd_strerror.restype = c.c_char_p
        L.rnnd_version.restype = c.c_int
        for name in ("rnnd_build", "rnnd_build_ex", "rnnd_workspace_bytes", "rnnd_random_graph",
                     "rnnd_update_neighbors", "rnnd_add_reverse_edges", "rnnd_export_graph", "rnnd_search",
                     "rnnd_set_kernel_variant", "rnnd_build_blocks", "rnnd_update_neighbors_blocks",
                     "rnnd_probe_gather", "rnnd_build_wide", "rnnd_build_static", "rnnd_release_workspace",
                     "rnnd_set_workspace_poison", "rnnd_add_reverse_edges_wide", "rnnd_set_transpose_path",
                     "rnnd_set_event_timing", "rnnd_probe_gather_map", "rnnd_set_scan_launches",
                     "rnnd_embed", "rnnd_embed_grad", "rnnd_embed_grad_workspace", "rnnd_contrast",
                     "rnnd_contrast_workspace", "rnnd_distill", "rnnd_distill_workspace", "rnnd_logprob", "rnnd_logprob_workspace", "rnnd_adamw"):
            getattr(L, name).restype = c.c_int
        _lib = L
    return _lib


def rnnd_strerror(status: int) -> str:
    return load_library().rnnd_strerror(status).decode()


def rnnd_version() -> int:
    return load_library().rnnd_version()


def _check(rc: int):
    if rc != 0:
        raise RnndError(rc, rnnd_strerror(rc))


_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _data_args(X):
    torch = _torch()
    if not (X.is_cuda and X.dim() == 2 and X.is_contiguous()):
        raise ValueError("X must be a contiguous 2-D tensor in device memory")
    if X.dtype == torch.uint8:
        dt = RNND_U8
    elif X.dtype == torch.float32:
        dt = RNND_F32
    elif X.dtype == torch.float16:
        dt = RNND_F16
    elif X.dtype == torch.bfloat16:
        dt = RNND_BF16
    else:
        raise ValueError("X must be uint8, float32, float16 or bfloat16")
    return X.data_ptr(), X.shape[0], X.shape[1], dt


def _stream(stream):
    torch = _torch()
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


RNND_STATIC_SCRATCH_BYTES = 64 << 20


def rnnd_workspace_bytes(N: int, d: int, dtype: int, R: int, rounds: int) -> int:
    b = ctypes.c_size_t(0)
    _check(load_library().rnnd_workspace_bytes(N, d, dtype, R, rounds, ctypes.byref(b)))
    return b.value


def rnnd_release_workspace():
    _check(load_library().rnnd_release_workspace())


def rnnd_set_workspace_poison(on: bool):
    _check(load_library().rnnd_set_workspace_poison(1 if on else 0))


def rnnd_set_event_timing(on: bool):
    """Per-round times of the statistics from HIP events (True) or from the device clock (False, the default)."""
    _check(load_library().rnnd_set_event_timing(1 if on else 0))


def rnnd_build_static(X, S: int, R: int, T1: int, T2: int, seed: int, graph, degree, metric: int = RNND_L2SQ,
                      stream=None):
    """rnnd_build_static: the caller passes the outputs (graph [N, R] int32, degree [N] int32, on X's device);
    nothing is allocated, here or in the library."""
    ptr, N, d, dt = _data_args(X)
    assert graph.is_cuda and graph.is_contiguous() and graph.shape == (N, R) and graph.element_size() == 4
    assert degree.is_cuda and degree.is_contiguous() and degree.shape == (N,) and degree.element_size() == 4
    _check(load_library().rnnd_build_static(ptr, N, d, dt, metric, S, R, T1, T2, seed, graph.data_ptr(),
                                            degree.data_ptr(), _stream(stream)))


def rnnd_build(X, S: int, R: int, T1: int, T2: int, seed: int, metric: int = RNND_L2SQ, stream=None):
    """rnnd_build: returns (graph [N, R] int32, -1 padded; degree [N] int32), both on X's device."""
    torch = _torch()
    ptr, N, d, dt = _data_args(X)
    graph = torch.empty((N, R), dtype=torch.int32, device=X.device)
    degree = torch.empty((N,), dtype=torch.int32, device=X.device)
    _check(load_library().rnnd_build(ptr, N, d, dt, metric, S, R, T1, T2, seed, graph.data_ptr(),
                                     degree.data_ptr(), _stream(stream)))
    return graph, degree


def rnnd_build_ex(X, S: int, R: int, T1: int, T2: int, seed: int, metric: int = RNND_L2SQ, stream=None,
                  want_keys: bool = True):
    """rnnd_build_ex: returns (graph, degree, keys [N, R] int64-typed uint64 or None, Stats)."""
    torch = _torch()
    ptr, N, d, dt = _data_args(X)
    graph = torch.empty((N, R), dtype=torch.int32, device=X.device)
    degree = torch.empty((N,), dtype=torch.int32, device=X.device)
    keys = torch.empty((N, R), dtype=torch.int64, device=X.device) if want_keys else None
    st = Stats()
    _check(load_library().rnnd_build_ex(ptr, N, d, dt, metric, S, R, T1, T2, seed, graph.data_ptr(),
                                        degree.data_ptr(), keys.data_ptr() if want_keys else None,
                                        ctypes.byref(st), _stream(stream)))
    return graph, degree, keys, st


def rnnd_build_wide(X, S: int, R: int, M: int, T1: int, T2: int, seed: int, metric: int = RNND_L2SQ, stream=None,
                    want_keys: bool = True):
    """rnnd_build_wide: returns (graph [N, M], degree, keys [N, M] int64-typed uint64 or None, Stats)."""
    torch = _torch()
    ptr, N, d, dt = _data_args(X)
    graph = torch.empty((N, M), dtype=torch.int32, device=X.device)
    degree = torch.empty((N,), dtype=torch.int32, device=X.device)
    keys = torch.empty((N, M), dtype=torch.int64, device=X.device) if want_keys else None
    st = Stats()
    _check(load_library().rnnd_build_wide(ptr, N, d, dt, metric, S, R, M, T1, T2, seed, graph.data_ptr(),
                                          degree.data_ptr(), keys.data_ptr() if want_keys else None,
                                          ctypes.byref(st), _stream(stream)))
    return graph, degree, keys, st


def rnnd_build_blocks(X, S: int, R: int, T1: int, T2: int, seed: int, blocks: int, metric: int = RNND_L2SQ,
                      stream=None, want_keys: bool = True):
    """rnnd_build_blocks: returns (graph, degree, keys [N, R] int64-typed uint64 or None, Stats)."""
    torch = _torch()
    ptr, N, d, dt = _data_args(X)
    graph = torch.empty((N, R), dtype=torch.int32, device=X.device)
    degree = torch.empty((N,), dtype=torch.int32, device=X.device)
    keys = torch.empty((N, R), dtype=torch.int64, device=X.device) if want_keys else None
    st = Stats()
    _check(load_library().rnnd_build_blocks(ptr, N, d, dt, metric, S, R, T1, T2, seed, blocks, graph.data_ptr(),
                                            degree.data_ptr(), keys.data_ptr() if want_keys else None,
                                            ctypes.byref(st), _stream(stream)))
    return graph, degree, keys, st


def rnnd_random_graph(X, S: int, R: int, seed: int, metric: int = RNND_L2SQ, stream=None):
    torch = _torch()
    ptr, N, d, dt = _data_args(X)
    keys = torch.empty((N, R), dtype=torch.int64, device=X.device)
    deg = torch.empty((N,), dtype=torch.int32, device=X.device)
    _check(load_library().rnnd_random_graph(ptr, N, d, dt, metric, S, R, seed, keys.data_ptr(),
                                            deg.data_ptr(), _stream(stream)))
    return keys, deg


def rnnd_update_neighbors(X, keys, deg, R: int, n_rounds: int = 1, metric: int = RNND_L2SQ, stream=None):
    """In place on (keys, deg); returns Stats."""
    ptr, N, d, dt = _data_args(X)
    assert keys.is_cuda and keys.is_contiguous() and keys.shape == (N, R) and keys.element_size() == 8
    assert deg.is_cuda and deg.is_contiguous() and deg.shape == (N,) and deg.element_size() == 4
    st = Stats()
    _check(load_library().rnnd_update_neighbors(ptr, N, d, dt, metric, R, keys.data_ptr(), deg.data_ptr(),
                                                n_rounds, ctypes.byref(st), _stream(stream)))
    return st


def rnnd_update_neighbors_blocks(X, keys, deg, R: int, blocks: int, n_passes: int = 1, metric: int = RNND_L2SQ,
                                 stream=None):
    """In place on (keys, deg); returns Stats."""
    ptr, N, d, dt = _data_args(X)
    assert keys.is_cuda and keys.is_contiguous() and keys.shape == (N, R) and keys.element_size() == 8
    assert deg.is_cuda and deg.is_contiguous() and deg.shape == (N,) and deg.element_size() == 4
    st = Stats()
    _check(load_library().rnnd_update_neighbors_blocks(ptr, N, d, dt, metric, R, keys.data_ptr(), deg.data_ptr(),
                                                       n_passes, blocks, ctypes.byref(st), _stream(stream)))
    return st


def rnnd_probe_gather(X, n_gather: int, seed: int = 1, stream=None) -> float:
    """GB/s of random whole-row gathers from X (measurement aid)."""
    assert X.is_cuda and X.is_contiguous() and X.dim() == 2
    out = ctypes.c_double(0.0)
    _check(load_library().rnnd_probe_gather(X.data_ptr(), X.shape[0], X.shape[1] * X.element_size(), n_gather, seed,
                                            ctypes.byref(out), _stream(stream)))
    return out.value


def rnnd_probe_gather_map(X, n_gather: int, lanes_per_row: int, seed: int = 1, stream=None) -> float:
    """GB/s of random whole-row gathers from X with lanes_per_row lanes reading a row together."""
    assert X.is_cuda and X.is_contiguous() and X.dim() == 2
    out = ctypes.c_double(0.0)
    _check(load_library().rnnd_probe_gather_map(X.data_ptr(), X.shape[0], X.shape[1] * X.element_size(), n_gather,
                                                lanes_per_row, seed, ctypes.byref(out), _stream(stream)))
    return out.value


def rnnd_add_reverse_edges(keys, deg, R: int, stream=None):
    N = keys.shape[0]
    assert keys.is_cuda and keys.is_contiguous() and keys.shape == (N, R) and keys.element_size() == 8
    assert deg.is_cuda and deg.is_contiguous() and deg.shape == (N,) and deg.element_size() == 4
    _check(load_library().rnnd_add_reverse_edges(N, R, keys.data_ptr(), deg.data_ptr(), _stream(stream)))


def rnnd_add_reverse_edges_wide(keys, deg, R: int, stream=None):
    """Rows are keys.shape[1] >= R slots wide."""
    N, M = keys.shape
    assert keys.is_cuda and keys.is_contiguous() and keys.element_size() == 8
    assert deg.is_cuda and deg.is_contiguous() and deg.shape == (N,) and deg.element_size() == 4
    _check(load_library().rnnd_add_reverse_edges_wide(N, R, M, keys.data_ptr(), deg.data_ptr(), _stream(stream)))


def rnnd_export_graph(keys, deg, R: int, stream=None):
    torch = _torch()
    N = keys.shape[0]
    graph = torch.empty((N, R), dtype=torch.int32, device=keys.device)
    degree = torch.empty((N,), dtype=torch.int32, device=keys.device)
    _check(load_library().rnnd_export_graph(N, R, keys.data_ptr(), deg.data_ptr(), graph.data_ptr(),
                                            degree.data_ptr(), _stream(stream)))
    return graph, degree


def rnnd_search(X, graph, degree, Q, L: int, K: int, k: int, seed: int, want_dist: bool = False,
                metric: int = RNND_L2SQ, stream=None):
    """Alg. 1 with the cap K on the GPU.  Returns (ids int32 [nq, k], dist_bits int32 [nq, k] or None, evals)."""
    torch = _torch()
    ptr, N, d, dt = _data_args(X)
    assert Q.is_cuda and Q.is_contiguous() and Q.dtype == X.dtype and Q.dim() == 2 and Q.shape[1] == d
    assert graph.is_cuda and graph.is_contiguous() and graph.dtype == torch.int32 and graph.shape[0] == N
    assert degree.is_cuda and degree.is_contiguous() and degree.dtype == torch.int32 and degree.shape == (N,)
    nq = Q.shape[0]
    ids = torch.empty((nq, k), dtype=torch.int32, device=X.device)
    dist = torch.empty((nq, k), dtype=torch.int32, device=X.device) if want_dist else None
    ev = ctypes.c_int64(0)
    _check(load_library().rnnd_search(ptr, N, d, dt, metric, graph.data_ptr(), degree.data_ptr(), graph.shape[1],
                                      Q.data_ptr(), nq, L, K, k, seed, ids.data_ptr(),
                                      dist.data_ptr() if want_dist else None, ctypes.byref(ev), _stream(stream)))
    return ids, dist, ev.value


def rnnd_set_transpose_path(path: int):
    _check(load_library().rnnd_set_transpose_path(path))


def rnnd_set_scan_launches(mode: int):
    _check(load_library().rnnd_set_scan_launches(mode))


def rnnd_set_kernel_variant(variant: int):
    _check(load_library().rnnd_set_kernel_variant(variant))


# ---- training the rows of an index.  These calls only enqueue their work.  Outputs and workspaces are allocated on the stream
# the call runs on; inputs are marked as in use there if it is not the current one.  They record no history for automatic
# differentiation (the gradients are calls of their own), so tensors that ask for one are refused.
_FLOAT_TYPES = {}


def _row_type(t, what):
    if not _FLOAT_TYPES:
        torch = _torch()
        _FLOAT_TYPES.update({torch.float32: RNND_F32, torch.float16: RNND_F16, torch.bfloat16: RNND_BF16})
    try:
        return _FLOAT_TYPES[t]
    except KeyError:
        raise ValueError("%s must be float32, float16 or bfloat16, not %s" % (what, t)) from None


def _need(ok, message, *values):
    if not ok:
        raise ValueError(message % values)


def _no_history(**tensors):
    for what, x in tensors.items():
        if x is not None and x.requires_grad and _torch().is_grad_enabled():
            raise ValueError("%s requires a gradient, but this call records no history: pass %s.detach(), or call under torch.no_grad()"
                             % (what, what))


def _rows(x, what, d=None):
    _need(x.is_cuda and x.dim() == 2 and x.is_contiguous(), "%s must be a contiguous 2-D tensor in device memory", what)
    _need(d is None or x.shape[1] == d, "%s must have rows of %s coordinates", what, d)
    return _row_type(x.dtype, what)


def _vector(x, what, n, dtype, device):
    if x is None:
        return None
    if not (x.is_cuda and x.device == device and x.dim() == 1 and x.is_contiguous() and x.dtype == dtype and (n is None or x.shape[0] == n)):
        raise ValueError("%s must be a contiguous %s vector%s on the same device" % (what, dtype, "" if n is None else " of %d" % n))
    return x.data_ptr()


class _On:
    """The device and stream of a call, current while it allocates and enqueues."""

    def __init__(self, device, stream, used):
        torch = _torch()
        self.context = None
        if stream is None:
            self.handle = _raw_stream(device.index)
            if torch.cuda.current_device() != device.index:
                self.context = torch.cuda.device(device)
        else:
            _need(stream.device == device, "the stream is of another device than the tensors")
            self.handle = stream.cuda_stream
            self.context = torch.cuda.stream(stream)
            if stream != torch.cuda.current_stream(device):
                for x in used:
                    if x is not None:
                        x.record_stream(stream)

    def __enter__(self):
        if self.context is not None:
            self.context.__enter__()
        return self.handle

    def __exit__(self, *error):
        if self.context is not None:
            return self.context.__exit__(*error)
        return False


def _raw_stream(index):
    """The current stream's handle, without an object around it where torch has that (2 us of a lookup's 10)."""
    torch = _torch()
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(index) if raw is not None else torch.cuda.current_stream(index).cuda_stream


def _work(workspace, need, device):
    torch = _torch()
    if workspace is None:
        return torch.empty(need, dtype=torch.uint8, device=device)
    _need(workspace.is_cuda and workspace.device == device and workspace.is_contiguous(),
          "workspace must be a contiguous tensor on the same device")
    return workspace


def rnnd_embed(table, ids, scale: float = 1.0, out_dtype=None, out=None, stream=None):
    """rnnd_embed: returns scale * table[ids] ([n, d], of table's type or out_dtype); rows of zeros for ids outside the table.
    Its gradient is rnnd_embed_grad; a table that requires gradients is refused outside torch.no_grad()."""
    torch = _torch()
    _no_history(table=table, out=out)
    dt, device = _rows(table, "table"), table.device
    n, (V, d) = ids.shape[0] if ids.dim() == 1 else -1, table.shape
    pi = _vector(ids, "ids", None, torch.int32, device)
    if out is not None:
        _need(out_dtype is None or out_dtype == out.dtype, "out_dtype is not that of out")
        _need(_rows(out, "out", d) is not None and out.shape[0] == n and out.device == device, "out must be [n, d] on the same device")
    with _On(device, stream, (table, ids, out)) as st:
        if out is None:
            out = torch.empty((n, d), dtype=out_dtype or table.dtype, device=device)
        _check(load_library().rnnd_embed(table.data_ptr(), V, d, dt, pi, n, scale, out.data_ptr(), _row_type(out.dtype, "out"), st))
    return out


def rnnd_embed_grad_workspace(n: int, d: int, V: int) -> int:
    b = ctypes.c_size_t(0)
    _check(load_library().rnnd_embed_grad_workspace(n, d, V, ctypes.byref(b)))
    return b.value


def rnnd_embed_grad(dout, ids, V: int, scale: float = 1.0, grad_dtype=None, grad=None, accumulate: bool = False,
                    workspace=None, stream=None):
    """rnnd_embed_grad: returns the gradient of the table ([V, d], float32 or grad_dtype).  grad: where to put it, or
    (accumulate) what to add it to."""
    torch = _torch()
    _no_history(dout=dout, grad=grad)
    dt, device = _rows(dout, "dout"), dout.device
    n, d = dout.shape
    pi = _vector(ids, "ids", n, torch.int32, device)
    _need(grad is not None or not accumulate, "accumulate needs the gradient to add to")
    if grad is not None:
        _need(grad_dtype is None or grad_dtype == grad.dtype, "grad_dtype is not that of grad")
        _need(_rows(grad, "grad", d) is not None and grad.shape[0] == V and grad.device == device, "grad must be [V, d] on the same device")
    need = rnnd_embed_grad_workspace(n, d, V)
    with _On(device, stream, (dout, ids, grad, workspace)) as st:
        if grad is None:
            grad = torch.empty((V, d), dtype=grad_dtype or torch.float32, device=device)
        w = _work(workspace, need, device)
        _check(load_library().rnnd_embed_grad(dout.data_ptr(), dt, pi, n, d, scale, V, grad.data_ptr(), _row_type(grad.dtype, "grad"),
                                              1 if accumulate else 0, w.data_ptr(), w.numel() * w.element_size(), st))
    return grad


def rnnd_contrast_workspace(B: int, M: int, d: int, dtype: int, want_grad: bool = True) -> int:
    b = ctypes.c_size_t(0)
    _check(load_library().rnnd_contrast_workspace(B, M, d, dtype, 1 if want_grad else 0, ctypes.byref(b)))
    return b.value


def rnnd_contrast(Q, K, target, scale: float, query_ids=None, key_ids=None, key_bias=None, row_weight=None,
                  want_grad: bool = True, metric: int = RNND_L2SQ, workspace=None, stream=None):
    """rnnd_contrast: returns (loss [B] float32, dQ, dK), the gradients None without want_grad.
    Inputs that require gradients are refused outside torch.no_grad(): dQ and dK are what there is."""
    torch = _torch()
    _no_history(Q=Q, K=K, key_bias=key_bias, row_weight=row_weight)
    dt, device = _rows(K, "K"), K.device
    M, d = K.shape
    _need(_rows(Q, "Q", d) == dt and Q.device == device, "Q and K must be of one type and on one device")
    B = Q.shape[0]
    pt = _vector(target, "target", B, torch.int32, device)
    pq = _vector(query_ids, "query_ids", B, torch.int32, device)
    pk = _vector(key_ids, "key_ids", M, torch.int32, device)
    pb = _vector(key_bias, "key_bias", M, torch.float32, device)
    pw = _vector(row_weight, "row_weight", B, torch.float32, device)
    need = rnnd_contrast_workspace(B, M, d, dt, want_grad)
    with _On(device, stream, (Q, K, target, query_ids, key_ids, key_bias, row_weight, workspace)) as st:
        loss = torch.empty(B, dtype=torch.float32, device=device)
        dQ, dK = (torch.empty_like(Q), torch.empty_like(K)) if want_grad else (None, None)
        w = _work(workspace, need, device)
        _check(load_library().rnnd_contrast(Q.data_ptr(), B, K.data_ptr(), M, d, dt, metric, pt, pq, pk, pb, pw, scale,
                                            loss.data_ptr(), dQ.data_ptr() if want_grad else None,
                                            dK.data_ptr() if want_grad else None, w.data_ptr(), w.numel() * w.element_size(), st))
    return loss, dQ, dK


def rnnd_distill_workspace(B: int, M: int, d: int, dtype: int, entries: int, want_grad: bool = True) -> int:
    b = ctypes.c_size_t(0)
    _check(load_library().rnnd_distill_workspace(B, M, d, dtype, entries, 1 if want_grad else 0, ctypes.byref(b)))
    return b.value


def rnnd_distill(Q, K, teacher_ids, teacher_logits, scale: float, tail: bool = False, query_ids=None, key_ids=None, key_bias=None,
                 row_weight=None, want_grad: bool = True, metric: int = RNND_L2SQ, workspace=None, stream=None):
    """rnnd_distill: returns (loss [B] float32, dQ, dK), the gradients None without want_grad.  teacher_ids (int32) and teacher_logits
    (float32) are [B, entries], as rnnd_logprob of the teacher returns them (tail=True) or any scores of candidates.
    Inputs that require gradients are refused outside torch.no_grad(): dQ and dK are what there is."""
    torch = _torch()
    _no_history(Q=Q, K=K, teacher_logits=teacher_logits, key_bias=key_bias, row_weight=row_weight)
    dt, device = _rows(K, "K"), K.device
    M, d = K.shape
    _need(_rows(Q, "Q", d) == dt and Q.device == device, "Q and K must be of one type and on one device")
    B = Q.shape[0]
    _need(teacher_ids.dim() == 2 and teacher_ids.shape[0] == B and teacher_logits.shape == teacher_ids.shape,
          "teacher_ids and teacher_logits must both be [%s, entries]", B)
    entries = teacher_ids.shape[1]
    for what, x, t in (("teacher_ids", teacher_ids, torch.int32), ("teacher_logits", teacher_logits, torch.float32)):
        _need(x.is_cuda and x.device == device and x.is_contiguous() and x.dtype == t, "%s must be a contiguous %s tensor on the same device", what, t)
    pq = _vector(query_ids, "query_ids", B, torch.int32, device)
    pk = _vector(key_ids, "key_ids", M, torch.int32, device)
    pb = _vector(key_bias, "key_bias", M, torch.float32, device)
    pw = _vector(row_weight, "row_weight", B, torch.float32, device)
    need = rnnd_distill_workspace(B, M, d, dt, entries, want_grad)
    with _On(device, stream, (Q, K, teacher_ids, teacher_logits, query_ids, key_ids, key_bias, row_weight, workspace)) as st:
        loss = torch.empty(B, dtype=torch.float32, device=device)
        dQ, dK = (torch.empty_like(Q), torch.empty_like(K)) if want_grad else (None, None)
        w = _work(workspace, need, device)
        _check(load_library().rnnd_distill(Q.data_ptr(), B, K.data_ptr(), M, d, dt, metric, teacher_ids.data_ptr(), teacher_logits.data_ptr(),
                                           entries, 1 if tail else 0, pq, pk, pb, pw, scale, loss.data_ptr(),
                                           dQ.data_ptr() if want_grad else None, dK.data_ptr() if want_grad else None,
                                           w.data_ptr(), w.numel() * w.element_size(), st))
    return loss, dQ, dK


def rnnd_logprob_workspace(B: int, M: int, d: int, dtype: int, alternatives: int = 0) -> int:
    b = ctypes.c_size_t(0)
    _check(load_library().rnnd_logprob_workspace(B, M, d, dtype, alternatives, ctypes.byref(b)))
    return b.value


def rnnd_logprob(Q, K, scale: float, target=None, alternatives: int = 0, query_ids=None, key_ids=None, key_bias=None,
                 metric: int = RNND_L2SQ, workspace=None, stream=None):
    """rnnd_logprob: returns (logprob [B] of the targets or None, entropy [B], top_ids int32 [B, alternatives], top_logprob
    [B, alternatives]), the last two None without alternatives.
    Inputs that require gradients are refused outside torch.no_grad(): the call records no history (rnnd_contrast has the gradients)."""
    torch = _torch()
    _no_history(Q=Q, K=K, key_bias=key_bias)
    dt, device = _rows(K, "K"), K.device
    M, d = K.shape
    _need(_rows(Q, "Q", d) == dt and Q.device == device, "Q and K must be of one type and on one device")
    B = Q.shape[0]
    pt = _vector(target, "target", B, torch.int32, device)
    pq = _vector(query_ids, "query_ids", B, torch.int32, device)
    pk = _vector(key_ids, "key_ids", M, torch.int32, device)
    pb = _vector(key_bias, "key_bias", M, torch.float32, device)
    need = rnnd_logprob_workspace(B, M, d, dt, alternatives)
    with _On(device, stream, (Q, K, target, query_ids, key_ids, key_bias, workspace)) as st:
        logprob = torch.empty(B, dtype=torch.float32, device=device) if target is not None else None
        entropy = torch.empty(B, dtype=torch.float32, device=device)
        ids = torch.empty((B, alternatives), dtype=torch.int32, device=device) if alternatives else None
        top = torch.empty((B, alternatives), dtype=torch.float32, device=device) if alternatives else None
        w = _work(workspace, need, device)
        _check(load_library().rnnd_logprob(Q.data_ptr(), B, K.data_ptr(), M, d, dt, metric, pt, pq, pk, pb, scale, alternatives,
                                           None if logprob is None else logprob.data_ptr(), entropy.data_ptr(),
                                           None if ids is None else ids.data_ptr(), None if top is None else top.data_ptr(),
                                           w.data_ptr(), w.numel() * w.element_size(), st))
    return logprob, entropy, ids, top


_ADAMW_KEYS = {"param", "grad", "m", "v", "m_scale", "v_scale", "copy", "counter"}


class AdamwTensors:
    """The tensors of an AdamW step, described once.  Each is a dict of 1-D views or whole contiguous tensors:
    param (float32), grad, m, v (float32, or one byte an element for 8-bit states with m_scale and v_scale, one
    byte per 128 elements), copy (float16 or bfloat16, optional) and counter (8 bits; by default the tensors' own elements,
    counted through, each starting at a multiple of 128).  The descriptors hold the tensors' addresses, and this object keeps the tensors: a program
    writes its gradients into the same tensors every step (rnnd_embed_grad's grad=); for gradients in new tensors it is made anew."""

    def __init__(self, tensors):
        torch = _torch()
        self.kept = [dict(t) for t in tensors]         # the descriptors hold addresses
        self.array = (AdamwTensor * max(1, len(self.kept)))()
        self.device, at = None, 0
        names = ("param", "grad", "m", "v", "m_scale", "v_scale", "copy")
        for i, t in enumerate(self.kept):
            if not t.keys() <= _ADAMW_KEYS:
                raise ValueError("tensor %d: unknown %s" % (i, sorted(t.keys() - _ADAMW_KEYS)))
            p, g, m, v = t["param"], t["grad"], t["m"], t["v"]
            ms, vs, copy = t.get("m_scale"), t.get("v_scale"), t.get("copy")
            n, eight = p.numel(), m.element_size() == 1
            if self.device is None:
                self.device, index = p.device, p.get_device()
            blocks = -(-n // 128)
            for name, x, count in zip(names, (p, g, m, v, ms, vs, copy), (n, n, n, n, blocks, blocks, n)):
                if x is not None and not (x.get_device() == index >= 0 and x.numel() == count and x.is_contiguous()):
                    raise ValueError("tensor %d: %s must be %d contiguous elements on one device" % (i, name, count))
            if p.dtype != torch.float32:
                raise ValueError("tensor %d: param must be float32" % i)
            if v.dtype != m.dtype or not (eight or m.dtype == torch.float32):
                raise ValueError("tensor %d: m and v must both be float32 or both bytes" % i)
            if (ms is None) == eight or (vs is None) == eight or (eight and ms.element_size() + vs.element_size() != 2):
                raise ValueError("tensor %d: 8-bit states need m_scale and v_scale of bytes, 32-bit states have none" % i)
            a = self.array[i]
            a.param, a.grad, a.m, a.v, a.n = p.data_ptr(), g.data_ptr(), m.data_ptr(), v.data_ptr(), n
            if eight:
                a.m_scale, a.v_scale = ms.data_ptr(), vs.data_ptr()
            a.grad_dtype, a.state_bits = _row_type(g.dtype, "grad"), 8 if eight else 32
            if copy is not None:
                a.copy, a.copy_dtype = copy.data_ptr(), _row_type(copy.dtype, "copy")
                if a.copy_dtype == RNND_F32:
                    raise ValueError("tensor %d: copy must be float16 or bfloat16" % i)
            a.counter = t.get("counter", at)
            at += -(-n // 128) * 128


def rnnd_adamw(tensors, step: int, lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
               weight_decay: float = 0.0, grad_scale: float = 1.0, seed: int = 0, stream=None):
    """rnnd_adamw on an AdamwTensors, in place."""
    if not tensors.kept:
        return
    used = ()
    if stream is not None:
        used = [x for t in tensors.kept for x in t.values() if hasattr(x, "record_stream")]
    with _On(tensors.device, stream, used) as st:
        _check(load_library().rnnd_adamw(tensors.array, len(tensors.kept), step, lr, beta1, beta2, eps, weight_decay, grad_scale,
                                         seed, st))


# ---- snapshot format helpers (host side, numpy): layout conversion only
def pack_keys(ids, dist_bits, flags, deg):
    """(ids int32 [N,R], dist_bits uint32 [N,R], flags uint8 [N,R], deg) -> uint64 keys [N,R]."""
    import numpy as np
    k = (dist_bits.astype(np.uint64) << np.uint64(32)) | \
        ((ids.astype(np.int64) & 0x7FFFFFFF).astype(np.uint64) << np.uint64(1)) | \
        (flags.astype(np.uint64) & np.uint64(1))
    pad = np.arange(ids.shape[1])[None, :] >= np.asarray(deg)[:, None]
    k[pad] = np.uint64(0xFFFFFFFFFFFFFFFF)
    return k


def unpack_keys(keys, deg):
    """uint64 keys [N,R] -> (ids int32 (-1 padded), dist_bits uint32, flags uint8)."""
    import numpy as np
    keys = keys.view(np.uint64) if keys.dtype != np.uint64 else keys
    ids = ((keys >> np.uint64(1)) & np.uint64(0x7FFFFFFF)).astype(np.int32)
    dist_bits = (keys >> np.uint64(32)).astype(np.uint32)
    flags = (keys & np.uint64(1)).astype(np.uint8)
    pad = np.arange(keys.shape[1])[None, :] >= np.asarray(deg)[:, None]
    ids[pad] = -1
    dist_bits[pad] = 0
    flags[pad] = 0
    return ids, dist_bits, flags
