"""Thin ctypes binding of liblaser_route.so (the C ABI in include/laser.h).

Argument marshalling only: torch supplies device memory and the stream; every
step of the routing path runs in the library's HIP kernels.  There is no CPU
fallback: if the library has not been built, importing the binding raises.
"""
from __future__ import annotations

import contextlib
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblaser_route.so")

DTYPE_F32 = 0
DTYPE_BF16 = 1
TRIM_TOP = 0
TRIM_RANDOM = 1

# include/laser.h
EXPORTS = ("laser_workspace_bytes", "laser_route", "laser_route_batched", "laser_route_stats",
           "laser_route_from_logits", "laser_imbalance", "laser_percentiles", "laser_summary_f32",
           "laser_strerror", "laser_status", "laser_static_workspace_bytes", "laser_route_static",
           "laser_status_static", "laser_experts_up", "laser_experts_workspace_bytes", "laser_experts_down",
           "laser_project_workspace_bytes", "laser_project_adapted")
# include/laser_bench.h
BENCH_EXPORTS = ("laser_bench_timer_create", "laser_bench_timer_destroy", "laser_bench_route",
                 "laser_bench_timer_read", "laser_bench_event_overhead", "laser_bench_plain_read")

STATUS_COMPLETE = 0
STATUS_TIMEOUT = 1
STATUS_INCONSISTENT = 2


class LaserParams(ctypes.Structure):
    _fields_ = [
        ("struct_bytes", ctypes.c_uint32),
        ("k", ctypes.c_int32),
        ("c", ctypes.c_int32),
        ("eps_high", ctypes.c_float),
        ("t_fix", ctypes.c_float),
        ("trim_mode", ctypes.c_int32),
        ("renormalize", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("seed", ctypes.c_uint64),
        ("token_offset", ctypes.c_uint64),
        ("stream", ctypes.c_uint32),
        ("poll_budget", ctypes.c_uint32),
        ("pipeline_tiles", ctypes.c_uint32),
        ("split_k", ctypes.c_uint32),
    ]


class LaserExpertsParams(ctypes.Structure):
    _fields_ = [
        ("struct_bytes", ctypes.c_uint32),
        ("k", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("first_expert", ctypes.c_int32),
    ]


class LaserAdapterParams(ctypes.Structure):
    _fields_ = [
        ("struct_bytes", ctypes.c_uint32),
        ("rank", ctypes.c_int32),
        ("adapters", ctypes.c_int32),
        ("requests", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("out_dtype", ctypes.c_int32),
    ]


class LaserError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"laser: {text} (code {code})")
        self.code = code


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it first (python -m paper_2510_03293_amd.build "
            "or __graft_entry__.build()); there is no fallback path")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    pp = ctypes.POINTER(LaserParams)
    lib.laser_workspace_bytes.argtypes = [i32, i32, i32, pp]
    lib.laser_workspace_bytes.restype = sz
    lib.laser_route.argtypes = [vp, vp, i32, i32, i32, pp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.laser_route.restype = ctypes.c_int
    lib.laser_route_batched.argtypes = [vp, vp, i32, i32, i32, i32, pp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.laser_route_batched.restype = ctypes.c_int
    lib.laser_route_stats.argtypes = [vp, vp, i32, i32, i32, pp, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                      vp, sz, vp]
    lib.laser_route_stats.restype = ctypes.c_int
    lib.laser_imbalance.argtypes = [vp, i32, i32, vp, i32, vp, vp, vp, vp, vp, vp]
    lib.laser_imbalance.restype = ctypes.c_int
    lib.laser_percentiles.argtypes = [vp, i32, ctypes.POINTER(ctypes.c_double), i32, vp, vp]
    lib.laser_percentiles.restype = ctypes.c_int
    lib.laser_summary_f32.argtypes = [vp, i32, ctypes.POINTER(ctypes.c_double), i32, vp, vp, vp]
    lib.laser_summary_f32.restype = ctypes.c_int
    lib.laser_route_from_logits.argtypes = [vp, i32, i32, pp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.laser_route_from_logits.restype = ctypes.c_int
    lib.laser_strerror.argtypes = [ctypes.c_int]
    lib.laser_strerror.restype = ctypes.c_char_p
    lib.laser_status.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_int32)]
    lib.laser_status.restype = ctypes.c_int
    lib.laser_static_workspace_bytes.argtypes = []
    lib.laser_static_workspace_bytes.restype = sz
    lib.laser_route_static.argtypes = [vp, vp, i32, i32, i32, pp, vp, vp, vp, vp, vp, vp, vp]
    lib.laser_route_static.restype = ctypes.c_int
    lib.laser_status_static.argtypes = [vp, ctypes.POINTER(ctypes.c_int32)]
    lib.laser_status_static.restype = ctypes.c_int
    ep, ap = ctypes.POINTER(LaserExpertsParams), ctypes.POINTER(LaserAdapterParams)
    lib.laser_experts_up.argtypes = [vp, vp, i32, i32, i32, i32, ep, vp, vp, vp, vp]
    lib.laser_experts_up.restype = ctypes.c_int
    lib.laser_experts_workspace_bytes.argtypes = [i32, i32, i32, i32, ep]
    lib.laser_experts_workspace_bytes.restype = sz
    lib.laser_experts_down.argtypes = [vp, vp, i32, i32, i32, i32, ep, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.laser_experts_down.restype = ctypes.c_int
    lib.laser_project_workspace_bytes.argtypes = [i32, i32, i32, ap]
    lib.laser_project_workspace_bytes.restype = sz
    lib.laser_project_adapted.argtypes = [vp, vp, i32, i32, i32, ap, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.laser_project_adapted.restype = ctypes.c_int
    lib.laser_bench_timer_create.argtypes = [i32, ctypes.POINTER(vp)]
    lib.laser_bench_timer_create.restype = ctypes.c_int
    lib.laser_bench_timer_destroy.argtypes = [vp]
    lib.laser_bench_timer_destroy.restype = None
    lib.laser_bench_route.argtypes = [vp] + lib.laser_route.argtypes
    lib.laser_bench_route.restype = ctypes.c_int
    lib.laser_bench_timer_read.argtypes = [vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double),
                                           ctypes.c_int64, ctypes.POINTER(ctypes.c_int64)]
    lib.laser_bench_timer_read.restype = ctypes.c_int
    lib.laser_bench_event_overhead.argtypes = [vp, ctypes.POINTER(ctypes.c_double)]
    lib.laser_bench_event_overhead.restype = ctypes.c_int
    lib.laser_bench_plain_read.argtypes = [vp, sz, sz, vp, vp, ctypes.POINTER(ctypes.c_double),
                                           ctypes.POINTER(ctypes.c_int64)]
    lib.laser_bench_plain_read.restype = ctypes.c_int
    return lib


_lib = _load()


def make_params(k: int, c: int, eps_high: float, t_fix: float, dtype: int = DTYPE_BF16,
                renormalize: bool = True, trim_mode: int = TRIM_TOP, seed: int = 0,
                stream: int = 0, token_offset: int = 0, poll_budget: int = 0,
                pipeline_tiles: int = 0, split_k: int = 0) -> LaserParams:
    return LaserParams(ctypes.sizeof(LaserParams), k, c, eps_high, t_fix, trim_mode,
                       1 if renormalize else 0, dtype, seed, token_offset, stream, poll_budget,
                       pipeline_tiles, split_k)


def laser_strerror(code: int) -> str:
    return _lib.laser_strerror(code).decode()


def _check(code: int) -> None:
    if code != 0:
        raise LaserError(code, laser_strerror(code))


def laser_workspace_bytes(T: int, H: int, E: int, params: LaserParams) -> int:
    return int(_lib.laser_workspace_bytes(T, H, E, ctypes.byref(params)))


def _ptr(t: torch.Tensor | None):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


# The current stream's handle without a Stream object around it, where torch offers that (of a call's
# 8 us on the host the object takes 3).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_handle(stream) -> ctypes.c_void_p:
    if stream is None and _raw_stream is not None:
        return ctypes.c_void_p(_raw_stream(torch.cuda.current_device()))
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def laser_route(hidden, w_gate, T, H, E, params, loads_inout, expert_ids, weights,
                permutation, expert_offsets, logits_out, workspace, stream=None) -> None:
    """Enqueue one layer's routing step; tensors are device tensors (see laser.h)."""
    _check(_lib.laser_route(_ptr(hidden), _ptr(w_gate), T, H, E, ctypes.byref(params),
                            _ptr(loads_inout), _ptr(expert_ids), _ptr(weights), _ptr(permutation),
                            _ptr(expert_offsets), _ptr(logits_out), _ptr(workspace),
                            workspace.numel() * workspace.element_size(), _stream_handle(stream)))


def laser_route_batched(hidden, w_gate, B, T, H, E, params, loads_inout, expert_ids, weights,
                        permutation, expert_offsets, logits_out, workspace, stream=None) -> None:
    """B independent problems of one size in one call; every tensor has a leading dimension B."""
    _check(_lib.laser_route_batched(_ptr(hidden), _ptr(w_gate), B, T, H, E, ctypes.byref(params),
                                    _ptr(loads_inout), _ptr(expert_ids), _ptr(weights),
                                    _ptr(permutation), _ptr(expert_offsets), _ptr(logits_out),
                                    _ptr(workspace),
                                    0 if workspace is None else workspace.numel() * workspace.element_size(),
                                    _stream_handle(stream)))


def laser_route_stats(hidden, w_gate, T, H, E, params, loads_inout, expert_ids, weights,
                      permutation, expert_offsets, logits_out, topk_mass, entropy, pool_size,
                      workspace, stream=None) -> None:
    """laser_route plus per-token top-k mass, entropy and pool size (each may be None)."""
    _check(_lib.laser_route_stats(_ptr(hidden), _ptr(w_gate), T, H, E, ctypes.byref(params),
                                  _ptr(loads_inout), _ptr(expert_ids), _ptr(weights),
                                  _ptr(permutation), _ptr(expert_offsets), _ptr(logits_out),
                                  _ptr(topk_mass), _ptr(entropy), _ptr(pool_size), _ptr(workspace),
                                  workspace.numel() * workspace.element_size(),
                                  _stream_handle(stream)))


def laser_route_from_logits(logits, T, E, params, loads_inout, expert_ids, weights,
                            permutation, expert_offsets, workspace, stream=None) -> None:
    _check(_lib.laser_route_from_logits(_ptr(logits), T, E, ctypes.byref(params),
                                        _ptr(loads_inout), _ptr(expert_ids), _ptr(weights),
                                        _ptr(permutation), _ptr(expert_offsets), _ptr(workspace),
                                        workspace.numel() * workspace.element_size(),
                                        _stream_handle(stream)))


def laser_imbalance(counts, placement=None, layer_weights=None, stream=None):
    """Imbalance metrics of device counts [L,E] (int32): dict of device fp64 tensors."""
    L, E = counts.shape
    G = 0 if placement is None else placement.shape[0]
    dev = counts.device
    out = {"I": torch.empty(L, dtype=torch.float64, device=dev),
           "MV": torch.empty(L, dtype=torch.float64, device=dev),
           "I_gpu": torch.empty(L, dtype=torch.float64, device=dev),
           "agg": torch.empty(2, dtype=torch.float64, device=dev)}
    _check(_lib.laser_imbalance(_ptr(counts), L, E, _ptr(placement), G, _ptr(layer_weights),
                                _ptr(out["I"]), _ptr(out["MV"]), _ptr(out["I_gpu"]),
                                _ptr(out["agg"]), _stream_handle(stream)))
    return out


def laser_percentiles(values, q, stream=None):
    """q-th percentiles (host sequence, each in [0, 100]) of a device fp64 vector; device fp64 [len(q)]."""
    qs = [float(x) for x in q]
    qa = (ctypes.c_double * max(len(qs), 1))(*qs)
    out = torch.empty(len(qs), dtype=torch.float64, device=values.device)
    _check(_lib.laser_percentiles(_ptr(values), values.numel(), qa, len(qs), _ptr(out),
                                  _stream_handle(stream)))
    return out


def laser_summary_f32(values, q, stream=None):
    """(mean, percentiles) of a device fp32 vector: device fp64 scalar and fp64 [len(q)]."""
    qs = [float(x) for x in q]
    qa = (ctypes.c_double * max(len(qs), 1))(*qs)
    mean = torch.empty((), dtype=torch.float64, device=values.device)
    out = torch.empty(len(qs), dtype=torch.float64, device=values.device)
    _check(_lib.laser_summary_f32(_ptr(values), values.numel(), qa, len(qs), _ptr(mean), _ptr(out),
                                  _stream_handle(stream)))
    return mean, out


def laser_status(workspace, stream=None) -> int:
    """STATUS_* of the last call that used `workspace` (waits for the stream)."""
    st = ctypes.c_int32(-1)
    _check(_lib.laser_status(_ptr(workspace), _stream_handle(stream), ctypes.byref(st)))
    return st.value


def laser_static_workspace_bytes() -> int:
    return int(_lib.laser_static_workspace_bytes())


def laser_route_static(hidden, w_gate, T, H, E, params, loads_inout, expert_ids, weights,
                       permutation, expert_offsets, logits_out, stream=None) -> None:
    """laser_route on the library's own per-GPU workspace (nothing is allocated)."""
    _check(_lib.laser_route_static(_ptr(hidden), _ptr(w_gate), T, H, E, ctypes.byref(params),
                                   _ptr(loads_inout), _ptr(expert_ids), _ptr(weights), _ptr(permutation),
                                   _ptr(expert_offsets), _ptr(logits_out), _stream_handle(stream)))


def laser_status_static(stream=None) -> int:
    st = ctypes.c_int32(-1)
    _check(_lib.laser_status_static(_stream_handle(stream), ctypes.byref(st)))
    return st.value


def make_experts_params(k: int, dtype: int = DTYPE_BF16, first_expert: int = 0) -> LaserExpertsParams:
    return LaserExpertsParams(ctypes.sizeof(LaserExpertsParams), k, dtype, first_expert)


def make_adapter_params(rank: int, adapters: int, requests: int, dtype: int = DTYPE_BF16,
                        out_dtype: int | None = None) -> LaserAdapterParams:
    return LaserAdapterParams(ctypes.sizeof(LaserAdapterParams), rank, adapters, requests, dtype,
                              dtype if out_dtype is None else out_dtype)


def laser_experts_up(hidden, w_up, T, H, F, E, params, permutation, expert_offsets, act, stream=None) -> None:
    """Enqueue the experts' first product and activation over the dispatch tables (see laser.h)."""
    _check(_lib.laser_experts_up(_ptr(hidden), _ptr(w_up), T, H, F, E, ctypes.byref(params),
                                 _ptr(permutation), _ptr(expert_offsets), _ptr(act), _stream_handle(stream)))


def laser_experts_workspace_bytes(T: int, H: int, F: int, E: int, params: LaserExpertsParams) -> int:
    return int(_lib.laser_experts_workspace_bytes(T, H, F, E, ctypes.byref(params)))


def laser_experts_down(act, w_down, T, H, F, E, params, permutation, expert_offsets, expert_ids, weights,
                       base, out, workspace, stream=None) -> None:
    """Enqueue the experts' second product, weighted and summed back into token order."""
    _check(_lib.laser_experts_down(_ptr(act), _ptr(w_down), T, H, F, E, ctypes.byref(params),
                                   _ptr(permutation), _ptr(expert_offsets), _ptr(expert_ids), _ptr(weights),
                                   _ptr(base), _ptr(out), _ptr(workspace),
                                   workspace.numel() * workspace.element_size(), _stream_handle(stream)))


def laser_project_workspace_bytes(T: int, H: int, N: int, params: LaserAdapterParams) -> int:
    return int(_lib.laser_project_workspace_bytes(T, H, N, ctypes.byref(params)))


def laser_project_adapted(x, w, T, H, N, params, a_down, a_up, scales, request_offsets, request_adapters,
                          out, workspace, stream=None) -> None:
    """Enqueue a shared projection with the adapters of the batch's requests beside it."""
    _check(_lib.laser_project_adapted(_ptr(x), _ptr(w), T, H, N, ctypes.byref(params), _ptr(a_down), _ptr(a_up),
                                      _ptr(scales), _ptr(request_offsets), _ptr(request_adapters), _ptr(out),
                                      _ptr(workspace), workspace.numel() * workspace.element_size(),
                                      _stream_handle(stream)))


class BenchTimer:
    """Event pool of include/laser_bench.h: times the stages of laser_bench_route calls."""

    def __init__(self, max_calls: int):
        self.capacity = max_calls
        self._h = ctypes.c_void_p()
        _check(_lib.laser_bench_timer_create(max_calls, ctypes.byref(self._h)))

    def route(self, hidden, w_gate, T, H, E, params, loads_inout, expert_ids, weights, permutation,
              expert_offsets, logits_out, workspace, stream=None) -> None:
        _check(_lib.laser_bench_route(self._h, _ptr(hidden), _ptr(w_gate), T, H, E, ctypes.byref(params),
                                      _ptr(loads_inout), _ptr(expert_ids), _ptr(weights),
                                      _ptr(permutation), _ptr(expert_offsets), _ptr(logits_out),
                                      _ptr(workspace), workspace.numel() * workspace.element_size(),
                                      _stream_handle(stream)))

    def read(self):
        """(first_ms, tail_ms): per timed call, projection + analysis and tail kernel (lists)."""
        a = (ctypes.c_double * self.capacity)()
        b = (ctypes.c_double * self.capacity)()
        n = ctypes.c_int64(0)
        _check(_lib.laser_bench_timer_read(self._h, a, b, self.capacity, ctypes.byref(n)))
        return list(a[:n.value]), list(b[:n.value])

    def close(self) -> None:
        if self._h:
            _lib.laser_bench_timer_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def laser_bench_event_overhead(stream=None) -> float:
    """Milliseconds a HIP event pair adds to the kernel it brackets (measured now)."""
    ms = ctypes.c_double(0.0)
    _check(_lib.laser_bench_event_overhead(_stream_handle(stream), ctypes.byref(ms)))
    return ms.value


def laser_bench_plain_read(buf, bytes_per_launch: int, sink, stream=None):
    """(milliseconds, launches) of a plain streaming read of `buf` in pieces."""
    ms = ctypes.c_double(0.0)
    n = ctypes.c_int64(0)
    nbytes = buf.numel() * buf.element_size()
    _check(_lib.laser_bench_plain_read(
        ctypes.c_void_p(buf.data_ptr()), ctypes.c_size_t(nbytes), ctypes.c_size_t(bytes_per_launch),
        ctypes.c_void_p(sink.data_ptr()), _stream_handle(stream), ctypes.byref(ms), ctypes.byref(n)))
    return ms.value, n.value


class RouteBuffers:
    """Output and workspace tensors for calls of one size, allocated once."""

    def __init__(self, T: int, H: int, E: int, params: LaserParams, device="cuda",
                 want_logits: bool = False):
        self.T, self.H, self.E, self.k = T, H, E, params.k
        nbytes = laser_workspace_bytes(T, H, E, params)
        if nbytes == 0:
            raise LaserError(-2, "laser_workspace_bytes rejected the arguments")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.expert_ids = torch.empty((T, params.k), dtype=torch.int32, device=device)
        self.weights = torch.empty((T, params.k), dtype=torch.float32, device=device)
        self.permutation = torch.empty(T * params.k, dtype=torch.int32, device=device)
        self.expert_offsets = torch.empty(E + 1, dtype=torch.int32, device=device)
        self.logits = torch.empty((T, E), dtype=torch.float32, device=device) if want_logits else None


def route(hidden, w_gate, params: LaserParams, loads_inout, buffers: RouteBuffers | None = None,
          want_logits: bool = False, stream=None) -> RouteBuffers:
    """Convenience wrapper: shapes from the tensors, buffers allocated if not given."""
    T, H = hidden.shape
    E = w_gate.shape[0]
    if buffers is None:
        buffers = RouteBuffers(T, H, E, params, device=hidden.device, want_logits=want_logits)
    laser_route(hidden, w_gate, T, H, E, params, loads_inout, buffers.expert_ids, buffers.weights,
                buffers.permutation, buffers.expert_offsets, buffers.logits, buffers.workspace,
                stream)
    return buffers


def route_from_logits(logits, params: LaserParams, loads_inout,
                      buffers: RouteBuffers | None = None, stream=None) -> RouteBuffers:
    T, E = logits.shape
    if buffers is None:
        buffers = RouteBuffers(T, 0, E, params, device=logits.device)
    laser_route_from_logits(logits, T, E, params, loads_inout, buffers.expert_ids, buffers.weights,
                            buffers.permutation, buffers.expert_offsets, buffers.workspace, stream)
    return buffers


_CODES = {torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16}


def _dtype_code(t: torch.Tensor, name: str) -> int:
    if t.dtype not in _CODES:
        raise ValueError(f"{name} must be float32 or bfloat16, not {t.dtype}")
    return _CODES[t.dtype]


def _expect(name: str, t, shape, dtype, device, optional: bool = False) -> None:
    """Checks one tensor of a wrapped call: its shape, type, device, and that it has no gaps."""
    if t is None:
        if optional:
            return
        raise ValueError(f"{name} is missing")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _expect_current(device, stream, workspace=None) -> None:
    """The library launches on the current device, so that is where the tensors and the stream have to be."""
    if device.type != "cuda" or device.index != torch.cuda.current_device():
        raise ValueError(f"tensors are on {device}: they must be on the current GPU")
    if stream is not None and stream.device != device:
        raise ValueError(f"the stream belongs to {stream.device}, not to {device}")
    if workspace is not None and (workspace.device != device or not workspace.is_contiguous()):
        raise ValueError(f"buffers.workspace must be contiguous and on {device}")


def _memory_of(stream):
    """Where a call allocates what it works in: memory of the call's own stream, which neither earlier
    work of the current stream uses any more nor later work of it gets while the call runs."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _expect_no_gradient(**operands) -> None:
    """The products have no backward pass: a result that would silently cut the graph is refused."""
    if torch.is_grad_enabled():
        for name, t in operands.items():
            if t is not None and t.requires_grad:
                raise ValueError(f"{name} requires a gradient and this call has none: detach it, or call under torch.no_grad()")


def _hold(stream, used, made=()) -> None:
    """Tensors of a call on a stream of its own may be dropped behind it: what the call uses stays until the
    call has run, and what it allocated on its stream until the current stream, which goes on with it, is
    through as well."""
    if stream is None:
        return
    for t in used:
        if t is not None:
            t.record_stream(stream)
    for t in made:
        t.record_stream(torch.cuda.current_stream())


class ExpertBuffers:
    """act, out and workspace of experts() for calls of one size, allocated once."""

    def __init__(self, T: int, H: int, F: int, E: int, k: int, dtype: torch.dtype, device="cuda"):
        if dtype not in _CODES:
            raise ValueError(f"dtype must be float32 or bfloat16, not {dtype}")
        nbytes = laser_experts_workspace_bytes(T, H, F, E, make_experts_params(k, _CODES[dtype]))
        if nbytes == 0:
            raise LaserError(-2, "laser_experts_workspace_bytes rejected the arguments")
        self.act = torch.empty((T * k, F), dtype=dtype, device=device)
        self.out = torch.empty((T, H), dtype=dtype, device=device)
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)


def experts(hidden, w_up, w_down, routed: RouteBuffers | None, base=None, first_expert: int = 0,
            buffers: ExpertBuffers | None = None, stream=None) -> ExpertBuffers:
    """Both products of the experts behind a routing call: laser_experts_up, then laser_experts_down
    with the call's weights.  w_up [E,2F,H], w_down [E,H,F]; routed None: one expert (E = 1) for every
    token.  The result is `out` of the returned buffers; forward only (operands that require a gradient are
    refused where gradients are enabled)."""
    code = _dtype_code(hidden, "hidden")
    if hidden.dim() != 2 or w_down.dim() != 3:
        raise ValueError("hidden must have 2 dimensions, w_down 3")
    (T, H), (E, _, F), dev, dt = hidden.shape, w_down.shape, hidden.device, hidden.dtype
    k = 1 if routed is None else routed.k
    _expect_no_gradient(hidden=hidden, w_up=w_up, w_down=w_down, base=base,
                        weights=None if routed is None else routed.weights)
    _expect("hidden", hidden, (T, H), dt, dev)
    _expect("w_up", w_up, (E, 2 * F, H), dt, dev)
    _expect("w_down", w_down, (E, H, F), dt, dev)
    _expect("base", base, (T, H), dt, dev, optional=True)
    if routed is not None:
        _expect("permutation", routed.permutation, (T * k,), torch.int32, dev)
        _expect("expert_ids", routed.expert_ids, (T, k), torch.int32, dev)
        _expect("weights", routed.weights, (T, k), torch.float32, dev)
        total = routed.expert_offsets.numel() - 1
        _expect("expert_offsets", routed.expert_offsets, (total + 1,), torch.int32, dev)
        if first_expert < 0 or first_expert + E > total:
            raise ValueError(f"experts {first_expert} to {first_expert + E - 1} of {total}")
    if buffers is not None:
        _expect("buffers.act", buffers.act, (T * k, F), dt, dev)
        _expect("buffers.out", buffers.out, (T, H), dt, dev)
    _expect_current(dev, stream, None if buffers is None else buffers.workspace)
    tables = (None,) * 4 if routed is None else (routed.permutation, routed.expert_offsets, routed.expert_ids,
                                                 routed.weights)
    made = ()
    if buffers is None:
        with _memory_of(stream):
            buffers = ExpertBuffers(T, H, F, E, k, dt, device=dev)
        made = (buffers.act, buffers.out)
    _hold(stream, (hidden, w_up, w_down, base, *tables, buffers.act, buffers.out, buffers.workspace), made)
    params = make_experts_params(k, code, first_expert)
    laser_experts_up(hidden, w_up, T, H, F, E, params, tables[0], tables[1], buffers.act, stream)
    laser_experts_down(buffers.act, w_down, T, H, F, E, params, *tables, base, buffers.out, buffers.workspace, stream)
    return buffers


class ProjectBuffers:
    """out and workspace of project_adapted() for calls of one size, allocated once."""

    def __init__(self, T: int, H: int, N: int, params: LaserAdapterParams, device="cuda"):
        nbytes = laser_project_workspace_bytes(T, H, N, params)
        if nbytes == 0:
            raise LaserError(-2, "laser_project_workspace_bytes rejected the arguments")
        dtype = torch.float32 if params.out_dtype == DTYPE_F32 else torch.bfloat16
        self.out = torch.empty((T, N), dtype=dtype, device=device)
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)


def project_adapted(x, w, a_down, a_up, scales, request_offsets, request_adapters, out_dtype=None,
                    buffers: ProjectBuffers | None = None, stream=None) -> torch.Tensor:
    """laser_project_adapted with sizes from the tensors: x [T,H], w [N,H], a_down [M,R,H], a_up [M,N,R],
    scales [M] fp32 or None, request_offsets [requests+1] and request_adapters [requests] int32.
    out_dtype: that of x (default) or float32.  Returns out [T,N]; forward only, as experts()."""
    code = _dtype_code(x, "x")
    if x.dim() != 2 or w.dim() != 2 or a_down.dim() != 3 or request_adapters.dim() != 1:
        raise ValueError("x and w must have 2 dimensions, a_down 3, request_adapters 1")
    (T, H), N, (M, R), n, dev, dt = x.shape, w.shape[0], a_down.shape[:2], request_adapters.numel(), x.device, x.dtype
    out_dtype = dt if out_dtype is None else out_dtype
    if out_dtype not in (dt, torch.float32):
        raise ValueError(f"out_dtype must be {dt} or float32, not {out_dtype}")
    _expect_no_gradient(x=x, w=w, a_down=a_down, a_up=a_up, scales=scales)
    _expect("x", x, (T, H), dt, dev)
    _expect("w", w, (N, H), dt, dev)
    _expect("a_down", a_down, (M, R, H), dt, dev)
    _expect("a_up", a_up, (M, N, R), dt, dev)
    _expect("scales", scales, (M,), torch.float32, dev, optional=True)
    _expect("request_offsets", request_offsets, (n + 1,), torch.int32, dev)
    _expect("request_adapters", request_adapters, (n,), torch.int32, dev)
    if buffers is not None:
        _expect("buffers.out", buffers.out, (T, N), out_dtype, dev)
    _expect_current(dev, stream, None if buffers is None else buffers.workspace)
    params = make_adapter_params(R, M, n, code, _CODES[out_dtype])
    made = ()
    if buffers is None:
        with _memory_of(stream):
            buffers = ProjectBuffers(T, H, N, params, device=dev)
        made = (buffers.out,)
    _hold(stream, (x, w, a_down, a_up, scales, request_offsets, request_adapters, buffers.out, buffers.workspace), made)
    laser_project_adapted(x, w, T, H, N, params, a_down, a_up, scales, request_offsets, request_adapters,
                          buffers.out, buffers.workspace, stream)
    return buffers.out
