"""Thin ctypes binding of libtrivance.so (the C ABI declared in include/trivance.h).

Argument marshalling only: every step of the emulated AllReduce runs in the library's HIP
kernels. Functions keep the C names. PyTorch provides device memory (tensors) and streams; it is
imported before the library is loaded so that both share one HIP runtime (both carry the soname
libamdhip64.so.7, and the first one loaded is reused).

There is no fallback: if the library is missing or a call fails, an exception is raised.
"""

from __future__ import annotations

import ctypes
import os

import numpy as np

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libtrivance.so")

LATENCY_OPT, BANDWIDTH_OPT, BRUCK_REF = 0, 1, 2
F32, I32, BF16, F16, I64 = 0, 1, 2, 3, 4
ROUTE_SCHEDULED, ROUTE_SHORTEST = 0, 1
PHASE_LATENCY, PHASE_REDUCE_SCATTER, PHASE_ALLGATHER = 0, 1, 2
MAX_DIMS = 8

_VARIANTS = {"L": LATENCY_OPT, "B": BANDWIDTH_OPT, "BRUCK": BRUCK_REF}
PLACE_BY_SCHEDULE = 1  # TRIVANCE_PLACE_BY_SCHEDULE
_PLACEMENTS = {"natural": 0, "schedule": PLACE_BY_SCHEDULE}
_ROUTING = {"scheduled": ROUTE_SCHEDULED, "shortest": ROUTE_SHORTEST}


class TrivanceError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what} failed: {_lib().trivance_strerror(status).decode()} ({status})")


class CostResult(ctypes.Structure):
    _fields_ = [("total", ctypes.c_double), ("latency", ctypes.c_double),
                ("transmission", ctypes.c_double), ("theta", ctypes.c_double),
                ("passes", ctypes.c_int)]


class Topology(ctypes.Structure):
    _fields_ = [("ndims", ctypes.c_int), ("dims", ctypes.c_int * MAX_DIMS),
                ("routing", ctypes.c_int)]


_LIB = None


def _lib():
    global _LIB
    if _LIB is not None:
        return _LIB
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is not built; run __graft_entry__.build() "
                           "(python -m paper_2602_17254_amd._build)")
    import torch  # noqa: F401  -- load torch's HIP runtime first (see module docstring)

    lib = ctypes.CDLL(LIB_PATH)
    P = ctypes.c_void_p
    i64 = ctypes.c_int64
    sig = {
        "trivance_plan": (ctypes.c_int, [ctypes.c_int, ctypes.POINTER(ctypes.c_int), ctypes.c_int,
                                         ctypes.c_int, ctypes.POINTER(P)]),
        "trivance_plan_ex": (ctypes.c_int, [ctypes.c_int, ctypes.POINTER(ctypes.c_int), ctypes.c_int,
                                            ctypes.c_int, ctypes.c_uint, ctypes.POINTER(P)]),
        "trivance_plan_destroy": (None, [P]),
        "trivance_plan_num_steps": (ctypes.c_int, [P]),
        "trivance_plan_num_passes": (ctypes.c_int, [P]),
        "trivance_plan_step": (ctypes.c_int, [P, ctypes.c_int, ctypes.c_int] +
                               [ctypes.POINTER(ctypes.c_int)] * 3),
        "trivance_plan_step_index": (ctypes.c_int, [P, ctypes.c_int]),
        "trivance_plan_with_dispatch_limit": (ctypes.c_int, [P, i64, ctypes.POINTER(P)]),
        "trivance_block_range": (ctypes.c_int, [P, i64, ctypes.c_int, ctypes.c_int,
                                                ctypes.POINTER(i64), ctypes.POINTER(i64)]),
        "trivance_algorithmic_bytes": (i64, [P, i64, ctypes.c_int]),
        "trivance_pass_bytes": (i64, [P, i64, ctypes.c_int, ctypes.c_int]),
        "trivance_allreduce_emulated": (ctypes.c_int, [P, ctypes.c_int, i64, ctypes.c_int, P, P]),
        "trivance_allreduce_emulated_steps": (ctypes.c_int, [P, ctypes.c_int, i64, ctypes.c_int,
                                                             P, P, ctypes.c_int, ctypes.c_int]),
        "trivance_workspace_bytes": (i64, [P, i64, ctypes.c_int]),
        "trivance_allreduce_emulated_ws": (ctypes.c_int, [P, ctypes.c_int, i64, ctypes.c_int, P, P,
                                                          i64, P]),
        "trivance_allreduce_emulated_steps_ws": (ctypes.c_int, [P, ctypes.c_int, i64, ctypes.c_int,
                                                                P, P, i64, P, ctypes.c_int,
                                                                ctypes.c_int]),
        "trivance_congestion": (i64, [P, ctypes.POINTER(Topology), ctypes.POINTER(i64), i64]),
        "trivance_congestion_device": (ctypes.c_int, [P, ctypes.POINTER(Topology), P, i64, P]),
        "trivance_congestion_noalloc": (i64, [P, ctypes.POINTER(Topology), ctypes.POINTER(i64), i64]),
        "trivance_fill_hash_uniform": (ctypes.c_int, [P, ctypes.c_int, i64, ctypes.c_uint64, P]),
        "trivance_copy_device": (ctypes.c_int, [P, P, i64, P]),
        "trivance_cost_model": (ctypes.c_int, [P, ctypes.c_double, ctypes.c_double, ctypes.c_double,
                                               ctypes.POINTER(ctypes.c_double), ctypes.c_int,
                                               ctypes.POINTER(CostResult)]),
        "trivance_layernorm_forward": (ctypes.c_int, [P] * 6 + [i64] * 7 +
                                       [ctypes.c_double, ctypes.c_int, ctypes.c_int, P]),
        "trivance_layernorm_workspace_bytes": (i64, [i64] * 3),
        "trivance_layernorm_backward": (ctypes.c_int, [P] * 8 + [i64] * 10 +
                                        [ctypes.c_int, ctypes.c_int, P, i64, P]),
        "trivance_balance_workspace_bytes": (i64, [i64] * 3),
        "trivance_balance_counts": (ctypes.c_int, [P] * 5 + [i64] * 8 +
                                    [ctypes.c_int, ctypes.c_int, P, i64, P]),
        "trivance_balance_loss": (ctypes.c_int, [P] * 3 + [i64] * 5 + [ctypes.c_double, P]),
        "trivance_balance_backward": (ctypes.c_int, [P] * 5 + [i64] * 9 +
                                      [ctypes.c_double, ctypes.c_int, P]),
        "trivance_orthogonalize_workspace_bytes": (i64, [i64] * 3),
        "trivance_orthogonalize": (ctypes.c_int, [P] * 2 + [i64] * 7 +
                                   [ctypes.POINTER(ctypes.c_float), ctypes.c_int, ctypes.c_double,
                                    ctypes.c_double, ctypes.c_int, P, i64, P]),
        "trivance_strerror": (ctypes.c_char_p, [ctypes.c_int]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _LIB = lib
    return lib


def exported_symbols() -> list:
    """Names the binding resolves (all of include/trivance.h)."""
    lib = ctypes.CDLL(LIB_PATH)
    names = ["trivance_plan", "trivance_plan_ex", "trivance_plan_destroy", "trivance_plan_num_steps",
             "trivance_plan_num_passes", "trivance_plan_step", "trivance_plan_step_index",
             "trivance_plan_with_dispatch_limit", "trivance_block_range",
             "trivance_algorithmic_bytes", "trivance_pass_bytes", "trivance_allreduce_emulated",
             "trivance_allreduce_emulated_steps", "trivance_workspace_bytes",
             "trivance_allreduce_emulated_ws", "trivance_allreduce_emulated_steps_ws",
             "trivance_congestion",
             "trivance_congestion_device", "trivance_congestion_noalloc", "trivance_fill_hash_uniform",
             "trivance_copy_device", "trivance_cost_model", "trivance_strerror",
             "trivance_layernorm_forward", "trivance_layernorm_workspace_bytes",
             "trivance_layernorm_backward", "trivance_balance_workspace_bytes",
             "trivance_balance_counts", "trivance_balance_loss", "trivance_balance_backward",
             "trivance_orthogonalize_workspace_bytes", "trivance_orthogonalize"]
    return [n for n in names if hasattr(lib, n)]


def _check(rc: int, what: str) -> int:
    if rc < 0:
        raise TrivanceError(int(rc), what)
    return rc


class Plan:
    """Owns a trivance_plan_t handle."""

    def __init__(self, handle, dims, variant, placement="natural"):
        self._h = handle
        self.dims = tuple(dims)
        self.variant = variant
        self.placement = placement
        self.n = int(np.prod(self.dims))
        self.D = len(self.dims)

    @property
    def handle(self):
        return self._h

    @property
    def num_steps(self) -> int:
        return _check(_lib().trivance_plan_num_steps(self._h), "trivance_plan_num_steps")

    @property
    def num_passes(self) -> int:
        return _check(_lib().trivance_plan_num_passes(self._h), "trivance_plan_num_passes")

    def __del__(self):
        if getattr(self, "_h", None) and _LIB is not None:
            _LIB.trivance_plan_destroy(self._h)
            self._h = None


def trivance_plan(dims, variant="L", placement="natural") -> Plan:
    """Build a plan for a ring (dims=(n,)) or torus; variant 'L', 'B' or 'BRUCK'; placement
    'natural' (block j at the j-th granule range) or 'schedule' (TRIVANCE_PLACE_BY_SCHEDULE)."""
    dims = tuple(int(d) for d in dims)
    arr = (ctypes.c_int * len(dims))(*dims)
    h = ctypes.c_void_p()
    n = int(np.prod(dims)) if dims else 0
    _check(_lib().trivance_plan_ex(n, arr, len(dims), _VARIANTS[variant], _PLACEMENTS[placement],
                                   ctypes.byref(h)), "trivance_plan_ex")
    return Plan(h, dims, variant, placement)


def trivance_plan_step(plan: Plan, pass_index: int, collective: int = 0) -> tuple:
    """(phase, dim, distance) of one pass for one collective."""
    out = [ctypes.c_int() for _ in range(3)]
    _check(_lib().trivance_plan_step(plan.handle, pass_index, collective,
                                     *[ctypes.byref(o) for o in out]), "trivance_plan_step")
    return tuple(o.value for o in out)


def trivance_plan_step_index(plan: Plan, pass_index: int) -> int:
    """Global step index t that a pass materialises (all-gather passes run t = S-1 .. 0)."""
    return _check(_lib().trivance_plan_step_index(plan.handle, pass_index),
                  "trivance_plan_step_index")


def trivance_plan_with_dispatch_limit(plan: Plan, work_items: int) -> Plan:
    """A new plan equal to `plan` whose launches are issued as dispatches of at most `work_items`
    work-items (1024 .. 2^31); `plan` itself is unchanged."""
    h = ctypes.c_void_p()
    _check(_lib().trivance_plan_with_dispatch_limit(plan.handle, int(work_items), ctypes.byref(h)),
           "trivance_plan_with_dispatch_limit")
    return Plan(h, plan.dims, plan.variant, plan.placement)


def trivance_block_range(plan: Plan, elems: int, collective: int, block: int) -> tuple:
    b, e = ctypes.c_int64(), ctypes.c_int64()
    _check(_lib().trivance_block_range(plan.handle, elems, collective, block, ctypes.byref(b),
                                       ctypes.byref(e)), "trivance_block_range")
    return b.value, e.value


def trivance_algorithmic_bytes(plan: Plan, elems: int, dtype: int = F32) -> int:
    return _check(_lib().trivance_algorithmic_bytes(plan.handle, elems, dtype),
                  "trivance_algorithmic_bytes")


def trivance_pass_bytes(plan: Plan, elems: int, pass_index: int, dtype: int = F32) -> int:
    return _check(_lib().trivance_pass_bytes(plan.handle, elems, dtype, pass_index),
                  "trivance_pass_bytes")


_TORCH = None
_DTYPES = {}
_FLOATS = {}  # the element types of activations, logits, weights and matrices
_IDS = {}  # of expert numbers
_current_device = None  # torch's call, without the checks of its public form where it has the private one


def _torch():
    """The torch module, and the element types it maps to; imported on the first call."""
    global _TORCH, _current_device
    if _TORCH is None:
        import torch

        _DTYPES.update({torch.float32: F32, torch.int32: I32})
        _FLOATS.update({torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16})
        _IDS.update({torch.int32: I32, torch.int64: I64})
        if _current_device is None:
            _current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        _TORCH = torch
    return _TORCH


def _stream_ptr(stream):
    if stream is None:
        torch = _torch()
        try:
            # the current stream's handle as current_stream().cuda_stream gives it, without the Stream
            # object: 0.3 us instead of 2.7 (a whole small AllReduce takes 8 with it and 5 without)
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        except AttributeError:  # these calls are private: a torch without them
            return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _buffer_args(buffers, plan: Plan):
    if not isinstance(buffers, _torch().Tensor) or not buffers.is_cuda:
        raise TypeError("buffers must be a CUDA (HIP) torch tensor")
    shape = buffers.shape
    if len(shape) != 2 or shape[0] != plan.n or not buffers.is_contiguous():
        raise ValueError(f"buffers must be a contiguous [{plan.n}, elems] tensor")
    dt = _DTYPES.get(buffers.dtype)
    if dt is None:
        raise TypeError("buffers must be float32 or int32")
    return buffers.data_ptr(), plan.n, shape[1], dt


def trivance_allreduce_emulated(buffers, plan: Plan, stream=None) -> None:
    """In-place emulated AllReduce over the rows of `buffers` (enqueued on `stream`)."""
    ptr, n, E, dt = _buffer_args(buffers, plan)
    _check(_lib().trivance_allreduce_emulated(ptr, n, E, dt, plan._h, _stream_ptr(stream)),
           "trivance_allreduce_emulated")


def trivance_allreduce_emulated_steps(buffers, plan: Plan, pass_begin: int, pass_end: int,
                                      stream=None) -> None:
    ptr, n, E, dt = _buffer_args(buffers, plan)
    _check(_lib().trivance_allreduce_emulated_steps(ptr, n, E, dt, plan.handle,
                                                    _stream_ptr(stream), pass_begin, pass_end),
           "trivance_allreduce_emulated_steps")


def trivance_workspace_bytes(plan: Plan, elems: int, dtype: int = F32) -> int:
    return _check(_lib().trivance_workspace_bytes(plan.handle, elems, dtype),
                  "trivance_workspace_bytes")


def _workspace_args(workspace):
    if workspace is None:
        return None, 0
    if not isinstance(workspace, _torch().Tensor) or not workspace.is_cuda or \
            not workspace.is_contiguous():
        raise TypeError("workspace must be a contiguous CUDA tensor")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def trivance_allreduce_emulated_ws(buffers, plan: Plan, workspace, stream=None) -> None:
    """In-place emulated AllReduce with a caller-owned device workspace (any contiguous CUDA tensor
    of at least trivance_workspace_bytes bytes)."""
    ptr, n, E, dt = _buffer_args(buffers, plan)
    wp, wb = _workspace_args(workspace)
    _check(_lib().trivance_allreduce_emulated_ws(ptr, n, E, dt, plan.handle, wp, wb,
                                                 _stream_ptr(stream)),
           "trivance_allreduce_emulated_ws")


def trivance_allreduce_emulated_steps_ws(buffers, plan: Plan, workspace, pass_begin: int,
                                         pass_end: int, stream=None) -> None:
    ptr, n, E, dt = _buffer_args(buffers, plan)
    wp, wb = _workspace_args(workspace)
    _check(_lib().trivance_allreduce_emulated_steps_ws(ptr, n, E, dt, plan.handle, wp, wb,
                                                       _stream_ptr(stream), pass_begin, pass_end),
           "trivance_allreduce_emulated_steps_ws")


def _topology(plan: Plan, routing: str) -> Topology:
    t = Topology()
    t.ndims = plan.D
    for i, d in enumerate(plan.dims):
        t.dims[i] = d
    t.routing = _ROUTING[routing]
    return t


def trivance_congestion(plan: Plan, routing: str = "scheduled") -> np.ndarray:
    """int64 loads[pass][rank][port] computed on the GPU (synchronous)."""
    lib = _lib()
    topo = _topology(plan, routing)
    need = _check(lib.trivance_congestion(plan.handle, ctypes.byref(topo), None, 0),
                  "trivance_congestion")
    out = np.zeros(need, dtype=np.int64)
    _check(lib.trivance_congestion(plan.handle, ctypes.byref(topo),
                                   out.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)), need),
           "trivance_congestion")
    return out.reshape(plan.num_passes, plan.n, 2 * plan.D)


def trivance_congestion_noalloc(plan: Plan, routing: str = "scheduled") -> np.ndarray:
    """trivance_congestion computed in the library's fixed device scratch (no device allocation;
    at most 2^20 entries)."""
    lib = _lib()
    topo = _topology(plan, routing)
    need = _check(lib.trivance_congestion_noalloc(plan.handle, ctypes.byref(topo), None, 0),
                  "trivance_congestion_noalloc")
    out = np.zeros(need, dtype=np.int64)
    _check(lib.trivance_congestion_noalloc(plan.handle, ctypes.byref(topo),
                                           out.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)), need),
           "trivance_congestion_noalloc")
    return out.reshape(plan.num_passes, plan.n, 2 * plan.D)


def trivance_congestion_device(plan: Plan, out, routing: str = "scheduled", stream=None) -> None:
    """Same counts written into a caller-owned int64 CUDA tensor (asynchronous)."""
    import torch

    if not isinstance(out, torch.Tensor) or not out.is_cuda or out.dtype != torch.int64 \
            or not out.is_contiguous():
        raise TypeError("out must be a contiguous int64 CUDA tensor")
    topo = _topology(plan, routing)
    _check(_lib().trivance_congestion_device(plan.handle, ctypes.byref(topo),
                                             ctypes.c_void_p(out.data_ptr()), out.numel(),
                                             _stream_ptr(stream)), "trivance_congestion_device")


def trivance_fill_hash_uniform(buffers, seed: int, stream=None) -> None:
    """Fill a float32 [n, elems] CUDA tensor with the counter-based U(-1, 1) inputs."""
    import torch

    if not isinstance(buffers, torch.Tensor) or not buffers.is_cuda or buffers.dtype != torch.float32 \
            or buffers.dim() != 2 or not buffers.is_contiguous():
        raise TypeError("buffers must be a contiguous float32 [n, elems] CUDA tensor")
    _check(_lib().trivance_fill_hash_uniform(ctypes.c_void_p(buffers.data_ptr()),
                                             buffers.shape[0], buffers.shape[1], seed,
                                             _stream_ptr(stream)), "trivance_fill_hash_uniform")


def trivance_copy_device(dst, src, stream=None) -> None:
    """Benchmark helper: copy the contiguous CUDA tensor `src` into `dst` (the same number of
    bytes, a multiple of 16) with the library's streaming copy kernel."""
    import torch

    for name, t in (("dst", dst), ("src", src)):
        if not isinstance(t, torch.Tensor) or not t.is_cuda or not t.is_contiguous():
            raise TypeError(f"{name} must be a contiguous CUDA tensor")
    nbytes = src.numel() * src.element_size()
    if dst.numel() * dst.element_size() != nbytes:
        raise ValueError("dst and src must hold the same number of bytes")
    _check(_lib().trivance_copy_device(ctypes.c_void_p(dst.data_ptr()),
                                       ctypes.c_void_p(src.data_ptr()), nbytes,
                                       _stream_ptr(stream)), "trivance_copy_device")


def trivance_cost_model(plan: Plan, bytes_per_rank: float, alpha: float = 0.0,
                        beta: float = 0.0) -> dict:
    """The Sec. 2.1 cost model of the plan for an AllReduce of `bytes_per_rank` bytes per rank:
    total, latency and transmission times, theta, passes, and the busiest link's bytes per
    pass."""
    P = plan.num_passes
    peaks = (ctypes.c_double * max(P, 1))()
    res = CostResult()
    _check(_lib().trivance_cost_model(plan.handle, float(bytes_per_rank), float(alpha), float(beta),
                                      peaks, max(P, 1), ctypes.byref(res)), "trivance_cost_model")
    return {"total": res.total, "latency": res.latency, "transmission": res.transmission,
            "theta": res.theta, "passes": res.passes, "pass_link_bytes": list(peaks)[:P]}


# The operators around the AllReduce. Tensors of activations and logits are [ranks, tokens, width], any
# strides with the last dimension's values consecutive; gradients, counts and sums are one row per
# rank and may be slices of a buffer that an AllReduce sums.


def _device(t, name):
    """The tensor's GPU, which has to be the current one: its stream takes the kernels."""
    dev = t.get_device()
    if dev != _current_device():
        raise ValueError(f"{name} is on GPU {dev}, which is not the current device")
    return dev


def _work(workspace, device):
    """(pointer, bytes) of a workspace on that GPU, (None, 0) for None."""
    if workspace is None:
        return None, 0
    args = _workspace_args(workspace)
    if workspace.get_device() != device:
        raise ValueError(f"workspace must be on GPU {device}")
    return args


def _rows(t, name):
    """(pointer, rank stride, token stride, type, device) of a [ranks, tokens, width] tensor."""
    if not isinstance(t, _torch().Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) torch tensor")
    dt = _FLOATS.get(t.dtype)
    if dt is None:
        raise TypeError(f"{name} must be float32, bfloat16 or float16")
    if t.dim() != 3:
        raise ValueError(f"{name} must be three-dimensional")
    s0, s1, s2 = t.stride()
    if s2 != 1 and t.shape[2] > 1:
        raise ValueError(f"the values of a row of {name} must be consecutive")
    return t.data_ptr(), s0, s1, dt, _device(t, name)


def _rows_like(t, name, shape, dtype, device):
    """(pointer, rank stride, token stride) of a tensor like another one."""
    if not isinstance(t, _TORCH.Tensor) or t.dtype is not dtype or t.get_device() != device:
        raise TypeError(f"{name} must be a {dtype} tensor on GPU {device}")
    if t.shape != shape:
        raise ValueError(f"{name} must be {tuple(shape)}")
    s0, s1, s2 = t.stride()
    if s2 != 1 and shape[2] > 1:
        raise ValueError(f"the values of a row of {name} must be consecutive")
    return t.data_ptr(), s0, s1


def _array(t, name, shape, dtype, device):
    """Pointer of a contiguous tensor, None for None."""
    if t is None:
        return None
    if not isinstance(t, _TORCH.Tensor) or t.dtype is not dtype or t.get_device() != device:
        raise TypeError(f"{name} must be a {dtype} tensor on GPU {device}")
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {tuple(shape)} tensor")
    return t.data_ptr()


def _rank_rows(t, name, ranks, width, dtype, device):
    """(pointer, stride) of one row of `width` values per rank, (None, 0) for None."""
    if t is None:
        return None, 0
    if not isinstance(t, _TORCH.Tensor) or t.dtype is not dtype or t.get_device() != device:
        raise TypeError(f"{name} must be a {dtype} tensor on GPU {device}")
    if t.shape != (ranks, width) or (width > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be [{ranks}, {width}] with consecutive values in a row")
    # the stride of a single row does not matter, and torch may give any
    return t.data_ptr(), t.stride(0) if ranks > 1 else width


def _weights(gamma, beta, width, device):
    """Pointers and the one type of the weights."""
    w = gamma if gamma is not None else beta
    if w is None:
        return None, None, F32
    dtype = getattr(w, "dtype", None)
    dt = _FLOATS.get(dtype)
    if dt is None:
        raise TypeError("weights must be float32, bfloat16 or float16 tensors")
    shape = (width,)
    return (_array(gamma, "gamma", shape, dtype, device), _array(beta, "beta", shape, dtype, device), dt)


def trivance_layernorm_forward(x, gamma, beta, y, mean=None, rstd=None, eps=1e-5,
                               stream=None) -> None:
    """y = layer norm of the rows of x [ranks, tokens, width], times gamma plus beta (either may be
    None); mean and rstd [ranks, tokens] receive the statistics for the backward pass."""
    xp, xr, xt, dt, dev = _rows(x, "x")
    shape = x.shape
    yp, yr, yt = _rows_like(y, "y", shape, x.dtype, dev)
    ranks, tokens, width = shape
    f32 = _TORCH.float32
    gp, bp, wt = _weights(gamma, beta, width, dev)
    mp = _array(mean, "mean", (ranks, tokens), f32, dev)
    sp = _array(rstd, "rstd", (ranks, tokens), f32, dev)
    _check(_lib().trivance_layernorm_forward(xp, gp, bp, yp, mp, sp, ranks, tokens, width, xr, xt, yr,
                                             yt, eps, dt, wt, _stream_ptr(stream)),
           "trivance_layernorm_forward")


def trivance_layernorm_workspace_bytes(ranks: int, tokens: int, width: int) -> int:
    return _check(_lib().trivance_layernorm_workspace_bytes(ranks, tokens, width),
                  "trivance_layernorm_workspace_bytes")


def trivance_layernorm_backward(dy, x, gamma, mean, rstd, dx, dgamma, dbeta, workspace=None,
                                stream=None) -> None:
    """dx, and each rank's dgamma and dbeta [ranks, width] (fp32 rows, equally far apart; either may be
    None), from dy and what the forward pass read and wrote."""
    xp, xr, xt, dt, dev = _rows(x, "x")
    shape, dtype = x.shape, x.dtype
    dyp, dyr, dyt = _rows_like(dy, "dy", shape, dtype, dev)
    dxp, dxr, dxt = _rows_like(dx, "dx", shape, dtype, dev)
    ranks, tokens, width = shape
    f32 = _TORCH.float32
    gp, _, wt = _weights(gamma, None, width, dev)
    mp = _array(mean, "mean", (ranks, tokens), f32, dev)
    sp = _array(rstd, "rstd", (ranks, tokens), f32, dev)
    dgp, dgs = _rank_rows(dgamma, "dgamma", ranks, width, f32, dev)
    dbp, dbs = _rank_rows(dbeta, "dbeta", ranks, width, f32, dev)
    if dgamma is not None and dbeta is not None and dgs != dbs:
        raise ValueError("the rows of dgamma and dbeta must be equally far apart")
    wp, wb = _work(workspace, dev)
    _check(_lib().trivance_layernorm_backward(dyp, xp, gp, mp, sp, dxp, dgp, dbp, ranks, tokens, width,
                                              dyr, dyt, xr, xt, dxr, dxt,
                                              dbs if dgamma is None else dgs, dt, wt, wp, wb,
                                              _stream_ptr(stream)),
           "trivance_layernorm_backward")


def trivance_balance_workspace_bytes(ranks: int, tokens: int, experts: int) -> int:
    return _check(_lib().trivance_balance_workspace_bytes(ranks, tokens, experts),
                  "trivance_balance_workspace_bytes")


def _mask(mask, shape, device):
    """Pointer of a mask of bools or bytes, None for None."""
    if mask is None:
        return None
    dtype = _TORCH.uint8 if getattr(mask, "dtype", None) is _TORCH.uint8 else _TORCH.bool
    return _array(mask, "mask", shape, dtype, device)


def trivance_balance_counts(logits, chosen, counts, probs, workspace=None, mask=None,
                            stream=None) -> None:
    """Each rank's expert counts and number of tokens, counts [ranks, experts + 1] (int32), and sums of
    probabilities, probs [ranks, experts] (float32), from the router's logits [ranks, tokens,
    experts], the experts chosen [ranks, tokens, top_k] (int32 or int64; negative: an empty slot)
    and an optional mask [ranks, tokens] of the tokens that count (bool or uint8)."""
    lp, lr, lt, dt, dev = _rows(logits, "logits")
    ranks, tokens, experts = logits.shape
    it = _IDS.get(getattr(chosen, "dtype", None))
    if it is None:
        raise TypeError("chosen must be an int32 or int64 tensor")
    if chosen.dim() != 3:
        raise ValueError("chosen must be [ranks, tokens, top_k]")
    k = chosen.shape[2]
    ip = _array(chosen, "chosen", (ranks, tokens, k), chosen.dtype, dev)
    mp = _mask(mask, (ranks, tokens), dev)
    cp, cs = _rank_rows(counts, "counts", ranks, experts + 1, _TORCH.int32, dev)
    pp, ps = _rank_rows(probs, "probs", ranks, experts, _TORCH.float32, dev)
    wp, wb = _work(workspace, dev)
    _check(_lib().trivance_balance_counts(lp, ip, mp, cp, pp, ranks, tokens, experts, k, lr, lt,
                                          cs, ps, dt, it, wp, wb, _stream_ptr(stream)),
           "trivance_balance_counts")


def trivance_balance_loss(counts, probs, top_k: int, loss, scale=1.0, stream=None) -> None:
    """loss [ranks]: the balance loss of every rank's row of counts and probs."""
    if not isinstance(probs, _torch().Tensor) or not probs.is_cuda or probs.dim() != 2:
        raise TypeError("probs must be a two-dimensional CUDA (HIP) torch tensor")
    ranks, experts = probs.shape
    dev = _device(probs, "probs")
    pp, ps = _rank_rows(probs, "probs", ranks, experts, _TORCH.float32, dev)
    cp, cs = _rank_rows(counts, "counts", ranks, experts + 1, _TORCH.int32, dev)
    op = _array(loss, "loss", (ranks,), _TORCH.float32, dev)
    _check(_lib().trivance_balance_loss(cp, pp, op, ranks, experts, top_k, cs, ps, scale,
                                        _stream_ptr(stream)), "trivance_balance_loss")


def trivance_balance_backward(logits, counts, top_k: int, dlogits, mask=None, scale=1.0, dloss=None,
                              stream=None) -> None:
    """dlogits: the gradient of the balance loss of `counts`, times dloss [ranks] (None: ones)."""
    lp, lr, lt, dt, dev = _rows(logits, "logits")
    dp, dr, dts = _rows_like(dlogits, "dlogits", logits.shape, logits.dtype, dev)
    ranks, tokens, experts = logits.shape
    mp = _mask(mask, (ranks, tokens), dev)
    cp, cs = _rank_rows(counts, "counts", ranks, experts + 1, _TORCH.int32, dev)
    gp = _array(dloss, "dloss", (ranks,), _TORCH.float32, dev)
    _check(_lib().trivance_balance_backward(lp, cp, mp, gp, dp, ranks, tokens, experts, top_k, lr, lt,
                                            dr, dts, cs, scale, dt, _stream_ptr(stream)),
           "trivance_balance_backward")


def trivance_orthogonalize_workspace_bytes(batch: int, rows: int, cols: int) -> int:
    return _check(_lib().trivance_orthogonalize_workspace_bytes(batch, rows, cols),
                  "trivance_orthogonalize_workspace_bytes")


# a, b, c of five steps that bring singular values from [0.003, 1] to about [0.7, 1.2]
QUINTIC_5 = ((3.4445, -4.7750, 2.0315),) * 5


def _coefficients(steps):
    """The steps' coefficients as a host array."""
    if steps is QUINTIC_5:
        return _HOST_QUINTIC_5
    if any(len(abc) != 3 for abc in steps):
        raise ValueError("coefficients must be three numbers for each step")
    flat = [float(v) for abc in steps for v in abc]
    return (ctypes.c_float * max(len(flat), 1))(*flat), len(steps)


_HOST_QUINTIC_5 = _coefficients(list(QUINTIC_5))


def trivance_orthogonalize(x, out, workspace, coefficients=QUINTIC_5, scale=1.0, eps=1e-7,
                           stream=None) -> None:
    """out = scale times x [batch, rows, cols] with the singular values of each matrix pushed towards
    one: X = x / (norm + eps), then X <- a X + (b A + c A A) X, A = X X', for each (a, b, c)."""
    xp, xb, xr, dt, dev = _rows(x, "x")
    op, ob, orow = _rows_like(out, "out", x.shape, x.dtype, dev)
    batch, rows, cols = x.shape
    k, steps = _coefficients(coefficients)
    wp, wb = _work(workspace, dev)
    _check(_lib().trivance_orthogonalize(xp, op, batch, rows, cols, xb, xr, ob, orow, k, steps, scale,
                                         eps, dt, wp, wb, _stream_ptr(stream)),
           "trivance_orthogonalize")
