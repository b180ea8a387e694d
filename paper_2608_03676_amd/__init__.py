"""MI355X-native TAOT per-step replica planner.

Thin Python binding of libtaot.so (include/taot.h).  Every step of the path
runs in the library's HIP kernels; this module only checks tensor
dtypes/devices, allocates outputs and workspace with torch on the GPU, and
passes raw pointers plus the current HIP stream.  There is no CPU fallback:
calls raise if the library is not built or a tensor is not on the GPU.

Steps (paper Sec. 3.2 / Appendix A): plan_loads (expert-load histogram and
marginals), sinkhorn_batched (Phase 1), round_schedule (Phases 2 and 3);
plan_step chains them.

Around them: add_rms_norm (residual addition, norm, 8-bit output) and route
(logits to expert ids, which plan_loads reads, and weights) before; then
dispatch_map (the schedule on the single copies), dispatch_rows and
combine_rows (rows to the send buffer and back).  The *_backward calls are
their gradients.  None of them is part of torch's graph: inputs whose gradient
is being recorded are refused.
"""
from __future__ import annotations

import ctypes
import dataclasses
import os
from typing import Optional

import numpy as np
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libtaot.so")

ST_BAD_ID, ST_BAD_INPUT, ST_ZERO_MASS, ST_UNFILLED, ST_STREAMED = 0x1, 0x2, 0x4, 0x8, 0x10
SK_NO_COLCAP, SK_FORCE_STREAM, SK_NO_REGISTER, SK_WAVES_1, SK_DENSE, SK_LINEAR = 0x1, 0x2, 0x4, 0x8, 0x10, 0x20
SCH_NO_TOPO, SCH_NO_FLOW, SCH_ROW_PRIORITY = 0x1, 0x2, 0x4  # Phase-2 ablations (round_schedule flags)
ROUTE_SIGMOID, ROUTE_RENORM, ROUTE_GROUP_TWO = 0x1, 0x2, 0x4  # route flags
STATUS_NAMES = {0: "ok", 1: "invalid argument", 2: "unsupported shape", 3: "workspace", 4: "launch"}

_lib = None
_devices = 0  # GPUs that the process sees, once the library is loaded
_P, _I32, _I64, _F32, _F64, _SZ, _U32 = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float,
                                         ctypes.c_double, ctypes.c_size_t, ctypes.c_uint32)


class TaotError(RuntimeError):
    def __init__(self, fn: str, code: int):
        super().__init__(f"{fn}: {lib().taot_status_string(code).decode()} (status {code})")
        self.code = code


def lib():
    """Load libtaot.so (raises if it has not been built)."""
    global _lib, _devices
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
        L = ctypes.CDLL(LIB_PATH)
        L.taot_status_string.restype = ctypes.c_char_p
        L.taot_status_string.argtypes = [ctypes.c_int]
        L.taot_plan_loads_workspace_size.restype = _SZ
        L.taot_plan_loads_workspace_size.argtypes = [_I32, _I32, _I32]
        L.taot_plan_loads.restype = ctypes.c_int
        L.taot_plan_loads.argtypes = [_P, _I32, _I32, _I64, _I32] + [_P] * 17 + [_P, _SZ, _P]
        L.taot_sinkhorn_workspace_size.restype = _SZ
        L.taot_sinkhorn_workspace_size.argtypes = [_I32, _I32]
        L.taot_sinkhorn_batched.restype = ctypes.c_int
        L.taot_sinkhorn_batched.argtypes = [_P, _P, _I32, _I32, _P, _I64, _F32, _I32, _U32, _P, _P, _P, _P,
                                            _P, _SZ, _P]
        L.taot_round_schedule_workspace_size.restype = _SZ
        L.taot_round_schedule_workspace_size.argtypes = [_I32, _I32, _I32, _I32]
        L.taot_round_schedule.restype = ctypes.c_int
        L.taot_round_schedule.argtypes = [_P] * 9 + [_I32] * 4 + [_F64, _I64, _U32] + [_P] * 6 + [_P, _SZ, _P]
        L.taot_add_rms_norm.restype = ctypes.c_int
        L.taot_add_rms_norm.argtypes = [_P] * 3 + [_I64, _I32, _I32, _I32, _F32, _I32] + [_P] * 6
        L.taot_add_rms_norm_backward_workspace_size.restype = _SZ
        L.taot_add_rms_norm_backward_workspace_size.argtypes = [_I64, _I32]
        L.taot_add_rms_norm_backward.restype = ctypes.c_int
        L.taot_add_rms_norm_backward.argtypes = [_P] * 5 + [_I64, _I32, _I32, _I32, _P, _P, _P, _SZ, _P]
        L.taot_route.restype = ctypes.c_int
        L.taot_route.argtypes = [_P, _P, _I64] + [_I32] * 4 + [_F32, _U32, _I32, _P, _P, _P]
        L.taot_route_backward.restype = ctypes.c_int
        L.taot_route_backward.argtypes = [_P] * 3 + [_I64, _I32, _I32, _F32, _U32, _I32, _P, _P]
        L.taot_dispatch_map_workspace_size.restype = _SZ
        L.taot_dispatch_map_workspace_size.argtypes = [_I32, _I32, _I64, _I32, _I32, _I32]
        L.taot_dispatch_map.restype = ctypes.c_int
        L.taot_dispatch_map.argtypes = [_P, _I32, _I32, _I32, _I64, _P, _I32, _I32, _I32] + [_P] * 7 + [_SZ, _P]
        L.taot_dispatch_rows.restype = ctypes.c_int
        L.taot_dispatch_rows.argtypes = [_P, _I64, _P, _I64, _I64, _I64, _I32] + [_P] * 4
        L.taot_combine_rows.restype = ctypes.c_int
        L.taot_combine_rows.argtypes = [_P] * 3 + [_I64, _I64, _I32, _I32, _I32, _P, _P]
        L.taot_combine_rows_backward.restype = ctypes.c_int
        L.taot_combine_rows_backward.argtypes = [_P] * 4 + [_I64, _I64, _I32, _I32, _I32, _P, _P, _P]
        L.taot_topology_pref.restype = ctypes.c_int
        L.taot_topology_pref.argtypes = [_P, _I32, _P, _P]
        _lib = L
        _devices = torch.cuda.device_count()
    return _lib


def _stream(stream) -> ctypes.c_void_p:
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _queue(stream, device) -> int:
    """The handle of the stream, or of the device's current one (without a torch.cuda.Stream for it: 3 us a call)."""
    return torch._C._cuda_getCurrentRawStream(device.index) if stream is None else stream.cuda_stream


def _dev(t: torch.Tensor, name: str, dtype) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _check(fn: str, code: int):
    if code != 0:
        raise TaotError(fn, code)


def _workspace(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device)


@dataclasses.dataclass
class Loads:
    n: torch.Tensor        # [B][R][E] int32
    load_e: torch.Tensor   # [B][E] int64
    load_r: torch.Tensor   # [B][R] int64
    excess: torch.Tensor   # [B][R] int64
    spare: torch.Tensor    # [B][R] int64
    spill: torch.Tensor    # [B][E] int64
    supply: torch.Tensor   # [B][R] float32
    demand: torch.Tensor   # [B][R] float32
    rho: torch.Tensor      # [B] float64
    alpha: torch.Tensor    # [B] float64
    bad_ids: torch.Tensor  # [B] int64
    status: torch.Tensor   # [B] int32 (uint32 bits)
    hot_idx: Optional[torch.Tensor] = None   # [B][R] int32: ranks with excess > 0, ascending, then -1
    cold_idx: Optional[torch.Tensor] = None  # [B][R] int32: ranks with spare > 0, ascending, then -1
    hot_cnt: Optional[torch.Tensor] = None   # [B] int32
    cold_cnt: Optional[torch.Tensor] = None  # [B] int32


def plan_loads(ids: torch.Tensor, home: torch.Tensor, E: int, out: Optional[Loads] = None,
               workspace: Optional[torch.Tensor] = None, stream=None) -> Loads:
    """Steps 1-2: histogram n_re and the load marginals (taot_plan_loads)."""
    _dev(ids, "ids", torch.int32)
    _dev(home, "home", torch.int32)
    B, R, N = ids.shape
    dev = ids.device
    if out is None:
        out = Loads(*(torch.empty(s, dtype=d, device=dev) for s, d in (
            ((B, R, E), torch.int32), ((B, E), torch.int64), ((B, R), torch.int64), ((B, R), torch.int64),
            ((B, R), torch.int64), ((B, E), torch.int64), ((B, R), torch.float32), ((B, R), torch.float32),
            ((B,), torch.float64), ((B,), torch.float64), ((B,), torch.int64), ((B,), torch.int32))))
    if out.hot_idx is None:
        out.hot_idx = torch.empty((B, R), dtype=torch.int32, device=dev)
        out.cold_idx = torch.empty((B, R), dtype=torch.int32, device=dev)
        out.hot_cnt = torch.empty((B,), dtype=torch.int32, device=dev)
        out.cold_cnt = torch.empty((B,), dtype=torch.int32, device=dev)
    need = lib().taot_plan_loads_workspace_size(B, R, E)
    ws = workspace if workspace is not None else _workspace(need, dev)
    _check("taot_plan_loads", lib().taot_plan_loads(
        ids.data_ptr(), B, R, N, E, home.data_ptr(), out.n.data_ptr(), out.load_e.data_ptr(),
        out.load_r.data_ptr(), out.excess.data_ptr(), out.spare.data_ptr(), out.spill.data_ptr(),
        out.supply.data_ptr(), out.demand.data_ptr(), out.rho.data_ptr(), out.alpha.data_ptr(),
        out.bad_ids.data_ptr(), _ptr(out.hot_idx), _ptr(out.cold_idx), _ptr(out.hot_cnt), _ptr(out.cold_cnt),
        out.status.data_ptr(), ws.data_ptr(), ws.numel(), _stream(stream)))
    return out


@dataclasses.dataclass
class Flow:
    T: torch.Tensor        # [B][R][R] float32
    f: torch.Tensor        # [B][R] float32
    g: torch.Tensor        # [B][R] float32
    status: torch.Tensor   # [B] int32


def sinkhorn_batched(a: torch.Tensor, b: torch.Tensor, C: torch.Tensor, eps: float, iters: int,
                     flags: int = 0, out: Optional[Flow] = None, workspace: Optional[torch.Tensor] = None,
                     stream=None) -> Flow:
    """Step 3: batched Phase-1 Sinkhorn (taot_sinkhorn_batched).  C is [R][R]
    (shared) or [B][R][R]."""
    _dev(a, "a", torch.float32)
    _dev(b, "b", torch.float32)
    _dev(C, "C", torch.float32)
    B, R = a.shape
    if tuple(b.shape) != (B, R) or tuple(C.shape[-2:]) != (R, R) or C.dim() not in (2, 3):
        raise ValueError("shape mismatch among a, b, C")
    stride = 0 if C.dim() == 2 else R * R
    if C.dim() == 3 and C.shape[0] != B:
        raise ValueError("per-problem C needs B matrices")
    dev = a.device
    if out is None:
        out = Flow(torch.empty((B, R, R), dtype=torch.float32, device=dev),
                   torch.empty((B, R), dtype=torch.float32, device=dev),
                   torch.empty((B, R), dtype=torch.float32, device=dev),
                   torch.empty((B,), dtype=torch.int32, device=dev))
    need = lib().taot_sinkhorn_workspace_size(B, R)
    ws = workspace if workspace is not None else _workspace(need, dev)
    _check("taot_sinkhorn_batched", lib().taot_sinkhorn_batched(
        a.data_ptr(), b.data_ptr(), B, R, C.data_ptr(), stride, float(eps), int(iters), int(flags),
        _ptr(out.T), _ptr(out.f), _ptr(out.g), _ptr(out.status), ws.data_ptr(), ws.numel(), _stream(stream)))
    return out


@dataclasses.dataclass
class Schedule:
    slot_expert: torch.Tensor  # [B][R*K] int32
    slot_amount: torch.Tensor  # [B][R*K] int64
    X: torch.Tensor            # [B][R][R*K] int32
    unfilled: torch.Tensor     # [B] int64
    rounds_used: torch.Tensor  # [B][2] int32
    status: torch.Tensor       # [B] int32


def round_schedule(n, spill, spare, excess, alpha, home, T, Bpref, Bauct, K: int,
                   price_step: float = 2.0 ** -6, t_max: int = 0, out: Optional[Schedule] = None,
                   workspace: Optional[torch.Tensor] = None, stream=None, flags: int = 0) -> Schedule:
    """Steps 4-5: Phase-2 matching and Phase-3 auction (taot_round_schedule).
    flags: SCH_NO_TOPO / SCH_NO_FLOW drop a Phase-2 score term, SCH_ROW_PRIORITY matches
    from the experts' side (ablations)."""
    _dev(n, "n", torch.int32)
    for name, t in (("spill", spill), ("spare", spare), ("excess", excess)):
        _dev(t, name, torch.int64)
    _dev(alpha, "alpha", torch.float64)
    _dev(home, "home", torch.int32)
    _dev(T, "T", torch.float32)
    _dev(Bpref, "Bpref", torch.float64)
    _dev(Bauct, "Bauct", torch.float64)
    B, R, E = n.shape
    S = R * K
    dev = n.device
    if out is None:
        out = Schedule(torch.empty((B, S), dtype=torch.int32, device=dev),
                       torch.empty((B, S), dtype=torch.int64, device=dev),
                       torch.empty((B, R, S), dtype=torch.int32, device=dev),
                       torch.empty((B,), dtype=torch.int64, device=dev),
                       torch.empty((B, 2), dtype=torch.int32, device=dev),
                       torch.empty((B,), dtype=torch.int32, device=dev))
    need = lib().taot_round_schedule_workspace_size(B, R, E, K)
    ws = workspace if workspace is not None else _workspace(need, dev)
    _check("taot_round_schedule", lib().taot_round_schedule(
        n.data_ptr(), spill.data_ptr(), spare.data_ptr(), excess.data_ptr(), alpha.data_ptr(),
        home.data_ptr(), T.data_ptr(), Bpref.data_ptr(), Bauct.data_ptr(), B, R, E, K, float(price_step),
        int(t_max), int(flags), _ptr(out.slot_expert), _ptr(out.slot_amount), _ptr(out.X), _ptr(out.unfilled),
        _ptr(out.rounds_used), _ptr(out.status), ws.data_ptr(), ws.numel(), _stream(stream)))
    return out


def topology_pref(C: np.ndarray):
    """Host helper (taot_topology_pref): (Bpref, Bauct) fp64 [R][R] from a cost matrix."""
    C = np.ascontiguousarray(C, dtype=np.float32)
    R = C.shape[0]
    Bp = np.empty((R, R), np.float64)
    Ba = np.empty((R, R), np.float64)
    _check("taot_topology_pref", lib().taot_topology_pref(C.ctypes.data, R, Bp.ctypes.data, Ba.ctypes.data))
    return Bp, Ba


def workspace_bytes(B: int, R: int, E: int, K: int) -> dict:
    L = lib()
    return dict(plan_loads=L.taot_plan_loads_workspace_size(B, R, E),
                sinkhorn=L.taot_sinkhorn_workspace_size(B, R),
                round_schedule=L.taot_round_schedule_workspace_size(B, R, E, K))


@dataclasses.dataclass
class Plan:
    loads: Loads
    flow: Flow
    schedule: Schedule


def plan_step(ids, home, C, E: int, eps: float, iters: int, K: int, Bpref=None, Bauct=None,
              price_step: float = 2.0 ** -6, t_max: int = 0, stream=None, flags: int = 0) -> Plan:
    """One full planner step over all B problems (three enqueued calls, no sync)."""
    if Bpref is None or Bauct is None:
        Bp, Ba = topology_pref(C.detach().cpu().numpy() if isinstance(C, torch.Tensor) else C)
        Bpref = torch.from_numpy(Bp).to(ids.device)
        Bauct = torch.from_numpy(Ba).to(ids.device)
    loads = plan_loads(ids, home, E, stream=stream)
    flow = sinkhorn_batched(loads.supply, loads.demand, C, eps, iters, stream=stream)
    sched = round_schedule(loads.n, loads.spill, loads.spare, loads.excess, loads.alpha, home, flow.T,
                           Bpref, Bauct, K, price_step, t_max, stream=stream, flags=flags)
    return Plan(loads, flow, sched)


# ---- around the planner: the ids' source, and a plan's execution on the tokens ----

_DTYPE = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}


def _rows(t: torch.Tensor, name: str, like: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Checks a contiguous GPU tensor of bfloat16, float16 or float32 (the type of `like`)."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if t.dtype not in _DTYPE or (like is not None and t.dtype != like.dtype):
        want = "bfloat16, float16 or float32" if like is None else like.dtype
        raise TypeError(f"{name} must be {want}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _shape(t: torch.Tensor, name: str, shape):
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")


def _inputs(fn: str, names: str, stream, *tensors):
    """Refuses tensors (and a stream) of several devices, and inputs whose gradient is being recorded: these calls are
    no part of torch's graph, and their results would carry none."""
    if torch.is_grad_enabled():
        for i, t in enumerate(tensors):
            if t is not None and t.requires_grad:
                raise RuntimeError(f"{names.split()[i]} requires a gradient, which {fn} does not record: detach it or "
                                   "call under torch.no_grad(), and take the gradients from the *_backward calls")
    if _devices == 1:
        return
    dev = tensors[0].get_device()
    for i, t in enumerate(tensors):
        if t is not None and t.get_device() != dev:
            raise ValueError(f"{names.split()[i]} is on cuda:{t.get_device()}, {names.split()[0]} on cuda:{dev}")
    if stream is not None and stream.device_index != dev:
        raise ValueError(f"the stream is of cuda:{stream.device_index}, {names.split()[0]} on cuda:{dev}")


def _launch(fn: str, device, stream, *args):
    """Calls the library with the tensors' device as the current one, which a launch goes to."""
    call = getattr(lib(), fn)
    if _devices == 1 or torch._C._cuda_getDevice() == device.index:
        code = call(*args, _queue(stream, device))
    else:
        with torch.cuda.device(device):
            code = call(*args, _queue(stream, device))
    if code != 0:
        raise TaotError(fn, code)


def _empty(shape, dtype, device, stream) -> torch.Tensor:
    """New memory of the stream that the call's work goes to: what used it before is done when that work begins, and
    it is not handed out again before that work is done."""
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _on(t: torch.Tensor, name: str, device):
    if _devices != 1 and t.get_device() != device.index:
        raise ValueError(f"{name} is on cuda:{t.get_device()}, the inputs on {device}")


def _into(t: Optional[torch.Tensor], name: str, shape, dtype, device, stream) -> torch.Tensor:
    """The caller's output tensor, checked, or a new one."""
    if t is None:
        return (torch.empty(tuple(shape), dtype=dtype, device=device) if stream is None else
                _empty(shape, dtype, device, stream))
    _shape(_dev(t, name, dtype), name, shape)
    _on(t, name, device)
    return t


def _like(t: Optional[torch.Tensor], name: str, x: torch.Tensor, stream) -> torch.Tensor:
    """The caller's output tensor of the shape and type of x, checked, or a new one."""
    if t is None and stream is None:
        return torch.empty_like(x)
    return _into(t, name, x.shape, x.dtype, x.device, stream)


def _room(workspace: Optional[torch.Tensor], nbytes: int, device, stream) -> torch.Tensor:
    if workspace is None:
        return _into(None, "workspace", (max(int(nbytes), 1),), torch.uint8, device, stream)
    if not isinstance(workspace, torch.Tensor):
        raise TypeError("workspace must be a GPU tensor")
    if not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous GPU tensor")
    _on(workspace, "workspace", device)
    return workspace


def _weight(t: torch.Tensor, like: torch.Tensor, H: int):
    f32 = isinstance(t, torch.Tensor) and t.dtype == torch.float32
    _shape(_rows(t, "weight", None if f32 else like), "weight", (H,))


@dataclasses.dataclass
class Norm:
    y: Optional[torch.Tensor] = None      # [..., H], x's type
    q: Optional[torch.Tensor] = None      # [..., H] float8_e4m3fn
    scale: Optional[torch.Tensor] = None  # [..., ceil(H / group)] float32 ([..., 1] for group = 0)
    rstd: Optional[torch.Tensor] = None   # [...] float32
    h: Optional[torch.Tensor] = None      # [..., H], x's type: x + residual (x itself without a residual)
    h_is_x: bool = False                  # h is the x of a call without a residual: no memory to write a sum to


def add_rms_norm(x: torch.Tensor, weight: torch.Tensor, eps: float, residual: Optional[torch.Tensor] = None,
                 group: Optional[int] = None, out: Optional[Norm] = None, stream=None) -> Norm:
    """h = x + residual, y = h * rsqrt(mean(h^2) + eps) * weight over the last dimension (taot_add_rms_norm).
    weight: [H] of x's type or float32.  group: also y in 8 bits with a scale for each `group` columns (a power
    of two from 8 to 512), 0: one scale a row; None: no 8-bit output, and none left in out.  out: tensors to write
    to, or an earlier call's result to use again."""
    _rows(x, "x")
    H = x.shape[-1] if x.dim() else 0
    _weight(weight, x, H)
    if residual is not None:
        _shape(_rows(residual, "residual", x), "residual", x.shape)
    _inputs("add_rms_norm", "x weight residual", stream, x, weight, residual)
    lead, dev = x.shape[:-1], x.device
    if out is None:
        out = Norm()
    y = _like(out.y, "out.y", x, stream)
    rstd = _into(out.rstd, "out.rstd", lead, torch.float32, dev, stream)
    h = x if residual is None else _like(None if out.h_is_x else out.h, "out.h", x, stream)
    q = s = None
    if group is not None:
        q = _into(out.q, "out.q", x.shape, torch.float8_e4m3fn, dev, stream)
        n = -(-H // group) if group > 0 else 1
        s = _into(out.scale, "out.scale", (*lead, n), torch.float32, dev, stream)
    T = x.numel() // H if H else 0
    _launch("taot_add_rms_norm", dev, stream,
        x.data_ptr(), _ptr(residual), weight.data_ptr(), T, H, _DTYPE[x.dtype], _DTYPE[weight.dtype], float(eps),
        int(group or 0), None if residual is None else h.data_ptr(), y.data_ptr(), _ptr(q), _ptr(s), rstd.data_ptr())
    # all of it at once: nothing of an earlier call stays beside this one's, and a refused call changes nothing
    out.y, out.q, out.scale, out.rstd, out.h, out.h_is_x = y, q, s, rstd, h, residual is None
    return out


@dataclasses.dataclass
class NormGrad:
    dx: Optional[torch.Tensor] = None       # [..., H], h's type: the gradient of x and of the residual
    dweight: Optional[torch.Tensor] = None  # [H] float32


def add_rms_norm_backward(dy: torch.Tensor, h: torch.Tensor, rstd: torch.Tensor, weight: torch.Tensor,
                          dh: Optional[torch.Tensor] = None, out: Optional[NormGrad] = None,
                          workspace: Optional[torch.Tensor] = None, stream=None) -> NormGrad:
    """Gradient of add_rms_norm (taot_add_rms_norm_backward) from its h and rstd: dy reaches y, dh reaches h."""
    _rows(h, "h")
    H = h.shape[-1] if h.dim() else 0
    _shape(_rows(dy, "dy", h), "dy", h.shape)
    if dh is not None:
        _shape(_rows(dh, "dh", h), "dh", h.shape)
    _weight(weight, h, H)
    _shape(_dev(rstd, "rstd", torch.float32), "rstd", h.shape[:-1])
    _inputs("add_rms_norm_backward", "dy h rstd weight dh", stream, dy, h, rstd, weight, dh)
    if out is None:
        out = NormGrad()
    out.dx = _like(out.dx, "out.dx", h, stream)
    out.dweight = _into(out.dweight, "out.dweight", (H,), torch.float32, h.device, stream)
    T = h.numel() // H if H else 0
    ws = _room(workspace, lib().taot_add_rms_norm_backward_workspace_size(T, H), h.device, stream)
    _launch("taot_add_rms_norm_backward", h.device, stream,
        dy.data_ptr(), _ptr(dh), h.data_ptr(), rstd.data_ptr(), weight.data_ptr(), T, H, _DTYPE[h.dtype],
        _DTYPE[weight.dtype], out.dx.data_ptr(), out.dweight.data_ptr(), ws.data_ptr(),
        ws.numel() * ws.element_size())
    return out


@dataclasses.dataclass
class Routing:
    ids: Optional[torch.Tensor] = None      # [..., top_k] int32, -1: none
    weights: Optional[torch.Tensor] = None  # [..., top_k] float32


def route(logits: torch.Tensor, top_k: int, bias: Optional[torch.Tensor] = None, groups: int = 1,
          top_groups: int = 1, scale: float = 1.0, flags: int = 0, out: Optional[Routing] = None,
          stream=None) -> Routing:
    """Chooses top_k of the E experts of each token by logits [..., E] and weighs them (taot_route; flags ROUTE_*).
    With logits [B][R][tokens][E], ids.view(B, R, -1) is plan_loads' input."""
    _rows(logits, "logits")
    E = logits.shape[-1] if logits.dim() else 0
    if bias is not None:
        _shape(_dev(bias, "bias", torch.float32), "bias", (E,))
    _inputs("route", "logits bias", stream, logits, bias)
    shape = (*logits.shape[:-1], top_k)
    if out is None:
        out = Routing()
    out.ids = _into(out.ids, "out.ids", shape, torch.int32, logits.device, stream)
    out.weights = _into(out.weights, "out.weights", shape, torch.float32, logits.device, stream)
    T = logits.numel() // E if E else 0
    _launch("taot_route", logits.device, stream,
        logits.data_ptr(), _ptr(bias), T, E, int(top_k), int(groups), int(top_groups), float(scale), int(flags),
        _DTYPE[logits.dtype], out.ids.data_ptr(), out.weights.data_ptr())
    return out


def route_backward(dweights: torch.Tensor, logits: torch.Tensor, ids: torch.Tensor, scale: float = 1.0,
                   flags: int = 0, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Gradient of route's weights by the logits (taot_route_backward): [..., E] of the logits' type."""
    _rows(logits, "logits")
    E = logits.shape[-1] if logits.dim() else 0
    top_k = ids.shape[-1] if _dev(ids, "ids", torch.int32).dim() else 0
    shape = (*logits.shape[:-1], top_k)
    _shape(ids, "ids", shape)
    _shape(_dev(dweights, "dweights", torch.float32), "dweights", shape)
    _inputs("route_backward", "logits ids dweights", stream, logits, ids, dweights)
    out = _like(out, "out", logits, stream)
    T = logits.numel() // E if E else 0
    _launch("taot_route_backward", logits.device, stream,
        dweights.data_ptr(), logits.data_ptr(), ids.data_ptr(), T, E, top_k, float(scale), int(flags),
        _DTYPE[logits.dtype], out.data_ptr())
    return out


@dataclasses.dataclass
class Dispatch:
    pos: Optional[torch.Tensor] = None      # [B][rows][N] int32 row of the send buffer (p < 0: nowhere)
    offsets: Optional[torch.Tensor] = None  # [B][rows][E + R*K + 1] int32 first row of each instance
    sends: Optional[torch.Tensor] = None    # [B][rows][R] int32 copies for each rank
    status: Optional[torch.Tensor] = None   # [B] int32 (uint32 bits)


def dispatch_map(ids: torch.Tensor, home: torch.Tensor, slot_expert: torch.Tensor, X: torch.Tensor, K: int,
                 rank0: int = 0, out: Optional[Dispatch] = None, workspace: Optional[torch.Tensor] = None,
                 stream=None) -> Dispatch:
    """Where a schedule sends each routed copy (taot_dispatch_map).  ids [B][rows][N] of the source ranks rank0 ..
    rank0 + rows - 1; slot_expert [B][R*K] and X [B][R][R*K] of the schedule."""
    _dev(ids, "ids", torch.int32)
    _dev(home, "home", torch.int32)
    _dev(slot_expert, "slot_expert", torch.int32)
    _dev(X, "X", torch.int32)
    if ids.dim() != 3 or X.dim() != 3 or home.dim() != 1:
        raise ValueError("ids must be [B][rows][N], X [B][R][R*K] and home [E]")
    B, rows, N = ids.shape
    E, R = home.shape[0], X.shape[1]
    S = R * K
    _shape(X, "X", (B, R, S))
    _shape(slot_expert, "slot_expert", (B, S))
    _inputs("dispatch_map", "ids home slot_expert X", stream, ids, home, slot_expert, X)
    dev = ids.device
    if out is None:
        out = Dispatch()
    out.pos = _like(out.pos, "out.pos", ids, stream)
    out.offsets = _into(out.offsets, "out.offsets", (B, rows, E + S + 1), torch.int32, dev, stream)
    out.sends = _into(out.sends, "out.sends", (B, rows, R), torch.int32, dev, stream)
    out.status = _into(out.status, "out.status", (B,), torch.int32, dev, stream)
    ws = _room(workspace, lib().taot_dispatch_map_workspace_size(B, rows, N, R, E, K), dev, stream)
    _launch("taot_dispatch_map", dev, stream,
        ids.data_ptr(), B, rows, int(rank0), N, home.data_ptr(), R, E, int(K), slot_expert.data_ptr(), X.data_ptr(),
        out.pos.data_ptr(), out.offsets.data_ptr(), out.sends.data_ptr(), out.status.data_ptr(), ws.data_ptr(),
        ws.numel() * ws.element_size())
    return out


def _tokens(pos: torch.Tensor, lead, name: str):
    """(rows, tokens, top_k) of positions [..., N] and a tensor of shape [*lead, tokens, ...]."""
    _dev(pos, "pos", torch.int32)
    if not pos.dim() or not len(lead):
        raise ValueError(f"{name} must be [..., rows, H] and pos [..., N]")
    N, tokens = pos.shape[-1], lead[-1]
    if tuple(pos.shape[:-1]) != tuple(lead[:-1]) or (N % tokens if tokens else N):
        raise ValueError(f"{name} of {tuple(lead)} tokens does not go with positions of shape {tuple(pos.shape)}")
    rows = 1
    for d in lead[:-1]:
        rows *= d
    return rows, tokens, N // tokens if tokens else 1


def _sent(y: torch.Tensor, pos: torch.Tensor):
    """Checks rows of a send buffer and the positions in it."""
    if _rows(y, "y").dim() < 2:
        raise ValueError(f"y must be [..., N, H], got {tuple(y.shape)}")
    _shape(_dev(pos, "pos", torch.int32), "pos", y.shape[:-1])


def dispatch_rows(x: torch.Tensor, pos: torch.Tensor, scale: Optional[torch.Tensor] = None,
                  out: Optional[torch.Tensor] = None, out_scale: Optional[torch.Tensor] = None, stream=None):
    """Tokens' rows x [..., tokens, H] (any type) at their places of the send buffer, [..., N, H] for pos [..., N]
    (taot_dispatch_rows).  With scale [..., tokens, G]: (rows, scales).  Its gradient is combine_rows, no weights."""
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise TypeError("x must be a GPU tensor")
    if not x.is_contiguous():
        raise ValueError("x must be contiguous")
    lead = x.shape[:-1]
    rows, tokens, k = _tokens(pos, lead, "x")
    if scale is not None:
        _shape(_dev(scale, "scale", torch.float32), "scale", (*lead, scale.shape[-1] if scale.dim() else 1))
    _inputs("dispatch_rows", "x pos scale", stream, x, pos, scale)
    out = _into(out, "out", (*pos.shape, x.shape[-1]), x.dtype, x.device, stream)
    more = 0
    if scale is not None:
        out_scale = _into(out_scale, "out_scale", (*pos.shape, scale.shape[-1]), torch.float32, x.device, stream)
        more = 4 * scale.shape[-1]
    _launch("taot_dispatch_rows", x.device, stream,
        x.data_ptr(), x.shape[-1] * x.element_size(), _ptr(scale), more, rows, tokens, k, pos.data_ptr(),
        out.data_ptr(), _ptr(out_scale) if scale is not None else None)
    return out if scale is None else (out, out_scale)


def combine_rows(y: torch.Tensor, pos: torch.Tensor, weights: Optional[torch.Tensor] = None, top_k: int = 1,
                 out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Weighted sum of each token's top_k rows of y [..., N, H] back in the tokens' order, [..., N / top_k, H]
    (taot_combine_rows).  weights [..., N] float32 or None (all 1), as route gives them: [..., tokens, top_k] too."""
    _sent(y, pos)
    N, H = y.shape[-2:]
    if top_k < 1 or N % top_k:
        raise ValueError(f"{N} copies are not top_k = {top_k} of each token")
    if weights is not None and _dev(weights, "weights", torch.float32).numel() != pos.numel():
        raise ValueError("weights must have a value for each copy")
    _inputs("combine_rows", "y pos weights", stream, y, pos, weights)
    lead = (*y.shape[:-2], N // top_k)
    out = _into(out, "out", (*lead, H), y.dtype, y.device, stream)
    rows, tokens, _ = _tokens(pos, lead, "y")
    _launch("taot_combine_rows", y.device, stream,
        y.data_ptr(), pos.data_ptr(), _ptr(weights), rows, tokens, int(top_k), H, _DTYPE[y.dtype], out.data_ptr())
    return out


@dataclasses.dataclass
class CombineGrad:
    dy: Optional[torch.Tensor] = None        # [..., N, H], y's type
    dweights: Optional[torch.Tensor] = None  # [..., N] float32

    def __iter__(self):
        return iter((self.dy, self.dweights))


def combine_rows_backward(dout: torch.Tensor, y: torch.Tensor, pos: torch.Tensor, weights: torch.Tensor,
                          out: Optional[CombineGrad] = None, stream=None) -> CombineGrad:
    """Gradient of combine_rows by y and the weights (taot_combine_rows_backward).  Without weights the gradient is
    dispatch_rows(dout, pos)."""
    _sent(y, pos)
    _rows(dout, "dout", y)
    H = y.shape[-1]
    rows, tokens, k = _tokens(pos, dout.shape[:-1], "dout")
    _shape(dout, "dout", (*dout.shape[:-1], H))
    if _dev(weights, "weights", torch.float32).numel() != pos.numel():
        raise ValueError("weights must have a value for each copy")
    _inputs("combine_rows_backward", "y pos dout weights", stream, y, pos, dout, weights)
    if out is None:
        out = CombineGrad()
    out.dy = _like(out.dy, "out.dy", y, stream)
    out.dweights = _like(out.dweights, "out.dweights", weights, stream)
    _launch("taot_combine_rows_backward", y.device, stream,
        dout.data_ptr(), y.data_ptr(), pos.data_ptr(), weights.data_ptr(), rows, tokens, k, H, _DTYPE[y.dtype],
        out.dy.data_ptr(), out.dweights.data_ptr())
    return out


@dataclasses.dataclass
class Quality:
    load_after: torch.Tensor  # [B][R] int64 rank loads once the planned tokens moved
    rho_after: torch.Tensor   # [B] float64 (R * max load - L) / L, 0 if L = 0
    intra: torch.Tensor       # [B] int64 replicas hosted in their expert's home node
    inter: torch.Tensor       # [B] int64 replicas hosted in another node
    weighted: torch.Tensor    # [B] float64 intra + w_inter * inter


def plan_quality(load_r: torch.Tensor, home: torch.Tensor, sched: Schedule, K: int,
                 ranks_per_node: int = 8, w_inter: float = 3.0) -> Quality:
    """Plan-quality metrics of one schedule per problem (Sec. 4.1): the
    imbalance left after the planned tokens move from each expert's home rank
    to the ranks hosting its replicas, and the replicas placed inside and
    across nodes (node = rank // ranks_per_node), weighted intra + w_inter *
    inter.  Evaluation of a plan, not a planner step: plain tensor ops on the
    schedule's device."""
    se = sched.slot_expert.long()
    B, S = se.shape
    R = load_r.shape[1]
    valid = se >= 0
    moved = sched.X.sum(dim=1, dtype=torch.int64) * valid           # [B][S]
    host = (torch.arange(S, device=se.device) // K).expand(B, S)      # [B][S]
    h = home.long()[se.clamp(min=0)]                                  # [B][S]
    la = load_r.to(torch.int64).clone()
    la.scatter_add_(1, h, -moved)
    la.scatter_add_(1, host, moved)
    L = load_r.to(torch.int64).sum(1)
    lmax = la.max(1).values
    rho = torch.where(L > 0, (R * lmax - L).double() / L.clamp(min=1).double(),
                      torch.zeros_like(L, dtype=torch.float64))
    same = (h // ranks_per_node) == (host // ranks_per_node)
    intra = (valid & same).sum(1)
    inter = (valid & ~same).sum(1)
    return Quality(la, rho, intra, inter, intra.double() + w_inter * inter.double())


def plan_report(plan: Plan, home: torch.Tensor, K: int, problems=None, ranks_per_node: int = 8,
                w_inter: float = 3.0) -> str:
    """Text report of a finished plan, one block per chosen problem (layer),
    in the four parts of the planner log described in Appendix B.3:
    [1] every rank's load, ranks above the integer mean starred, and each
        expert that spills, with its home rank, load and spill;
    [2] one line per filled guest slot (expert, its home rank, the hosting
        rank and slot, same node or not, tokens the slot receives), then the
        copy counts and their weighted cost;
    [3] every rank's load once the planned tokens have moved;
    [4] rho and the largest rank load before and after, the share of all
        tokens sent to a replica, and the copy counts and cost.
    Formats on the host what the plan already holds."""
    L, sched = plan.loads, plan.schedule
    q = plan_quality(L.load_r, home, sched, K, ranks_per_node, w_inter)
    load_r, load_e = L.load_r.cpu().numpy(), L.load_e.cpu().numpy()
    excess, spill = L.excess.cpu().numpy(), L.spill.cpu().numpy()
    rho0, la, rho1 = L.rho.cpu().numpy(), q.load_after.cpu().numpy(), q.rho_after.cpu().numpy()
    se, X = sched.slot_expert.cpu().numpy(), sched.X.cpu().numpy()
    hm = home.cpu().numpy()
    B, R = load_r.shape
    problems = range(B) if problems is None else problems
    out = []

    def ranks(vals, marks=None):
        cells = [f"{r:4d}:{int(v):>9d}{'*' if marks is not None and marks[r] else ' '}" for r, v in enumerate(vals)]
        return ["   " + " ".join(cells[i:i + 8]) for i in range(0, len(cells), 8)]

    for b in problems:
        tot = int(load_r[b].sum())
        mean = tot / R if R else 0.0
        out.append(f"== plan report, problem {b}: R = {R}, E = {hm.shape[0]}, K = {K}, "
                   f"L = {tot}, mean {mean:.1f} ==")
        out.append("[1] load before routing (* hot rank: load above the integer mean)")
        out += ranks(load_r[b], excess[b] > 0)
        hot = np.nonzero(spill[b] > 0)[0]
        out.append(f"    hot experts (spill > 0): {len(hot)}")
        for e in hot:
            out.append(f"      expert {e:5d} on rank {hm[e]:4d}: load {int(load_e[b, e])}, spill {int(spill[b, e])}")
        out.append("[2] cloning plan")
        moved_tot, ni, no = 0, 0, 0
        for s_ in np.nonzero(se[b] >= 0)[0]:
            e, host = int(se[b, s_]), int(s_) // K
            moved = int(X[b, :, s_].sum())
            moved_tot += moved
            intra = hm[e] // ranks_per_node == host // ranks_per_node
            ni, no = ni + intra, no + (not intra)
            out.append(f"      expert {e:5d} (rank {hm[e]:4d}) -> slot {s_ % K} of rank {host:4d}: "
                       f"{'intra' if intra else 'inter'}-node, {moved} tokens")
        out.append(f"    topology: {ni} intra-node, {no} inter-node copies; weighted cost "
                   f"{ni + w_inter * no:.1f} (intra + {w_inter:g} x inter)")
        out.append("[3] projected load after routing")
        out += ranks(la[b])
        pk0, pk1 = int(load_r[b].max()), int(la[b].max())
        out.append("[4] summary")
        out.append(f"    imbalance rho {rho0[b]:.4f} -> {rho1[b]:.4f}; peak load {pk0} -> {pk1} "
                   f"({100.0 * (pk0 - pk1) / pk0 if pk0 else 0.0:.1f} % lower); rerouted {moved_tot} of "
                   f"{tot} tokens ({100.0 * moved_tot / tot if tot else 0.0:.2f} %); "
                   f"copies {ni} intra / {no} inter, weighted cost {ni + w_inter * no:.1f}")
    return "\n".join(out) + "\n"
