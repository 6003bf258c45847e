"""Python binding of libmoesched (argument marshalling only).

Every step of the path -- greedy max-weight decomposition (paper Sec. 3.2),
Birkhoff-von Neumann decomposition (Sec. 3.1) and schedule scoring (Sec. 4.1) --
runs in the CUDA kernels behind the C ABI declared in include/moesched.h.
PyTorch is used for device memory and streams only. There is no CPU fallback:
a missing library or a non-CUDA tensor raises.
"""
from __future__ import annotations

import ctypes
import math
import os
from dataclasses import dataclass

import torch

from .workload import DEFAULT_MODEL, PROFILED_MODEL, bvn_capacity  # noqa: F401  (re-exported)

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmoesched.so")

ST_OK, ST_TRUNCATED, ST_BAD_INPUT, ST_INTERNAL = 0, 1, -1, -2
WORK_FIELDS = 10
MAX_N = 256


class MoeschedError(RuntimeError):
    pass


class _Model(ctypes.Structure):
    _fields_ = [("bytes_per_token", ctypes.c_int64), ("link_gbps", ctypes.c_int64),
                ("reconfig_ns", ctypes.c_int64), ("expert_fixed_ns", ctypes.c_int64),
                ("expert_ps_per_token", ctypes.c_int64), ("expert_knee_tokens", ctypes.c_int64)]


class _PathArgs(ctypes.Structure):
    """moesched_path_t of include/moesched.h."""
    _fields_ = ([(n, ctypes.c_int64) for n in ("k_mw", "k_bvn", "score_stride")] +
                [(n, ctypes.c_void_p) for n in (
                    "mw_perm", "bvn_perm", "mw_dur", "mw_count", "mw_status", "mw_eval_status", "bvn_coef", "bvn_count",
                    "bvn_status", "bvn_eval_status", "mw_work", "bvn_work", "mw_scores", "bvn_scores", "bvn_scratch",
                    "side_stream", "fork_event", "join_event", "done_event")])


_lib = None

# Argument types of the entry points: i = int, p = pointer (an address, or None), q = int64, d = double. With them declared,
# addresses go in as plain integers.
_ARGTYPES = {"i": ctypes.c_int, "p": ctypes.c_void_p, "q": ctypes.c_int64, "d": ctypes.c_double}
_SIGNATURES = {
    "moesched_mw_decompose": "iipippppppp", "moesched_bvn_decompose": "iipipppppppp",
    "moesched_bvn_decompose_static": "iipippppppp", "moesched_schedule_eval": "iipippp" + "p" * 8,
    "moesched_schedule_prefix_eval": "iipippp" + "p" * 10, "moesched_ideal_a2a": "iipppppp",
    "moesched_sinkhorn_scale": "iipidipppppp", "moesched_sinkhorn_durations": "iipppipp",
    "moesched_schedule_order": "iipippp" + "p" * 8, "moesched_schedule_permute": "iiipppppp",
    "moesched_best_budget": "iipppqppp", "moesched_bvn_real_decompose": "iipdipppppppp",
    "moesched_route_demand": "iiii" + "p" * 6, "moesched_schedule_slots": "iipipppi" + "p" * 9,
    "moesched_expert_ffn": "i" * 7 + "p" * 11, "moesched_expert_ffn_backward": "i" * 7 + "p" * 15,
    "moesched_expert_matvec4": "i" * 8 + "p" * 9,
    "moesched_path_run": "piippip", "moesched_last_cuda_error": "",
}


def _open(path):
    if not os.path.exists(path):
        raise MoeschedError(f"{path} is missing: run `python -m paper_2605_26845_b200.build` "
                            "(there is no CPU fallback)")
    lib = ctypes.CDLL(path)
    lib.moesched_strerror.restype = ctypes.c_char_p
    lib.moesched_status_str.restype = ctypes.c_char_p
    lib.moesched_workspace_bytes.restype = ctypes.c_size_t
    for name, signature in _SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = ctypes.c_int, [_ARGTYPES[c] for c in signature]
    lib.moesched_bvn_scratch_bytes.restype = ctypes.c_size_t
    lib.moesched_order_scratch_bytes.restype = ctypes.c_size_t
    lib.moesched_expert_scratch_bytes.restype = ctypes.c_size_t
    lib.moesched_slots_scratch_bytes.restype = ctypes.c_size_t
    lib.moesched_probe_int_ops.restype = ctypes.c_longlong
    lib.moesched_debug_index_faults.restype = ctypes.c_longlong
    return lib


def load_library():
    """dlopen libmoesched.so (built in-tree by paper_2605_26845_b200/build.py)."""
    global _lib
    if _lib is None:
        _lib = _open(LIB_PATH)
    return _lib


def use_library(path=None):
    """Route every call of this binding through another build of the library, e.g. the checked one
    (libmoesched_checked.so, see build.py); None goes back to the regular library. Returns the path."""
    global _lib
    path = LIB_PATH if path is None else path
    _lib = _open(path)
    return path


def debug_index_faults() -> int:
    """Out-of-range indices the checked build has caught on the current device (-1: no checks compiled in)."""
    return int(load_library().moesched_debug_index_faults())


def _check(rc, what):
    if rc != 0:
        lib = load_library()
        msg = lib.moesched_strerror(rc).decode()
        raise MoeschedError(f"{what}: {msg} (rc={rc}, cuda error {lib.moesched_last_cuda_error()})")


def _dev(t, dtype, what):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise MoeschedError(f"{what} must be a CUDA tensor (the library has no CPU path)")
    if t.dtype != dtype or not t.is_contiguous():
        raise MoeschedError(f"{what} must be contiguous {dtype}")
    return t


def _ptr(t):
    return t.data_ptr() if t is not None else None


def _call(name, device, *args):
    """Entry point `name` with `args` and the current stream of `device`, with that device current."""
    index = device.index
    stream = torch._C._cuda_getCurrentRawStream(index)
    fn = getattr(load_library(), name)
    if torch._C._cuda_getDevice() == index:
        rc = fn(*args, stream)
    else:
        with torch.cuda.device(device):
            rc = fn(*args, stream)
    if rc != 0:
        _check(rc, name)


@dataclass
class Schedule:
    """Ordered matchings of a batch: perm [B, k_max, N] uint8 (perm[b, k, i] = destination of
    source i), dur [B, k_max] int32 tokens, count [B], status [B]; extra = residual (greedy) or
    augmented matrix (BvN) if requested; work = per-matrix work counters if requested."""
    perm: torch.Tensor
    dur: torch.Tensor
    count: torch.Tensor
    status: torch.Tensor
    extra: torch.Tensor | None = None
    work: torch.Tensor | None = None


def _new_schedule(demand, k_max, want_extra, want_work):
    B, N, _ = demand.shape
    dev = demand.device
    return Schedule(perm=torch.empty((B, k_max, N), dtype=torch.uint8, device=dev),
                    dur=torch.empty((B, k_max), dtype=torch.int32, device=dev),
                    count=torch.empty(B, dtype=torch.int32, device=dev),
                    status=torch.empty(B, dtype=torch.int32, device=dev),
                    extra=torch.empty_like(demand) if want_extra else None,
                    work=torch.empty((B, WORK_FIELDS), dtype=torch.int64, device=dev) if want_work else None)


def _check_demand(demand):
    demand = _dev(demand, torch.int32, "demand")
    if demand.dim() != 3 or demand.shape[1] != demand.shape[2]:
        raise MoeschedError("demand must have shape [B, N, N]")
    return demand


def mw_decompose(demand, k_max, want_residual=False, want_work=False, out=None) -> Schedule:
    """Greedy max-weight decomposition of every matrix of `demand` [B, N, N] int32 (CUDA)."""
    demand = _check_demand(demand)
    B, N, _ = demand.shape
    if out is None:
        out = _new_schedule(demand, int(k_max), want_residual, want_work)
    _call("moesched_mw_decompose", demand.device, B, N, _ptr(demand), int(k_max), _ptr(out.perm), _ptr(out.dur),
          _ptr(out.count), _ptr(out.extra), _ptr(out.status), _ptr(out.work))
    return out


def bvn_scratch_bytes(B, N) -> int:
    return int(load_library().moesched_bvn_scratch_bytes(int(B), int(N)))


def workspace_bytes(B, N, k_max) -> int:
    """Device working memory a pass of the whole path can use beyond its inputs and outputs."""
    return int(load_library().moesched_workspace_bytes(int(B), int(N), int(k_max)))


def status_str(status) -> str:
    """Text for one per-matrix status value."""
    return load_library().moesched_status_str(int(status)).decode()


def bvn_decompose(demand, k_max=None, want_aug=False, want_work=False, out=None, scratch=True) -> Schedule:
    """Birkhoff-von Neumann decomposition; k_max defaults to N^2 - 2N + 2 (always enough).

    scratch: True allocates the working buffer of the fast path, a uint8 CUDA tensor of at least
    bvn_scratch_bytes(B, N) bytes is used as given, False / None selects the shared-memory path."""
    demand = _check_demand(demand)
    B, N, _ = demand.shape
    dev = demand.device
    if k_max is None:
        k_max = bvn_capacity(N)
    if out is None:
        out = _new_schedule(demand, int(k_max), want_aug, want_work)
    if scratch is True:
        scratch = torch.empty(max(1, bvn_scratch_bytes(B, N)), dtype=torch.uint8, device=dev)
    elif scratch is False:
        scratch = None
    if scratch is not None:
        _dev(scratch, torch.uint8, "scratch")
        if scratch.numel() < bvn_scratch_bytes(B, N):
            raise MoeschedError("scratch is smaller than bvn_scratch_bytes(B, N)")
    _call("moesched_bvn_decompose", dev, B, N, _ptr(demand), int(k_max), _ptr(out.perm), _ptr(out.dur), _ptr(out.count),
          _ptr(out.extra), _ptr(scratch), _ptr(out.status), _ptr(out.work))
    return out


STATIC_SCRATCH_BYTES = 16 * 1024 * 1024


def bvn_decompose_static(demand, out: Schedule) -> Schedule:
    """BvN decomposition through the entry point that allocates nothing: for callers that may
    not allocate device memory (a host framework owns the pool, or an allocation would stall a
    latency-critical loop). `out` must be a complete, caller-made Schedule; the working copy sits
    in the library's built-in 16 MiB array, so B * N * roundup(N, 8) * 4 must fit in it. Calls
    that may overlap on one GPU share that array and must be serialised."""
    demand = _check_demand(demand)
    B, N, _ = demand.shape
    _call("moesched_bvn_decompose_static", demand.device, B, N, _ptr(demand), int(out.perm.shape[1]), _ptr(out.perm),
          _ptr(out.dur), _ptr(out.count), _ptr(out.extra), _ptr(out.status), _ptr(out.work))
    return out


def probe_int_rate(device=None, blocks=148 * 8, iters=20000, reps=3) -> float:
    """Measured integer lane-operations per second of the GPU (add / min / logic mix)."""
    lib = load_library()
    dev = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    out = torch.empty(blocks * 256, dtype=torch.int32, device=dev)
    best = 0.0
    with torch.cuda.device(dev):
        for _ in range(reps + 1):
            e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            e0.record()
            ops = lib.moesched_probe_int_ops(blocks, iters, ctypes.c_void_p(_ptr(out)),
                                             ctypes.c_void_p(torch.cuda.current_stream(dev).cuda_stream))
            e1.record()
            if ops < 0:
                _check(int(ops), "moesched_probe_int_ops")
            e1.synchronize()
            best = max(best, ops / (e0.elapsed_time(e1) * 1e-3))
    return best


def sinkhorn_scale(demand, iters=20, smooth=0.5, scale_bits=20, out=None) -> dict:
    """Sinkhorn-Knopp scaling of a batch (paper Sec. 3.1). Returns scaled [B, N, N] float64, fixed
    [B, N, N] int32 (= round(scaled * 2^scale_bits), the input of bvn_decompose), stretch [B], row_err [B]
    float64 and status [B]; `out` may hand back the dict of an earlier call of the same shape for reuse."""
    demand = _check_demand(demand)
    B, N, _ = demand.shape
    dev = demand.device
    if out is None:
        out = dict(scaled=torch.empty((B, N, N), dtype=torch.float64, device=dev),
                   fixed=torch.empty((B, N, N), dtype=torch.int32, device=dev),
                   stretch=torch.empty(B, dtype=torch.float64, device=dev),
                   row_err=torch.empty(B, dtype=torch.float64, device=dev),
                   status=torch.empty(B, dtype=torch.int32, device=dev))
    else:
        _dev(out["scaled"], torch.float64, "out['scaled']")
        _dev(out["fixed"], torch.int32, "out['fixed']")
        if out["scaled"].shape != demand.shape or out["fixed"].shape != demand.shape:
            raise MoeschedError("out has the wrong shape")
    _call("moesched_sinkhorn_scale", dev, B, N, _ptr(demand), int(iters), float(smooth), int(scale_bits),
          _ptr(out["scaled"]), _ptr(out["fixed"]), _ptr(out["stretch"]), _ptr(out["row_err"]), _ptr(out["status"]))
    return out


def sinkhorn_durations(coef, count, stretch, scale_bits=20, out=None) -> torch.Tensor:
    """Token length of each matching of a decomposition of sinkhorn_scale(...)["fixed"]:
    ceil(coef * stretch / 2^scale_bits) for the first count[b] matchings of every schedule."""
    coef = _dev(coef, torch.int32, "coef")
    count = _dev(count, torch.int32, "count")
    stretch = _dev(stretch, torch.float64, "stretch")
    B, K = coef.shape
    if out is None:
        out = torch.zeros_like(coef)
    _call("moesched_sinkhorn_durations", coef.device, B, K, _ptr(coef), _ptr(count), _ptr(stretch), int(scale_bits),
          _ptr(_dev(out, torch.int32, "out")))
    return out


def bvn_real_decompose(matrix, k_max=None, tol=1e-12) -> dict:
    """Real-valued Birkhoff-von Neumann decomposition A = sum_k lambda_k P_k (paper Sec. 3.1) of [B, N, N]
    float64 matrices, e.g. sinkhorn_scale(...)["scaled"]. Returns perm [B, k_max, N] uint8, lam [B, k_max]
    float64, count, sum_lambda, max_left (largest entry remaining) and status [B]."""
    matrix = _dev(matrix, torch.float64, "matrix")
    if matrix.dim() != 3 or matrix.shape[1] != matrix.shape[2]:
        raise MoeschedError("matrix must have shape [B, N, N]")
    B, N, _ = matrix.shape
    dev = matrix.device
    k_max = bvn_capacity(N) if k_max is None else int(k_max)
    out = dict(perm=torch.empty((B, k_max, N), dtype=torch.uint8, device=dev),
               lam=torch.empty((B, k_max), dtype=torch.float64, device=dev),
               count=torch.empty(B, dtype=torch.int32, device=dev),
               sum_lambda=torch.empty(B, dtype=torch.float64, device=dev),
               max_left=torch.empty(B, dtype=torch.float64, device=dev),
               status=torch.empty(B, dtype=torch.int32, device=dev))
    scratch = torch.empty(max(1, B * N * ((N + 7) // 8 * 8)), dtype=torch.float64, device=dev)
    _call("moesched_bvn_real_decompose", dev, B, N, _ptr(matrix), float(tol), k_max, _ptr(out["perm"]), _ptr(out["lam"]),
          _ptr(out["count"]), _ptr(out["sum_lambda"]), _ptr(out["max_left"]), _ptr(scratch), _ptr(out["status"]))
    return out


_models = {}    # models of plain ints that have been used lately, in their C form (never changed once made)


def _model(model):
    """Reference to the C form of a model dict; it keeps the structure alive for as long as it is held itself, which a call's
    arguments do until the call is over."""
    items = tuple((model or DEFAULT_MODEL).items())
    try:
        made = _models.get(items)
    except TypeError:           # a value that has no hash
        made = None
    if made is None:
        made = _Model(**{k: int(v) for k, v in items})
        if all(type(v) is int for _, v in items):   # (what else is equal to them has the same values)
            if len(_models) >= 256:
                _models.clear()
            _models[items] = made
    return ctypes.byref(made)


def ideal_a2a(demand, model=None) -> dict:
    """Idealised congestion-free all-to-all of every matrix: 'comm_ns' (one exchange at line rate of
    the busiest port), 'makespan_ns' (dispatch + compute + combine, run to completion), 'status'."""
    demand = _check_demand(demand)
    B, N, _ = demand.shape
    dev = demand.device
    m = _model(model)
    comm, makespan = torch.empty((2, B), dtype=torch.int64, device=dev).unbind(0)
    status = torch.empty(B, dtype=torch.int32, device=dev)
    _call("moesched_ideal_a2a", dev, B, N, _ptr(demand), m, _ptr(comm), _ptr(makespan), _ptr(status))
    return {"comm_ns": comm, "makespan_ns": makespan, "status": status}


SCORE_FIELDS = ("makespan_overlap_ns", "makespan_serial_ns", "compute_idle_ns", "link_idle_tokens",
                "unserved_tokens")


def schedule_eval(demand, perm, dur, count, model=None, out=None, status=None, prefix=False) -> dict:
    """Score schedules under the dispatch-compute-combine model. Returns a dict of [B] int64
    tensors (SCORE_FIELDS) plus 'status' [B] int32; `out` may supply a [5, B] int64 tensor and
    `status` a [B] int32 tensor. With prefix=True the dict also holds 'prefix_overlap_ns' and
    'prefix_unserved_tokens', [B, k_stride] int64: the scores of the schedule cut after each
    matching (-1 beyond count)."""
    demand = _dev(demand, torch.int32, "demand")
    perm = _dev(perm, torch.uint8, "perm")
    dur = _dev(dur, torch.int32, "dur")
    count = _dev(count, torch.int32, "count")
    B, N, _ = demand.shape
    if perm.dim() != 3 or perm.shape[0] != B or perm.shape[2] != N or dur.shape != perm.shape[:2]:
        raise MoeschedError("perm must be [B, k_stride, N] and dur [B, k_stride]")
    m = _model(model)
    dev = demand.device
    scores = out if out is not None else torch.empty((5, B), dtype=torch.int64, device=dev)
    if status is None:
        status = torch.empty(B, dtype=torch.int32, device=dev)
    K = int(perm.shape[1])
    pre = torch.empty((2, B, K), dtype=torch.int64, device=dev) if prefix else None
    # (a caller's own may be a sequence, and hold more)
    rows = scores.unbind(0) if out is None else [out[i] for i in range(len(SCORE_FIELDS))]
    args = (B, N, _ptr(demand), K, _ptr(perm), _ptr(dur), _ptr(count), m, *(r.data_ptr() for r in rows), _ptr(status))
    res = dict(zip(SCORE_FIELDS, rows))
    if prefix:
        overlap, unserved = pre.unbind(0)
        _call("moesched_schedule_prefix_eval", dev, *args, _ptr(overlap), _ptr(unserved))
        res["prefix_overlap_ns"], res["prefix_unserved_tokens"] = overlap, unserved
    else:
        _call("moesched_schedule_eval", dev, *args)
    res["status"] = status
    return res


ORDER_MAX_K = 1024


def schedule_order(demand, perm, dur, count, model=None) -> dict:
    """Best of five orders of the matchings on the job times of the emission-order replay (paper
    Sec. 3.3). Returns 'order' [B, k_stride] int32 (position -> original index, -1 beyond count),
    'makespan_ns', 'emission_ns' [B] int64, 'rule', 'status' [B] int32."""
    lib = load_library()
    demand = _check_demand(demand)
    perm = _dev(perm, torch.uint8, "perm")
    dur = _dev(dur, torch.int32, "dur")
    count = _dev(count, torch.int32, "count")
    B, N, _ = demand.shape
    K = int(perm.shape[1])
    if perm.dim() != 3 or perm.shape[0] != B or perm.shape[2] != N or dur.shape != perm.shape[:2]:
        raise MoeschedError("perm must be [B, k_stride, N] and dur [B, k_stride]")
    dev = demand.device
    m = _model(model)
    order = torch.empty((B, K), dtype=torch.int32, device=dev)
    makespan, emission = torch.empty((2, B), dtype=torch.int64, device=dev).unbind(0)
    rule, status = torch.empty((2, B), dtype=torch.int32, device=dev).unbind(0)
    scratch = torch.empty(max(8, int(lib.moesched_order_scratch_bytes(B, K))), dtype=torch.uint8, device=dev)
    _call("moesched_schedule_order", dev, B, N, _ptr(demand), K, _ptr(perm), _ptr(dur), _ptr(count), m, _ptr(order),
          _ptr(makespan), _ptr(emission), _ptr(rule), _ptr(status), _ptr(scratch))
    return {"order": order, "makespan_ns": makespan, "emission_ns": emission, "rule": rule, "status": status}


def schedule_permute(perm, dur, order):
    """(perm, dur) with the matchings in the given order; positions whose order entry is -1 hold zeros."""
    perm = _dev(perm, torch.uint8, "perm")
    dur = _dev(dur, torch.int32, "dur")
    order = _dev(order, torch.int32, "order")
    B, K, N = perm.shape
    perm_out, dur_out = torch.zeros_like(perm), torch.zeros_like(dur)
    _call("moesched_schedule_permute", perm.device, B, N, K, _ptr(perm), _ptr(dur), _ptr(order), _ptr(perm_out),
          _ptr(dur_out))
    return perm_out, dur_out


def best_budget(count, prefix_overlap_ns, prefix_unserved_tokens, ns_per_unserved_token) -> dict:
    """Number of matchings (1..count) minimising prefix makespan + price * unserved tokens."""
    count = _dev(count, torch.int32, "count")
    po = _dev(prefix_overlap_ns, torch.int64, "prefix_overlap_ns")
    pu = _dev(prefix_unserved_tokens, torch.int64, "prefix_unserved_tokens")
    B, K = po.shape
    best_k = torch.empty(B, dtype=torch.int32, device=po.device)
    best_cost = torch.empty(B, dtype=torch.int64, device=po.device)
    _call("moesched_best_budget", po.device, B, K, _ptr(count), _ptr(po), _ptr(pu), int(ns_per_unserved_token),
          _ptr(best_k), _ptr(best_cost))
    return {"best_k": best_k, "best_cost": best_cost}


MAX_EXPERTS = 1024


try:
    from torch._C._dynamo.guards import _empty_strided_cuda     # (an allocation on the current device, without the dispatcher)
except ImportError:
    _empty_strided_cuda = None


_INT_MAX = 0x7fffffff                                    # (the binding of the C entry points cuts longer numbers off)


def _allocator(device):
    """Function of (shape, strides, dtype) that makes a tensor on `device`. (torch.empty takes 2.3 us, torch.empty_strided 1.5 and the
    allocation underneath 0.8, which counts beside kernels of a few microseconds.) Not the one underneath where the dispatcher has something to
    do: fill uninitialised memory (deterministic algorithms), or tell a dispatch mode."""
    if (_empty_strided_cuda is not None and device.index == torch._C._cuda_getDevice() and not torch._C._get_deterministic_algorithms()
            and not torch._C._len_torch_dispatch_stack()):
        return _empty_strided_cuda
    return lambda shape, strides, dtype: torch.empty_strided(shape, strides, dtype=dtype, device=device)


def _empty(dtype, device, *shape):
    """Densely packed tensor of one to three dimensions."""
    n = len(shape)
    strides = (1,) if n == 1 else (shape[1], 1) if n == 2 else (shape[1] * shape[2], shape[2], 1)
    return _allocator(device)(shape, strides, dtype)


def route_demand(experts, num_experts, out=None) -> dict:
    """Demand matrices from the router's choices: experts [B, N, S] int32 (expert of every choice of every rank, -1 for none).
    The num_experts experts sit in equal blocks on the N ranks. Returns 'demand' [B, N, N], 'counts' [B, N, num_experts], 'slot'
    [B, N, S] (row of every choice in its rank's send buffer, which lies by expert; -1 for none) and 'status' [B, N], all
    int32; `out` may hand back the dict of an earlier call of the same shape for reuse."""
    experts = _dev(experts, torch.int32, "experts")
    if experts.dim() != 3:
        raise MoeschedError("experts must have shape [B, N, S]")
    B, N, S = experts.shape
    E, dev = int(num_experts), experts.device
    if not 1 <= N <= E <= MAX_EXPERTS or E % N != 0 or max(B, S) > _INT_MAX:
        raise MoeschedError(f"num_experts must be a multiple of N and {MAX_EXPERTS} at most, B and S less than 2^31")
    if out is None:
        make, i32 = _allocator(dev), torch.int32
        out = {"demand": make((B, N, N), (N * N, N, 1), i32), "counts": make((B, N, E), (N * E, E, 1), i32),
               "slot": make((B, N, S), (N * S, S, 1), i32), "status": make((B, N), (N, 1), i32)}
    else:
        for k, shape in dict(demand=(B, N, N), counts=(B, N, E), slot=(B, N, S), status=(B, N)).items():
            if _dev(out[k], torch.int32, f"out['{k}']").shape != shape or out[k].device != dev:
                raise MoeschedError("out has the wrong shape or device")
    _call("moesched_route_demand", dev, B, N, S, E, _ptr(experts), _ptr(out["demand"]), _ptr(out["counts"]), _ptr(out["slot"]),
          _ptr(out["status"]))
    return out


def schedule_slots(demand, perm, dur, count, counts=None) -> dict:
    """Place of every transfer of a schedule: 'start' (first token of the pair's), 'length' (tokens) and 'row' (first row in
    the receiver's buffer), [B, k_stride, N] int32 by matching and source; 'rows' [B, N] (tokens that a rank receives);
    'status' [B]. With counts (route_demand's) also 'offsets' [B, N, k_stride * P + 1], P = experts per rank: the rows
    of every matching and expert in a rank's receive buffer, as expert_ffn and expert_matvec4 take them."""
    demand = _check_demand(demand)
    perm = _dev(perm, torch.uint8, "perm")
    dur = _dev(dur, torch.int32, "dur")
    count = _dev(count, torch.int32, "count")
    B, N, _ = demand.shape
    if perm.dim() != 3:
        raise MoeschedError("perm must be [B, k_stride, N]")
    K, P, dev = perm.shape[1], 0, demand.device
    if max(B, K) > _INT_MAX:
        raise MoeschedError("B and k_stride must be less than 2^31")
    if N < 1 or perm.shape != (B, K, N) or dur.shape != (B, K) or count.shape != (B,):
        raise MoeschedError("perm must be [B, k_stride, N], dur [B, k_stride] and count [B]")
    if counts is not None:
        counts = _dev(counts, torch.int32, "counts")
        wide = counts.shape
        if len(wide) != 3 or wide[0] != B or wide[1] != N or wide[2] % N != 0 or not N <= wide[2] <= MAX_EXPERTS:
            raise MoeschedError(f"counts must be [B, N, N * experts per rank], {MAX_EXPERTS} experts at most")
        P = wide[2] // N
    if perm.device != dev or dur.device != dev or count.device != dev or (counts is not None and counts.device != dev):
        raise MoeschedError("all tensors must be on one device")
    make, i32, shape, strides = _allocator(dev), torch.int32, (B, K, N), (K * N, N, 1)
    start, length, row = make(shape, strides, i32), make(shape, strides, i32), make(shape, strides, i32)
    rows, status = make((B, N), (N, 1), i32), make((B,), (1,), i32)
    res = {"start": start, "length": length, "row": row, "rows": rows, "status": status}
    offsets = None
    if counts is not None:
        res["offsets"] = offsets = make((B, N, K * P + 1), (N * (K * P + 1), K * P + 1, 1), i32)
    scratch = None
    if K > 224:                                          # (shorter schedules never use any)
        with torch.cuda.device(dev):
            need = int(load_library().moesched_slots_scratch_bytes(B, N, K))
        if need:
            scratch = make((need,), (1,), torch.uint8)
    _call("moesched_schedule_slots", dev, B, N, demand.data_ptr(), K, perm.data_ptr(), dur.data_ptr(), count.data_ptr(), P, _ptr(counts),
          start.data_ptr(), length.data_ptr(), row.data_ptr(), rows.data_ptr(), _ptr(offsets), _ptr(scratch), status.data_ptr())
    return res


_ACTS = {"silu": 0, "gelu": 1}
_MAX_ROWS, _MAX_GROUPS, _MAX_WIDTH = 1 << 30, 1 << 24, 65536
_TYPES = {torch.bfloat16: 0, torch.float16: 1}


def _act(act):
    if act not in _ACTS:
        raise MoeschedError(f"act must be one of {sorted(_ACTS)}")
    return _ACTS[act]


def _no_graph(what, *tensors):
    """Refuses tensors that want a gradient where autograd records: the experts' calls are not recorded, and the gradient would be lost
    without a sign."""
    if torch.is_grad_enabled():
        for t in tensors:
            if isinstance(t, torch.Tensor) and t.requires_grad:
                raise MoeschedError(f"{what} is not recorded by autograd, but an argument requires a gradient: call it under torch.no_grad() "
                                    "(gradients come from expert_ffn_backward), or detach the argument")


def _expert_rows(x, offsets, num_experts):
    """Element type of x [R, width] and number of groups of offsets; both checked."""
    if not isinstance(x, torch.Tensor) or x.dtype not in _TYPES:
        raise MoeschedError("x must be bfloat16 or float16")
    x = _dev(x, x.dtype, "x")
    offsets = _dev(offsets, torch.int32, "offsets")
    groups = offsets.numel() - 1
    if x.dim() != 2 or offsets.dim() != 1 or num_experts < 1 or groups < 1 or groups % num_experts != 0:
        raise MoeschedError("x must be [R, width] and offsets [groups + 1], groups a multiple of the number of experts")
    if x.shape[0] > _MAX_ROWS or groups > _MAX_GROUPS:
        raise MoeschedError("at most 2^30 rows and 2^24 groups")
    return _TYPES[x.dtype], groups


def _like(t, like, shape, what):
    """`t`, or a new tensor, of the type and device of `like` and the given shape."""
    if t is None:
        return _empty(like.dtype, like.device, *shape)
    _dev(t, like.dtype, what)
    if t.shape != tuple(shape) or t.device != like.device:
        raise MoeschedError(f"{what} must have shape {tuple(shape)}, on the device of x")
    return t


def _expert_weights(x, w_gate, w_up, w_down):
    if not isinstance(w_gate, torch.Tensor) or w_gate.dim() != 3 or x.dim() != 2:
        raise MoeschedError("x must be [R, D], w_gate and w_up [E, I, D] and w_down [E, D, I]")
    E, I, D = w_gate.shape
    dtype, dev = x.dtype, x.device
    for t, shape, what in ((w_gate, (E, I, D), "w_gate"), (w_up, (E, I, D), "w_up"), (w_down, (E, D, I), "w_down")):
        if _dev(t, dtype, what).shape != shape or t.device != dev:
            raise MoeschedError(f"{what} must have shape {shape}, on the device of x")
    if x.shape[1] != D:
        raise MoeschedError("x must be [R, D] with the D of the weights")
    if max(D, I) > _MAX_WIDTH or E > MAX_EXPERTS:
        raise MoeschedError(f"D and I must be {_MAX_WIDTH} at most, and there may be {MAX_EXPERTS} experts")
    return E, I, D


def _status_of(status, device):
    """The caller's, or a new one, which the call has to hold on to until it has launched: memory that is free again another
    thread may be given on the same stream, for work that is launched earlier."""
    if status is None:
        return _empty(torch.int32, device, 1)
    _dev(status, torch.int32, "status")
    if status.numel() != 1 or status.device != device:
        raise MoeschedError("status must hold one int32, on the device of x")
    return status


def _expert_scratch(scratch, x, I, groups, backward):
    """256-byte aligned working memory: the caller's (uint8), or new."""
    need = int(load_library().moesched_expert_scratch_bytes(x.shape[0], I, groups, backward))
    if scratch is None:
        return _empty(torch.uint8, x.device, max(1, need))
    _dev(scratch, torch.uint8, "scratch")
    if scratch.numel() < need or scratch.device != x.device:
        raise MoeschedError("scratch is smaller than expert_scratch_bytes, or on another device")
    return scratch


def expert_scratch_bytes(rows, width, groups, backward=False) -> int:
    """Working memory of expert_ffn (or its backward pass) for that many rows, a hidden width of `width` and `groups` groups."""
    rows, width, groups = int(rows), int(width), int(groups)
    if max(rows, width, groups) > _INT_MAX or min(rows, width, groups) < 0:              # (the library answers the others)
        return 0
    return int(load_library().moesched_expert_scratch_bytes(rows, width, groups, int(backward)))


def expert_ffn(x, w_gate, w_up, w_down, offsets, act="silu", save=False, out=None, scratch=None, status=None):
    """Gated feed-forward block of the experts, y = (act(x Wg^T) * (x Wu^T)) Wd^T, on rows grouped by expert: group g of
    x [R, D] is rows offsets[g] .. offsets[g+1]-1 and belongs to expert g % E. w_gate, w_up [E, I, D], w_down [E, D, I], bfloat16
    or float16; offsets [groups + 1] int32, groups a multiple of E (schedule_slots' offsets of a rank, or the part of them for one matching).
    act(x Wg^T) * (x Wu^T) is rounded to the type before the second product: in float16, infinite beyond 65504.
    Returns y [R, D]; rows outside the groups are left as they were (undefined in a tensor made here). With save=True
    returns (y, saved) for expert_ffn_backward. `status` [1] int32 takes the outcome; where it is not
    ST_OK (ST_BAD_INPUT: offsets out of order) the results are NaN, with or without a status. `scratch` is working memory of
    expert_scratch_bytes(R, I, groups). Autograd does not record the call: tensors that require gradients are refused unless it is off
    (torch.no_grad(), or within an autograd function); the gradients come from expert_ffn_backward."""
    _no_graph("expert_ffn", x, w_gate, w_up, w_down, out)
    E, I, D = _expert_weights(x, w_gate, w_up, w_down)
    dtype, groups = _expert_rows(x, offsets, E)
    if offsets.device != x.device:
        raise MoeschedError("all tensors must be on one device")
    R, dev = x.shape[0], x.device
    out = _like(out, x, (R, D), "out")
    saved = {k: _empty(torch.float32, dev, R, I) for k in ("gate", "up")} if save else {}
    scratch, status = _expert_scratch(scratch, x, I, groups, 0), _status_of(status, dev)
    _call("moesched_expert_ffn", dev, R, D, I, E, groups, dtype, _act(act), _ptr(x), _ptr(w_gate), _ptr(w_up), _ptr(w_down),
          _ptr(offsets), _ptr(out), _ptr(saved.get("gate")), _ptr(saved.get("up")), _ptr(scratch), _ptr(status))
    return (out, saved) if save else out


def expert_ffn_backward(dy, x, w_gate, w_up, w_down, offsets, saved, act="silu", out=None, scratch=None, status=None) -> dict:
    """Gradients of expert_ffn: 'dx' [R, D], 'dw_gate', 'dw_up' [E, I, D] and 'dw_down' [E, D, I] (0 for an expert without rows)
    from dy [R, D], the inputs of the forward call and what it saved. (The gradients of x Wg^T and x Wu^T are rounded to the type on the way:
    in float16, fewer digits below 6e-5 and 0 below 3e-8.) Rows of dx outside the groups are left as they were (undefined in a
    tensor made here); NaN throughout, as in expert_ffn, if the offsets are out of order. `out` may hand back the dict of an earlier
    call for reuse; `scratch` is working memory of expert_scratch_bytes(R, I, groups, True). Not recorded by autograd, like expert_ffn."""
    _no_graph("expert_ffn_backward", dy, x, w_gate, w_up, w_down)
    E, I, D = _expert_weights(x, w_gate, w_up, w_down)
    dtype, groups = _expert_rows(x, offsets, E)
    R, dev = x.shape[0], x.device
    if offsets.device != dev:
        raise MoeschedError("all tensors must be on one device")
    if dy is None:
        raise MoeschedError("dy is missing")
    _like(dy, x, (R, D), "dy")
    for k in ("gate", "up"):
        if _dev(saved[k], torch.float32, f"saved['{k}']").shape != (R, I) or saved[k].device != dev:
            raise MoeschedError(f"saved['{k}'] must be [R, I], on the device of x")
    shapes = dict(dx=(R, D), dw_gate=(E, I, D), dw_up=(E, I, D), dw_down=(E, D, I))
    grads = {k: _like(None if out is None else out[k], x, v, k) for k, v in shapes.items()}
    scratch, status = _expert_scratch(scratch, x, I, groups, 1), _status_of(status, dev)
    _call("moesched_expert_ffn_backward", dev, R, D, I, E, groups, dtype, _act(act), _ptr(dy), _ptr(x), _ptr(w_gate), _ptr(w_up),
          _ptr(w_down), _ptr(offsets), _ptr(saved["gate"]), _ptr(saved["up"]), *(_ptr(grads[k]) for k in shapes), _ptr(scratch),
          _ptr(status))
    return grads


def expert_matvec4(x, weight, scale, offsets, weight_up=None, scale_up=None, act="silu", out=None, status=None):
    """Products of a few rows with their experts' 4-bit weights: y[r, n] = sum_k (q - 8) scale[e, n, k // group] x[r, k], the q of
    k = 2m in the low half of byte m of weight [E, N, K / 2] uint8, scale [E, N, K / group] in the type of x (bfloat16
    or float16), group 32, 64 or 128. With weight_up and scale_up, act(x W^T) * (x W_up^T). Rows lie by group as in expert_ffn, and
    the result is NaN, whether or not `status` [1] int32 is there to take the outcome, if the offsets are out of order.
    Not recorded by autograd, like expert_ffn."""
    _no_graph("expert_matvec4", x, scale, scale_up, out)
    dtype, groups = _expert_rows(x, offsets, 1)
    weight = _dev(weight, torch.uint8, "weight")
    scale = _dev(scale, x.dtype, "scale")
    if weight.dim() != 3 or scale.dim() != 3:
        raise MoeschedError("weight must be [E, N, K / 2] and scale [E, N, K / group]")
    E, N, half = weight.shape
    R, K = x.shape
    parts, dev = scale.shape[2], x.device
    if half == 0 or K != 2 * half or scale.shape[:2] != (E, N) or parts == 0 or K % parts != 0:
        raise MoeschedError("x must be [R, K], weight [E, N, K / 2] and scale [E, N, K / group]")
    if E < 1 or groups % E != 0 or max(N, K) > 1 << 24:
        raise MoeschedError("the groups of offsets must be a multiple of the number of experts, N and K 2^24 at most")
    if (weight_up is None) != (scale_up is None):
        raise MoeschedError("weight_up and scale_up go together")
    if weight.device != dev or scale.device != dev or offsets.device != dev:
        raise MoeschedError("all tensors must be on one device")
    if weight_up is not None:
        if _dev(weight_up, torch.uint8, "weight_up").shape != weight.shape or weight_up.device != dev:
            raise MoeschedError("weight_up must be like weight, on the device of x")
        if _dev(scale_up, x.dtype, "scale_up").shape != scale.shape or scale_up.device != dev:
            raise MoeschedError("scale_up must be like scale, on the device of x")
    out, status = _like(out, x, (R, N), "out"), _status_of(status, dev)
    _call("moesched_expert_matvec4", dev, R, K, N, E, groups, K // parts, dtype, _act(act), x.data_ptr(), weight.data_ptr(),
          scale.data_ptr(), _ptr(weight_up), _ptr(scale_up), offsets.data_ptr(), out.data_ptr(), status.data_ptr())
    return out


def _expert_curve(tokens, times):
    """Fixed cost, slope and knee of the curve that is nearest to the times, of those with one of the counts as the knee. Near is a ratio, so
    that half of a time is as far off as twice (a difference relative to the time would put curves below)."""
    best = None
    for knee in tokens:
        flat = [ns for g, ns in zip(tokens, times) if g <= knee]
        fixed = sum(flat) / len(flat)
        beyond = [(g - knee, ns - fixed) for g, ns in zip(tokens, times) if g > knee]
        slope = max(0.0, sum(g * ns for g, ns in beyond) / sum(g * g for g, _ in beyond)) if beyond else 0.0
        off = sum(math.log((fixed + max(0, g - knee) * slope) / ns) ** 2 for g, ns in zip(tokens, times))
        if best is None or off < best[0]:
            best = off, fixed, slope, knee
    return best[1:]


def probe_expert(weights, tokens=(1, 16, 64, 256, 1024, 4096), act="silu", base=None, reps=20) -> dict:
    """Compute model of the experts of one rank, measured (the paper profiles its experts, Fig. 1): the batches of expert_ffn
    are timed for every count in `tokens`, spread evenly over the experts, and the model's curve is laid through the times: a fixed cost up
    to a knee, linear beyond. weights = (w_gate, w_up, w_down) as expert_ffn takes them, or three (weight, scale) pairs in 4
    bits, timed with expert_matvec4. Returns 'model' (base, or DEFAULT_MODEL, with the experts' three numbers and the bytes of a token,
    as schedule_eval, Path and the others take it), 'tokens' and 'ns'. A time is that of the GPU alone: batches are replayed from a graph, behind
    work that keeps the GPU busy until they are queued, and find the weights in memory, not in the L2 (another layer's were there
    before). Synchronises: a measurement, not for a serving loop."""
    quantised = isinstance(weights[0], (tuple, list))
    first = weights[0][0] if quantised else weights[0]
    typed = weights[0][1] if quantised else weights[0]
    if not isinstance(first, torch.Tensor) or not first.is_cuda or first.dim() != 3:
        raise MoeschedError("weights must be CUDA tensors of three dimensions, or pairs of them")
    tokens = sorted({int(g) for g in tokens})
    if not tokens or tokens[0] < 1 or reps < 1:
        raise MoeschedError("tokens must be counts of at least 1, reps at least 1")
    E, dev = first.shape[0], first.device
    D = first.shape[2] * (2 if quantised else 1)
    gen = torch.Generator(dev)
    gen.manual_seed(0)
    times = []
    with torch.cuda.device(dev), torch.no_grad():
        other = torch.zeros(torch.cuda.get_device_properties(dev).L2_cache_size, dtype=torch.float32, device=dev)     # (four times the L2)
        for g in tokens:
            x = torch.randn((g, D), generator=gen, device=dev).to(typed.dtype)
            offsets = torch.tensor([g * e // E for e in range(E + 1)], dtype=torch.int32, device=dev)
            if quantised:
                (wg, sg), (wu, su), (wd, sd) = weights

                def batch():
                    return expert_matvec4(expert_matvec4(x, wg, sg, offsets, wu, su, act=act), wd, sd, offsets)
            else:
                def batch():
                    return expert_ffn(x, *weights, offsets, act=act)
            for _ in range(3):
                batch()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=torch.cuda.Stream(dev), capture_error_mode="thread_local"):
                batch()
            events = [(torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)) for _ in range(reps)]
            for start, end in events:
                other.sum()                              # (read, not written: nothing is left to be written back)
                start.record()
                graph.replay()
                end.record()
            torch.cuda.current_stream(dev).synchronize()
            times.append(sorted(s.elapsed_time(e) for s, e in events)[reps // 2] * 1e6)
    fixed, slope, knee = _expert_curve(tokens, times)
    model = dict(base or DEFAULT_MODEL, bytes_per_token=2 * D, expert_fixed_ns=round(fixed), expert_knee_tokens=knee,
                 expert_ps_per_token=round(slope * 1000))
    return {"model": model, "tokens": tokens, "ns": times}


class Path:
    """The whole path for batches of one shape: greedy max-weight and BvN decomposition, both scored.

    All buffers (schedules, scores, BvN scratch) are allocated once here. The two decompositions do not
    depend on each other: run() enqueues BvN and its scoring on the caller's current stream and greedy and its
    scoring on a side stream forked from it and joined back, so that the greedy warps fill the SMs beside the BvN
    warps. run(overlap=False) keeps everything on the current stream. The launches, the fork and the join are
    one call into the library (moesched_path_run), since a small batch is done in microseconds."""

    def __init__(self, B, N, k_mw, k_bvn=None, device=None, want_work=False):
        dev = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
        self.device, self.B, self.N = dev, B, N
        self.k_mw, self.k_bvn = int(k_mw), int(bvn_capacity(N) if k_bvn is None else k_bvn)

        def sched(k):
            return Schedule(perm=torch.empty((B, k, N), dtype=torch.uint8, device=dev),
                            dur=torch.empty((B, k), dtype=torch.int32, device=dev),
                            count=torch.empty(B, dtype=torch.int32, device=dev),
                            status=torch.empty(B, dtype=torch.int32, device=dev),
                            work=torch.zeros((B, WORK_FIELDS), dtype=torch.int64, device=dev) if want_work else None)

        self.mw, self.bvn = sched(self.k_mw), sched(self.k_bvn)
        self.score_mw = torch.empty((5, B), dtype=torch.int64, device=dev)
        self.score_bvn = torch.empty((5, B), dtype=torch.int64, device=dev)
        self.eval_status_mw = torch.empty(B, dtype=torch.int32, device=dev)
        self.eval_status_bvn = torch.empty(B, dtype=torch.int32, device=dev)
        self.scratch = torch.empty(max(1, bvn_scratch_bytes(B, N)), dtype=torch.uint8, device=dev)
        with torch.cuda.device(dev):
            self._side = torch.cuda.Stream(dev)
            self._events = tuple(torch.cuda.Event() for _ in range(3))   # fork, join, done
            for event in self._events:
                event.record()                                           # an event gets its handle when first recorded
        self._made = (None, None)                                        # addresses, and the C form made of them
        self._arguments()

    def _arguments(self):
        """The C form of the buffers as they are at this call: a caller may have put others of the same shapes and types in
        their place."""
        mw, bvn = self.mw, self.bvn
        at = (mw.perm.data_ptr(), bvn.perm.data_ptr(), mw.dur.data_ptr(), mw.count.data_ptr(), mw.status.data_ptr(),
              self.eval_status_mw.data_ptr(), bvn.dur.data_ptr(), bvn.count.data_ptr(), bvn.status.data_ptr(),
              self.eval_status_bvn.data_ptr(), _ptr(mw.work), _ptr(bvn.work), self.score_mw.data_ptr(),
              self.score_bvn.data_ptr(), self.scratch.data_ptr())
        made_of, args = self._made
        if made_of != at:
            args = _PathArgs(self.k_mw, self.k_bvn, self.B, *at, self._side.cuda_stream, *(e.cuda_event for e in self._events))
            self._made = (at, args)
        return args

    def outputs(self):
        return [self.mw.perm, self.mw.dur, self.mw.count, self.mw.status, self.bvn.perm, self.bvn.dur,
                self.bvn.count, self.bvn.status, self.score_mw, self.score_bvn]

    def run_graph(self, demand, model=None):
        """The same launches replayed from a CUDA graph: for small matrices the step is a handful of
        microsecond kernels and the cost of launching them one by one dominates. The graph is captured
        on first use and again whenever the demand tensor's address, its shape, the model or one of the buffers changes."""
        demand = _check_demand(demand)                   # also where the graph is replayed
        key = (demand.data_ptr(), demand.device, demand.shape, bytes(_model(model)._obj), bytes(self._arguments()))
        if getattr(self, "_graph_key", None) != key:
            self.run(demand, model)                      # first-use set-up outside the capture
            torch.cuda.current_stream(self.device).synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                self.run(demand, model)
            self._graph, self._graph_key, self._graph_demand = graph, key, demand
        self._graph.replay()
        return self

    def run(self, demand, model=None, overlap=True):
        """Enqueue the four kernels; results are ready when the caller's current stream reaches this point. Runs of one Path
        follow one another whatever streams they are called on (captured ones are ordered by their graph alone).

        A smaller batch is taken too. Its results lie densely packed at the start of the buffers ([B, k, N] with its own
        B and N), so with fewer matrices of the Path's own N they are rows 0 .. B-1 of outputs(); what lies behind them is
        left as it was."""
        demand = _check_demand(demand)
        B, N, _ = demand.shape
        if B > self.B or N > self.N:
            raise MoeschedError("demand is larger than the Path was made for")
        _call("moesched_path_run", demand.device, ctypes.byref(self._arguments()), B, N, _ptr(demand), _model(model), int(overlap))
        return self


class HostPipeline:
    """The whole path for batches that live in host memory, double-buffered.

    submit() enqueues, for one batch: the copy of the demand from (pinned) host memory to the device
    on an upload stream, the four kernels on the slot's compute stream, and the copy of all schedules and scores
    back to pinned host memory on a download stream. With two slots the download of one batch and the
    upload of the next overlap the kernels of the batch in between, so a stream of batches runs at the
    speed of the slowest of the three stages instead of their sum."""

    def __init__(self, B, N, k_mw, k_bvn=None, device=None, slots=2):
        dev = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
        self.device, self.slots = dev, slots
        self.paths = [Path(B, N, k_mw, k_bvn, device=dev) for _ in range(slots)]
        self.d_in = [torch.empty((B, N, N), dtype=torch.int32, device=dev) for _ in range(slots)]
        self.h_out = [[torch.empty(t.shape, dtype=t.dtype, pin_memory=True) for t in p.outputs()] for p in self.paths]
        self.up, self.down = torch.cuda.Stream(dev), torch.cuda.Stream(dev)
        # A batch that leaves the schedulers with little to choose from is bound by the latency of its chains, so two of
        # them run side by side, a compute stream per slot; larger ones would only
        # get in each other's way.
        sms = torch.cuda.get_device_properties(dev).multi_processor_count
        shared = None if B < 12 * sms else torch.cuda.Stream(dev)
        self.compute = [shared or torch.cuda.Stream(dev) for _ in range(slots)]
        self.ev_in = [torch.cuda.Event() for _ in range(slots)]
        self.ev_done = [torch.cuda.Event() for _ in range(slots)]
        self.ev_out = [torch.cuda.Event() for _ in range(slots)]
        self._next = 0
        self.h2d_bytes = B * N * N * 4
        self.d2h_bytes = sum(t.numel() * t.element_size() for t in self.paths[0].outputs())

    def submit(self, demand_host, model=None) -> int:
        """Enqueue one batch (a [B, N, N] int32 CPU tensor, ideally pinned); returns its slot."""
        s = self._next
        self._next = (s + 1) % self.slots
        self.ev_out[s].synchronize()            # the slot's previous results must have left the device
        self.up.wait_event(self.ev_done[s])     # and its previous kernels must be done with the input
        with torch.cuda.stream(self.up):
            self.d_in[s].copy_(demand_host, non_blocking=True)
            self.ev_in[s].record(self.up)
        compute = self.compute[s]
        compute.wait_event(self.ev_in[s])
        with torch.cuda.stream(compute):
            self.paths[s].run(self.d_in[s], model)
            self.ev_done[s].record(compute)
        self.down.wait_event(self.ev_done[s])
        with torch.cuda.stream(self.down):
            for h, t in zip(self.h_out[s], self.paths[s].outputs()):
                h.copy_(t, non_blocking=True)
            self.ev_out[s].record(self.down)
        return s

    def result(self, slot):
        """Block until the slot's results are in host memory; returns the pinned host tensors in the
        order of Path.outputs(). They are overwritten when the slot is submitted again."""
        self.ev_out[slot].synchronize()
        return self.h_out[slot]
