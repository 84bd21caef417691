"""Thin ctypes binding of the C-ABI library (argument marshalling only).

Function names and argument order follow ``include/routepack.h``.  Arrays may be numpy
arrays (host memory) or torch tensors (host or CUDA); outputs are allocated here when the
caller passes none.  Nothing in this module computes any step of the method: if the CUDA
library cannot be loaded, every call raises.
"""
from __future__ import annotations

import ctypes as C
import functools
import operator
import os
import warnings
from typing import Optional, Sequence, Tuple

import numpy as np

from . import build as _build

_lib = None

STATUS_NAMES = {0: "RP_OK", -1: "RP_ERR_ARG", -2: "RP_ERR_SHAPE", -3: "RP_ERR_CONSERVATION",
                -4: "RP_ERR_INFEASIBLE", -5: "RP_ERR_RANGE", -6: "RP_ERR_CUDA", -7: "RP_ERR_STATE",
                -8: "RP_ERR_TIMEOUT", -9: "RP_ERR_INVALID_PLAN"}
RP_OK = 0

EXPORTS = ("rp_window_load", "rp_place_experts", "rp_pack_rows", "rp_seed_population", "rp_pair_population", "rp_select_population", "rp_init_population", "rp_eval_population", "rp_eval_layouts_noalloc", "rp_diagnostics", "rp_anneal",
           "rp_best", "rp_destroy", "rp_release_cached_memory", "rp_strerror", "rp_last_cuda_error", "rp_debug_dump",
           "rp_debug_set_trace", "rp_debug_set_knob", "rp_debug_set_stage_timing", "rp_debug_stage_times",
           "rp_debug_nl2", "rp_debug_exp2neg", "rp_debug_philox", "rp_debug_launch_count", "rp_debug_l2_read_rate",
           "rp_debug_chain_kernel", "rp_debug_chain_form",
           "rp_count_routes", "rp_window_load_routes", "rp_route_workspace", "rp_route", "rp_route_grad",
           "rp_rotate", "rp_rotate_workspace", "rp_rotate_grad", "rp_attend_workspace", "rp_attend",
           "rp_attend_grad_workspace", "rp_attend_grad", "rp_attend_window", "rp_attend_window_grad_workspace",
           "rp_attend_window_grad", "rp_attend_step_workspace", "rp_attend_step", "rp_rotate_axes", "rp_rotate_axes_grad",
           "rp_debug_set_wait_limit")


class RpError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().rp_strerror(status).decode()
        extra = f" (cudaError {lib().rp_last_cuda_error()})" if status == -6 else ""
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)}: {msg}{extra}")


class rp_config(C.Structure):
    _fields_ = [("n_samples", C.c_int32), ("n_layers", C.c_int32), ("n_experts", C.c_int32),
                ("top_k", C.c_int32), ("token_cap", C.c_int32), ("dp_width", C.c_int32),
                ("ep_width", C.c_int32), ("edp_of_dp", C.c_void_p), ("n_stages", C.c_int32),
                ("alpha", C.c_void_p), ("beta", C.c_void_p), ("pop_size", C.c_int32),
                ("min_rows", C.c_int32), ("seed", C.c_uint64)]


class rp_anneal_params(C.Structure):
    _fields_ = [("n_levels", C.c_int32), ("steps_per_level", C.c_int32), ("t0", C.c_double),
                ("t_ratio", C.c_double), ("p_reloc", C.c_double), ("p_guide", C.c_double)]


class rp_anneal_stats(C.Structure):
    _fields_ = [("proposed", C.c_int64), ("feasible", C.c_int64), ("accepted", C.c_int64),
                ("improved", C.c_int64), ("ms_chains", C.c_double),
                ("move_bytes", C.c_int64), ("gather_bytes", C.c_int64), ("staging_bytes", C.c_int64),
                ("kernel_launches", C.c_int64)]


class rp_router(C.Structure):
    _fields_ = [("n_experts", C.c_int32), ("top_k", C.c_int32), ("type", C.c_int32), ("score", C.c_int32), ("normalise", C.c_int32),
                ("scale", C.c_float), ("loss_coef", C.c_float)]


class rp_rotary(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("rotary_dim", C.c_int32), ("layout", C.c_int32), ("type", C.c_int32), ("weight_type", C.c_int32),
                ("eps", C.c_float), ("mscale", C.c_float)]


class rp_heads(C.Structure):
    _fields_ = [("n_heads", C.c_int32), ("x", C.c_void_p), ("x_token", C.c_int64), ("x_head", C.c_int64),
                ("y", C.c_void_p), ("y_token", C.c_int64), ("y_head", C.c_int64), ("weight", C.c_void_p),
                ("y_grad", C.c_void_p), ("g_token", C.c_int64), ("g_head", C.c_int64), ("weight_grad", C.c_void_p)]


class rp_axes(C.Structure):
    _fields_ = [("n_axes", C.c_int32), ("axis", C.c_void_p), ("position", C.c_void_p), ("axis_stride", C.c_int64), ("token_stride", C.c_int64)]


class rp_attend_config(C.Structure):
    _fields_ = [("q_heads", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("type", C.c_int32), ("causal", C.c_int32),
                ("scale", C.c_float)]


class rp_view(C.Structure):
    _fields_ = [("x", C.c_void_p), ("token", C.c_int64), ("head", C.c_int64)]


class rp_diag(C.Structure):
    _fields_ = [("cv_identity", C.c_double), ("cv_placed", C.c_double), ("s_ep", C.c_int64), ("t_ep", C.c_int64),
                ("n_ep", C.c_int64), ("eta_ep", C.c_double), ("attention", C.c_double), ("joint", C.c_double)]


def library_path() -> str:
    return _build.LIB


def lib():
    """Load the CUDA library; raises if it has not been built (there is no fallback)."""
    global _lib
    if _lib is None:
        path = library_path()
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing: run paper_2608_12146_b200.build.build() (needs nvcc)")
        L = C.CDLL(path)
        L.rp_strerror.restype = C.c_char_p
        L.rp_strerror.argtypes = [C.c_int]
        L.rp_last_cuda_error.restype = C.c_int
        L.rp_destroy.restype = None
        L.rp_destroy.argtypes = [C.c_void_p]
        L.rp_window_load.argtypes = [C.POINTER(C.c_void_p), C.POINTER(rp_config), C.c_void_p, C.c_void_p, C.c_void_p]
        L.rp_place_experts.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p]
        L.rp_pack_rows.argtypes = [C.c_void_p, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
        L.rp_seed_population.argtypes = [C.c_void_p, C.c_int32, C.POINTER(C.c_int32)]
        L.rp_pair_population.argtypes = [C.c_void_p, C.c_int32, C.POINTER(C.c_int32)]
        L.rp_select_population.argtypes = [C.c_void_p, C.c_int32, C.c_int64, C.POINTER(C.c_int32), C.c_void_p]
        L.rp_init_population.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int64, C.POINTER(C.c_int32), C.c_void_p]
        L.rp_eval_population.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p]
        L.rp_eval_layouts_noalloc.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p]
        L.rp_diagnostics.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(rp_diag)]
        L.rp_anneal.argtypes = [C.c_void_p, C.POINTER(rp_anneal_params), C.POINTER(rp_anneal_stats)]
        L.rp_best.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.rp_debug_dump.argtypes = [C.c_void_p, C.c_int, C.c_int32, C.c_void_p, C.c_int64]
        L.rp_debug_set_trace.argtypes = [C.c_void_p, C.c_int]
        L.rp_debug_set_knob.argtypes = [C.c_void_p, C.c_int, C.c_int64]
        L.rp_debug_set_stage_timing.argtypes = [C.c_int]
        L.rp_debug_stage_times.argtypes = [C.c_void_p, C.c_void_p]
        L.rp_debug_nl2.argtypes = [C.c_void_p, C.c_void_p, C.c_int64]
        L.rp_debug_exp2neg.argtypes = [C.c_void_p, C.c_void_p, C.c_int64]
        L.rp_debug_philox.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64]
        L.rp_debug_launch_count.restype = C.c_int64
        L.rp_debug_l2_read_rate.argtypes = [C.c_int64, C.c_int32, C.POINTER(C.c_double)]
        L.rp_debug_chain_kernel.argtypes = [C.c_void_p, C.POINTER(C.c_int32)]
        L.rp_debug_chain_form.argtypes = [C.c_void_p, C.POINTER(C.c_int32)]
        L.rp_debug_set_wait_limit.argtypes = [C.c_int64]
        V, I, Q = C.c_void_p, C.c_int32, C.c_int64
        L.rp_count_routes.argtypes = [V, I, Q, I, I, I, Q, Q, V, I, V, V]
        L.rp_window_load_routes.argtypes = [C.POINTER(C.c_void_p), C.POINTER(rp_config), V, V, I, Q, Q, Q, V]
        L.rp_route_workspace.restype = Q
        L.rp_route_workspace.argtypes = [C.POINTER(rp_router), I]
        L.rp_route.argtypes = [C.POINTER(rp_router), V, Q, Q, V, V, I, I, V, I, Q, V, V, V, V, Q, V]
        L.rp_route_grad.argtypes = [C.POINTER(rp_router), V, Q, Q, V, I, Q, V, V, V, I, V, V, Q, V]
        H = C.POINTER(rp_heads)
        L.rp_rotate.argtypes = [C.POINTER(rp_rotary), Q, V, V, I, V, H, H, V]
        L.rp_rotate_workspace.restype = Q
        L.rp_rotate_workspace.argtypes = [C.POINTER(rp_rotary)]
        L.rp_rotate_grad.argtypes = [C.POINTER(rp_rotary), Q, V, V, I, V, H, H, V, Q, V]
        L.rp_rotate_axes.argtypes = [C.POINTER(rp_rotary), Q, V, C.POINTER(rp_axes), H, H, V]
        L.rp_rotate_axes_grad.argtypes = [C.POINTER(rp_rotary), Q, V, C.POINTER(rp_axes), H, H, V, Q, V]
        W = C.POINTER(rp_view)
        L.rp_attend_workspace.restype = Q
        L.rp_attend_workspace.argtypes = [C.POINTER(rp_attend_config), Q, I]
        L.rp_attend.argtypes = [C.POINTER(rp_attend_config), Q, W, W, W, V, I, W, W, V, Q, V]
        L.rp_attend_grad_workspace.restype = Q
        L.rp_attend_grad_workspace.argtypes = [C.POINTER(rp_attend_config), Q, I]
        L.rp_attend_grad.argtypes = [C.POINTER(rp_attend_config), Q, W, W, W, W, W, W, V, I, W, W, W, V, Q, V]
        L.rp_attend_window.argtypes = [C.POINTER(rp_attend_config), I, I, Q, W, W, W, V, I, W, W, V, Q, V]
        L.rp_attend_window_grad_workspace.restype = Q
        L.rp_attend_window_grad_workspace.argtypes = [C.POINTER(rp_attend_config), I, I, Q, I]
        L.rp_attend_window_grad.argtypes = [C.POINTER(rp_attend_config), I, I, Q, W, W, W, W, W, W, V, I, W, W, W, V, Q, V]
        L.rp_attend_step_workspace.restype = Q
        L.rp_attend_step_workspace.argtypes = [C.POINTER(rp_attend_config), I, I, Q, I]
        L.rp_attend_step.argtypes = [C.POINTER(rp_attend_config), I, I, Q, W, W, W, V, I, V, W, W, V, Q, V]
        _lib = L
    return _lib


def _ptr(a) -> Optional[int]:
    """Address of a numpy array or torch tensor (host or device); None stays NULL."""
    if a is None:
        return None
    if isinstance(a, np.ndarray):
        if not a.flags["C_CONTIGUOUS"]:
            raise ValueError("array must be C-contiguous")
        return a.ctypes.data
    if hasattr(a, "data_ptr"):
        if not a.is_contiguous():
            raise ValueError("tensor must be contiguous")
        return a.data_ptr()
    raise TypeError(f"unsupported array type {type(a)}")


def _check(status: int, where: str):
    if status != RP_OK:
        raise RpError(status, where)


def _stream_handle(stream) -> Optional[int]:
    if stream is None:
        return None
    if isinstance(stream, int):
        return stream
    return int(stream.cuda_stream)           # torch.cuda.Stream


class Context:
    """Owner of one rp_ctx*; destroyed with close() or at garbage collection."""

    def __init__(self, handle: int, cfg: rp_config, keep: tuple):
        self.handle = C.c_void_p(handle)
        self.cfg = cfg
        self._keep = keep                    # input arrays adopted by the library must stay alive
        self.n_rows = 0
        self.n_shards = 0

    def close(self):
        if self.handle:
            lib().rp_destroy(self.handle)
            self.handle = C.c_void_p(None)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _window_config(n, l, e, top_k, token_cap, dp_width, ep_width, pop_size, edp_of_dp, alpha, beta, min_rows, seed):
    """rp_config and the arrays it points to."""
    al = np.ascontiguousarray(alpha, dtype=np.float64)
    be = np.ascontiguousarray(beta, dtype=np.float64)
    edp = None if edp_of_dp is None else np.ascontiguousarray(edp_of_dp, dtype=np.int32)
    cfg = rp_config(n, l, e, top_k, token_cap, dp_width, ep_width, _ptr(edp), len(al), _ptr(al), _ptr(be),
                    pop_size, min_rows, seed)
    return cfg, al, be, edp


def rp_window_load(lengths, demand, *, top_k: int, token_cap: int, dp_width: int, ep_width: int,
                   pop_size: int, edp_of_dp: Optional[Sequence[int]] = None,
                   alpha: Sequence[float] = (1.0, 1.0), beta: Sequence[float] = (0.0, 1.0),
                   min_rows: int = 0, seed: int = 0, stream=None) -> Context:
    """``stream``: by default that of the input, where it is a CUDA tensor (torch's current one, on which it is written), or the default stream."""
    n, l, e = tuple(demand.shape)
    if stream is None:
        stream = next((_current_stream(x.get_device()) for x in (demand, lengths) if getattr(x, "is_cuda", False)), None)
    cfg, al, be, edp = _window_config(n, l, e, top_k, token_cap, dp_width, ep_width, pop_size, edp_of_dp, alpha, beta, min_rows, seed)
    out = C.c_void_p(None)
    st = lib().rp_window_load(C.byref(out), C.byref(cfg), _ptr(lengths), _ptr(demand), _stream_handle(stream))
    _check(st, "rp_window_load")
    ctx = Context(out.value, cfg, (lengths, demand, al, be, edp))
    ctx.n_shards = dp_width if edp is None else int(edp.max()) + 1
    return ctx


def rp_window_load_routes(lengths, routes, n_experts: int, *, token_cap: int, dp_width: int, ep_width: int, pop_size: int,
                          edp_of_dp: Optional[Sequence[int]] = None, alpha: Sequence[float] = (1.0, 1.0),
                          beta: Sequence[float] = (0.0, 1.0), min_rows: int = 0, seed: int = 0, stream=None) -> Context:
    """A window from recorded routes (CUDA tensor [n_tokens, n_layers, top_k] of integers, any strides with the choices side by side).

    ``stream``: torch's current one by default, on which the record is written; the context works on it.
    """
    T, l, k = routes.shape
    size, ts, ls = _route_layout(routes)
    if stream is None:
        stream = _current_stream(routes.get_device())
    cfg, al, be, edp = _window_config(int(lengths.shape[0]), l, n_experts, k, token_cap, dp_width, ep_width, pop_size, edp_of_dp, alpha, beta,
                                      min_rows, seed)
    out = C.c_void_p(None)
    st = lib().rp_window_load_routes(C.byref(out), C.byref(cfg), _ptr(lengths), routes.data_ptr(), size, T, ts, ls, _stream_handle(stream))
    _check(st, "rp_window_load_routes")
    ctx = Context(out.value, cfg, (lengths, al, be, edp))
    ctx.n_shards = dp_width if edp is None else int(edp.max()) + 1
    return ctx


def rp_place_experts(ctx: Context, pi=None, rank_load=None):
    c = ctx.cfg
    if pi is None:
        pi = np.empty((c.n_layers, c.n_experts), np.int32)
    if rank_load is None:
        rank_load = np.empty((c.n_layers, c.ep_width), np.int64)
    _check(lib().rp_place_experts(ctx.handle, _ptr(pi), _ptr(rank_load)), "rp_place_experts")
    return pi, rank_load


def rp_pack_rows(ctx: Context) -> Tuple[int, int]:
    r, cert = C.c_int32(0), C.c_int32(0)
    _check(lib().rp_pack_rows(ctx.handle, C.byref(r), C.byref(cert)), "rp_pack_rows")
    ctx.n_rows = r.value
    return r.value, cert.value


def rp_seed_population(ctx: Context, choice_width: int) -> int:
    """Randomized seeds, one trial per member; returns how many members carry their own trial."""
    own = C.c_int32(0)
    _check(lib().rp_seed_population(ctx.handle, choice_width, C.byref(own)), "rp_seed_population")
    return own.value


def rp_pair_population(ctx: Context, choice_width: int) -> int:
    """EDPAwarePair on every member but the first; returns how many layouts changed."""
    changed = C.c_int32(0)
    _check(lib().rp_pair_population(ctx.handle, choice_width, C.byref(changed)), "rp_pair_population")
    return int(changed.value)


def rp_select_population(ctx: Context, n_proj: int = 8, eta_q16: int = 1 << 16):
    """CanonicalMap + QualityDiversitySelect over the population; returns (n_distinct, order [P_pop])."""
    nd = C.c_int32(0)
    order = np.zeros(ctx.cfg.pop_size, np.int32)
    _check(lib().rp_select_population(ctx.handle, n_proj, eta_q16, C.byref(nd), _ptr(order)), "rp_select_population")
    return int(nd.value), order


def rp_init_population(ctx: Context, n_candidates: int, choice_width: int = 4, n_proj: int = 8, eta_q16: int = 1 << 16):
    """Algorithm 2 over n_candidates fixed-row candidates; returns (n_distinct, picked [P_pop])."""
    nd = C.c_int32(0)
    picked = np.zeros(ctx.cfg.pop_size, np.int32)
    _check(lib().rp_init_population(ctx.handle, n_candidates, choice_width, n_proj, eta_q16, C.byref(nd), _ptr(picked)),
           "rp_init_population")
    return int(nd.value), picked


def rp_eval_population(ctx: Context, layouts=None, score_fx=None, score_f64=None):
    n = ctx.cfg.pop_size if layouts is None else int(layouts.shape[0])
    if score_fx is None:
        score_fx = np.empty((n, 3), np.int64)
    if score_f64 is None:
        score_f64 = np.empty((n, 3), np.float64)
    _check(lib().rp_eval_population(ctx.handle, _ptr(layouts), n, _ptr(score_fx), _ptr(score_f64)),
           "rp_eval_population")
    return score_fx, score_f64


def rp_eval_layouts_noalloc(ctx: Context, layouts, score_fx, score_f64):
    """Scores of device-resident layouts into device-resident outputs without any allocation.

    For callers that may not allocate once running (all device memory already belongs to a
    framework's pool, or an allocation would stall the device).  ``layouts`` [n][N] int32 and
    the outputs [n][3] int64 / float64 must be CUDA tensors; nothing is allocated here either.
    """
    n = int(layouts.shape[0])
    _check(lib().rp_eval_layouts_noalloc(ctx.handle, _ptr(layouts), n, _ptr(score_fx), _ptr(score_f64)),
           "rp_eval_layouts_noalloc")
    return score_fx, score_f64


def rp_diagnostics(ctx: Context, layout=None) -> dict:
    """Load-balance diagnostics of a layout (None = the incumbent) as a dict."""
    d = rp_diag()
    _check(lib().rp_diagnostics(ctx.handle, _ptr(layout), C.byref(d)), "rp_diagnostics")
    return {name: getattr(d, name) for name, _ in rp_diag._fields_}


def rp_anneal(ctx: Context, *, n_levels: int, steps_per_level: int, t0: float, t_ratio: float,
              p_reloc: float, p_guide: float, want_stats: bool = True) -> Optional[rp_anneal_stats]:
    prm = rp_anneal_params(n_levels, steps_per_level, t0, t_ratio, p_reloc, p_guide)
    stats = rp_anneal_stats() if want_stats else None
    _check(lib().rp_anneal(ctx.handle, C.byref(prm), C.byref(stats) if want_stats else None), "rp_anneal")
    return stats


def rp_best(ctx: Context, cell_of_sample=None, score_fx=None, score_f64=None):
    if cell_of_sample is None:
        cell_of_sample = np.empty(ctx.cfg.n_samples, np.int32)
    if score_fx is None:
        score_fx = np.empty(3, np.int64)
    if score_f64 is None:
        score_f64 = np.empty(3, np.float64)
    _check(lib().rp_best(ctx.handle, _ptr(cell_of_sample), _ptr(score_fx), _ptr(score_f64)), "rp_best")
    return cell_of_sample, score_fx, score_f64


def rp_destroy(ctx: Context):
    ctx.close()


def rp_release_cached_memory():
    _check(lib().rp_release_cached_memory(), "rp_release_cached_memory")


# ---- operators on the tokens of a window ------------------------------------------------
# Arrays are CUDA tensors of one GPU; calls queue on ``stream`` (default: torch's current stream of that GPU) and return.
# Outputs that the caller does not pass are allocated on that stream.
# Autograd does not record them: the forward calls warn where an input needs a gradient, the way back is a call of its own (rp_..._grad).
_TYPES = {}


def _torch():
    import torch
    if not _TYPES:
        _TYPES.update({torch.float32: 0, torch.float16: 1, torch.bfloat16: 2})
    return torch


def _current_stream(device: int) -> int:
    """Handle of torch's current stream of a GPU (without the stream object, which takes ten times as long to make)."""
    raw = getattr(_torch()._C, "_cuda_getCurrentRawStream", None)
    return raw(device) if raw is not None else _torch().cuda.current_stream(device).cuda_stream


class _Queue:
    """Stream of a call: its handle, and as a context the stream that new tensors belong to."""
    __slots__ = ("handle", "scope")

    def __init__(self, torch, tensor, stream):
        self.scope = None
        if stream is None:
            self.handle = _current_stream(tensor.get_device())
            return
        if isinstance(stream, int):
            stream = torch.cuda.ExternalStream(stream, device=tensor.device)
        self.handle = stream.cuda_stream
        self.scope = torch.cuda.stream(stream)

    def __enter__(self):
        if self.scope is not None:
            self.scope.__enter__()
        return self

    def __exit__(self, *exc):
        if self.scope is not None:
            self.scope.__exit__(*exc)


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _unrecorded(torch, call: str, *inputs, back: bool = True):
    """Says so where autograd would be expected to follow a call that it does not see."""
    if torch.is_grad_enabled() and any(x is not None and x.requires_grad for x in inputs):
        how = f"call it inside a torch.autograd.Function (or under torch.no_grad()) with {call}_grad for the way back" if back else "it has no way back"
        warnings.warn(f"{call}: an input needs a gradient, but autograd does not record this call and its outputs have none; {how}", stacklevel=3)


def _dense(t, dtype, shape, what: str):
    """Address of a contiguous CUDA tensor of a type and shape; None stays NULL."""
    if t is None:
        return None
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous() or not t.is_cuda:
        raise ValueError(f"{what}: contiguous CUDA tensor {tuple(shape)} of {dtype} wanted, got {tuple(t.shape)} of {t.dtype} on {t.device}")
    return t.data_ptr()


def _starts(torch, start):
    """(address, number of samples) of a tensor of starts."""
    if start.dim() != 1 or start.shape[0] < 2:
        raise ValueError("start: [n + 1] wanted")
    return _dense(start, torch.int64, start.shape, "start"), start.shape[0] - 1


_ROUTE_TYPES = ("torch.uint8", "torch.int16", "torch.int32", "torch.int64")


def _route_layout(routes):
    """(bytes of a route, strides of all dimensions but the last) of recorded routes."""
    if str(routes.dtype) not in _ROUTE_TYPES or not routes.is_cuda:
        raise ValueError(f"routes: a CUDA tensor of uint8, int16, int32 or int64 wanted, got {routes.dtype} on {routes.device}")
    if routes.shape[-1] != 1 and routes.stride(-1) != 1:
        raise ValueError("routes: a token's choices have to lie side by side")
    return (routes.element_size(), *routes.stride()[:-1])


def rp_count_routes(routes, start, n_experts: int, demand=None, stream=None):
    """Per-expert counts [n_samples, n_layers, n_experts] int32 of recorded routes [n_tokens, n_layers, top_k]."""
    torch = _torch()
    _need(routes.dim() == 3, "routes: [n_tokens, n_layers, top_k] wanted")
    T, L, k = routes.shape
    size, ts, ls = _route_layout(routes)
    at, n = _starts(torch, start)
    with _Queue(torch, routes, stream) as queue:
        if demand is None:
            demand = routes.new_empty((n, L, n_experts), dtype=torch.int32)
        _check(lib().rp_count_routes(routes.data_ptr() or at, size, T, L, k, n_experts, ts, ls, at, n,
                                     _dense(demand, torch.int32, (n, L, n_experts), "demand"), queue.handle), "rp_count_routes")
    return demand


SCORES = dict(softmax=0, sigmoid=1)


# Structures are kept for numbers, never for objects: what a caller's tensor or array holds may be another number at the next call.
@functools.lru_cache(maxsize=256)
def _router(n_experts, top_k, kind, score, normalise, scale, loss_coef):
    r = rp_router(n_experts, top_k, kind, SCORES[score], normalise, scale, loss_coef)
    return r, C.byref(r)


def _rows(x, what: str):
    """Stride of the rows of a matrix."""
    if x.dim() != 2 or not x.is_cuda or (x.shape[1] != 1 and x.stride(1) != 1):
        raise ValueError(f"{what}: a CUDA tensor [n_tokens, n] with its last dimension side by side wanted")
    return x.stride(0)


def _kind(x, what: str):
    kind = _TYPES.get(x.dtype)
    if kind is None:
        raise ValueError(f"{what}: float32, float16 or bfloat16 wanted, got {x.dtype}")
    return kind


def rp_route(logits, top_k: int, start, *, score: str = "softmax", normalise: bool = True, scale: float = 1.0, loss_coef: float = 0.0,
             choice_bias=None, replay=None, routes=None, gates=None, counts=None, loss=None, stream=None):
    """Router of one layer: (routes [T, k], gates [T, k] float32, counts [n_groups, E] int32, loss [1] float32).

    ``replay``: routes of an earlier pass to be taken in place of the largest logits (returned as they are).  ``routes``: where the chosen
    ones go (any integer type, rows with a stride: a slice of a record); int32 by default.
    """
    torch = _torch()
    _unrecorded(torch, "rp_route", logits)
    row = _rows(logits, "logits")
    T, E = logits.shape
    at, n = _starts(torch, start)
    r, ref = _router(E, operator.index(top_k), _kind(logits, "logits"), score, int(normalise), float(scale), float(loss_coef))
    with _Queue(torch, logits, stream) as queue:
        if replay is not None:
            routes = replay
        elif routes is None:
            routes = logits.new_empty((T, top_k), dtype=torch.int32)
        if routes.shape != (T, top_k):
            raise ValueError(f"routes: {(T, top_k)} wanted, got {tuple(routes.shape)}")
        size, step = _route_layout(routes)
        if gates is None:
            gates = logits.new_empty((T, top_k), dtype=torch.float32)
        if counts is None:
            counts = logits.new_empty((n, E), dtype=torch.int32)
        if loss is None:
            loss = logits.new_empty(1, dtype=torch.float32)
        nbytes = lib().rp_route_workspace(ref, n)
        space = logits.new_empty(nbytes, dtype=torch.uint8)
        # (an empty tensor has no address: any will do)
        _check(lib().rp_route(ref, logits.data_ptr() or at, row, T, _dense(choice_bias, torch.float32, (E,), "choice_bias"), at, n,
                              int(replay is not None), routes.data_ptr() or at, size, step,
                              _dense(gates, torch.float32, (T, top_k), "gates") or at, _dense(counts, torch.int32, (n, E), "counts"),
                              _dense(loss, torch.float32, (1,), "loss"), space.data_ptr(), nbytes, queue.handle), "rp_route")
    return routes, gates, counts, loss


def rp_route_grad(logits, routes, start, counts, *, gates_grad=None, loss_grad=None, score: str = "softmax", normalise: bool = True,
                  scale: float = 1.0, loss_coef: float = 0.0, logits_grad=None, stream=None):
    """Gradient for the logits of the gates (``gates_grad`` [T, k] float32) and the balance loss (``loss_grad`` [1] float32) of rp_route."""
    torch = _torch()
    row = _rows(logits, "logits")
    T, E = logits.shape
    if routes.dim() != 2 or routes.shape[0] != T:
        raise ValueError("routes: [n_tokens, top_k] wanted")
    k = routes.shape[1]
    size, step = _route_layout(routes)
    at, n = _starts(torch, start)
    r, ref = _router(E, k, _kind(logits, "logits"), score, int(normalise), float(scale), float(loss_coef))
    with _Queue(torch, logits, stream) as queue:
        if logits_grad is None:
            logits_grad = logits.new_empty((T, E))
        if logits_grad.shape != logits.shape or logits_grad.dtype != logits.dtype:
            raise ValueError("logits_grad: shape and type of the logits wanted")
        if T:
            _check(lib().rp_route_grad(ref, logits.data_ptr(), row, T, routes.data_ptr(), size, step,
                                       _dense(gates_grad, torch.float32, (T, k), "gates_grad"), _dense(loss_grad, torch.float32, (1,), "loss_grad"),
                                       at, n, _dense(counts, torch.int32, (n, E), "counts"), logits_grad.data_ptr(),
                                       _rows(logits_grad, "logits_grad"), queue.handle), "rp_route_grad")
    return logits_grad


LAYOUTS = dict(half=0, interleaved=1)


@functools.lru_cache(maxsize=256)
def _rotary(head_dim, rotary_dim, layout, kind, weight_kind, eps, mscale):
    r = rp_rotary(head_dim, rotary_dim, LAYOUTS[layout], kind, weight_kind, eps, mscale)
    return r, C.byref(r)


def _head_strides(x, like, what: str):
    """Strides of tokens and heads of a tensor of the shape and type of `like`."""
    step = x.stride()
    if (x is not like and (x.shape != like.shape or x.dtype != like.dtype)) or not x.is_cuda or (step[2] != 1 and x.shape[2] != 1):
        raise ValueError(f"{what}: CUDA tensor {tuple(like.shape)} of {like.dtype} with its last dimension side by side wanted, "
                         f"got {tuple(x.shape)} of {x.dtype}")
    return step[0], step[1]


def _rotate(q, k, inv_freq, start, first_position, weights, eps, layout, mscale, outs, grads, stream, axes=None):
    """``axes``: (axis, position) in the place of ``start`` and ``first_position``."""
    torch = _torch()
    _need(q.dim() == 3 and (k is None or (k.dim() == 3 and k.dtype == q.dtype and k.shape[0] == q.shape[0] and k.shape[2] == q.shape[2])),
          "q and k: [n_tokens, n_heads, head_dim] of one type, as many tokens and one head size wanted")
    T, _, d = q.shape
    kind = _kind(q, "q")
    if axes is None:
        at, n = _starts(torch, start)
    else:
        _need(inv_freq is not None, "inv_freq: [rotary_dim / 2] wanted")
        axis, place = axes
        if place.dim() != 2 or place.shape[1] != T or place.dtype != torch.int64 or not place.is_cuda:
            raise ValueError(f"position: CUDA tensor [n_axes, {T}] of int64 wanted, got {tuple(place.shape)} of {place.dtype} on {place.device}")
        table = rp_axes(place.shape[0], _dense(axis, torch.int32, inv_freq.shape, "axis"), place.data_ptr(), *place.stride())
    w_type = next((w.dtype for w in weights if w is not None), q.dtype)
    _need(w_type == q.dtype or w_type == torch.float32, "weights: float32 or the type of q wanted")
    back = grads[0] is not None
    with _Queue(torch, q, stream) as queue:
        sides, results, dws = [None, None], [None, None], [None, None]
        for i in (0, 1) if k is not None else (0,):
            x, w, out, g = (q, k)[i], weights[i], outs[i], grads[i]
            xt, xh = _head_strides(x, x, "input")
            if out is None:
                out = _like(torch, x)
                yt, yh = x.shape[1] * d, d
            else:
                yt, yh = _head_strides(out, x, "output")
            results[i] = out
            if not back:
                side = rp_heads(x.shape[1], x.data_ptr(), xt, xh, out.data_ptr(), yt, yh, _dense(w, w_type, (d,), "weight"))
            else:
                gt, gh = _head_strides(g, x, "gradient")
                if w is not None:
                    dws[i] = (x.new_empty if x.shape[1] else x.new_zeros)(d, dtype=torch.float32)        # (without heads nothing is written)
                side = rp_heads(x.shape[1], x.data_ptr(), xt, xh, out.data_ptr(), yt, yh, _dense(w, w_type, (d,), "weight"), g.data_ptr(), gt, gh,
                                None if w is None else dws[i].data_ptr())
            sides[i] = C.byref(side)
        freq = None if inv_freq is None else _dense(inv_freq, torch.float64, inv_freq.shape, "inv_freq")
        r, ref = _rotary(d, 0 if inv_freq is None else 2 * inv_freq.numel(), layout, kind, _TYPES[w_type], float(eps), float(mscale))
        if axes is None:
            forward, backward, name = lib().rp_rotate, lib().rp_rotate_grad, "rp_rotate"
            args = (ref, T, freq, at, n, _dense(first_position, torch.int64, (n,), "first_position"), *sides)
        else:
            forward, backward, name = lib().rp_rotate_axes, lib().rp_rotate_axes_grad, "rp_rotate_axes"
            args = (ref, T, freq, C.byref(table), *sides)
        if not T:
            for dw in dws:
                if dw is not None:
                    dw.zero_()
        elif not back:
            _check(forward(*args, queue.handle), name)
        else:
            space, nbytes = None, 0
            if dws[0] is not None or dws[1] is not None:
                nbytes = lib().rp_rotate_workspace(ref)
                space = q.new_empty(nbytes, dtype=torch.uint8)
            _check(backward(*args, None if space is None else space.data_ptr(), nbytes, queue.handle), name + "_grad")
    return results, dws


def rp_rotate(q, k, inv_freq, start, *, first_position=None, q_weight=None, k_weight=None, eps: float = 1e-6, layout: str = "half",
              mscale: float = 1.0, q_out=None, k_out=None, stream=None):
    """Norm of each head (where there is a weight) and rotation by the position in the sample: (q, k) of [n_tokens, n_heads, head_dim].

    ``inv_freq`` float64 [rotary_dim / 2] on the GPU, radians per position (None: no rotation); ``k`` may be None; outputs may be the inputs.
    """
    _unrecorded(_torch(), "rp_rotate", q, k, q_weight, k_weight)
    results, _ = _rotate(q, k, inv_freq, start, first_position, (q_weight, k_weight), eps, layout, mscale, (q_out, k_out), (None, None), stream)
    return tuple(results)


def rp_rotate_grad(q_out_grad, k_out_grad, q, k, inv_freq, start, *, first_position=None, q_weight=None, k_weight=None, eps: float = 1e-6,
                   layout: str = "half", mscale: float = 1.0, q_grad=None, k_grad=None, stream=None):
    """Gradients of rp_rotate: (q_grad, k_grad, q_weight_grad, k_weight_grad), the weights' in float32, None where there is no weight."""
    _need(q_out_grad is not None and (k is None) == (k_out_grad is None), "a gradient for each of q and k wanted")
    results, dws = _rotate(q, k, inv_freq, start, first_position, (q_weight, k_weight), eps, layout, mscale, (q_grad, k_grad),
                           (q_out_grad, k_out_grad), stream)
    return (*results, *dws)


def rp_rotate_axes(q, k, inv_freq, axis, position, *, q_weight=None, k_weight=None, eps: float = 1e-6, layout: str = "half", mscale: float = 1.0,
                   q_out=None, k_out=None, stream=None):
    """rp_rotate with positions on several axes: pair p of token t is turned by position[axis[p], t] * inv_freq[p].

    ``axis`` int32 [rotary_dim / 2] (what is none of the axes turns nothing), ``position`` int64 [n_axes, n_tokens] with any strides, 8 axes at most, all on the GPU.
    """
    _unrecorded(_torch(), "rp_rotate_axes", q, k, q_weight, k_weight)
    results, _ = _rotate(q, k, inv_freq, None, None, (q_weight, k_weight), eps, layout, mscale, (q_out, k_out), (None, None), stream, (axis, position))
    return tuple(results)


def rp_rotate_axes_grad(q_out_grad, k_out_grad, q, k, inv_freq, axis, position, *, q_weight=None, k_weight=None, eps: float = 1e-6, layout: str = "half",
                        mscale: float = 1.0, q_grad=None, k_grad=None, stream=None):
    """Gradients of rp_rotate_axes, as those of rp_rotate."""
    _need(q_out_grad is not None and (k is None) == (k_out_grad is None), "a gradient for each of q and k wanted")
    results, dws = _rotate(q, k, inv_freq, None, None, (q_weight, k_weight), eps, layout, mscale, (q_grad, k_grad), (q_out_grad, k_out_grad), stream,
                           (axis, position))
    return (*results, *dws)


@functools.lru_cache(maxsize=256)
def _attention(q_heads, kv_heads, head_dim, kind, causal, scale):
    a = rp_attend_config(q_heads, kv_heads, head_dim, kind, causal, head_dim ** -0.5 if scale is None else scale)
    return a, C.byref(a)


def _config(q, k, causal, scale):
    """What a call's heads and numbers are kept by."""
    return q.shape[1], k.shape[1], q.shape[2], _kind(q, "q"), int(causal), None if scale is None else float(scale)


def _view(x, like, what: str):
    token, head = _head_strides(x, like, what)
    return C.byref(rp_view(x.data_ptr(), token, head))


def _lse_view(x, T, H, torch):
    if x.shape != (T, H) or x.dtype != torch.float32 or not x.is_cuda:
        raise ValueError(f"lse: CUDA tensor {(T, H)} of float32 wanted, got {tuple(x.shape)} of {x.dtype}")
    return C.byref(rp_view(x.data_ptr(), x.stride(0), x.stride(1)))


def _attend_args(torch, q, k, v, start, causal, scale):
    _need(q.dim() == 3 and k.dim() == 3 and k.shape == v.shape and k.dtype == q.dtype and v.dtype == q.dtype and k.shape[0] == q.shape[0]
          and k.shape[2] == q.shape[2], "q, k and v: [n_tokens, n_heads, head_dim] of one type, as many tokens and one head size wanted")
    at, n = _starts(torch, start)
    return _config(q, k, causal, scale), at, n


def _hand_out(status, space, T, torch):
    """What the kernels leave at the front of their workspace goes into a tensor of the caller's."""
    if status is not None:
        status.copy_(space[:4].view(torch.int32)) if T else status.zero_()


def _like(torch, x):
    """A new dense tensor of the shape and type of `x` (the shorter way where it is dense itself)."""
    return torch.empty_like(x) if x.is_contiguous() else x.new_empty(x.shape)


@functools.lru_cache(maxsize=256)
def _attend_space(call: str, config, *sizes):
    """Bytes of the workspace that a call with these heads and sizes wants."""
    return getattr(lib(), call + "_workspace")(_attention(*config)[1], *sizes)


def _int32(x, what: str) -> int:
    """A whole number for the C entries, what lies outside 32 bits as the next that does not (a window longer than any row, or one that is refused)."""
    try:
        return max(-0x80000000, min(0x7fffffff, operator.index(x)))
    except TypeError:
        raise ValueError(f"{what}: a whole number wanted, got {x!r}") from None


def _attend(window, q, k, v, start, causal, scale, out, lse, status, stream):
    torch = _torch()
    config, at, n = _attend_args(torch, q, k, v, start, causal, scale)
    ref = _attention(*config)[1]
    T, H, _ = q.shape
    _dense(status, torch.int32, (1,), "status")
    with _Queue(torch, q, stream) as queue:
        if out is None:
            out = _like(torch, q)
        if lse is None:
            lse = q.new_empty((H, T), dtype=torch.float32).t()      # a head's rows side by side: what the backward pass reads fastest
        nbytes = _attend_space("rp_attend", config, T, n)
        space = q.new_empty(max(nbytes, 16), dtype=torch.uint8)
        if T:
            args = (T, _view(q, q, "q"), _view(k, k, "k"), _view(v, v, "v"), at, n, _view(out, q, "out"), _lse_view(lse, T, H, torch), space.data_ptr(), nbytes,
                    queue.handle)
            if window is None:
                _check(lib().rp_attend(ref, *args), "rp_attend")
            else:
                _check(lib().rp_attend_window(ref, *window, *args), "rp_attend_window")
        _hand_out(status, space, T, torch)
    return out, lse


def _attend_grad(window, out_grad, q, k, v, out, lse, start, causal, scale, q_grad, k_grad, v_grad, status, stream):
    torch = _torch()
    config, at, n = _attend_args(torch, q, k, v, start, causal, scale)
    ref = _attention(*config)[1]
    T, H, _ = q.shape
    _dense(status, torch.int32, (1,), "status")
    with _Queue(torch, q, stream) as queue:
        q_grad = _like(torch, q) if q_grad is None else q_grad
        k_grad = _like(torch, k) if k_grad is None else k_grad
        v_grad = _like(torch, v) if v_grad is None else v_grad
        nbytes = _attend_space("rp_attend_grad", config, T, n) if window is None else _attend_space("rp_attend_window_grad", config, *window, T, n)
        space = q.new_empty(max(nbytes, 16), dtype=torch.uint8)
        if T:
            args = (T, _view(q, q, "q"), _view(k, k, "k"), _view(v, v, "v"), _view(out, q, "out"), _lse_view(lse, T, H, torch), _view(out_grad, q, "out_grad"), at, n,
                    _view(q_grad, q, "q_grad"), _view(k_grad, k, "k_grad"), _view(v_grad, v, "v_grad"), space.data_ptr(), nbytes, queue.handle)
            if window is None:
                _check(lib().rp_attend_grad(ref, *args), "rp_attend_grad")
            else:
                _check(lib().rp_attend_window_grad(ref, *window, *args), "rp_attend_window_grad")
        _hand_out(status, space, T, torch)
    return q_grad, k_grad, v_grad


def rp_attend(q, k, v, start, *, causal: bool = True, scale: Optional[float] = None, out=None, lse=None, status=None, stream=None):
    """Attention inside the samples of a packed row: (out [n_tokens, q_heads, head_dim], lse [n_tokens, q_heads] float32).

    ``q`` [n_tokens, q_heads, head_dim], ``k`` and ``v`` [n_tokens, kv_heads, head_dim] of float16 or bfloat16; ``scale`` is head_dim ** -0.5 by default.
    ``status``: [1] int32 on the GPU, receives 0, or -8 (RP_ERR_TIMEOUT) where a wait inside the kernel ran out (outputs that were not worked out are NaN then).
    """
    _unrecorded(_torch(), "rp_attend", q, k, v)
    return _attend(None, q, k, v, start, causal, scale, out, lse, status, stream)


def rp_attend_grad(out_grad, q, k, v, out, lse, start, *, causal: bool = True, scale: Optional[float] = None, q_grad=None, k_grad=None, v_grad=None,
                   status=None, stream=None):
    """Gradients (q_grad, k_grad, v_grad) of rp_attend from that of its output, its inputs, ``out`` and ``lse``; ``status`` as there."""
    return _attend_grad(None, out_grad, q, k, v, out, lse, start, causal, scale, q_grad, k_grad, v_grad, status, stream)


def rp_attend_window(q, k, v, start, *, window: int, sinks: int = 0, scale: Optional[float] = None, out=None, lse=None, status=None, stream=None):
    """Attention with a sliding window: token i of a sample sees its tokens j <= i with i - j < ``window`` or j < ``sinks`` (0 to 128); all else as rp_attend."""
    _unrecorded(_torch(), "rp_attend_window", q, k, v)
    return _attend((_int32(window, "window"), _int32(sinks, "sinks")), q, k, v, start, True, scale, out, lse, status, stream)


def rp_attend_window_grad(out_grad, q, k, v, out, lse, start, *, window: int, sinks: int = 0, scale: Optional[float] = None, q_grad=None, k_grad=None,
                          v_grad=None, status=None, stream=None):
    """Gradients (q_grad, k_grad, v_grad) of rp_attend_window, as those of rp_attend."""
    return _attend_grad((_int32(window, "window"), _int32(sinks, "sinks")), out_grad, q, k, v, out, lse, start, True, scale, q_grad, k_grad, v_grad, status, stream)


def rp_attend_step(q, k, v, start, *, length=None, window: int = 0, sinks: int = 0, scale: Optional[float] = None, out=None, lse=None, status=None,
                   stream=None):
    """Attention of one new token of each sequence against its cache: (out [n_samples, q_heads, head_dim], lse [n_samples, q_heads] float32).

    ``q`` [n_samples, q_heads, head_dim]; ``k`` and ``v`` [n_tokens, kv_heads, head_dim]: sequence i has the rows start[i] to start[i + 1], the first ``length[i]`` of
    them filled (int64; None: all), the last of those the new token's own.  The token sees the last ``window`` filled rows (0: all) and the first ``sinks``.
    ``status`` as in rp_attend.
    """
    torch = _torch()
    _unrecorded(torch, "rp_attend_step", q, k, v, back=False)
    _need(q.dim() == 3 and k.dim() == 3 and k.shape == v.shape and k.dtype == q.dtype and v.dtype == q.dtype and k.shape[2] == q.shape[2],
          "q [n_samples, q_heads, head_dim], k and v [n_tokens, kv_heads, head_dim] of one type and head size wanted")
    at, n = _starts(torch, start)
    N, H, _ = q.shape
    _need(N == n, "q: a token for each sequence wanted")
    config = _config(q, k, True, scale)
    ref = _attention(*config)[1]
    window, sinks, T = _int32(window, "window"), _int32(sinks, "sinks"), k.shape[0]
    _dense(status, torch.int32, (1,), "status")
    with _Queue(torch, q, stream) as queue:
        if out is None:
            out = _like(torch, q)
        if lse is None:
            lse = q.new_empty((N, H), dtype=torch.float32)
        nbytes = _attend_space("rp_attend_step", config, window, sinks, T, n)
        space = q.new_empty(max(nbytes, 16), dtype=torch.uint8)
        _check(lib().rp_attend_step(ref, window, sinks, T, _view(q, q, "q"), _view(k, k, "k"), _view(v, v, "v"), at, n, _dense(length, torch.int64, (n,), "length"),
                                    _view(out, q, "out"), _lse_view(lse, N, H, torch), space.data_ptr(), nbytes, queue.handle), "rp_attend_step")
        _hand_out(status, space, 1, torch)
    return out, lse


# ---- inspection hooks -------------------------------------------------------------------
DUMP = dict(LAGG=1, Q=2, SEED_LAYOUT=3, POPULATION=4, W=5, CELL_T=6, CELL_Q=7, CELL_CNT=8, ESUM=9,
            TRACE_TERM=10, TRACE_BEST=11, TRACE_BEST_STEP=12, TRACE_DIGEST=13, TRACE_ANC=14,
            TRACE_INCUMBENT=15, EVAL_W=16, SELECT_DIST=17, SLACK=18)


def rp_debug_set_trace(ctx: Context, on: bool = True):
    _check(lib().rp_debug_set_trace(ctx.handle, int(on)), "rp_debug_set_trace")


STAGES = ("check_reduce", "placement", "projection", "pack_rows", "seed_eval", "best_check")


def rp_debug_set_stage_timing(on: bool = True):
    _check(lib().rp_debug_set_stage_timing(int(on)), "rp_debug_set_stage_timing")


def rp_debug_stage_times(ctx: Context) -> dict:
    """Device milliseconds of the front-end stages of this context (None where a stage has not run)."""
    ms = np.zeros(6, np.float64)
    _check(lib().rp_debug_stage_times(ctx.handle, _ptr(ms)), "rp_debug_stage_times")
    return {k: (float(v) if v >= 0 else None) for k, v in zip(STAGES, ms)}


KNOB = dict(BARRIER_WORKSPACE=1, WAIT_POLLS=2, STALL_ONE_CHAIN=3, RANK_LOAD_SLICES=4, LAUNCH_PER_LEVEL=5,
            CHAIN_KERNEL=6, RESIDENT_SMS=7)


def rp_debug_set_knob(ctx: Context, knob: str, value: int):
    _check(lib().rp_debug_set_knob(ctx.handle, KNOB[knob], int(value)), f"rp_debug_set_knob({knob})")


def rp_debug_set_wait_limit(nanoseconds: int = 2_000_000_000):
    """Limit of the waits inside the attention kernels; 0: they give up at once."""
    _check(lib().rp_debug_set_wait_limit(int(nanoseconds)), "rp_debug_set_wait_limit")


def rp_debug_dump(ctx: Context, what: str, shape, dtype, index: int = 0) -> np.ndarray:
    out = np.empty(shape, dtype)
    _check(lib().rp_debug_dump(ctx.handle, DUMP[what], index, _ptr(out), out.nbytes), f"rp_debug_dump({what})")
    return out


def rp_debug_nl2(x) -> np.ndarray:
    x = np.ascontiguousarray(x, np.uint32)
    out = np.empty(x.shape, np.uint64)
    _check(lib().rp_debug_nl2(_ptr(x), _ptr(out), x.size), "rp_debug_nl2")
    return out


def rp_debug_exp2neg(z) -> np.ndarray:
    z = np.ascontiguousarray(z, np.uint64)
    out = np.empty(z.shape, np.uint64)
    _check(lib().rp_debug_exp2neg(_ptr(z), _ptr(out), z.size), "rp_debug_exp2neg")
    return out


def rp_debug_l2_read_rate(nbytes: int = 32 << 20, reps: int = 50) -> float:
    """Measured read bandwidth (GB/s) of a buffer of `nbytes` that stays in L2."""
    out = C.c_double(0.0)
    _check(lib().rp_debug_l2_read_rate(nbytes, reps, C.byref(out)), "rp_debug_l2_read_rate")
    return float(out.value)


CHAIN_KERNELS = ("k_anneal_wpc", "k_anneal_level", "k_anneal_warp", "k_anneal_row")


def rp_debug_chain_kernel(ctx: Context) -> str:
    """Name of the chain kernel rp_anneal runs for this context (after rp_pack_rows)."""
    out = C.c_int32(-1)
    _check(lib().rp_debug_chain_kernel(ctx.handle, C.byref(out)), "rp_debug_chain_kernel")
    return CHAIN_KERNELS[out.value]


CHAIN_FORMS = ("none", "all levels", "whole layers", "dealt out", "compressed", "two to a warp")


def rp_debug_chain_form(ctx: Context) -> str:
    """Form of the one-layer-per-lane kernel that the last rp_anneal call ran."""
    out = C.c_int32(-1)
    _check(lib().rp_debug_chain_form(ctx.handle, C.byref(out)), "rp_debug_chain_form")
    return CHAIN_FORMS[out.value]


def rp_debug_launch_count() -> int:
    return int(lib().rp_debug_launch_count())


def rp_debug_philox(ctr, key) -> np.ndarray:
    ctr = np.ascontiguousarray(ctr, np.uint32)
    key = np.ascontiguousarray(key, np.uint32)
    out = np.empty(ctr.shape, np.uint32)
    _check(lib().rp_debug_philox(_ptr(ctr), _ptr(key), _ptr(out), ctr.shape[0]), "rp_debug_philox")
    return out
