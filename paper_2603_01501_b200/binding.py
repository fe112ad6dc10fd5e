"""Thin ctypes binding of the C ABI in ``include/gac.h``: argument marshalling
only.  Every step of the path runs in the CUDA library; if the library is
missing this module raises -- there is no CPU fallback.

PyTorch appears here only as the owner of device memory and streams.
"""
from __future__ import annotations

import ctypes
import os
import struct
from dataclasses import dataclass
from typing import List, Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# GAC_B200_LIBRARY selects another build of the same library (a debug build, or one compiled with
# another launch-geometry table through -DGAC_GEOMETRY_HEADER); the default is the in-tree build.
LIB_PATH = os.environ.get("GAC_B200_LIBRARY") or os.path.join(_HERE, "libgac_b200.so")

GAC_OK, GAC_ERR_INVALID_ARG, GAC_ERR_DTYPE, GAC_ERR_CUDA, GAC_ERR_STATE, GAC_ERR_NONFINITE, \
    GAC_ERR_TIMEOUT = range(7)
GAC_F32, GAC_BF16 = 0, 1
GAC_REGIME_SAFE, GAC_REGIME_PROJECT, GAC_REGIME_VIOLATION = 0, 1, 2
GAC_MODE_ADAPTIVE, GAC_MODE_FIXED = 0, 1
GAC_STATE_RAW, GAC_STATE_PROJECTED, GAC_STATE_HOLD, GAC_STATE_EXCHANGE = 0, 1, 2, 3
GAC_SET_G, GAC_SET_D = 0, 1
REGIME_NAMES = {0: "safe", 1: "project", 2: "violation"}


class gac_tensor(ctypes.Structure):
    _fields_ = [("g", ctypes.c_void_p), ("d", ctypes.c_void_p), ("numel", ctypes.c_uint64)]


class gac_hparams(ctypes.Structure):
    _fields_ = [("c_low", ctypes.c_double), ("c_high", ctypes.c_double), ("eps", ctypes.c_double),
                ("beta", ctypes.c_double), ("mode", ctypes.c_int32), ("state_mode", ctypes.c_int32),
                ("alpha_fixed", ctypes.c_double), ("zero_on_violation", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("clip_max_norm", ctypes.c_double),
                ("clip_eps", ctypes.c_double)]


class gac_result(ctypes.Structure):
    _fields_ = [("dot", ctypes.c_double), ("gg", ctypes.c_double), ("dd", ctypes.c_double),
                ("cos", ctypes.c_double), ("alpha", ctypes.c_double), ("coef64", ctypes.c_double),
                ("coef", ctypes.c_float), ("regime", ctypes.c_int32), ("nonfinite", ctypes.c_int32),
                ("staleness", ctypes.c_uint32), ("step", ctypes.c_uint64),
                ("out_norm", ctypes.c_double), ("clip_scale", ctypes.c_double),
                ("applied_steps", ctypes.c_uint64), ("g_set", ctypes.c_uint32),
                ("out_set", ctypes.c_uint32), ("ref_lost", ctypes.c_uint32),
                ("timed_out", ctypes.c_uint32)]

    def as_dict(self):
        return {k: getattr(self, k) for k, _ in self._fields_}


class gac_opt_tensor(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("m", ctypes.c_void_p), ("v", ctypes.c_void_p)]


class gac_adamw(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("weight_decay", ctypes.c_double)]


class gac_info(ctypes.Structure):
    _fields_ = [("total_elems", ctypes.c_uint64), ("n_chunks", ctypes.c_uint64),
                ("n_tensors", ctypes.c_uint32), ("grid", ctypes.c_uint32),
                ("threads", ctypes.c_uint32), ("chunk_elems", ctypes.c_uint32),
                ("launches", ctypes.c_uint64), ("misaligned_tensors", ctypes.c_uint32),
                ("reserved", ctypes.c_uint32)]


GAC_ROTARY_HALF, GAC_ROTARY_INTERLEAVED = 0, 1
GAC_ROTARY_NONE, GAC_ROTARY_LINEAR, GAC_ROTARY_BASE, GAC_ROTARY_PARTS = 0, 1, 2, 3
ROTARY_LAYOUTS = {"half": GAC_ROTARY_HALF, "interleaved": GAC_ROTARY_INTERLEAVED}
ROTARY_SCALINGS = {"none": GAC_ROTARY_NONE, "linear": GAC_ROTARY_LINEAR, "base": GAC_ROTARY_BASE,
                   "parts": GAC_ROTARY_PARTS}


class gac_clip_tensor(ctypes.Structure):
    _fields_ = [("g", ctypes.c_void_p), ("out", ctypes.c_void_p), ("numel", ctypes.c_uint64),
                ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class gac_clip_result(ctypes.Structure):
    _fields_ = [("sumsq", ctypes.c_double), ("norm", ctypes.c_double), ("scale", ctypes.c_double),
                ("nonfinite", ctypes.c_int32), ("timed_out", ctypes.c_int32)]


class gac_rotary_heads(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("y", ctypes.c_void_p), ("x_token", ctypes.c_int64),
                ("x_head", ctypes.c_int64), ("y_token", ctypes.c_int64), ("y_head", ctypes.c_int64)]


class gac_rotary_args(ctypes.Structure):
    _fields_ = [("qk", gac_rotary_heads * 2), ("heads", ctypes.c_uint32 * 2), ("n_tokens", ctypes.c_uint32),
                ("n_seqs", ctypes.c_uint32), ("head_dim", ctypes.c_uint32), ("rot_dim", ctypes.c_uint32),
                ("dtype", ctypes.c_int32), ("layout", ctypes.c_int32), ("inverse", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("positions", ctypes.c_void_p), ("cu_seqlens", ctypes.c_void_p),
                ("freqs", ctypes.c_void_p), ("scale", ctypes.c_double)]


class gac_attn_heads(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("token", ctypes.c_int64), ("head", ctypes.c_int64)]


class gac_attn(ctypes.Structure):
    _fields_ = [("q", gac_attn_heads), ("k", gac_attn_heads), ("v", gac_attn_heads), ("o", gac_attn_heads),
                ("lse", ctypes.c_void_p), ("cu_seqlens", ctypes.c_void_p), ("n_tokens", ctypes.c_uint32),
                ("n_seqs", ctypes.c_uint32), ("q_heads", ctypes.c_uint32), ("kv_heads", ctypes.c_uint32),
                ("head_dim", ctypes.c_uint32), ("dtype", ctypes.c_int32), ("scale", ctypes.c_float),
                ("reserved", ctypes.c_int32)]


class gac_attn_grad(ctypes.Structure):
    _fields_ = [("d_o", gac_attn_heads), ("d_q", gac_attn_heads), ("d_k", gac_attn_heads), ("d_v", gac_attn_heads),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


EXPORTS = ["gac_default_hparams", "gac_init", "gac_stats", "gac_stats_partial", "gac_decide",
           "gac_project", "gac_free", "gac_last_error", "gac_set_launch", "gac_get_info",
           "gac_stats_static", "gac_default_adamw", "gac_attach_adamw", "gac_project_adamw",
           "gac_rebind", "gac_next_gradient_set", "gac_exchange_bytes", "gac_exchange_attach",
           "gac_stats_exchange", "gac_decide_exchange", "gac_clip_init", "gac_clip_rebind", "gac_clip_sumsq",
           "gac_clip_apply", "gac_clip_grad_norm", "gac_clip_set_timeout", "gac_clip_free", "gac_rotary_freqs", "gac_rotary",
           "gac_attn_workspace",
           "gac_attn_forward", "gac_attn_backward", "gac_attn_check"]

_lib = None


class GacError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"gac status {status}: {message}")
        self.status = status


def load_library() -> ctypes.CDLL:
    """Loads the in-tree CUDA library; raises if it was not built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with "
                          "`python -m paper_2603_01501_b200.build` (needs nvcc); "
                          "this package has no CPU fallback")
    L = ctypes.CDLL(LIB_PATH)
    vp, u32, u64, i32 = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_int
    L.gac_default_hparams.argtypes = [ctypes.POINTER(gac_hparams)]
    L.gac_default_hparams.restype = None
    L.gac_init.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(gac_tensor), u32, i32, i32,
                           ctypes.POINTER(gac_hparams), i32]
    L.gac_stats.argtypes = [vp, u64, u32, vp, ctypes.POINTER(gac_result)]
    L.gac_stats_partial.argtypes = [vp, u64, u32, vp, vp]
    L.gac_decide.argtypes = [vp, vp, vp, ctypes.POINTER(gac_result)]
    L.gac_project.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(gac_result)]
    L.gac_free.argtypes = [vp]
    L.gac_last_error.argtypes = [vp]
    L.gac_last_error.restype = ctypes.c_char_p
    L.gac_set_launch.argtypes = [vp, i32, i32]
    L.gac_get_info.argtypes = [vp, ctypes.POINTER(gac_info)]
    L.gac_stats_static.argtypes = [ctypes.POINTER(gac_tensor), u32, i32, i32,
                                   ctypes.POINTER(gac_hparams), u64, u32, i32, vp, vp]
    L.gac_stats_static.restype = i32
    L.gac_rebind.argtypes = [vp, ctypes.POINTER(gac_tensor), u32]
    L.gac_rebind.restype = i32
    L.gac_next_gradient_set.argtypes = [vp, ctypes.POINTER(ctypes.c_int)]
    L.gac_next_gradient_set.restype = i32
    L.gac_default_adamw.argtypes = [ctypes.POINTER(gac_adamw)]
    L.gac_default_adamw.restype = None
    L.gac_attach_adamw.argtypes = [vp, ctypes.POINTER(gac_opt_tensor), u32, u64]
    L.gac_attach_adamw.restype = i32
    L.gac_project_adamw.argtypes = [vp, vp, ctypes.POINTER(gac_adamw), ctypes.POINTER(ctypes.c_float),
                                    ctypes.POINTER(gac_result)]
    L.gac_project_adamw.restype = i32
    L.gac_exchange_bytes.argtypes = [u32]
    L.gac_exchange_bytes.restype = ctypes.c_size_t
    L.gac_exchange_attach.argtypes = [vp, u32, u32, ctypes.POINTER(vp), u32]
    L.gac_exchange_attach.restype = i32
    L.gac_stats_exchange.argtypes = [vp, u64, u32, vp]
    L.gac_stats_exchange.restype = i32
    L.gac_decide_exchange.argtypes = [vp, vp, ctypes.POINTER(gac_result)]
    L.gac_decide_exchange.restype = i32
    P, f64 = ctypes.POINTER, ctypes.c_double
    L.gac_clip_init.argtypes = [P(vp), P(gac_clip_tensor), u32, i32]
    L.gac_clip_rebind.argtypes = [vp, P(gac_clip_tensor), u32, vp]
    L.gac_clip_sumsq.argtypes = [vp, vp, vp]
    L.gac_clip_apply.argtypes = [vp, vp, vp, f64, f64, vp, P(gac_clip_result)]
    L.gac_clip_grad_norm.argtypes = [vp, vp, f64, f64, vp, P(gac_clip_result)]
    L.gac_clip_set_timeout.argtypes = [vp, u32]
    L.gac_clip_free.argtypes = [vp]
    L.gac_rotary_freqs.argtypes = [P(f64), u32, f64, i32, f64, f64, f64, f64]
    # the structs travel as packed bytes (or ctypes.byref of the structures above)
    L.gac_rotary.argtypes = [vp, i32, vp]
    L.gac_attn_workspace.argtypes = [vp]
    L.gac_attn_workspace.restype = ctypes.c_size_t
    L.gac_attn_forward.argtypes = [vp, i32, vp]
    L.gac_attn_backward.argtypes = [vp, vp, i32, vp]
    L.gac_attn_check.argtypes = [i32, vp]
    for name in ("gac_clip_init", "gac_clip_rebind", "gac_clip_sumsq", "gac_clip_apply", "gac_clip_grad_norm", "gac_clip_set_timeout",
                 "gac_clip_free", "gac_rotary_freqs", "gac_rotary", "gac_attn_forward", "gac_attn_backward", "gac_attn_check"):
        getattr(L, name).restype = i32
    for name in ("gac_init", "gac_stats", "gac_stats_partial", "gac_decide", "gac_project",
                 "gac_free", "gac_set_launch", "gac_get_info"):
        getattr(L, name).restype = i32
    _lib = L
    return L


@dataclass
class HParams:
    """Algorithm 1 inputs (c_low, c_high), the cosine's eps (App. A.1) and the
    gains of Eq. 3 / Eq. 5; defaults are the paper's."""
    c_low: float = 0.05
    c_high: float = 0.3
    eps: float = 1e-8
    beta: float = 1.0
    mode: int = GAC_MODE_ADAPTIVE
    alpha_fixed: float = 0.0
    state_mode: int = GAC_STATE_RAW
    zero_on_violation: int = 0
    clip_max_norm: float = 0.0     # > 0 folds global-norm clipping into the projection pass
    clip_eps: float = 1e-6

    def c(self) -> gac_hparams:
        return gac_hparams(self.c_low, self.c_high, self.eps, self.beta, self.mode,
                           self.state_mode, self.alpha_fixed, self.zero_on_violation, 0,
                           self.clip_max_norm, self.clip_eps)


_DT = {torch.float32: GAC_F32, torch.bfloat16: GAC_BF16}


def _stream_ptr(stream) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


class GacContext:
    """Owner of one ``gac_ctx``.  Keeps references to the tensors so that the
    device pointers in the chunk table stay valid."""

    def __init__(self, handle: int, g_list, d_list):
        self.handle = ctypes.c_void_p(handle)
        self._keep = (list(g_list), list(d_list))

    def _check(self, rc: int, allow_nonfinite: bool = False):
        if rc != GAC_OK and not (allow_nonfinite and rc == GAC_ERR_NONFINITE):
            raise GacError(rc, load_library().gac_last_error(self.handle).decode())

    def __del__(self):
        try:
            gac_free(self)
        except Exception:
            pass


def gac_init(g_list: Sequence[torch.Tensor], d_list: Sequence[torch.Tensor],
             hp: Optional[HParams] = None, device: Optional[int] = None) -> GacContext:
    """gac_init of the C ABI on lists of CUDA tensors (g_i, d_i)."""
    L = load_library()
    hp = hp or HParams()
    if len(g_list) != len(d_list):
        raise ValueError("g and d lists differ in length")
    n = len(g_list)
    arr = (gac_tensor * max(n, 1))()
    g_dt = d_dt = None
    for i, (g, d) in enumerate(zip(g_list, d_list)):
        if not (g.is_cuda and d.is_cuda and g.is_contiguous() and d.is_contiguous()):
            raise ValueError("tensors must be contiguous CUDA tensors")
        if g.numel() != d.numel():
            raise ValueError(f"tensor {i}: g and d differ in numel")
        if g.dtype not in _DT or d.dtype not in _DT:
            raise GacError(GAC_ERR_DTYPE, f"unsupported dtype {g.dtype}/{d.dtype}")
        if g_dt is None:
            g_dt, d_dt = g.dtype, d.dtype
        elif (g.dtype, d.dtype) != (g_dt, d_dt):
            raise GacError(GAC_ERR_DTYPE, "all tensors of a list must share one (g,d) dtype pair")
        arr[i] = gac_tensor(g.data_ptr(), d.data_ptr(), g.numel())
    if device is None:
        device = g_list[0].device.index if n else torch.cuda.current_device()
    out = ctypes.c_void_p()
    chp = hp.c()
    rc = L.gac_init(ctypes.byref(out), arr, n, _DT.get(g_dt, 0), _DT.get(d_dt, 0),
                    ctypes.byref(chp), device)
    if rc != GAC_OK:
        raise GacError(rc, L.gac_last_error(None).decode())
    return GacContext(out.value, g_list, d_list)


def gac_stats(ctx: GacContext, step: int, staleness: int = 0, stream=None,
              fetch: bool = True) -> Optional[gac_result]:
    """gac_stats; with fetch=False nothing leaves the device and None is returned."""
    L = load_library()
    res = gac_result() if fetch else None
    rc = L.gac_stats(ctx.handle, step, staleness, _stream_ptr(stream),
                     ctypes.byref(res) if fetch else None)
    ctx._check(rc, allow_nonfinite=True)
    return res


def gac_stats_partial(ctx: GacContext, step: int, sums_out: torch.Tensor, staleness: int = 0,
                      stream=None) -> None:
    if not (sums_out.is_cuda and sums_out.dtype == torch.float64 and sums_out.numel() >= 3):
        raise ValueError("sums_out must be a CUDA float64 tensor of 3 elements")
    ctx._check(load_library().gac_stats_partial(ctx.handle, step, staleness, _stream_ptr(stream),
                                                sums_out.data_ptr()))


def gac_decide(ctx: GacContext, sums_in: torch.Tensor, stream=None,
               fetch: bool = True) -> Optional[gac_result]:
    if not (sums_in.is_cuda and sums_in.dtype == torch.float64 and sums_in.numel() >= 3):
        raise ValueError("sums_in must be a CUDA float64 tensor of 3 elements")
    res = gac_result() if fetch else None
    rc = load_library().gac_decide(ctx.handle, _stream_ptr(stream), sums_in.data_ptr(),
                                   ctypes.byref(res) if fetch else None)
    ctx._check(rc, allow_nonfinite=True)
    return res


def gac_exchange_bytes(world: int) -> int:
    """Size of one rank's slot array for the peer exchange of the three sums."""
    return int(load_library().gac_exchange_bytes(world))


def gac_exchange_attach(ctx: GacContext, rank: int, world: int, slots: Sequence[torch.Tensor],
                        timeout_ms: int = 0) -> None:
    """gac_exchange_attach: `slots[r]` is rank r's slot array (a zero-filled CUDA uint8 tensor of
    gac_exchange_bytes(world) bytes, or an integer device address of one mapped from a peer)."""
    arr = (ctypes.c_void_p * max(world, 1))()
    for r, t in enumerate(slots):
        if isinstance(t, torch.Tensor):
            if not (t.is_cuda and t.is_contiguous() and t.numel() * t.element_size() >= gac_exchange_bytes(world)):
                raise ValueError("a slot array must be a contiguous CUDA tensor of gac_exchange_bytes(world) bytes")
            arr[r] = t.data_ptr()
        else:
            arr[r] = int(t)
    if len(slots) != world:
        raise ValueError("one slot array per rank")
    ctx._check(load_library().gac_exchange_attach(ctx.handle, rank, world, arr, timeout_ms))
    ctx._keep_slots = list(slots)


def gac_stats_exchange(ctx: GacContext, step: int, staleness: int = 0, stream=None) -> None:
    ctx._check(load_library().gac_stats_exchange(ctx.handle, step, staleness, _stream_ptr(stream)))


def gac_decide_exchange(ctx: GacContext, stream=None, fetch: bool = True) -> Optional[gac_result]:
    """gac_decide_exchange; raises GacError(GAC_ERR_TIMEOUT) when fetching a record whose wait ran out."""
    res = gac_result() if fetch else None
    rc = load_library().gac_decide_exchange(ctx.handle, _stream_ptr(stream), ctypes.byref(res) if fetch else None)
    ctx._check(rc, allow_nonfinite=True)
    return res


def gac_project(ctx: GacContext, stream=None, coef_override: Optional[float] = None,
                fetch: bool = False) -> Optional[gac_result]:
    L = load_library()
    res = gac_result() if fetch else None
    k = ctypes.c_float(coef_override) if coef_override is not None else None
    rc = L.gac_project(ctx.handle, _stream_ptr(stream),
                       ctypes.byref(k) if k is not None else None,
                       ctypes.byref(res) if fetch else None)
    ctx._check(rc, allow_nonfinite=True)
    return res


def gac_next_gradient_set(ctx: GacContext) -> int:
    """Exchange mode: GAC_SET_G or GAC_SET_D, the buffer set the next gradient belongs in."""
    out = ctypes.c_int(0)
    ctx._check(load_library().gac_next_gradient_set(ctx.handle, ctypes.byref(out)))
    return out.value


def gac_free(ctx: GacContext) -> None:
    if ctx.handle:
        load_library().gac_free(ctx.handle)
        ctx.handle = ctypes.c_void_p(None)
    # the library no longer touches the buffers: let go of them, so that their owner can free them
    ctx._keep = ([], [])
    for extra in ("_keep_opt", "_keep_slots", "_keep_symm"):
        if hasattr(ctx, extra):
            setattr(ctx, extra, None)


def gac_set_launch(ctx: GacContext, chunk_elems: int = 0, ctas_per_sm: int = 0) -> None:
    ctx._check(load_library().gac_set_launch(ctx.handle, chunk_elems, ctas_per_sm))


def gac_get_info(ctx: GacContext) -> gac_info:
    info = gac_info()
    ctx._check(load_library().gac_get_info(ctx.handle, ctypes.byref(info)))
    return info


def gac_stats_static(g_list: Sequence[torch.Tensor], d_list: Sequence[torch.Tensor], hp: HParams,
                     step: int, result_dev: torch.Tensor, staleness: int = 0, stream=None) -> None:
    """gac_stats_static of the C ABI: the statistics and the decision of one step
    without any allocation by the library (work memory is built into it).
    `result_dev` is a caller-owned CUDA uint8 tensor of at least
    ``ctypes.sizeof(gac_result)`` bytes that receives the record on the stream;
    read it with ``result_from_tensor`` after synchronising."""
    L = load_library()
    if not (result_dev.is_cuda and result_dev.dtype == torch.uint8 and result_dev.is_contiguous()
            and result_dev.numel() >= ctypes.sizeof(gac_result) and result_dev.data_ptr() % 8 == 0):
        raise ValueError("result_dev must be an 8-byte aligned CUDA uint8 tensor of >= sizeof(gac_result) bytes")
    n = len(g_list)
    arr = (gac_tensor * max(n, 1))()
    for i, (g, d) in enumerate(zip(g_list, d_list)):
        arr[i] = gac_tensor(g.data_ptr(), d.data_ptr(), g.numel())
    chp = hp.c()
    g_dt = _DT[g_list[0].dtype] if n else 0
    d_dt = _DT[d_list[0].dtype] if n else 0
    dev = result_dev.device.index
    rc = L.gac_stats_static(arr, n, g_dt, d_dt, ctypes.byref(chp), step, staleness, dev,
                            _stream_ptr(stream), result_dev.data_ptr())
    if rc != GAC_OK:
        raise GacError(rc, L.gac_last_error(None).decode())


def result_from_tensor(t: torch.Tensor) -> gac_result:
    """Decodes a gac_result held in a uint8 tensor (copied to the host here)."""
    raw = bytes(t.detach().cpu().numpy().tobytes()[: ctypes.sizeof(gac_result)])
    return gac_result.from_buffer_copy(raw)


@dataclass
class AdamW:
    """AdamW hyper-parameters; defaults are the paper's (Table 2)."""
    lr: float = 1e-6
    beta1: float = 0.9
    beta2: float = 0.999
    eps: float = 1e-8
    weight_decay: float = 1e-2

    def c(self) -> gac_adamw:
        return gac_adamw(self.lr, self.beta1, self.beta2, self.eps, self.weight_decay)


def gac_attach_adamw(ctx: GacContext, p_list: Sequence[torch.Tensor], m_list: Sequence[torch.Tensor],
                     v_list: Sequence[torch.Tensor], applied_steps: int = 0) -> None:
    """Binds float32 parameters and AdamW moments (one per tensor of the context's list)."""
    n = len(p_list)
    arr = (gac_opt_tensor * max(n, 1))()
    for i, (p, m, v) in enumerate(zip(p_list, m_list, v_list)):
        for t in (p, m, v):
            if not (t.is_cuda and t.is_contiguous() and t.dtype == torch.float32):
                raise ValueError("p, m, v must be contiguous float32 CUDA tensors")
            if t.numel() != ctx._keep[0][i].numel():
                raise ValueError(f"tensor {i}: optimizer state differs in numel from the gradient")
        arr[i] = gac_opt_tensor(p.data_ptr(), m.data_ptr(), v.data_ptr())
    ctx._check(load_library().gac_attach_adamw(ctx.handle, arr, n, applied_steps))
    ctx._keep_opt = (list(p_list), list(m_list), list(v_list))


def gac_project_adamw(ctx: GacContext, opt: AdamW, stream=None, coef_override: Optional[float] = None,
                      fetch: bool = False) -> Optional[gac_result]:
    L = load_library()
    res = gac_result() if fetch else None
    k = ctypes.c_float(coef_override) if coef_override is not None else None
    copt = opt.c()
    rc = L.gac_project_adamw(ctx.handle, _stream_ptr(stream), ctypes.byref(copt),
                             ctypes.byref(k) if k is not None else None,
                             ctypes.byref(res) if fetch else None)
    ctx._check(rc, allow_nonfinite=True)
    return res


def gac_rebind(ctx: GacContext, g_list: Sequence[torch.Tensor], d_list: Sequence[torch.Tensor]) -> None:
    """Points the context at moved buffers of the same sizes (gac_rebind of the C ABI)."""
    n = len(g_list)
    arr = (gac_tensor * max(n, 1))()
    for i, (g, d) in enumerate(zip(g_list, d_list)):
        if not (g.is_cuda and d.is_cuda and g.is_contiguous() and d.is_contiguous()):
            raise ValueError("tensors must be contiguous CUDA tensors")
        arr[i] = gac_tensor(g.data_ptr(), d.data_ptr(), g.numel())
    ctx._check(load_library().gac_rebind(ctx.handle, arr, n))
    ctx._keep = (list(g_list), list(d_list))


# ---------------------------------------------------------------- around the rule: packed rollouts
#
# The calls on lists of gradients (gac_project, gac_clip_*) write tensors that autograd does not save in ordinary use and
# leave their versions alone; gac_rotary in place, on activations, raises them.


# Packed forms of gac_rotary_args, gac_attn and gac_attn_grad: one call instead of one per field.
_ROTARY = struct.Struct("=QQqqqqQQqqqqIIIIIIiiiiQQQd")
_ATTN = struct.Struct("=QqqQqqQqqQqqQQIIIIIifi")
_ATTN_GRAD = struct.Struct("=QqqQqqQqqQqqQQ")
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _on(stream, device: torch.device):
    """(raw stream to launch on, torch stream or None for the current one of the tensors' device).  What a call
    allocates is allocated on that stream, so that the caching allocator hands the memory on in its order."""
    if stream is None:
        return _raw_stream(device.index), None
    if not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(int(stream), device=device)
    return stream.cuda_stream, stream


def _empty(like: torch.Tensor, shape, stream, dtype=None) -> torch.Tensor:
    if stream is None:
        return like.new_empty(shape) if dtype is None else like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(stream):
        return like.new_empty(shape) if dtype is None else like.new_empty(shape, dtype=dtype)


def _check(rc: int) -> None:
    if rc != GAC_OK:
        raise GacError(rc, load_library().gac_last_error(None).decode())


class ClipContext:
    """Owner of one ``gac_clip_ctx``; keeps references to the tensors in its table, unless told that the caller does."""

    def __init__(self, handle: int, device: int, keep: bool):
        self.handle = ctypes.c_void_p(handle)
        self.device = torch.device("cuda", device)
        self._keeps, self._keep = keep, ()

    def _hold(self, g_list, out_list):
        if self._keeps:
            self._keep = (list(g_list), list(out_list))

    def __del__(self):
        try:
            gac_clip_free(self)
        except Exception:
            pass


def _clip_list(g_list, outs, device: int):
    if len(g_list) != len(outs):
        raise ValueError("gradient and output lists differ in length")
    arr = (gac_clip_tensor * max(len(g_list), 1))()
    for i, (g, o) in enumerate(zip(g_list, outs)):
        if not (g.is_cuda and o.is_cuda and g.is_contiguous() and o.is_contiguous()):
            raise ValueError("tensors must be contiguous CUDA tensors")
        if g.numel() != o.numel() or g.dtype != o.dtype:
            raise ValueError(f"tensor {i}: gradient and output differ in numel or dtype")
        if g.dtype not in _DT:
            raise GacError(GAC_ERR_DTYPE, f"unsupported dtype {g.dtype}")
        arr[i] = gac_clip_tensor(g.data_ptr(), o.data_ptr(), g.numel(), _DT[g.dtype], 0)
    if any(t.device.index != device for t in g_list) or any(t.device.index != device for t in outs):
        raise ValueError("all tensors of a list must be on one device")
    return arr


def gac_clip_init(g_list: Sequence[torch.Tensor], out_list: Optional[Sequence[torch.Tensor]] = None,
                  device: Optional[int] = None, keep: bool = True) -> ClipContext:
    """gac_clip_init of the C ABI on a list of contiguous CUDA tensors, float32 and bfloat16 mixed as
    they come.  ``out_list``: where the clipped gradients go; None clips in place.  ``keep=False``: the context holds
    no references, the caller sees to it that the tensors of the last init or rebind are there at every call."""
    L = load_library()
    outs = g_list if out_list is None else out_list
    if device is None:
        device = g_list[0].device.index if len(g_list) else torch.cuda.current_device()
    arr = _clip_list(g_list, outs, device)
    out = ctypes.c_void_p()
    _check(L.gac_clip_init(ctypes.byref(out), arr, len(g_list), device))
    ctx = ClipContext(out.value, device, keep)
    ctx._hold(g_list, outs)
    return ctx


def gac_clip_rebind(ctx: ClipContext, g_list: Sequence[torch.Tensor], out_list: Optional[Sequence[torch.Tensor]] = None,
                    stream=None) -> None:
    """Points the context at moved tensors of the same sizes and types, in stream order and without waiting."""
    outs = g_list if out_list is None else out_list
    arr = _clip_list(g_list, outs, ctx.device.index)
    _check(load_library().gac_clip_rebind(ctx.handle, arr, len(g_list), _on(stream, ctx.device)[0]))
    ctx._hold(g_list, outs)


def _clip_result(rc: int, res) -> Optional[gac_clip_result]:
    if rc not in (GAC_OK, GAC_ERR_NONFINITE):
        _check(rc)
    return res


def _scalar_ptr(t: Optional[torch.Tensor], name: str, dtype: torch.dtype, ctx: ClipContext) -> Optional[int]:
    if t is None:
        return None
    if not (t.is_cuda and t.device == ctx.device and t.dtype == dtype and t.numel() >= 1):
        raise ValueError(f"{name} must be a {str(dtype)[6:]} tensor on the list's device")
    return t.data_ptr()


def gac_clip_grad_norm(ctx: ClipContext, max_norm: float, eps: float = 1e-6, norm_out: Optional[torch.Tensor] = None,
                       stream=None, fetch: bool = False) -> Optional[gac_clip_result]:
    """Norm of the list, and the list scaled by min(1, max_norm/(norm + eps)).  With fetch=False nothing
    leaves the device; a non-finite norm leaves every output as it was and is told by the record.  So is a wait that
    ran out, as a norm of NaN and, with fetch=True, as GacError(GAC_ERR_TIMEOUT)."""
    res = gac_clip_result() if fetch else None
    raw = _on(stream, ctx.device)[0]
    rc = load_library().gac_clip_grad_norm(ctx.handle, raw, max_norm, eps, _scalar_ptr(norm_out, "norm_out", torch.float32, ctx),
                                           ctypes.byref(res) if fetch else None)
    return _clip_result(rc, res)


def gac_clip_sumsq(ctx: ClipContext, sumsq_out: torch.Tensor, stream=None) -> None:
    """Sharded form: this rank's sum of squares into a CUDA float64 tensor, for the caller's all-reduce."""
    to = _scalar_ptr(sumsq_out, "sumsq_out", torch.float64, ctx)
    _check(load_library().gac_clip_sumsq(ctx.handle, _on(stream, ctx.device)[0], to))


def gac_clip_apply(ctx: ClipContext, sumsq_in: torch.Tensor, max_norm: float, eps: float = 1e-6,
                   norm_out: Optional[torch.Tensor] = None, stream=None, fetch: bool = False) -> Optional[gac_clip_result]:
    """Sharded form: scales this rank's list by the factor that follows from the global sum of squares."""
    res = gac_clip_result() if fetch else None
    rc = load_library().gac_clip_apply(ctx.handle, _on(stream, ctx.device)[0],
                                       _scalar_ptr(sumsq_in, "sumsq_in", torch.float64, ctx), max_norm, eps,
                                       _scalar_ptr(norm_out, "norm_out", torch.float32, ctx), ctypes.byref(res) if fetch else None)
    return _clip_result(rc, res)


def gac_clip_set_timeout(ctx: ClipContext, timeout_ms: int) -> None:
    """Longest wait of the CTAs for one another inside gac_clip_grad_norm (1000 ms unless set)."""
    _check(load_library().gac_clip_set_timeout(ctx.handle, timeout_ms))


def gac_clip_free(ctx: ClipContext) -> None:
    if ctx.handle:
        load_library().gac_clip_free(ctx.handle)
        ctx.handle = ctypes.c_void_p(None)
    ctx._keep = ()


def gac_rotary_freqs(rot_dim: int, base: float = 1e4, scaling: str = "none", factor: float = 1.0,
                     trained: float = 4096.0, low: float = 1.0, high: float = 4.0):
    """Radians per position of each pair (a float64 array of rot_dim/2), stretched for contexts ``factor``
    times as long as the trained one; see gac.h for the scalings."""
    import numpy as np
    freqs = np.zeros(max(rot_dim // 2, 1), dtype=np.float64)
    _check(load_library().gac_rotary_freqs(freqs.ctypes.data_as(ctypes.POINTER(ctypes.c_double)), rot_dim, base,
                                           ROTARY_SCALINGS[scaling], factor, trained, low, high))
    return freqs


def _int32_ptr(t: Optional[torch.Tensor], name: str, device: torch.device) -> int:
    if t is None:
        return 0
    if t.dtype is not torch.int32 or t.device != device or t.dim() != 1 or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 vector on the tensors' device")
    return t.data_ptr()


def _heads(t: torch.Tensor, name: str, like: torch.Tensor):
    """Checks one [tokens, heads, head_dim] operand; returns (address, token stride, head stride, heads)."""
    if t.dim() != 3 or t.device != like.device or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor [tokens, heads, head_dim]")
    n, h, d = t.shape
    if t is not like and (t.dtype is not like.dtype or n != like.shape[0] or d != like.shape[2]):
        raise ValueError(f"{name} differs in dtype, tokens or head_dim")
    s0, s1, s2 = t.stride()
    if s2 != 1 and d > 1:
        raise ValueError(f"the last dimension of {name} must be contiguous")
    return t.data_ptr(), s0, s1, h


def gac_rotary(q: torch.Tensor, k: Optional[torch.Tensor], freqs, positions: Optional[torch.Tensor] = None,
               cu_seqlens: Optional[torch.Tensor] = None, layout: str = "half", scale: float = 1.0,
               inverse: bool = False, in_place: bool = False, stream=None):
    """Rotary positions on q (and k, or None), [tokens, heads, head_dim] float32 or bfloat16 views.
    ``freqs``: float64 radians per position (gac_rotary_freqs); it turns the first 2 * len(freqs) elements of
    a head.  Positions are given, or follow from ``cu_seqlens``.  Returns (q', k'): new contiguous tensors, or
    the given ones when ``in_place``."""
    import numpy as np
    dtype, device = q.dtype, q.device
    if dtype not in _DT:
        raise GacError(GAC_ERR_DTYPE, f"unsupported dtype {dtype}")
    qx, q0, q1, qh = _heads(q, "q", q)
    kx = k0 = k1 = kh = 0
    if k is not None:
        kx, k0, k1, kh = _heads(k, "k", q)
    if (positions is None) == (cu_seqlens is None):
        raise ValueError("give positions or cu_seqlens")
    tokens, _, dim = q.shape
    if positions is not None and positions.numel() != tokens:
        raise ValueError("one position per token")
    if cu_seqlens is not None and cu_seqlens.numel() < 1:
        raise ValueError("cu_seqlens has one entry more than there are sequences")
    if not (isinstance(freqs, np.ndarray) and freqs.dtype == np.float64 and freqs.flags.c_contiguous):
        freqs = np.ascontiguousarray(freqs, dtype=np.float64)
    raw, stream = _on(stream, device)
    if in_place:
        yq, yk = q, k
        qy, kout = (qx, q0, q1), (kx, k0, k1)
    else:
        yq = _empty(q, (tokens, qh, dim), stream)
        yk = _empty(q, (tokens, kh, dim), stream) if k is not None else None
        qy = (yq.data_ptr(), qh * dim, dim)
        kout = (yk.data_ptr(), kh * dim, dim) if k is not None else (0, 0, 0)
    args = _ROTARY.pack(qx, qy[0], q0, q1, qy[1], qy[2], kx, kout[0], k0, k1, kout[1], kout[2], qh, kh, tokens,
                        0 if cu_seqlens is None else cu_seqlens.numel() - 1, dim, 2 * freqs.size, _DT[dtype],
                        ROTARY_LAYOUTS[layout], 1 if inverse else 0, 0, _int32_ptr(positions, "positions", device),
                        _int32_ptr(cu_seqlens, "cu_seqlens", device), freqs.__array_interface__["data"][0], scale)
    _check(load_library().gac_rotary(args, device.index, raw))
    if in_place:   # autograd has to notice that what it may have saved has changed
        torch.autograd.graph.increment_version(q if k is None else (q, k))
    return yq, yk


def _attn_args(q, k, v, o, lse, cu_seqlens, scale) -> bytes:
    if q.dtype not in _DT:
        raise GacError(GAC_ERR_DTYPE, f"unsupported dtype {q.dtype}")
    qp, q0, q1, qh = _heads(q, "q", q)
    kp, k0, k1, kh = _heads(k, "k", q)
    vp, v0, v1, vh = _heads(v, "v", q)
    op, o0, o1, oh = _heads(o, "o", q)
    tokens, _, dim = q.shape
    if vh != kh or oh != qh:
        raise ValueError("k and v, and o and q, must have the same shape")
    if lse.dtype is not torch.float32 or lse.device != q.device or lse.shape != (qh, tokens) or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous float32 tensor [q_heads, tokens]")
    n = cu_seqlens.numel()
    if n < 1:
        raise ValueError("cu_seqlens has one entry more than there are sequences")
    return _ATTN.pack(qp, q0, q1, kp, k0, k1, vp, v0, v1, op, o0, o1, lse.data_ptr(),
                      _int32_ptr(cu_seqlens, "cu_seqlens", q.device), tokens, n - 1, qh, kh, dim, _DT[q.dtype],
                      dim ** -0.5 if scale is None else scale, 0)


def gac_attn_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_seqlens: torch.Tensor,
                     scale: Optional[float] = None, stream=None):
    """Causal attention over packed sequences: q [tokens, q_heads, head_dim], k and v [tokens, kv_heads,
    head_dim], bfloat16 views.  Returns (o, lse): o like q, contiguous; lse [q_heads, tokens] float32."""
    if q.dim() != 3 or not q.is_cuda:
        raise ValueError("q must be a CUDA tensor [tokens, heads, head_dim]")
    device = q.device
    raw, stream = _on(stream, device)
    tokens, heads, dim = q.shape
    o = _empty(q, (tokens, heads, dim), stream)
    lse = _empty(q, (heads, tokens), stream, torch.float32)
    _check(load_library().gac_attn_forward(_attn_args(q, k, v, o, lse, cu_seqlens, scale), device.index, raw))
    return o, lse


def gac_attn_backward(d_o: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor,
                      lse: torch.Tensor, cu_seqlens: torch.Tensor, scale: Optional[float] = None, stream=None):
    """Gradients (d_q, d_k, d_v) of gac_attn_forward's o, given d_o; new contiguous tensors."""
    L = load_library()
    args = _attn_args(q, k, v, o, lse, cu_seqlens, scale)
    gp, g0, g1, gh = _heads(d_o, "d_o", q)
    tokens, qh, dim = q.shape
    kh = k.shape[1]
    if gh != qh:
        raise ValueError("d_o must have q's shape")
    device = q.device
    raw, stream = _on(stream, device)
    d_q = _empty(q, (tokens, qh, dim), stream)
    d_k = _empty(q, (tokens, kh, dim), stream)
    d_v = _empty(q, (tokens, kh, dim), stream)
    need = max(L.gac_attn_workspace(args), 16)
    workspace = _empty(q, (need,), stream, torch.uint8)
    grad = _ATTN_GRAD.pack(gp, g0, g1, d_q.data_ptr(), qh * dim, dim, d_k.data_ptr(), kh * dim, dim, d_v.data_ptr(),
                           kh * dim, dim, workspace.data_ptr(), need)
    _check(L.gac_attn_backward(args, grad, device.index, raw))
    return d_q, d_k, d_v


def gac_attn_check(device: Optional[int] = None, stream=None) -> None:
    """Synchronises the stream and raises GacError(GAC_ERR_TIMEOUT) if a wait inside an attention kernel of this device ran
    out since this thread last asked on this stream."""
    dev = torch.device("cuda", torch.cuda.current_device() if device is None else device)
    _check(load_library().gac_attn_check(dev.index, _on(stream, dev)[0]))
