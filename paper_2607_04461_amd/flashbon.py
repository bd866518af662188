"""Python binding of ``libflashbon.so`` (include/flashbon.h, include/flashbon_ops.h).

Argument marshalling only: every step of the draft path runs in the library's HIP kernels.  Device
buffers are anything with ``data_ptr()`` (torch CUDA tensors); ``stream=None`` means torch's current
stream on the current device.  The library must have been built (``__graft_entry__.build()``); a
missing library raises, there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, Optional, Sequence

import numpy as np

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libflashbon.so")
_lib: Optional[ctypes.CDLL] = None

OK, EINVAL, ESHAPE, ENOMEM, EHIP, ESTATE = 0, -1, -2, -3, -4, -5
FP32, BF16 = 0, 1
COMPUTE, SKIP, PROXY = 0, 1, 2
EPI_STORE, EPI_GELU, EPI_STORE_F32, EPI_RESIDUAL = 0, 1, 2, 3
NORM_NONE, NORM_LAYER, NORM_RMS = 0, 1, 2
SITES = ["qkv", "attn_self", "out", "cross_q", "attn_cross", "out_cross", "mlp_up", "mlp_down", "norm",
         "proxy", "embed", "head", "time", "text"]


class FlashbonError(RuntimeError):
    def __init__(self, status: int, where: str, msg: str):
        super().__init__(f"{where} failed with status {status}: {msg}")
        self.status = status


class ModelConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("num_blocks", "hidden", "heads", "mlp_hidden",
                                               "latent_channels", "patch", "freq_dim", "text_dim",
                                               "dtype")] + \
               [("ln_eps", ctypes.c_float)] + \
               [(n, ctypes.c_int32) for n in ("max_n", "max_tokens", "max_text_len", "max_cond", "qk_norm_rope")]


class CacheMeta(ctypes.Structure):
    _fields_ = [("count", ctypes.c_int32), ("head", ctypes.c_int32), ("t", ctypes.c_float * 3)]


class TraceEntry(ctypes.Structure):
    _fields_ = [("action", ctypes.c_int8), ("order", ctypes.c_int8), ("slot", ctypes.c_int8),
                ("live", ctypes.c_int8)]


class StepArgs(ctypes.Structure):
    _fields_ = [
        ("n", ctypes.c_int32), ("latent_h", ctypes.c_int32), ("latent_w", ctypes.c_int32),
        ("latents", ctypes.c_void_p), ("t_cur", ctypes.c_float), ("t_next", ctypes.c_float),
        ("text", ctypes.c_void_p), ("n_cond", ctypes.c_int32), ("text_len", ctypes.c_int32),
        ("cond_index", ctypes.POINTER(ctypes.c_int32)), ("text_kv", ctypes.c_void_p),
        ("text_kv_valid", ctypes.POINTER(ctypes.c_int32)),
        ("skip", ctypes.POINTER(ctypes.c_uint8)), ("proxy", ctypes.POINTER(ctypes.c_uint8)),
        ("cache", ctypes.c_void_p), ("meta", ctypes.POINTER(CacheMeta)),
        ("trace", ctypes.POINTER(TraceEntry)), ("hidden_dump", ctypes.c_void_p),
        ("stream", ctypes.c_void_p),
        ("sde_a", ctypes.c_float), ("sde_step", ctypes.c_int32), ("sde_seed", ctypes.c_uint64),
        ("sde_row0", ctypes.c_int32), ("preview", ctypes.c_void_p),
        ("cfg", ctypes.c_int32), ("cfg_scale", ctypes.c_float), ("uncond_index", ctypes.POINTER(ctypes.c_int32)),
        ("proxy_mode", ctypes.c_int32),
    ]


EXPORTS = [
    "flashbon_weight_count", "flashbon_init_model", "flashbon_text_kv_bytes", "flashbon_cache_bytes",
    "flashbon_draft_step", "flashbon_refine_step", "flashbon_free", "flashbon_plan_step",
    "flashbon_last_error", "flashbon_set_timing", "flashbon_read_timing", "flashbon_op_linear", "flashbon_op_linear_residual", "flashbon_op_linear_plan", "flashbon_op_attention", "flashbon_op_ln_mod",
    "flashbon_op_proxy", "flashbon_op_normals", "flashbon_op_unpatch_sde", "flashbon_select",
    "flashbon_refine_step_noalloc", "flashbon_op_linear_ws",
    "flashbon_op_quant_rows", "flashbon_op_linear_i8", "flashbon_op_norm_residual",
    "flashbon_op_layer_norm", "flashbon_op_layer_norm_grad", "flashbon_op_layer_norm_grad_workspace",
    "flashbon_op_cross_attention", "flashbon_op_cross_attention_workspace", "flashbon_op_cross_attention_grad",
    "flashbon_op_cross_attention_grad_workspace", "flashbon_op_adapters", "flashbon_op_adapters_grad",
    "flashbon_op_adapters_grad_workspace",
]
NOALLOC_SCRATCH_BYTES = 128 << 20

JUDGE_FN = ctypes.CFUNCTYPE(ctypes.c_int32, ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32,
                            ctypes.POINTER(ctypes.c_int32))


def lib_path() -> str:
    return _LIB_PATH


def load() -> ctypes.CDLL:
    """Load the built library (raises FileNotFoundError if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise FileNotFoundError(f"{_LIB_PATH} is not built; run __graft_entry__.build()")
    L = ctypes.CDLL(_LIB_PATH)
    vp, i32, i64, f32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
    L.flashbon_weight_count.argtypes = [ctypes.POINTER(ModelConfig)]
    L.flashbon_weight_count.restype = sz
    L.flashbon_init_model.argtypes = [ctypes.POINTER(ModelConfig), vp, sz, ctypes.POINTER(vp)]
    L.flashbon_init_model.restype = i32
    L.flashbon_text_kv_bytes.argtypes = [vp, i32, i32]
    L.flashbon_text_kv_bytes.restype = sz
    L.flashbon_cache_bytes.argtypes = [vp, i32, i32]
    L.flashbon_cache_bytes.restype = sz
    L.flashbon_draft_step.argtypes = [vp, ctypes.POINTER(StepArgs)]
    L.flashbon_draft_step.restype = i32
    L.flashbon_refine_step.argtypes = [vp, ctypes.POINTER(StepArgs)]
    L.flashbon_refine_step.restype = i32
    L.flashbon_refine_step_noalloc.argtypes = [vp, ctypes.POINTER(StepArgs)]
    L.flashbon_refine_step_noalloc.restype = i32
    L.flashbon_free.argtypes = [vp]
    L.flashbon_free.restype = None
    L.flashbon_plan_step.argtypes = [i32, ctypes.POINTER(ctypes.c_uint8), ctypes.POINTER(ctypes.c_uint8),
                                     ctypes.POINTER(CacheMeta), f32, ctypes.POINTER(TraceEntry), i32]
    L.flashbon_plan_step.restype = i32
    L.flashbon_set_timing.argtypes = [vp, ctypes.c_uint32]
    L.flashbon_set_timing.restype = i32
    L.flashbon_read_timing.argtypes = [vp, i32, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64)]
    L.flashbon_read_timing.restype = i32
    L.flashbon_last_error.argtypes = []
    L.flashbon_last_error.restype = ctypes.c_char_p
    L.flashbon_op_linear.argtypes = [i32, i32, i32, i32, vp, vp, vp, i32, vp, vp, vp, vp]
    L.flashbon_op_linear.restype = i32
    L.flashbon_op_linear_ws.argtypes = [i32, i32, i32, i32, vp, vp, vp, i32, vp, vp, vp, vp, sz,
                                        ctypes.POINTER(ctypes.c_int32), vp]
    L.flashbon_op_linear_ws.restype = i32
    L.flashbon_op_linear_residual.argtypes = [i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp]
    L.flashbon_op_linear_residual.restype = i32
    L.flashbon_op_linear_plan.argtypes = [i32, i32, i32, i32, i32, ctypes.POINTER(ctypes.c_int32), ctypes.c_char_p, i32]
    L.flashbon_op_linear_plan.restype = i32
    L.flashbon_op_attention.argtypes = [i32, i32, i32, i32, i32, i32, vp, i64, i64, vp, vp, i64, i64,
                                        vp, i32, vp, i64, i64, vp]
    L.flashbon_op_attention.restype = i32
    L.flashbon_op_ln_mod.argtypes = [i32, i32, i32, f32, vp, vp, vp, vp, vp]
    L.flashbon_op_ln_mod.restype = i32
    L.flashbon_op_proxy.argtypes = [i64, vp, vp, vp, i32, f32, f32, f32, vp, vp]
    L.flashbon_op_proxy.restype = i32
    L.flashbon_op_normals.argtypes = [i64, i32, i32, ctypes.c_uint64, vp, vp, vp]
    L.flashbon_op_normals.restype = i32
    L.flashbon_op_unpatch_sde.argtypes = [i32, i32, i32, i32, i32, vp, vp, f32, f32, f32, ctypes.c_uint64,
                                          i32, i32, vp]
    L.flashbon_op_unpatch_sde.restype = i32
    L.flashbon_op_quant_rows.argtypes = [i32, i32, i32, vp, i64, vp, vp, vp]
    L.flashbon_op_quant_rows.restype = i32
    L.flashbon_op_linear_i8.argtypes = [i32, i32, i32, i32, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp, vp]
    L.flashbon_op_linear_i8.restype = i32
    L.flashbon_op_norm_residual.argtypes = [i32, i32, i32, f32, vp, f32, vp, i32, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp]
    L.flashbon_op_norm_residual.restype = i32
    L.flashbon_op_layer_norm.argtypes = [i32, i32, i32, f32, vp, i32, vp, i32, vp, vp, vp, vp, vp]
    L.flashbon_op_layer_norm.restype = i32
    L.flashbon_op_layer_norm_grad.argtypes = [i32, i32, i32, vp, i32, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.flashbon_op_layer_norm_grad.restype = i32
    L.flashbon_op_layer_norm_grad_workspace.argtypes = [i32] * 3
    L.flashbon_op_layer_norm_grad_workspace.restype = sz
    cross = [i32] * 7 + [vp, i64, i64, vp, vp, i64, i64, vp, i32, vp, vp, i64, i64, vp]
    L.flashbon_op_cross_attention.argtypes = cross + [vp, sz, vp]
    L.flashbon_op_cross_attention.restype = i32
    L.flashbon_op_cross_attention_workspace.argtypes = [i32] * 7
    L.flashbon_op_cross_attention_workspace.restype = sz
    L.flashbon_op_cross_attention_grad.argtypes = cross + [vp, vp, vp, vp, vp, sz, vp]
    L.flashbon_op_cross_attention_grad.restype = i32
    L.flashbon_op_cross_attention_grad_workspace.argtypes = [i32] * 8
    L.flashbon_op_cross_attention_grad_workspace.restype = sz
    adapters = [i32] * 6 + [vp, vp, vp, vp, vp, i32]
    L.flashbon_op_adapters.argtypes = adapters + [i32, vp, vp, vp, vp, vp]
    L.flashbon_op_adapters.restype = i32
    L.flashbon_op_adapters_grad.argtypes = adapters + [vp, vp, i32, vp, vp, vp, vp, vp, sz, vp]
    L.flashbon_op_adapters_grad.restype = i32
    L.flashbon_op_adapters_grad_workspace.argtypes = [i32] * 7
    L.flashbon_op_adapters_grad_workspace.restype = sz
    L.flashbon_select.argtypes = [i32, ctypes.POINTER(ctypes.c_int32), ctypes.c_double, ctypes.c_double,
                                  ctypes.c_double, JUDGE_FN, vp, ctypes.POINTER(ctypes.c_int32),
                                  ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int32)]
    L.flashbon_select.restype = i32
    _lib = L
    return L


def _check(status: int, where: str) -> None:
    if status != OK:
        raise FlashbonError(status, where, load().flashbon_last_error().decode())


def _ptr(t) -> Optional[int]:
    return None if t is None else int(t.data_ptr())


def _stream(stream) -> Optional[int]:
    if stream is not None:
        return int(stream)
    import torch
    return int(torch.cuda.current_stream().cuda_stream)


def _u8(mask: Optional[Sequence[int]], n: int):
    if mask is None:
        return None, None
    a = np.ascontiguousarray(np.asarray(mask, dtype=np.uint8))
    if a.shape != (n,):
        raise ValueError(f"mask must have shape ({n},)")
    c = _c_array(ctypes.c_uint8, a)
    return c, c


def _c_array(ctype, a: np.ndarray):
    """The values of a contiguous array as a ctypes array, which pointer arguments and fields take as it is
    (ndarray.ctypes.data_as costs several times as much, on every step)."""
    return (ctype * a.size).from_buffer_copy(a)


def make_config(shape, dtype: int, max_n: int, max_tokens: int, max_text_len: int, max_cond: int) -> ModelConfig:
    return ModelConfig(shape.num_blocks, shape.hidden, shape.heads, shape.mlp_hidden,
                       shape.latent_channels, shape.patch, shape.freq_dim, shape.text_dim, dtype,
                       shape.ln_eps, max_n, max_tokens, max_text_len, max_cond,
                       1 if getattr(shape, "qk_norm_rope", False) else 0)


def flashbon_weight_count(cfg: ModelConfig) -> int:
    return int(load().flashbon_weight_count(ctypes.byref(cfg)))


# Shape of every live model handle, so that the step wrappers can check the caller's tensors before
# their addresses cross the C ABI (which cannot see sizes, dtypes or devices).
_MODELS: Dict[int, ModelConfig] = {}


def flashbon_init_model(cfg: ModelConfig, host_weights: np.ndarray) -> int:
    w = np.ascontiguousarray(host_weights, dtype=np.float32)
    h = ctypes.c_void_p()
    _check(load().flashbon_init_model(ctypes.byref(cfg), w.ctypes.data, w.size, ctypes.byref(h)),
           "flashbon_init_model")
    kept = ModelConfig()
    ctypes.pointer(kept)[0] = cfg
    _MODELS[int(h.value)] = kept
    return int(h.value)


def flashbon_free(model: Optional[int]) -> None:
    if model:
        _MODELS.pop(int(model), None)
        load().flashbon_free(model)


def model_config(model: int) -> ModelConfig:
    """The configuration a live handle was created with (ValueError for an unknown handle)."""
    try:
        return _MODELS[int(model)]
    except (KeyError, TypeError):
        raise ValueError("not a live model handle from flashbon_init_model") from None


def text_kv_nbytes(cfg: ModelConfig, n_cond: int, text_len: int) -> int:
    """flashbon_text_kv_bytes for a configuration: [L][n_cond][text_len][2 D] act elements."""
    return cfg.num_blocks * n_cond * text_len * 2 * cfg.hidden * (2 if cfg.dtype == BF16 else 4)


def cache_nbytes(cfg: ModelConfig, rows: int, tokens: int) -> int:
    """flashbon_cache_bytes for a configuration: fp32 [L][3][rows][tokens][D]."""
    return cfg.num_blocks * 3 * rows * tokens * cfg.hidden * 4


def _nbytes(t) -> int:
    return int(t.numel()) * int(t.element_size())


def _check_tensor(name: str, t, *, dtype=None, ndim=None, require_device: bool = True, device: Optional[int] = None) -> None:
    """``device``: the current device's index, where the caller has it."""
    import torch
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} must be a torch tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if ndim is not None and t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dimensions, got shape {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if require_device:
        if not t.is_cuda:
            raise ValueError(f"{name} must be on the current device (a GPU), got {t.device}")
        if device is None:
            device = torch.cuda.current_device()
        if t.device.index != device:
            raise ValueError(f"{name} must be on the current device (cuda:{device}), got {t.device}")


def validate_step(cfg: ModelConfig, latents, text, text_kv, *, draft: bool, guided: bool = False,
                  cache=None, hidden_dump=None, preview=None, meta=None, trace=None,
                  require_device: bool = True) -> None:
    """Raise ValueError unless every buffer a step would hand to the library has the dtype, layout,
    device and size the step's kernels read and write (include/flashbon.h, flashbon_step_args).
    ``require_device=False`` skips only the device check (host-only tests of the other checks)."""
    import torch
    f32 = torch.float32
    device = torch.cuda.current_device() if require_device and isinstance(latents, torch.Tensor) and latents.is_cuda else None
    _check_tensor("latents", latents, dtype=f32, ndim=4, require_device=require_device, device=device)
    n, C, H, W = (int(x) for x in latents.shape)
    if C != cfg.latent_channels:
        raise ValueError(f"latents have {C} channels, the model {cfg.latent_channels}")
    _check_tensor("text", text, dtype=f32, ndim=3, require_device=require_device, device=device)
    n_cond, text_len, text_dim = (int(x) for x in text.shape)
    if text_dim != cfg.text_dim:
        raise ValueError(f"text tokens are {text_dim} wide, the model takes {cfg.text_dim}")
    _check_tensor("text_kv", text_kv, require_device=require_device, device=device)
    need = text_kv_nbytes(cfg, n_cond, text_len)
    if _nbytes(text_kv) < need:
        raise ValueError(f"text_kv holds {_nbytes(text_kv)} bytes, needs {need}")
    rows = 2 * n if guided else n
    p = max(cfg.patch, 1)
    tokens = (H // p) * (W // p)
    if draft:
        if cache is None:
            raise ValueError("a draft step needs the activation cache")
        _check_tensor("cache", cache, dtype=f32, require_device=require_device, device=device)
        need = cache_nbytes(cfg, rows, tokens)
        if _nbytes(cache) < need:
            raise ValueError(f"cache holds {_nbytes(cache)} bytes, needs {need} for {rows} rows x {tokens} tokens")
        if meta is None or len(meta) != cfg.num_blocks:
            raise ValueError(f"meta must hold {cfg.num_blocks} entries")
    if trace is not None and len(trace) != cfg.num_blocks:
        raise ValueError(f"trace must hold {cfg.num_blocks} entries")
    if hidden_dump is not None:
        _check_tensor("hidden_dump", hidden_dump, dtype=f32, require_device=require_device, device=device)
        need = (cfg.num_blocks + 1) * rows * tokens * cfg.hidden
        if int(hidden_dump.numel()) < need:
            raise ValueError(f"hidden_dump holds {int(hidden_dump.numel())} floats, needs {need}")
    if preview is not None:
        _check_tensor("preview", preview, dtype=f32, ndim=4, require_device=require_device, device=device)
        if tuple(preview.shape) != tuple(latents.shape):
            raise ValueError(f"preview must have the latents' shape {tuple(latents.shape)}")
        a0, a1 = latents.data_ptr(), latents.data_ptr() + _nbytes(latents)
        b0, b1 = preview.data_ptr(), preview.data_ptr() + _nbytes(preview)
        if a0 < b1 and b0 < a1:
            raise ValueError("preview must not overlap latents")


def flashbon_text_kv_bytes(model: int, n_cond: int, text_len: int) -> int:
    return int(load().flashbon_text_kv_bytes(model, n_cond, text_len))


def flashbon_cache_bytes(model: int, n: int, tokens: int) -> int:
    return int(load().flashbon_cache_bytes(model, n, tokens))


def new_meta(num_blocks: int):
    return (CacheMeta * num_blocks)()


def new_trace(num_blocks: int):
    return (TraceEntry * num_blocks)()


def trace_list(trace) -> list:
    return [(e.action, e.order, e.slot, e.live) for e in trace]


def _step(fn, where, model, latents, t_cur, t_next, text, cond_index, text_kv, text_kv_valid,
          skip=None, proxy=None, cache=None, meta=None, trace=None, hidden_dump=None, stream=None,
          num_blocks=None, sde=None, preview=None, cfg=None, proxy_mode=0, draft=True):
    validate_step(model_config(model), latents, text, text_kv, draft=draft, guided=cfg is not None,
                  cache=cache, hidden_dump=hidden_dump, preview=preview, meta=meta, trace=trace)
    a = step_args(latents, t_cur, t_next, text, cond_index, text_kv, text_kv_valid, skip, proxy, cache,
                  meta, trace, hidden_dump, stream, num_blocks, sde, preview, cfg, proxy_mode)
    _check(fn(model, ctypes.byref(a)), where)


def step_args(latents, t_cur, t_next, text, cond_index, text_kv, text_kv_valid, skip=None, proxy=None,
              cache=None, meta=None, trace=None, hidden_dump=None, stream=None, num_blocks=None, sde=None,
              preview=None, cfg=None, proxy_mode=0) -> StepArgs:
    """flashbon_step_args for the given buffers, without any check (the library validates the rest;
    tests of the library's own validation build arguments with this).  The host arrays it points to
    are kept alive on the returned structure."""
    n, C, H, W = (int(x) for x in latents.shape)
    n_cond, text_len = int(text.shape[0]), int(text.shape[1])
    cond = np.ascontiguousarray(np.asarray(cond_index, dtype=np.int32))
    if cond.shape != (n,):
        raise ValueError(f"cond_index must have shape ({n},)")
    L = num_blocks if num_blocks is not None else (len(meta) if meta is not None else None)
    sk, skp = _u8(skip, L) if skip is not None else (None, None)
    px, pxp = _u8(proxy, L) if proxy is not None else (None, None)
    a = StepArgs()
    a.n, a.latent_h, a.latent_w = n, H, W
    a.latents = _ptr(latents)
    a.t_cur, a.t_next = float(t_cur), float(t_next)
    a.text = _ptr(text)
    a.n_cond, a.text_len = n_cond, text_len
    cond = a.cond_index = _c_array(ctypes.c_int32, cond)
    a.text_kv = _ptr(text_kv)
    a.text_kv_valid = ctypes.pointer(text_kv_valid)
    a.skip, a.proxy = skp, pxp
    a.cache = _ptr(cache)
    a.meta = meta
    a.trace = trace
    a.hidden_dump = _ptr(hidden_dump)
    a.preview = _ptr(preview)
    a.proxy_mode = int(proxy_mode)
    if cfg is not None:
        unc = np.ascontiguousarray(np.asarray(cfg[1], dtype=np.int32))
        if unc.shape != (n,):
            raise ValueError(f"uncond_index must have shape ({n},)")
        a.cfg, a.cfg_scale = 1, float(cfg[0])
        unc = a.uncond_index = _c_array(ctypes.c_int32, unc)
    a.stream = _stream(stream)
    if sde is not None:
        a.sde_a, a.sde_seed, a.sde_step = float(sde[0]), int(sde[1]), int(sde[2])
        a.sde_row0 = int(sde[3]) if len(sde) > 3 else 0
    a._keep = (cond, sk, px, unc if cfg is not None else None, text_kv_valid)
    return a


def flashbon_draft_step(model, latents, t_cur, t_next, text, cond_index, text_kv, text_kv_valid,
                        skip, proxy, cache, meta, trace=None, hidden_dump=None, stream=None, sde=None,
                        preview=None, cfg=None, proxy_mode=0):
    """One draft step; ``text_kv_valid`` is a ctypes.c_int32, ``meta``/``trace`` ctypes arrays;
    ``sde = (a, seed, step[, row0])`` selects the stochastic update (None or a = 0: Euler);
    ``preview`` (device [n, C, H, W] fp32) receives z - t_cur v; ``cfg = (scale, uncond_index)``
    turns on classifier-free guidance (the cache then holds 2n rows); ``proxy_mode`` 1 takes the
    residual-delta reading of the proxy."""
    _step(load().flashbon_draft_step, "flashbon_draft_step", model, latents, t_cur, t_next, text,
          cond_index, text_kv, text_kv_valid, skip, proxy, cache, meta, trace, hidden_dump, stream,
          num_blocks=len(meta), sde=sde, preview=preview, cfg=cfg, proxy_mode=proxy_mode)


def flashbon_refine_step(model, latents, t_cur, t_next, text, cond_index, text_kv, text_kv_valid,
                         trace=None, hidden_dump=None, stream=None, sde=None, preview=None, cfg=None):
    _step(load().flashbon_refine_step, "flashbon_refine_step", model, latents, t_cur, t_next, text,
          cond_index, text_kv, text_kv_valid, None, None, None, None, trace, hidden_dump, stream, sde=sde,
          preview=preview, cfg=cfg, draft=False)


def flashbon_refine_step_noalloc(model, latents, t_cur, t_next, text, cond_index, text_kv, text_kv_valid,
                                 trace=None, hidden_dump=None, stream=None, sde=None, preview=None, cfg=None):
    """flashbon_refine_step with its working buffers in the library's static per-GPU scratch array
    (allocates nothing; overlapping calls on one GPU race)."""
    _step(load().flashbon_refine_step_noalloc, "flashbon_refine_step_noalloc", model, latents, t_cur, t_next,
          text, cond_index, text_kv, text_kv_valid, None, None, None, None, trace, hidden_dump, stream, sde=sde,
          preview=preview, cfg=cfg, draft=False)


def flashbon_select(scores, judge, rho1=0.5, rho2=0.5, kappa=1.5):
    """Multi-stage Elo selection; ``judge(a, b) -> (winner, confidence)`` is the verifier.
    Returns (winner, ratings [m] float64, pairwise calls)."""
    sc = np.ascontiguousarray(np.asarray(scores, dtype=np.int32))
    m = int(sc.size)
    failure = []

    def _cb(_ctx, a, b, conf):
        try:
            w, c = judge(int(a), int(b))
            conf[0] = int(c)
            return int(w)
        except BaseException as e:  # the exception cannot cross the C frame; report it afterwards
            failure.append(e)
            return -1

    cb = JUDGE_FN(_cb)
    winner, calls = ctypes.c_int32(), ctypes.c_int32()
    ratings = np.zeros(m, np.float64)
    st = load().flashbon_select(m, sc.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), rho1, rho2, kappa, cb,
                                None, ctypes.byref(winner),
                                ratings.ctypes.data_as(ctypes.POINTER(ctypes.c_double)), ctypes.byref(calls))
    if failure:
        raise failure[0]
    _check(st, "flashbon_select")
    return int(winner.value), ratings, int(calls.value)


def flashbon_plan_step(skip, proxy, meta, t_cur: float, trace=None, proxy_mode: int = 0):
    L = len(meta)
    sk, skp = _u8(skip, L)
    px, pxp = _u8(proxy, L)
    if trace is None:
        trace = new_trace(L)
    _check(load().flashbon_plan_step(L, skp, pxp, meta, float(t_cur), trace, int(proxy_mode)),
           "flashbon_plan_step")
    return trace


def flashbon_set_timing(model: int, sites) -> None:
    """Time the named launch sites (see SITES) on later steps; empty = off."""
    mask = 0
    for name in sites:
        mask |= 1 << SITES.index(name)
    _check(load().flashbon_set_timing(model, mask), "flashbon_set_timing")


def flashbon_read_timing(model: int, site: str):
    """(total device ms, launches) of one site since the last read."""
    ms, n = ctypes.c_double(), ctypes.c_int64()
    _check(load().flashbon_read_timing(model, SITES.index(site), ctypes.byref(ms), ctypes.byref(n)),
           "flashbon_read_timing")
    return ms.value, n.value


# --------------------------------------------------------------------------- kernel-level entry points

def flashbon_op_linear(dtype, M, N, K, A, W, bias, epilogue, out, gate=None, cache_out=None, stream=None):
    _check(load().flashbon_op_linear(dtype, M, N, K, _ptr(A), _ptr(W), _ptr(bias), epilogue, _ptr(out),
                                     _ptr(gate), _ptr(cache_out), _stream(stream)), "flashbon_op_linear")


def flashbon_op_linear_ws(dtype, M, N, K, A, W, bias, epilogue, out, workspace, gate=None, cache_out=None,
                          stream=None) -> int:
    """flashbon_op_linear with a split-K workspace (a device tensor); returns the number of K ranges."""
    sp = ctypes.c_int32()
    nbytes = 0 if workspace is None else int(workspace.numel()) * int(workspace.element_size())
    _check(load().flashbon_op_linear_ws(dtype, M, N, K, _ptr(A), _ptr(W), _ptr(bias), epilogue, _ptr(out),
                                        _ptr(gate), _ptr(cache_out), _ptr(workspace), nbytes, ctypes.byref(sp),
                                        _stream(stream)), "flashbon_op_linear_ws")
    return sp.value


def flashbon_op_linear_residual(dtype, M, N, K, A, W, bias, gate, residual_in, out, stream=None):
    _check(load().flashbon_op_linear_residual(dtype, M, N, K, _ptr(A), _ptr(W), _ptr(bias), _ptr(gate),
                                              _ptr(residual_in), _ptr(out), _stream(stream)),
           "flashbon_op_linear_residual")


def flashbon_op_linear_plan(dtype, M, N, K, epilogue):
    """(number of kernel launches, description) of the tile plan flashbon_op_linear takes."""
    n = ctypes.c_int32()
    buf = ctypes.create_string_buffer(256)
    _check(load().flashbon_op_linear_plan(dtype, M, N, K, epilogue, ctypes.byref(n), buf, len(buf)),
           "flashbon_op_linear_plan")
    return n.value, buf.value.decode()


def flashbon_op_attention(dtype, batch, heads, head_dim, tq, tk, q, q_bs, q_rs, k, v, kv_bs, kv_rs,
                          kv_index, n_kv, out, o_bs, o_rs, stream=None):
    _check(load().flashbon_op_attention(dtype, batch, heads, head_dim, tq, tk, _ptr(q), q_bs, q_rs, _ptr(k),
                                        _ptr(v), kv_bs, kv_rs, _ptr(kv_index), n_kv, _ptr(out), o_bs, o_rs,
                                        _stream(stream)), "flashbon_op_attention")


def flashbon_op_ln_mod(dtype, M, D, eps, x, shift, scale, out, stream=None):
    _check(load().flashbon_op_ln_mod(dtype, M, D, eps, _ptr(x), _ptr(shift), _ptr(scale), _ptr(out),
                                     _stream(stream)), "flashbon_op_ln_mod")


def flashbon_op_proxy(count, h1, h2, h3, order, tau1, tau2, t_cur, out, stream=None):
    _check(load().flashbon_op_proxy(count, _ptr(h1), _ptr(h2), _ptr(h3), order, tau1, tau2, t_cur, _ptr(out),
                                    _stream(stream)), "flashbon_op_proxy")


def flashbon_op_normals(count, candidate, step, seed, words=None, normals=None, stream=None):
    _check(load().flashbon_op_normals(count, candidate, step, seed, _ptr(words), _ptr(normals),
                                      _stream(stream)), "flashbon_op_normals")


def flashbon_op_unpatch_sde(n, C, H, W, p, v, z, t_cur, t_next, a, seed, step, row0=0, stream=None):
    _check(load().flashbon_op_unpatch_sde(n, C, H, W, p, _ptr(v), _ptr(z), t_cur, t_next, a, seed, step, row0,
                                          _stream(stream)), "flashbon_op_unpatch_sde")


# 8-bit layers.  Sizes are given, as in the calls above; every tensor is checked against them.

_torch = None


def _with_torch():
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


def _act(dtype):
    torch = _with_torch()
    if dtype not in (FP32, BF16):
        raise ValueError("dtype must be FP32 or BF16")
    return torch.bfloat16 if dtype == BF16 else torch.float32


def _current_device(require_device: bool) -> Optional[int]:
    return _with_torch().cuda.current_device() if require_device else None


def _raw_stream(stream, device: int) -> int:
    """``_stream`` on ``device``, the current one: torch's call for the address alone, which is no public one, takes a tenth
    of the time of a Stream object; without it the public one."""
    raw = getattr(_torch._C, "_cuda_getCurrentRawStream", None) if stream is None else None
    return raw(device) if raw is not None else _stream(stream)


def _int32(*sizes) -> None:
    """Refuses integers that the ABI's 32 bits would wrap."""
    if max(sizes) > 0x7FFFFFFF or min(sizes) < -0x80000000:
        raise ValueError(f"integers must be below 2^31 in magnitude, got {sizes}")


def _pointers(device: Optional[int], *wanted) -> list:
    """Addresses of the tensors in ``wanted``, (name, tensor or None, dtype, elements, required) each: of that dtype,
    contiguous, of at least so many elements, on the GPU ``device`` (None: anywhere)."""
    found = []
    for name, t, dtype, count, required in wanted:
        if t is None:
            if required:
                raise ValueError(f"{name} is required")
            found.append(None)
            continue
        if t.dtype is not dtype:
            raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        if t.numel() < count:
            raise ValueError(f"{name} holds {t.numel()} elements, needs {count}")
        if device is not None and t.get_device() != device:
            raise ValueError(f"{name} must be on the current device (cuda:{device}), got {t.device}")
        found.append(t.data_ptr())
    return found


def validate_quant_rows(dtype, M, K, x, x_row_stride, q, scale, *, require_device: bool = True) -> list:
    """Raise ValueError unless the tensors are what flashbon_op_quant_rows reads and writes; their addresses.  ``x`` may
    be a view of wider rows: 2-D with a unit column stride."""
    act, device = _act(dtype), _current_device(require_device)
    _int32(M, K)
    if M < 1 or K < 1 or x_row_stride < K:
        raise ValueError(f"need M, K >= 1 and a row stride of at least K, got {M}, {K}, {x_row_stride}")
    if x is None:
        raise ValueError("x is required")
    if x.dtype is not act:
        raise ValueError(f"x must be {act}, got {x.dtype}")
    if x.is_contiguous():
        if x.numel() < (M - 1) * x_row_stride + K:
            raise ValueError(f"x holds {x.numel()} elements, {M} rows of {K} at stride {x_row_stride} need more")
    elif x.dim() != 2 or x.stride(1) != 1 or x.stride(0) != x_row_stride or x.shape[0] < M or x.shape[1] < K:
        raise ValueError(f"x must be contiguous or [{M}, {K}] with strides ({x_row_stride}, 1), got "
                         f"{tuple(x.shape)} with {x.stride()}")
    if device is not None and x.get_device() != device:
        raise ValueError(f"x must be on the current device (cuda:{device}), got {x.device}")
    return [x.data_ptr()] + _pointers(device, ("q", q, _torch.int8, M * K, True), ("scale", scale, _torch.float32, M, True))


def flashbon_op_quant_rows(dtype, M, K, x, q, scale, x_row_stride=None, stream=None):
    """Rows x [M][K] to int8 codes q and one scale a row; ``x_row_stride`` in elements (None: a matrix's own, else K)."""
    if x_row_stride is None:
        x_row_stride = int(x.stride(0)) if x is not None and x.dim() == 2 and x.shape[0] > 1 else K
    px, pq, ps = validate_quant_rows(dtype, M, K, x, x_row_stride, q, scale)
    _check(load().flashbon_op_quant_rows(dtype, M, K, px, x_row_stride, pq, ps, _raw_stream(stream, x.get_device())),
           "flashbon_op_quant_rows")


def validate_linear_i8(dtype, M, N, K, A, a_scale, W, w_scale, bias, epilogue, out, gate=None, residual_in=None,
                       cache_out=None, *, require_device: bool = True) -> list:
    """Raise ValueError unless the tensors are what flashbon_op_linear_i8 reads and writes; their addresses."""
    act, device = _act(dtype), _current_device(require_device)
    i8, f32 = _torch.int8, _torch.float32
    _int32(M, N, K, epilogue)
    found = _pointers(device, ("A", A, i8, M * K, True), ("a_scale", a_scale, f32, M, True), ("W", W, i8, N * K, True),
                      ("w_scale", w_scale, f32, N, True), ("bias", bias, f32, N, False),
                      ("out", out, act if epilogue == EPI_STORE or epilogue == EPI_GELU else f32, M * N, True))
    if epilogue == EPI_RESIDUAL:
        return found + _pointers(device, ("gate", gate, f32, N, False), ("residual_in", residual_in, f32, M * N, False),
                                 ("cache_out", cache_out, f32, M * N, False))
    return found + [None, None, None]


def flashbon_op_linear_i8(dtype, M, N, K, A, a_scale, W, w_scale, bias, epilogue, out, gate=None, residual_in=None,
                          cache_out=None, stream=None):
    """Linear layer on int8 rows A [M][K] and weights W [N][K] with a scale a token and an output channel."""
    pa, psa, pw, psw, pb, po, pg, pr, pc = validate_linear_i8(dtype, M, N, K, A, a_scale, W, w_scale, bias, epilogue, out,
                                                              gate, residual_in, cache_out)
    _check(load().flashbon_op_linear_i8(dtype, M, N, K, pa, psa, pw, psw, pb, epilogue, po, pg, pr, pc,
                                        _raw_stream(stream, A.get_device())), "flashbon_op_linear_i8")


def validate_norm_residual(dtype, M, D, x, y=None, out=None, q=None, q_scale=None, x_out=None, post_gain=None, gate=None,
                           shift=None, scale=None, *, require_device: bool = True) -> list:
    """Raise ValueError unless the tensors are what flashbon_op_norm_residual reads and writes; their addresses."""
    act, device = _act(dtype), _current_device(require_device)
    f32 = _torch.float32
    _int32(M, D)
    return _pointers(device, ("x", x, f32, M * D, True), ("y", y, act, M * D, False), ("post_gain", post_gain, f32, D, False),
                     ("gate", gate, f32, D, False), ("x_out", x_out, f32, M * D, False), ("shift", shift, f32, D, False),
                     ("scale", scale, f32, D, False), ("out", out, act, M * D, False), ("q", q, _torch.int8, M * D, False),
                     ("q_scale", q_scale, f32, M, False))


def flashbon_op_norm_residual(dtype, M, D, eps, x, y=None, *, alpha=1.0, post_norm=NORM_NONE, post_gain=None, gate=None,
                              x_out=None, pre_norm=NORM_LAYER, shift=None, scale=None, out=None, q=None, q_scale=None,
                              stream=None):
    """h = alpha x + gate (post_norm(y) post_gain) -> x_out; pre_norm(h) (1 + scale) + shift -> out, or q and q_scale."""
    px, py, pp, pg, ph, psh, psc, po, pq, pqs = validate_norm_residual(dtype, M, D, x, y, out, q, q_scale, x_out, post_gain,
                                                                       gate, shift, scale)
    _check(load().flashbon_op_norm_residual(dtype, M, D, eps, px, alpha, py, post_norm, pp, pg, ph, pre_norm, psh, psc, po,
                                            pq, pqs, _raw_stream(stream, x.get_device())), "flashbon_op_norm_residual")


# The cross-attention branch with a prompt and an adapter per candidate, and its gradients.  Tensors are checked as above;
# a workspace is a tensor of any type, of as many bytes as the ``_workspace`` function of the same sizes says.

def _workspace_pointer(device: Optional[int], workspace) -> tuple:
    """Address and bytes of a workspace (None: none)."""
    if workspace is None:
        return None, 0
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    if device is not None and workspace.get_device() != device:
        raise ValueError(f"workspace must be on the current device (cuda:{device}), got {workspace.device}")
    return workspace.data_ptr(), _nbytes(workspace)


def _rows_of_heads(device: Optional[int], *wanted) -> list:
    """Addresses of the tensors in ``wanted``, (name, tensor or None, dtype, batches, batch stride, rows, row stride, width,
    required) each, strides in elements: views whose memory holds all of that."""
    found = []
    for name, t, dtype, n, batch_stride, rows, row_stride, width, required in wanted:
        if t is None:
            if required:
                raise ValueError(f"{name} is required")
            found.append(None)
            continue
        if t.dtype is not dtype:
            raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
        if not (0 <= batch_stride < 1 << 36 and 0 <= row_stride < 1 << 36):
            raise ValueError(f"strides of {name} must be in [0, 2^36), got {batch_stride} and {row_stride}")
        need = (n - 1) * batch_stride + (rows - 1) * row_stride + width
        if t.numel() < need or not t.is_contiguous():      # a view of wider rows: what its memory holds from its first element on
            held = t.untyped_storage().nbytes() // t.element_size() - t.storage_offset()
            if held < need:
                raise ValueError(f"{name} holds {held} elements from its first on, needs {need}")
        if device is not None and t.get_device() != device:
            raise ValueError(f"{name} must be on the current device (cuda:{device}), got {t.device}")
        found.append(t.data_ptr())
    return found


def _groups(rows: int, rows_per_group: int) -> int:
    if rows_per_group < 1:
        raise ValueError(f"rows_per_group must be at least 1, got {rows_per_group}")
    return -(-rows // rows_per_group)


def validate_layer_norm(dtype, M, D, x, out, weight=None, bias=None, rows_per_group=1, mean=None, rstd=None, *,
                        require_device: bool = True) -> list:
    """Raise ValueError unless the tensors are what flashbon_op_layer_norm reads and writes; their addresses."""
    act, device = _act(dtype), _current_device(require_device)
    f32 = _torch.float32
    _int32(M, D, rows_per_group)
    vectors = _groups(M, rows_per_group) * D
    return _pointers(device, ("x", x, f32, M * D, True), ("weight", weight, f32, vectors, False),
                     ("bias", bias, f32, vectors, False), ("out", out, act, M * D, True), ("mean", mean, f32, M, False),
                     ("rstd", rstd, f32, M, False))


def flashbon_op_layer_norm(dtype, M, D, eps, x, out, *, weight=None, bias=None, rows_per_group=None, modulated=False,
                           mean=None, rstd=None, stream=None):
    """LayerNorm of x [M][D] times weight (``modulated``: 1 + weight) plus bias, a vector for each ``rows_per_group`` rows
    (None: one for all); ``mean`` and ``rstd`` [M] for the gradient."""
    per = max(int(M), 1) if rows_per_group is None else rows_per_group
    px, pw, pb, po, pm, pr = validate_layer_norm(dtype, M, D, x, out, weight, bias, per, mean, rstd)
    _check(load().flashbon_op_layer_norm(dtype, M, D, eps, px, per, pw, int(bool(modulated)), pb, po, pm, pr,
                                         _raw_stream(stream, x.get_device())), "flashbon_op_layer_norm")


def flashbon_op_layer_norm_grad_workspace(M, D, rows_per_group=None) -> int:
    """Bytes of the workspace flashbon_op_layer_norm_grad needs."""
    per = max(int(M), 1) if rows_per_group is None else rows_per_group
    _int32(M, D, per)
    return int(load().flashbon_op_layer_norm_grad_workspace(M, D, per))


def validate_layer_norm_grad(dtype, M, D, x, mean, rstd, dy, dx=None, weight=None, rows_per_group=1, residual=None,
                             dweight=None, dbias=None, workspace=None, *, require_device: bool = True) -> list:
    """Raise ValueError unless the tensors are what flashbon_op_layer_norm_grad reads and writes; their addresses."""
    act, device = _act(dtype), _current_device(require_device)
    f32 = _torch.float32
    _int32(M, D, rows_per_group)
    vectors = _groups(M, rows_per_group) * D
    return _pointers(device, ("x", x, f32, M * D, True), ("weight", weight, f32, vectors, False), ("mean", mean, f32, M, True),
                     ("rstd", rstd, f32, M, True), ("dy", dy, act, M * D, True), ("residual", residual, f32, M * D, False),
                     ("dx", dx, f32, M * D, False), ("dweight", dweight, f32, vectors, False),
                     ("dbias", dbias, f32, vectors, False)) + list(_workspace_pointer(device, workspace))


def flashbon_op_layer_norm_grad(dtype, M, D, x, mean, rstd, dy, dx=None, *, weight=None, rows_per_group=None, modulated=False,
                                residual=None, dweight=None, dbias=None, workspace=None, stream=None):
    """dx = residual + the gradient of x, and dweight and dbias, from dy and the saved statistics."""
    per = max(int(M), 1) if rows_per_group is None else rows_per_group
    px, pw, pm, pr, py, pres, pdx, pdw, pdb, ws, nbytes = validate_layer_norm_grad(
        dtype, M, D, x, mean, rstd, dy, dx, weight, per, residual, dweight, dbias, workspace)
    _check(load().flashbon_op_layer_norm_grad(dtype, M, D, px, per, pw, int(bool(modulated)), pm, pr, py, pres, pdx, pdw, pdb,
                                              ws, nbytes, _raw_stream(stream, x.get_device())), "flashbon_op_layer_norm_grad")


def _cross_tensors(dtype, batch, heads, kv_heads, head_dim, tq, tk, n_kv, device, rows, vectors) -> list:
    sizes = (batch, heads, kv_heads, head_dim, tq, tk, n_kv)
    if min(sizes) < 1 or max(sizes) > 0x7FFFFFFF:
        raise ValueError(f"batch, heads, kv_heads, head_dim, tq, tk and n_kv must be at least 1 and below 2^31, got {sizes}")
    return _rows_of_heads(device, *rows) + _pointers(device, *vectors)


def validate_cross_attention(dtype, batch, heads, kv_heads, head_dim, tq, tk, q, q_bs, q_rs, k, v, kv_bs, kv_rs, kv_index, n_kv,
                             kv_len, out, o_bs, o_rs, lse=None, workspace=None, *, require_device: bool = True) -> list:
    """Raise ValueError unless the tensors are what flashbon_op_cross_attention reads and writes; their addresses."""
    act, device = _act(dtype), _current_device(require_device)
    wide, narrow, i32 = heads * head_dim, kv_heads * head_dim, _torch.int32
    return _cross_tensors(
        dtype, batch, heads, kv_heads, head_dim, tq, tk, n_kv, device,
        (("q", q, act, batch, q_bs, tq, q_rs, wide, True), ("k", k, act, n_kv, kv_bs, tk, kv_rs, narrow, True),
         ("v", v, act, n_kv, kv_bs, tk, kv_rs, narrow, True), ("out", out, act, batch, o_bs, tq, o_rs, wide, True)),
        (("kv_index", kv_index, i32, batch, False), ("kv_len", kv_len, i32, n_kv, False),
         ("lse", lse, _torch.float32, batch * heads * tq, False))) + list(_workspace_pointer(device, workspace))


def flashbon_op_cross_attention(dtype, batch, heads, kv_heads, head_dim, tq, tk, q, q_bs, q_rs, k, v, kv_bs, kv_rs, kv_index,
                                n_kv, kv_len, out, o_bs, o_rs, *, lse=None, workspace=None, stream=None):
    """Attention of each batch row to the first kv_len of its prompt's tk keys; ``lse`` [batch][heads][tq] for the gradient."""
    pq, pk, pv, po, pi, pn, pl, ws, nbytes = validate_cross_attention(
        dtype, batch, heads, kv_heads, head_dim, tq, tk, q, q_bs, q_rs, k, v, kv_bs, kv_rs, kv_index, n_kv, kv_len, out, o_bs,
        o_rs, lse, workspace)
    _check(load().flashbon_op_cross_attention(dtype, batch, heads, kv_heads, head_dim, tq, tk, pq, q_bs, q_rs, pk, pv, kv_bs,
                                              kv_rs, pi, n_kv, pn, po, o_bs, o_rs, pl, ws, nbytes,
                                              _raw_stream(stream, q.get_device())), "flashbon_op_cross_attention")


def flashbon_op_cross_attention_workspace(dtype, batch, heads, kv_heads, head_dim, tq, tk) -> int:
    """Bytes of the workspace with which flashbon_op_cross_attention cuts long keys into ranges."""
    _int32(batch, heads, kv_heads, head_dim, tq, tk)
    return int(load().flashbon_op_cross_attention_workspace(dtype, batch, heads, kv_heads, head_dim, tq, tk))


def validate_cross_attention_grad(dtype, batch, heads, kv_heads, head_dim, tq, tk, q, q_bs, q_rs, k, v, kv_bs, kv_rs, kv_index,
                                  n_kv, kv_len, out, o_bs, o_rs, lse, dout, dq=None, dk=None, dv=None, workspace=None, *,
                                  require_device: bool = True) -> list:
    """Raise ValueError unless the tensors are what flashbon_op_cross_attention_grad reads and writes; their addresses."""
    act, device = _act(dtype), _current_device(require_device)
    wide, narrow, i32 = heads * head_dim, kv_heads * head_dim, _torch.int32
    return _cross_tensors(
        dtype, batch, heads, kv_heads, head_dim, tq, tk, n_kv, device,
        (("q", q, act, batch, q_bs, tq, q_rs, wide, True), ("k", k, act, n_kv, kv_bs, tk, kv_rs, narrow, True),
         ("v", v, act, n_kv, kv_bs, tk, kv_rs, narrow, True), ("out", out, act, batch, o_bs, tq, o_rs, wide, True),
         ("dout", dout, act, batch, o_bs, tq, o_rs, wide, True), ("dq", dq, act, batch, q_bs, tq, q_rs, wide, False),
         ("dk", dk, act, n_kv, kv_bs, tk, kv_rs, narrow, False), ("dv", dv, act, n_kv, kv_bs, tk, kv_rs, narrow, False)),
        (("kv_index", kv_index, i32, batch, False), ("kv_len", kv_len, i32, n_kv, False),
         ("lse", lse, _torch.float32, batch * heads * tq, True))) + list(_workspace_pointer(device, workspace))


def flashbon_op_cross_attention_grad(dtype, batch, heads, kv_heads, head_dim, tq, tk, q, q_bs, q_rs, k, v, kv_bs, kv_rs,
                                     kv_index, n_kv, kv_len, out, o_bs, o_rs, lse, dout, dq=None, dk=None, dv=None, *,
                                     workspace=None, stream=None):
    """dq (q's strides), dk and dv (k's) from dout (out's), out and lse; dq, or dk and dv, may be None."""
    pq, pk, pv, po, pdo, pdq, pdk, pdv, pi, pn, pl, ws, nbytes = validate_cross_attention_grad(
        dtype, batch, heads, kv_heads, head_dim, tq, tk, q, q_bs, q_rs, k, v, kv_bs, kv_rs, kv_index, n_kv, kv_len, out, o_bs,
        o_rs, lse, dout, dq, dk, dv, workspace)
    _check(load().flashbon_op_cross_attention_grad(dtype, batch, heads, kv_heads, head_dim, tq, tk, pq, q_bs, q_rs, pk, pv,
                                                   kv_bs, kv_rs, pi, n_kv, pn, po, o_bs, o_rs, pl, pdo, pdq, pdk, pdv, ws,
                                                   nbytes, _raw_stream(stream, q.get_device())),
           "flashbon_op_cross_attention_grad")


def flashbon_op_cross_attention_grad_workspace(dtype, batch, heads, kv_heads, head_dim, tq, tk, n_kv) -> int:
    """Bytes of the workspace flashbon_op_cross_attention_grad needs."""
    _int32(batch, heads, kv_heads, head_dim, tq, tk, n_kv)
    return int(load().flashbon_op_cross_attention_grad_workspace(dtype, batch, heads, kv_heads, head_dim, tq, tk, n_kv))


def validate_adapters(dtype, M, N, K, rank, n_adapters, x, down, up, scales, index, rows_per_group, epilogue, base, out, u,
                      gate=None, *, require_device: bool = True) -> list:
    """Raise ValueError unless the tensors are what flashbon_op_adapters reads and writes; their addresses."""
    act, device = _act(dtype), _current_device(require_device)
    f32 = _torch.float32
    _int32(M, N, K, rank, n_adapters, rows_per_group, epilogue)
    groups, outs = _groups(M, rows_per_group), act if epilogue == EPI_STORE else f32
    return _pointers(device, ("x", x, act, M * K, True), ("down", down, act, n_adapters * rank * K, True),
                     ("up", up, act, n_adapters * N * rank, True), ("scales", scales, f32, n_adapters, False),
                     ("index", index, _torch.int32, groups, False),
                     ("gate", gate if epilogue == EPI_RESIDUAL else None, f32, N, False), ("base", base, outs, M * N, False),
                     ("out", out, outs, M * N, True), ("u", u, f32, M * rank, True))


def flashbon_op_adapters(dtype, M, N, K, rank, n_adapters, x, down, up, scales, index, rows_per_group, epilogue, base, out, u,
                         *, gate=None, stream=None):
    """out = base + gate scales[a] (x down[a]^T) up[a]^T, a = index of each ``rows_per_group`` rows; u = x down^T (fp32)."""
    px, pd, pu, ps, pi, pg, pb, po, pmid = validate_adapters(dtype, M, N, K, rank, n_adapters, x, down, up, scales, index,
                                                             rows_per_group, epilogue, base, out, u, gate)
    _check(load().flashbon_op_adapters(dtype, M, N, K, rank, n_adapters, px, pd, pu, ps, pi, rows_per_group, epilogue, pg, pb,
                                       po, pmid, _raw_stream(stream, x.get_device())), "flashbon_op_adapters")


def flashbon_op_adapters_grad_workspace(dtype, M, N, K, rank, n_adapters, rows_per_group) -> int:
    """Bytes of the workspace flashbon_op_adapters_grad needs."""
    _int32(M, N, K, rank, n_adapters, rows_per_group)
    return int(load().flashbon_op_adapters_grad_workspace(dtype, M, N, K, rank, n_adapters, rows_per_group))


def validate_adapters_grad(dtype, M, N, K, rank, n_adapters, x, down, up, scales, index, rows_per_group, u, dy, epilogue, base,
                           dx=None, d_down=None, d_up=None, workspace=None, *, require_device: bool = True) -> list:
    """Raise ValueError unless the tensors are what flashbon_op_adapters_grad reads and writes; their addresses."""
    act, device = _act(dtype), _current_device(require_device)
    f32 = _torch.float32
    _int32(M, N, K, rank, n_adapters, rows_per_group, epilogue)
    groups, outs = _groups(M, rows_per_group), act if epilogue == EPI_STORE else f32
    downs, ups = n_adapters * rank * K, n_adapters * N * rank
    return _pointers(device, ("x", x, act, M * K, True), ("down", down, act, downs, True), ("up", up, act, ups, True),
                     ("scales", scales, f32, n_adapters, False), ("index", index, _torch.int32, groups, False),
                     ("u", u, f32, M * rank, True), ("dy", dy, act, M * N, True), ("base", base, outs, M * K, False),
                     ("dx", dx, outs, M * K, False), ("d_down", d_down, f32, downs, False),
                     ("d_up", d_up, f32, ups, False)) + list(_workspace_pointer(device, workspace))


def flashbon_op_adapters_grad(dtype, M, N, K, rank, n_adapters, x, down, up, scales, index, rows_per_group, u, dy, epilogue,
                              base, dx=None, d_down=None, d_up=None, *, workspace=None, stream=None):
    """dx = base + the adapters' gradient of x, d_down and d_up (fp32), from dy and u."""
    px, pd, pu, ps, pi, pmid, py, pb, pdx, pdd, pdu, ws, nbytes = validate_adapters_grad(
        dtype, M, N, K, rank, n_adapters, x, down, up, scales, index, rows_per_group, u, dy, epilogue, base, dx, d_down, d_up,
        workspace)
    _check(load().flashbon_op_adapters_grad(dtype, M, N, K, rank, n_adapters, px, pd, pu, ps, pi, rows_per_group, pmid, py,
                                            epilogue, pb, pdx, pdd, pdu, ws, nbytes, _raw_stream(stream, x.get_device())),
           "flashbon_op_adapters_grad")
