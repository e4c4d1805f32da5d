"""ctypes binding of the FreqFormer C ABI (include/freqformer.h).

Argument marshalling only: every step of the path runs inside the CUDA library.  PyTorch is
used for device memory and streams.  There is no CPU fallback: if the library has not been
built (``python -m paper_2604_22808_b200.build``) loading it raises.
"""
from __future__ import annotations

import ctypes as C
import os
from array import array
from typing import Optional, Sequence

import numpy as np

from .configs import CrossAttentionConfig, FFConfig, FFNConfig, LayerNormConfig, RotaryConfig

# FF_LIBRARY_VARIANT=debug loads the build with device-side range checks (python -m paper_2604_22808_b200.build --debug),
# =clocks the one with cycle sums (--clocks)
_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), {
    "debug": "libfreqformer_debug.so", "clocks": "libfreqformer_clocks.so"}.get(os.environ.get("FF_LIBRARY_VARIANT"), "libfreqformer.so"))
_lib = None

FF_OK = 0
STATUS_NAMES = {0: "FF_OK", 1: "FF_ERR_INVALID_ARG", 2: "FF_ERR_UNSUPPORTED", 3: "FF_ERR_WORKSPACE",
                4: "FF_ERR_CUDA", 5: "FF_ERR_TIMEOUT", 6: "FF_ERR_EMPTY_BAND", 7: "FF_ERR_NOT_ROUTED"}
FF_BF16, FF_FP32 = 0, 1
FF_BAND_LOW, FF_BAND_MID, FF_BAND_HIGH = 1, 2, 4
(TAP_SPEC_LOW, TAP_SPEC_MID, TAP_SPEC_HIGH, TAP_POOLED_LOW, TAP_Y_LOW, TAP_Y_MID, TAP_Y_HIGH, TAP_SUMMARY,
 TAP_ENERGY, TAP_ALLOC, TAP_PI) = range(11)

EXPORTS = ("ff_config_validate", "ff_band_sizes", "ff_band_rank", "ff_workspace_bytes", "ff_workspace_bytes_host",
           "ff_plan_create", "ff_plan_workspace_bytes", "ff_band_info", "ff_plan_set_workspace", "ff_destroy", "ff_last_error",
           "ff_route", "ff_forward", "ff_forward_host", "ff_forward_projected", "ff_plan_device_status", "ff_plan_last_launches", "ff_plan_kernel_info",
           "ff_get_tap", "ff_plan_set_attention_impl", "ff_plan_set_profiling", "ff_plan_stage_times", "ff_high_attention_noalloc",
           "ff_plan_selftest_bounded_wait", "ff_rotary_create", "ff_rotary_destroy", "ff_rotary_last_error", "ff_rotary_frequencies",
           "ff_rotary_apply", "ff_qk_norm", "ff_qk_norm_backward", "ff_qk_norm_workspace_bytes", "ff_forward_projected_rotary", "ff_ffn_validate",
           "ff_ffn_workspace_bytes", "ff_ffn_create", "ff_ffn_destroy", "ff_ffn_last_error", "ff_ffn_forward", "ff_ffn_backward",
           "ff_ffn_device_status", "ff_layer_norm_create", "ff_layer_norm_destroy", "ff_layer_norm_last_error", "ff_layer_norm_forward",
           "ff_layer_norm_backward", "ff_layer_norm_workspace_bytes", "ff_cross_attention_validate", "ff_cross_attention_workspace_bytes",
           "ff_cross_attention_create", "ff_cross_attention_destroy", "ff_cross_attention_last_error", "ff_cross_attention_forward",
           "ff_cross_attention_backward", "ff_cross_attention_device_status")
STAGES = ("transform", "router", "attention", "summary", "inverse")


class ff_config_t(C.Structure):
    _fields_ = [("batch", C.c_int32), ("T", C.c_int32), ("H", C.c_int32), ("W", C.c_int32), ("heads", C.c_int32),
                ("head_dim", C.c_int32), ("dtype", C.c_int32), ("low_cut", C.c_int32 * 3), ("mid_cut", C.c_int32 * 3),
                ("low_compress", C.c_int32), ("mid_block", C.c_int32), ("mid_stride", C.c_int32),
                ("high_radius", C.c_int32), ("n_summary", C.c_int32), ("router_hidden", C.c_int32),
                ("t_embed_dim", C.c_int32), ("transform", C.c_int32), ("mid_pattern", C.c_int32)]


class ff_weights_t(C.Structure):
    _fields_ = [("W1", C.c_void_p), ("b1", C.c_void_p), ("W2", C.c_void_p), ("b2", C.c_void_p), ("U", C.c_void_p)]


class ff_rotary_config_t(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("rot_dim", C.c_int32), ("dtype", C.c_int32), ("layout", C.c_int32), ("scaling", C.c_int32),
                ("axis_pairs", C.c_int32 * 3), ("grid", C.c_int32 * 3), ("original_length", C.c_int32), ("base", C.c_double),
                ("factor", C.c_double)]


class ff_ffn_config_t(C.Structure):
    _fields_ = [("dim", C.c_int32), ("hidden", C.c_int32), ("activation", C.c_int32)]


class ff_layer_norm_config_t(C.Structure):
    _fields_ = [("dim", C.c_int32), ("dtype", C.c_int32), ("unit_offset", C.c_int32), ("eps", C.c_float)]


class ff_cross_attention_config_t(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("heads", C.c_int32), ("kv_heads", C.c_int32), ("scale", C.c_float)]


class ff_rows_t(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride_batch", C.c_int64), ("stride_token", C.c_int64)]


class ff_heads_t(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride_batch", C.c_int64), ("stride_head", C.c_int64), ("stride_token", C.c_int64),
                ("heads", C.c_int32)]


class FFError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


def library() -> C.CDLL:
    """Load the CUDA library; fails loudly when it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise FFError(4, f"{_LIB_PATH} is missing: build it with `python -m paper_2604_22808_b200.build` "
                             "(there is no CPU fallback)")
        lib = C.CDLL(_LIB_PATH)
        lib.ff_last_error.restype = C.c_char_p
        lib.ff_last_error.argtypes = [C.c_void_p]
        for name in ("ff_rotary_last_error", "ff_ffn_last_error", "ff_layer_norm_last_error", "ff_cross_attention_last_error"):
            getattr(lib, name).restype = C.c_char_p
            getattr(lib, name).argtypes = [C.c_void_p]
        for name in EXPORTS:
            if not name.endswith("last_error"):
                getattr(lib, name).restype = C.c_int32
        lib.ff_plan_create.argtypes = [C.POINTER(ff_config_t), C.POINTER(ff_weights_t), C.POINTER(C.c_void_p)]
        lib.ff_plan_workspace_bytes.argtypes = [C.c_void_p, C.POINTER(C.c_size_t)]
        lib.ff_plan_set_workspace.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t]
        lib.ff_band_info.argtypes = [C.c_void_p, C.POINTER(C.c_int64)]
        lib.ff_destroy.argtypes = [C.c_void_p]
        lib.ff_route.argtypes = [C.c_void_p] + [C.c_void_p] * 3 + [C.c_void_p] * 4 + [C.c_void_p]
        lib.ff_forward.argtypes = [C.c_void_p] + [C.c_void_p] * 3 + [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        lib.ff_forward_host.argtypes = [C.c_void_p] + [C.c_void_p] * 3 + [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        lib.ff_forward_projected.argtypes = [C.c_void_p] + [C.c_void_p] * 3 + [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        lib.ff_plan_device_status.argtypes = [C.c_void_p, C.c_void_p]
        lib.ff_plan_last_launches.argtypes = [C.c_void_p, C.POINTER(C.c_int64)]
        lib.ff_plan_kernel_info.argtypes = [C.c_void_p, C.POINTER(C.c_int32)]
        lib.ff_get_tap.argtypes = [C.c_void_p, C.c_int32, C.POINTER(C.c_void_p), C.POINTER(C.c_size_t)]
        lib.ff_plan_set_attention_impl.argtypes = [C.c_void_p, C.c_int32]
        lib.ff_plan_set_profiling.argtypes = [C.c_void_p, C.c_int32]
        lib.ff_plan_stage_times.argtypes = [C.c_void_p, C.POINTER(C.c_float), C.POINTER(C.c_int64)]
        lib.ff_high_attention_noalloc.argtypes = [C.c_void_p] * 4 + [C.c_int32, C.c_int64, C.c_int32, C.c_int32, C.c_void_p]
        lib.ff_plan_selftest_bounded_wait.argtypes = [C.c_void_p, C.c_int64, C.POINTER(C.c_int32), C.c_void_p]
        heads, place = C.c_void_p, [C.c_void_p, C.c_int64, C.c_int64, C.c_void_p, C.c_int64]
        lib.ff_rotary_create.argtypes = [C.POINTER(ff_rotary_config_t), C.POINTER(C.c_void_p)]
        lib.ff_rotary_destroy.argtypes = [C.c_void_p]
        lib.ff_rotary_frequencies.argtypes = [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_double)]
        lib.ff_rotary_apply.argtypes = place + [heads, heads, C.c_int32, heads, heads, C.c_void_p]
        lib.ff_qk_norm.argtypes = place + [heads, heads, C.c_void_p, C.c_void_p, C.c_float, heads, heads, C.c_void_p]
        lib.ff_qk_norm_backward.argtypes = (place + [heads, heads, C.c_void_p, C.c_void_p, C.c_float] + [heads] * 4
                                            + [C.c_void_p] * 3 + [C.c_size_t, C.c_void_p])
        lib.ff_forward_projected_rotary.argtypes = ([C.c_void_p] * 6 + [C.c_int64, C.c_void_p, C.c_void_p, C.c_float] + [C.c_void_p] * 4)
        lib.ff_qk_norm_workspace_bytes.argtypes = [C.c_void_p, C.POINTER(C.c_size_t)]
        lib.ff_ffn_validate.argtypes = [C.POINTER(ff_ffn_config_t)]
        lib.ff_ffn_workspace_bytes.argtypes = [C.POINTER(ff_ffn_config_t), C.c_int64, C.c_int32, C.POINTER(C.c_size_t)]
        lib.ff_ffn_create.argtypes = [C.POINTER(ff_ffn_config_t), C.POINTER(C.c_void_p)]
        lib.ff_ffn_destroy.argtypes = [C.c_void_p]
        lib.ff_ffn_forward.argtypes = [C.c_void_p, C.c_int64] + [C.c_void_p] * 8 + [C.c_size_t, C.c_void_p]
        lib.ff_ffn_backward.argtypes = [C.c_void_p, C.c_int64] + [C.c_void_p] * 12 + [C.c_size_t, C.c_void_p]
        lib.ff_ffn_device_status.argtypes = [C.c_void_p, C.c_void_p]
        lib.ff_layer_norm_create.argtypes = [C.POINTER(ff_layer_norm_config_t), C.POINTER(C.c_void_p)]
        lib.ff_layer_norm_destroy.argtypes = [C.c_void_p]
        lib.ff_layer_norm_workspace_bytes.argtypes = [C.c_void_p, C.c_int64, C.c_int64, C.c_int32, C.POINTER(C.c_size_t)]
        lib.ff_layer_norm_forward.argtypes = [C.c_void_p, C.c_int64, C.c_int64] + [C.c_void_p] * 3 + [C.c_int32, C.c_void_p, C.c_void_p]
        lib.ff_layer_norm_backward.argtypes = ([C.c_void_p, C.c_int64, C.c_int64, C.c_void_p, C.c_void_p, C.c_int32] + [C.c_void_p] * 5
                                               + [C.c_size_t, C.c_void_p])
        lib.ff_cross_attention_validate.argtypes = [C.POINTER(ff_cross_attention_config_t)]
        lib.ff_cross_attention_workspace_bytes.argtypes = ([C.POINTER(ff_cross_attention_config_t)] + [C.c_int64] * 3
                                                           + [C.c_int32, C.POINTER(C.c_size_t)])
        lib.ff_cross_attention_create.argtypes = [C.POINTER(ff_cross_attention_config_t), C.POINTER(C.c_void_p)]
        lib.ff_cross_attention_destroy.argtypes = [C.c_void_p]
        lib.ff_cross_attention_forward.argtypes = [C.c_void_p] + [C.c_int64] * 3 + [C.c_void_p] * 8 + [C.c_size_t, C.c_void_p]
        lib.ff_cross_attention_backward.argtypes = [C.c_void_p] + [C.c_int64] * 3 + [C.c_void_p] * 12 + [C.c_size_t, C.c_void_p]
        lib.ff_cross_attention_device_status.argtypes = [C.c_void_p, C.c_void_p]
        lib.ff_config_validate.argtypes = [C.POINTER(ff_config_t)]
        lib.ff_band_sizes.argtypes = [C.POINTER(ff_config_t), C.POINTER(C.c_int64)]
        lib.ff_band_rank.argtypes = [C.POINTER(ff_config_t), C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_int32),
                                     C.POINTER(C.c_int64)]
        lib.ff_workspace_bytes.argtypes = [C.POINTER(ff_config_t), C.POINTER(C.c_size_t)]
        lib.ff_workspace_bytes_host.argtypes = [C.POINTER(ff_config_t), C.POINTER(C.c_size_t)]
        _lib = lib
    return _lib


def c_config(cfg: FFConfig) -> ff_config_t:
    c = ff_config_t()
    c.batch, c.T, c.H, c.W, c.heads, c.head_dim = cfg.batch, cfg.T, cfg.H, cfg.W, cfg.heads, cfg.head_dim
    c.dtype = FF_FP32 if cfg.dtype == "fp32" else FF_BF16
    c.low_cut = (C.c_int32 * 3)(*cfg.low_cut)
    c.mid_cut = (C.c_int32 * 3)(*cfg.mid_cut)
    c.low_compress, c.mid_block, c.mid_stride, c.high_radius = cfg.r, cfg.b, cfg.s, cfg.R
    c.n_summary, c.router_hidden, c.t_embed_dim = cfg.m, cfg.router_hidden, cfg.t_embed_dim
    c.transform = {"dct": 0, "haar": 1}[cfg.transform]
    c.mid_pattern = {"strided": 0, "anchor": 1}[cfg.mid_pattern]
    return c


def _check(status: int, plan=None):
    if status != FF_OK:
        raise FFError(status, library().ff_last_error(plan).decode())


# ---- host-only helpers ------------------------------------------------------------------------
def ff_config_validate(cfg: FFConfig) -> int:
    return library().ff_config_validate(C.byref(c_config(cfg)))


def ff_band_sizes(cfg: FFConfig):
    out = (C.c_int64 * 4)()
    _check(library().ff_band_sizes(C.byref(c_config(cfg)), out))
    return tuple(int(x) for x in out)


def ff_band_rank(cfg: FFConfig, kt: int, kh: int, kw: int):
    band, rank = C.c_int32(), C.c_int64()
    _check(library().ff_band_rank(C.byref(c_config(cfg)), kt, kh, kw, C.byref(band), C.byref(rank)))
    return band.value, rank.value


def ff_workspace_bytes(cfg: FFConfig, host_staging: bool = False) -> int:
    out = C.c_size_t()
    fn = library().ff_workspace_bytes_host if host_staging else library().ff_workspace_bytes
    _check(fn(C.byref(c_config(cfg)), C.byref(out)))
    return out.value


# ---- the plan -----------------------------------------------------------------------------------
def _f32(a) -> Optional[np.ndarray]:
    return None if a is None else np.ascontiguousarray(a, dtype=np.float32)


def _floats(values, count: int):
    """A host float array for a call that reads `count` of them: a sequence of numbers, or one number (None stays None)."""
    if values is None:
        return None
    if isinstance(values, np.ndarray):
        values = values.ravel()
    try:
        out = (C.c_float * len(values))(*values)
    except TypeError:                                    # a number, a nested sequence
        flat = np.ascontiguousarray(values, dtype=np.float32).ravel()
        out = (C.c_float * flat.size)(*flat)
    if len(out) < count:
        raise FFError(1, f"expected {count} timesteps (one per sample), got {len(out)}")
    return out


def _ptr(a: Optional[np.ndarray]):
    return None if a is None else a.ctypes.data_as(C.c_void_p)


def _stream_getter(torch):
    """Device index -> handle of the current stream.  A Stream object per call takes 1.3 us, the handle alone 0.07; torch
    has a private name for that, which another version may lack."""
    return getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


class Plan:
    """Owns an ff_plan_t and (through torch) its workspace."""

    def __init__(self, cfg: FFConfig, weights: Optional[dict] = None, U: Optional[np.ndarray] = None,
                 host_staging: bool = False, device: str = "cuda:0"):
        import torch
        self.cfg = cfg
        self._torch = torch
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.handle = C.c_void_p()
        lib = library()
        w = ff_weights_t()
        keep = []
        if weights is not None:
            for name in ("W1", "b1", "W2", "b2"):
                arr = _f32(weights[name]); keep.append(arr)
                setattr(w, name, arr.ctypes.data)
        if U is not None:
            arr = _f32(U); keep.append(arr)
            w.U = arr.ctypes.data
        with torch.cuda.device(self.device):
            _check(lib.ff_plan_create(C.byref(c_config(cfg)), C.byref(w), C.byref(self.handle)))
            nbytes = ff_workspace_bytes(cfg, host_staging)
            self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            _check(lib.ff_plan_set_workspace(self.handle, self.workspace.data_ptr(), nbytes), self.handle)
        self.workspace_bytes = nbytes
        self._shape = torch.Size((cfg.batch, cfg.heads, cfg.T, cfg.H, cfg.W, cfg.head_dim))
        self._dtype = torch.float32 if cfg.dtype == "fp32" else torch.bfloat16
        self._raw_stream = _stream_getter(torch)

    # -- lifetime
    def destroy(self):
        if self.handle:
            library().ff_destroy(self.handle)
            self.handle = C.c_void_p()
            self.workspace = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def band_info(self):
        """(N_low, ceil(N_low / r), N_mid, N_high) of the plan's configuration."""
        out = (C.c_int64 * 4)()
        _check(library().ff_band_info(self.handle, out), self.handle)
        return tuple(int(x) for x in out)

    def _stream(self):
        return self._raw_stream(self.device.index)

    @property
    def torch_dtype(self):
        return self._dtype

    def _check_io(self, *tensors):
        shape, dtype, device = self._shape, self._dtype, self.device
        for t in tensors:
            if t.shape != shape or t.dtype != dtype or not t.is_contiguous():
                raise FFError(1, f"expected a contiguous {dtype} tensor of shape {tuple(shape)}")
            if t.device != device:
                raise FFError(1, f"expected a tensor on {self.device}, got one on {t.device}")

    def _check_masks(self, masks):
        """The device pointer of a tensor of batch * heads band masks, one byte each (None stays None)."""
        if masks is None:
            return None
        n = self.cfg.batch * self.cfg.heads
        if masks.element_size() != 1 or masks.numel() < n or not masks.is_contiguous() or masks.device != self.device:
            raise FFError(1, f"expected a contiguous uint8 tensor of {n} band masks on {self.device}")
        return masks.data_ptr()

    def _check_host(self, *tensors):
        n = self._shape.numel() * self._dtype.itemsize
        for t in tensors:
            if t.numel() * t.element_size() < n or not t.is_contiguous():
                raise FFError(1, f"expected a contiguous {self._dtype} tensor of shape {tuple(self._shape)}")

    # -- the path
    def route(self, Q, K, V, timesteps: Sequence[float], alloc_out=None, want_host: bool = True):
        self._check_io(Q, K, V)
        ts = _floats(timesteps, self.cfg.batch)
        assert len(ts) == self.cfg.batch
        alloc_h = np.zeros(self.cfg.batch * self.cfg.heads, np.uint8) if want_host else None
        pi_h = np.zeros((self.cfg.batch, 3), np.float32) if want_host else None
        _check(library().ff_route(self.handle, Q.data_ptr(), K.data_ptr(), V.data_ptr(), ts,
                                  self._check_masks(alloc_out), _ptr(alloc_h), _ptr(pi_h),
                                  self._stream()), self.handle)
        return alloc_h, pi_h

    def forward(self, Q, K, V, out, alloc=None, timesteps: Optional[Sequence[float]] = None):
        """alloc: uint8 CUDA tensor [batch*heads] of band masks, or None to route from timesteps."""
        self._check_io(Q, K, V, out)
        ts = _floats(timesteps, self.cfg.batch)
        _check(library().ff_forward(self.handle, Q.data_ptr(), K.data_ptr(), V.data_ptr(), self._check_masks(alloc), ts,
                                    out.data_ptr(), self._stream()), self.handle)
        return out

    def forward_host(self, Qh, Kh, Vh, out_h, alloc_host: Optional[np.ndarray] = None,
                     timesteps: Optional[Sequence[float]] = None):
        """Host tensors (ideally pinned) in and out; the copies are part of the call."""
        self._check_host(Qh, Kh, Vh, out_h)
        ts = _floats(timesteps, self.cfg.batch)
        al = None if alloc_host is None else np.ascontiguousarray(alloc_host, dtype=np.uint8)
        if al is not None and al.size < self.cfg.batch * self.cfg.heads:
            raise FFError(1, f"expected {self.cfg.batch * self.cfg.heads} band masks, got {al.size}")
        _check(library().ff_forward_host(self.handle, Qh.data_ptr(), Kh.data_ptr(), Vh.data_ptr(), _ptr(al), ts,
                                         out_h.data_ptr(), self._stream()), self.handle)
        return out_h

    def forward_projected(self, X, Wqkv, Wo, out, alloc=None, timesteps: Optional[Sequence[float]] = None,
                          rotary: Optional["Rotary"] = None, wq=None, wk=None, eps: float = 0.0, positions=None):
        """X, out: bf16 CUDA tensors [batch][T*H*W][heads*head_dim]; Wqkv [3][D][D], Wo [D][D] (y = x W).
        The plan must have been created with host_staging=True (Q, K, V and the attention output live there).
        rotary: Q and K are turned before the attention, and with eps > 0 normed first (times wq, wk: fp32 [head_dim] or None);
        positions as for Rotary, None: the plan's grid, or the token's index."""
        torch = self._torch
        cfg = self.cfg
        D = cfg.heads * cfg.head_dim
        for t, shape in ((X, (cfg.batch, cfg.N, D)), (out, (cfg.batch, cfg.N, D)), (Wqkv, (3, D, D)), (Wo, (D, D))):
            if (tuple(t.shape) != shape or t.dtype != torch.bfloat16 or not t.is_contiguous() or not t.is_cuda
                    or t.device != self.device):
                raise FFError(1, f"expected a contiguous bf16 tensor of shape {shape} on {self.device}")
        ts = _floats(timesteps, self.cfg.batch)
        if rotary is not None:
            if eps and C.c_float(eps).value == 0:
                raise FFError(1, "eps is 0 in fp32, which means no norm")
            w, (pos, stride) = [rotary._weight(t, self.device) for t in (wq, wk)], rotary._positions(positions, cfg.batch, cfg.N, self.device)
            _check(library().ff_forward_projected_rotary(self.handle, X.data_ptr(), Wqkv.data_ptr(), Wo.data_ptr(), rotary.handle, pos, stride,
                                                         *w, eps, self._check_masks(alloc), ts, out.data_ptr(), self._stream()), self.handle)
            return out
        if wq is not None or wk is not None or eps or positions is not None:
            raise FFError(1, "norm weights, eps and positions belong to a rotary handle")
        _check(library().ff_forward_projected(self.handle, X.data_ptr(), Wqkv.data_ptr(), Wo.data_ptr(),
                                              self._check_masks(alloc), ts, out.data_ptr(), self._stream()), self.handle)
        return out

    def device_status(self) -> int:
        return library().ff_plan_device_status(self.handle, self._stream())

    def selftest_bounded_wait(self, limit_cycles: int) -> int:
        """Runs the bounded-wait self-test; returns how many of its two waits were abandoned."""
        n = C.c_int32(-1)
        _check(library().ff_plan_selftest_bounded_wait(self.handle, int(limit_cycles), C.byref(n), self._stream()), self.handle)
        return n.value

    def kernel_info(self) -> dict:
        info = (C.c_int32 * 4)()
        _check(library().ff_plan_kernel_info(self.handle, info), self.handle)
        return {"transform_fused": bool(info[0] & 1), "forward_axis_in_registers": bool(info[0] & 2),
                "inverse_t_in_registers": bool(info[1]), "attention_tensor_core": bool(info[2]), "low_band_tensor_core": bool(info[3])}

    def last_launches(self) -> int:
        n = C.c_int64()
        _check(library().ff_plan_last_launches(self.handle, C.byref(n)), self.handle)
        return n.value

    def set_attention_impl(self, impl: int):
        _check(library().ff_plan_set_attention_impl(self.handle, impl), self.handle)

    def set_profiling(self, enable: bool):
        _check(library().ff_plan_set_profiling(self.handle, int(enable)), self.handle)

    def stage_times(self):
        """{stage: (ms, launches)} of the last forward (profiling must be enabled)."""
        ms, n = (C.c_float * len(STAGES))(), (C.c_int64 * len(STAGES))()
        _check(library().ff_plan_stage_times(self.handle, ms, n), self.handle)
        return {name: (float(ms[i]), int(n[i])) for i, name in enumerate(STAGES)}

    # -- inspection
    def tap(self, which: int):
        """A torch view (no copy) of an intermediate buffer inside the workspace."""
        torch = self._torch
        ptr, nbytes = C.c_void_p(), C.c_size_t()
        _check(library().ff_get_tap(self.handle, which, C.byref(ptr), C.byref(nbytes)), self.handle)
        off = ptr.value - self.workspace.data_ptr()
        raw = self.workspace[off:off + nbytes.value]
        cfg = self.cfg
        n_low, n_bar, n_mid, n_high = ff_band_sizes(cfg)
        BH, d = cfg.batch * cfg.heads, cfg.head_dim
        st = self.torch_dtype
        shapes = {TAP_SPEC_LOW: (torch.float32, (3, BH, n_low, d)), TAP_SPEC_MID: (st, (3, BH, n_mid, d)),
                  TAP_SPEC_HIGH: (st, (3, BH, n_high, d)), TAP_POOLED_LOW: (torch.float32, (3, BH, n_bar, d)),
                  TAP_Y_LOW: (torch.float32, (BH, n_bar, d)), TAP_Y_MID: (st, (BH, n_mid, d)),
                  TAP_Y_HIGH: (st, (BH, n_high, d)), TAP_SUMMARY: (torch.float32, (BH, 3, cfg.m, d)),
                  TAP_ENERGY: (torch.float64, (cfg.batch, 3, d)), TAP_ALLOC: (torch.uint8, (BH,)),
                  TAP_PI: (torch.float32, (cfg.batch, 3))}
        dt, shape = shapes[which]
        return raw.view(dt).view(shape)


# ---- queries and keys between the projections and the attention ---------------------------------------
class Rotary:
    """Rotary positions of queries and keys, alone or with the norm of every head row in the same pass.

    q, k and the tensors written are CUDA tensors [batch][heads][tokens][head_dim] of the configuration's type, with
    contiguous channels and any strides for the rest (a transposed view of [batch][tokens][heads][head_dim] is one; for
    interleaved pairs addresses and strides have to be multiples of two elements); q and k may have different numbers of heads,
    and k and its output may be None.  An output may be its own input.  positions: an int32 CUDA tensor [tokens] or
    [batch][tokens], with a last dimension of 3 (t, h, w) where the configuration divides the pairs over axes; None: the token's
    index, or its cell in the configuration's grid."""

    def __init__(self, cfg: RotaryConfig):
        import torch
        self.cfg = cfg
        self._torch = torch
        self.handle = C.c_void_p()
        c = ff_rotary_config_t()
        c.head_dim, c.rot_dim, c.original_length = cfg.head_dim, cfg.rot_dim, cfg.original_length
        c.base, c.factor = cfg.base, cfg.factor
        try:
            c.dtype = {"bf16": FF_BF16, "fp32": FF_FP32}[cfg.dtype]
            c.layout = {"half": 0, "interleaved": 1}[cfg.layout]
            c.scaling = {"none": 0, "linear": 1, "ntk": 2, "by_parts": 3}[cfg.scaling]
        except KeyError as e:
            raise FFError(1, f"unknown dtype, layout or scaling: {e}") from None
        c.axis_pairs = (C.c_int32 * 3)(*cfg.axis_pairs)
        c.grid = (C.c_int32 * 3)(*cfg.grid)
        _check(library().ff_rotary_create(C.byref(c), C.byref(self.handle)))
        self._dtype = torch.float32 if cfg.dtype == "fp32" else torch.bfloat16
        self._axes = 3 if any(cfg.axis_pairs) else 1
        self._int32, self._float32, self._channels, self._lib = torch.int32, torch.float32, torch.Size((cfg.head_dim,)), library()
        self._raw_stream = _stream_getter(torch)
        n = C.c_size_t()
        _check(library().ff_qk_norm_workspace_bytes(self.handle, C.byref(n)))
        self.workspace_bytes = n.value

    def destroy(self):
        if self.handle:
            library().ff_rotary_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def frequencies(self):
        """(radians per position of every pair, magnitude of the rotation)"""
        theta, m = (C.c_double * (self.cfg.rot_dim // 2))(), C.c_double()
        self._status(library().ff_rotary_frequencies(self.handle, theta, C.byref(m)))
        return np.array(theta), m.value

    def _status(self, status: int):
        if status != FF_OK:
            raise FFError(status, library().ff_rotary_last_error(self.handle).decode())

    def _arguments(self, positions, q, k, *others):
        """Checks the tensors of a call, `others` q- and k-like in turns: the arguments (batch, tokens, positions, stride between the
        samples' positions), the addresses of the tensors' ff_heads_t (None for None), and the array that holds those."""
        dtype, device, qs = self._dtype, q.device, q.shape
        if len(qs) != 4 or qs[3] != self.cfg.head_dim or not q.is_cuda or q.dtype != dtype:
            raise FFError(1, f"expected q a {dtype} tensor [batch][heads][tokens][{self.cfg.head_dim}] on a GPU")
        B, Hq, N, d = qs
        sb, sh, st, sc = q.stride()
        rows, at, contiguous = [q.data_ptr(), sb, sh, st, Hq], [0], sc == 1      # (the layout of ff_heads_t, heads in its low half word)
        if k is None:
            ks, Hk = None, 0
            at.append(None)
        else:
            ks = k.shape
            if len(ks) != 4 or ks[0] != B or ks[2] != N or ks[3] != d or k.dtype != dtype or k.device != device:
                raise FFError(1, f"expected k a {dtype} tensor [{B}][heads][{N}][{d}] on {device}")
            Hk = ks[1]
            sb, sh, st, sc = k.stride()
            at.append(40)
            rows += (k.data_ptr(), sb, sh, st, Hk)
            contiguous &= sc == 1
        like_k = False
        for t in others:
            shape, heads = (ks, Hk) if like_k else (qs, Hq)
            like_k = not like_k
            if t is None or shape is None:
                if t is not shape:
                    raise FFError(1, "k comes with its outputs and gradients, or none of them is given")
                at.append(None)
                continue
            if t.shape != shape or t.dtype != dtype or t.device != device:
                raise FFError(1, f"expected a {dtype} tensor of shape {tuple(shape)} on {device}")
            sb, sh, st, sc = t.stride()
            at.append(8 * len(rows))
            rows += (t.data_ptr(), sb, sh, st, heads)
            contiguous &= sc == 1
        if not contiguous:
            raise FFError(1, "the channels of a head must be contiguous")
        rows = array("q", rows)
        base = rows.buffer_info()[0]
        at = [None if o is None else base + o for o in at]
        pos, stride = self._positions(positions, B, N, device)
        return (B, N, pos, stride), at, rows

    def _positions(self, p, B, N, device):
        """Address of the positions and the elements between the samples' (None: none given), checked."""
        if p is None:
            return None, 0
        ps, tail = p.shape, (N,) if self._axes == 1 else (N, 3)
        if p.dtype != self._int32 or p.device != device or not p.is_contiguous() or (ps != tail and ps != (B,) + tail):
            raise FFError(1, f"expected contiguous int32 positions of shape {tail} or {(B,) + tail} on {device}")
        return p.data_ptr(), N * self._axes if len(ps) > len(tail) else 0

    def _weight(self, w, device):
        if w is None:
            return None
        if w.dtype != self._float32 or w.shape != self._channels or not w.is_contiguous() or w.device != device:
            raise FFError(1, f"expected contiguous fp32 weights of shape [{self.cfg.head_dim}] on {device}")
        return w.data_ptr()

    def _call(self, device, fn, *args):
        """The call on the tensors' device (made current for it where another one is) and its current stream."""
        torch = self._torch
        if torch.cuda.current_device() == device.index:
            return self._status(fn(self.handle, *args, self._raw_stream(device.index)))
        with torch.cuda.device(device):
            return self._status(fn(self.handle, *args, self._raw_stream(device.index)))

    def apply(self, q, q_out, k=None, k_out=None, positions=None, inverse: bool = False):
        """The rotation of q and k; inverse: its transpose, the backward pass."""
        place, (hq, hk, hqo, hko), keep = self._arguments(positions, q, k, q_out, k_out)
        self._call(q.device, self._lib.ff_rotary_apply, *place, hq, hk, int(inverse), hqo, hko)
        return q_out, k_out

    def qk_norm(self, q, k, wq, wk, q_out, k_out, eps: float = 1e-6, positions=None):
        """Norm of every row, times wq / wk (fp32 [head_dim], None: ones), then the rotation."""
        place, (hq, hk, hqo, hko), keep = self._arguments(positions, q, k, q_out, k_out)
        dev = q.device
        self._call(dev, self._lib.ff_qk_norm, *place, hq, hk, self._weight(wq, dev), self._weight(wk, dev), eps, hqo, hko)
        return q_out, k_out

    def qk_norm_backward(self, q, k, wq, wk, dq_out, dk_out, dq, dk, dwq=None, dwk=None, eps: float = 1e-6, positions=None):
        """Gradients of q, k (and of the weights, fp32 [head_dim], where given) from those of qk_norm's outputs; dwk without k: zeros."""
        place, (hq, hk, hgq, hgk, hdq, hdk), keep = self._arguments(positions, q, k, dq_out, dk_out, dq, dk)
        dev = q.device
        # (a workspace per call: calls on different streams and captured graphs share none)
        ws = self._torch.empty(self.workspace_bytes, dtype=self._torch.uint8, device=dev)
        self._call(dev, self._lib.ff_qk_norm_backward, *place, hq, hk, self._weight(wq, dev), self._weight(wk, dev), eps, hgq, hgk, hdq, hdk,
                   self._weight(dwq, dev), self._weight(dwk, dev), ws.data_ptr(), self.workspace_bytes)
        return dq, dk


# ---- the gated feed-forward block ----------------------------------------------------------------------
class GatedFFN:
    """out = (act(X Wg) * (X Wu)) Wd on contiguous bf16 CUDA tensors: X, out [..., dim], Wg, Wu [dim][hidden], Wd [hidden][dim]
    (y = x W).  The leading dimensions of X are its tokens."""

    def __init__(self, cfg: FFNConfig, device: str = "cuda:0"):
        import torch
        self.cfg = cfg
        self._torch = torch
        self.handle = C.c_void_p()
        self._c = c = ff_ffn_config_t(cfg.dim, cfg.hidden, {"silu": 0, "gelu_tanh": 1, "gelu": 2}.get(cfg.activation, -1))
        _check(library().ff_ffn_validate(C.byref(c)))
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        with torch.cuda.device(self.device):
            _check(library().ff_ffn_create(C.byref(c), C.byref(self.handle)))
        self._sized, self._bytes = None, 0                       # the workspace's size for the last number of tokens
        self._lib, self._bf16, self._uint8 = library(), torch.bfloat16, torch.uint8
        self._into, self._back = torch.Size((cfg.dim, cfg.hidden)), torch.Size((cfg.hidden, cfg.dim))
        self._raw_stream = _stream_getter(torch)

    def destroy(self):
        if self.handle:
            library().ff_ffn_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def _status(self, status: int):
        if status != FF_OK:
            raise FFError(status, library().ff_ffn_last_error(self.handle).decode())

    def _pointers(self, *tensors):
        """Addresses of (tensor or None, shape) in turns: bf16, contiguous, of that shape and here."""
        bf16, device, at = self._bf16, self.device, []
        for t, shape in zip(tensors[::2], tensors[1::2]):
            if t is None:
                at.append(None)
                continue
            if t.shape != shape or t.dtype != bf16 or t.device != device or not t.is_contiguous():
                raise FFError(1, f"expected a contiguous bf16 tensor of shape {tuple(shape)} on {device}")
            at.append(t.data_ptr())
        return at

    def _shapes(self, X):
        """Number of tokens, shape of X and of the hidden activations."""
        xs = X.shape
        if not xs or xs[-1] != self.cfg.dim:
            raise FFError(1, f"expected X of shape [...][{self.cfg.dim}]")
        return X.numel() // self.cfg.dim, xs, xs[:-1] + (self.cfg.hidden,)

    def _call(self, fn, training, tokens, pointers):
        torch, dev = self._torch, self.device
        if self._sized != (tokens, training):
            size = C.c_size_t()
            _check(library().ff_ffn_workspace_bytes(C.byref(self._c), tokens, training, C.byref(size)))
            self._sized, self._bytes = (tokens, training), size.value
        n = self._bytes
        # (a workspace per call: calls on different streams and captured graphs share none)
        ws = torch.empty(n, dtype=self._uint8, device=dev)
        if torch.cuda.current_device() == dev.index:
            return self._status(fn(self.handle, tokens, *pointers, ws.data_ptr(), n, self._raw_stream(dev.index)))
        with torch.cuda.device(dev):
            return self._status(fn(self.handle, tokens, *pointers, ws.data_ptr(), n, self._raw_stream(dev.index)))

    def forward(self, X, Wg, Wu, Wd, out, gate=None, up=None):
        """gate, up [..., hidden]: X Wg and X Wu are written there, for backward; they overlap nothing.  out may be X."""
        M, xs, hs = self._shapes(X)
        into, back = self._into, self._back
        self._call(self._lib.ff_ffn_forward, False, M, self._pointers(X, xs, Wg, into, Wu, into, Wd, back, gate, hs, up, hs, out, xs))
        return out

    def backward(self, X, Wg, Wu, Wd, gate, up, dout, dX=None, dWg=None, dWu=None, dWd=None):
        """Gradients of X and the weights, where given, from that of out (dWg and dWu together).  dX may be neither X (where dWg is
        given) nor dout (where dWd is): other gradients are made from those in the same launch."""
        M, xs, hs = self._shapes(X)
        into, back = self._into, self._back
        self._call(self._lib.ff_ffn_backward, True, M, self._pointers(X, xs, Wg, into, Wu, into, Wd, back, gate, hs, up, hs, dout, xs, dX, xs,
                                                                      dWg, into, dWu, into, dWd, back))
        return dX, dWg, dWu, dWd

    def device_status(self) -> int:
        with self._torch.cuda.device(self.device):               # (its default stream is 0, as every device's is)
            return library().ff_ffn_device_status(self.handle, self._raw_stream(self.device.index))


# ---- layer norm ----------------------------------------------------------------------------------------
class LayerNorm:
    """y = (x - mean) / sqrt(variance + eps) * weight + bias on CUDA tensors [batch][tokens][dim] (or [tokens][dim]) of any strides whose
    rows are contiguous; weight, bias: contiguous fp32, [dim], or [batch][dim] for each sample its own, or None."""

    def __init__(self, cfg: LayerNormConfig):
        import torch
        self.cfg = cfg
        self._torch = torch
        self.handle = C.c_void_p()
        c = ff_layer_norm_config_t(cfg.dim, {"bf16": 0, "fp32": 1}.get(cfg.dtype, -1), int(cfg.unit_offset), cfg.eps)
        _check(library().ff_layer_norm_create(C.byref(c), C.byref(self.handle)))
        self._dtype = torch.float32 if cfg.dtype == "fp32" else torch.bfloat16
        self._float32, self._model, self._lib = torch.float32, torch.Size((cfg.dim,)), library()
        self._sized, self._bytes = None, 0                       # the workspace's size for the last sizes of a backward call
        self._raw_stream = _stream_getter(torch)

    def destroy(self):
        if self.handle:
            library().ff_layer_norm_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def _status(self, status: int):
        if status != FF_OK:
            raise FFError(status, library().ff_layer_norm_last_error(self.handle).decode())

    def _rows(self, x, *others):
        """Checks the tensors of a call: (batch, tokens), the addresses of their ff_rows_t (None for None), the array that holds those."""
        dtype, device, shape, rank = self._dtype, x.device, x.shape, x.dim()
        if rank not in (2, 3) or shape[-1] != self.cfg.dim or not x.is_cuda or x.dtype != dtype:
            raise FFError(1, f"expected x a {dtype} tensor [batch][tokens][{self.cfg.dim}] or [tokens][{self.cfg.dim}] on a GPU")
        rows, at = [], []
        for t in (x,) + others:
            if t is None:
                at.append(None)
                continue
            if t.shape != shape or t.dtype != dtype or t.device != device:
                raise FFError(1, f"expected a {dtype} tensor of shape {tuple(shape)} on {device}")
            st = t.stride()
            if st[-1] != 1 and shape[-1] > 1:
                raise FFError(1, "the values of a row must be contiguous")
            at.append(8 * len(rows))
            rows += (t.data_ptr(), st[0] if rank == 3 else 0, st[-2])
        rows = array("q", rows)
        base = rows.buffer_info()[0]
        return (shape[0] if rank == 3 else 1, shape[-2]), [None if o is None else base + o for o in at], rows

    def _weights(self, batch, device, *weights):
        """Whether they are each sample's, and their addresses."""
        per_sample, shape, at = 0, None, []
        for w in weights:
            if w is None:
                at.append(None)
                continue
            if shape is None:
                shape = self._model if w.shape == self._model else self._torch.Size((batch, self.cfg.dim))
                per_sample = int(shape is not self._model)
            if w.dtype != self._float32 or w.shape != shape or not w.is_contiguous() or w.device != device:
                raise FFError(1, f"expected contiguous fp32 weights and biases, all [{self.cfg.dim}] or all [{batch}][{self.cfg.dim}], on {device}")
            at.append(w.data_ptr())
        return per_sample, at

    def _call(self, device, fn, *args):
        """The call on the tensors' device (made current for it where another one is) and its current stream."""
        torch = self._torch
        if torch.cuda.current_device() == device.index:
            return self._status(fn(self.handle, *args, self._raw_stream(device.index)))
        with torch.cuda.device(device):
            return self._status(fn(self.handle, *args, self._raw_stream(device.index)))

    def forward(self, x, weight, bias, y):
        """y may be x."""
        size, (ax, ay), keep = self._rows(x, y)
        per_sample, (w, b) = self._weights(size[0], x.device, weight, bias)
        self._call(x.device, self._lib.ff_layer_norm_forward, *size, ax, w, b, per_sample, ay)
        return y

    def backward(self, x, weight, dy, dx, dweight=None, dbias=None):
        """Gradients of x (dx may be dy or x, or None) and, where given, of weight and bias, from the input x and the gradient of y."""
        size, (ax, ag, ad), keep = self._rows(x, dy, dx)
        per_sample, (w, dw, db) = self._weights(size[0], x.device, weight, dweight, dbias)
        if self._sized != (size, per_sample):
            n = C.c_size_t()
            self._status(self._lib.ff_layer_norm_workspace_bytes(self.handle, *size, per_sample, C.byref(n)))
            self._sized, self._bytes = (size, per_sample), n.value
        # (a workspace per call: calls on different streams and captured graphs share none)
        ws = self._torch.empty(self._bytes, dtype=self._torch.uint8, device=x.device)
        self._call(x.device, self._lib.ff_layer_norm_backward, *size, ax, w, per_sample, ag, ad, dw, db, ws.data_ptr(), self._bytes)
        return dx, dweight, dbias


# ---- cross attention -----------------------------------------------------------------------------------
class CrossAttention:
    """out = softmax(scale q k^T) v over the keys that count, on bf16 CUDA tensors [batch][heads][tokens][head_dim] of any strides (16-byte
    multiples) whose channels are contiguous; k and v have kv_heads heads and the encoder's number of states.
    lengths: int32 [batch], keys from there on do not count;  mask: bool or uint8 [batch][keys], false: the key does not count."""

    def __init__(self, cfg: CrossAttentionConfig, device: str = "cuda:0"):
        import torch
        self.cfg = cfg
        self._torch = torch
        self.handle = C.c_void_p()
        self._c = c = ff_cross_attention_config_t(cfg.head_dim, cfg.heads, cfg.kv_heads, cfg.scale)
        _check(library().ff_cross_attention_validate(C.byref(c)))
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        with torch.cuda.device(self.device):
            _check(library().ff_cross_attention_create(C.byref(c), C.byref(self.handle)))
        self._sized, self._bytes = None, 0                       # the workspace's size for the last sizes of a call
        self._lib, self._bf16, self._uint8, self._float32, self._int32 = library(), torch.bfloat16, torch.uint8, torch.float32, torch.int32
        self._mask_types = (torch.bool, torch.uint8)
        self._raw_stream = _stream_getter(torch)

    def destroy(self):
        if self.handle:
            library().ff_cross_attention_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def _status(self, status: int):
        if status != FF_OK:
            raise FFError(status, library().ff_cross_attention_last_error(self.handle).decode())

    def _heads(self, q, k, *others):
        """Checks the tensors of a call, `others` as (tensor or None, is it like k) in turns: (batch, queries, keys), the addresses of
        their ff_heads_t (None for None), and the array that holds those."""
        c, bf16, device = self.cfg, self._bf16, self.device
        qs, ks = q.shape, k.shape
        if len(qs) != 4 or qs[1] != c.heads or qs[3] != c.head_dim:
            raise FFError(1, f"expected q a tensor [batch][{c.heads}][queries][{c.head_dim}]")
        if len(ks) != 4 or ks[0] != qs[0] or ks[1] != c.kv_heads or ks[3] != c.head_dim:
            raise FFError(1, f"expected k a tensor [{qs[0]}][{c.kv_heads}][keys][{c.head_dim}]")
        rows, at = [], []
        for t, like_k in ((q, False), (k, True)) + tuple(zip(others[::2], others[1::2])):
            if t is None:
                at.append(None)
                continue
            if t.shape != (ks if like_k else qs) or t.dtype != bf16 or t.device != device:
                raise FFError(1, f"expected a bf16 tensor of shape {tuple(ks if like_k else qs)} on {device}")
            sb, sh, st, sc = t.stride()
            if sc != 1:
                raise FFError(1, "the channels of a head must be contiguous")
            at.append(8 * len(rows))
            rows += (t.data_ptr(), sb, sh, st, c.kv_heads if like_k else c.heads)         # (the layout of ff_heads_t, heads in its low half word)
        rows = array("q", rows)
        base = rows.buffer_info()[0]
        return (qs[0], qs[2], ks[2]), [None if o is None else base + o for o in at], rows

    def _keys(self, size, lengths, mask):
        """Addresses of the lengths and the mask, checked."""
        at = []
        for t, types, shape, what in ((lengths, (self._int32,), size[:1], "int32 lengths"), (mask, self._mask_types, size[::2], "a bool mask")):
            if t is None:
                at.append(None)
                continue
            if t.dtype not in types or t.shape != shape or not t.is_contiguous() or t.device != self.device:
                raise FFError(1, f"expected {what}, contiguous, of shape {tuple(shape)} on {self.device}")
            at.append(t.data_ptr())
        return at

    def _lse(self, size, lse):
        if lse is None:
            return None
        shape = (size[0], self.cfg.heads, size[1])
        if lse.dtype != self._float32 or lse.shape != shape or not lse.is_contiguous() or lse.device != self.device:
            raise FFError(1, f"expected lse a contiguous fp32 tensor of shape {shape} on {self.device}")
        return lse.data_ptr()

    def _call(self, fn, training, size, *args):
        torch, dev = self._torch, self.device
        if self._sized != (size, training):
            n = C.c_size_t()
            _check(self._lib.ff_cross_attention_workspace_bytes(C.byref(self._c), *size, training, C.byref(n)))
            self._sized, self._bytes = (size, training), n.value
        n = self._bytes
        # (a workspace per call that takes one: calls on different streams and captured graphs share none)
        ws = torch.empty(n, dtype=self._uint8, device=dev) if n else None
        at = ws.data_ptr() if n else None
        if torch.cuda.current_device() == dev.index:
            return self._status(fn(self.handle, *size, *args, at, n, self._raw_stream(dev.index)))
        with torch.cuda.device(dev):
            return self._status(fn(self.handle, *size, *args, at, n, self._raw_stream(dev.index)))

    def forward(self, q, k, v, out, lse=None, lengths=None, mask=None):
        """lse (fp32 [batch][heads][queries]): the logarithms of the rows' sums are written there, for backward.  out may be q."""
        size, (aq, ak, av, ao), keep = self._heads(q, k, v, True, out, False)
        self._call(self._lib.ff_cross_attention_forward, False, size, aq, ak, av, *self._keys(size, lengths, mask), ao, self._lse(size, lse))
        return out

    def backward(self, q, k, v, out, lse, dout, dq=None, dk=None, dv=None, lengths=None, mask=None):
        """Gradients of q, k and v, where given (dk and dv together), from that of out and what forward left in out and lse.  They
        overlap no other tensor."""
        size, (aq, ak, av, ao, ag, adq, adk, adv), keep = self._heads(q, k, v, True, out, False, dout, False, dq, False, dk, True, dv, True)
        self._call(self._lib.ff_cross_attention_backward, True, size, aq, ak, av, *self._keys(size, lengths, mask), ao, self._lse(size, lse), ag, adq,
                   adk, adv)
        return dq, dk, dv

    def device_status(self) -> int:
        with self._torch.cuda.device(self.device):               # (its default stream is 0, as every device's is)
            return library().ff_cross_attention_device_status(self.handle, self._raw_stream(self.device.index))


# Same names as the C entry points, for callers that prefer the flat API.
def ff_plan_create(cfg: FFConfig, weights=None, U=None, host_staging=False, device="cuda:0") -> Plan:
    return Plan(cfg, weights, U, host_staging, device)


def ff_route(plan: Plan, Q, K, V, timesteps, alloc_out=None):
    return plan.route(Q, K, V, timesteps, alloc_out)


def ff_forward(plan: Plan, Q, K, V, out, alloc=None, timesteps=None):
    return plan.forward(Q, K, V, out, alloc, timesteps)


def ff_forward_host(plan: Plan, Qh, Kh, Vh, out_h, alloc_host=None, timesteps=None):
    return plan.forward_host(Qh, Kh, Vh, out_h, alloc_host, timesteps)


def ff_forward_projected(plan: Plan, X, Wqkv, Wo, out, alloc=None, timesteps=None):
    return plan.forward_projected(X, Wqkv, Wo, out, alloc, timesteps)


def ff_forward_projected_rotary(plan: Plan, X, Wqkv, Wo, out, rotary: Rotary, wq=None, wk=None, eps=0.0, positions=None, alloc=None,
                                timesteps=None):
    return plan.forward_projected(X, Wqkv, Wo, out, alloc, timesteps, rotary, wq, wk, eps, positions)


def ff_rotary_create(cfg: RotaryConfig) -> Rotary:
    return Rotary(cfg)


def ff_rotary_apply(rotary: Rotary, q, q_out, k=None, k_out=None, positions=None, inverse=False):
    return rotary.apply(q, q_out, k, k_out, positions, inverse)


def ff_qk_norm(rotary: Rotary, q, k, wq, wk, q_out, k_out, eps=1e-6, positions=None):
    return rotary.qk_norm(q, k, wq, wk, q_out, k_out, eps, positions)


def ff_qk_norm_backward(rotary: Rotary, q, k, wq, wk, dq_out, dk_out, dq, dk, dwq=None, dwk=None, eps=1e-6, positions=None):
    return rotary.qk_norm_backward(q, k, wq, wk, dq_out, dk_out, dq, dk, dwq, dwk, eps, positions)


def ff_ffn_create(cfg: FFNConfig, device="cuda:0") -> GatedFFN:
    return GatedFFN(cfg, device)


def ff_ffn_forward(ffn: GatedFFN, X, Wg, Wu, Wd, out, gate=None, up=None):
    return ffn.forward(X, Wg, Wu, Wd, out, gate, up)


def ff_ffn_backward(ffn: GatedFFN, X, Wg, Wu, Wd, gate, up, dout, dX=None, dWg=None, dWu=None, dWd=None):
    return ffn.backward(X, Wg, Wu, Wd, gate, up, dout, dX, dWg, dWu, dWd)


def ff_layer_norm_create(cfg: LayerNormConfig) -> LayerNorm:
    return LayerNorm(cfg)


def ff_layer_norm_forward(norm: LayerNorm, x, weight, bias, y):
    return norm.forward(x, weight, bias, y)


def ff_layer_norm_backward(norm: LayerNorm, x, weight, dy, dx, dweight=None, dbias=None):
    return norm.backward(x, weight, dy, dx, dweight, dbias)


def ff_cross_attention_create(cfg: CrossAttentionConfig, device="cuda:0") -> CrossAttention:
    return CrossAttention(cfg, device)


def ff_cross_attention_forward(attention: CrossAttention, q, k, v, out, lse=None, lengths=None, mask=None):
    return attention.forward(q, k, v, out, lse, lengths, mask)


def ff_cross_attention_backward(attention: CrossAttention, q, k, v, out, lse, dout, dq=None, dk=None, dv=None, lengths=None, mask=None):
    return attention.backward(q, k, v, out, lse, dout, dq, dk, dv, lengths, mask)


def ff_high_attention_noalloc(q, k, v, y, radius: int, sync: bool = True):
    """High-band sliding-window attention on bf16 CUDA tensors [heads][n][128] without any device
    allocation inside the call (the kernel's scratch is a fixed array in the library): for hosts
    whose device memory is fully owned by their own pool, or that cannot tolerate the device-wide
    synchronisation of an allocation.  Calls on one device share that scratch: do not overlap them."""
    import torch
    for t in (q, k, v, y):
        if (not t.is_cuda or t.device != q.device or t.dtype != torch.bfloat16 or not t.is_contiguous() or t.dim() != 3
                or t.shape[2] != 128 or t.shape != q.shape):
            raise FFError(1, "expected contiguous bf16 CUDA tensors of one shape [heads][n][128] on one device")
    stream = C.c_void_p(torch.cuda.current_stream(q.device).cuda_stream)
    with torch.cuda.device(q.device):
        _check(library().ff_high_attention_noalloc(q.data_ptr(), k.data_ptr(), v.data_ptr(), y.data_ptr(), q.shape[0],
                                                   q.shape[1], radius, int(sync), stream))
    return y


def ff_destroy(plan: Plan):
    plan.destroy()
