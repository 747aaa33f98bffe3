"""Thin Python binding of libhot, the MI355X implementation of the HOT linear-layer
backward pass (arxiv 2503.21261).

Argument marshalling only: every step runs in the HIP kernels behind the C ABI
declared in ``include/hot.h``; function names here are the C names.  torch is
used for device memory and streams.  There is no CPU fallback: if the library
has not been built, importing the entry points raises.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional, Sequence, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libhot.so")

HOT_OK = 0
HOT_ERR_ARG, HOT_ERR_SHAPE, HOT_ERR_WORKSPACE, HOT_ERR_DEVICE, HOT_ERR_UNIMPLEMENTED = 1, 2, 3, 4, 5
HOT_ERR_SCRATCH_LIMIT = 6
HOT_NOALLOC_SCRATCH_BYTES = 64 << 20
HOT_Q_PER_TENSOR, HOT_Q_PER_TOKEN = 0, 1
HOT_ROUND_NEAREST_EVEN, HOT_ROUND_PSEUDO_STOCHASTIC, HOT_ROUND_DRAWN = 0, 1, 3

EXPORTS = (
    "hot_default_config", "hot_status_string", "hot_act_buffer_bytes", "hot_workspace_bytes",
    "hot_weight_buffer_bytes", "hot_gx_cached_workspace_bytes", "hot_quantize_weight", "hot_linear_backward_gx_cached",
    "hot_debug_unpack_weight", "hot_compress_activation", "hot_linear_backward_gx", "hot_linear_backward_gw",
    "hot_linear_backward", "hot_linear_backward_gx_noalloc", "hot_lowpass_l1_rows", "hot_select_quantizer", "hot_debug_unpack_activation",
    "hot_debug_gx_operands", "hot_debug_gw_operands", "hot_debug_fused_operands", "hot_debug_set_exchange_wait_us",
    "hot_debug_set_backward_strategy", "hot_debug_set_gemm_mode", "hot_debug_profile_begin", "hot_debug_profile_end", "hot_debug_profile_end_all", "hot_debug_profile_sequence",
    "hot_debug_stage_name", "hot_debug_probe", "hot_debug_gemm_plan", "hot_debug_linear_plan",
    "hot_checkpoint_bytes", "hot_checkpoint_write", "hot_checkpoint_read", "hot_activation_forward",
    "hot_activation_backward_workspace_bytes", "hot_activation_backward", "hot_layer_norm_forward",
    "hot_layer_norm_backward_workspace_bytes", "hot_layer_norm_backward", "hot_linear_forward_workspace_bytes",
    "hot_linear_forward",
    "hot_adapter_forward_workspace_bytes", "hot_adapter_backward_workspace_bytes", "hot_adapter_forward", "hot_adapter_backward",
    "hot_token_logprobs_workspace_bytes", "hot_token_logprobs", "hot_token_logprobs_backward",
    "hot_adamw_state_bytes", "hot_adamw_state_read", "hot_adamw_state_write", "hot_adamw_table_bytes", "hot_adamw_table", "hot_adamw_step",
)
HOT_NUM_STAGES, HOT_NUM_STAGES_ALL = 15, 36
HOT_WS_PREFIX_BYTES = 24832
HOT_F32, HOT_BF16 = 0, 1
HOT_ACT_NONE, HOT_ACT_RELU, HOT_ACT_GELU, HOT_ACT_GELU_TANH, HOT_ACT_SILU = range(5)
ACT_FNS = {"none": HOT_ACT_NONE, "relu": HOT_ACT_RELU, "gelu": HOT_ACT_GELU, "gelu_tanh": HOT_ACT_GELU_TANH,
           "silu": HOT_ACT_SILU}
HOT_MAX_TOP, HOT_MAX_RANK = 32, 128
HOT_STATE_F32, HOT_STATE_8BIT = 0, 1
HOT_MOMENT_M, HOT_MOMENT_V = 0, 1


class hot_config(C.Structure):
    _fields_ = [("block", C.c_int32), ("keep", C.c_int32), ("keep_idx", C.POINTER(C.c_int32)),
                ("gx_bits", C.c_int32), ("gw_bits", C.c_int32), ("rounding", C.c_int32),
                ("lqs_threshold", C.c_float), ("sample_tokens", C.c_int32), ("replayable", C.c_int32)]


class hot_gemm_plan(C.Structure):
    _fields_ = [("one_launch", C.c_int32)] + [(f, C.c_int32 * 5) for f in ("gx", "gw", "gx_alone", "gw_alone")]


class hot_linear_plan(C.Structure):
    _fields_ = [(f, C.c_int32) for f in ("way", "tile_rows", "tile_cols", "tiles", "whole", "slices", "masked", "streams")]


class hot_adamw_tensor(C.Structure):
    _fields_ = ([(f, C.c_void_p) for f in ("grad", "param", "m", "v", "param_out", "m_out", "v_out", "copy")] +
                [("n", C.c_int64), ("param_type", C.c_int32), ("grad_type", C.c_int32), ("weight_decay", C.c_float), ("lr_factor", C.c_float)])


class hot_adamw_config(C.Structure):
    _fields_ = ([(f, C.c_double) for f in ("lr", "beta1", "beta2", "eps")] +
                [("step", C.c_int64), ("rounding", C.c_int32), ("dynamic_count", C.c_int32), ("dynamic", C.c_void_p)])


class HotError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (hot_status {status})")


_lib: Optional[C.CDLL] = None


def lib() -> C.CDLL:
    """Loads libhot.so; fails loudly if it has not been built (no fallback)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2503_21261_amd.build` "
                "(or __graft_entry__.build()); there is no CPU fallback")
        l = C.CDLL(LIB_PATH)
        i64, vp, sz = C.c_int64, C.c_void_p, C.c_size_t
        cfgp = C.POINTER(hot_config)
        l.hot_default_config.argtypes = [cfgp]
        l.hot_default_config.restype = None
        l.hot_status_string.argtypes = [C.c_int]
        l.hot_status_string.restype = C.c_char_p
        l.hot_act_buffer_bytes.argtypes = [cfgp, i64, i64]
        l.hot_act_buffer_bytes.restype = sz
        l.hot_workspace_bytes.argtypes = [cfgp, i64, i64, i64]
        l.hot_workspace_bytes.restype = sz
        l.hot_compress_activation.argtypes = [cfgp, vp, i64, i64, vp, vp, sz, vp]
        l.hot_linear_backward_gx.argtypes = [cfgp, vp, vp, i64, i64, i64, C.c_int, vp, vp, sz, vp]
        l.hot_linear_backward_gx_noalloc.argtypes = [cfgp, vp, vp, i64, i64, i64, C.c_int, vp, vp]
        l.hot_linear_backward_gw.argtypes = [cfgp, vp, vp, i64, i64, i64, vp, vp, sz, vp]
        l.hot_linear_backward.argtypes = [cfgp, vp, vp, vp, i64, i64, i64, C.c_int, vp, vp, vp, sz, vp]
        l.hot_select_quantizer.argtypes = [cfgp, vp, i64, i64, C.POINTER(C.c_int),
                                           C.POINTER(C.c_double), C.POINTER(C.c_double), vp, sz, vp]
        l.hot_lowpass_l1_rows.argtypes = [C.c_int32, C.c_int32, C.POINTER(C.c_int32)]
        l.hot_debug_unpack_activation.argtypes = [cfgp, vp, i64, i64, vp, vp, vp]
        l.hot_debug_gx_operands.argtypes = [cfgp, vp, i64, i64, i64, C.c_int, vp, vp, vp, vp, vp, vp]
        l.hot_debug_gw_operands.argtypes = [cfgp, vp, vp, i64, i64, i64, vp, vp, vp, vp]
        l.hot_debug_fused_operands.argtypes = [cfgp, vp, vp, i64, i64, i64, C.c_int] + [vp] * 9
        l.hot_debug_set_exchange_wait_us.argtypes = [C.c_int]
        l.hot_debug_set_backward_strategy.argtypes = [C.c_int]
        l.hot_debug_set_gemm_mode.argtypes = [C.c_int]
        l.hot_debug_profile_begin.argtypes = []
        l.hot_debug_profile_end.argtypes = [C.POINTER(C.c_float), C.POINTER(C.c_int64)]
        l.hot_debug_profile_end_all.argtypes = [C.POINTER(C.c_float), C.POINTER(C.c_int64), C.c_int32]
        l.hot_debug_linear_plan.argtypes = [C.c_int, C.c_int, i64, i64, i64, C.c_int32, C.POINTER(hot_linear_plan)]
        l.hot_debug_gemm_plan.argtypes = [cfgp, i64, i64, i64, C.POINTER(hot_gemm_plan)]
        l.hot_debug_probe.argtypes = [C.c_int, vp, sz, C.c_int, vp]
        l.hot_debug_profile_sequence.argtypes = [C.POINTER(C.c_int32), C.c_int64]
        l.hot_weight_buffer_bytes.argtypes = [cfgp, i64, i64]
        l.hot_weight_buffer_bytes.restype = sz
        l.hot_gx_cached_workspace_bytes.argtypes = [cfgp, i64, i64, i64]
        l.hot_gx_cached_workspace_bytes.restype = sz
        l.hot_quantize_weight.argtypes = [cfgp, vp, i64, i64, vp, vp, sz, vp]
        l.hot_linear_backward_gx_cached.argtypes = [cfgp, vp, vp, i64, i64, i64, C.c_int, vp, vp, sz, vp]
        l.hot_debug_unpack_weight.argtypes = [cfgp, vp, i64, i64, vp, vp, vp]
        en = C.c_int
        l.hot_checkpoint_write.argtypes = [vp, en, i64, i64, vp, vp]
        l.hot_checkpoint_read.argtypes = [vp, i64, i64, vp, en, vp]
        l.hot_activation_forward.argtypes = [en, vp, en, i64, i64, vp, vp, vp]
        l.hot_activation_backward.argtypes = [en, vp, en, vp, vp, i64, i64, vp, vp, vp, sz, vp]
        l.hot_layer_norm_forward.argtypes = [vp, en, vp, vp, vp, C.c_float, i64, i64, vp, vp, en, vp, vp, vp, vp]
        l.hot_layer_norm_backward.argtypes = [vp, en, vp, vp, en, vp, vp, vp, vp, i64, i64, vp, vp, vp, vp, sz, vp]
        l.hot_linear_forward.argtypes = [vp, vp, en, vp, vp, i64, i64, i64, en, vp, en, vp, vp, sz, vp]
        l.hot_adapter_forward.argtypes = [vp, vp, vp, en, vp, vp, vp] + [i64] * 6 + [vp, vp, vp, vp, sz, vp]
        l.hot_adapter_backward.argtypes = [vp, vp, vp, vp, vp, en, vp, vp, vp] + [i64] * 6 + [vp, vp, vp, vp, vp, sz, vp]
        l.hot_token_logprobs.argtypes = [vp, en, i64, i64, vp, vp, vp, vp, C.c_int32, vp, vp, vp, sz, vp]
        l.hot_token_logprobs_backward.argtypes = [vp, en, i64, i64, vp, vp, vp, vp, vp, vp, vp]
        l.hot_adamw_state_read.argtypes = [vp, en, i64, vp, en, vp]
        l.hot_adamw_state_write.argtypes = [vp, en, en, i64, vp, vp]
        l.hot_adamw_table.argtypes = [C.POINTER(hot_adamw_tensor), C.c_int32, en, vp, sz]
        l.hot_adamw_step.argtypes = [vp, C.POINTER(hot_adamw_config), vp]
        sizes = {"hot_adapter_forward_workspace_bytes": [en] + [i64] * 6, "hot_adapter_backward_workspace_bytes": [en] + [i64] * 6,
                 "hot_token_logprobs_workspace_bytes": [en, i64, i64, C.c_int32], "hot_adamw_state_bytes": [en, i64],
                 "hot_adamw_table_bytes": [C.c_int32], "hot_checkpoint_bytes": [i64, i64], "hot_activation_backward_workspace_bytes": [i64, i64],
                 "hot_layer_norm_backward_workspace_bytes": [i64, i64],
                 "hot_linear_forward_workspace_bytes": [en, i64, i64, i64]}
        for name, args in sizes.items():
            getattr(l, name).argtypes = args
            getattr(l, name).restype = sz
        for name in EXPORTS[6:]:
            if name in sizes:
                continue
            if name not in ("hot_debug_stage_name", "hot_debug_profile_sequence"):
                getattr(l, name).restype = C.c_int
        l.hot_debug_profile_sequence.restype = C.c_int64
        l.hot_debug_stage_name.argtypes = [C.c_int]
        l.hot_debug_stage_name.restype = C.c_char_p
        _lib = l
    return _lib


def status_string(status: int) -> str:
    return lib().hot_status_string(int(status)).decode()


@dataclass
class Config:
    """Python mirror of ``hot_config`` (paper defaults: n=16, r=8, INT4/INT8, PSR, 0.5)."""
    block: int = 16
    keep: int = 8
    keep_idx: Optional[Sequence[int]] = None
    gx_bits: int = 4
    gw_bits: int = 8
    rounding: int = HOT_ROUND_PSEUDO_STOCHASTIC
    lqs_threshold: float = 0.5
    sample_tokens: int = 0
    replayable: bool = False     # launch tags from the workspace epoch: calls may be recorded into a HIP graph

    def reduced_tokens(self, L: int) -> int:
        """L' = tokens after HLA: L*r/n, or B * ceil(S/n) * r with per-sample tiling."""
        if self.sample_tokens:
            return L // self.sample_tokens * (-(-self.sample_tokens // self.block)) * self.keep
        return L // self.block * self.keep

    def c(self) -> hot_config:
        keep_idx = None
        self._keep_arr = None
        if self.keep_idx is not None:
            self._keep_arr = (C.c_int32 * len(self.keep_idx))(*[int(k) for k in self.keep_idx])
            keep_idx = C.cast(self._keep_arr, C.POINTER(C.c_int32))
        return hot_config(int(self.block), int(self.keep), keep_idx, int(self.gx_bits), int(self.gw_bits),
                          int(self.rounding), float(self.lqs_threshold), int(self.sample_tokens),
                          1 if self.replayable else 0)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


# The current stream's handle alone, a Stream object of which costs a call over a microsecond; private to torch, so
# that a torch without it takes the object.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> Optional[int]:
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device()) or None
        stream = torch.cuda.current_stream()
    return stream.cuda_stream or None


def _check(status: int, where: str) -> None:
    if status != HOT_OK:
        raise HotError(status, where)


def _dev_f32(t: torch.Tensor, shape: Tuple[int, ...], name: str) -> None:
    if not (t.is_cuda and t.dtype == torch.float32 and t.is_contiguous() and t.shape == shape):
        raise ValueError(f"{name}: expected contiguous float32 device tensor of shape {shape}")


def hot_act_buffer_bytes(cfg: Config, L: int, I: int) -> int:
    return int(lib().hot_act_buffer_bytes(C.byref(cfg.c()), L, I))


def hot_workspace_bytes(cfg: Config, L: int, O: int, I: int) -> int:
    return int(lib().hot_workspace_bytes(C.byref(cfg.c()), L, O, I))


def alloc_workspace(cfg: Config, L: int, O: int, I: int, device="cuda") -> torch.Tensor:
    n = hot_workspace_bytes(cfg, L, O, I)
    if n == 0:
        raise HotError(HOT_ERR_SHAPE, "hot_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def alloc_act_buffer(cfg: Config, L: int, I: int, device="cuda") -> torch.Tensor:
    n = hot_act_buffer_bytes(cfg, L, I)
    if n == 0:
        raise HotError(HOT_ERR_SHAPE, "hot_act_buffer_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def hot_weight_buffer_bytes(cfg: Config, O: int, I: int) -> int:
    return int(lib().hot_weight_buffer_bytes(C.byref(cfg.c()), O, I))


def hot_gx_cached_workspace_bytes(cfg: Config, L: int, O: int, I: int) -> int:
    return int(lib().hot_gx_cached_workspace_bytes(C.byref(cfg.c()), L, O, I))


def alloc_weight_buffer(cfg: Config, O: int, I: int, device="cuda") -> torch.Tensor:
    n = hot_weight_buffer_bytes(cfg, O, I)
    if n == 0:
        raise HotError(HOT_ERR_SHAPE, "hot_weight_buffer_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def hot_quantize_weight(cfg: Config, w: torch.Tensor, wq_buf: torch.Tensor, ws: torch.Tensor,
                        stream=None) -> torch.Tensor:
    O, I = w.shape
    _dev_f32(w, (O, I), "w")
    st = lib().hot_quantize_weight(C.byref(cfg.c()), _ptr(w), O, I, _ptr(wq_buf), _ptr(ws),
                                   ws.numel(), _stream(stream))
    _check(st, "hot_quantize_weight")
    return wq_buf


def hot_linear_backward_gx_cached(cfg: Config, g_y: torch.Tensor, wq_buf: torch.Tensor, I: int,
                                  gy_quantizer: int, g_x: torch.Tensor, ws: torch.Tensor,
                                  stream=None) -> torch.Tensor:
    L, O = g_y.shape
    _dev_f32(g_y, (L, O), "g_y"); _dev_f32(g_x, (L, I), "g_x")
    st = lib().hot_linear_backward_gx_cached(C.byref(cfg.c()), _ptr(g_y), _ptr(wq_buf), L, O, I,
                                             int(gy_quantizer), _ptr(g_x), _ptr(ws), ws.numel(),
                                             _stream(stream))
    _check(st, "hot_linear_backward_gx_cached")
    return g_x


def hot_debug_unpack_weight(cfg: Config, wq_buf: torch.Tensor, O: int, I: int, stream=None):
    """Returns (codes int8 [O, I], scale float32 [1]) on the device."""
    codes = torch.empty((O, I), dtype=torch.int8, device=wq_buf.device)
    scale = torch.empty(1, dtype=torch.float32, device=wq_buf.device)
    st = lib().hot_debug_unpack_weight(C.byref(cfg.c()), _ptr(wq_buf), O, I, _ptr(codes),
                                       _ptr(scale), _stream(stream))
    _check(st, "hot_debug_unpack_weight")
    return codes, scale


def hot_compress_activation(cfg: Config, x: torch.Tensor, act_buf: torch.Tensor,
                            ws: torch.Tensor, stream=None) -> torch.Tensor:
    L, I = x.shape
    _dev_f32(x, (L, I), "x")
    st = lib().hot_compress_activation(C.byref(cfg.c()), _ptr(x), L, I, _ptr(act_buf), _ptr(ws),
                                       ws.numel(), _stream(stream))
    _check(st, "hot_compress_activation")
    return act_buf


def hot_linear_backward_gx(cfg: Config, g_y: torch.Tensor, w: torch.Tensor, gy_quantizer: int,
                           g_x: torch.Tensor, ws: torch.Tensor, stream=None) -> torch.Tensor:
    L, O = g_y.shape
    I = w.shape[1]
    _dev_f32(g_y, (L, O), "g_y"); _dev_f32(w, (O, I), "w"); _dev_f32(g_x, (L, I), "g_x")
    st = lib().hot_linear_backward_gx(C.byref(cfg.c()), _ptr(g_y), _ptr(w), L, O, I,
                                      int(gy_quantizer), _ptr(g_x), _ptr(ws), ws.numel(),
                                      _stream(stream))
    _check(st, "hot_linear_backward_gx")
    return g_x


def hot_linear_backward_gx_noalloc(cfg: Config, g_y: torch.Tensor, w: torch.Tensor, gy_quantizer: int,
                                   g_x: torch.Tensor, stream=None) -> torch.Tensor:
    """hot_linear_backward_gx with the library's built-in scratch instead of a workspace."""
    L, O = g_y.shape
    I = w.shape[1]
    _dev_f32(g_y, (L, O), "g_y"); _dev_f32(w, (O, I), "w"); _dev_f32(g_x, (L, I), "g_x")
    st = lib().hot_linear_backward_gx_noalloc(C.byref(cfg.c()), _ptr(g_y), _ptr(w), L, O, I,
                                              int(gy_quantizer), _ptr(g_x), _stream(stream))
    _check(st, "hot_linear_backward_gx_noalloc")
    return g_x


def hot_linear_backward_gw(cfg: Config, g_y: torch.Tensor, act_buf: torch.Tensor, I: int,
                           g_w: torch.Tensor, ws: torch.Tensor, stream=None) -> torch.Tensor:
    L, O = g_y.shape
    _dev_f32(g_y, (L, O), "g_y"); _dev_f32(g_w, (O, I), "g_w")
    st = lib().hot_linear_backward_gw(C.byref(cfg.c()), _ptr(g_y), _ptr(act_buf), L, O, I,
                                      _ptr(g_w), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "hot_linear_backward_gw")
    return g_w


def hot_linear_backward(cfg: Config, g_y: torch.Tensor, w: torch.Tensor, act_buf: torch.Tensor,
                        gy_quantizer: int, g_x: torch.Tensor, g_w: torch.Tensor, ws: torch.Tensor,
                        stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    L, O = g_y.shape
    I = w.shape[1]
    _dev_f32(g_y, (L, O), "g_y"); _dev_f32(w, (O, I), "w")
    _dev_f32(g_x, (L, I), "g_x"); _dev_f32(g_w, (O, I), "g_w")
    st = lib().hot_linear_backward(C.byref(cfg.c()), _ptr(g_y), _ptr(w), _ptr(act_buf), L, O, I,
                                   int(gy_quantizer), _ptr(g_x), _ptr(g_w), _ptr(ws), ws.numel(),
                                   _stream(stream))
    _check(st, "hot_linear_backward")
    return g_x, g_w


def hot_select_quantizer(cfg: Config, g_y: torch.Tensor, ws: torch.Tensor,
                         stream=None) -> Tuple[int, float, float]:
    """Returns (choice, mse_token, mse_tensor)."""
    L, O = g_y.shape
    _dev_f32(g_y, (L, O), "g_y")
    choice, mt, mn = C.c_int(-1), C.c_double(0), C.c_double(0)
    st = lib().hot_select_quantizer(C.byref(cfg.c()), _ptr(g_y), L, O, C.byref(choice),
                                    C.byref(mt), C.byref(mn), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "hot_select_quantizer")
    return choice.value, mt.value, mn.value


def hot_lowpass_l1_rows(block: int, keep: int):
    """The `keep` low-pass rows of a block by the LP_L1 criterion, as a list for Config.keep_idx."""
    out = (C.c_int32 * keep)()
    _check(lib().hot_lowpass_l1_rows(int(block), int(keep), out), "hot_lowpass_l1_rows")
    return [int(k) for k in out]


# ---- the operators around the linear backward -----------------------------------------------------------------------
# Tensors are contiguous [rows, cols] of float32 or bfloat16 on the current device; the argument checks below hold for each.

_TYPES = {torch.float32: HOT_F32, torch.bfloat16: HOT_BF16}


# The index alone; private to torch, so that a torch without it takes the public call.
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _stream_of(stream, device: int) -> Optional[int]:
    """As _stream(), for the current device that the caller has asked for already."""
    if stream is None and _raw_stream is not None:
        return _raw_stream(device) or None
    return _stream(stream)


def _expect(name: str, t: torch.Tensor, dtype: torch.dtype, shape: Tuple[int, ...], device: int) -> int:
    """The tensor's address; raises unless it is a contiguous `dtype` tensor of `shape` on CUDA device `device`."""
    if t.get_device() != device or t.dtype is not dtype or t.shape != shape or not t.is_contiguous():   # a host tensor's device is -1
        raise ValueError(f"{name}: expected contiguous {dtype} tensor of shape {tuple(shape)} on cuda:{device}, the current device")
    return t.data_ptr()


def _typed(name: str, t: torch.Tensor) -> int:
    """hot_type of a tensor that sets the type of others; raises unless it is a matrix of a supported type on a GPU."""
    ty = _TYPES.get(t.dtype)
    if ty is None or t.dim() != 2 or not t.is_cuda:
        raise ValueError(f"{name}: expected a float32 or bfloat16 device tensor of two dimensions")
    return ty


def _bytes(name: str, t: torch.Tensor, least: int, device: int) -> int:
    """Address of an opaque uint8 buffer of at least `least` bytes."""
    if t.get_device() != device or t.dtype is not torch.uint8 or t.numel() < least or not t.is_contiguous():
        raise ValueError(f"{name}: expected contiguous uint8 tensor of at least {least} bytes on cuda:{device}, the current device")
    return t.data_ptr()


def _ckpt(t: torch.Tensor, rows: int, cols: int, device: int) -> int:
    """Address of a checkpoint of [rows, cols]; its size is hot_checkpoint_bytes()'s, worked out here without a call."""
    pitch = cols + 31 & -32
    return _bytes("ckpt", t, (rows * pitch + 255 & -256) + rows * pitch // 32, device)


def hot_checkpoint_bytes(rows: int, cols: int) -> int:
    return int(lib().hot_checkpoint_bytes(rows, cols))


def hot_activation_backward_workspace_bytes(rows: int, cols: int) -> int:
    return int(lib().hot_activation_backward_workspace_bytes(rows, cols))


def hot_layer_norm_backward_workspace_bytes(rows: int, cols: int) -> int:
    return int(lib().hot_layer_norm_backward_workspace_bytes(rows, cols))


def _type_of(name: str, dtype: torch.dtype) -> int:
    if dtype not in _TYPES:
        raise ValueError(f"{name}: expected torch.float32 or torch.bfloat16, not {dtype}")
    return _TYPES[dtype]


def hot_linear_forward_workspace_bytes(dtype: torch.dtype, L: int, O: int, I: int) -> int:
    return int(lib().hot_linear_forward_workspace_bytes(_type_of("dtype", dtype), L, O, I))


def _alloc(n: int, where: str, device) -> torch.Tensor:
    if n == 0:
        raise HotError(HOT_ERR_SHAPE, where)
    return torch.empty(n, dtype=torch.uint8, device=device)


def alloc_checkpoint(rows: int, cols: int, device="cuda") -> torch.Tensor:
    return _alloc(hot_checkpoint_bytes(rows, cols), "hot_checkpoint_bytes", device)


def alloc_activation_workspace(rows: int, cols: int, device="cuda") -> torch.Tensor:
    """Scratch of hot_activation_backward with g_bias."""
    return _alloc(hot_activation_backward_workspace_bytes(rows, cols), "hot_activation_backward_workspace_bytes", device)


def alloc_layer_norm_workspace(rows: int, cols: int, device="cuda") -> torch.Tensor:
    """Scratch of hot_layer_norm_backward with parameter gradients."""
    return _alloc(hot_layer_norm_backward_workspace_bytes(rows, cols), "hot_layer_norm_backward_workspace_bytes", device)


def alloc_linear_workspace(dtype: torch.dtype, L: int, O: int, I: int, device="cuda") -> Optional[torch.Tensor]:
    """Scratch of hot_linear_forward for these sizes (others may need more, smaller ones too); None where it needs none."""
    n = hot_linear_forward_workspace_bytes(dtype, L, O, I)
    if not (0 < L < 1 << 31 and 0 < O < 1 << 24 and 0 < I < 1 << 24):
        raise HotError(HOT_ERR_SHAPE, "hot_linear_forward_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def hot_checkpoint_write(x: torch.Tensor, ckpt: torch.Tensor, stream=None) -> torch.Tensor:
    """Stores x in 8 bits; returns the buffer."""
    ty, dev = _typed("x", x), _current_device()
    rows, cols = x.shape
    st = lib().hot_checkpoint_write(_expect("x", x, x.dtype, x.shape, dev), ty, rows, cols,
                                    _ckpt(ckpt, rows, cols, dev), _stream_of(stream, dev))
    if st:
        _check(st, "hot_checkpoint_write")
    return ckpt


def hot_checkpoint_read(ckpt: torch.Tensor, x: torch.Tensor, stream=None) -> torch.Tensor:
    """Fills x [rows, cols] with the values that the checkpoint of its shape holds; returns x."""
    ty, dev = _typed("x", x), _current_device()
    rows, cols = x.shape
    st = lib().hot_checkpoint_read(_ckpt(ckpt, rows, cols, dev), rows, cols,
                                   _expect("x", x, x.dtype, x.shape, dev), ty, _stream_of(stream, dev))
    if st:
        _check(st, "hot_checkpoint_read")
    return x


def hot_activation_forward(fn: int, x: torch.Tensor, y: torch.Tensor, ckpt: Optional[torch.Tensor] = None,
                           stream=None) -> torch.Tensor:
    """y = f(x), and the checkpoint of x where a buffer is given; returns y."""
    ty, dev = _typed("x", x), _current_device()
    rows, cols = x.shape
    st = lib().hot_activation_forward(int(fn), _expect("x", x, x.dtype, x.shape, dev), ty, rows, cols,
                                      _expect("y", y, x.dtype, x.shape, dev),
                                      None if ckpt is None else _ckpt(ckpt, rows, cols, dev),
                                      _stream_of(stream, dev))
    if st:
        _check(st, "hot_activation_forward")
    return y


def hot_activation_backward(fn: int, g_y: torch.Tensor, g_x: torch.Tensor, x: Optional[torch.Tensor] = None,
                            ckpt: Optional[torch.Tensor] = None, g_bias: Optional[torch.Tensor] = None,
                            ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """g_x = g_y f'(x) with x or its checkpoint, g_bias = the sum of g_x over the rows; returns g_x."""
    ty, dev = _typed("g_y", g_y), _current_device()
    rows, cols = shape = g_y.shape
    st = lib().hot_activation_backward(
        int(fn), _expect("g_y", g_y, g_y.dtype, shape, dev), ty, None if x is None else _expect("x", x, g_y.dtype, shape, dev),
        None if ckpt is None else _ckpt(ckpt, rows, cols, dev), rows, cols,
        _expect("g_x", g_x, g_y.dtype, shape, dev),
        None if g_bias is None else _expect("g_bias", g_bias, torch.float32, (cols,), dev),
        *((None, 0) if ws is None else (_bytes("ws", ws, 0, dev), ws.numel())), _stream_of(stream, dev))
    if st:
        _check(st, "hot_activation_backward")
    return g_x


def hot_layer_norm_forward(x: torch.Tensor, gamma: Optional[torch.Tensor], beta: Optional[torch.Tensor], eps: float,
                           y: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, residual: Optional[torch.Tensor] = None,
                           h: Optional[torch.Tensor] = None, ckpt: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """h = x + residual, y = layer norm of h, with its mean and rstd per row, and the checkpoint of h; returns y."""
    tx, ty, dev = _typed("x", x), _typed("y", y), _current_device()
    rows, cols = shape = x.shape
    f32 = torch.float32
    st = lib().hot_layer_norm_forward(
        _expect("x", x, x.dtype, shape, dev), tx, None if residual is None else _expect("residual", residual, x.dtype, shape, dev),
        None if gamma is None else _expect("gamma", gamma, f32, (cols,), dev),
        None if beta is None else _expect("beta", beta, f32, (cols,), dev), eps, rows, cols,
        None if h is None else _expect("h", h, x.dtype, shape, dev), _expect("y", y, y.dtype, shape, dev), ty,
        _expect("mean", mean, f32, (rows,), dev), _expect("rstd", rstd, f32, (rows,), dev),
        None if ckpt is None else _ckpt(ckpt, rows, cols, dev), _stream_of(stream, dev))
    if st:
        _check(st, "hot_layer_norm_forward")
    return y


def hot_layer_norm_backward(g_y: torch.Tensor, gamma: Optional[torch.Tensor], mean: torch.Tensor, rstd: torch.Tensor,
                            g_x: torch.Tensor, g_gamma: Optional[torch.Tensor] = None, g_beta: Optional[torch.Tensor] = None,
                            ws: Optional[torch.Tensor] = None, h: Optional[torch.Tensor] = None,
                            ckpt: Optional[torch.Tensor] = None, g_residual: Optional[torch.Tensor] = None,
                            stream=None) -> torch.Tensor:
    """Gradients of the layer norm of h (or of its checkpoint); g_residual is added to g_x; returns g_x."""
    ty, tx, dev = _typed("g_y", g_y), _typed("g_x", g_x), _current_device()
    rows, cols = shape = g_y.shape
    f32 = torch.float32
    st = lib().hot_layer_norm_backward(
        _expect("g_y", g_y, g_y.dtype, shape, dev), ty, None if h is None else _expect("h", h, g_x.dtype, shape, dev),
        None if ckpt is None else _ckpt(ckpt, rows, cols, dev), tx,
        None if gamma is None else _expect("gamma", gamma, f32, (cols,), dev),
        _expect("mean", mean, f32, (rows,), dev), _expect("rstd", rstd, f32, (rows,), dev),
        None if g_residual is None else _expect("g_residual", g_residual, g_x.dtype, shape, dev), rows, cols,
        _expect("g_x", g_x, g_x.dtype, shape, dev),
        None if g_gamma is None else _expect("g_gamma", g_gamma, f32, (cols,), dev),
        None if g_beta is None else _expect("g_beta", g_beta, f32, (cols,), dev),
        *((None, 0) if ws is None else (_bytes("ws", ws, 0, dev), ws.numel())), _stream_of(stream, dev))
    if st:
        _check(st, "hot_layer_norm_backward")
    return g_x


def hot_linear_forward(x: torch.Tensor, w: torch.Tensor, y: torch.Tensor, ws: Optional[torch.Tensor] = None,
                       bias: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None, fn: int = HOT_ACT_NONE,
                       ckpt: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """y = f(x.w^T + bias) + residual, and the checkpoint of x.w^T + bias; returns y."""
    tx, ty, dev = _typed("x", x), _typed("y", y), _current_device()
    _typed("w", w)
    (L, I), O = x.shape, w.shape[0]
    st = lib().hot_linear_forward(
        _expect("x", x, x.dtype, (L, I), dev), _expect("w", w, x.dtype, (O, I), dev), tx,
        None if bias is None else _expect("bias", bias, torch.float32, (O,), dev),
        None if residual is None else _expect("residual", residual, y.dtype, (L, O), dev), L, O, I, int(fn),
        _expect("y", y, y.dtype, (L, O), dev), ty,
        None if ckpt is None else _ckpt(ckpt, L, O, dev),
        *((None, 0) if ws is None else (_bytes("ws", ws, 0, dev), ws.numel())), _stream_of(stream, dev))
    if st:
        _check(st, "hot_linear_forward")
    return y


# ---- the operators of a fine-tuning step ------------------------------------------------------------------------------

def _opt(name: str, t: Optional[torch.Tensor], dtype: torch.dtype, shape: Tuple[int, ...], device: int) -> Optional[int]:
    return None if t is None else _expect(name, t, dtype, shape, device)


def _scratch(ws: Optional[torch.Tensor], device: int) -> Tuple[Optional[int], int]:
    return (None, 0) if ws is None else (_bytes("ws", ws, 0, device), ws.numel())


def hot_adapter_forward_workspace_bytes(dtype: torch.dtype, L: int, O: int, I: int, rank: int, adapters: int, segments: int = 0) -> int:
    return int(lib().hot_adapter_forward_workspace_bytes(_type_of("dtype", dtype), L, O, I, rank, adapters, segments))


def hot_adapter_backward_workspace_bytes(dtype: torch.dtype, L: int, O: int, I: int, rank: int, adapters: int, segments: int = 0) -> int:
    return int(lib().hot_adapter_backward_workspace_bytes(_type_of("dtype", dtype), L, O, I, rank, adapters, segments))


def _adapter_shape(x: torch.Tensor, a: torch.Tensor, b: torch.Tensor) -> Tuple[int, int, int, int, int]:
    if x.dim() != 2 or a.dim() != 3 or b.dim() != 3:
        raise ValueError("expected x [L, I], a [adapters, rank, I] and b [adapters, O, rank]")
    (L, I), (K, rank, _), O = x.shape, a.shape, b.shape[1]
    return L, O, I, rank, K


def alloc_adapter_workspace(x: torch.Tensor, a: torch.Tensor, b: torch.Tensor, segments: int = 0, backward: bool = True) -> torch.Tensor:
    """Scratch of hot_adapter_forward and, with `backward`, of hot_adapter_backward for tensors of these shapes."""
    L, O, I, rank, K = _adapter_shape(x, a, b)
    sizes = (x.dtype, L, O, I, rank, K, segments)
    n = hot_adapter_forward_workspace_bytes(*sizes)
    if n and backward:
        n = max(n, hot_adapter_backward_workspace_bytes(*sizes))
    return _alloc(n, "hot_adapter_forward_workspace_bytes", x.device)


def _batch(offsets: Optional[torch.Tensor], index: Optional[torch.Tensor], device: int):
    if offsets is None and index is None:
        return None, None, 0
    if offsets is None or index is None or index.dim() != 1 or not index.shape[0]:
        raise ValueError("offsets, index: expected both, of segments + 1 and segments int32 numbers, or neither")
    n = index.shape[0]
    return _expect("offsets", offsets, torch.int32, (n + 1,), device), _expect("index", index, torch.int32, (n,), device), n


def hot_adapter_forward(x: torch.Tensor, a: torch.Tensor, b: torch.Tensor, y: torch.Tensor, ws: torch.Tensor,
                        scale: Optional[torch.Tensor] = None, offsets: Optional[torch.Tensor] = None,
                        index: Optional[torch.Tensor] = None, base: Optional[torch.Tensor] = None,
                        u: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """y = base + scale_k (x.A_k^T).B_k^T with the adapter k of each row's request; u = x.A_k^T where a tensor is given; returns y."""
    ty, dev = _typed("x", x), _current_device()
    L, O, I, rank, K = _adapter_shape(x, a, b)
    t, f32 = x.dtype, torch.float32
    at, ix, n = _batch(offsets, index, dev)
    st = lib().hot_adapter_forward(
        _expect("x", x, t, (L, I), dev), _expect("a", a, t, (K, rank, I), dev), _expect("b", b, t, (K, O, rank), dev), ty,
        _opt("scale", scale, f32, (K,), dev), at, ix, n, K, L, O, I, rank, _opt("base", base, t, (L, O), dev),
        _expect("y", y, t, (L, O), dev), _opt("u", u, f32, (L, rank), dev), *_scratch(ws, dev), _stream_of(stream, dev))
    if st:
        _check(st, "hot_adapter_forward")
    return y


def hot_adapter_backward(g_y: torch.Tensor, x: torch.Tensor, u: Optional[torch.Tensor], a: torch.Tensor, b: torch.Tensor,
                         ws: torch.Tensor, g_x: Optional[torch.Tensor] = None, g_a: Optional[torch.Tensor] = None,
                         g_b: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                         offsets: Optional[torch.Tensor] = None, index: Optional[torch.Tensor] = None,
                         g_base: Optional[torch.Tensor] = None, stream=None) -> None:
    """g_x = g_base + g_u.A_k with g_u = scale_k g_y.B_k, and fp32 g_a and g_b of each adapter, of those that are given."""
    ty, dev = _typed("x", x), _current_device()
    L, O, I, rank, K = _adapter_shape(x, a, b)
    t, f32 = x.dtype, torch.float32
    at, ix, n = _batch(offsets, index, dev)
    st = lib().hot_adapter_backward(
        _expect("g_y", g_y, t, (L, O), dev), _expect("x", x, t, (L, I), dev), _opt("u", u, f32, (L, rank), dev),
        _expect("a", a, t, (K, rank, I), dev), _expect("b", b, t, (K, O, rank), dev), ty, _opt("scale", scale, f32, (K,), dev), at, ix, n,
        K, L, O, I, rank, _opt("g_base", g_base, t, (L, I), dev), _opt("g_x", g_x, t, (L, I), dev),
        _opt("g_a", g_a, f32, (K, rank, I), dev), _opt("g_b", g_b, f32, (K, O, rank), dev), *_scratch(ws, dev), _stream_of(stream, dev))
    if st:
        _check(st, "hot_adapter_backward")


def hot_token_logprobs_workspace_bytes(dtype: torch.dtype, rows: int, vocab: int, top: int = 0) -> int:
    return int(lib().hot_token_logprobs_workspace_bytes(_type_of("dtype", dtype), rows, vocab, top))


def alloc_logprobs_workspace(logits: torch.Tensor, top: int = 0) -> Optional[torch.Tensor]:
    """Scratch of hot_token_logprobs for logits of this shape (fewer rows may need more); None where it needs none."""
    rows, vocab = logits.shape
    n = hot_token_logprobs_workspace_bytes(logits.dtype, rows, vocab, top)
    if not (0 < rows < 1 << 31 and 0 < vocab < 1 << 24 and 0 <= top <= min(vocab, HOT_MAX_TOP)):
        raise HotError(HOT_ERR_SHAPE, "hot_token_logprobs_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=logits.device) if n else None


def hot_token_logprobs(logits: torch.Tensor, targets: Optional[torch.Tensor], logp: Optional[torch.Tensor],
                       ws: Optional[torch.Tensor] = None, entropy: Optional[torch.Tensor] = None,
                       stats: Optional[torch.Tensor] = None, top_logp: Optional[torch.Tensor] = None,
                       top_ids: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
    """logp[row] = log softmax(logits[row])[targets[row]] (0 where the target is no token), and what else is given; returns logp."""
    ty, dev = _typed("logits", logits), _current_device()
    rows, vocab = shape = logits.shape
    f32 = torch.float32
    top = 0
    if top_logp is not None or top_ids is not None:
        if top_logp is None or top_ids is None or top_logp.dim() != 2:
            raise ValueError("top_logp, top_ids: expected both, of shape [rows, top], or neither")
        top = top_logp.shape[1]
    st = lib().hot_token_logprobs(
        _expect("logits", logits, logits.dtype, shape, dev), ty, rows, vocab, _opt("targets", targets, torch.int64, (rows,), dev),
        _opt("logp", logp, f32, (rows,), dev), _opt("entropy", entropy, f32, (rows,), dev), _opt("stats", stats, f32, (rows, 2), dev), top,
        _opt("top_logp", top_logp, f32, (rows, top), dev), _opt("top_ids", top_ids, torch.int32, (rows, top), dev),
        *_scratch(ws, dev), _stream_of(stream, dev))
    if st:
        _check(st, "hot_token_logprobs")
    return logp


def hot_token_logprobs_backward(logits: torch.Tensor, targets: Optional[torch.Tensor], stats: torch.Tensor, g_logits: torch.Tensor,
                                g_logp: Optional[torch.Tensor] = None, entropy: Optional[torch.Tensor] = None,
                                g_entropy: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Gradient of the logits (g_logits may be logits) from those of logp and of the entropy; returns g_logits."""
    ty, dev = _typed("logits", logits), _current_device()
    rows, vocab = shape = logits.shape
    f32 = torch.float32
    st = lib().hot_token_logprobs_backward(
        _expect("logits", logits, logits.dtype, shape, dev), ty, rows, vocab, _opt("targets", targets, torch.int64, (rows,), dev),
        _expect("stats", stats, f32, (rows, 2), dev), _opt("entropy", entropy, f32, (rows,), dev), _opt("g_logp", g_logp, f32, (rows,), dev),
        _opt("g_entropy", g_entropy, f32, (rows,), dev), _expect("g_logits", g_logits, logits.dtype, shape, dev), _stream_of(stream, dev))
    if st:
        _check(st, "hot_token_logprobs_backward")
    return g_logits


_STATES = {"f32": HOT_STATE_F32, "8bit": HOT_STATE_8BIT}
_MOMENTS = {"m": HOT_MOMENT_M, "v": HOT_MOMENT_V}


def hot_adamw_state_bytes(state: str, n: int) -> int:
    return int(lib().hot_adamw_state_bytes(_STATES[state], n))


def alloc_adamw_state(state: str, n: int, device="cuda") -> torch.Tensor:
    """One moment of n elements at the first step (all zeros): float32 [n], or the bytes of the 8-bit form."""
    size = hot_adamw_state_bytes(state, n)
    if size == 0:
        raise HotError(HOT_ERR_SHAPE, "hot_adamw_state_bytes")
    return torch.zeros(n, dtype=torch.float32, device=device) if state == "f32" else torch.zeros(size, dtype=torch.uint8, device=device)


def _flat(name: str, t: torch.Tensor) -> int:
    ty = _TYPES.get(t.dtype)
    if ty is None or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous float32 or bfloat16 device tensor")
    return ty


def hot_adamw_state_read(buf: torch.Tensor, moment: str, x: torch.Tensor, stream=None) -> torch.Tensor:
    """Fills x with the values that an 8-bit moment ("m" or "v") of as many elements holds; returns x."""
    ty, dev, n = _flat("x", x), _current_device(), x.numel()
    st = lib().hot_adamw_state_read(_bytes("buf", buf, hot_adamw_state_bytes("8bit", n), dev), _MOMENTS[moment], n,
                                    _expect("x", x, x.dtype, x.shape, dev), ty, _stream_of(stream, dev))
    if st:
        _check(st, "hot_adamw_state_read")
    return x


def hot_adamw_state_write(x: torch.Tensor, moment: str, buf: torch.Tensor, stream=None) -> torch.Tensor:
    """Stores x as an 8-bit moment, rounded to the nearest; returns buf."""
    ty, dev, n = _flat("x", x), _current_device(), x.numel()
    st = lib().hot_adamw_state_write(_expect("x", x, x.dtype, x.shape, dev), ty, _MOMENTS[moment], n,
                                     _bytes("buf", buf, hot_adamw_state_bytes("8bit", n), dev), _stream_of(stream, dev))
    if st:
        _check(st, "hot_adamw_state_write")
    return buf


class AdamWTensors:
    """The tensors of an optimiser step: a list of dicts with param, grad, m and v, and where wanted copy (bfloat16), param_out, m_out,
    v_out (in place without), weight_decay and lr_factor.  Checked once, and held as long as this object lives: zero or write the gradients
    where they are (gradients allocated anew need another object, some microseconds a tensor)."""

    def __init__(self, tensors: Sequence[dict], state: str = "f32"):
        form = _STATES[state]
        self.tensors = [dict(t) for t in tensors]
        self.state, self.device = state, -1
        count = len(self.tensors)
        entries = (hot_adamw_tensor * max(count, 1))()

        def address(name: str, i: int, x: torch.Tensor, dtype: torch.dtype, n: int) -> int:
            if x.numel() != n or x.dtype is not dtype or x.get_device() != self.device or not x.is_contiguous():
                raise ValueError(f"{name} of tensor {i}: expected {n} contiguous {dtype} elements on cuda:{self.device}")
            return x.data_ptr()

        for i, t in enumerate(self.tensors):
            p, g, e, get = t["param"], t["grad"], entries[i], t.get
            n, dev = p.numel(), p.get_device()
            e.param_type, e.grad_type = _flat(f"param of tensor {i}", p), _flat(f"grad of tensor {i}", g)
            if self.device not in (-1, dev):
                raise ValueError(f"tensor {i}: on cuda:{dev}, others on cuda:{self.device}")
            self.device = dev
            e.n, e.weight_decay, e.lr_factor = n, get("weight_decay", 0.0), get("lr_factor", 1.0)
            e.param, e.grad = p.data_ptr(), address("grad", i, g, g.dtype, n)
            x = get("param_out")
            if x is not None:
                e.param_out = address("param_out", i, x, p.dtype, n)
            x = get("copy")
            if x is not None:
                e.copy = address("copy", i, x, torch.bfloat16, n)
            for name in ("m", "v", "m_out", "v_out"):
                x = get(name)
                if x is None:
                    continue
                if form == HOT_STATE_F32:
                    setattr(e, name, address(name, i, x, torch.float32, n))
                else:      # blocks of 1024 codes and 32 exponents
                    setattr(e, name, _bytes(f"{name} of tensor {i}", x, (n + 1023) // 1024 * 1056, dev))
        size = int(lib().hot_adamw_table_bytes(count))
        self.table = (C.c_uint64 * max((size + 7) // 8, 1))()
        _check(lib().hot_adamw_table(entries, count, form, self.table, size), "hot_adamw_table")


def hot_adamw_step(tensors: AdamWTensors, lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, step: int = 1,
                   rounding: int = HOT_ROUND_DRAWN, dynamic: Optional[torch.Tensor] = None, stream=None) -> None:
    """One AdamW step over the tensors.  dynamic: float32 [4] on the device, lr, 1 - beta1^step, 1 - beta2^step and a factor of every
    gradient, in place of lr and step (for recorded calls); [5] with a number that no two steps share (the step, say), which goes
    into the rounding of 8-bit moments where the first three no longer change."""
    dev = _current_device()
    if tensors.device != dev:
        raise ValueError(f"tensors: expected on cuda:{dev}, the current device")
    count = 5 if dynamic is not None and tuple(dynamic.shape) == (5,) else 4
    cfg = hot_adamw_config(float(lr), float(beta1), float(beta2), float(eps), int(step), int(rounding), count,
                           _opt("dynamic", dynamic, torch.float32, (count,), dev))
    st = lib().hot_adamw_step(tensors.table, C.byref(cfg), _stream_of(stream, dev))
    if st:
        _check(st, "hot_adamw_step")


def hot_debug_unpack_activation(cfg: Config, act_buf: torch.Tensor, L: int, I: int, stream=None):
    """Returns (codes int8 [L*r/n, I], scale float32 [1]) on the device; with gw_bits = 16
    the codes are bfloat16 bit patterns (int16) and the scale is 1."""
    Lr = cfg.reduced_tokens(L)
    codes = torch.empty((Lr, I), dtype=torch.int16 if cfg.gw_bits == 16 else torch.int8,
                        device=act_buf.device)
    scale = torch.empty(1, dtype=torch.float32, device=act_buf.device)
    st = lib().hot_debug_unpack_activation(C.byref(cfg.c()), _ptr(act_buf), L, I, _ptr(codes),
                                           _ptr(scale), _stream(stream))
    _check(st, "hot_debug_unpack_activation")
    return codes, scale


def hot_debug_gx_operands(cfg: Config, ws: torch.Tensor, L: int, O: int, I: int, gy_quantizer: int,
                          want_acc: bool = True, stream=None):
    """Returns dict(qg [L,O] int8, sg [L]|[1], qw [O,I] int8, sw [1], acc [L,I] int32)."""
    dev = ws.device
    qg = torch.empty((L, O), dtype=torch.int8, device=dev)
    sg = torch.empty(L if gy_quantizer == HOT_Q_PER_TOKEN else 1, dtype=torch.float32, device=dev)
    qw = torch.empty((O, I), dtype=torch.int8, device=dev)
    sw = torch.empty(1, dtype=torch.float32, device=dev)
    acc = torch.empty((L, I), dtype=torch.int32, device=dev) if want_acc else None
    st = lib().hot_debug_gx_operands(C.byref(cfg.c()), _ptr(ws), L, O, I, int(gy_quantizer),
                                     _ptr(qg), _ptr(sg), _ptr(qw), _ptr(sw), _ptr(acc),
                                     _stream(stream))
    _check(st, "hot_debug_gx_operands")
    return dict(qg=qg, sg=sg, qw=qw, sw=sw, acc=acc)


def hot_debug_gw_operands(cfg: Config, ws: torch.Tensor, act_buf: torch.Tensor, L: int, O: int,
                          I: int, want_acc: bool = True, stream=None):
    """Returns dict(qg [L*r/n,O] int8, sg [1], acc [O,I] int32); with gw_bits = 16 qg holds
    bfloat16 bit patterns (int16) and acc the fp32 accumulators (float32)."""
    dev = ws.device
    Lr = cfg.reduced_tokens(L)
    qg = torch.empty((Lr, O), dtype=torch.int16 if cfg.gw_bits == 16 else torch.int8, device=dev)
    sg = torch.empty(1, dtype=torch.float32, device=dev)
    acc = torch.empty((O, I), dtype=torch.int32, device=dev) if want_acc else None
    st = lib().hot_debug_gw_operands(C.byref(cfg.c()), _ptr(ws), _ptr(act_buf), L, O, I, _ptr(qg),
                                     _ptr(sg), _ptr(acc), _stream(stream))
    _check(st, "hot_debug_gw_operands")
    if acc is not None and cfg.gw_bits == 16:
        acc = acc.view(torch.float32)
    return dict(qg=qg, sg=sg, acc=acc)


def hot_debug_fused_operands(cfg: Config, ws: torch.Tensor, act_buf: torch.Tensor, L: int, O: int,
                             I: int, gy_quantizer: int, want_acc: bool = True, stream=None):
    """Operands of the last hot_linear_backward: dict(qg, sg, qw, sw, acc_gx, qgh, sgh, acc_gw)."""
    dev = ws.device
    Lr = cfg.reduced_tokens(L)
    qg = torch.empty((L, O), dtype=torch.int8, device=dev)
    sg = torch.empty(L if gy_quantizer == HOT_Q_PER_TOKEN else 1, dtype=torch.float32, device=dev)
    qw = torch.empty((O, I), dtype=torch.int8, device=dev)
    sw = torch.empty(1, dtype=torch.float32, device=dev)
    qgh = torch.empty((Lr, O), dtype=torch.int8, device=dev)
    sgh = torch.empty(1, dtype=torch.float32, device=dev)
    acc_gx = torch.empty((L, I), dtype=torch.int32, device=dev) if want_acc else None
    acc_gw = torch.empty((O, I), dtype=torch.int32, device=dev) if want_acc else None
    st = lib().hot_debug_fused_operands(C.byref(cfg.c()), _ptr(ws), _ptr(act_buf), L, O, I,
                                        int(gy_quantizer), _ptr(qg), _ptr(sg), _ptr(qw), _ptr(sw),
                                        _ptr(acc_gx), _ptr(qgh), _ptr(sgh), _ptr(acc_gw),
                                        _stream(stream))
    _check(st, "hot_debug_fused_operands")
    return dict(qg=qg, sg=sg, qw=qw, sw=sw, acc_gx=acc_gx, qgh=qgh, sgh=sgh, acc_gw=acc_gw)


def hot_debug_set_backward_strategy(strategy: int) -> None:
    """0 = library's choice, 1 = separate paths, 2 = shared g_y passes where they exist."""
    _check(lib().hot_debug_set_backward_strategy(int(strategy)), "hot_debug_set_backward_strategy")


def hot_debug_set_gemm_mode(mode: int) -> None:
    """0: library's choice, 1: one workgroup per output tile, s >= 2: s K slices where a split applies."""
    _check(lib().hot_debug_set_gemm_mode(int(mode)), "hot_debug_set_gemm_mode")


def hot_debug_set_exchange_wait_us(us: int) -> None:
    _check(lib().hot_debug_set_exchange_wait_us(int(us)), "hot_debug_set_exchange_wait_us")


def hot_debug_profile_begin() -> None:
    _check(lib().hot_debug_profile_begin(), "hot_debug_profile_begin")


def hot_debug_profile_end():
    """Returns {stage name: (total ms, launches)} for the stages that ran."""
    ms = (C.c_float * HOT_NUM_STAGES_ALL)()
    cnt = (C.c_int64 * HOT_NUM_STAGES_ALL)()
    _check(lib().hot_debug_profile_end_all(ms, cnt, HOT_NUM_STAGES_ALL), "hot_debug_profile_end_all")
    return {lib().hot_debug_stage_name(i).decode(): (float(ms[i]), int(cnt[i]))
            for i in range(HOT_NUM_STAGES_ALL) if cnt[i]}


def hot_debug_profile_sequence():
    """Stage names of the recording closed by the last hot_debug_profile_end, in launch order."""
    n = int(lib().hot_debug_profile_sequence(None, 0))
    buf = (C.c_int32 * max(n, 1))()
    lib().hot_debug_profile_sequence(buf, n)
    return [lib().hot_debug_stage_name(int(buf[i])).decode() for i in range(n)]


def hot_debug_gemm_plan(cfg: Config, L: int, O: int, I: int) -> dict:
    """{one_launch: bool, gx / gw / gx_alone / gw_alone: (tile rows, tile columns, K slices, added by a second kernel),
    streams: which of the four store their output with the streaming hint}."""
    p = hot_gemm_plan()
    _check(lib().hot_debug_gemm_plan(C.byref(cfg.c()), L, O, I, C.byref(p)), "hot_debug_gemm_plan")
    names = ("gx", "gw", "gx_alone", "gw_alone")
    return dict(one_launch=bool(p.one_launch), streams={f for f in names if getattr(p, f)[4]},
                **{f: (*list(getattr(p, f))[:3], bool(getattr(p, f)[3])) for f in names})


def hot_debug_linear_plan(dtype: torch.dtype, L: int, O: int, I: int, y_dtype: Optional[torch.dtype] = None, ckpt: bool = False) -> dict:
    """How hot_linear_forward works on a product: its way ("rows", "direct", "tiles", "packed"), rows and outputs a workgroup, tiles, tiles
    with a workgroup each, slices of the others, whether row ends are masked, whether y is streamed."""
    p = hot_linear_plan()
    _check(lib().hot_debug_linear_plan(_type_of("dtype", dtype), _type_of("y_dtype", y_dtype or dtype), L, O, I, int(ckpt), C.byref(p)), "hot_debug_linear_plan")
    return dict(way=("rows", "direct", "tiles", "packed")[p.way], tile=(p.tile_rows, p.tile_cols), tiles=p.tiles, whole=p.whole,
                slices=p.slices, masked=bool(p.masked), streams=bool(p.streams))


def hot_debug_probe(kind: int, buf: torch.Tensor, iters: int = 1, stream=None) -> None:
    _check(lib().hot_debug_probe(int(kind), _ptr(buf), buf.numel() * buf.element_size(), int(iters),
                                 _stream(stream)), "hot_debug_probe")
