"""Python binding of liboctree_nca.so, the MI355X (gfx950) OctreeNCA inference
library (arXiv 2508.06993).

Argument marshalling only: every function here checks and converts its
arguments, then calls the C entry point of the same name (include/octree_nca.h).
All arithmetic runs in the library's HIP kernels.  PyTorch supplies device
memory and the current stream.  There is no CPU fallback: if the library is
missing, every call raises ``OctreeNCAError``.
"""
from __future__ import annotations

import ctypes
import functools
import os
from dataclasses import dataclass
from typing import Optional, Sequence

import numpy as np
import torch

from .build import LIB_PATH

__all__ = [
    "OctreeNCAError", "Model", "lib", "library_path", "level_weights_struct",
    "octree_nca_build_pyramid", "octree_nca_upsample", "octree_nca_run_level",
    "octree_nca_readout", "octree_nca_readout_classes", "octree_nca_workspace_bytes",
    "octree_nca_infer", "octree_nca_infer_batch", "octree_nca_infer_launches",
    "octree_nca_infer_static", "OCTNCA_STATIC_SCRATCH_BYTES",
    "octree_nca_first_level_steps",
    "octree_nca_fire_mask", "octree_nca_strerror", "octree_nca_abi_version",
    "octree_nca_step_backward_workspace_bytes", "octree_nca_step_backward",
    "octree_nca_upsample_backward", "octree_nca_readout_mse_workspace_bytes",
    "octree_nca_readout_mse", "octree_nca_train_workspace_bytes", "octree_nca_train_step",
    "level_grads_struct", "check_train_weights", "StateCacheBuffers", "state_cache_refs",
    "octree_nca_state_cache_write", "octree_nca_state_cache_read", "param_structs",
    "octree_nca_param_table_bytes", "octree_nca_param_table", "octree_nca_grad_norm",
    "octree_nca_clip_grads", "octree_nca_adamw", "octree_nca_train_kept_workspace_bytes",
    "octree_nca_train_step_kept", "MX4Buffers", "mx4_shapes", "octree_nca_mx4_code_bytes",
    "octree_nca_mx4_quantise", "octree_nca_mx4_dequantise", "octree_nca_mx4_product",
    "octree_nca_mx4_linear", "octree_nca_mx4_backward_workspace_bytes", "octree_nca_mx4_backward",
    "octree_nca_dropout", "CODE_NAMES", "OCTNCA_BF16", "OCTNCA_CODE_I8", "OCTNCA_CODE_F8",
    "EXPORTED_SYMBOLS", "OCTNCA_OK", "OCTNCA_EINVAL",
    "OCTNCA_EUNSUPPORTED", "OCTNCA_ESHAPE",
    "OCTNCA_EHIP", "OCTNCA_ESPACE", "OCTNCA_F32", "OCTNCA_F16", "KERNEL_NAMES", "kernel_fields",
]

OCTNCA_OK, OCTNCA_EINVAL, OCTNCA_EUNSUPPORTED, OCTNCA_ESHAPE, OCTNCA_EHIP, OCTNCA_ESPACE = \
    0, -1, -2, -3, -4, -5
OCTNCA_F32, OCTNCA_F16, OCTNCA_BF16 = 0, 1, 2
OCTNCA_CODE_I8, OCTNCA_CODE_F8 = 0, 1
CODE_NAMES = {"i8": OCTNCA_CODE_I8, "f8": OCTNCA_CODE_F8}   # formats of a state cache
(OCTNCA_MLP_AUTO, OCTNCA_MLP_F32, OCTNCA_MLP_BF16X3, OCTNCA_MLP_F16, OCTNCA_MLP_F16S,
 OCTNCA_MLP_VALU) = range(6)
OCTNCA_LAYOUT_AUTO, OCTNCA_LAYOUT_ROWS, OCTNCA_LAYOUT_TILES = range(3)
OCTNCA_STATIC_SCRATCH_BYTES = 64 << 20   # octree_nca_infer_static's device array

# Step-kernel names accepted by Model(kernel=...): a comma-separated list of
# these, each setting one field of the C model description (octnca_model).
KERNEL_NAMES = {
    "mfma": {},                                   # the library's default
    "mfma_f32": {"mlp": OCTNCA_MLP_F32},
    "mfma_bf16x3": {"mlp": OCTNCA_MLP_BF16X3},
    "mfma_f16": {"mlp": OCTNCA_MLP_F16},
    "mfma_f16s": {"mlp": OCTNCA_MLP_F16S},
    "valu": {"mlp": OCTNCA_MLP_VALU},
    "mfma_rows": {"layout2d": OCTNCA_LAYOUT_ROWS},
    "mfma_tiles": {"layout2d": OCTNCA_LAYOUT_TILES},
    "mfma_1step": {"steps_per_launch": 1},
}


def kernel_fields(kernel: str) -> dict:
    """octnca_model step-kernel fields (mlp, layout2d, steps_per_launch) of a
    name such as "mfma_rows,mfma_1step"."""
    out = {"mlp": OCTNCA_MLP_AUTO, "layout2d": OCTNCA_LAYOUT_AUTO, "steps_per_launch": 0}
    for name in kernel.split(","):
        if name not in KERNEL_NAMES:
            raise ValueError(f"unknown step kernel {name!r}; known: {sorted(KERNEL_NAMES)}")
        out.update(KERNEL_NAMES[name])
    return out

EXPORTED_SYMBOLS = (
    "octree_nca_build_pyramid", "octree_nca_upsample", "octree_nca_run_level",
    "octree_nca_readout", "octree_nca_readout_classes", "octree_nca_workspace_bytes",
    "octree_nca_infer", "octree_nca_infer_batch", "octree_nca_infer_launches",
    "octree_nca_infer_static",
    "octree_nca_first_level_steps",
    "octree_nca_fire_mask", "octree_nca_strerror", "octree_nca_abi_version",
    "octree_nca_step_backward_workspace_bytes", "octree_nca_step_backward",
    "octree_nca_upsample_backward", "octree_nca_readout_mse_workspace_bytes",
    "octree_nca_readout_mse", "octree_nca_train_workspace_bytes", "octree_nca_train_step",
    "octree_nca_state_cache_write", "octree_nca_state_cache_read",
    "octree_nca_param_table_bytes", "octree_nca_param_table", "octree_nca_grad_norm",
    "octree_nca_clip_grads", "octree_nca_adamw", "octree_nca_train_kept_workspace_bytes",
    "octree_nca_train_step_kept", "octree_nca_mx4_code_bytes", "octree_nca_mx4_quantise",
    "octree_nca_mx4_dequantise", "octree_nca_mx4_product", "octree_nca_mx4_linear",
    "octree_nca_mx4_backward_workspace_bytes", "octree_nca_mx4_backward", "octree_nca_dropout",
)


class OctreeNCAError(RuntimeError):
    def __init__(self, msg, status=None):
        super().__init__(msg)
        self.status = status


class _Model(ctypes.Structure):
    _fields_ = [("ndim", ctypes.c_int32), ("channels", ctypes.c_int32),
                ("hidden", ctypes.c_int32), ("n_in", ctypes.c_int32),
                ("state_dtype", ctypes.c_int32), ("mlp", ctypes.c_int32),
                ("layout2d", ctypes.c_int32), ("steps_per_launch", ctypes.c_int32)]


class _Extent(ctypes.Structure):
    _fields_ = [("d", ctypes.c_int64), ("h", ctypes.c_int64), ("w", ctypes.c_int64)]


class _LevelWeights(ctypes.Structure):
    _fields_ = [("conv_w", ctypes.c_void_p), ("conv_b", ctypes.c_void_p),
                ("w1", ctypes.c_void_p), ("b1", ctypes.c_void_p), ("w2", ctypes.c_void_p)]


class _LevelGrads(ctypes.Structure):
    _fields_ = [("conv_w", ctypes.c_void_p), ("conv_b", ctypes.c_void_p),
                ("w1", ctypes.c_void_p), ("b1", ctypes.c_void_p), ("w2", ctypes.c_void_p)]


class _StateCache(ctypes.Structure):
    _fields_ = [("code", ctypes.c_int32), ("block", ctypes.c_int32), ("slots", ctypes.c_int64),
                ("cells", ctypes.c_int64), ("codes", ctypes.c_void_p),
                ("scales", ctypes.c_void_p)]


class _Keep(ctypes.Structure):
    _fields_ = [("code", ctypes.c_int32), ("block", ctypes.c_int32)]


class _Param(ctypes.Structure):
    _fields_ = [("count", ctypes.c_int64), ("grad", ctypes.c_void_p),
                ("clipped", ctypes.c_void_p), ("param", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("ema", ctypes.c_void_p), ("grad_dtype", ctypes.c_int32),
                ("clipped_dtype", ctypes.c_int32)]


class _ParamList(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("chunks", ctypes.c_int64),
                ("elements", ctypes.c_int64), ("bytes", ctypes.c_int64),
                ("has", ctypes.c_int32)]


class _AdamW(ctypes.Structure):
    _fields_ = [(k, ctypes.c_double) for k in
                ("lr", "beta1", "beta2", "eps", "weight_decay", "max_norm", "scale", "ema_decay")]


class _Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("stride", ctypes.c_int64), ("dtype", ctypes.c_int32)]


class _MX4(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("codes", ctypes.c_void_p),
                ("scales", ctypes.c_void_p)]
    device = None    # its memory's; None: not known


class _Dropout(ctypes.Structure):
    _fields_ = [("rate", ctypes.c_float), ("seed", ctypes.c_uint64), ("index", ctypes.c_uint64),
                ("step", ctypes.c_void_p)]


_P = ctypes.c_void_p
_I32 = ctypes.c_int32
_I64 = ctypes.c_int64
_SIGS = {
    "octree_nca_build_pyramid": (_I32, [ctypes.POINTER(_Model), _P, _Extent, _I32,
                                        ctypes.POINTER(_I32), ctypes.POINTER(_P), _P]),
    "octree_nca_upsample": (_I32, [ctypes.POINTER(_Model), _P, _Extent, ctypes.POINTER(_I32),
                                   _P, _P, _P]),
    "octree_nca_run_level": (_I32, [ctypes.POINTER(_Model), _P, _P, _Extent,
                                    ctypes.POINTER(_LevelWeights), _I32, _I32, ctypes.c_float,
                                    ctypes.c_uint64, ctypes.POINTER(_I32), _P]),
    "octree_nca_readout": (_I32, [ctypes.POINTER(_Model), _P, _Extent, _P, _P]),
    "octree_nca_readout_classes": (_I32, [ctypes.POINTER(_Model), _P, _Extent, _I32, _P, _P]),
    "octree_nca_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(_Model), _Extent, _I32,
                                                     ctypes.POINTER(_I32), _I32]),
    "octree_nca_infer_launches": (_I32, [ctypes.POINTER(_Model), _Extent, _I32,
                                         ctypes.POINTER(_I32), ctypes.POINTER(_I32),
                                         ctypes.POINTER(_I32)]),
    "octree_nca_infer": (_I32, [ctypes.POINTER(_Model), _P, _Extent, _I32, ctypes.POINTER(_I32),
                                ctypes.POINTER(_LevelWeights), ctypes.POINTER(_I32),
                                ctypes.c_float, ctypes.c_uint64, _P, ctypes.c_size_t, _P, _P,
                                ctypes.POINTER(_P), _P]),
    "octree_nca_infer_static": (_I32, [ctypes.POINTER(_Model), _P, _Extent, _I32,
                                       ctypes.POINTER(_I32), ctypes.POINTER(_LevelWeights),
                                       ctypes.POINTER(_I32), ctypes.c_float, ctypes.c_uint64, _P,
                                       _P, _P]),
    "octree_nca_infer_batch": (_I32, [ctypes.POINTER(_Model), _P, _I32, _Extent, _I32,
                                      ctypes.POINTER(_I32), ctypes.POINTER(_LevelWeights),
                                      ctypes.POINTER(_I32), ctypes.c_float, ctypes.c_uint64, _P,
                                      ctypes.c_size_t, _P, _P, _P]),
    "octree_nca_fire_mask": (_I32, [ctypes.c_uint64, _I32, _I32, _Extent, ctypes.c_float, _P,
                                    _P]),
    "octree_nca_first_level_steps": (_I32, [ctypes.c_float, _Extent]),
    "octree_nca_step_backward_workspace_bytes": (ctypes.c_size_t,
                                                 [ctypes.POINTER(_Model), _Extent]),
    "octree_nca_step_backward": (_I32, [ctypes.POINTER(_Model), _P, _P, _Extent,
                                        ctypes.POINTER(_LevelWeights), _I32, _I32,
                                        ctypes.c_float, ctypes.c_uint64, _P,
                                        ctypes.POINTER(_LevelGrads), _P, ctypes.c_size_t, _P]),
    "octree_nca_upsample_backward": (_I32, [ctypes.POINTER(_Model), _P, _Extent,
                                            ctypes.POINTER(_I32), _P, _P]),
    "octree_nca_readout_mse_workspace_bytes": (ctypes.c_size_t, [_Extent]),
    "octree_nca_readout_mse": (_I32, [ctypes.POINTER(_Model), _P, _P, _Extent, _P, _P, _P,
                                      ctypes.c_size_t, _P]),
    "octree_nca_train_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(_Model), _Extent, _I32,
                                                           ctypes.POINTER(_I32),
                                                           ctypes.POINTER(_I32)]),
    "octree_nca_train_step": (_I32, [ctypes.POINTER(_Model), _P, _Extent, _I32,
                                     ctypes.POINTER(_I32), ctypes.POINTER(_LevelWeights),
                                     ctypes.POINTER(_I32), ctypes.c_float, ctypes.c_uint64, _P,
                                     _P, ctypes.c_size_t, ctypes.POINTER(_LevelGrads), _P, _P,
                                     _P]),
    "octree_nca_state_cache_write": (_I32, [ctypes.POINTER(_Model), ctypes.POINTER(_StateCache),
                                            _P, _I64, _I64, _I32, _P, _I64, _P]),
    "octree_nca_state_cache_read": (_I32, [ctypes.POINTER(_Model), ctypes.POINTER(_StateCache),
                                           _P, _I64, _I64, _I32, _P, _I64, _P]),
    "octree_nca_train_kept_workspace_bytes": (ctypes.c_size_t,
                                              [ctypes.POINTER(_Model), _Extent, _I32,
                                               ctypes.POINTER(_I32), ctypes.POINTER(_I32),
                                               ctypes.POINTER(_Keep)]),
    "octree_nca_train_step_kept": (_I32, [ctypes.POINTER(_Model), _P, _Extent, _I32,
                                          ctypes.POINTER(_I32), ctypes.POINTER(_LevelWeights),
                                          ctypes.POINTER(_I32), ctypes.c_float, ctypes.c_uint64,
                                          _P, ctypes.POINTER(_Keep), _P, ctypes.c_size_t,
                                          ctypes.POINTER(_LevelGrads), _P, _P, _P]),
    "octree_nca_param_table_bytes": (ctypes.c_size_t, [ctypes.POINTER(_Param), _I32]),
    "octree_nca_param_table": (_I32, [ctypes.POINTER(_Param), _I32, _P, ctypes.c_size_t,
                                      ctypes.POINTER(_ParamList), _P]),
    "octree_nca_grad_norm": (_I32, [ctypes.POINTER(_ParamList), ctypes.c_float, _P, _P]),
    "octree_nca_clip_grads": (_I32, [ctypes.POINTER(_ParamList), ctypes.c_float, ctypes.c_float,
                                     _P, _P]),
    "octree_nca_adamw": (_I32, [ctypes.POINTER(_ParamList), ctypes.POINTER(_AdamW), _P, _P, _P]),
    "octree_nca_mx4_code_bytes": (ctypes.c_size_t, [_I64, _I64]),
    "octree_nca_mx4_quantise": (_I32, [ctypes.POINTER(_Rows), ctypes.POINTER(_MX4), _P]),
    "octree_nca_mx4_dequantise": (_I32, [ctypes.POINTER(_MX4), ctypes.POINTER(_Rows), _P]),
    "octree_nca_mx4_product": (_I32, [ctypes.POINTER(_MX4), ctypes.POINTER(_MX4), _P, _I32,
                                      ctypes.POINTER(_Rows), _P]),
    "octree_nca_mx4_linear": (_I32, [ctypes.POINTER(_Rows), ctypes.POINTER(_MX4),
                                     ctypes.POINTER(_MX4), _P, _I32, ctypes.POINTER(_Rows), _P]),
    "octree_nca_mx4_backward_workspace_bytes": (ctypes.c_size_t, [_I64, _I64, _I64]),
    "octree_nca_mx4_backward": (_I32, [ctypes.POINTER(_Rows), ctypes.POINTER(_MX4),
                                       ctypes.POINTER(_MX4), ctypes.POINTER(_Rows), _P, _P, _P,
                                       ctypes.c_size_t, _P]),
    "octree_nca_dropout": (_I32, [ctypes.POINTER(_Dropout)] + [ctypes.POINTER(_Rows)] * 4 +
                           [_I64, _I64, _P]),
    "octree_nca_strerror": (ctypes.c_char_p, [ctypes.c_int]),
    "octree_nca_abi_version": (ctypes.c_int, []),
}

_lib = None


def library_path() -> str:
    return os.environ.get("OCTREE_NCA_LIB", LIB_PATH)


def lib():
    """The loaded library (loaded on first use).  Raises if it is not built."""
    global _lib
    if _lib is None:
        path = library_path()
        if not os.path.exists(path):
            raise OctreeNCAError(
                f"HIP library {path} is not built; run `python -m paper_2508_06993_amd.build` "
                "(there is no CPU fallback)")
        handle = ctypes.CDLL(path)
        for name, (res, args) in _SIGS.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _lib = handle
    return _lib


# ---------------------------------------------------------------------------
# marshalling helpers
# ---------------------------------------------------------------------------

@dataclass(frozen=True)
class Model:
    ndim: int
    n_in: int
    dtype: str = "f32"          # storage of states and images: "f32" or "f16"
    channels: int = 16
    hidden: int = 64
    kernel: str = "mfma"        # step kernel: names of KERNEL_NAMES, comma-separated

    @property
    def torch_dtype(self):
        return torch.float16 if self.dtype == "f16" else torch.float32

    def struct(self) -> _Model:
        k = kernel_fields(self.kernel)
        return _Model(self.ndim, self.channels, self.hidden, self.n_in,
                      OCTNCA_F16 if self.dtype == "f16" else OCTNCA_F32, k["mlp"],
                      k["layout2d"], k["steps_per_launch"])


def _extent(ext: Sequence[int]) -> _Extent:
    d, h, w = (int(v) for v in ext)
    return _Extent(d, h, w)


def _ptr(t: Optional[torch.Tensor], dtype=None, name="tensor"):
    """Address of a contiguous device tensor (an int; None for None)."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch.Tensor")
    if not t.is_cuda:
        raise OctreeNCAError(f"{name}: must be a device (cuda) tensor")
    if not t.is_contiguous():
        raise OctreeNCAError(f"{name}: must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise OctreeNCAError(f"{name}: expected {dtype}, got {t.dtype}")
    return t.data_ptr()


# the current stream's handle comes from these; torch.cuda.current_stream() would
# also make a Stream object, 2.7 us a call
_current_device = getattr(torch._C, "_cuda_getDevice", None)
_current_handle = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if type(stream) is int:
        return stream
    if stream is None:
        return _current_handle(_current_device())
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _factors(factors: Sequence[Sequence[int]], levels: int):
    """Array of three factors for each level but the coarsest; the library reads
    that many."""
    flat = [int(v) for f in factors for v in f]
    if len(flat) < 3 * (levels - 1):
        raise OctreeNCAError(f"factors: {len(flat)} values for {levels} levels, expected "
                             f"{3 * (levels - 1)}")
    arr = (_I32 * max(1, len(flat)))(*flat)
    return arr


def _check(status: int, what: str):
    if status != OCTNCA_OK:
        msg = lib().octree_nca_strerror(status).decode()
        raise OctreeNCAError(f"{what} failed: {msg} ({status})", status)


def level_weights_struct(w) -> _LevelWeights:
    """``w`` has device fp32 tensors conv_w [C][taps], conv_b [C], w1 [H][2C],
    b1 [H], w2 [C][H] (attributes or a dict)."""
    get = (lambda k: w[k]) if isinstance(w, dict) else (lambda k: getattr(w, k))
    return _LevelWeights(*(_ptr(get(k), torch.float32, k) for k in
                           ("conv_w", "conv_b", "w1", "b1", "w2")))


# ---------------------------------------------------------------------------
# entry points (same names as the C ABI)
# ---------------------------------------------------------------------------

def octree_nca_abi_version() -> int:
    return lib().octree_nca_abi_version()


def octree_nca_strerror(status: int) -> str:
    return lib().octree_nca_strerror(status).decode()


def octree_nca_build_pyramid(model: Model, image: torch.Tensor, factors, level_images,
                             stream=None) -> None:
    levels = len(level_images) + 1
    d, h, w = image.shape[:3]
    imgs = (_P * max(1, levels - 1))(*[_ptr(t, model.torch_dtype, "level image")
                                       for t in level_images])
    st = lib().octree_nca_build_pyramid(ctypes.byref(model.struct()),
                                        _ptr(image, model.torch_dtype, "image"),
                                        _extent((d, h, w)), levels, _factors(factors, levels), imgs,
                                        _stream(stream))
    _check(st, "octree_nca_build_pyramid")


def octree_nca_upsample(model: Model, coarse_state: torch.Tensor, factor, fine_image,
                        fine_state, stream=None) -> None:
    d, h, w = coarse_state.shape[:3]
    st = lib().octree_nca_upsample(ctypes.byref(model.struct()),
                                   _ptr(coarse_state, model.torch_dtype, "coarse_state"),
                                   _extent((d, h, w)), (_I32 * 3)(*[int(v) for v in factor]),
                                   _ptr(fine_image, model.torch_dtype, "fine_image"),
                                   _ptr(fine_state, model.torch_dtype, "fine_state"),
                                   _stream(stream))
    _check(st, "octree_nca_upsample")


def octree_nca_run_level(model: Model, buf0, buf1, weights, level: int, steps: int,
                         fire_rate: float, seed: int, stream=None) -> int:
    """Returns 1 if the final state is in buf1, 0 if in buf0 (steps % 2)."""
    d, h, w = buf0.shape[:3]
    res = _I32(0)
    st = lib().octree_nca_run_level(ctypes.byref(model.struct()),
                                    _ptr(buf0, model.torch_dtype, "buf0"),
                                    _ptr(buf1, model.torch_dtype, "buf1"), _extent((d, h, w)),
                                    ctypes.byref(level_weights_struct(weights)), int(level),
                                    int(steps), float(fire_rate), int(seed), ctypes.byref(res),
                                    _stream(stream))
    _check(st, "octree_nca_run_level")
    return int(res.value)


def octree_nca_readout(model: Model, state, seg, stream=None) -> None:
    d, h, w = state.shape[:3]
    st = lib().octree_nca_readout(ctypes.byref(model.struct()),
                                  _ptr(state, model.torch_dtype, "state"), _extent((d, h, w)),
                                  _ptr(seg, torch.uint8, "seg"), _stream(stream))
    _check(st, "octree_nca_readout")


def octree_nca_readout_classes(model: Model, state, classes: int, seg, stream=None) -> None:
    d, h, w = state.shape[:3]
    st = lib().octree_nca_readout_classes(ctypes.byref(model.struct()),
                                          _ptr(state, model.torch_dtype, "state"),
                                          _extent((d, h, w)), int(classes),
                                          _ptr(seg, torch.uint8, "seg"), _stream(stream))
    _check(st, "octree_nca_readout_classes")


def octree_nca_workspace_bytes(model: Model, finest, factors, with_final_state=True) -> int:
    levels = len(factors) + 1
    n = lib().octree_nca_workspace_bytes(ctypes.byref(model.struct()), _extent(finest), levels,
                                         _factors(factors, levels), 1 if with_final_state else 0)
    if n == 0:
        raise OctreeNCAError("octree_nca_workspace_bytes: invalid arguments", OCTNCA_EINVAL)
    return int(n)


def octree_nca_infer_launches(model: Model, finest, factors, steps) -> list:
    """Launch units of the steps per level (index 0 = finest) with the model's
    step kernel: the step launches that octree_nca_infer enqueues, but one per
    step on small 2D levels, where a launch runs several."""
    levels = len(factors) + 1
    out = (_I32 * levels)()
    st = lib().octree_nca_infer_launches(ctypes.byref(model.struct()), _extent(finest), levels,
                                         _factors(factors, levels), (_I32 * levels)(*steps), out)
    _check(st, "octree_nca_infer_launches")
    return [int(v) for v in out]


def octree_nca_infer(model: Model, image, factors, weights, steps, fire_rate: float, seed: int,
                     workspace, final_state=None, seg=None, level_events=None,
                     stream=None) -> None:
    levels = len(steps)
    d, h, w = image.shape[:3]
    ws = (_LevelWeights * levels)(*[level_weights_struct(x) for x in weights])
    ev = None
    if level_events is not None:
        ev = (_P * (2 * levels))(*[ctypes.c_void_p(int(e)) if e else None
                                   for e in level_events])
    st = lib().octree_nca_infer(ctypes.byref(model.struct()),
                                _ptr(image, model.torch_dtype, "image"), _extent((d, h, w)),
                                levels, _factors(factors, levels), ws,
                                (_I32 * levels)(*[int(s) for s in steps]), float(fire_rate),
                                int(seed), _ptr(workspace, torch.uint8, "workspace"),
                                workspace.numel(),
                                _ptr(final_state, model.torch_dtype, "final_state"),
                                _ptr(seg, torch.uint8, "seg"), ev, _stream(stream))
    _check(st, "octree_nca_infer")


def octree_nca_infer_static(model: Model, image, factors, weights, steps, fire_rate: float,
                            seed: int, final_state, seg=None, stream=None) -> None:
    """octree_nca_infer with the library's static device workspace (no
    allocation in the call); final_state is required.  Calls on one device
    share that workspace and must not overlap."""
    levels = len(steps)
    d, h, w = image.shape[:3]
    ws = (_LevelWeights * levels)(*[level_weights_struct(x) for x in weights])
    st = lib().octree_nca_infer_static(ctypes.byref(model.struct()),
                                       _ptr(image, model.torch_dtype, "image"),
                                       _extent((d, h, w)), levels, _factors(factors, levels), ws,
                                       (_I32 * levels)(*[int(s) for s in steps]),
                                       float(fire_rate), int(seed),
                                       _ptr(final_state, model.torch_dtype, "final_state"),
                                       _ptr(seg, torch.uint8, "seg"), _stream(stream))
    _check(st, "octree_nca_infer_static")


def octree_nca_infer_batch(model: Model, images, factors, weights, steps, fire_rate: float,
                           seed: int, workspace, final_states=None, segs=None,
                           stream=None) -> None:
    """images: [batch][d][h][w][n_in]; final_states [batch][d][h][w][C] or None;
    segs [batch][d][h][w] uint8 or None."""
    levels = len(steps)
    batch, d, h, w = images.shape[:4]
    ws = (_LevelWeights * levels)(*[level_weights_struct(x) for x in weights])
    st = lib().octree_nca_infer_batch(ctypes.byref(model.struct()),
                                      _ptr(images, model.torch_dtype, "images"), int(batch),
                                      _extent((d, h, w)), levels, _factors(factors, levels), ws,
                                      (_I32 * levels)(*[int(s) for s in steps]),
                                      float(fire_rate), int(seed),
                                      _ptr(workspace, torch.uint8, "workspace"),
                                      workspace.numel(),
                                      _ptr(final_states, model.torch_dtype, "final_states"),
                                      _ptr(segs, torch.uint8, "segs"), _stream(stream))
    _check(st, "octree_nca_infer_batch")


def octree_nca_first_level_steps(alpha0: float, coarsest) -> int:
    """Steps of the coarsest level under the alpha0 * max(H, W, D) rule."""
    n = lib().octree_nca_first_level_steps(float(alpha0), _extent(coarsest))
    if n < 0:
        raise OctreeNCAError("octree_nca_first_level_steps: invalid arguments", OCTNCA_EINVAL)
    return int(n)


def octree_nca_fire_mask(seed: int, level: int, step: int, extent, fire_rate: float, mask,
                         stream=None) -> None:
    st = lib().octree_nca_fire_mask(int(seed), int(level), int(step), _extent(extent),
                                    float(fire_rate), _ptr(mask, torch.uint8, "mask"),
                                    _stream(stream))
    _check(st, "octree_nca_fire_mask")


# ---------------------------------------------------------------------------
# training gradients (fp32 states)
# ---------------------------------------------------------------------------

def level_grads_struct(g) -> _LevelGrads:
    """``g`` has device fp32 tensors conv_w, conv_b, w1, b1, w2 shaped like the
    weights (attributes or a dict); the library writes into them."""
    get = (lambda k: g[k]) if isinstance(g, dict) else (lambda k: getattr(g, k))
    return _LevelGrads(*(_ptr(get(k), torch.float32, k) for k in
                         ("conv_w", "conv_b", "w1", "b1", "w2")))


def octree_nca_step_backward_workspace_bytes(model: Model, extent) -> int:
    return int(lib().octree_nca_step_backward_workspace_bytes(ctypes.byref(model.struct()),
                                                              _extent(extent)))


def octree_nca_step_backward(model: Model, state, grad_out, weights, level: int, step: int,
                             fire_rate: float, seed: int, grad_in, grads, workspace,
                             stream=None) -> None:
    """Backward of one step: grad_in <- dL/dS, grads += the weight gradients."""
    d, h, w = state.shape[:3]
    st = lib().octree_nca_step_backward(
        ctypes.byref(model.struct()), _ptr(state, torch.float32, "state"),
        _ptr(grad_out, torch.float32, "grad_out"), _extent((d, h, w)),
        ctypes.byref(level_weights_struct(weights)), int(level), int(step), float(fire_rate),
        int(seed), _ptr(grad_in, torch.float32, "grad_in"), ctypes.byref(level_grads_struct(grads)),
        _ptr(workspace, None, "workspace"), workspace.numel() * workspace.element_size(),
        _stream(stream))
    _check(st, "octree_nca_step_backward")


def octree_nca_upsample_backward(model: Model, grad_fine, factor, grad_coarse,
                                 stream=None) -> None:
    d, h, w = grad_coarse.shape[:3]
    f = (_I32 * 3)(*[int(v) for v in factor])
    st = lib().octree_nca_upsample_backward(ctypes.byref(model.struct()),
                                            _ptr(grad_fine, torch.float32, "grad_fine"),
                                            _extent((d, h, w)), f,
                                            _ptr(grad_coarse, torch.float32, "grad_coarse"),
                                            _stream(stream))
    _check(st, "octree_nca_upsample_backward")


def octree_nca_readout_mse_workspace_bytes(extent) -> int:
    return int(lib().octree_nca_readout_mse_workspace_bytes(_extent(extent)))


def octree_nca_readout_mse(model: Model, state, target, grad, loss, workspace,
                           stream=None) -> None:
    """loss: device float64 tensor of one element."""
    d, h, w = state.shape[:3]
    st = lib().octree_nca_readout_mse(ctypes.byref(model.struct()),
                                      _ptr(state, torch.float32, "state"),
                                      _ptr(target, torch.float32, "target"), _extent((d, h, w)),
                                      _ptr(grad, torch.float32, "grad"),
                                      _ptr(loss, torch.float64, "loss"),
                                      _ptr(workspace, None, "workspace"),
                                      workspace.numel() * workspace.element_size(),
                                      _stream(stream))
    _check(st, "octree_nca_readout_mse")


def octree_nca_train_workspace_bytes(model: Model, finest, factors, steps) -> int:
    levels = len(steps)
    s = (_I32 * levels)(*[int(v) for v in steps])
    return int(lib().octree_nca_train_workspace_bytes(ctypes.byref(model.struct()),
                                                      _extent(finest), levels,
                                                      _factors(factors, levels), s))


def _expect_elements(t, n: int, name: str) -> None:
    if t.numel() != n:
        raise OctreeNCAError(f"{name}: expected {n} elements, got {t.numel()}")


def check_train_weights(model: Model, levels: int, weights, what="weights") -> None:
    """Raises OctreeNCAError unless ``weights`` (or gradients) is a set per level,
    each tensor of the model's size."""
    if len(weights) != levels:
        raise OctreeNCAError(f"{what}: {len(weights)} sets for {levels} levels")
    c, h = model.channels, model.hidden
    sizes = (("conv_w", c * 3 ** model.ndim), ("conv_b", c), ("w1", 2 * c * h), ("b1", h),
             ("w2", c * h))
    for lvl, w in enumerate(weights):
        get = w.__getitem__ if isinstance(w, dict) else functools.partial(getattr, w)
        for k, n in sizes:
            if get(k).numel() != n:
                _expect_elements(get(k), n, f"{what} {k} of level {lvl}")


def _check_train(model: Model, levels: int, image, weights, target, grads, final_state) -> None:
    """The library sees addresses only, and takes the sizes from the model and
    the image's extent."""
    d, h, w = image.shape[:3]
    cells = d * h * w
    _expect_elements(image, model.n_in * cells, "image")
    _expect_elements(target, 2 * cells, "target")
    if final_state is not None:
        _expect_elements(final_state, model.channels * cells, "final_state")
    check_train_weights(model, levels, weights)
    check_train_weights(model, levels, grads, "grads")


def octree_nca_train_step(model: Model, image, factors, weights, steps, fire_rate: float,
                          seed: int, target, workspace, grads, loss, final_state=None,
                          stream=None) -> None:
    """One training step; ``grads`` is a list (index = level) of gradient sets,
    overwritten; ``loss`` a device float64 tensor of one element; ``target`` is
    [d][h][w][2].  Sizes that do not fit raise OctreeNCAError."""
    levels = len(steps)
    _check_train(model, levels, image, weights, target, grads, final_state)
    d, h, w = image.shape[:3]
    ws = (_LevelWeights * levels)(*[level_weights_struct(x) for x in weights])
    gs = (_LevelGrads * levels)(*[level_grads_struct(x) for x in grads])
    s = (_I32 * levels)(*[int(v) for v in steps])
    st = lib().octree_nca_train_step(
        ctypes.byref(model.struct()), _ptr(image, torch.float32, "image"), _extent((d, h, w)),
        levels, _factors(factors, levels), ws, s, float(fire_rate), int(seed),
        _ptr(target, torch.float32, "target"), _ptr(workspace, None, "workspace"),
        workspace.numel() * workspace.element_size(), gs, _ptr(loss, torch.float64, "loss"),
        _ptr(final_state, torch.float32, "final_state"), _stream(stream))
    _check(st, "octree_nca_train_step")


# ---------------------------------------------------------------------------
# state cache: states in 8 bits
# ---------------------------------------------------------------------------

@dataclass(frozen=True)
class StateCacheBuffers:
    """A cache's description and device memory (octnca_state_cache): codes int8
    or uint8 [slots][cells][C], scales fp32 [slots][ceil(cells / block)][C]."""
    codes: torch.Tensor
    scales: torch.Tensor
    cells: int
    code: str = "i8"
    block: int = 64

    def struct(self, model: Model) -> _StateCache:
        if self.code not in CODE_NAMES:
            raise ValueError(f"unknown code {self.code!r}; known: {sorted(CODE_NAMES)}")
        if self.block not in (32, 64, 128):
            raise ValueError(f"block is 32, 64 or 128 cells, got {self.block}")
        if self.codes.dtype not in (torch.int8, torch.uint8):
            raise OctreeNCAError(f"codes: expected int8 or uint8, got {self.codes.dtype}")
        slots, c = self.codes.shape[0], model.channels
        if tuple(self.codes.shape) != (slots, self.cells, c):
            raise OctreeNCAError(f"codes: expected shape {(slots, self.cells, c)}, "
                                 f"got {tuple(self.codes.shape)}")
        want = (slots, -(-self.cells // self.block), c)
        if tuple(self.scales.shape) != want:
            raise OctreeNCAError(f"scales: expected shape {want}, got {tuple(self.scales.shape)}")
        return _StateCache(CODE_NAMES[self.code], self.block, slots, self.cells,
                           _ptr(self.codes, None, "codes"),
                           _ptr(self.scales, torch.float32, "scales"))


def _cache_call(call, model, refs, states, from_cell, slots, first, stream):
    """A state-cache call (a function of lib()): states [n][cells...][C], refs of
    state_cache_refs."""
    shape = states.shape
    n, c = shape[0], shape[-1]
    if c != model.channels:
        raise OctreeNCAError(f"states: expected {model.channels} channels, got {c}")
    if slots is not None and slots.shape != (n,):
        raise OctreeNCAError(f"slots: expected shape {(n,)}, got {tuple(slots.shape)}")
    st = call(*refs, _ptr(states, model.torch_dtype, "states"), from_cell,
              states.numel() // (n * c) if n else 0, n, _ptr(slots, torch.int64, "slots"), first,
              _stream(stream))
    if st:
        _check(st, call.__name__)


def state_cache_refs(model: Model, cache: StateCacheBuffers):
    """The two structs of a call; a caller of many keeps them."""
    return ctypes.byref(model.struct()), ctypes.byref(cache.struct(model))


def octree_nca_state_cache_write(model: Model, cache: StateCacheBuffers, states, from_cell=0,
                                 slots=None, first=0, stream=None, refs=None) -> None:
    """Quantise states [n][...cells][C] into the slots ``slots`` (device int64
    [n]) or first, first + 1, ..."""
    _cache_call(lib().octree_nca_state_cache_write, model, refs or state_cache_refs(model, cache),
                states, from_cell, slots, first, stream)


def octree_nca_state_cache_read(model: Model, cache: StateCacheBuffers, states, from_cell=0,
                                slots=None, first=0, stream=None, refs=None) -> None:
    """Fill states [n][...cells][C] with the values of the slots."""
    _cache_call(lib().octree_nca_state_cache_read, model, refs or state_cache_refs(model, cache),
                states, from_cell, slots, first, stream)


def _keep(code, block) -> _Keep:
    if code not in CODE_NAMES:
        raise ValueError(f"unknown code {code!r}; known: {sorted(CODE_NAMES)}")
    return _Keep(CODE_NAMES[code], int(block))


def octree_nca_train_kept_workspace_bytes(model: Model, finest, factors, steps, code="i8",
                                          block=64) -> int:
    levels = len(steps)
    return int(lib().octree_nca_train_kept_workspace_bytes(
        ctypes.byref(model.struct()), _extent(finest), levels, _factors(factors, levels),
        (_I32 * levels)(*[int(v) for v in steps]), ctypes.byref(_keep(code, block))))


def octree_nca_train_step_kept(model: Model, image, factors, weights, steps, fire_rate: float,
                               seed: int, target, workspace, grads, loss, final_state=None,
                               code="i8", block=64, stream=None) -> None:
    """octree_nca_train_step with the states kept in 8 bits (``code``, ``block``)."""
    levels = len(steps)
    _check_train(model, levels, image, weights, target, grads, final_state)
    d, h, w = image.shape[:3]
    ws = (_LevelWeights * levels)(*[level_weights_struct(x) for x in weights])
    gs = (_LevelGrads * levels)(*[level_grads_struct(x) for x in grads])
    s = (_I32 * levels)(*[int(v) for v in steps])
    st = lib().octree_nca_train_step_kept(
        ctypes.byref(model.struct()), _ptr(image, torch.float32, "image"), _extent((d, h, w)),
        levels, _factors(factors, levels), ws, s, float(fire_rate), int(seed),
        _ptr(target, torch.float32, "target"), ctypes.byref(_keep(code, block)),
        _ptr(workspace, None, "workspace"), workspace.numel() * workspace.element_size(), gs,
        _ptr(loss, torch.float64, "loss"), _ptr(final_state, torch.float32, "final_state"),
        _stream(stream))
    _check(st, "octree_nca_train_step_kept")


# ---------------------------------------------------------------------------
# gradients of many tensors
# ---------------------------------------------------------------------------

_GRAD_TYPES = {torch.float32: OCTNCA_F32, torch.float16: OCTNCA_F16, torch.bfloat16: OCTNCA_BF16}


def _grad_type(t, name):
    if t.dtype not in _GRAD_TYPES:
        raise OctreeNCAError(f"{name}: expected fp32, fp16 or bf16, got {t.dtype}")
    return _GRAD_TYPES[t.dtype]


def _addresses(tensors, counts, device, dtype, name):
    """Addresses of a list of contiguous device tensors of the given sizes."""
    out = [_ptr(t, dtype, name) for t in tensors]
    for t, n in zip(tensors, counts):
        if t.numel() != n:
            raise OctreeNCAError(f"{name}: {t.numel()} elements for {n} of the gradient")
        if t.device != device:
            raise OctreeNCAError(f"{name}: on {t.device}, the first gradient on {device}")
    return out


def param_structs(grads, params=None, m=None, v=None, ema=None, clipped=None):
    """Array of octnca_param for lists of device tensors (index = tensor)."""
    for k, x in (("param", params), ("m", m), ("v", v), ("ema", ema), ("clipped", clipped)):
        if x is not None and len(x) != len(grads):
            raise OctreeNCAError(f"{k}: {len(x)} tensors for {len(grads)} gradients")
    if not grads:
        return (_Param * 1)()
    counts = [g.numel() for g in grads]
    device = grads[0].device
    out = np.zeros(len(grads), np.dtype(_Param))
    out["count"] = counts
    out["grad"] = _addresses(grads, counts, device, None, "grad")
    out["grad_dtype"] = [_grad_type(g, "grad") for g in grads]
    for k, x in (("param", params), ("m", m), ("v", v), ("ema", ema)):
        if x is not None:
            out[k] = _addresses(x, counts, device, torch.float32, k)
    if clipped is not None:
        out["clipped"] = _addresses(clipped, counts, device, None, "clipped")
        out["clipped_dtype"] = [_grad_type(t, "clipped") for t in clipped]
    return (_Param * len(grads)).from_buffer(out)


def octree_nca_param_table_bytes(structs, n: int) -> int:
    size = int(lib().octree_nca_param_table_bytes(structs, n))
    if size == 0:
        raise OctreeNCAError("octree_nca_param_table_bytes: invalid list", OCTNCA_EINVAL)
    return size


def octree_nca_param_table(structs, n: int, table, stream=None) -> _ParamList:
    """Writes the table of a list (param_structs) to the uint8 tensor ``table``."""
    out = _ParamList()
    st = lib().octree_nca_param_table(structs, n, _ptr(table, torch.uint8, "table"),
                                      table.numel(), ctypes.byref(out), _stream(stream))
    _check(st, "octree_nca_param_table")
    return out


def octree_nca_grad_norm(plist: _ParamList, norm, scale=1.0, stream=None) -> None:
    """norm: device fp32 tensor of one element."""
    st = lib().octree_nca_grad_norm(ctypes.byref(plist), float(scale),
                                    _ptr(norm, torch.float32, "norm"), _stream(stream))
    _check(st, "octree_nca_grad_norm")


def octree_nca_clip_grads(plist: _ParamList, max_norm: float, scale=1.0, norm=None,
                          stream=None) -> None:
    st = lib().octree_nca_clip_grads(ctypes.byref(plist), float(scale), float(max_norm),
                                     _ptr(norm, torch.float32, "norm"), _stream(stream))
    _check(st, "octree_nca_clip_grads")


def octree_nca_adamw(plist: _ParamList, step, lr: float, betas=(0.9, 0.99), eps=1e-8,
                     weight_decay=0.0, max_norm=float("inf"), scale=1.0, ema_decay=0.0, norm=None,
                     stream=None) -> None:
    """step: device int64 tensor of one element, the updates made so far."""
    h = _AdamW(lr, betas[0], betas[1], eps, weight_decay, max_norm, scale, ema_decay)
    st = lib().octree_nca_adamw(ctypes.byref(plist), ctypes.byref(h),
                                _ptr(step, torch.int64, "step"),
                                _ptr(norm, torch.float32, "norm"), _stream(stream))
    _check(st, "octree_nca_adamw")


# ---------------------------------------------------------------------------
# cell layers: matrices in microscaled 4 bits, dropout
# ---------------------------------------------------------------------------

def _on_device(t, name):
    """Refuses tensors that the current device's kernels would not be given."""
    device = t.get_device()
    if device < 0:
        raise OctreeNCAError(f"{name}: must be a device (cuda) tensor")
    if device != _current_device():
        raise OctreeNCAError(f"{name}: on {t.device}, the current device is {_current_device()}")


def _here(*matrices):
    """Refuses matrices in 4 bits whose memory the current device's kernels would not be
    given."""
    for m in matrices:
        if m.device is not None and m.device != _current_device():
            raise OctreeNCAError(f"matrix in 4 bits: on cuda:{m.device}, the current device is "
                                 f"{_current_device()}")


def _rows(t, name, rows=None, cols=None):
    """octnca_rows of a tensor [..., cols]: rows any distance apart (two
    dimensions) or contiguous; checked against a size if one is given."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch.Tensor")
    dtype = _GRAD_TYPES.get(t.dtype)
    if dtype is None:
        raise OctreeNCAError(f"{name}: expected fp32, fp16 or bf16, got {t.dtype}")
    _on_device(t, name)
    shape = t.shape
    if len(shape) == 2:
        r, c = shape
        stride, step = t.stride()
        if (step != 1 and c > 1) or (stride < c and r > 1):
            raise OctreeNCAError(f"{name}: columns must be contiguous and rows apart, got strides "
                                 f"{(stride, step)}")
    else:
        if not shape or not t.is_contiguous():
            raise OctreeNCAError(f"{name}: expected rows of columns or a contiguous tensor")
        c = shape[-1]
        r = t.numel() // c if c else 0
        stride = c
    if rows is not None and (r, c) != (rows, cols):
        raise OctreeNCAError(f"{name}: expected {(rows, cols)}, got {(r, c)}")
    return _Rows(t.data_ptr(), stride, dtype), r, c


def _vector(t, name, n):
    if t is None:
        return None
    if t.numel() != n:
        raise OctreeNCAError(f"{name}: expected {n} elements, got {t.numel()}")
    _on_device(t, name)
    return _ptr(t, torch.float32, name)


def mx4_shapes(rows: int, cols: int):
    """Shapes of the codes and scales (uint8) of a matrix in 4 bits."""
    groups, blocks = -(-rows // 16), -(-cols // 32)
    return (groups, blocks, 16, 16), (groups, blocks, 16)


@dataclass(frozen=True)
class MX4Buffers:
    """A matrix in microscaled 4 bits (octnca_mx4): codes and scales uint8 of
    mx4_shapes, or of more rows."""
    rows: int
    cols: int
    codes: torch.Tensor
    scales: torch.Tensor

    def struct(self) -> _MX4:
        for t, want, name in zip((self.codes, self.scales), mx4_shapes(self.rows, self.cols),
                                 ("codes", "scales")):
            shape = tuple(t.shape)
            if shape[1:] != want[1:] or len(shape) != len(want) or shape[0] < want[0]:
                raise OctreeNCAError(f"{name}: expected shape {want}, got {shape}")
            _on_device(t, name)
        m = _MX4(self.rows, self.cols, _ptr(self.codes, torch.uint8, "codes"),
                 _ptr(self.scales, torch.uint8, "scales"))
        m.device = self.codes.get_device()
        return m


def octree_nca_mx4_code_bytes(rows: int, cols: int) -> int:
    return int(lib().octree_nca_mx4_code_bytes(rows, cols))


def octree_nca_mx4_quantise(x, m: _MX4, stream=None) -> None:
    """m (MX4Buffers.struct) = x [rows][cols] in 4 bits."""
    _here(m)
    st = lib().octree_nca_mx4_quantise(_rows(x, "x", m.rows, m.cols)[0], m, _stream(stream))
    if st:
        _check(st, "octree_nca_mx4_quantise")


def octree_nca_mx4_dequantise(m: _MX4, x, stream=None) -> None:
    """x [rows][cols] = the values of m."""
    _here(m)
    st = lib().octree_nca_mx4_dequantise(m, _rows(x, "x", m.rows, m.cols)[0], _stream(stream))
    if st:
        _check(st, "octree_nca_mx4_dequantise")


def octree_nca_mx4_product(a: _MX4, w: _MX4, out, bias=None, relu=False, stream=None) -> None:
    """out [a.rows][w.rows] = a times w transposed, plus bias; relu."""
    _here(a, w)
    st = lib().octree_nca_mx4_product(a, w, _vector(bias, "bias", w.rows), relu,
                                      _rows(out, "out", a.rows, w.rows)[0], _stream(stream))
    if st:
        _check(st, "octree_nca_mx4_product")


def octree_nca_mx4_linear(x, kept: _MX4, w: _MX4, out, bias=None, relu=False,
                          stream=None) -> None:
    """kept = x in 4 bits, out = kept times w transposed, plus bias; relu."""
    _here(kept, w)
    st = lib().octree_nca_mx4_linear(_rows(x, "x", kept.rows, kept.cols)[0], kept, w,
                                     _vector(bias, "bias", w.rows), relu,
                                     _rows(out, "out", kept.rows, w.rows)[0], _stream(stream))
    if st:
        _check(st, "octree_nca_mx4_linear")


def octree_nca_mx4_backward_workspace_bytes(rows: int, cols: int, outs: int) -> int:
    return int(lib().octree_nca_mx4_backward_workspace_bytes(rows, cols, outs))


def octree_nca_mx4_backward(grad_out, a: _MX4, w: _MX4, grad_in=None, grad_weight=None,
                            grad_bias=None, workspace=None, stream=None) -> None:
    """Gradients of the product of a and w for the gradient grad_out
    [a.rows][w.rows]; grad_weight fp32 [w.rows][a.cols], grad_bias fp32 [w.rows]."""
    _here(a, w)
    if workspace is not None:
        _on_device(workspace, "workspace")
    st = lib().octree_nca_mx4_backward(
        _rows(grad_out, "grad_out", a.rows, w.rows)[0], a, w,
        None if grad_in is None else _rows(grad_in, "grad_in", a.rows, a.cols)[0],
        _vector(grad_weight, "grad_weight", w.rows * a.cols),
        _vector(grad_bias, "grad_bias", w.rows), _ptr(workspace, None, "workspace"),
        0 if workspace is None else workspace.numel() * workspace.element_size(),
        _stream(stream))
    if st:
        _check(st, "octree_nca_mx4_backward")


def octree_nca_dropout(x, out, rate: float, seed: int, index=0, step=None, gate=None, add=None,
                       stream=None) -> None:
    """out = add + dropout of x (gated); step: device int64 [1] added to index."""
    if step is not None:
        if step.numel() != 1:
            raise OctreeNCAError(f"step: expected 1 element, got {step.numel()}")
        _on_device(step, "step")
    rx, r, c = _rows(x, "x")
    st = lib().octree_nca_dropout(
        _Dropout(rate, seed, index, _ptr(step, torch.int64, "step")), rx,
        None if gate is None else _rows(gate, "gate", r, c)[0],
        None if add is None else _rows(add, "add", r, c)[0], _rows(out, "out", r, c)[0], r, c,
        _stream(stream))
    if st:
        _check(st, "octree_nca_dropout")
