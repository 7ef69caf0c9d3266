"""ctypes binding of ``libdamoe.so`` (the C-ABI declared in ``include/damoe.h``).

Argument marshalling only: every step of the path runs in the library's HIP
kernels.  Tensors are passed as device pointers (``tensor.data_ptr()``) and
streams as raw ``hipStream_t`` handles; PyTorch is only used by callers to own
device memory.  Loading fails loudly if the library has not been built.
"""
from __future__ import annotations

import ctypes
import os
import struct
from dataclasses import dataclass

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdamoe.so")

N_TILE_SIZES = 5
W_BF16, W_FP8_B128, W_MXFP4 = 0, 1, 2
DEVERR_EXPERT_ID, DEVERR_TILES, DEVERR_VARIANT, DEVERR_COUNTS = 1, 2, 4, 8
LAYOUT_ROWMAJOR, LAYOUT_FRAG16, LAYOUT_TILE32 = 0, 1, 2
BF16, F32 = 0, 1
SCORE_SOFTMAX, SCORE_SIGMOID = 0, 1

STATUS = {0: "ok", -1: "invalid argument", -2: "unsupported", -3: "workspace too small",
          -4: "table mismatch", -5: "hip error", -6: "out of memory", -7: "io error"}

EXPORTED = [
    "damoe_status_string", "damoe_workspace_layout", "damoe_workspace_size", "damoe_route_histogram",
    "damoe_table_create", "damoe_table_destroy", "damoe_table_info", "damoe_table_save",
    "damoe_table_load", "damoe_dispatch", "damoe_fused_moe", "damoe_num_variants", "damoe_variant_name",
    "damoe_variant_tile_m", "damoe_variant_supports", "damoe_tune", "damoe_alpha_search",
    "damoe_read_device_error", "damoe_fused_moe_stage", "damoe_route_dispatch", "damoe_pack_weights",
    "damoe_table_candidates", "damoe_router", "damoe_router_workspace_size", "damoe_route_dispatch_effexp",
    "damoe_table_effexp_map", "damoe_table_effexp_candidates", "damoe_noalloc_scratch_bytes",
    "damoe_moe_layer_noalloc", "damoe_router_loss_workspace_size", "damoe_router_loss", "damoe_router_loss_grad",
    "damoe_mxfp4_bytes", "damoe_mxfp4_quantise", "damoe_mxfp4_dequantise", "damoe_mxfp4_pack",
    "damoe_mxfp4_linear_workspace_size", "damoe_mxfp4_linear", "damoe_call_words",
]


class DamoeError(RuntimeError):
    def __init__(self, fn: str, code: int):
        super().__init__(f"{fn} failed: {code} ({STATUS.get(code, 'unknown')})")
        self.code = code


class Layer(ctypes.Structure):
    _fields_ = [("E", ctypes.c_int32), ("k", ctypes.c_int32), ("H", ctypes.c_int32),
                ("I", ctypes.c_int32), ("wdtype", ctypes.c_int32), ("layout", ctypes.c_int32),
                ("w1", ctypes.c_void_p),
                ("w3", ctypes.c_void_p), ("w2", ctypes.c_void_p), ("s1", ctypes.c_void_p),
                ("s3", ctypes.c_void_p), ("s2", ctypes.c_void_p)]


class WsLayout(ctypes.Structure):
    _fields_ = [("total", ctypes.c_size_t), ("ctrl", ctypes.c_size_t),
                ("tiles", ctypes.c_size_t * N_TILE_SIZES), ("tiles_cap", ctypes.c_size_t),
                ("h", ctypes.c_size_t), ("out", ctypes.c_size_t), ("route", ctypes.c_size_t)]


class TableDesc(ctypes.Structure):
    _fields_ = [("E", ctypes.c_int32), ("k", ctypes.c_int32), ("H", ctypes.c_int32),
                ("I", ctypes.c_int32), ("wdtype", ctypes.c_int32), ("n_buckets", ctypes.c_int32),
                ("bucket_T", ctypes.c_void_p), ("n_ex", ctypes.c_void_p), ("Q", ctypes.c_void_p),
                ("kid", ctypes.c_void_p), ("noda", ctypes.c_void_p)]


class TuneConfig(ctypes.Structure):
    _fields_ = [("n_buckets", ctypes.c_int32), ("bucket_T", ctypes.c_void_p),
                ("n_skews", ctypes.c_int32), ("skew_X", ctypes.c_void_p), ("samples", ctypes.c_int32),
                ("reps", ctypes.c_int32), ("alpha_samples", ctypes.c_int32),
                ("alpha_iters", ctypes.c_int32), ("seed", ctypes.c_uint64), ("x", ctypes.c_void_p),
                ("verbose", ctypes.c_int32), ("ep", ctypes.c_int32), ("n_repeat", ctypes.c_int32),
                ("repeat_f", ctypes.c_void_p), ("flush_mib", ctypes.c_int32)]


_lib = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built: run __graft_entry__.build() "
                               "(the fused-MoE path has no fallback)")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, u32, u64, sz, f64 = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint32, ctypes.c_uint64,
                                      ctypes.c_size_t, ctypes.c_double)
        i64, f32 = ctypes.c_int64, ctypes.c_float
        sigs = {
            "damoe_status_string": ([i32], ctypes.c_char_p),
            "damoe_workspace_layout": ([i32, i32, i32, i32, i32, vp], i32),
            "damoe_workspace_size": ([vp, i32], sz),
            "damoe_route_histogram": ([vp, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp], i32),
            "damoe_table_create": ([vp, vp], i32),
            "damoe_table_destroy": ([vp], None),
            "damoe_table_info": ([vp, vp, vp, vp, vp, vp, vp, vp], i32),
            "damoe_table_save": ([vp, ctypes.c_char_p], i32),
            "damoe_table_load": ([ctypes.c_char_p, vp], i32),
            "damoe_dispatch": ([vp, vp, i32, vp, vp, sz, vp], i32),
            "damoe_route_dispatch": ([vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp], i32),
            "damoe_fused_moe": ([vp, vp, vp, i32, vp, vp, vp, i32, u32, vp, vp, sz, vp], i32),
            "damoe_fused_moe_stage": ([vp, i32, vp, vp, i32, vp, vp, vp, i32, u32, vp, vp, sz, vp], i32),
            "damoe_table_candidates": ([vp, i32], u32),
            "damoe_num_variants": ([], i32),
            "damoe_variant_name": ([i32], ctypes.c_char_p),
            "damoe_variant_tile_m": ([i32], i32),
            "damoe_variant_supports": ([i32, i32], i32),
            "damoe_tune": ([vp, vp, vp, vp], i32),
            "damoe_alpha_search": ([i32, f64, i32, i32, u64], f64),
            "damoe_read_device_error": ([vp, vp, vp], i32),
            "damoe_pack_weights": ([vp, vp, vp, vp, vp], i32),
            "damoe_router": ([vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, vp, sz, vp], i32),
            "damoe_router_workspace_size": ([i32, i32, i32], sz),
            "damoe_route_dispatch_effexp": ([vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp], i32),
            "damoe_table_effexp_map": ([vp, i32, vp], i32),
            "damoe_table_effexp_candidates": ([vp, i32], u32),
            "damoe_noalloc_scratch_bytes": ([], sz),
            "damoe_moe_layer_noalloc": ([vp, vp, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp], i32),
            "damoe_router_loss_workspace_size": ([i32, i32, i32], sz),
            "damoe_router_loss": ([vp, i32, i64, vp, vp, vp, i32, i32, i32, i32, i32, f32, f32, vp, vp, vp, vp, vp, sz,
                                   vp], i32),
            "damoe_router_loss_grad": ([vp, i32, i64, vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, f32, f32, vp,
                                        vp, i64, vp], i32),
            "damoe_mxfp4_bytes": ([i64, i32, i32], sz),
            "damoe_mxfp4_quantise": ([vp, i32, i64, i32, i64, i32, vp, vp, vp], i32),
            "damoe_mxfp4_dequantise": ([vp, vp, i64, i32, i32, vp, i32, i64, vp], i32),
            "damoe_mxfp4_pack": ([vp, vp, i64, i32, vp, vp], i32),
            "damoe_mxfp4_linear_workspace_size": ([i32, i32, i32], sz),
            "damoe_call_words": ([i32, ctypes.c_char_p, sz], i32),
            "damoe_mxfp4_linear": ([vp, i32, i64, i32, i32, vp, i32, vp, i64, vp, i32, i64, vp, sz, vp], i32),
        }
        for name, (args, res) in sigs.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = res
        _lib = L
    return _lib


def _check(fn: str, rc: int):
    if rc != 0:
        raise DamoeError(fn, rc)


def _p(t) -> int:
    """Device (or host numpy) pointer of a tensor, or 0 for None."""
    if t is None:
        return 0
    try:
        return t.data_ptr()
    except AttributeError:
        return t.ctypes.data


def _stream(stream) -> int:
    if stream is None:  # the handle alone: torch.cuda.current_stream() builds a Stream object, 2.7 us a call
        import torch
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


_torch = None  # set by _types()


def _stream_on(fn: str, stream, dev: int, dtype: int, rows: int = 1) -> int:
    """The stream's handle for a call on tensors of device number `dev` (-1: the host's memory), which a kernel on
    the current device would fault on unless it is that device.  Without rows nothing is launched."""
    if dev < 0 or dev != _torch._C._cuda_getDevice():
        if dtype < 0:  # what the library refuses by itself is named as it does
            raise DamoeError(fn, -2)
        if rows == 0:
            return 0
        raise ValueError(f"{fn}: tensors of the current device are wanted, not of "
                         + (f"cuda:{dev} (torch.cuda.device makes it the current one)" if dev >= 0 else "the host"))
    if stream is None:
        return _torch._C._cuda_getCurrentRawStream(dev)
    if isinstance(stream, int):
        return stream
    if getattr(stream, "device_index", dev) != dev:
        raise ValueError(f"{fn}: a stream of cuda:{stream.device_index}, the tensors are on cuda:{dev}")
    return stream.cuda_stream


# ---------------------------------------------------------------- registry / layout

def num_variants() -> int:
    return int(lib().damoe_num_variants())


def variant_name(v: int) -> str:
    n = lib().damoe_variant_name(v)
    return n.decode() if n else ""


def variant_tile_m(v: int) -> int:
    return int(lib().damoe_variant_tile_m(v))


def variant_supports(v: int, wdtype: int) -> bool:
    return bool(lib().damoe_variant_supports(v, wdtype))


def workspace_layout(E: int, k: int, H: int, I: int, T: int) -> dict:
    lo = WsLayout()
    _check("damoe_workspace_layout", lib().damoe_workspace_layout(E, k, H, I, T, ctypes.byref(lo)))
    return {"total": lo.total, "ctrl": lo.ctrl, "tiles": list(lo.tiles), "tiles_cap": lo.tiles_cap,
            "h": lo.h, "out": lo.out, "route": lo.route}


def make_layer(E, k, H, I, wdtype, w1, w3, w2, s1=None, s3=None, s2=None, layout=LAYOUT_ROWMAJOR) -> Layer:
    return Layer(E, k, H, I, wdtype, layout, _p(w1), _p(w3), _p(w2), _p(s1), _p(s3), _p(s2))


def pack_weights(layer: Layer, w1, w3, w2, stream=None):
    _check("damoe_pack_weights", lib().damoe_pack_weights(ctypes.byref(layer), _p(w1), _p(w3), _p(w2),
                                                          _stream(stream)))


def workspace_size(layer: Layer, T_max: int) -> int:
    return int(lib().damoe_workspace_size(ctypes.byref(layer), T_max))


def alpha_search(E: int, target: float, samples: int = 64, iters: int = 60, seed: int = 0) -> float:
    return float(lib().damoe_alpha_search(E, float(target), samples, iters, seed))


# ---------------------------------------------------------------- stream-ordered calls

def route_histogram(ids, T, k, E, counts, offsets, perm, inv_perm, numden, bucket, ws, stream=None):
    _check("damoe_route_histogram", lib().damoe_route_histogram(
        _p(ids), T, k, E, _p(counts), _p(offsets), _p(perm), _p(inv_perm), _p(numden), _p(bucket),
        _p(ws), ws.numel() * ws.element_size(), _stream(stream)))


def route_dispatch(table: "Table", ids, T, k, E, counts, offsets, perm, inv_perm, numden, bucket,
                   variant_id, ws, stream=None):
    _check("damoe_route_dispatch", lib().damoe_route_dispatch(
        table.handle, _p(ids), T, k, E, _p(counts), _p(offsets), _p(perm), _p(inv_perm), _p(numden),
        _p(bucket), _p(variant_id), _p(ws), ws.numel() * ws.element_size(), _stream(stream)))


def route_dispatch_effexp(table: "Table", ids, T, k, E, counts, offsets, perm, inv_perm, numden, bucket,
                          variant_id, ws, stream=None):
    _check("damoe_route_dispatch_effexp", lib().damoe_route_dispatch_effexp(
        table.handle, _p(ids), T, k, E, _p(counts), _p(offsets), _p(perm), _p(inv_perm), _p(numden),
        _p(bucket), _p(variant_id), _p(ws), ws.numel() * ws.element_size(), _stream(stream)))


def dispatch(table: "Table", counts, T, variant_id, ws, stream=None):
    _check("damoe_dispatch", lib().damoe_dispatch(table.handle, _p(counts), T, _p(variant_id), _p(ws),
                                                  ws.numel() * ws.element_size(), _stream(stream)))


def fused_moe(layer: Layer, x, w, T, perm, inv_perm, variant_id, force_variant, y, ws, stream=None,
              candidates: int = 0):
    """candidates: bit mask of the variant ids *variant_id may hold (Table.candidates(T)); 0 = all."""
    _check("damoe_fused_moe", lib().damoe_fused_moe(
        ctypes.byref(layer), _p(x), _p(w), T, _p(perm), _p(inv_perm), _p(variant_id), int(force_variant),
        int(candidates), _p(y), _p(ws), ws.numel() * ws.element_size(), _stream(stream)))


def fused_moe_stage(layer: Layer, stage, x, w, T, perm, inv_perm, variant_id, force_variant, y, ws,
                    stream=None, candidates: int = 0):
    _check("damoe_fused_moe_stage", lib().damoe_fused_moe_stage(
        ctypes.byref(layer), int(stage), _p(x), _p(w), T, _p(perm), _p(inv_perm), _p(variant_id),
        int(force_variant), int(candidates), _p(y), _p(ws), ws.numel() * ws.element_size(),
        _stream(stream)))


def noalloc_scratch_bytes() -> int:
    return int(lib().damoe_noalloc_scratch_bytes())


def moe_layer_noalloc(table: "Table", layer: Layer, x, ids, w, T, counts, offsets, perm, inv_perm, numden, bucket,
                      variant_id, y, stream=None):
    """route_dispatch + fused_moe with the library's own fixed workspace (no workspace argument)."""
    _check("damoe_moe_layer_noalloc", lib().damoe_moe_layer_noalloc(
        table.handle, ctypes.byref(layer), _p(x), _p(ids), _p(w), T, _p(counts), _p(offsets), _p(perm),
        _p(inv_perm), _p(numden), _p(bucket), _p(variant_id), _p(y), _stream(stream)))


def router_workspace_size(E: int, H: int, T_max: int) -> int:
    return int(lib().damoe_router_workspace_size(E, H, T_max))


def router(x, wg, bias, T, H, E, k, logits, ids, w, ws, stream=None):
    _check("damoe_router", lib().damoe_router(_p(x), _p(wg), _p(bias), T, H, E, k, _p(logits), _p(ids), _p(w),
                                              _p(ws), ws.numel() * ws.element_size(), _stream(stream)))


# torch types, filled by the first call
_DTYPES = {}  # element types of matrices; anything else gets a code that the library refuses
_INT32, _FLOAT32, _BYTES = set(), set(), set()


def _types():
    global _torch
    import torch
    _torch = torch
    _BYTES.update((torch.uint8, torch.bool, torch.int8))
    _FLOAT32.add(torch.float32)
    _INT32.add(torch.int32)
    _DTYPES.update({torch.bfloat16: BF16, torch.float32: F32})  # last: another thread takes it for all


def _dtype(t) -> int:
    if not _DTYPES:
        _types()
    return _DTYPES.get(t.dtype, -1)


def _ld(name: str, t, rows: int, cols: int, ld) -> int:
    """Row stride of a matrix in elements: as given, the tensor's own (2-D), or `cols`.  The elements of a row
    lie side by side and the tensor holds rows x cols of them; any other is refused."""
    if ld is None:
        shape = t.shape
        if len(shape) == 2:
            if shape[0] >= rows and shape[1] >= cols:
                if t.is_contiguous():
                    return shape[1]
                stride = t.stride()
                if stride[1] == 1 or shape[1] == 1:
                    return max(cols, stride[0]) if shape[0] == 1 else stride[0]
        elif t.numel() >= rows * cols and t.is_contiguous():
            return cols
    elif rows <= 0 or (rows - 1) * ld + cols <= _reach(t):
        return int(ld)
    raise ValueError(f"{name}: {rows} rows of {cols} elements side by side are wanted, not {tuple(t.shape)} with strides "
                     f"{t.stride()}" + ("" if ld is None else f" taken with a row stride of {ld}"))


def _elsewhere(name: str, t):
    raise ValueError(f"{name}: a tensor on {t.device}, others of the call are on another device")


def _reach(t) -> int:
    """Elements from a tensor's first to its last."""
    if t.is_contiguous():
        return t.numel()
    return 1 + sum((n - 1) * s for n, s in zip(t.shape, t.stride())) if t.numel() else 0


def _list(name: str, t, types: set, n: int, dev: int) -> int:
    """Pointer of a tensor on device number `dev`, 0 for None.  Refuses one that is not n elements side by side of one of
    the types: an int64 list of offsets or of counts, or the gradient of a sum, whose elements are all the same one, would
    be taken for something else, and a shorter list or output be read or written past its end."""
    if t is None:
        return 0
    if t.dtype in types and t.numel() >= n and t.is_contiguous():
        if t.get_device() != dev:
            _elsewhere(name, t)
        return t.data_ptr()
    raise ValueError(f"{name}: {n} contiguous elements of {'/'.join(str(d) for d in types)} are wanted, "
                     f"not {tuple(t.shape)} of {t.dtype}, strides {t.stride()}")


def _room(name: str, t, n: int, dev: int) -> int:
    """Pointer of a buffer of at least n bytes side by side on device number `dev`, 0 for None."""
    if t is None:
        return 0
    if t.nbytes >= n and t.is_contiguous():
        if t.get_device() != dev:
            _elsewhere(name, t)
        return t.data_ptr()
    raise ValueError(f"{name}: {n} contiguous bytes are wanted, not {t.nbytes} in {tuple(t.shape)} with strides {t.stride()}")


def _offsets(t, S: int, dev: int) -> int:
    """_list for offsets, of S sequences and no other number of them: a longer list would lose its last sequences."""
    if t is None or t.dtype in _INT32 and t.numel() == S + 1 and t.is_contiguous() and t.get_device() == dev:
        return 0 if t is None else t.data_ptr()
    _list("seq_offsets", t, _INT32, S + 1, dev)
    raise ValueError(f"seq_offsets: S = {S} sequences have {S + 1} offsets, not {t.numel()}")


# damoe_call_words: ctypes takes 50 to 85 ns to convert an argument, and these calls have 15 to 21 (as words: 0.8 us less,
# what the checks of their tensors cost).
_LOSS_WORDS, _GRAD_WORDS, _LINEAR_WORDS = (struct.Struct(f).pack for f in ("=11q2d7q", "=15q2d4q", "=15q"))


def router_loss_workspace_size(T_max: int, E: int, S: int = 1) -> int:
    return int(lib().damoe_router_loss_workspace_size(T_max, E, S))


def router_loss(logits, ids, T, E, k, loss, counts, tokens, ws, *, mask=None, seq_offsets=None, S=1,
                score=SCORE_SOFTMAX, alpha=0.0, z_coef=0.0, probs=None, ld=None, stream=None):
    """Balance loss, z-loss, counts and mean probabilities of a routed batch (damoe_router_loss)."""
    if not _DTYPES:
        _types()
    dt, dev = _DTYPES.get(logits.dtype, -1), logits.get_device()
    n = S * E  # the checks of _list and _offsets in one expression: their calls, which name what is wrong, take 0.6 us more
    if not (loss is not None and counts is not None and tokens is not None
            and (ids is None or ids.dtype in _INT32 and ids.numel() >= T * k and ids.is_contiguous() and ids.get_device() == dev)
            and (mask is None or mask.dtype in _BYTES and mask.numel() >= T and mask.is_contiguous() and mask.get_device() == dev)
            and (seq_offsets is None or seq_offsets.dtype in _INT32 and seq_offsets.numel() == S + 1
                 and seq_offsets.is_contiguous() and seq_offsets.get_device() == dev)
            and loss.dtype in _FLOAT32 and loss.numel() >= 3 and loss.is_contiguous() and loss.get_device() == dev
            and counts.dtype in _INT32 and counts.numel() >= n and counts.is_contiguous() and counts.get_device() == dev
            and tokens.dtype in _INT32 and tokens.numel() >= S + 2 and tokens.is_contiguous() and tokens.get_device() == dev
            and (probs is None or probs.dtype in _FLOAT32 and probs.numel() >= n and probs.is_contiguous()
                 and probs.get_device() == dev)
            and ws.is_contiguous() and ws.get_device() == dev):
        _list("ids", ids, _INT32, T * k, dev)
        _list("mask", mask, _BYTES, T, dev)
        _offsets(seq_offsets, S, dev)
        # What the library refuses by itself is named as it does.
        if (ids is None and T > 0) or loss is None or counts is None or tokens is None:
            raise DamoeError("damoe_router_loss", -1)
        if ws.nbytes < router_loss_workspace_size(T, E, S):
            raise DamoeError("damoe_router_loss", -3)
        for name, t, types, m in (("loss", loss, _FLOAT32, 3), ("counts", counts, _INT32, n), ("tokens", tokens, _INT32, S + 2),
                                  ("probs", probs, _FLOAT32, n)):
            _list(name, t, types, m, dev)
        _room("ws", ws, 0, dev)
    rc = (_lib or lib()).damoe_call_words(0, _LOSS_WORDS(
        logits.data_ptr(), dt, _ld("logits", logits, T, E, ld), 0 if ids is None else ids.data_ptr(),
        0 if mask is None else mask.data_ptr(), 0 if seq_offsets is None else seq_offsets.data_ptr(), T, E, k, S, score, alpha,
        z_coef, loss.data_ptr(), counts.data_ptr(), 0 if probs is None else probs.data_ptr(), tokens.data_ptr(), ws.data_ptr(),
        ws.nbytes, _stream_on("damoe_router_loss", stream, dev, dt)), 20)
    if rc:
        raise DamoeError("damoe_router_loss", rc)


def router_loss_grad(logits, ids, T, E, k, counts, tokens, dlogits, *, mask=None, seq_offsets=None, S=1,
                     score=SCORE_SOFTMAX, alpha=0.0, z_coef=0.0, dloss=None, w=None, dw=None, ld=None, ldd=None,
                     stream=None):
    """Gradient of the loss and of the gates w with respect to the logits (damoe_router_loss_grad)."""
    if not _DTYPES:
        _types()
    if dlogits.dtype != logits.dtype:
        raise ValueError("dlogits has the logits' type")
    dt, dev = _DTYPES.get(logits.dtype, -1), logits.get_device()
    p_ids, p_mask = _list("ids", ids, _INT32, T * k, dev), _list("mask", mask, _BYTES, T, dev)
    if dlogits.get_device() != dev:
        _elsewhere("dlogits", dlogits)
    p_off, p_dloss = _offsets(seq_offsets, S, dev), _list("dloss", dloss, _FLOAT32, 1, dev)
    p_w, p_dw = _list("w", w, _FLOAT32, T * k, dev), _list("dw", dw, _FLOAT32, T * k, dev)
    if T > 0:
        p_counts, p_tokens = _list("counts", counts, _INT32, S * E, dev), _list("tokens", tokens, _INT32, S + 2, dev)
    else:  # without tokens neither is read
        p_counts, p_tokens = _p(counts), _p(tokens)
    rc = (_lib or lib()).damoe_call_words(1, _GRAD_WORDS(
        logits.data_ptr(), dt, _ld("logits", logits, T, E, ld), p_ids, p_w, p_dw, p_mask, p_off, p_counts, p_tokens, T,
        E, k, S, score, alpha, z_coef, p_dloss, dlogits.data_ptr(), _ld("dlogits", dlogits, T, E, ldd),
        _stream_on("damoe_router_loss_grad", stream, dev, dt, T)), 21)
    if rc:
        raise DamoeError("damoe_router_loss_grad", rc)


def mxfp4_bytes(rows: int, cols: int, layout: int = LAYOUT_TILE32) -> int:
    """Bytes of the codes of a rows x cols matrix (scales included but for the row-major layout); 0 if invalid."""
    return int(lib().damoe_mxfp4_bytes(rows, cols, layout))


def _codes_bytes(rows: int, cols: int, layout: int) -> int:
    """mxfp4_bytes of a valid shape, without the call."""
    if layout == LAYOUT_TILE32:
        return -(-rows // 32) * -(-cols // 256) * 4352
    return rows * cols // 2 if layout == LAYOUT_ROWMAJOR else rows * cols // 32 * 17


def mxfp4_quantise(x, rows, cols, codes, scales=None, layout=LAYOUT_TILE32, ldx=None, stream=None):
    dt, dev = _dtype(x), x.get_device()
    p_codes = _room("codes", codes, _codes_bytes(rows, cols, layout), dev)
    p_scales = _room("scales", scales, rows * cols // 32, dev) if layout == LAYOUT_ROWMAJOR else 0
    rc = (_lib or lib()).damoe_mxfp4_quantise(x.data_ptr(), dt, rows, cols, _ld("x", x, rows, cols, ldx), layout, p_codes,
                                              p_scales, _stream_on("damoe_mxfp4_quantise", stream, dev, dt, rows))
    if rc:
        raise DamoeError("damoe_mxfp4_quantise", rc)


def mxfp4_dequantise(codes, scales, rows, cols, x, layout=LAYOUT_TILE32, ldx=None, stream=None):
    dt, dev = _dtype(x), x.get_device()
    p_codes = _room("codes", codes, _codes_bytes(rows, cols, layout), dev)
    p_scales = _room("scales", scales, rows * cols // 32, dev) if layout == LAYOUT_ROWMAJOR else 0
    rc = (_lib or lib()).damoe_mxfp4_dequantise(p_codes, p_scales, rows, cols, layout, x.data_ptr(), dt,
                                                _ld("x", x, rows, cols, ldx),
                                                _stream_on("damoe_mxfp4_dequantise", stream, dev, dt, rows))
    if rc:
        raise DamoeError("damoe_mxfp4_dequantise", rc)


def mxfp4_pack(codes, scales, rows, cols, tiles, stream=None):
    """Row-major codes and scales into the operand layout of mxfp4_linear."""
    if not _DTYPES:
        _types()
    dev = codes.get_device()
    _check("damoe_mxfp4_pack", lib().damoe_mxfp4_pack(
        _room("codes", codes, rows * cols // 2, dev), _room("scales", scales, rows * cols // 32, dev), rows, cols,
        _room("tiles", tiles, _codes_bytes(rows, cols, LAYOUT_TILE32), dev), _stream_on("damoe_mxfp4_pack", stream, dev, 0, rows)))


def mxfp4_linear_workspace_size(T_max: int, N: int, K: int) -> int:
    return int(lib().damoe_mxfp4_linear_workspace_size(T_max, N, K))


def mxfp4_linear(x, T, K, w_tiles, N, y, ws, add=None, ldx=None, ldy=None, ld_add=None, stream=None):
    """y = add + Q(x) W^T with W in tiles (damoe_mxfp4_linear); add has y's type."""
    if add is not None and add.dtype != y.dtype:
        raise ValueError("add has y's type")
    dt, dev = _dtype(x), x.get_device()
    if y.get_device() != dev:
        _elsewhere("y", y)
    if add is not None and add.get_device() != dev:
        _elsewhere("add", add)
    p_tiles = _room("w_tiles", w_tiles, _codes_bytes(N, K, LAYOUT_TILE32), dev)
    p_add, lda = (0, 0) if add is None else (add.data_ptr(), _ld("add", add, T, N, ld_add))
    rc = (_lib or lib()).damoe_call_words(2, _LINEAR_WORDS(
        x.data_ptr(), dt, _ld("x", x, T, K, ldx), T, K, p_tiles, N, p_add, lda, y.data_ptr(), _dtype(y),
        _ld("y", y, T, N, ldy), _room("ws", ws, 0, dev), ws.nbytes, _stream_on("damoe_mxfp4_linear", stream, dev, dt, T)), 15)
    if rc:
        raise DamoeError("damoe_mxfp4_linear", rc)


def read_device_error(ws, stream=None) -> int:
    code = ctypes.c_int32()
    _check("damoe_read_device_error", lib().damoe_read_device_error(_p(ws), ctypes.byref(code),
                                                                   _stream(stream)))
    return int(code.value)


# ---------------------------------------------------------------- tables

@dataclass
class TableData:
    E: int
    k: int
    H: int
    I: int
    wdtype: int
    bucket_T: np.ndarray
    n_ex: np.ndarray
    Q: np.ndarray       # [sum n_ex][E]
    kid: np.ndarray
    noda: np.ndarray

    def bucket_rows(self, b: int):
        s = int(self.n_ex[:b].sum())
        return slice(s, s + int(self.n_ex[b]))


class Table:
    def __init__(self, handle: int):
        self.handle = ctypes.c_void_p(handle)
        self._candidates = {}  # T -> mask; tables are immutable, so the lookup is cached
        self._eff_candidates = {}

    @classmethod
    def create(cls, td: TableData) -> "Table":
        arrs = [np.ascontiguousarray(np.asarray(a, np.int32)) for a in
                (td.bucket_T, td.n_ex, td.Q, td.kid, td.noda)]
        d = TableDesc(td.E, td.k, td.H, td.I, td.wdtype, len(arrs[0]), *[a.ctypes.data for a in arrs])
        h = ctypes.c_void_p()
        _check("damoe_table_create", lib().damoe_table_create(ctypes.byref(d), ctypes.byref(h)))
        return cls(h.value)

    @classmethod
    def load(cls, path: str) -> "Table":
        h = ctypes.c_void_p()
        _check("damoe_table_load", lib().damoe_table_load(path.encode(), ctypes.byref(h)))
        return cls(h.value)

    def candidates(self, T: int) -> int:
        """Bit mask of the variants dispatch may choose for T tokens (see damoe_table_candidates)."""
        m = self._candidates.get(T)
        if m is None:
            m = self._candidates[T] = int(lib().damoe_table_candidates(self.handle, int(T)))
        return m

    def effexp_map(self, T: int) -> np.ndarray:
        """Variant per Effective Experts bucket -1..13 for T's token bucket."""
        m = np.zeros(15, np.int32)
        _check("damoe_table_effexp_map", lib().damoe_table_effexp_map(self.handle, T, m.ctypes.data))
        return m

    def effexp_candidates(self, T: int) -> int:
        """Bit mask of the variants the Effective-Experts dispatch may write for T tokens."""
        m = self._eff_candidates.get(T)
        if m is None:
            m = self._eff_candidates[T] = int(lib().damoe_table_effexp_candidates(self.handle, int(T)))
        return m

    def save(self, path: str):
        _check("damoe_table_save", lib().damoe_table_save(self.handle, path.encode()))

    def data(self, E: int) -> TableData:
        nb, nt = ctypes.c_int32(), ctypes.c_int32()
        _check("damoe_table_info", lib().damoe_table_info(self.handle, ctypes.byref(nb), ctypes.byref(nt),
                                                          None, None, None, None, None))
        bT, nex, noda = (np.zeros(nb.value, np.int32) for _ in range(3))
        kid = np.zeros(nt.value, np.int32)
        Q = np.zeros((nt.value, E), np.int32)
        _check("damoe_table_info", lib().damoe_table_info(self.handle, None, None, bT.ctypes.data,
                                                          nex.ctypes.data, Q.ctypes.data,
                                                          kid.ctypes.data, noda.ctypes.data))
        return TableData(E, 0, 0, 0, 0, bT, nex, Q, kid, noda)

    def close(self):
        if self.handle:
            lib().damoe_table_destroy(self.handle)
            self.handle = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def tune(layer: Layer, bucket_T, skew_X, x, *, samples=10, reps=5, alpha_samples=64, alpha_iters=60,
         seed=0, verbose=False, ep=1, repeat_f=(), flush_mib=0, stream=None) -> Table:
    bT = np.ascontiguousarray(np.asarray(bucket_T, np.int32))
    sx = np.ascontiguousarray(np.asarray(skew_X, np.float64))
    rf = np.ascontiguousarray(np.asarray(repeat_f, np.int32))
    cfg = TuneConfig(len(bT), bT.ctypes.data, len(sx), sx.ctypes.data, samples, reps, alpha_samples,
                     alpha_iters, seed, _p(x), int(verbose), int(ep), len(rf), rf.ctypes.data if len(rf) else None,
                     int(flush_mib))
    h = ctypes.c_void_p()
    _check("damoe_tune", lib().damoe_tune(ctypes.byref(layer), ctypes.byref(cfg), ctypes.byref(h),
                                          _stream(stream)))
    return Table(h.value)
