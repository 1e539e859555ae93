"""B200-native activation compress / decompress (the DAF hot path): thin Python binding.

Every function here only marshals arguments for the C ABI declared in ``include/daf.h``
(``libdaf.so``, hand-written sm_100a kernels), in Python through ctypes or, for the operators of a transformer's step, in the
compiled module ``_marshal`` (``csrc/marshal.cpp``).  PyTorch supplies device memory and streams;
all arithmetic of the path runs in the CUDA library.  There is no CPU fallback: if the
library is missing or fails to load, the first call raises.
"""
from __future__ import annotations

import ctypes
import importlib
import os
from dataclasses import dataclass

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdaf.so")

OK, ERR_INVALID_ARG, ERR_SHAPE, ERR_BUDGET, ERR_CAPACITY, ERR_CUDA, ERR_TIMEOUT, ERR_UNSUPPORTED = range(8)
F32, F16, BF16 = 0, 1, 2
ROUND_STOCHASTIC, ROUND_NEAREST = 0, 1
FLAG_STREAM_ALWAYS, FLAG_STREAM_NEVER, FLAG_KEEP_WORKSPACE, FLAG_ONE_PASS, FLAG_TWO_PASS = 1, 2, 4, 8, 16


# daf_params.flags used by make_params when the caller gives none (the GPU tests set FLAG_STREAM_ALWAYS here so
# that their small tensors still go through both compress kernels).
DEFAULT_FLAGS = 0


def flag_poll_limit(n: int) -> int:
    """daf_params.flags value that makes bounded device-side waits give up after n polls (diagnostic)."""
    return int(n) << 8

BATCH_MAX = 64
DEFAULT_WINDOW = 16384


class daf_params(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_uint32), ("numel", ctypes.c_uint64),
                ("group_size", ctypes.c_uint32), ("window_elems", ctypes.c_uint32), ("width_mask", ctypes.c_uint32),
                ("bit_budget", ctypes.c_float), ("rounding", ctypes.c_uint32), ("flags", ctypes.c_uint32),
                ("seed", ctypes.c_uint64), ("elem_index_base", ctypes.c_uint64)]


class daf_pool_stats(ctypes.Structure):
    _fields_ = [(n, ctypes.c_uint64) for n in ("arena_bytes", "page_bytes", "pages_total", "pages_used",
                                               "live_allocations", "bytes_requested", "largest_free_run_pages",
                                               "evictions")]


class daf_store_config(ctypes.Structure):
    _fields_ = [("mem_budget_bytes", ctypes.c_uint64), ("time_budget", ctypes.c_double), ("page_bytes", ctypes.c_uint64),
                ("step_bytes", ctypes.c_uint64), ("width_mask", ctypes.c_uint32), ("reserved", ctypes.c_uint32)]


class daf_store_move(ctypes.Structure):
    _fields_ = [(n, ctypes.c_uint64) for n in ("id", "from_offset", "to_offset", "bytes")]


class daf_store_stats(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_uint64) for n in ("arena_bytes", "mem_budget_bytes", "used_bytes", "planned_bytes")]
                + [("time_budget", ctypes.c_double), ("used_time", ctypes.c_double)]
                + [(n, ctypes.c_uint64) for n in ("entries", "kept", "evictions", "resizes", "grows", "shrinks", "moves")])


_u64x3 = ctypes.c_uint64 * 3


class daf_attention_params(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_uint32) for n in ("struct_size", "dtype", "batch", "queries", "keys", "heads", "kv_heads", "head_dim",
                                                "causal")]
                + [("scale", ctypes.c_float), ("reserved", ctypes.c_uint32 * 2)]
                + [(n, _u64x3) for n in ("q_stride", "k_stride", "v_stride", "out_stride", "grad_out_stride", "grad_q_stride",
                                         "grad_k_stride", "grad_v_stride")])


class daf_norm_params(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_uint32), ("param_dtype", ctypes.c_uint32),
                ("kind", ctypes.c_uint32), ("rows", ctypes.c_uint64), ("width", ctypes.c_uint32), ("gates", ctypes.c_uint32),
                ("residual_scale", ctypes.c_float), ("eps", ctypes.c_float), ("reserved", ctypes.c_uint32)]


class daf_embedding_params(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_uint32), ("table_dtype", ctypes.c_uint32),
                ("token_bytes", ctypes.c_uint32), ("tokens", ctypes.c_uint64), ("vocabulary", ctypes.c_uint64), ("width", ctypes.c_uint32),
                ("scale", ctypes.c_float), ("padding", ctypes.c_int64), ("reserved", ctypes.c_uint64)]


class daf_rotary_params(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_uint32) for n in ("struct_size", "dtype", "param_dtype", "style", "batch", "tokens", "heads", "kv_heads",
                                                "head_dim", "rotary_dim", "position_bytes", "shared_positions")]
                + [("first_position", ctypes.c_int64), ("base", ctypes.c_double), ("eps", ctypes.c_float), ("reserved", ctypes.c_uint32 * 3)]
                + [(n, _u64x3) for n in ("q_stride", "k_stride", "q_out_stride", "k_out_stride", "grad_q_stride", "grad_k_stride")])


class daf_orthogonalize_params(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("steps", ctypes.c_uint32), ("coefficients", ctypes.c_float * 3), ("eps", ctypes.c_float),
                ("reserved", ctypes.c_uint32 * 2)]


class DafError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().daf_status_string(status).decode() if _lib is not None else str(status)
        super().__init__(f"{where}: {msg} (status {status})")


_lib = None
_u64p = ctypes.POINTER(ctypes.c_uint64)
_vp = ctypes.c_void_p

# name -> (restype, argtypes): every symbol include/daf.h declares
SIGNATURES = {
    "daf_sizes": (ctypes.c_int, [ctypes.POINTER(daf_params), _u64p, _u64p, _u64p, _u64p]),
    "daf_shard": (ctypes.c_int, [ctypes.POINTER(daf_params), ctypes.c_uint32, ctypes.c_uint32, ctypes.POINTER(daf_params), _u64p]),
    "daf_compress": (ctypes.c_int, [ctypes.POINTER(daf_params), _vp, _vp, ctypes.c_uint64, _vp, _vp, _vp, _vp, _vp,
                                    ctypes.c_uint64, _vp]),
    "daf_relu_compress": (ctypes.c_int, [ctypes.POINTER(daf_params), _vp, _vp, _vp, ctypes.c_uint64, _vp, _vp, _vp, _vp, _vp,
                                         ctypes.c_uint64, _vp]),
    "daf_act_compress": (ctypes.c_int, [ctypes.POINTER(daf_params), ctypes.c_uint32, _vp, _vp, _vp, ctypes.c_uint64, _vp, _vp,
                                        _vp, _vp, _vp, ctypes.c_uint64, _vp]),
    "daf_decompress_act_grad": (ctypes.c_int, [ctypes.POINTER(daf_params), ctypes.c_uint32, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                               _vp]),
    "daf_compress_static": (ctypes.c_int, [ctypes.POINTER(daf_params), _vp, _vp, ctypes.c_uint64, _vp, _vp, _vp, _vp, _vp, _vp]),
    "daf_decompress": (ctypes.c_int, [ctypes.POINTER(daf_params), _vp, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_uint64, _vp]),
    "daf_decompress_relu_grad": (ctypes.c_int, [ctypes.POINTER(daf_params), _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "daf_group_offsets": (ctypes.c_int, [_vp, ctypes.c_uint64, ctypes.c_uint32, _vp, _vp, ctypes.c_uint64, _vp]),
    "daf_group_offsets_diag": (ctypes.c_int, [_vp, ctypes.c_uint64, ctypes.c_uint32, _vp, _vp, ctypes.c_uint64, ctypes.c_uint32,
                                              _vp]),
    "daf_group_offsets_workspace": (ctypes.c_uint64, [ctypes.c_uint64]),
    "daf_poll_status": (ctypes.c_int, [_vp, _vp]),
    "daf_batch_workspace": (ctypes.c_uint64, [ctypes.c_uint32, ctypes.POINTER(daf_params)]),
    "daf_compress_batch": (ctypes.c_int, [ctypes.c_uint32, ctypes.POINTER(daf_params), _vp, _vp, _u64p, _vp, _vp, _vp, _vp,
                                          _vp, ctypes.c_uint64, _vp]),
    "daf_decompress_batch": (ctypes.c_int, [ctypes.c_uint32, ctypes.POINTER(daf_params), _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "daf_tensor_minmax": (ctypes.c_int, [ctypes.c_uint32, _vp, ctypes.c_uint64, _vp, _vp]),
    "daf_tensor_compress": (ctypes.c_int, [ctypes.c_uint32, _vp, ctypes.c_uint64, ctypes.c_uint32, ctypes.c_uint32,
                                           ctypes.c_uint64, ctypes.c_uint64, _vp, _vp, _vp, _vp]),
    "daf_tensor_decompress": (ctypes.c_int, [ctypes.c_uint32, _vp, ctypes.c_uint64, ctypes.c_uint32, _vp, _vp, _vp]),
    "daf_device_status": (ctypes.c_int, [_vp]),
    "daf_device_status_word": (ctypes.c_int, [ctypes.POINTER(_vp)]),
    "daf_attention": (ctypes.c_int, [ctypes.POINTER(daf_attention_params)] + [_vp] * 7 + [ctypes.c_uint64, _vp]),
    "daf_attention_workspace": (ctypes.c_uint64, [ctypes.POINTER(daf_attention_params)]),
    "daf_attention_grad_workspace": (ctypes.c_uint64, [ctypes.POINTER(daf_attention_params)]),
    "daf_attention_grad": (ctypes.c_int, [ctypes.POINTER(daf_attention_params)] + [_vp] * 11 + [ctypes.c_uint64, _vp]),
    "daf_residual_norm": (ctypes.c_int, [ctypes.POINTER(daf_norm_params)] + [_vp] * 10),
    "daf_residual_norm_grad_workspace": (ctypes.c_uint64, [ctypes.POINTER(daf_norm_params)]),
    "daf_residual_norm_grad": (ctypes.c_int, [ctypes.POINTER(daf_norm_params)] + [_vp] * 16 + [ctypes.c_uint64, _vp]),
    "daf_clip_norm_workspace": (ctypes.c_uint64, [ctypes.c_uint32]),
    "daf_clip_norm_batch": (ctypes.c_int, [ctypes.c_uint32, _vp, _vp, _vp, _vp, ctypes.c_float, ctypes.c_float, _vp, _vp,
                                           ctypes.c_uint64, _vp]),
    "daf_embedding": (ctypes.c_int, [ctypes.POINTER(daf_embedding_params)] + [_vp] * 4),
    "daf_embedding_workspace": (ctypes.c_uint64, [ctypes.POINTER(daf_embedding_params)]),
    "daf_embedding_checked": (ctypes.c_int, [ctypes.POINTER(daf_embedding_params)] + [_vp] * 4 + [ctypes.c_uint64, _vp]),
    "daf_embedding_grad_workspace": (ctypes.c_uint64, [ctypes.POINTER(daf_embedding_params)]),
    "daf_embedding_grad": (ctypes.c_int, [ctypes.POINTER(daf_embedding_params)] + [_vp] * 4 + [ctypes.c_uint64, _vp]),
    "daf_rotary_norm": (ctypes.c_int, [ctypes.POINTER(daf_rotary_params)] + [_vp] * 9),
    "daf_rotary_norm_grad_workspace": (ctypes.c_uint64, [ctypes.POINTER(daf_rotary_params)]),
    "daf_rotary_norm_grad": (ctypes.c_int, [ctypes.POINTER(daf_rotary_params)] + [_vp] * 13 + [ctypes.c_uint64, _vp]),
    "daf_orthogonalize_workspace": (ctypes.c_uint64, [ctypes.POINTER(daf_orthogonalize_params), ctypes.c_uint32, _vp, _vp, _vp]),
    "daf_orthogonalize": (ctypes.c_int, [ctypes.POINTER(daf_orthogonalize_params), ctypes.c_uint32] + [_vp] * 6 + [ctypes.c_uint64, _vp]),
    "daf_pool_create": (_vp, [ctypes.c_uint64, ctypes.c_uint64]),
    "daf_pool_destroy": (None, [_vp]),
    "daf_pool_alloc": (ctypes.c_uint64, [_vp, ctypes.c_uint64, ctypes.c_double, _u64p]),
    "daf_pool_free": (ctypes.c_int, [_vp, ctypes.c_uint64]),
    "daf_pool_evict_lowest": (ctypes.c_uint64, [_vp]),
    "daf_pool_get_stats": (ctypes.c_int, [_vp, ctypes.POINTER(daf_pool_stats)]),
    "daf_store_bytes": (ctypes.c_uint64, [ctypes.c_uint64, ctypes.c_uint32, ctypes.c_uint32]),
    "daf_store_create": (_vp, [ctypes.POINTER(daf_store_config)]),
    "daf_store_destroy": (None, [_vp]),
    "daf_store_estimate": (ctypes.c_int, [_vp, ctypes.c_uint64, ctypes.c_uint64, ctypes.c_uint32, ctypes.c_double,
                                          ctypes.c_double, ctypes.POINTER(ctypes.c_uint32), _u64p,
                                          ctypes.POINTER(ctypes.c_uint32)]),
    "daf_store_admit": (ctypes.c_int, [_vp, ctypes.c_uint64, ctypes.c_double, ctypes.POINTER(ctypes.c_uint32), _u64p, _u64p,
                                       ctypes.POINTER(ctypes.c_uint32)]),
    "daf_store_width": (ctypes.c_int, [_vp, ctypes.c_uint64, ctypes.POINTER(ctypes.c_uint32), _u64p]),
    "daf_store_release": (ctypes.c_int, [_vp, ctypes.c_uint64]),
    "daf_store_set_budget": (ctypes.c_int, [_vp, ctypes.c_uint64, ctypes.c_double, ctypes.POINTER(daf_store_move),
                                            ctypes.POINTER(ctypes.c_uint32), _u64p, ctypes.POINTER(ctypes.c_uint32)]),
    "daf_store_get_stats": (ctypes.c_int, [_vp, ctypes.POINTER(daf_store_stats)]),
    "daf_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "daf_version": (ctypes.c_uint32, []),
}


def lib() -> ctypes.CDLL:
    """The loaded C-ABI library; raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2507_07149_b200.build` "
                               "(nvcc, sm_100a); there is no CPU fallback")
        handle = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype, fn.argtypes = res, args
        _lib = handle
    return _lib


def _check(status: int, where: str):
    if status != OK:
        raise DafError(status, where)


# ------------------------------------------------------------------------------------ params / sizes
def width_mask(widths) -> int:
    m = 0
    for b in widths:
        m |= 1 << int(b)
    return m


def make_params(dtype: int, numel: int, group_size: int, widths, bit_budget: float, *, window_elems: int = 0,
                rounding: int = ROUND_STOCHASTIC, seed: int = 0, elem_index_base: int = 0,
                flags: int | None = None) -> daf_params:
    if flags is None:
        flags = DEFAULT_FLAGS
    return daf_params(ctypes.sizeof(daf_params), dtype, numel, group_size, window_elems, width_mask(widths),
                      bit_budget, rounding, flags, seed, elem_index_base)


@dataclass
class Sizes:
    n_groups: int
    n_windows: int
    packed_capacity: int
    workspace: int


def daf_sizes(params: daf_params) -> Sizes:
    v = [ctypes.c_uint64() for _ in range(4)]
    _check(lib().daf_sizes(ctypes.byref(params), *[ctypes.byref(x) for x in v]), "daf_sizes")
    return Sizes(*[int(x.value) for x in v])


def daf_shard(params: daf_params, rank: int, world: int):
    """(parameters of rank's window-aligned slice, its first element); the slice's numel is 0 when there is none."""
    shard, first = daf_params(), ctypes.c_uint64()
    _check(lib().daf_shard(ctypes.byref(params), rank, world, ctypes.byref(shard), ctypes.byref(first)), "daf_shard")
    return shard, int(first.value)


def _torch():
    import torch
    return torch


_codes = {}


def _dtype_codes() -> dict:
    """torch dtype -> daf_dtype."""
    if not _codes:
        torch = _torch()
        _codes.update({torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16})
    return _codes


def dtype_code(t) -> int:
    return _dtype_codes()[t.dtype]


def _raw_stream(index: int, stream) -> int:
    """The cudaStream_t of `stream`, or of torch's current stream of device `index`."""
    if stream is not None:
        return stream.cuda_stream
    torch = _torch()
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)       # the same without a Stream object
    return raw(index) if raw is not None else torch.cuda.current_stream(index).cuda_stream


def _call(fn, ref, stream, *args) -> int:
    """Calls fn(*args, stream) with the device of tensor `ref` current in this thread (the library launches on the
    current device) and, unless a stream is given, on torch's current stream OF THAT DEVICE.  Returns the status."""
    torch = _torch()
    index = ref.get_device()
    if index < 0:                                                    # torch would take -1 for the current device
        raise ValueError(f"expected a CUDA tensor, got one on {ref.device}")
    raw = _raw_stream(index, stream)
    if index == torch._C._cuda_getDevice():
        return int(fn(*args, raw))
    with torch.cuda.device(index):
        return int(fn(*args, raw))


def _ptr(t) -> int:
    return 0 if t is None else int(t.data_ptr())


# ------------------------------------------------------------------------------------ raw entry points
def daf_compress(params, d_in, d_packed, packed_capacity, d_bits, d_min, d_scale, d_window_offsets, d_workspace,
                 workspace_bytes, stream=None):
    """Tensors (or None) in, status checked; everything else is the C call."""
    status = _call(lib().daf_compress, d_in, stream, ctypes.byref(params), _ptr(d_in), _ptr(d_packed),
                   packed_capacity, _ptr(d_bits), _ptr(d_min), _ptr(d_scale), _ptr(d_window_offsets),
                   _ptr(d_workspace), workspace_bytes)
    _check(status, "daf_compress")


def daf_relu_compress(params, d_in, d_act, d_packed, packed_capacity, d_bits, d_min, d_scale, d_window_offsets, d_workspace,
                      workspace_bytes, stream=None):
    """Fused producer: d_act = max(d_in, +0) is written and compressed in one pass (d_act may be d_in)."""
    status = _call(lib().daf_relu_compress, d_in, stream, ctypes.byref(params), _ptr(d_in), _ptr(d_act),
                   _ptr(d_packed), packed_capacity, _ptr(d_bits), _ptr(d_min), _ptr(d_scale), _ptr(d_window_offsets),
                   _ptr(d_workspace), workspace_bytes)
    _check(status, "daf_relu_compress")


ACT_RELU, ACT_RELU6, ACT_GELU = 1, 2, 3


def daf_act_compress(params, act, d_in, d_act, d_packed, packed_capacity, d_bits, d_min, d_scale, d_window_offsets, d_workspace,
                     workspace_bytes, stream=None):
    """Fused producer for ReLU / ReLU6 / GELU: d_act = act(d_in) written in the same pass that compresses (the
    activation for ReLU and ReLU6, the input for GELU)."""
    status = _call(lib().daf_act_compress, d_in, stream, ctypes.byref(params), act, _ptr(d_in), _ptr(d_act),
                   _ptr(d_packed), packed_capacity, _ptr(d_bits), _ptr(d_min), _ptr(d_scale), _ptr(d_window_offsets),
                   _ptr(d_workspace), workspace_bytes)
    _check(status, "daf_act_compress")


def daf_decompress_act_grad(params, act, d_packed, d_bits, d_min, d_scale, d_window_offsets, d_grad_out, d_grad_in, stream=None):
    """Fused consumer: the gradient of the activation from its compressed form (may be in place)."""
    status = _call(lib().daf_decompress_act_grad, d_grad_out, stream, ctypes.byref(params), act, _ptr(d_packed),
                   _ptr(d_bits), _ptr(d_min), _ptr(d_scale), _ptr(d_window_offsets), _ptr(d_grad_out),
                   _ptr(d_grad_in))
    _check(status, "daf_decompress_act_grad")


STATIC_MAX_WINDOWS = 65536


def daf_compress_static(params, d_in, d_packed, packed_capacity, d_bits, d_min, d_scale, d_window_offsets, d_status=None,
                        stream=None):
    """daf_compress for callers that cannot allocate a workspace: the kernel's scratch is a fixed
    array inside the library (at most STATIC_MAX_WINDOWS windows; calls must not overlap on the GPU).
    d_status: optional int32 tensor of one element that receives the device status word."""
    status = _call(lib().daf_compress_static, d_in, stream, ctypes.byref(params), _ptr(d_in), _ptr(d_packed),
                   packed_capacity, _ptr(d_bits), _ptr(d_min), _ptr(d_scale), _ptr(d_window_offsets), _ptr(d_status))
    _check(status, "daf_compress_static")


def daf_decompress_relu_grad(params, d_packed, d_bits, d_min, d_scale, d_window_offsets, d_grad_out, d_grad_in, stream=None):
    """Fused consumer: d_grad_in = d_grad_out where the restored activation is > 0, else 0 (may be in place)."""
    status = _call(lib().daf_decompress_relu_grad, d_grad_out, stream, ctypes.byref(params), _ptr(d_packed),
                   _ptr(d_bits), _ptr(d_min), _ptr(d_scale), _ptr(d_window_offsets), _ptr(d_grad_out),
                   _ptr(d_grad_in))
    _check(status, "daf_decompress_relu_grad")


def daf_decompress(params, d_packed, d_bits, d_min, d_scale, d_window_offsets, d_out, d_workspace=None,
                   workspace_bytes=0, stream=None):
    status = _call(lib().daf_decompress, d_out, stream, ctypes.byref(params), _ptr(d_packed), _ptr(d_bits),
                   _ptr(d_min), _ptr(d_scale), _ptr(d_window_offsets), _ptr(d_out), _ptr(d_workspace),
                   workspace_bytes)
    _check(status, "daf_decompress")


def daf_group_offsets_workspace(n_groups: int) -> int:
    return int(lib().daf_group_offsets_workspace(n_groups))


def daf_group_offsets(d_bits, n_groups, group_size, d_offsets, d_ws, ws_bytes, stream=None):
    status = _call(lib().daf_group_offsets, d_bits, stream, _ptr(d_bits), n_groups, group_size, _ptr(d_offsets),
                   _ptr(d_ws), ws_bytes)
    _check(status, "daf_group_offsets")


def daf_group_offsets_diag(d_bits, n_groups, group_size, d_offsets, d_ws, ws_bytes, flags, stream=None):
    """daf_group_offsets with diagnostic flags (FLAG_KEEP_WORKSPACE, flag_poll_limit(n)): for tests of the bounded wait."""
    status = _call(lib().daf_group_offsets_diag, d_bits, stream, _ptr(d_bits), n_groups, group_size, _ptr(d_offsets),
                   _ptr(d_ws), ws_bytes, flags)
    _check(status, "daf_group_offsets_diag")


def daf_poll_status(d_workspace, stream=None) -> int:
    return _call(lib().daf_poll_status, d_workspace, stream, _ptr(d_workspace))


def daf_device_status(device=None, stream=None) -> int:
    """The largest error that an operator's call on `device` (the current one) has recorded since the last such question."""
    torch = _torch()
    with torch.cuda.device(device):                                  # None: stays
        return int(lib().daf_device_status(_raw_stream(torch.cuda.current_device(), stream)))


def daf_device_status_word(device=None) -> int:
    """The device address of the word that daf_device_status reads."""
    word = _vp()
    with _torch().cuda.device(device):
        _check(int(lib().daf_device_status_word(ctypes.byref(word))), "daf_device_status_word")
    return word.value


def check_device(device=None, stream=None) -> None:
    """Waits for the stream and raises if an attention or orthogonalisation call on `device` gave up, or an embedding call met a
    token that is none, since the last question.  These calls do not wait for the device (unless called with check) and keep
    nothing that could be asked later, so ask here once a step or once an epoch."""
    _check(daf_device_status(device, stream), "operators (device status)")


def _ptr_array(tensors):
    return (ctypes.c_void_p * len(tensors))(*[_ptr(t) for t in tensors])


def daf_batch_workspace(params_list) -> int:
    arr = (daf_params * len(params_list))(*params_list)
    return int(lib().daf_batch_workspace(len(params_list), arr))


def daf_compress_batch(params_list, d_in, d_packed, capacities, d_bits, d_min, d_scale, d_window_offsets, d_workspace,
                       workspace_bytes, stream=None):
    n = len(params_list)
    arr = (daf_params * n)(*params_list)
    caps = (ctypes.c_uint64 * n)(*capacities)
    status = _call(lib().daf_compress_batch, d_in[0], stream, n, arr, _ptr_array(d_in), _ptr_array(d_packed), caps,
                   _ptr_array(d_bits), _ptr_array(d_min), _ptr_array(d_scale), _ptr_array(d_window_offsets),
                   _ptr(d_workspace), workspace_bytes)
    _check(status, "daf_compress_batch")


def daf_decompress_batch(params_list, d_packed, d_bits, d_min, d_scale, d_window_offsets, d_out, stream=None):
    n = len(params_list)
    arr = (daf_params * n)(*params_list)
    status = _call(lib().daf_decompress_batch, d_out[0], stream, n, arr, _ptr_array(d_packed), _ptr_array(d_bits),
                   _ptr_array(d_min), _ptr_array(d_scale), _ptr_array(d_window_offsets), _ptr_array(d_out))
    _check(status, "daf_decompress_batch")


def daf_version() -> int:
    return int(lib().daf_version())


def daf_status_string(status: int) -> str:
    return lib().daf_status_string(status).decode()


# ------------------------------------------------------------------------------------ conveniences (allocation only)
@dataclass
class CompressedTensor:
    """Device buffers written by daf_compress for one tensor (owned by torch)."""
    params: daf_params
    shape: tuple
    packed: object
    bits: object
    min: object
    scale: object
    window_offsets: object
    workspace: object
    sizes: Sizes

    def packed_bytes(self) -> int:
        return int(self.window_offsets[-1].item())


def alloc_outputs(params: daf_params, device, shape=None) -> CompressedTensor:
    torch = _torch()
    sz = daf_sizes(params)
    return CompressedTensor(
        params, tuple(shape) if shape is not None else (int(params.numel),),
        torch.empty(max(sz.packed_capacity, 16), dtype=torch.uint8, device=device),
        torch.empty(sz.n_groups, dtype=torch.uint8, device=device),
        torch.empty(sz.n_groups, dtype=torch.float32, device=device),
        torch.empty(sz.n_groups, dtype=torch.float32, device=device),
        torch.empty(sz.n_windows + 1, dtype=torch.int64, device=device),
        torch.empty(sz.workspace, dtype=torch.uint8, device=device), sz)


def compress(x, group_size: int, widths, bit_budget: float, *, window_elems: int = 0, rounding: int = ROUND_STOCHASTIC,
             seed: int = 0, elem_index_base: int = 0, flags: int | None = None, out: CompressedTensor | None = None,
             check: bool = False, stream=None) -> CompressedTensor:
    """Allocate outputs with torch (unless given) and call daf_compress on the current stream."""
    if not x.is_cuda or not x.is_contiguous():
        raise ValueError("compress expects a contiguous CUDA tensor")
    params = make_params(dtype_code(x), x.numel(), group_size, widths, bit_budget, window_elems=window_elems,
                         rounding=rounding, seed=seed, elem_index_base=elem_index_base, flags=flags)
    c = out if out is not None else alloc_outputs(params, x.device, x.shape)
    c.params = params
    daf_compress(params, x, c.packed, c.sizes.packed_capacity, c.bits, c.min, c.scale, c.window_offsets, c.workspace,
                 c.sizes.workspace, stream)
    if check:
        _check(daf_poll_status(c.workspace, stream), "daf_compress (device status)")
    return c


def relu_compress(x, group_size: int, widths, bit_budget: float, *, rounding: int = ROUND_STOCHASTIC, seed: int = 0,
                  elem_index_base: int = 0, flags: int | None = None, inplace: bool = False, out: CompressedTensor | None = None,
                  check: bool = False, stream=None, act: int = ACT_RELU):
    """(act(x), compressed form) in one pass over x (daf_act_compress); ``inplace`` overwrites x.  The compressed
    form holds act(x) for ReLU and ReLU6, and x itself for GELU."""
    if not x.is_cuda or not x.is_contiguous():
        raise ValueError("relu_compress expects a contiguous CUDA tensor")
    params = make_params(dtype_code(x), x.numel(), group_size, widths, bit_budget, rounding=rounding, seed=seed,
                         elem_index_base=elem_index_base, flags=flags)
    c = out if out is not None else alloc_outputs(params, x.device, x.shape)
    c.params = params
    y = x if inplace else _torch().empty_like(x)
    daf_act_compress(params, act, x, y, c.packed, c.sizes.packed_capacity, c.bits, c.min, c.scale, c.window_offsets,
                     c.workspace, c.sizes.workspace, stream)
    if check:
        _check(daf_poll_status(c.workspace, stream), "daf_act_compress (device status)")
    return y, c


def decompress(c: CompressedTensor, out=None, stream=None):
    torch = _torch()
    dt = {F32: torch.float32, F16: torch.float16, BF16: torch.bfloat16}[int(c.params.dtype)]
    if out is None:
        out = torch.empty(c.shape, dtype=dt, device=c.packed.device)
    daf_decompress(c.params, c.packed, c.bits, c.min, c.scale, c.window_offsets, out, None, 0, stream)
    return out


def relu_grad(c: CompressedTensor, grad_out, out=None, stream=None, act: int = ACT_RELU):
    """Gradient of the activation from its compressed form (daf_decompress_act_grad)."""
    torch = _torch()
    if not grad_out.is_contiguous():
        grad_out = grad_out.contiguous()
    if out is None:
        out = torch.empty_like(grad_out)
    daf_decompress_act_grad(c.params, act, c.packed, c.bits, c.min, c.scale, c.window_offsets, grad_out, out, stream)
    return out


# ------------------------------------------------------------------------------------ per-tensor path
def daf_tensor_minmax(d_in, d_stats, stream=None):
    """min, max and range of the whole tensor into d_stats (8 x 32-bit words on the device: floats 0-2, scratch 4-7)."""
    status = _call(lib().daf_tensor_minmax, d_in, stream, dtype_code(d_in), _ptr(d_in), d_in.numel(), _ptr(d_stats))
    _check(status, "daf_tensor_minmax")


def daf_tensor_compress(d_in, width, d_stats, d_packed, d_min_scale, *, rounding=ROUND_STOCHASTIC, seed=0, elem_index_base=0,
                        stream=None):
    status = _call(lib().daf_tensor_compress, d_in, stream, dtype_code(d_in), _ptr(d_in), d_in.numel(), width, rounding, seed,
                   elem_index_base, _ptr(d_stats), _ptr(d_packed), _ptr(d_min_scale))
    _check(status, "daf_tensor_compress")


def daf_tensor_decompress(d_packed, width, d_min_scale, d_out, stream=None):
    status = _call(lib().daf_tensor_decompress, d_out, stream, dtype_code(d_out), _ptr(d_packed), d_out.numel(), width,
                   _ptr(d_min_scale), _ptr(d_out))
    _check(status, "daf_tensor_decompress")


def tensor_compress(x, width: int, *, rounding: int = ROUND_STOCHASTIC, seed: int = 0, elem_index_base: int = 0, stream=None):
    """Eq. 1 with one min / max / width for the whole tensor: (packed uint8 tensor, min_scale float tensor, stats)."""
    torch = _torch()
    if not x.is_cuda or not x.is_contiguous():
        raise ValueError("tensor_compress expects a contiguous CUDA tensor")
    stats = torch.empty(8, dtype=torch.int32, device=x.device)
    packed = torch.empty(max(x.numel() * width // 8, 16), dtype=torch.uint8, device=x.device)
    min_scale = torch.empty(2, dtype=torch.float32, device=x.device)
    daf_tensor_minmax(x, stats, stream)
    daf_tensor_compress(x, width, stats, packed, min_scale, rounding=rounding, seed=seed, elem_index_base=elem_index_base,
                        stream=stream)
    return packed, min_scale, stats


def tensor_decompress(packed, width: int, min_scale, shape, dtype, stream=None):
    out = _torch().empty(shape, dtype=dtype, device=packed.device)
    daf_tensor_decompress(packed, width, min_scale, out, stream)
    return out


# ------------------------------------------------------------------------------------ operators of a transformer's step
NORM_LAYER, NORM_RMS = 0, 1


def daf_attention(params, d_q, d_k, d_v, d_key_lengths, d_out, d_lse, d_workspace, workspace_bytes, stream=None):
    status = _call(lib().daf_attention, d_q, stream, ctypes.byref(params), _ptr(d_q), _ptr(d_k), _ptr(d_v), _ptr(d_key_lengths),
                   _ptr(d_out), _ptr(d_lse), _ptr(d_workspace), workspace_bytes)
    _check(status, "daf_attention")


def daf_attention_workspace(params) -> int:
    return int(lib().daf_attention_workspace(ctypes.byref(params)))


def daf_attention_grad_workspace(params) -> int:
    return int(lib().daf_attention_grad_workspace(ctypes.byref(params)))


def daf_attention_grad(params, d_q, d_k, d_v, d_key_lengths, d_out, d_lse, d_grad_out, d_grad_q, d_grad_k, d_grad_v, d_workspace,
                       workspace_bytes, stream=None):
    status = _call(lib().daf_attention_grad, d_q, stream, ctypes.byref(params), _ptr(d_q), _ptr(d_k), _ptr(d_v),
                   _ptr(d_key_lengths), _ptr(d_out), _ptr(d_lse), _ptr(d_grad_out), _ptr(d_grad_q), _ptr(d_grad_k),
                   _ptr(d_grad_v), _ptr(d_workspace), workspace_bytes)
    _check(status, "daf_attention_grad")


def daf_residual_norm(params, d_x, d_y, d_weight, d_bias, d_gate, d_post_weight, d_post_bias, d_z, d_h, stream=None):
    status = _call(lib().daf_residual_norm, d_x, stream, ctypes.byref(params), _ptr(d_x), _ptr(d_y), _ptr(d_weight), _ptr(d_bias),
                   _ptr(d_gate), _ptr(d_post_weight), _ptr(d_post_bias), _ptr(d_z), _ptr(d_h))
    _check(status, "daf_residual_norm")


def daf_residual_norm_grad_workspace(params) -> int:
    return int(lib().daf_residual_norm_grad_workspace(ctypes.byref(params)))


def daf_residual_norm_grad(params, d_z, d_y, d_weight, d_gate, d_post_weight, d_post_bias, d_grad_z, d_grad_h, d_grad_x, d_grad_y,
                           d_grad_weight, d_grad_bias, d_grad_gate, d_grad_post_weight, d_grad_post_bias, d_workspace,
                           workspace_bytes, stream=None):
    status = _call(lib().daf_residual_norm_grad, d_z, stream, ctypes.byref(params), _ptr(d_z), _ptr(d_y), _ptr(d_weight),
                   _ptr(d_gate), _ptr(d_post_weight), _ptr(d_post_bias), _ptr(d_grad_z), _ptr(d_grad_h), _ptr(d_grad_x),
                   _ptr(d_grad_y), _ptr(d_grad_weight), _ptr(d_grad_bias), _ptr(d_grad_gate), _ptr(d_grad_post_weight),
                   _ptr(d_grad_post_bias), _ptr(d_workspace), workspace_bytes)
    _check(status, "daf_residual_norm_grad")


def daf_clip_norm_workspace(n: int) -> int:
    return int(lib().daf_clip_norm_workspace(n))


def daf_clip_norm_batch(d_in, d_out, max_norm, eps, d_norm, d_workspace, workspace_bytes, stream=None):
    """d_in, d_out: lists of tensors (d_out None: the norm alone)."""
    n = len(d_in)
    status = _call(lib().daf_clip_norm_batch, d_norm, stream, n, (ctypes.c_uint32 * n)(*[dtype_code(t) for t in d_in]),
                   _ptr_array(d_in), None if d_out is None else _ptr_array(d_out), (ctypes.c_uint64 * n)(*[t.numel() for t in d_in]),
                   max_norm, eps, _ptr(d_norm), _ptr(d_workspace), workspace_bytes)
    _check(status, "daf_clip_norm_batch")


def daf_embedding(params, d_tokens, d_weight, d_out, stream=None):
    _check(_call(lib().daf_embedding, d_out, stream, ctypes.byref(params), _ptr(d_tokens), _ptr(d_weight), _ptr(d_out)), "daf_embedding")


def daf_embedding_workspace(params) -> int:
    return int(lib().daf_embedding_workspace(ctypes.byref(params)))


def daf_embedding_checked(params, d_tokens, d_weight, d_out, d_workspace, workspace_bytes, stream=None):
    status = _call(lib().daf_embedding_checked, d_out, stream, ctypes.byref(params), _ptr(d_tokens), _ptr(d_weight), _ptr(d_out), _ptr(d_workspace),
                   workspace_bytes)
    _check(status, "daf_embedding_checked")


def daf_embedding_grad_workspace(params) -> int:
    return int(lib().daf_embedding_grad_workspace(ctypes.byref(params)))


def daf_embedding_grad(params, d_tokens, d_grad_out, d_grad_weight, d_workspace, workspace_bytes, stream=None):
    status = _call(lib().daf_embedding_grad, d_grad_weight, stream, ctypes.byref(params), _ptr(d_tokens), _ptr(d_grad_out),
                   _ptr(d_grad_weight), _ptr(d_workspace), workspace_bytes)
    _check(status, "daf_embedding_grad")


def _frequencies(params, frequencies):
    if frequencies is None:
        return None
    if len(frequencies) != params.rotary_dim // 2:                  # the library reads that many
        raise ValueError(f"frequencies: {len(frequencies)} of them, expected rotary_dim / 2 = {params.rotary_dim // 2}")
    return (ctypes.c_double * len(frequencies))(*frequencies)


def daf_rotary_norm(params, frequencies, d_q, d_k, d_q_weight, d_k_weight, d_positions, d_q_out, d_k_out, stream=None):
    """frequencies: rotary_dim / 2 numbers (ValueError if it is another count) or None, as for ``rotary_norm``."""
    status = _call(lib().daf_rotary_norm, d_q, stream, ctypes.byref(params), _frequencies(params, frequencies), _ptr(d_q), _ptr(d_k), _ptr(d_q_weight),
                   _ptr(d_k_weight), _ptr(d_positions), _ptr(d_q_out), _ptr(d_k_out))
    _check(status, "daf_rotary_norm")


def daf_rotary_norm_grad_workspace(params) -> int:
    return int(lib().daf_rotary_norm_grad_workspace(ctypes.byref(params)))


def daf_rotary_norm_grad(params, frequencies, d_q, d_k, d_q_weight, d_k_weight, d_positions, d_grad_q_out, d_grad_k_out, d_grad_q, d_grad_k,
                         d_grad_q_weight, d_grad_k_weight, d_workspace, workspace_bytes, stream=None):
    status = _call(lib().daf_rotary_norm_grad, d_q, stream, ctypes.byref(params), _frequencies(params, frequencies), _ptr(d_q), _ptr(d_k),
                   _ptr(d_q_weight), _ptr(d_k_weight), _ptr(d_positions), _ptr(d_grad_q_out), _ptr(d_grad_k_out), _ptr(d_grad_q),
                   _ptr(d_grad_k), _ptr(d_grad_q_weight), _ptr(d_grad_k_weight), _ptr(d_workspace), workspace_bytes)
    _check(status, "daf_rotary_norm_grad")


def _matrices(tensors):
    """Types, rows and columns of matrices (dimensions behind the first are one), as the C ABI takes them."""
    n = len(tensors)
    rows = [t.shape[0] for t in tensors]
    return ((ctypes.c_uint32 * n)(*[dtype_code(t) for t in tensors]), (ctypes.c_uint64 * n)(*rows),
            (ctypes.c_uint64 * n)(*[t.numel() // r if r else 0 for t, r in zip(tensors, rows)]))


def daf_orthogonalize_workspace(params, d_in) -> int:
    types, rows, cols = _matrices(d_in)
    return int(lib().daf_orthogonalize_workspace(ctypes.byref(params), len(d_in), types, rows, cols))


def daf_orthogonalize(params, d_in, d_out, d_workspace, workspace_bytes, stream=None):
    """d_in, d_out: lists of contiguous matrices, as many of one as of the other."""
    if len(d_out) != len(d_in):                                     # the library reads as many addresses
        raise ValueError(f"daf_orthogonalize: {len(d_out)} outputs for {len(d_in)} matrices")
    types, rows, cols = _matrices(d_in)
    status = _call(lib().daf_orthogonalize, d_workspace, stream, ctypes.byref(params), len(d_in), types, _ptr_array(d_in), _ptr_array(d_out), rows,
                   cols, _ptr(d_workspace), workspace_bytes)
    _check(status, "daf_orthogonalize")


_native_module = None


def _native():
    """The compiled marshalling module of the functions below; raises if it has not been built."""
    global _native_module
    if _native_module is None:
        lib()
        _torch()                                                     # its libraries are what the module links against
        try:
            _native_module = importlib.import_module("._marshal", __name__)
        except ImportError as e:
            raise RuntimeError(f"paper_2507_07149_b200/_marshal.so cannot be loaded ({e}): build it with "
                               "`python -m paper_2507_07149_b200.build`") from e
    return _native_module


def attention(q, k, v, *, causal: bool = False, scale: float | None = None, key_lengths=None, out=None, lse=None,
              check: bool = False, stream=None):
    """(out, lse): softmax attention of q [B, Sq, H, D] over k, v [B, Sk, Hkv, D] and the logarithm of each row's sum of
    exponentials [B, H, Sq] that the backward pass needs (daf_attention).  Slices of a packed projection are read in place;
    tensors the kernels cannot address (D not contiguous, rows off 16-byte boundaries, broadcast dimensions) are copied
    first.  scale: 1 / sqrt(D) by default; key_lengths: int32 [B]; causal: query i sees keys up to i + Sk - Sq.  check waits
    for the device and raises on an error there (without it, ``check_device`` tells later).  With a stream, results and scratch
    belong to that stream."""
    if stream is not None:
        with _torch().cuda.stream(stream):
            return attention(q, k, v, causal=causal, scale=scale, key_lengths=key_lengths, out=out, lse=lse, check=check)
    out, lse, status = _native().attention(q, k, v, key_lengths, out, lse, causal, scale, check)
    _check(status, "daf_attention")
    return out, lse


def attention_grad(q, k, v, out, lse, grad_out, *, causal: bool = False, scale: float | None = None, key_lengths=None, grads=None,
                   check: bool = False, stream=None):
    """(grad_q, grad_k, grad_v) of ``attention`` from its inputs, its two results and grad_out (daf_attention_grad).  grads:
    three tensors to write into (they may be slices of one packed gradient), fresh contiguous ones by default."""
    if stream is not None:
        with _torch().cuda.stream(stream):
            return attention_grad(q, k, v, out, lse, grad_out, causal=causal, scale=scale, key_lengths=key_lengths, grads=grads, check=check)
    gq, gk, gv = (None, None, None) if grads is None else grads
    gq, gk, gv, status = _native().attention_grad(q, k, v, out, lse, grad_out, key_lengths, gq, gk, gv, causal, scale, check)
    _check(status, "daf_attention_grad")
    return gq, gk, gv


_KINDS = {"layer": NORM_LAYER, "rms": NORM_RMS}


def _kind(where: str, kind: str) -> int:
    if kind not in _KINDS:
        raise ValueError(f"{where}: kind is 'layer' or 'rms'")
    return _KINDS[kind]


def residual_norm(x, y, weight, bias=None, *, gate=None, post_weight=None, post_bias=None, residual_scale: float = 1.0,
                  kind: str = "layer", eps: float = 1e-6, out=None, stream=None):
    """(z, h): z = x + residual_scale * gate * post_norm(y), h = norm(z) * weight + bias over the last dimension, in one pass
    (daf_residual_norm).  post_norm only with post_weight; gate [C], or [G, C] for G equal runs of rows; parameters in the
    activations' type or float32.  Tensors are contiguous; what does not start on the kernels' boundaries is copied first.  out:
    (z, h) to write into, z may be x and h may be y."""
    if stream is not None:
        with _torch().cuda.stream(stream):
            return residual_norm(x, y, weight, bias, gate=gate, post_weight=post_weight, post_bias=post_bias, residual_scale=residual_scale,
                                 kind=kind, eps=eps, out=out)
    z, h = (None, None) if out is None else out
    made_z, made_h, status = _native().residual_norm(x, y, weight, bias, gate, post_weight, post_bias, residual_scale,
                                                     _kind("residual_norm", kind), eps, z, h)
    _check(status, "daf_residual_norm")
    return (made_z, made_h) if out is None else (z, h)


def residual_norm_grad(z, y, weight, bias, grad_z, grad_h, *, gate=None, post_weight=None, post_bias=None,
                       residual_scale: float = 1.0, kind: str = "layer", eps: float = 1e-6, stream=None) -> dict:
    """Gradients of ``residual_norm`` from z, y and those of z (None: zero) and h (daf_residual_norm_grad): a dict with "x", "y",
    "weight", "bias", "gate", "post_weight" and "post_bias", None where there is no such parameter."""
    if stream is not None:
        with _torch().cuda.stream(stream):
            return residual_norm_grad(z, y, weight, bias, grad_z, grad_h, gate=gate, post_weight=post_weight, post_bias=post_bias,
                                      residual_scale=residual_scale, kind=kind, eps=eps)
    gx, gy, gw, gb, gg, gpw, gpb, status = _native().residual_norm_grad(
        z, y, weight, bias, gate, post_weight, post_bias, residual_scale, _kind("residual_norm_grad", kind), eps, grad_z, grad_h)
    _check(status, "daf_residual_norm_grad")
    return {"x": gx, "y": gy, "weight": gw, "bias": gb, "gate": gg, "post_weight": gpw, "post_bias": gpb}


def gap_free(t) -> bool:
    """Whether a tensor fills its memory without gaps or overlaps, in whatever order of dimensions."""
    return _native().gap_free(t)


def clip_grad_norm(grads, max_norm: float, *, eps: float = 1e-6, out=None, stream=None):
    """Scales the tensors of ``grads`` in place (or into ``out``, tensors of the same types, sizes and orders) by
    min(1, max_norm / (norm + eps)), norm being the 2-norm over all of them; returns the norm as a float32 scalar tensor on
    their device, zero on the current one for no tensors (daf_clip_norm_batch).  Nothing is read back."""
    if stream is not None:
        with _torch().cuda.stream(stream):
            return clip_grad_norm(grads, max_norm, eps=eps, out=out)
    grads = list(grads)
    if not grads:
        torch = _torch()
        return torch.zeros((), dtype=torch.float32, device="cuda" if torch.cuda.is_available() else "cpu")
    norm, status = _native().clip_grad_norm(grads, None if out is None else list(out), max_norm, eps)
    _check(status, "daf_clip_norm_batch")
    return norm


def embedding(tokens, weight, *, scale: float = 1.0, dtype=None, out=None, check: bool = False, stream=None):
    """scale * weight[tokens]: rows of weight [vocabulary, width] for int32 or int64 tokens of any shape (daf_embedding).  dtype:
    the output's type, the weight's by default, any of the three where the weight is float32.  A token outside the vocabulary
    gives zeros and is recorded for ``check_device``; with check the call waits and raises for its own tokens, and records nothing there."""
    if stream is not None:
        with _torch().cuda.stream(stream):
            return embedding(tokens, weight, scale=scale, dtype=dtype, out=out, check=check)
    made, status = _native().embedding(tokens, weight, scale, dtype, out, check)
    _check(status, "daf_embedding")
    return made if out is None else out


def embedding_grad(tokens, grad_out, vocabulary: int, *, scale: float = 1.0, padding: int | None = None, dtype=None, out=None,
                   check: bool = False, stream=None):
    """The gradient of ``embedding`` with respect to its weight, [vocabulary, width]: scale times the sum of grad_out's rows over
    each token's places, in their order and in float32, zero for the others and for the padding token (daf_embedding_grad).
    dtype: the gradient's type, grad_out's by default, or float32."""
    if stream is not None:
        with _torch().cuda.stream(stream):
            return embedding_grad(tokens, grad_out, vocabulary, scale=scale, padding=padding, dtype=dtype, out=out, check=check)
    made, status = _native().embedding_grad(tokens, grad_out, vocabulary, scale, padding, dtype, out, check)
    _check(status, "daf_embedding_grad")
    return made if out is None else out


ROTARY_HALVES, ROTARY_PAIRS = 0, 1
_STYLES = {"halves": ROTARY_HALVES, "pairs": ROTARY_PAIRS}


def _style(where: str, style: str) -> int:
    if style not in _STYLES:
        raise ValueError(f"{where}: style is 'halves' or 'pairs'")
    return _STYLES[style]


def rotary_norm(q, k, q_weight=None, k_weight=None, *, positions=None, rotary_dim: int | None = None, base: float = 10000.0,
                style: str = "halves", eps: float = 1e-6, frequencies=None, out=None, stream=None):
    """(q, k): every row of q [B, S, H, D] and k [B, S, Hkv, D] (None: queries alone) divided by its root mean square, times
    the weight [D], its first rotary_dim elements turned by position (daf_rotary_norm).  positions: int32 or int64, [B, S] or [S], a
    whole number (the first token's position in every sequence), or None for 0.  style: pairs (i, i + rotary_dim / 2) or
    (2 i, 2 i + 1), turned by position * base^(-2 i / rotary_dim), or by position * frequencies[i].  Slices of a packed projection
    are read in place; what the kernels cannot address is copied first.  out: (q, k) to write into, which may be q and k."""
    if stream is not None:
        with _torch().cuda.stream(stream):
            return rotary_norm(q, k, q_weight, k_weight, positions=positions, rotary_dim=rotary_dim, base=base, style=style, eps=eps,
                               frequencies=frequencies, out=out)
    qo, ko = (None, None) if out is None else out
    frequencies = None if frequencies is None else [float(f) for f in frequencies]
    qo, ko, status = _native().rotary_norm(q, k, q_weight, k_weight, positions, rotary_dim, base, _style("rotary_norm", style), eps,
                                           frequencies, qo, ko)
    _check(status, "daf_rotary_norm")
    return qo, ko


def rotary_norm_grad(q, k, q_weight, k_weight, grad_q_out, grad_k_out, *, positions=None, rotary_dim: int | None = None,
                     base: float = 10000.0, style: str = "halves", eps: float = 1e-6, frequencies=None, grads=None, stream=None):
    """(grad_q, grad_k, grad_q_weight, grad_k_weight) of ``rotary_norm`` from its inputs and the gradients of its outputs
    (daf_rotary_norm_grad); None where there is no such input.  grads: (grad_q, grad_k) to write into, e.g. slices of one packed
    gradient."""
    if stream is not None:
        with _torch().cuda.stream(stream):
            return rotary_norm_grad(q, k, q_weight, k_weight, grad_q_out, grad_k_out, positions=positions, rotary_dim=rotary_dim, base=base,
                                    style=style, eps=eps, frequencies=frequencies, grads=grads)
    gq, gk = (None, None) if grads is None else grads
    frequencies = None if frequencies is None else [float(f) for f in frequencies]
    *made, status = _native().rotary_norm_grad(q, k, q_weight, k_weight, positions, rotary_dim, base, _style("rotary_norm_grad", style), eps,
                                               frequencies, grad_q_out, grad_k_out, gq, gk)
    _check(status, "daf_rotary_norm_grad")
    return tuple(made)


def orthogonalize(updates, *, steps: int = 5, coefficients=(3.4445, -4.7750, 2.0315), eps: float = 1e-7, out=None, check: bool = False,
                  stream=None) -> list:
    """The matrices of ``updates`` (dimensions behind the first count as one) with their singular values taken towards one: x =
    g / (norm(g) + eps), then ``steps`` times x = a x + (b x x^T + c (x x^T)^2) x (daf_orthogonalize).  All matrices of a call run
    together, so give them at once.  out: contiguous tensors to write into, which may be the updates themselves."""
    if stream is not None:
        with _torch().cuda.stream(stream):
            return orthogonalize(updates, steps=steps, coefficients=coefficients, eps=eps, out=out, check=check)
    updates = list(updates)
    if not updates:
        return []
    made, status = _native().orthogonalize(updates, None if out is None else list(out), steps, tuple(coefficients), eps, check)
    _check(status, "daf_orthogonalize")
    return made if out is None else list(out)


class Pool:
    """Host-side page pool (bookkeeping only) over a caller-owned arena."""

    def __init__(self, arena_bytes: int, page_bytes: int = 0):
        self._h = lib().daf_pool_create(arena_bytes, page_bytes)
        if not self._h:
            raise DafError(ERR_INVALID_ARG, "daf_pool_create")

    def alloc(self, nbytes: int, importance: float):
        off = ctypes.c_uint64()
        h = int(lib().daf_pool_alloc(self._h, nbytes, importance, ctypes.byref(off)))
        return (h, int(off.value)) if h else (0, None)

    def free(self, handle: int):
        _check(lib().daf_pool_free(self._h, handle), "daf_pool_free")

    def evict_lowest(self) -> int:
        return int(lib().daf_pool_evict_lowest(self._h))

    def stats(self) -> dict:
        s = daf_pool_stats()
        _check(lib().daf_pool_get_stats(self._h, ctypes.byref(s)), "daf_pool_get_stats")
        return {n: int(getattr(s, n)) for n, _ in daf_pool_stats._fields_}

    def close(self):
        if self._h:
            lib().daf_pool_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def store_bytes(numel: int, group_size: int, width: int) -> int:
    """Bytes one activation occupies in a store at the given width (see daf_store_bytes)."""
    return int(lib().daf_store_bytes(numel, group_size, width))


class Store:
    """Importance-aware store (Sec. 3.4 of the paper): per-activation width under a memory and a time budget, two
    ordered indices, first-fit pages in an arena that follows the budget in steps.  Bookkeeping only."""

    NOT_STORED = (1 << 64) - 1
    _MAX_OUT = 4096

    def __init__(self, mem_budget_bytes: int, time_budget: float, widths=(1, 2, 4, 8), page_bytes: int = 0,
                 step_bytes: int = 0):
        cfg = daf_store_config(mem_budget_bytes, time_budget, page_bytes, step_bytes, width_mask(widths), 0)
        self._h = lib().daf_store_create(ctypes.byref(cfg))
        if not self._h:
            raise DafError(ERR_INVALID_ARG, "daf_store_create")

    def estimate(self, ident: int, numel: int, group_size: int, importance: float, time_cost: float, evicted=None) -> int:
        """Width planned for the activation; ids that lost their place in the call are appended to `evicted`."""
        w, n = ctypes.c_uint32(), ctypes.c_uint32(self._MAX_OUT)
        ev = (ctypes.c_uint64 * self._MAX_OUT)()
        _check(lib().daf_store_estimate(self._h, ident, numel, group_size, importance, time_cost, ctypes.byref(w), ev,
                                        ctypes.byref(n)), "daf_store_estimate")
        if evicted is not None:
            evicted.extend(int(ev[i]) for i in range(min(n.value, self._MAX_OUT)))
        return int(w.value)

    def admit(self, ident: int, importance: float):
        """(width, offset or None, ids evicted to make room)"""
        w, off, n = ctypes.c_uint32(), ctypes.c_uint64(), ctypes.c_uint32(self._MAX_OUT)
        ev = (ctypes.c_uint64 * self._MAX_OUT)()
        _check(lib().daf_store_admit(self._h, ident, importance, ctypes.byref(w), ctypes.byref(off), ev, ctypes.byref(n)),
               "daf_store_admit")
        return int(w.value), (None if off.value == self.NOT_STORED else int(off.value)), [int(ev[i]) for i in range(min(n.value, self._MAX_OUT))]

    def width(self, ident: int):
        w, off = ctypes.c_uint32(), ctypes.c_uint64()
        _check(lib().daf_store_width(self._h, ident, ctypes.byref(w), ctypes.byref(off)), "daf_store_width")
        return int(w.value), (None if off.value == self.NOT_STORED else int(off.value))

    def release(self, ident: int):
        _check(lib().daf_store_release(self._h, ident), "daf_store_release")

    def set_budget(self, mem_budget_bytes: int, time_budget: float):
        """(moves as (id, from, to, bytes), ids evicted)"""
        nm, ne = ctypes.c_uint32(self._MAX_OUT), ctypes.c_uint32(self._MAX_OUT)
        mv, ev = (daf_store_move * self._MAX_OUT)(), (ctypes.c_uint64 * self._MAX_OUT)()
        _check(lib().daf_store_set_budget(self._h, mem_budget_bytes, time_budget, mv, ctypes.byref(nm), ev, ctypes.byref(ne)),
               "daf_store_set_budget")
        return ([(int(m.id), int(m.from_offset), int(m.to_offset), int(m.bytes)) for m in mv[:min(nm.value, self._MAX_OUT)]],
                [int(ev[i]) for i in range(min(ne.value, self._MAX_OUT))])

    def stats(self) -> dict:
        s = daf_store_stats()
        _check(lib().daf_store_get_stats(self._h, ctypes.byref(s)), "daf_store_get_stats")
        return {n: getattr(s, n) for n, _ in daf_store_stats._fields_}

    def close(self):
        if self._h:
            lib().daf_store_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class HostRoundTrip:
    """Compress + decompress of a tensor that lives in pinned HOST memory, streamed through the device in window-aligned
    chunks: while chunk i is compressed and restored, chunk i+1 is on its way in and chunk i-1 on its way out (three
    streams, two sets of device buffers).  The chunks are shards in the sense of daf_shard -- same seed, counter base
    moved -- so the restored values are exactly those of one call on the whole tensor.  The packed form of a chunk only
    lives until the next chunk reuses its slot: this is the end-to-end path of the benchmark and of callers that want
    the effect of the round trip (what the backward pass will see), not a way to keep the packed bytes."""

    def __init__(self, dtype, group_size: int, widths, bit_budget: float, *, seed: int = 0, rounding: int = ROUND_STOCHASTIC,
                 chunk_elems: int = 1 << 25, device="cuda"):
        torch = _torch()
        if chunk_elems % DEFAULT_WINDOW:
            raise ValueError("chunk_elems must be a multiple of the window")
        self.kw = dict(group_size=group_size, widths=tuple(widths), bit_budget=float(bit_budget), seed=seed, rounding=rounding)
        self.chunk, self.device = int(chunk_elems), torch.device(device)
        self.s_in, self.s_run, self.s_out = (torch.cuda.Stream(self.device) for _ in range(3))
        self.x = [torch.empty(self.chunk, dtype=dtype, device=self.device) for _ in range(2)]
        self.y = [torch.empty(self.chunk, dtype=dtype, device=self.device) for _ in range(2)]
        code = dtype_code(self.x[0])
        full = make_params(code, self.chunk, group_size, widths, bit_budget, rounding=rounding, seed=seed)
        self.c = [alloc_outputs(full, self.device) for _ in range(2)]
        self.free = [torch.cuda.Event() for _ in range(2)]

    def __call__(self, h_in, h_out) -> None:
        """h_in, h_out: flat pinned host tensors of the same length (a multiple of the group size).  Returns when the
        work has been enqueued; the calling stream waits for it (so events recorded on it afterwards see it done)."""
        torch = _torch()
        n = h_in.numel()
        cur = torch.cuda.current_stream(self.device)
        for s in (self.s_in, self.s_run, self.s_out):
            s.wait_stream(cur)
        for i, lo in enumerate(range(0, n, self.chunk)):
            m, k = min(self.chunk, n - lo), i & 1
            ev_in, ev_run = torch.cuda.Event(), torch.cuda.Event()
            with torch.cuda.stream(self.s_in):
                if i >= 2:
                    self.s_in.wait_event(self.free[k])            # the slot's last chunk has left the device
                self.x[k][:m].copy_(h_in[lo:lo + m], non_blocking=True)
                ev_in.record()
            with torch.cuda.stream(self.s_run):
                self.s_run.wait_event(ev_in)
                kw = self.kw
                c = compress(self.x[k][:m], kw["group_size"], kw["widths"], kw["bit_budget"], rounding=kw["rounding"],
                             seed=kw["seed"], elem_index_base=lo, out=self.c[k] if m == self.chunk else None)
                decompress(c, out=self.y[k][:m])
                ev_run.record()
            with torch.cuda.stream(self.s_out):
                self.s_out.wait_event(ev_run)
                h_out[lo:lo + m].copy_(self.y[k][:m], non_blocking=True)
                self.free[k].record()
        cur.wait_stream(self.s_out)
