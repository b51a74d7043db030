"""Thin ctypes binding of ``libciera.so``: same names as the C ABI, argument marshalling only.

Every step of the codec runs in the library's CUDA kernels.  torch is used for device memory
and streams, nothing else.  Importing this module loads the library and raises if it has not
been built (``python -m paper_2609_04609_b200.build``): there is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional

import numpy as np
import torch

from .workloads import UNIT_DTYPE

BF16 = 0
FP32 = 1
FP16 = 2
DTYPE_CODES = {"bf16": BF16, "fp32": FP32, "fp16": FP16}

OK = 0
ERR_INVALID_ARG = -1
ERR_UNSUPPORTED = -2
ERR_MISALIGNED = -3
ERR_CAPACITY = -4
ERR_CUDA = -5
ERR_TIMEOUT = -6
ERR_CORRUPT = -7
ERR_NOT_BOUND = -8
ERR_TOO_LARGE = -9
NOALLOC_MAX_TILES = 65536

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libciera.so")
if not os.path.exists(_LIB_PATH):
    raise ImportError(
        f"{_LIB_PATH} is missing: build the CUDA library first (python -m paper_2609_04609_b200.build). "
        "There is no fallback path."
    )
_lib = ctypes.CDLL(_LIB_PATH)

_u64, _u32, _i32, _vp, _sz, _dbl = (ctypes.c_uint64, ctypes.c_uint32, ctypes.c_int, ctypes.c_void_p,
                                    ctypes.c_size_t, ctypes.c_double)


SCORE_SOFTMAX, SCORE_SIGMOID = 0, 1
FP8_BLOCK = 128
SOURCE_ROWS, SOURCE_SWIGLU, SOURCE_SWIGLU_BACKWARD = 0, 1, 2
PRODUCT_DENSE, PRODUCT_ROWS, PRODUCT_CONTRACT = 0, 1, 2
FP4_GROUP = 32
FP4_ATOM = 512  # scale bytes of 128 rows and 128 columns
WEIGHTS_FP8, WEIGHTS_FP4 = 0, 1
EXPERT_TOKENS_MAX = 64
EXPERT_TOKENS_HEAD = 8448


class RouteConfig(ctypes.Structure):
    """How tokens choose experts (see ``ciera_route_config`` in ciera.h); fields by keyword, the rest zero."""

    _fields_ = [("n_experts", _u32), ("top_k", _u32), ("n_groups", _u32), ("top_groups", _u32), ("group_best", _u32),
                ("score", ctypes.c_int32), ("renormalise", ctypes.c_int32), ("scale", ctypes.c_float)]


class _Fp8Rows(ctypes.Structure):
    _fields_ = [("source", ctypes.c_int32), ("dtype", ctypes.c_int32), ("rows", _u64), ("cols", _u64), ("x_rows", _u64),
                ("x", _vp), ("x_stride", _u64), ("grad", _vp), ("grad_stride", _u64), ("slot_of_row", _vp),
                ("row_weights", _vp), ("starts", _vp), ("top_k", _u32), ("n_experts", _u32), ("q", _vp), ("q_stride", _u64),
                ("scales", _vp), ("scales_stride", _u64), ("qt", _vp), ("qt_stride", _u64), ("scales_t", _vp),
                ("scales_t_stride", _u64)]


class _Fp8Blocks(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("matrices", _u32), ("rows", _u64), ("cols", _u64), ("x", _vp),
                ("x_stride", _u64), ("x_matrix_stride", _u64), ("q", _vp), ("q_stride", _u64), ("q_matrix_stride", _u64),
                ("scales", _vp), ("scales_stride", _u64), ("scales_matrix_stride", _u64), ("qt", _vp), ("qt_stride", _u64),
                ("qt_matrix_stride", _u64), ("scales_t", _vp), ("scales_t_stride", _u64), ("scales_t_matrix_stride", _u64)]


class _Fp8Product(ctypes.Structure):
    _fields_ = [("mode", ctypes.c_int32), ("out_dtype", ctypes.c_int32), ("b_blocks", ctypes.c_int32), ("n_experts", _u32),
                ("m", _u64), ("n", _u64), ("k", _u64), ("a", _vp), ("a_stride", _u64), ("a_scales", _vp),
                ("a_scales_stride", _u64), ("b", _vp), ("b_stride", _u64), ("b_matrix_stride", _u64), ("b_scales", _vp),
                ("b_scales_stride", _u64), ("b_scales_matrix_stride", _u64), ("starts", _vp), ("out", _vp),
                ("out_stride", _u64), ("out_matrix_stride", _u64), ("status", _vp)]


class _Fp4Rows(ctypes.Structure):
    _fields_ = [("source", ctypes.c_int32), ("dtype", ctypes.c_int32), ("rows", _u64), ("cols", _u64), ("x_rows", _u64),
                ("x", _vp), ("x_stride", _u64), ("slot_of_row", _vp), ("starts", _vp), ("top_k", _u32), ("n_experts", _u32),
                ("q", _vp), ("q_stride", _u64), ("scales", _vp), ("scales_stride", _u64)]


class _Fp4Matrices(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("matrices", _u32), ("rows", _u64), ("cols", _u64), ("x", _vp),
                ("x_stride", _u64), ("x_matrix_stride", _u64), ("q", _vp), ("q_stride", _u64), ("q_matrix_stride", _u64),
                ("scales", _vp), ("scales_stride", _u64), ("scales_matrix_stride", _u64), ("qt", _vp), ("qt_stride", _u64),
                ("qt_matrix_stride", _u64), ("scales_t", _vp), ("scales_t_stride", _u64), ("scales_t_matrix_stride", _u64)]


class _Fp4Values(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("matrices", _u32), ("rows", _u64), ("cols", _u64), ("q", _vp), ("q_stride", _u64),
                ("q_matrix_stride", _u64), ("scales", _vp), ("scales_stride", _u64), ("scales_matrix_stride", _u64),
                ("out", _vp), ("out_stride", _u64), ("out_matrix_stride", _u64)]


class _Fp4Product(ctypes.Structure):
    _fields_ = [("mode", ctypes.c_int32), ("out_dtype", ctypes.c_int32), ("n_experts", _u32), ("m", _u64), ("n", _u64),
                ("k", _u64), ("a", _vp), ("a_stride", _u64), ("a_scales", _vp), ("a_scales_stride", _u64), ("b", _vp),
                ("b_stride", _u64), ("b_matrix_stride", _u64), ("b_scales", _vp), ("b_scales_stride", _u64),
                ("b_scales_matrix_stride", _u64), ("starts", _vp), ("out", _vp), ("out_stride", _u64), ("status", _vp)]


class _ExpertTokens(ctypes.Structure):
    _fields_ = [("route", RouteConfig), ("format", ctypes.c_int32), ("dtype", ctypes.c_int32), ("logits_dtype", ctypes.c_int32),
                ("n_tokens", _u32), ("d_model", _u32), ("d_ff", _u32), ("x", _vp), ("x_stride", _u64), ("logits", _vp),
                ("logits_stride", _u64), ("bias", _vp), ("w1", _vp), ("w1_stride", _u64), ("w1_matrix_stride", _u64),
                ("w1_scales", _vp), ("w1_scales_stride", _u64), ("w1_scales_matrix_stride", _u64), ("w2", _vp),
                ("w2_stride", _u64), ("w2_matrix_stride", _u64), ("w2_scales", _vp), ("w2_scales_stride", _u64),
                ("w2_scales_matrix_stride", _u64), ("out", _vp), ("out_stride", _u64), ("experts", _vp), ("weights", _vp),
                ("workspace", _vp), ("workspace_bytes", _u64), ("status", _vp)]


class GainIn(ctypes.Structure):
    _fields_ = [
        ("n_values", _u64), ("dtype", ctypes.c_int32), ("block", _u32), ("q", _dbl),
        ("world_size", ctypes.c_int32), ("overlapped", ctypes.c_int32), ("alpha", _dbl), ("beta", _dbl),
        ("table_bytes", ctypes.POINTER(_dbl)), ("table_secs", ctypes.POINTER(_dbl)), ("n_points", ctypes.c_int32),
        ("t_hash", _dbl), ("t_cmp", _dbl), ("t_decmp", _dbl),
    ]


_SIGS = {
    "ciera_message_capacity": ([_u64, _i32, _u32], _sz),
    "ciera_sm_offset": ([_u64, _u32], _sz),
    "ciera_payload_offset": ([_u64, _i32, _u32], _sz),
    "ciera_message_bytes": ([_u64, _i32, _u32, _u64], _sz),
    "ciera_plan_create": ([_vp, _u32, _i32, _u32, ctypes.POINTER(_vp)], _i32),
    "ciera_plan_destroy": ([_vp], None),
    "ciera_plan_n_units": ([_vp], _u32),
    "ciera_plan_n_tiles": ([_vp], _u32),
    "ciera_plan_tile_values": ([_vp], _u32),
    "ciera_plan_total_values": ([_vp], _u64),
    "ciera_plan_device_bytes": ([_vp], _sz),
    "ciera_plan_host_image": ([_vp], _vp),
    "ciera_plan_workspace_bytes": ([_vp], _sz),
    "ciera_workspace_init": ([_vp, _vp, _vp], _i32),
    "ciera_plan_bind": ([_vp, _vp, _sz, _vp], _i32),
    "ciera_cache_init": ([_vp, _vp, _vp, _vp], _i32),
    "ciera_cache_update": ([_vp, _vp, _vp, _vp], _i32),
    "ciera_encode": ([_vp] * 9, _i32),
    "ciera_encode_noalloc": ([_vp] * 8, _i32),
    "ciera_plan_hash_cache_bytes": ([_vp], _sz),
    "ciera_plan_unit_hash_offset": ([_vp, _u32], _sz),
    "ciera_plan_hashed_workspace_bytes": ([_vp], _sz),
    "ciera_hash_cache_init": ([_vp] * 4, _i32),
    "ciera_encode_hashed": ([_vp] * 9, _i32),
    "ciera_plan_entropy_scratch_bytes": ([_vp], _sz),
    "ciera_entropy_encode": ([_vp] * 5, _i32),
    "ciera_entropy_decode": ([_vp] * 6, _i32),
    "ciera_transport": ([_vp] * 7, _i32),
    "ciera_decode": ([_vp] * 8, _i32),
    "ciera_step": ([_vp] * 12, _i32),
    "ciera_roundtrip_host": ([_vp, _vp, _sz, _vp, _vp, _vp, _vp], _i32),
    "ciera_should_compress": ([ctypes.POINTER(GainIn), ctypes.POINTER(_dbl), ctypes.POINTER(_i32)], _i32),
    "ciera_select_shards": ([ctypes.POINTER(GainIn), _u32, _u64, _i32, _vp, _vp, _vp, _vp, _vp], _i32),
    "ciera_route": ([ctypes.POINTER(RouteConfig), _i32, _vp, _u64, _u64, _vp, _vp, _vp, _vp], _i32),
    "ciera_route_backward": ([ctypes.POINTER(RouteConfig), _i32, _vp, _u64, _u64, _vp, _vp, _vp, _u64, _vp], _i32),
    "ciera_expert_rows_capacity": ([_u64, _u32], _u64),
    "ciera_expert_layout_workspace_bytes": ([_u64, _u32], _sz),
    "ciera_expert_layout": ([_vp, _u64, _u32] + [_vp] * 6, _i32),
    "ciera_fp8_quantize_rows": ([ctypes.POINTER(_Fp8Rows), _vp], _i32),
    "ciera_fp8_quantize_blocks": ([ctypes.POINTER(_Fp8Blocks), _vp], _i32),
    "ciera_fp8_matmul": ([ctypes.POINTER(_Fp8Product), _vp], _i32),
    "ciera_fp4_quantize_rows": ([ctypes.POINTER(_Fp4Rows), _vp], _i32),
    "ciera_fp4_quantize_matrices": ([ctypes.POINTER(_Fp4Matrices), _vp], _i32),
    "ciera_fp4_values": ([ctypes.POINTER(_Fp4Values), _vp], _i32),
    "ciera_fp4_matmul": ([ctypes.POINTER(_Fp4Product), _vp], _i32),
    "ciera_expert_tokens_workspace_bytes": ([_u32] * 4, _sz),
    "ciera_expert_tokens": ([ctypes.POINTER(_ExpertTokens), _vp], _i32),
    "ciera_expert_combine": ([_i32, _vp, _u64, _u64, _vp, _vp, _u64, _u32, _u64, _vp, _u64, _vp], _i32),
    "ciera_expert_combine_backward": ([_i32, _vp, _u64, _vp, _u64, _u64, _vp, _vp, _u64, _u32, _u64, _vp, _vp, _u64, _vp],
                                      _i32),
    "ciera_selftest_bounded_waits": ([_u32, _vp, _vp, _vp, _vp], _i32),
    "ciera_last_cuda_error": ([], _i32),
    "ciera_kernel_launch_count": ([], _u64),
    "ciera_status_string": ([_i32], ctypes.c_char_p),
}
for _name, (_args, _res) in _SIGS.items():
    _f = getattr(_lib, _name)
    _f.argtypes, _f.restype = _args, _res

EXPORTS = tuple(_SIGS)



def _packed(name: str, layout: str, structure):
    """An entry point whose arguments are packed in one go, microseconds less than a structure with as many fields takes."""
    pack = struct.Struct(layout)
    assert pack.size == ctypes.sizeof(structure)
    f = _lib[name]
    f.argtypes, f.restype = [ctypes.c_char_p, _vp], _i32
    return f, pack.pack


_fp4_rows, _pack_fp4_rows = _packed("ciera_fp4_quantize_rows", "=2i7Q2I4Q", _Fp4Rows)
_fp4_matrices, _pack_fp4_matrices = _packed("ciera_fp4_quantize_matrices", "=iI17Q", _Fp4Matrices)
_fp4_value, _pack_fp4_value = _packed("ciera_fp4_values", "=iI11Q", _Fp4Values)
_fp4_product, _pack_fp4_product = _packed("ciera_fp4_matmul", "=2iI4x17Q", _Fp4Product)
_tokens, _pack_tokens = _packed("ciera_expert_tokens", "=32s6i24Q", _ExpertTokens)


class CieraError(RuntimeError):
    def __init__(self, where: str, status: int):
        self.status = status
        msg = _lib.ciera_status_string(status).decode()
        if status == ERR_CUDA:
            msg += f" (cudaError {_lib.ciera_last_cuda_error()})"
        super().__init__(f"{where}: {msg} [{status}]")


def _check(where: str, status: int) -> None:
    if status != OK:
        raise CieraError(where, status)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    return t.data_ptr()


# the current stream's handle without a Stream object around it: torch.cuda.current_stream() takes 3.2 us, as long
# as the rest of the binding (small tables are stepped in 6 us), this 0.1 us
_current_device = getattr(torch._C, "_cuda_getDevice", None)
_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream: Optional[torch.cuda.Stream]) -> Optional[int]:
    if stream is not None:
        return stream.cuda_stream or None
    if _current_raw_stream is None or _current_device is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream or None
    return _current_raw_stream(_current_device()) or None


# ------------------------------------------------------------------------------ sizes (host)


def message_capacity(n: int, dtype: int, block: int) -> int:
    return int(_lib.ciera_message_capacity(n, dtype, block))


def sm_offset(n: int, block: int) -> int:
    return int(_lib.ciera_sm_offset(n, block))


def payload_offset(n: int, dtype: int, block: int) -> int:
    return int(_lib.ciera_payload_offset(n, dtype, block))


def message_bytes(n: int, dtype: int, block: int, payload_bytes: int) -> int:
    return int(_lib.ciera_message_bytes(n, dtype, block, payload_bytes))


def kernel_launch_count() -> int:
    return int(_lib.ciera_kernel_launch_count())


def selftest_bounded_waits(max_polls: int, scratch: torch.Tensor, status: torch.Tensor, report: torch.Tensor,
                           stream=None) -> None:
    """Runs the library's two kinds of bounded device wait with a short limit on things nobody completes
    (see ciera.h): ``status`` receives ERR_TIMEOUT, ``report`` (4 x int32) says which waits gave up."""
    _check("ciera_selftest_bounded_waits",
           _lib.ciera_selftest_bounded_waits(max_polls, _ptr(scratch), _ptr(status), _ptr(report), _stream(stream)))


# ------------------------------------------------------------------------------ plan


class Plan:
    """Owner of a ``ciera_plan`` handle and of the device memory its tile table lives in."""

    def __init__(self, units: np.ndarray, dtype: int, block: int, device: Optional[torch.device] = None):
        units = np.ascontiguousarray(units, dtype=UNIT_DTYPE)
        self.units = units
        self.dtype, self.block = dtype, block
        h = _vp()
        _check("ciera_plan_create",
               _lib.ciera_plan_create(units.ctypes.data if units.size else None, units.size, dtype, block,
                                      ctypes.byref(h)))
        self._h = h
        self.n_units = int(_lib.ciera_plan_n_units(h))
        self.n_tiles = int(_lib.ciera_plan_n_tiles(h))
        self.tile_values = int(_lib.ciera_plan_tile_values(h))
        self.total_values = int(_lib.ciera_plan_total_values(h))
        self.device_bytes = int(_lib.ciera_plan_device_bytes(h))
        self.workspace_bytes = int(_lib.ciera_plan_workspace_bytes(h))
        self.hash_cache_bytes = int(_lib.ciera_plan_hash_cache_bytes(h))
        self.entropy_scratch_bytes = int(_lib.ciera_plan_entropy_scratch_bytes(h))
        self.hashed_workspace_bytes = int(_lib.ciera_plan_hashed_workspace_bytes(h))
        self.table = None
        if device is not None:
            self.bind(device)

    def host_image(self) -> np.ndarray:
        n = self.device_bytes
        if n == 0:
            return np.zeros(0, np.uint8)
        buf = (ctypes.c_uint8 * n).from_address(_lib.ciera_plan_host_image(self._h))
        return np.frombuffer(buf, np.uint8).copy()

    def bind(self, device) -> "Plan":
        self.table = torch.empty(self.device_bytes, dtype=torch.uint8, device=device)
        with torch.cuda.device(self.table.device):
            _check("ciera_plan_bind",
                   _lib.ciera_plan_bind(self._h, self.table.data_ptr(), self.table.numel(), _stream(None)))
        return self

    def new_workspace(self) -> torch.Tensor:
        """A fresh workspace, zero-filled through ``ciera_workspace_init`` as the sender calls expect it."""
        ws = torch.empty(max(self.workspace_bytes, 16), dtype=torch.uint8, device=self.table.device)
        workspace_init(self, ws)
        return ws

    @property
    def handle(self):
        return self._h

    def __del__(self):
        h = getattr(self, "_h", None)
        if h:
            _lib.ciera_plan_destroy(h)
            self._h = None


# ------------------------------------------------------------------------------ device calls


def workspace_init(plan: "Plan", workspace: torch.Tensor, stream=None) -> None:
    """Zero-fills a workspace: once after allocating it, and again after a call that reported a device-side error."""
    with torch.cuda.device(workspace.device):
        _check("ciera_workspace_init", _lib.ciera_workspace_init(plan.handle, _ptr(workspace), _stream(stream)))


def cache_init(plan: Plan, cache: torch.Tensor, weights: Optional[torch.Tensor], stream=None) -> None:
    _check("ciera_cache_init", _lib.ciera_cache_init(plan.handle, _ptr(cache), _ptr(weights), _stream(stream)))


def cache_update(plan: Plan, cache: torch.Tensor, weights: torch.Tensor, stream=None) -> None:
    _check("ciera_cache_update", _lib.ciera_cache_update(plan.handle, _ptr(cache), _ptr(weights), _stream(stream)))


def encode(plan: Plan, weights, sender_cache, messages, wire_bytes, changed_blocks, workspace, status=None,
           stream=None) -> None:
    _check("ciera_encode",
           _lib.ciera_encode(plan.handle, _ptr(weights), _ptr(sender_cache), _ptr(messages), _ptr(wire_bytes),
                             _ptr(changed_blocks), _ptr(workspace), _ptr(status), _stream(stream)))


def encode_noalloc(plan: Plan, weights, sender_cache, messages, wire_bytes, changed_blocks, status=None,
                   stream=None) -> None:
    """``ciera_encode`` without a scratch argument: for callers that can pass the buffers they own
    but cannot allocate one more (see ciera.h).  At most NOALLOC_MAX_TILES tiles per call; calls
    that may overlap on the GPU must not both use it."""
    _check("ciera_encode_noalloc",
           _lib.ciera_encode_noalloc(plan.handle, _ptr(weights), _ptr(sender_cache), _ptr(messages), _ptr(wire_bytes),
                                     _ptr(changed_blocks), _ptr(status), _stream(stream)))


def unit_hash_offset(plan: Plan, unit: int) -> int:
    """Byte offset of the unit's first block in the plan's HashCache."""
    return int(_lib.ciera_plan_unit_hash_offset(plan.handle, unit))


def hash_cache_init(plan: Plan, hash_cache: torch.Tensor, weights: Optional[torch.Tensor], stream=None) -> None:
    _check("ciera_hash_cache_init",
           _lib.ciera_hash_cache_init(plan.handle, _ptr(hash_cache), _ptr(weights), _stream(stream)))


def encode_hashed(plan: Plan, weights, hash_cache, messages, wire_bytes, changed_blocks, workspace, status=None,
                  stream=None) -> None:
    """Sender step with a 128-bit hash per block in place of the exponent cache (blocks of 16 values
    and more); ``workspace`` holds ``plan.hashed_workspace_bytes``."""
    _check("ciera_encode_hashed",
           _lib.ciera_encode_hashed(plan.handle, _ptr(weights), _ptr(hash_cache), _ptr(messages), _ptr(wire_bytes),
                                    _ptr(changed_blocks), _ptr(workspace), _ptr(status), _stream(stream)))


def entropy_encode(plan: Plan, messages, wire_bytes, scratch, stream=None) -> None:
    """rANS-codes the payload of every message in place where that shortens it (after encode)."""
    _check("ciera_entropy_encode",
           _lib.ciera_entropy_encode(plan.handle, _ptr(messages), _ptr(wire_bytes), _ptr(scratch), _stream(stream)))


def entropy_decode(plan: Plan, messages, wire_bytes, scratch, status=None, stream=None) -> None:
    """Restores the raw payload of every message in place (before decode)."""
    _check("ciera_entropy_decode",
           _lib.ciera_entropy_decode(plan.handle, _ptr(messages), _ptr(wire_bytes), _ptr(scratch), _ptr(status),
                                     _stream(stream)))


def transport(plan: Plan, src_messages, dst_messages, wire_bytes, workspace, status=None, stream=None) -> None:
    _check("ciera_transport",
           _lib.ciera_transport(plan.handle, _ptr(src_messages), _ptr(dst_messages), _ptr(wire_bytes),
                                _ptr(workspace), _ptr(status), _stream(stream)))


def decode(plan: Plan, messages, receiver_cache, weights_out, wire_bytes=None, workspace=None, status=None,
           stream=None) -> None:
    _check("ciera_decode",
           _lib.ciera_decode(plan.handle, _ptr(messages), _ptr(receiver_cache), _ptr(weights_out), _ptr(wire_bytes),
                             _ptr(workspace), _ptr(status), _stream(stream)))


def step(plan: Plan, weights, sender_cache, msg_send, msg_recv, receiver_cache, weights_out, wire_bytes, changed_blocks,
         workspace, status=None, stream=None) -> None:
    """``encode``, ``transport`` and ``decode`` of one table in one launch (sender and receiver on this GPU)."""
    _check("ciera_step",
           _lib.ciera_step(plan.handle, _ptr(weights), _ptr(sender_cache), _ptr(msg_send), _ptr(msg_recv),
                           _ptr(receiver_cache), _ptr(weights_out), _ptr(wire_bytes), _ptr(changed_blocks),
                           _ptr(workspace), _ptr(status), _stream(stream)))


class DeviceBuffers(ctypes.Structure):
    _fields_ = [(n, _vp) for n in ("weights_dev", "sender_cache_dev", "msg_send_dev", "msg_recv_dev",
                                   "receiver_cache_dev", "weights_out_dev", "wire_bytes_dev", "changed_blocks_dev",
                                   "workspace_dev", "status_dev")]


def roundtrip_host(plan: Plan, weights_host: torch.Tensor, weights_out_host: torch.Tensor,
                   wire_bytes_host: Optional[torch.Tensor], bufs: DeviceBuffers, stream=None) -> None:
    """Host weights in, host weights out (both CPU tensors, ideally pinned); see ciera.h."""
    nbytes = weights_host.numel() * weights_host.element_size()
    _check("ciera_roundtrip_host",
           _lib.ciera_roundtrip_host(plan.handle, _ptr(weights_host), nbytes, _ptr(weights_out_host),
                                     _ptr(wire_bytes_host), ctypes.addressof(bufs), _stream(stream)))


# ------------------------------------------------------------------------------ the MoE layer behind the gather

_CODE_OF = {torch.bfloat16: BF16, torch.float32: FP32, torch.float16: FP16}
_E4M3 = torch.float8_e4m3fn
_I32, _F32, _U8 = torch.int32, torch.float32, torch.uint8
_Tensor = torch.Tensor


def _refuse(where: str, status: int = ERR_INVALID_ARG):
    raise CieraError(where, status)


def _device_of(where: str, t) -> int:
    """The CUDA device that the call's first tensor lives on; the others have to live there too."""
    device = t.get_device() if isinstance(t, _Tensor) else -1
    if device < 0:
        raise CieraError(where, ERR_INVALID_ARG)
    return device


def _whole(where: str, device: int, t, shape, dtype) -> int:
    """The address of a contiguous tensor of this shape and type."""
    if not isinstance(t, _Tensor) or t.dtype is not dtype or t.shape != shape or t.get_device() != device \
            or not t.is_contiguous():
        raise CieraError(where, ERR_INVALID_ARG)
    return t.data_ptr()


def _matrix(where: str, device: int, t, shape, dtype):
    """The address and the stride of the rows of a 2-D tensor of this type and, unless None, shape."""
    if not isinstance(t, _Tensor) or t.dtype is not dtype or t.get_device() != device or t.dim() != 2 \
            or (shape is not None and t.shape != shape):
        raise CieraError(where, ERR_INVALID_ARG)
    stride = t.stride()
    if stride[1] != 1 and t.shape[1] > 1:
        raise CieraError(where, ERR_INVALID_ARG)
    return t.data_ptr(), stride[0]


def _matrices(where: str, device: int, t, shape, dtype):
    """The address and the strides of the rows and of the matrices of a 3-D tensor of this type and, unless None, shape."""
    if not isinstance(t, _Tensor) or t.dtype is not dtype or t.get_device() != device or t.dim() != 3 \
            or (shape is not None and t.shape != shape):
        raise CieraError(where, ERR_INVALID_ARG)
    stride = t.stride()
    if stride[2] != 1 and t.shape[2] > 1:
        raise CieraError(where, ERR_INVALID_ARG)
    return t.data_ptr(), stride[1], stride[0]


def _scale_lines(where: str, device: int, t, cols: int, rows: int):
    """The same of scale bytes [ceil(cols / 128), at least rows]."""
    at = _matrix(where, device, t, None, _U8)
    shape = t.shape
    if shape[0] != -(-cols // FP8_BLOCK) or shape[1] < rows:
        raise CieraError(where, ERR_INVALID_ARG)
    return at


def _code(where: str, t) -> int:
    code = _CODE_OF.get(t.dtype)
    if code is None:
        raise CieraError(where, ERR_INVALID_ARG)
    return code


def _enqueue(where: str, device: int, stream, f, *args) -> None:
    """Calls the library for tensors on ``device``, which need not be the current one."""
    if device == _current_device():
        status = f(*args, (_current_raw_stream(device) if stream is None else stream.cuda_stream) or None)
    else:
        with torch.cuda.device(device):
            status = f(*args, (_current_raw_stream(device) if stream is None else stream.cuda_stream) or None)
    if status != OK:
        raise CieraError(where, status)


def route(config: RouteConfig, logits, bias, experts, weights, stream=None) -> None:
    """Scores of ``logits`` [T, E], the top k experts of every token (``experts`` int32 [T, k], -1 where none is left) and their
    ``weights`` (fp32 [T, k]); ``bias`` (fp32 [E] or None) counts for the choice only."""
    w = "ciera_route"
    device = _device_of(w, logits)
    code = _code(w, logits)
    at, stride = _matrix(w, device, logits, None, logits.dtype)
    t, e = logits.shape
    if e != config.n_experts:
        _refuse(w)
    k = config.top_k
    _enqueue(w, device, stream, _lib.ciera_route, config, code, at, t, stride,
             None if bias is None else _whole(w, device, bias, (e,), _F32), _whole(w, device, experts, (t, k), _I32),
             _whole(w, device, weights, (t, k), _F32))


def route_backward(config: RouteConfig, logits, experts, dweights, dlogits, stream=None) -> None:
    """Gradient of the logits (``dlogits``, their shape and type) from that of the weights, for the choice in ``experts``."""
    w = "ciera_route_backward"
    device = _device_of(w, logits)
    code = _code(w, logits)
    at, stride = _matrix(w, device, logits, None, logits.dtype)
    shape = logits.shape
    t, e = shape
    if e != config.n_experts:
        _refuse(w)
    k = config.top_k
    _enqueue(w, device, stream, _lib.ciera_route_backward, config, code, at, t, stride,
             _whole(w, device, experts, (t, k), _I32), _whole(w, device, dweights, (t, k), _F32),
             *_matrix(w, device, dlogits, shape, logits.dtype))


def expert_rows_capacity(n_slots: int, n_experts: int) -> int:
    """Rows that the experts' segments can take at most."""
    return int(_lib.ciera_expert_rows_capacity(n_slots, n_experts))


def expert_layout_workspace_bytes(n_slots: int, n_experts: int) -> int:
    return int(_lib.ciera_expert_layout_workspace_bytes(n_slots, n_experts))


def expert_layout(experts, n_experts: int, starts, counts, row_of_slot, slot_of_row, workspace, stream=None) -> None:
    """Slots (``experts``, int32, any shape) in the order of the experts, segments of a multiple of 128 rows: ``starts`` int32
    [E + 1], ``counts`` int32 [E], ``row_of_slot`` int32 of the shape of ``experts``, ``slot_of_row`` int32
    [expert_rows_capacity], ``workspace`` uint8 [expert_layout_workspace_bytes]."""
    w = "ciera_expert_layout"
    device = _device_of(w, experts)
    shape = experts.shape
    n = experts.numel()
    room = slot_of_row.numel() if isinstance(slot_of_row, _Tensor) else -1
    scratch = workspace.numel() if isinstance(workspace, _Tensor) else -1
    args = (_whole(w, device, experts, shape, _I32), n, n_experts, _whole(w, device, starts, (n_experts + 1,), _I32),
            _whole(w, device, counts, (n_experts,), _I32), _whole(w, device, row_of_slot, shape, _I32),
            _whole(w, device, slot_of_row, (room,), _I32), _whole(w, device, workspace, (scratch,), _U8))
    if room < _lib.ciera_expert_rows_capacity(n, n_experts) or \
            scratch < _lib.ciera_expert_layout_workspace_bytes(n, n_experts):
        _refuse(w, ERR_CAPACITY)
    _enqueue(w, device, stream, _lib.ciera_expert_layout, *args)


def fp8_quantize_rows(x, q, scales, qt=None, scales_t=None, *, kind: int = SOURCE_ROWS, grad=None, slot_of_row=None,
                      top_k: int = 1, row_weights=None, starts=None, stream=None) -> None:
    """Rows formed from ``x`` and rounded to e4m3: ``q`` [rows, cols] with ``scales`` uint8 [ceil(cols / 128), >= rows], and, if
    given, the transposed ``qt`` [cols, rows] with ``scales_t`` uint8 [ceil(rows / 128), >= cols] (see ``ciera_fp8_rows``)."""
    w = "ciera_fp8_quantize_rows"
    device = _device_of(w, x)
    code = _code(w, x)
    x_at = _matrix(w, device, x, None, x.dtype)
    x_rows, x_cols = x.shape
    q_at = _matrix(w, device, q, None, _E4M3)
    rows, cols = q.shape
    if x_cols != (2 * cols if kind == SOURCE_SWIGLU else cols) or (qt is None) != (scales_t is None) or \
            (grad is None) == (kind == SOURCE_SWIGLU_BACKWARD):
        _refuse(w)
    s_at = _scale_lines(w, device, scales, cols, rows)
    t_at, st_at, g_at = (None, 0), (None, 0), (None, 0)
    if qt is not None:
        t_at = _matrix(w, device, qt, (cols, rows), _E4M3)
        st_at = _scale_lines(w, device, scales_t, rows, cols)
    if grad is not None:
        g_at = _matrix(w, device, grad, (x_rows, cols // 2), x.dtype)
    slots = weights = begin = None
    n_experts = 0
    if slot_of_row is not None:
        slots = _whole(w, device, slot_of_row, slot_of_row.shape, _I32)
        if slot_of_row.dim() != 1 or slot_of_row.numel() < rows:
            _refuse(w)
    if row_weights is not None:
        weights = _whole(w, device, row_weights, (x_rows, top_k), _F32)
    if starts is not None:
        n_experts = starts.numel() - 1
        begin = _whole(w, device, starts, (n_experts + 1,), _I32)
    args = _Fp8Rows(kind, code, rows, cols, x_rows, *x_at, *g_at, slots, weights, begin, top_k, max(n_experts, 0), *q_at, *s_at,
                    *t_at, *st_at)
    _enqueue(w, device, stream, _lib.ciera_fp8_quantize_rows, args)


def fp8_quantize_blocks(x, q, scales, qt=None, scales_t=None, stream=None) -> None:
    """Matrices ``x`` [matrices, rows, cols] rounded to e4m3 with one scale for each 128 x 128 block: ``q`` of that shape with
    ``scales`` uint8 [matrices, ceil(rows / 128), ceil(cols / 128)], and, if given, the transposed ``qt`` and ``scales_t``."""
    w = "ciera_fp8_quantize_blocks"
    device = _device_of(w, x)
    code = _code(w, x)
    x_at = _matrices(w, device, x, None, x.dtype)
    shape = x.shape
    m, r, c = shape
    rb, cb = -(-r // FP8_BLOCK), -(-c // FP8_BLOCK)
    if (qt is None) != (scales_t is None):
        _refuse(w)
    turned = () if qt is None else (*_matrices(w, device, qt, (m, c, r), _E4M3),
                                    *_matrices(w, device, scales_t, (m, cb, rb), _U8))
    args = _Fp8Blocks(code, m, r, c, *x_at, *_matrices(w, device, q, shape, _E4M3),
                      *_matrices(w, device, scales, (m, rb, cb), _U8), *turned)
    _enqueue(w, device, stream, _lib.ciera_fp8_quantize_blocks, args)


def fp8_matmul(a, a_scales, b, b_scales, out, starts=None, contract: bool = False, status=None, stream=None) -> None:
    """``out`` = ``a`` times ``b`` transposed, of operands as the two calls above make them (see ``ciera_fp8_product``).

    ``starts`` None: a [m, k], b [n, k] with a scale for each row and 128 columns, or b [1, n, k] with one for each block.
    ``starts`` int32 [E + 1]: rows of ``a`` and ``out`` [rows, n] by segments, each with its own matrix of b [E, n, k]; with
    ``contract`` a [m, rows], b [n, rows], out [E, m, n], each from the columns of its own segment."""
    w = "ciera_fp8_matmul"
    device = _device_of(w, a)
    a_at = _matrix(w, device, a, None, _E4M3)
    m, k = a.shape
    begin, experts = None, 0
    mode = PRODUCT_DENSE
    if starts is not None:
        experts = starts.numel() - 1
        begin = _whole(w, device, starts, (experts + 1,), _I32)
        mode = PRODUCT_CONTRACT if contract else PRODUCT_ROWS
    elif contract:
        _refuse(w)
    blocks = isinstance(b, _Tensor) and b.dim() == 3
    if blocks != (mode == PRODUCT_ROWS) and mode != PRODUCT_DENSE:
        _refuse(w)
    if blocks:
        b_at = _matrices(w, device, b, None, _E4M3)
        matrices, n, bk = b.shape
        if matrices != (experts if mode == PRODUCT_ROWS else 1):
            _refuse(w)
        bs_at = _matrices(w, device, b_scales, (matrices, -(-n // FP8_BLOCK), -(-k // FP8_BLOCK)), _U8)
    else:
        b_at = (*_matrix(w, device, b, None, _E4M3), 0)
        n, bk = b.shape
        bs_at = (*_scale_lines(w, device, b_scales, k, n), 0)
    if bk != k:
        _refuse(w)
    code = _code(w, out)
    if contract:
        o_at = _matrices(w, device, out, (experts, m, n), out.dtype)
    else:
        o_at = (*_matrix(w, device, out, (m, n), out.dtype), 0)
    args = _Fp8Product(mode, code, blocks, max(experts, 0), m, n, k, *a_at, *_scale_lines(w, device, a_scales, k, m), *b_at,
                       *bs_at, begin, *o_at, None if status is None else _whole(w, device, status, (1,), _I32))
    _enqueue(w, device, stream, _lib.ciera_fp8_matmul, args)


def _codes(where: str, device: int, t, rows: int, cols: int):
    """The address and the stride of the rows of 4-bit codes [rows, ceil(cols / 2)]."""
    return _matrix(where, device, t, (rows, (cols + 1) // 2), _U8)


def _atom_lines(where: str, device: int, t, rows: int, cols: int):
    """The address and the stride of the lines of scale bytes [ceil(rows / 128), ceil(cols / 128), 512]."""
    atoms = -(-cols // 128)
    if not isinstance(t, _Tensor) or t.dtype is not _U8 or t.shape != (-(-rows // 128), atoms, FP4_ATOM) or t.get_device() != device:
        raise CieraError(where, ERR_INVALID_ARG)
    stride = t.stride()
    if stride[2] != 1 or (stride[1] != FP4_ATOM and atoms > 1):
        raise CieraError(where, ERR_INVALID_ARG)
    return t.data_ptr(), stride[0]


def _atom_stack(where: str, device: int, t, matrices: int, rows: int, cols: int):
    """The same of [matrices, ...], and the stride of the matrices."""
    atoms = -(-cols // 128)
    if not isinstance(t, _Tensor) or t.dtype is not _U8 or t.shape != (matrices, -(-rows // 128), atoms, FP4_ATOM) or \
            t.get_device() != device:
        raise CieraError(where, ERR_INVALID_ARG)
    stride = t.stride()
    if stride[3] != 1 or (stride[2] != FP4_ATOM and atoms > 1):
        raise CieraError(where, ERR_INVALID_ARG)
    return t.data_ptr(), stride[1], stride[0]


def fp4_quantize_rows(x, q, scales, *, kind: int = SOURCE_ROWS, slot_of_row=None, top_k: int = 1, starts=None,
                      stream=None) -> None:
    """Rows formed from ``x`` (as ``fp8_quantize_rows`` forms them, ``SOURCE_ROWS`` or ``SOURCE_SWIGLU``) and rounded to e2m1 with
    a power of two for each 32 values: ``q`` uint8 [rows, ceil(cols / 2)], two values a byte, and ``scales`` uint8
    [ceil(rows / 128), ceil(cols / 128), 512] (see ``ciera_fp4_rows``)."""
    w = "ciera_fp4_quantize_rows"
    device = _device_of(w, x)
    code = _code(w, x)
    x_at = _matrix(w, device, x, None, x.dtype)
    x_rows, cols = x.shape
    if kind == SOURCE_SWIGLU:
        if cols % 2:
            _refuse(w)
        cols //= 2
    if not isinstance(q, _Tensor) or q.dim() != 2:
        _refuse(w)
    rows = q.shape[0]
    q_at = _codes(w, device, q, rows, cols)
    s_at = _atom_lines(w, device, scales, rows, cols)
    slots = begin = n_experts = 0
    if slot_of_row is not None:
        n = slot_of_row.numel() if isinstance(slot_of_row, _Tensor) else -1
        slots = _whole(w, device, slot_of_row, (n,), _I32)
        if n < rows:
            _refuse(w)
    if starts is not None:
        n_experts = starts.numel() - 1 if isinstance(starts, _Tensor) else 0
        begin = _whole(w, device, starts, (n_experts + 1,), _I32)
    if not 0 <= kind <= 2 or not 0 <= top_k < 1 << 32:
        _refuse(w)
    _enqueue(w, device, stream, _fp4_rows, _pack_fp4_rows(kind, code, rows, cols, x_rows, *x_at, slots, begin, top_k,
                                                          max(n_experts, 0), *q_at, *s_at))


def fp4_quantize_matrices(x, q=None, scales=None, qt=None, scales_t=None, stream=None) -> None:
    """Matrices ``x`` [matrices, rows, cols] rounded to e2m1: ``q`` uint8 [matrices, rows, ceil(cols / 2)] with ``scales`` uint8
    [matrices, ceil(rows / 128), ceil(cols / 128), 512], or transposed, ``qt`` and ``scales_t`` of [cols, rows], or both."""
    w = "ciera_fp4_quantize_matrices"
    device = _device_of(w, x)
    code = _code(w, x)
    x_at = _matrices(w, device, x, None, x.dtype)
    m, r, c = x.shape
    if (q is None) != (scales is None) or (qt is None) != (scales_t is None):
        _refuse(w)
    at = turned = (0, 0, 0, 0, 0, 0)
    if q is not None:
        at = (*_matrices(w, device, q, (m, r, (c + 1) // 2), _U8), *_atom_stack(w, device, scales, m, r, c))
    if qt is not None:
        turned = (*_matrices(w, device, qt, (m, c, (r + 1) // 2), _U8), *_atom_stack(w, device, scales_t, m, c, r))
    _enqueue(w, device, stream, _fp4_matrices, _pack_fp4_matrices(code, m, r, c, *x_at, *at, *turned))


def fp4_values(q, scales, out, stream=None) -> None:
    """``out`` ([rows, cols] or [matrices, rows, cols]) = the values that ``q`` and ``scales`` stand for."""
    w = "ciera_fp4_values"
    device = _device_of(w, out)
    code = _code(w, out)
    if out.dim() == 3:
        m, r, c = out.shape
        o_at = _matrices(w, device, out, None, out.dtype)
        q_at, s_at = _matrices(w, device, q, (m, r, (c + 1) // 2), _U8), _atom_stack(w, device, scales, m, r, c)
    else:
        o_at = (*_matrix(w, device, out, None, out.dtype), 0)
        m, (r, c) = 1, out.shape
        q_at, s_at = (*_codes(w, device, q, r, c), 0), (*_atom_lines(w, device, scales, r, c), 0)
    _enqueue(w, device, stream, _fp4_value, _pack_fp4_value(code, m, r, c, *q_at, *s_at, *o_at))


def fp4_matmul(a, a_scales, b, b_scales, out, starts=None, status=None, stream=None) -> None:
    """``out`` [m, n] = ``a`` times ``b`` transposed, of operands as the calls above make them (see ``ciera_fp4_product``).

    ``starts`` None: b [n, ceil(k / 2)] with scales of [n, k].  ``starts`` int32 [E + 1]: rows of ``a`` and ``out`` by segments, each
    with its own matrix of b [E, n, ceil(k / 2)]."""
    w = "ciera_fp4_matmul"
    device = _device_of(w, a)
    a_at = _matrix(w, device, a, None, _U8)
    m, line = a.shape
    k = 2 * line
    begin = experts = 0
    if starts is not None:
        experts = starts.numel() - 1 if isinstance(starts, _Tensor) else 0
        begin = _whole(w, device, starts, (experts + 1,), _I32)
        b_at = _matrices(w, device, b, None, _U8)
        matrices, n, b_line = b.shape
        if matrices != experts:
            _refuse(w)
        bs_at = _atom_stack(w, device, b_scales, experts, n, k)
    else:
        b_at = (*_matrix(w, device, b, None, _U8), 0)
        n, b_line = b.shape
        bs_at = (*_atom_lines(w, device, b_scales, n, k), 0)
    if b_line != line:
        _refuse(w)
    code = _code(w, out)
    args = _pack_fp4_product(PRODUCT_DENSE if starts is None else PRODUCT_ROWS, code, max(experts, 0), m, n, k, *a_at,
                             *_atom_lines(w, device, a_scales, m, k), *b_at, *bs_at, begin,
                             *_matrix(w, device, out, (m, n), out.dtype),
                             0 if status is None else _whole(w, device, status, (1,), _I32))
    _enqueue(w, device, stream, _fp4_product, args)


def expert_tokens_workspace_bytes(config: RouteConfig, n_tokens: int, d_model: int, d_ff: int) -> int:
    return int(_lib.ciera_expert_tokens_workspace_bytes(n_tokens, config.top_k, d_model, d_ff))


def expert_tokens(config: RouteConfig, x, logits, bias, w1, w1_scales, w2, w2_scales, out, experts, weights, workspace,
                  status=None, stream=None) -> None:
    """A whole MoE layer for up to ``EXPERT_TOKENS_MAX`` tokens (see ``ciera_expert_tokens_args``): ``x`` and ``out`` [T, d_model],
    ``logits`` [T, E], ``bias`` fp32 [E] or None; ``experts`` int32 and ``weights`` fp32 [T, top_k] receive the choice.

    Weights in 8 bits: ``w1`` e4m3 [E, 2 d_ff, d_model] with a scale for each 128 x 128 block, ``w2`` [E, d_model, d_ff].  In 4 bits:
    uint8, half as wide, with scales [E, rows / 128, cols / 128, 512].  ``workspace`` uint8
    [expert_tokens_workspace_bytes(config, T, d_model, d_ff) or more], zeros before the first call; every call leaves it fit for the
    next, but for one that was given up (``status`` ERR_TIMEOUT), behind which it has to be filled with zeros again."""
    w = "ciera_expert_tokens"
    device = _device_of(w, x)
    dtype = x.dtype
    code = _code(w, x)
    x_at = _matrix(w, device, x, None, dtype)
    t, d = shape = x.shape
    e, k = config.n_experts, config.top_k
    if not isinstance(logits, _Tensor) or not isinstance(w1, _Tensor) or w1.dim() != 3 or w1.shape[1] % 2 or not isinstance(workspace, _Tensor):
        _refuse(w)
    logits_code = _code(w, logits)
    f = w1.shape[1] // 2
    if w1.dtype is _U8:
        form = WEIGHTS_FP4
        at = (*_matrices(w, device, w1, (e, 2 * f, d // 2), _U8), *_atom_stack(w, device, w1_scales, e, 2 * f, d),
              *_matrices(w, device, w2, (e, d, f // 2), _U8), *_atom_stack(w, device, w2_scales, e, d, f))
    else:
        form = WEIGHTS_FP8
        fb, db = -(-f // FP8_BLOCK), -(-d // FP8_BLOCK)
        at = (*_matrices(w, device, w1, (e, 2 * f, d), _E4M3),
              *_matrices(w, device, w1_scales, (e, -(-2 * f // FP8_BLOCK), db), _U8),
              *_matrices(w, device, w2, (e, d, f), _E4M3), *_matrices(w, device, w2_scales, (e, db, fb), _U8))
    choice = (t, k)
    room = workspace.numel()
    args = _pack_tokens(bytes(config), form, code, logits_code, t, d, f, *x_at, *_matrix(w, device, logits, (t, e), logits.dtype),
                        0 if bias is None else _whole(w, device, bias, (e,), _F32), *at, *_matrix(w, device, out, shape, dtype),
                        _whole(w, device, experts, choice, _I32), _whole(w, device, weights, choice, _F32),
                        _whole(w, device, workspace, (room,), _U8), room,
                        0 if status is None else _whole(w, device, status, (1,), _I32))
    _enqueue(w, device, stream, _tokens, args)


def expert_combine(rows, row_of_slot, weights, out, stream=None) -> None:
    """``out`` [T, cols] = the weighted sum of every token's ``rows`` (``row_of_slot`` int32 [T, k], entries outside passed
    over; ``weights`` fp32 [T, k], or None for 1)."""
    w = "ciera_expert_combine"
    device = _device_of(w, rows)
    code = _code(w, rows)
    r_at = _matrix(w, device, rows, None, rows.dtype)
    n_rows, cols = rows.shape
    if not isinstance(row_of_slot, _Tensor) or row_of_slot.dim() != 2:
        _refuse(w)
    shape = row_of_slot.shape
    t, k = shape
    _enqueue(w, device, stream, _lib.ciera_expert_combine, code, r_at[0], n_rows, r_at[1],
             _whole(w, device, row_of_slot, shape, _I32), None if weights is None else _whole(w, device, weights, shape, _F32),
             t, k, cols, *_matrix(w, device, out, (t, cols), rows.dtype))


def expert_combine_backward(dout, rows, row_of_slot, weights, dweights, drows=None, stream=None) -> None:
    """Gradients of ``expert_combine``: ``dweights`` fp32 [T, k] and, if given, ``drows`` (shape and type of ``rows``; rows that
    no slot names are left as they were)."""
    w = "ciera_expert_combine_backward"
    device = _device_of(w, rows)
    code = _code(w, rows)
    r_at = _matrix(w, device, rows, None, rows.dtype)
    n_rows, cols = rows.shape
    if not isinstance(row_of_slot, _Tensor) or row_of_slot.dim() != 2:
        _refuse(w)
    shape = row_of_slot.shape
    t, k = shape
    d_at = (None, 0) if drows is None else _matrix(w, device, drows, (n_rows, cols), rows.dtype)
    _enqueue(w, device, stream, _lib.ciera_expert_combine_backward, code, *_matrix(w, device, dout, (t, cols), rows.dtype), r_at[0],
             n_rows, r_at[1], _whole(w, device, row_of_slot, shape, _I32),
             None if weights is None else _whole(w, device, weights, shape, _F32), t, k, cols,
             _whole(w, device, dweights, shape, _F32), *d_at)


# ------------------------------------------------------------------------------ gain rule (host)


def _fill_gain_in(gi, keep, n_values, dtype, block, q, world_size=2, alpha=0.0, beta=1.0, table=None, t_hash=0.0,
                  t_cmp=0.0, t_decmp=0.0, overlapped=False):
    gi.n_values, gi.dtype, gi.block, gi.q = n_values, dtype, block, q
    gi.world_size, gi.overlapped, gi.alpha, gi.beta = world_size, int(overlapped), alpha, beta
    gi.t_hash, gi.t_cmp, gi.t_decmp = t_hash, t_cmp, t_decmp
    if table:
        tb = (_dbl * len(table))(*[float(p[0]) for p in table])
        ts = (_dbl * len(table))(*[float(p[1]) for p in table])
        keep.append((tb, ts))  # the arrays must outlive the call
        gi.table_bytes, gi.table_secs, gi.n_points = tb, ts, len(table)
    else:
        gi.n_points = 0


def select_shards(shards, cache_budget_bytes: int, with_sender_cache: bool = False):
    """``shards``: a list of dicts with the keyword arguments of ``should_compress``.  Returns a dict with
    ``ranking``, ``selected``, ``gains``, ``footprints`` (lists) and ``used`` (bytes)."""
    n = len(shards)
    arr = (GainIn * max(n, 1))()
    keep = []
    for gi, sh in zip(arr, shards):
        _fill_gain_in(gi, keep, **sh)
    ranking = (_u32 * max(n, 1))()
    selected = (ctypes.c_uint8 * max(n, 1))()
    gains = (_dbl * max(n, 1))()
    fps = (_u64 * max(n, 1))()
    used = _u64(0)
    _check("ciera_select_shards",
           _lib.ciera_select_shards(arr, n, int(cache_budget_bytes), int(with_sender_cache),
                                    ctypes.cast(ranking, _vp), ctypes.cast(selected, _vp), ctypes.cast(gains, _vp),
                                    ctypes.cast(fps, _vp), ctypes.cast(ctypes.pointer(used), _vp)))
    del keep
    return {"ranking": list(ranking)[:n], "selected": [bool(x) for x in list(selected)[:n]],
            "gains": list(gains)[:n], "footprints": list(fps)[:n], "used": int(used.value)}


def should_compress(n_values: int, dtype: int, block: int, q: float, world_size: int = 2, alpha: float = 0.0,
                    beta: float = 1.0, table=None, t_hash: float = 0.0, t_cmp: float = 0.0, t_decmp: float = 0.0,
                    overlapped: bool = False):
    """Returns (gain_seconds, decision)."""
    gi = GainIn()
    keep = []
    _fill_gain_in(gi, keep, n_values, dtype, block, q, world_size, alpha, beta, table, t_hash, t_cmp, t_decmp, overlapped)
    g = _dbl(0.0)
    d = _i32(0)
    _check("ciera_should_compress", _lib.ciera_should_compress(ctypes.byref(gi), ctypes.byref(g), ctypes.byref(d)))
    del keep
    return float(g.value), bool(d.value)
