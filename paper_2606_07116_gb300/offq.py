"""Python binding of liboffq.so (the OffQ W4A4 linear path on GB300).

The functions named ``offq_*`` mirror the C ABI in ``include/offq.h`` one to
one: they take torch CUDA tensors, pass their device pointers, sizes and the
current CUDA stream to the library, and raise :class:`OffqError` on a non-zero
status. All computation happens in the library's kernels; torch supplies device
memory and streams only. The helpers without the prefix (``quantize_act``,
``w4a4_linear``, ...) allocate the outputs with torch and call the same entry
points. Activation and weight code buffers are [ceil(R/32)*32, K/2] uint8
tensors holding the tiled operand layout of include/offq.h.
"""

from __future__ import annotations

import ctypes
import functools
import inspect
import math
import os
import re
from typing import NamedTuple, Optional, Tuple

import torch

from . import build as _build

OFFQ_OK = 0
OFFQ_ERR_INVALID_ARG = -1
OFFQ_ERR_UNSUPPORTED = -2
OFFQ_ERR_MISALIGNED = -3
OFFQ_ERR_CUDA = -4
OFFQ_ERR_TIMEOUT = -5

OFFQ_F32, OFFQ_BF16, OFFQ_F16 = 0, 1, 2
OFFQ_ROTATE, OFFQ_OFFSET, OFFQ_INTERLEAVED, OFFQ_ROTATE_V = 1, 2, 4, 8
OFFQ_FORM_FEW, OFFQ_FORM_MID, OFFQ_FORM_PAIR = 1, 2, 3

_DTYPE_CODE = {torch.float32: OFFQ_F32, torch.bfloat16: OFFQ_BF16, torch.float16: OFFQ_F16}
_CODE_DTYPE = {v: k for k, v in _DTYPE_CODE.items()}

_c_vp = ctypes.c_void_p
_c_i64 = ctypes.c_int64
_c_i32 = ctypes.c_int32
_c_int = ctypes.c_int
_c_f32 = ctypes.c_float

_SIGNATURES = {
    "offq_quantize_act": (_c_int, [_c_vp, _c_int, _c_i64, _c_i64, _c_i64, _c_i32, _c_i32, _c_vp, _c_vp, _c_vp, _c_vp]),
    "offq_w4a4_linear": (_c_int, [_c_vp, _c_vp, _c_vp, _c_i64, _c_i64, _c_i64, _c_i32, _c_vp, _c_vp, _c_vp, _c_vp,
                                  _c_int, _c_i64, _c_vp, _c_vp]),
    "offq_w4a4_linear_form": (_c_int, [_c_i64, _c_i64, _c_i64, _c_i32]),
    "offq_kv4_quantize": (_c_int, [_c_vp, _c_int, _c_i64, _c_i32, _c_i32, _c_i64, _c_i32, _c_vp, _c_vp, _c_vp, _c_vp]),
    "offq_prepare_weight": (_c_int, [_c_vp, _c_int, _c_i64, _c_i64, _c_i32, _c_i32, _c_vp, _c_vp, _c_vp, _c_vp]),
    "offq_get_device_status": (_c_int, [_c_vp]),
    "offq_set_wait_cycles": (_c_int, [_c_i64]),
    "offq_quantize_act_mx": (_c_int, [_c_vp, _c_int, _c_i64, _c_i64, _c_i64, _c_i32, _c_i32, _c_vp, _c_vp, _c_vp,
                                      _c_vp, _c_vp]),
    "offq_prepare_weight_mx": (_c_int, [_c_vp, _c_int, _c_i64, _c_i64, _c_i32, _c_i32, _c_vp, _c_vp, _c_vp, _c_vp,
                                        _c_vp]),
    "offq_mx_linear": (_c_int, [_c_vp, _c_vp, _c_vp, _c_vp, _c_i64, _c_i64, _c_i64, _c_i32, _c_vp, _c_vp, _c_vp,
                                _c_vp, _c_vp, _c_int, _c_i64, _c_vp]),
    "offq_mx_shift_bytes": (_c_i64, [_c_i64, _c_i64]),
    "offq_status_string": (ctypes.c_char_p, [_c_int]),
    "offq_abi_version": (_c_int, []),
    "offq_act_codes_bytes": (_c_i64, [_c_i64, _c_i64]),
    "offq_weight_codes_bytes": (_c_i64, [_c_i64, _c_i64]),
    "offq_quantize_act_group": (_c_int, [_c_vp, _c_int, _c_i64, _c_i64, _c_i64, _c_i32, _c_i32, _c_i32, _c_vp, _c_vp,
                                         _c_vp, _c_vp]),
    "offq_weight_group_sums": (_c_int, [_c_vp, _c_i64, _c_i64, _c_i32, _c_vp, _c_vp]),
    "offq_w4a4_linear_group": (_c_int, [_c_vp, _c_vp, _c_vp, _c_i64, _c_i64, _c_i64, _c_i32, _c_vp, _c_vp, _c_vp,
                                        _c_vp, _c_int, _c_i64, _c_vp]),
    "offq_kv4_quantize_rotated": (_c_int, [_c_vp, _c_int, _c_i64, _c_i32, _c_i32, _c_i64, _c_vp, _c_i32, _c_vp,
                                           _c_vp, _c_vp, _c_vp]),
    "offq_rotate_heads": (_c_int, [_c_vp, _c_int, _c_i64, _c_i32, _c_i32, _c_i64, _c_vp, _c_vp, _c_int, _c_i64,
                                   _c_vp]),
    "offq_prepare_key_rotation": (_c_int, [_c_vp, _c_i32, _c_i32, _c_vp, _c_vp]),
    "offq_kv4_quantize_prepared": (_c_int, [_c_vp, _c_int, _c_i64, _c_i32, _c_i32, _c_i64, _c_vp, _c_i32, _c_vp,
                                            _c_vp, _c_vp, _c_vp]),
    "offq_rotate_heads_prepared": (_c_int, [_c_vp, _c_int, _c_i64, _c_i32, _c_i32, _c_i64, _c_vp, _c_vp, _c_int,
                                            _c_i64, _c_vp]),
    "offq_prepare_key_reflection": (_c_int, [_c_vp, _c_vp, _c_i32, _c_i32, _c_vp]),
    "offq_kv4_quantize_reflected": (_c_int, [_c_vp, _c_int, _c_i64, _c_i32, _c_i32, _c_i64, _c_vp, _c_i32, _c_vp,
                                             _c_vp, _c_vp, _c_vp]),
    "offq_rotate_heads_reflected": (_c_int, [_c_vp, _c_int, _c_i64, _c_i32, _c_i32, _c_i64, _c_vp, _c_vp, _c_int,
                                             _c_i64, _c_vp]),
    "offq_top1_tokens": (_c_int, [_c_vp, _c_int, _c_i64, _c_i64, _c_i64, _c_i64, _c_i64, _c_vp, _c_vp, _c_vp]),
    "offq_top1_direction": (_c_int, [_c_vp, _c_i64, _c_i64, _c_i32, _c_vp, _c_vp, _c_vp, _c_vp]),
    "offq_reflect_rows": (_c_int, [_c_vp, _c_i64, _c_i64, _c_vp, _c_vp, _c_vp]),
    "offq_column_absmax": (_c_int, [_c_vp, _c_i64, _c_i64, _c_vp, _c_vp]),
    "offq_sorted_grouping": (_c_int, [_c_vp, _c_i64, _c_i32, _c_vp]),
    "offq_fuse_rotation": (_c_int, [_c_vp, _c_i64, _c_i64, _c_vp, _c_vp, _c_i32, _c_vp, _c_vp]),
    "offq_rope_heads": (_c_int, [_c_vp, _c_int, _c_i64, _c_i32, _c_i32, _c_i64, _c_vp, _c_vp, _c_i64, _c_i32, _c_vp,
                                 _c_f32, _c_i32, _c_vp, _c_int, _c_i64, _c_vp]),
    "offq_kv4_paged_write": (_c_int, [_c_vp, _c_vp, _c_vp, _c_int, _c_i64, _c_i32, _c_i32, _c_i32, _c_i64, _c_i64,
                                      _c_i64, _c_vp, _c_vp, _c_i64, _c_i32, _c_vp, _c_vp, _c_f32, _c_i32, _c_vp,
                                      _c_vp, _c_vp, _c_vp, _c_vp, _c_i64, _c_i32, _c_vp, _c_int, _c_i64, _c_vp]),
    "offq_kv4_paged_read": (_c_int, [_c_vp, _c_vp, _c_vp, _c_vp, _c_i64, _c_i32, _c_i32, _c_i32, _c_vp, _c_i64,
                                     _c_i32, _c_vp, _c_vp, _c_int, _c_i64, _c_i64, _c_vp]),
    "offq_paged_attention": (_c_int, [_c_vp, _c_int, _c_i64, _c_i32, _c_i32, _c_i32, _c_i64, _c_vp, _c_vp, _c_vp,
                                      _c_vp, _c_i64, _c_i32, _c_vp, _c_i64, _c_vp, _c_vp, _c_i32, _c_i32, _c_f32,
                                      _c_vp, _c_i64, _c_vp, _c_vp, _c_i64, _c_vp]),
    "offq_paged_attention_workspace": (_c_i64, [_c_i64, _c_i32, _c_i32, _c_i32, _c_i32, _c_i32]),
    "offq_prompt_attention": (_c_int, [_c_vp, _c_vp, _c_vp, _c_int, _c_i64, _c_i32, _c_i32, _c_i32, _c_i64, _c_i64,
                                       _c_i64, _c_vp, _c_i32, _c_f32, _c_i32, _c_vp, _c_i64, _c_vp, _c_vp]),
}

_lib = None


class OffqError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__(f"{fn} failed: {status_string(status)} ({status})")


def library_path() -> str:
    return _build.LIB_PATH


def load_library(path: Optional[str] = None) -> ctypes.CDLL:
    """Loads liboffq.so (raises if it was not built: there is no fallback)."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or library_path()
    if not os.path.exists(p):
        raise RuntimeError(f"liboffq.so not found at {p}; build it with "
                           "paper_2606_07116_gb300.build.build() (no CPU fallback exists)")
    lib = ctypes.CDLL(p)
    for name, (res, args) in _SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    if path is None:
        _lib = lib
    return lib


def declared_symbols(header: Optional[str] = None):
    """Names of the functions include/offq.h declares."""
    header = header or os.path.join(_build.INCLUDE, "offq.h")
    with open(header) as f:
        text = f.read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(offq_[a-z0-9_]+)\s*\(", text)))


def status_string(status: int) -> str:
    return load_library().offq_status_string(status).decode()


def abi_version() -> int:
    return load_library().offq_abi_version()


def _check(fn: str, rc: int):
    if rc != OFFQ_OK:
        raise OffqError(fn, rc)


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("tensors passed to liboffq must live on a CUDA device")
    return t.data_ptr()


def _stream(stream):
    if stream is None:  # the current stream's handle, without an object around it (3 us of a 20 us call)
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    if isinstance(stream, torch.cuda.Stream):
        return ctypes.c_void_p(stream.cuda_stream)
    return ctypes.c_void_p(int(stream))


def _on(stream):
    """Context in which torch takes memory from, and runs behind, a stream given as such or as its handle."""
    if not isinstance(stream, torch.cuda.Stream):
        handle = int(stream)
        # 0, 1 and 2 are the runtime's names for the default stream and the per-thread one, which is ordered with it.
        stream = torch.cuda.ExternalStream(handle) if handle > 2 else torch.cuda.default_stream()
    return torch.cuda.stream(stream)


def _on_its_stream(helper):
    """With a stream given, what the helper allocates and copies is that stream's too: memory let go on the current
    stream may still be in use there, and a copy made there would not be ordered with the call. What it returns is
    memory of the call's stream, as under torch.cuda.stream."""
    at = list(inspect.signature(helper).parameters).index("stream")

    @functools.wraps(helper)
    def call(*args, **kwargs):
        stream = args[at] if len(args) > at else kwargs.get("stream")
        if stream is None:
            return helper(*args, **kwargs)
        with _on(stream):
            return helper(*args, **kwargs)
    return call


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype not in _DTYPE_CODE:
        raise ValueError(f"unsupported dtype {t.dtype}")
    return _DTYPE_CODE[t.dtype]


# ---------------------------------------------------------------------------
# One-to-one wrappers of the C ABI.
# ---------------------------------------------------------------------------

def offq_quantize_act(x: torch.Tensor, T: int, K: int, ldx: int, g: int, flags: int,
                      codes: torch.Tensor, scale: torch.Tensor, offset: Optional[torch.Tensor],
                      stream=None) -> None:
    _check("offq_quantize_act", load_library().offq_quantize_act(
        _ptr(x), _dtype_code(x), T, K, ldx, g, flags, _ptr(codes), _ptr(scale), _ptr(offset), _stream(stream)))


def offq_w4a4_linear(a_codes: torch.Tensor, a_scale: torch.Tensor, a_offset: Optional[torch.Tensor],
                     T: int, N: int, K: int, g: int, w_codes: torch.Tensor, w_scale: torch.Tensor,
                     w_offsum: torch.Tensor, out: torch.Tensor, ldo: int,
                     acc_debug: Optional[torch.Tensor] = None, stream=None) -> None:
    _check("offq_w4a4_linear", load_library().offq_w4a4_linear(
        _ptr(a_codes), _ptr(a_scale), _ptr(a_offset), T, N, K, g, _ptr(w_codes), _ptr(w_scale),
        _ptr(w_offsum), _ptr(out), _dtype_code(out), ldo, _ptr(acc_debug), _stream(stream)))


def offq_w4a4_linear_form(T: int, N: int, K: int, g: int) -> int:
    """Which of the kernels behind offq_w4a4_linear takes the shape (OFFQ_FORM_*)."""
    form = load_library().offq_w4a4_linear_form(T, N, K, g)
    if form < 0:
        raise OffqError("offq_w4a4_linear_form", form)
    return form


def offq_kv4_quantize(kv: torch.Tensor, T: int, H: int, head_dim: int, ld_token: int, flags: int,
                      codes: torch.Tensor, scale: torch.Tensor, offset: Optional[torch.Tensor],
                      stream=None) -> None:
    _check("offq_kv4_quantize", load_library().offq_kv4_quantize(
        _ptr(kv), _dtype_code(kv), T, H, head_dim, ld_token, flags, _ptr(codes), _ptr(scale), _ptr(offset),
        _stream(stream)))


def offq_prepare_weight(w: torch.Tensor, N: int, K: int, g: int, rotate: bool, w_codes: torch.Tensor,
                        w_scale: torch.Tensor, w_offsum: torch.Tensor, stream=None) -> None:
    _check("offq_prepare_weight", load_library().offq_prepare_weight(
        _ptr(w), _dtype_code(w), N, K, g, 1 if rotate else 0, _ptr(w_codes), _ptr(w_scale), _ptr(w_offsum),
        _stream(stream)))


def offq_quantize_act_group(x: torch.Tensor, T: int, K: int, ldx: int, g: int, group: int, flags: int,
                            codes: torch.Tensor, scale: torch.Tensor, zero: torch.Tensor, stream=None) -> None:
    _check("offq_quantize_act_group", load_library().offq_quantize_act_group(
        _ptr(x), _dtype_code(x), T, K, ldx, g, group, flags, _ptr(codes), _ptr(scale), _ptr(zero), _stream(stream)))


def offq_weight_group_sums(w_codes: torch.Tensor, N: int, K: int, group: int, w_groupsum: torch.Tensor,
                           stream=None) -> None:
    _check("offq_weight_group_sums", load_library().offq_weight_group_sums(
        _ptr(w_codes), N, K, group, _ptr(w_groupsum), _stream(stream)))


def offq_w4a4_linear_group(a_codes: torch.Tensor, a_scale: torch.Tensor, a_zero: torch.Tensor, T: int, N: int,
                           K: int, group: int, w_codes: torch.Tensor, w_scale: torch.Tensor,
                           w_groupsum: torch.Tensor, out: torch.Tensor, ldo: int, stream=None) -> None:
    _check("offq_w4a4_linear_group", load_library().offq_w4a4_linear_group(
        _ptr(a_codes), _ptr(a_scale), _ptr(a_zero), T, N, K, group, _ptr(w_codes), _ptr(w_scale),
        _ptr(w_groupsum), _ptr(out), _dtype_code(out), ldo, _stream(stream)))


def offq_kv4_quantize_rotated(kv: torch.Tensor, T: int, H: int, head_dim: int, ld_token: int, rot: torch.Tensor,
                              flags: int, codes: torch.Tensor, scale: torch.Tensor, offset: Optional[torch.Tensor],
                              stream=None) -> None:
    _check("offq_kv4_quantize_rotated", load_library().offq_kv4_quantize_rotated(
        _ptr(kv), _dtype_code(kv), T, H, head_dim, ld_token, _ptr(rot), flags, _ptr(codes), _ptr(scale),
        _ptr(offset), _stream(stream)))


def offq_rotate_heads(x: torch.Tensor, T: int, H: int, head_dim: int, ld_token: int, rot: torch.Tensor,
                      out: torch.Tensor, ld_out: int, stream=None) -> None:
    _check("offq_rotate_heads", load_library().offq_rotate_heads(
        _ptr(x), _dtype_code(x), T, H, head_dim, ld_token, _ptr(rot), _ptr(out), _dtype_code(out), ld_out,
        _stream(stream)))


def offq_prepare_key_rotation(rot: torch.Tensor, H: int, head_dim: int, prepared: torch.Tensor,
                              stream=None) -> None:
    _check("offq_prepare_key_rotation", load_library().offq_prepare_key_rotation(
        _ptr(rot), H, head_dim, _ptr(prepared), _stream(stream)))


def offq_kv4_quantize_prepared(kv: torch.Tensor, T: int, H: int, head_dim: int, ld_token: int,
                               prepared: torch.Tensor, flags: int, codes: torch.Tensor, scale: torch.Tensor,
                               offset: Optional[torch.Tensor], stream=None) -> None:
    _check("offq_kv4_quantize_prepared", load_library().offq_kv4_quantize_prepared(
        _ptr(kv), _dtype_code(kv), T, H, head_dim, ld_token, _ptr(prepared), flags, _ptr(codes), _ptr(scale),
        _ptr(offset), _stream(stream)))


def offq_rotate_heads_prepared(x: torch.Tensor, T: int, H: int, head_dim: int, ld_token: int,
                               prepared: torch.Tensor, out: torch.Tensor, ld_out: int, stream=None) -> None:
    _check("offq_rotate_heads_prepared", load_library().offq_rotate_heads_prepared(
        _ptr(x), _dtype_code(x), T, H, head_dim, ld_token, _ptr(prepared), _ptr(out), _dtype_code(out), ld_out,
        _stream(stream)))


def offq_prepare_key_reflection(v: torch.Tensor, perm: torch.Tensor, H: int, head_dim: int,
                                prepared: torch.Tensor) -> None:
    """Host call: v [H, hd] float32, perm [H, hd] int32 and prepared (uint8) all in host memory."""
    for t in (v, perm, prepared):
        if t.device.type != "cpu" or not t.is_contiguous():
            raise ValueError("offq_prepare_key_reflection takes contiguous host tensors")
    _check("offq_prepare_key_reflection", load_library().offq_prepare_key_reflection(
        ctypes.c_void_p(v.data_ptr()), ctypes.c_void_p(perm.data_ptr()), H, head_dim,
        ctypes.c_void_p(prepared.data_ptr())))


def offq_kv4_quantize_reflected(kv: torch.Tensor, T: int, H: int, head_dim: int, ld_token: int,
                                prepared: torch.Tensor, flags: int, codes: torch.Tensor, scale: torch.Tensor,
                                offset: Optional[torch.Tensor], stream=None) -> None:
    _check("offq_kv4_quantize_reflected", load_library().offq_kv4_quantize_reflected(
        _ptr(kv), _dtype_code(kv), T, H, head_dim, ld_token, _ptr(prepared), flags, _ptr(codes), _ptr(scale),
        _ptr(offset), _stream(stream)))


def offq_rotate_heads_reflected(x: torch.Tensor, T: int, H: int, head_dim: int, ld_token: int,
                                prepared: torch.Tensor, out: torch.Tensor, ld_out: int, stream=None) -> None:
    _check("offq_rotate_heads_reflected", load_library().offq_rotate_heads_reflected(
        _ptr(x), _dtype_code(x), T, H, head_dim, ld_token, _ptr(prepared), _ptr(out), _dtype_code(out), ld_out,
        _stream(stream)))


def offq_get_device_status(stream=None) -> int:
    return load_library().offq_get_device_status(_stream(stream))


def offq_set_wait_cycles(cycles: int) -> None:
    """Test hook: budget of the persistent quantizers' waits for staged rows
    (0 restores the default)."""
    _check("offq_set_wait_cycles", load_library().offq_set_wait_cycles(cycles))


def offq_act_codes_bytes(T: int, K: int) -> int:
    return load_library().offq_act_codes_bytes(T, K)


def offq_weight_codes_bytes(N: int, K: int) -> int:
    return load_library().offq_weight_codes_bytes(N, K)


def padded_rows(R: int) -> int:
    """Rows a tiled code buffer holds for R rows (a multiple of 32)."""
    return (R + 31) // 32 * 32


# ---------------------------------------------------------------------------
# Allocating helpers (torch allocates; the entry points above compute).
# ---------------------------------------------------------------------------

@_on_its_stream
def quantize_act(x: torch.Tensor, g: int, rotate: bool = True, offset: bool = True,
                 stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    T, K = x.shape
    codes = torch.empty((padded_rows(T), K // 2), dtype=torch.uint8, device=x.device)
    scale = torch.empty((T,), dtype=torch.float32, device=x.device)
    off = torch.empty((T, K // g), dtype=torch.float32, device=x.device)
    flags = (OFFQ_ROTATE if rotate else 0) | (OFFQ_OFFSET if offset else 0)
    offq_quantize_act(x, T, K, x.stride(0), g, flags, codes, scale, off, stream)
    return codes, scale, off


@_on_its_stream
def kv4_quantize(kv: torch.Tensor, rotate: bool = True, offset: bool = True,
                 stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    T, H, hd = kv.shape
    if kv.stride(2) != 1 or kv.stride(1) != hd:
        raise ValueError("heads of a token must be contiguous")
    codes = torch.empty((T, H, hd // 2), dtype=torch.uint8, device=kv.device)
    scale = torch.empty((T, H), dtype=torch.float32, device=kv.device)
    off = torch.empty((T, H), dtype=torch.float32, device=kv.device)
    flags = (OFFQ_ROTATE if rotate else 0) | (OFFQ_OFFSET if offset else 0)
    offq_kv4_quantize(kv, T, H, hd, kv.stride(0), flags, codes, scale, off, stream)
    return codes, scale, off


@_on_its_stream
def prepare_weight(w: torch.Tensor, g: int, rotate: bool = True,
                   stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    N, K = w.shape
    w = w.contiguous()
    codes = torch.empty((padded_rows(N), K // 2), dtype=torch.uint8, device=w.device)
    scale = torch.empty((N,), dtype=torch.float32, device=w.device)
    rowsum = torch.empty((K // g, N), dtype=torch.float32, device=w.device)
    offq_prepare_weight(w, N, K, g, rotate, codes, scale, rowsum, stream)
    return codes, scale, rowsum


@_on_its_stream
def w4a4_linear(a_codes: torch.Tensor, a_scale: torch.Tensor, a_offset: Optional[torch.Tensor],
                w_codes: torch.Tensor, w_scale: torch.Tensor, w_offsum: torch.Tensor, g: int,
                out_dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None,
                acc_debug: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    T = a_scale.shape[0]
    K = a_codes.shape[1] * 2
    N = w_scale.shape[0]
    if out is None:
        out = torch.empty((T, N), dtype=out_dtype, device=a_codes.device)
    offq_w4a4_linear(a_codes, a_scale, a_offset, T, N, K, g, w_codes, w_scale, w_offsum, out, out.stride(0),
                     acc_debug, stream)
    return out


GROUP = 128  # activation group size of the per-group path (the paper's evaluated setting)


@_on_its_stream
def quantize_act_group(x: torch.Tensor, g: int, group: int = GROUP, rotate: bool = True,
                       stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Per-group asymmetric codes, scales and zero-points of token rows x [T, K]."""
    T, K = x.shape
    codes = torch.empty((padded_rows(T), K // 2), dtype=torch.uint8, device=x.device)
    scale = torch.empty((T, K // group), dtype=torch.float32, device=x.device)
    zero = torch.empty((T, K // group), dtype=torch.float32, device=x.device)
    offq_quantize_act_group(x, T, K, x.stride(0), g, group, OFFQ_ROTATE if rotate else 0, codes, scale, zero,
                            stream)
    return codes, scale, zero


@_on_its_stream
def weight_group_sums(w_codes: torch.Tensor, N: int, K: int, group: int = GROUP, stream=None) -> torch.Tensor:
    """Integer row sums of the weight codes per activation group, [K/group, N] float32."""
    sums = torch.empty((K // group, N), dtype=torch.float32, device=w_codes.device)
    offq_weight_group_sums(w_codes, N, K, group, sums, stream)
    return sums


@_on_its_stream
def w4a4_linear_group(a_codes: torch.Tensor, a_scale: torch.Tensor, a_zero: torch.Tensor,
                      w_codes: torch.Tensor, w_scale: torch.Tensor, w_groupsum: torch.Tensor,
                      group: int = GROUP, out_dtype: torch.dtype = torch.bfloat16,
                      out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    T = a_scale.shape[0]
    K = a_codes.shape[1] * 2
    N = w_scale.shape[0]
    if out is None:
        out = torch.empty((T, N), dtype=out_dtype, device=a_codes.device)
    offq_w4a4_linear_group(a_codes, a_scale, a_zero, T, N, K, group, w_codes, w_scale, w_groupsum, out,
                           out.stride(0), stream)
    return out


@_on_its_stream
def kv4_quantize_rotated(kv: torch.Tensor, rot: torch.Tensor, offset: bool = True,
                         stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Key-cache codes, scales and offsets of kv [T, H, hd] under per-head rotations rot [H, hd, hd]."""
    T, H, hd = kv.shape
    if kv.stride(2) != 1 or kv.stride(1) != hd:
        raise ValueError("heads of a token must be contiguous")
    codes = torch.empty((T, H, hd // 2), dtype=torch.uint8, device=kv.device)
    scale = torch.empty((T, H), dtype=torch.float32, device=kv.device)
    off = torch.empty((T, H), dtype=torch.float32, device=kv.device)
    offq_kv4_quantize_rotated(kv, T, H, hd, kv.stride(0), rot.contiguous(), OFFQ_OFFSET if offset else 0, codes,
                              scale, off, stream)
    return codes, scale, off


@_on_its_stream
def rotate_heads(x: torch.Tensor, rot: torch.Tensor, out_dtype: torch.dtype = torch.float32,
                 stream=None) -> torch.Tensor:
    """x [T, H, hd] rotated per head by rot [H, hd, hd] (y = x rot[h])."""
    T, H, hd = x.shape
    if x.stride(2) != 1 or x.stride(1) != hd:
        raise ValueError("heads of a token must be contiguous")
    out = torch.empty((T, H, hd), dtype=out_dtype, device=x.device)
    offq_rotate_heads(x, T, H, hd, x.stride(0), rot.contiguous(), out, out.stride(0), stream)
    return out


KEY_ROTATION_BYTES = 98304  # OFFQ_KEY_ROTATION_BYTES: one head's prepared rotation


@_on_its_stream
def prepare_key_rotation(rot: torch.Tensor, stream=None) -> torch.Tensor:
    """rot [H, hd, hd] float32 -> the prepared image [H, KEY_ROTATION_BYTES] (uint8)."""
    H, hd, _ = rot.shape
    prep = torch.empty((H, KEY_ROTATION_BYTES), dtype=torch.uint8, device=rot.device)
    offq_prepare_key_rotation(rot.contiguous(), H, hd, prep, stream)
    return prep


@_on_its_stream
def kv4_quantize_prepared(kv: torch.Tensor, prepared: torch.Tensor, offset: bool = True,
                          stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """kv4_quantize_rotated for bf16 kv [T, H, hd] with M given as prepare_key_rotation's image."""
    T, H, hd = kv.shape
    if kv.stride(2) != 1 or kv.stride(1) != hd:
        raise ValueError("heads of a token must be contiguous")
    codes = torch.empty((T, H, hd // 2), dtype=torch.uint8, device=kv.device)
    scale = torch.empty((T, H), dtype=torch.float32, device=kv.device)
    off = torch.empty((T, H), dtype=torch.float32, device=kv.device)
    offq_kv4_quantize_prepared(kv, T, H, hd, kv.stride(0), prepared, OFFQ_OFFSET if offset else 0, codes, scale,
                               off, stream)
    return codes, scale, off


@_on_its_stream
def rotate_heads_prepared(x: torch.Tensor, prepared: torch.Tensor, out_dtype: torch.dtype = torch.float32,
                          stream=None) -> torch.Tensor:
    """rotate_heads for bf16 x [T, H, hd] with M given as prepare_key_rotation's image."""
    T, H, hd = x.shape
    if x.stride(2) != 1 or x.stride(1) != hd:
        raise ValueError("heads of a token must be contiguous")
    out = torch.empty((T, H, hd), dtype=out_dtype, device=x.device)
    offq_rotate_heads_prepared(x, T, H, hd, x.stride(0), prepared, out, out.stride(0), stream)
    return out


KEY_REFLECTION_BYTES = 37376  # OFFQ_KEY_REFLECTION_BYTES: one head's structured rotation


def prepare_key_reflection(v: torch.Tensor, perm: torch.Tensor, device=None) -> torch.Tensor:
    """Top-1 directions v [H, hd] and permutations perm [H, hd] -> the structured
    image [H, KEY_REFLECTION_BYTES] (uint8), built on the host and copied to `device`."""
    H, hd = v.shape
    vh = v.detach().to("cpu", torch.float32).contiguous()
    ph = perm.detach().to("cpu", torch.int32).contiguous()
    img = torch.empty((H, KEY_REFLECTION_BYTES), dtype=torch.uint8)
    offq_prepare_key_reflection(vh, ph, H, hd, img)
    return img.to(device) if device is not None else img


@_on_its_stream
def kv4_quantize_reflected(kv: torch.Tensor, prepared: torch.Tensor, offset: bool = True,
                           stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Key-cache codes, scales and offsets of bf16 kv [T, H, hd] under the structured M = U3 P3 H3."""
    T, H, hd = kv.shape
    if kv.stride(2) != 1 or kv.stride(1) != hd:
        raise ValueError("heads of a token must be contiguous")
    codes = torch.empty((T, H, hd // 2), dtype=torch.uint8, device=kv.device)
    scale = torch.empty((T, H), dtype=torch.float32, device=kv.device)
    off = torch.empty((T, H), dtype=torch.float32, device=kv.device)
    offq_kv4_quantize_reflected(kv, T, H, hd, kv.stride(0), prepared, OFFQ_OFFSET if offset else 0, codes, scale,
                                off, stream)
    return codes, scale, off


@_on_its_stream
def rotate_heads_reflected(x: torch.Tensor, prepared: torch.Tensor, out_dtype: torch.dtype = torch.float32,
                           stream=None) -> torch.Tensor:
    """bf16 x [T, H, hd] rotated per head by the structured M = U3 P3 H3."""
    T, H, hd = x.shape
    if x.stride(2) != 1 or x.stride(1) != hd:
        raise ValueError("heads of a token must be contiguous")
    out = torch.empty((T, H, hd), dtype=out_dtype, device=x.device)
    offq_rotate_heads_reflected(x, T, H, hd, x.stride(0), prepared, out, out.stride(0), stream)
    return out


# ---------------------------------------------------------------------------
# Offline transform builder
# ---------------------------------------------------------------------------

@_on_its_stream
def top1_tokens(x: torch.Tensor, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """x [S, L, D] (contiguous tokens): per sequence the token of largest L-inf norm."""
    S, L, D = x.shape
    if x.stride(2) != 1:
        raise ValueError("channels must be contiguous")
    index = torch.empty((S,), dtype=torch.int32, device=x.device)
    rows = torch.empty((S, D), dtype=torch.float32, device=x.device)
    _check("offq_top1_tokens", load_library().offq_top1_tokens(
        _ptr(x), _dtype_code(x), S, L, D, x.stride(1), x.stride(0), _ptr(index), _ptr(rows), _stream(stream)))
    return index, rows


@_on_its_stream
def top1_direction(X: torch.Tensor, iters: int = 100, v0: Optional[torch.Tensor] = None,
                   stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Leading eigenvector of X^T X / N by power iteration (and X v)."""
    N, D = X.shape
    X = X.contiguous()
    v0 = torch.ones((D,), dtype=torch.float32, device=X.device) if v0 is None else v0.contiguous()
    v = torch.empty((D,), dtype=torch.float32, device=X.device)
    proj = torch.empty((N,), dtype=torch.float32, device=X.device)
    _check("offq_top1_direction", load_library().offq_top1_direction(
        _ptr(X), N, D, iters, _ptr(v0), _ptr(v), _ptr(proj), _stream(stream)))
    return v, proj


@_on_its_stream
def reflect_rows(A: torch.Tensor, v: torch.Tensor, stream=None) -> torch.Tensor:
    R, D = A.shape
    A = A.contiguous()
    out = torch.empty((R, D), dtype=torch.float32, device=A.device)
    _check("offq_reflect_rows", load_library().offq_reflect_rows(
        _ptr(A), R, D, _ptr(v), _ptr(out), _stream(stream)))
    return out


@_on_its_stream
def column_absmax(A: torch.Tensor, stream=None) -> torch.Tensor:
    R, D = A.shape
    A = A.contiguous()
    mag = torch.empty((D,), dtype=torch.float32, device=A.device)
    _check("offq_column_absmax", load_library().offq_column_absmax(
        _ptr(A), R, D, _ptr(mag), _stream(stream)))
    return mag


def sorted_grouping(mag: torch.Tensor, G: int) -> torch.Tensor:
    """Host call: the sorted-grouping permutation (int32, on the host)."""
    m = mag.detach().to("cpu", torch.float32).contiguous()
    perm = torch.empty((m.numel(),), dtype=torch.int32)
    _check("offq_sorted_grouping", load_library().offq_sorted_grouping(
        ctypes.c_void_p(m.data_ptr()), m.numel(), G, ctypes.c_void_p(perm.data_ptr())))
    return perm


@_on_its_stream
def fuse_rotation(W: torch.Tensor, v: torch.Tensor, perm: torch.Tensor, g: int, stream=None) -> torch.Tensor:
    N, D = W.shape
    W, perm = W.contiguous(), perm.to(W.device, torch.int32).contiguous()
    out = torch.empty((N, D), dtype=torch.float32, device=W.device)
    _check("offq_fuse_rotation", load_library().offq_fuse_rotation(
        _ptr(W), N, D, _ptr(v), _ptr(perm), g, _ptr(out), _stream(stream)))
    return out


# ---------------------------------------------------------------------------
# MXFP4 residuals with the offset as zero-point
# ---------------------------------------------------------------------------

def offq_quantize_act_mx(x: torch.Tensor, T: int, K: int, ldx: int, g: int, flags: int, codes: torch.Tensor,
                         shifts: torch.Tensor, row_scale: torch.Tensor, offset: Optional[torch.Tensor],
                         stream=None) -> None:
    _check("offq_quantize_act_mx", load_library().offq_quantize_act_mx(
        _ptr(x), _dtype_code(x), T, K, ldx, g, flags, _ptr(codes), _ptr(shifts), _ptr(row_scale), _ptr(offset),
        _stream(stream)))


def offq_prepare_weight_mx(w: torch.Tensor, N: int, K: int, g: int, rotate: int, w_codes: torch.Tensor,
                           w_shifts: torch.Tensor, w_scale: torch.Tensor, w_offsum: torch.Tensor,
                           stream=None) -> None:
    _check("offq_prepare_weight_mx", load_library().offq_prepare_weight_mx(
        _ptr(w), _dtype_code(w), N, K, g, rotate, _ptr(w_codes), _ptr(w_shifts), _ptr(w_scale), _ptr(w_offsum),
        _stream(stream)))


def offq_mx_linear(a_codes, a_shifts, a_scale, a_offset, T: int, N: int, K: int, g: int, w_codes, w_shifts,
                   w_scale, w_offsum, out: torch.Tensor, ldo: int, stream=None) -> None:
    _check("offq_mx_linear", load_library().offq_mx_linear(
        _ptr(a_codes), _ptr(a_shifts), _ptr(a_scale), _ptr(a_offset), T, N, K, g, _ptr(w_codes), _ptr(w_shifts),
        _ptr(w_scale), _ptr(w_offsum), _ptr(out), _dtype_code(out), ldo, _stream(stream)))


def mx_shift_bytes(R: int, K: int) -> int:
    return load_library().offq_mx_shift_bytes(R, K)


def quantize_act_mx(x: torch.Tensor, g: int, rotate: bool = True, offset: bool = True):
    """Allocating wrapper: (codes, shifts, row_scale, offset) for rows x [T, K]."""
    T, K = x.shape
    dev = x.device
    codes = torch.empty((padded_rows(T), K // 2), dtype=torch.uint8, device=dev)
    shifts = torch.empty((mx_shift_bytes(T, K),), dtype=torch.uint8, device=dev)
    scale = torch.empty((T,), dtype=torch.float32, device=dev)
    off = torch.empty((T, K // g), dtype=torch.float32, device=dev)
    flags = (OFFQ_ROTATE if rotate else 0) | (OFFQ_OFFSET if offset else 0)
    offq_quantize_act_mx(x, T, K, x.stride(0), g, flags, codes, shifts, scale, off)
    return codes, shifts, scale, off


def prepare_weight_mx(w: torch.Tensor, g: int, rotate: bool = True):
    """Allocating wrapper: (codes, shifts, scale, offsum) for weights w [N, K]."""
    N, K = w.shape
    dev = w.device
    codes = torch.empty((padded_rows(N), K // 2), dtype=torch.uint8, device=dev)
    shifts = torch.empty((mx_shift_bytes(N, K),), dtype=torch.uint8, device=dev)
    scale = torch.empty((N,), dtype=torch.float32, device=dev)
    offsum = torch.empty((K // g, N), dtype=torch.float32, device=dev)
    offq_prepare_weight_mx(w.contiguous(), N, K, g, 1 if rotate else 0, codes, shifts, scale, offsum)
    return codes, shifts, scale, offsum


# ---------------------------------------------------------------------------
# Between the projections and attention: norm, rotary positions and H3 of heads,
# the paged 4-bit cache, attention
# ---------------------------------------------------------------------------

class KV4Cache(NamedTuple):
    """The paged 4-bit cache of one layer: codes [pages, H, page_size, hd / 2] uint8 and
    (scale, offset) pairs [pages, H, page_size, 2] float32 of keys and of values."""
    k_codes: torch.Tensor
    k_params: torch.Tensor
    v_codes: torch.Tensor
    v_params: torch.Tensor


def kv4_cache(pages: int, heads: int, head_dim: int = 128, page_size: int = 64, device=None) -> KV4Cache:
    """Uninitialised pages (a slot means something once a token was written to it)."""
    def codes():
        return torch.empty((pages, heads, page_size, head_dim // 2), dtype=torch.uint8, device=device or "cuda")

    def params():
        return torch.empty((pages, heads, page_size, 2), dtype=torch.float32, device=device or "cuda")
    return KV4Cache(codes(), params(), codes(), params())


def rope_table(max_pos: int, rot_dim: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
               original_len: int = 4096, beta_fast: float = 32.0, beta_slow: float = 1.0, device=None) -> torch.Tensor:
    """Rotary table [max_pos, rot_dim] float32: cosines of rot_dim / 2 angles, then their sines, computed in float64.

    Frequencies are f_m = base^(-2m / rot_dim). Contexts ``factor`` times longer than the trained ``original_len``:
      linear  positions divided by factor;
      ntk     base * factor^(rot_dim / (rot_dim - 2)): the slowest frequency is divided by factor, the fastest kept;
      yarn    f_m / factor where the trained length holds fewer than beta_slow turns, f_m where it holds more than
              beta_fast, a linear ramp between, and cosines and sines times 0.1 ln(factor) + 1.
    """
    if rot_dim < 2 or rot_dim % 2 or max_pos < 1:
        raise ValueError("rope_table needs max_pos >= 1 and an even rot_dim >= 2")
    if scaling not in ("none", "linear", "ntk", "yarn") or factor < 1.0:
        raise ValueError(f"unknown scaling {scaling!r} or factor below 1")
    m = torch.arange(rot_dim // 2, dtype=torch.float64)
    if scaling == "ntk":
        if rot_dim < 4:
            raise ValueError("ntk scaling needs rot_dim >= 4")
        base = base * factor ** (rot_dim / (rot_dim - 2))
    freq = base ** (-2.0 * m / rot_dim)
    amp = 1.0
    if scaling == "linear":
        freq = freq / factor
    elif scaling == "yarn":
        def at(turns):  # the m whose frequency makes that many turns over the trained length
            return rot_dim * math.log(original_len / (2 * math.pi * turns)) / (2 * math.log(base))
        lo, hi = max(0.0, math.floor(at(beta_fast))), min(rot_dim - 1.0, math.ceil(at(beta_slow)))
        ramp = ((m - lo) / max(hi - lo, 1e-3)).clamp(0.0, 1.0)
        freq = freq / factor * ramp + freq * (1.0 - ramp)
        amp = 0.1 * math.log(factor) + 1.0
    a = torch.arange(max_pos, dtype=torch.float64)[:, None] * freq
    return torch.cat([a.cos() * amp, a.sin() * amp], 1).to(torch.float32).to(device or "cuda")


def offq_rope_heads(x: torch.Tensor, T: int, H: int, head_dim: int, ld_token: int, positions: Optional[torch.Tensor],
                    table: Optional[torch.Tensor], max_pos: int, rot_dim: int, norm: Optional[torch.Tensor], eps: float,
                    flags: int, out: torch.Tensor, ld_out: int, stream=None) -> None:
    _check("offq_rope_heads", load_library().offq_rope_heads(
        _ptr(x), _dtype_code(x), T, H, head_dim, ld_token, _ptr(positions), _ptr(table), max_pos, rot_dim, _ptr(norm),
        eps, flags, _ptr(out), _dtype_code(out), ld_out, _stream(stream)))


def offq_kv4_paged_write(q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, T: int, Hq: int, H: int,
                         head_dim: int, ld_q: int, ld_k: int, ld_v: int, positions: Optional[torch.Tensor],
                         table: Optional[torch.Tensor], max_pos: int, rot_dim: int, q_norm: Optional[torch.Tensor],
                         k_norm: Optional[torch.Tensor], eps: float, flags: int, slots: torch.Tensor,
                         cache: KV4Cache, pages: int, page_size: int, q_out: Optional[torch.Tensor], ld_q_out: int,
                         stream=None) -> None:
    _check("offq_kv4_paged_write", load_library().offq_kv4_paged_write(
        _ptr(q), _ptr(k), _ptr(v), _dtype_code(k), T, Hq, H, head_dim, ld_q, ld_k, ld_v, _ptr(positions), _ptr(table),
        max_pos, rot_dim, _ptr(q_norm), _ptr(k_norm), eps, flags, _ptr(slots), _ptr(cache.k_codes),
        _ptr(cache.k_params), _ptr(cache.v_codes), _ptr(cache.v_params), pages, page_size, _ptr(q_out),
        _dtype_code(q_out) if q_out is not None else OFFQ_F32, ld_q_out, _stream(stream)))


def offq_kv4_paged_read(cache: KV4Cache, pages: int, page_size: int, H: int, head_dim: int, slots: torch.Tensor, T: int,
                        flags: int, k_out: Optional[torch.Tensor], v_out: Optional[torch.Tensor], out_dtype: int,
                        ld_k: int, ld_v: int, stream=None) -> None:
    _check("offq_kv4_paged_read", load_library().offq_kv4_paged_read(
        _ptr(cache.k_codes), _ptr(cache.k_params), _ptr(cache.v_codes), _ptr(cache.v_params), pages, page_size, H,
        head_dim, _ptr(slots), T, flags, _ptr(k_out), _ptr(v_out), out_dtype, ld_k, ld_v, _stream(stream)))


def offq_paged_attention(q: torch.Tensor, Tq: int, Hq: int, H: int, head_dim: int, ld_q: int, cache: KV4Cache,
                         pages: int, page_size: int, block_table: torch.Tensor, ld_table: int, lens: torch.Tensor,
                         cu_q: torch.Tensor, B: int, max_q: int, scale: float, out: torch.Tensor, ld_out: int,
                         lse: Optional[torch.Tensor], workspace: Optional[torch.Tensor], workspace_bytes: int,
                         stream=None) -> None:
    _check("offq_paged_attention", load_library().offq_paged_attention(
        _ptr(q), _dtype_code(q), Tq, Hq, H, head_dim, ld_q, _ptr(cache.k_codes), _ptr(cache.k_params),
        _ptr(cache.v_codes), _ptr(cache.v_params), pages, page_size, _ptr(block_table), ld_table, _ptr(lens),
        _ptr(cu_q), B, max_q, scale, _ptr(out), ld_out, _ptr(lse), _ptr(workspace), workspace_bytes, _stream(stream)))


def paged_attention_workspace(Tq: int, Hq: int, H: int, head_dim: int, B: int, max_q: int) -> int:
    return load_library().offq_paged_attention_workspace(Tq, Hq, H, head_dim, B, max_q)


@functools.lru_cache(maxsize=1024)
def _workspace_bytes(device: int, Tq: int, Hq: int, H: int, head_dim: int, B: int, max_q: int) -> int:
    need = paged_attention_workspace(Tq, Hq, H, head_dim, B, max_q)
    if need < 0:
        raise LookupError  # not kept; the call itself says what is wrong with its sizes
    return need


def offq_prompt_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, T: int, Hq: int, H: int, head_dim: int,
                          ld_q: int, ld_k: int, ld_v: int, cu: torch.Tensor, B: int, scale: float, causal: bool,
                          out: torch.Tensor, ld_out: int, lse: Optional[torch.Tensor], stream=None) -> None:
    _check("offq_prompt_attention", load_library().offq_prompt_attention(
        _ptr(q), _ptr(k), _ptr(v), _dtype_code(q), T, Hq, H, head_dim, ld_q, ld_k, ld_v, _ptr(cu), B, scale,
        1 if causal else 0, _ptr(out), ld_out, _ptr(lse), _stream(stream)))


def _heads(x: torch.Tensor) -> Tuple[int, int, int, int]:
    """(T, H, hd, ld_token) of x [T, H, hd] with contiguous heads."""
    T, H, hd = x.shape
    ld, between, inner = x.stride()
    if inner != 1 or (H > 1 and between != hd):
        raise ValueError("heads of a token must be contiguous")
    return T, H, hd, ld if T > 1 else H * hd


def _like(what: str, t: Optional[torch.Tensor], dtype: torch.dtype, shape: tuple) -> None:
    """t is a contiguous tensor of that type and shape, or None."""
    if t is not None and (t.dtype is not dtype or t.shape != shape or not t.is_contiguous()):
        raise ValueError(f"{what} must be a contiguous {dtype} tensor of shape {tuple(shape)}")


def _rotary(positions, table, T):
    """(max_pos, rot_dim) of a rotary table, (0, 0) without one."""
    if table is None:
        return 0, 0
    if positions is None or table.dim() != 2:
        raise ValueError("a rotary table [max_pos, rot_dim] goes with positions [T]")
    _like("positions", positions, torch.int32, (T,))
    _like("table", table, torch.float32, table.shape)
    return table.shape


def _cache_shape(cache: KV4Cache, H: Optional[int], hd: Optional[int]):
    kc, kp, vc, vp = cache
    pages, heads, page_size, half = shape = kc.shape
    if (H is not None and heads != H) or (hd is not None and 2 * half != hd):
        raise ValueError(f"the cache holds {heads} heads of {2 * half}")
    _like("cache codes", kc, torch.uint8, shape)
    _like("cache codes", vc, torch.uint8, shape)
    _like("cache params", kp, torch.float32, (pages, heads, page_size, 2))
    _like("cache params", vp, torch.float32, (pages, heads, page_size, 2))
    return pages, heads, page_size, 2 * half


@_on_its_stream
def rope_heads(x: torch.Tensor, positions: Optional[torch.Tensor] = None, table: Optional[torch.Tensor] = None,
               norm: Optional[torch.Tensor] = None, eps: float = 1e-6, interleaved: bool = False, rotate: bool = False,
               out_dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """x [T, H, hd]: RMS norm (norm [H, hd]), rotary positions (rope_table) and H3, each if asked for, in one pass."""
    T, H, hd, ld = _heads(x)
    max_pos, rot = _rotary(positions, table, T)
    _like("norm", norm, torch.float32, (H, hd))
    ld_out = H * hd
    if out is None:
        out = torch.empty((T, H, hd), dtype=out_dtype or x.dtype, device=x.device)
    elif out.shape != x.shape:
        raise ValueError("out has x's shape")
    else:
        ld_out = _heads(out)[3]
    flags = (OFFQ_ROTATE if rotate else 0) | (OFFQ_INTERLEAVED if interleaved else 0)
    offq_rope_heads(x, T, H, hd, ld, positions, table, max_pos, rot, norm, eps, flags, out, ld_out, stream)
    return out


@_on_its_stream
def kv4_paged_write(cache: KV4Cache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor,
                    positions: Optional[torch.Tensor] = None, table: Optional[torch.Tensor] = None,
                    q: Optional[torch.Tensor] = None, q_norm: Optional[torch.Tensor] = None,
                    k_norm: Optional[torch.Tensor] = None, eps: float = 1e-6, interleaved: bool = False,
                    rotate: bool = True, rotate_v: bool = False, offset: bool = True,
                    out_dtype: Optional[torch.dtype] = None, stream=None) -> Optional[torch.Tensor]:
    """Keys and values [T, H, hd] into the slots [T] (int64) of the cache, the keys after k_norm, rotary positions and
    H3; returns the queries q [T, Hq, hd] after the same (None without q)."""
    T, H, hd, ld_k = _heads(k)
    if v.shape != k.shape or v.dtype != k.dtype:
        raise ValueError("keys and values have one shape and type")
    pages, _, page_size, _ = _cache_shape(cache, H, hd)
    max_pos, rot = _rotary(positions, table, T)
    _like("slots", slots, torch.int64, (T,))
    _like("k_norm", k_norm, torch.float32, (H, hd))
    Hq, ld_q, q_out = 0, 0, None
    if q is not None:
        Tq, Hq, hq, ld_q = _heads(q)
        if (Tq, hq) != (T, hd) or q.dtype != k.dtype:
            raise ValueError("queries have the keys' tokens, head size and type")
        _like("q_norm", q_norm, torch.float32, (Hq, hd))
        q_out = torch.empty((T, Hq, hd), dtype=out_dtype or q.dtype, device=q.device)
    flags = ((OFFQ_ROTATE if rotate else 0) | (OFFQ_OFFSET if offset else 0) | (OFFQ_INTERLEAVED if interleaved else 0)
             | (OFFQ_ROTATE_V if rotate_v else 0))
    offq_kv4_paged_write(q, k, v, T, Hq, H, hd, ld_q, ld_k, _heads(v)[3], positions, table, max_pos, rot, q_norm, k_norm,
                         eps, flags, slots, cache, pages, page_size, q_out, Hq * hd, stream)
    return q_out


@_on_its_stream
def kv4_paged_read(cache: KV4Cache, slots: torch.Tensor, rotate: bool = True, rotate_v: bool = False,
                   out_dtype: torch.dtype = torch.bfloat16, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Keys (H3 undone with rotate) and values [T, H, hd] of the tokens in slots [T] (int64)."""
    pages, H, page_size, hd = _cache_shape(cache, None, None)
    T = slots.shape[0]
    _like("slots", slots, torch.int64, (T,))
    k = torch.empty((T, H, hd), dtype=out_dtype, device=slots.device)
    v = torch.empty((T, H, hd), dtype=out_dtype, device=slots.device)
    flags = (OFFQ_ROTATE if rotate else 0) | (OFFQ_ROTATE_V if rotate_v else 0)
    offq_kv4_paged_read(cache, pages, page_size, H, hd, slots, T, flags, k, v, _dtype_code(k), H * hd, H * hd, stream)
    return k, v


@_on_its_stream
def paged_attention(q: torch.Tensor, cache: KV4Cache, block_table: torch.Tensor, lens: torch.Tensor,
                    cu_q: torch.Tensor, max_q: int, scale: Optional[float] = None, lse: bool = False,
                    out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None):
    """New tokens' queries q [Tq, Hq, hd] over the pages block_table [B, width] (int32) of lens [B] cached tokens;
    sequence b's queries are rows cu_q[b] .. cu_q[b + 1] - 1 and its last tokens. A length may not pass the columns of
    block_table (a part of a wider table is copied). Returns out, or (out, lse [Tq, Hq])."""
    Tq, Hq, hd, ld_q = _heads(q)
    pages, H, page_size, _ = _cache_shape(cache, None, hd)
    B = lens.shape[0]
    _like("lens", lens, torch.int32, (B,))
    _like("cu_q", cu_q, torch.int32, (B + 1,))
    if block_table.dim() != 2:
        raise ValueError("block_table must be int32 [B, width] with contiguous rows")
    listed, width = block_table.shape
    ld_table, inner = block_table.stride()
    if block_table.dtype is not torch.int32 or listed != B or (width > 1 and inner != 1):
        raise ValueError("block_table must be int32 [B, width] with contiguous rows")
    if B > 1 and ld_table != width:
        # The library's ld_table is the pages a sequence can hold as well as the way to the next row: columns that were
        # not given would count as pages.
        block_table = block_table.contiguous()
    ld_out = Hq * hd
    if out is None:
        out = torch.empty((Tq, Hq, hd), dtype=q.dtype, device=q.device)
    elif out.shape != q.shape or out.dtype != q.dtype:
        raise ValueError("out has q's shape and type")
    else:
        ld_out = _heads(out)[3]
    if workspace is None:
        try:
            need = _workspace_bytes(q.get_device(), Tq, Hq, H, hd, B, max_q)
        except LookupError:
            need = 0
        workspace = torch.empty((need,), dtype=torch.uint8, device=q.device) if need > 0 else None
    stats = torch.empty((Tq, Hq), dtype=torch.float32, device=q.device) if lse else None
    offq_paged_attention(q, Tq, Hq, H, hd, ld_q, cache, pages, page_size, block_table,
                         width, lens, cu_q, B, max_q,
                         scale if scale is not None else hd ** -0.5, out, ld_out, stats, workspace,
                         workspace.nbytes if workspace is not None else 0, stream)
    return (out, stats) if lse else out


@_on_its_stream
def prompt_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu: torch.Tensor, scale: Optional[float] = None,
                     causal: bool = True, lse: bool = False, out: Optional[torch.Tensor] = None, stream=None):
    """Attention inside packed sequences: rows cu[b] .. cu[b + 1] - 1 of q [T, Hq, hd] and k, v [T, H, hd] are sequence
    b. Returns out, or (out, lse [T, Hq])."""
    T, Hq, hd, ld_q = _heads(q)
    Tk, H, hk, ld_k = _heads(k)
    if (Tk, hk) != (T, hd) or v.shape != k.shape or k.dtype != q.dtype or v.dtype != q.dtype:
        raise ValueError("queries, keys and values have the same tokens, head size and type")
    _like("cu", cu, torch.int32, cu.shape[:1])
    ld_out = Hq * hd
    if out is None:
        out = torch.empty((T, Hq, hd), dtype=q.dtype, device=q.device)
    elif out.shape != q.shape or out.dtype != q.dtype:
        raise ValueError("out has q's shape and type")
    else:
        ld_out = _heads(out)[3]
    stats = torch.empty((T, Hq), dtype=torch.float32, device=q.device) if lse else None
    offq_prompt_attention(q, k, v, T, Hq, H, hd, ld_q, ld_k, _heads(v)[3], cu, cu.shape[0] - 1,
                          scale if scale is not None else hd ** -0.5, causal, out, ld_out, stats, stream)
    return (out, stats) if lse else out
