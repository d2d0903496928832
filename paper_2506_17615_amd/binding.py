"""Thin Python binding of libequarx.so: argument marshalling only.

The ordinary call -- plain contiguous GPU tensors, nothing to refuse -- is marshalled by the extension `_marshal`
(csrc/marshal.cpp); whatever that one hands back goes through the checks written out here.

Every function has the name and meaning of the C entry point declared in
``include/equarx.h``; tensors are torch CUDA tensors used purely as device
memory, and work is enqueued on torch's current stream.  There is no CPU
fallback: if the HIP library is missing, loading raises.
"""
from __future__ import annotations

import ctypes
import importlib.util
import os
import warnings
from typing import NamedTuple

import torch

from . import build as _build

_lib = None


class _Unloaded:
    """Stands in for the extension until the first call needs the library."""

    def __getattr__(self, name):
        load()
        return getattr(_native, name)


_native = _Unloaded()


class _PythonOnly:
    """In the extension's place where there is none for this interpreter and this torch: hands every call to the checks here."""

    def __getattr__(self, name):
        return lambda *args: -1


def _extension(addresses):
    """The extension, bound to the library; or, with a warning that says why, _PythonOnly."""
    path = _build.MARSHAL_PATH
    try:
        if not os.path.exists(path):
            raise ImportError(f"{path} is missing: build it (python -m paper_2506_17615_amd.build)")
        spec = importlib.util.spec_from_file_location(__package__ + "._marshal", path)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        if module.torch_version != torch.__version__:
            raise ImportError(f"{path} was built for torch {module.torch_version}, this is {torch.__version__}: build it again")
        module.bind(addresses)
        return module
    except ImportError as e:
        warnings.warn(f"calls are marshalled in Python, 5 to 11 us each: {e}", RuntimeWarning, stacklevel=3)
        return _PythonOnly()


STATUS_OK = 0
STATUS_NULL_POINTER = 1
STATUS_BAD_SHAPE = 2
STATUS_BAD_BLOCK = 3
STATUS_MISALIGNED = 4
STATUS_WORKSPACE_TOO_SMALL = 5
STATUS_DEVICE_ERROR = 6
MAX_PARTIALS = 64
BLOCK_SIZES = (32, 64, 128, 256, 512)
SEMI_LOOP, RS_UNQUANTIZED, AG_UNQUANTIZED, RING_ORDER = 1, 2, 4, 8

class _CCache(ctypes.Structure):
    """equarx_cache of include/equarx.h."""
    _fields_ = [("k_codes", ctypes.c_void_p), ("k_scales", ctypes.c_void_p), ("v_codes", ctypes.c_void_p),
                ("v_scales", ctypes.c_void_p), ("pages", ctypes.c_int64), ("heads", ctypes.c_int32), ("page", ctypes.c_int32),
                ("dim", ctypes.c_int32), ("block", ctypes.c_int32)]


# name -> (restype, argtypes); SIGNATURES mirrors include/equarx.h, DEVTOOLS_SIGNATURES include/equarx_devtools.h
_vp, _i64, _i32, _sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t
SIGNATURES = {
    "equarx_quantize": (ctypes.c_int, [_vp, _i64, _i32, _vp, _vp, _vp]),
    "equarx_quantize_batch": (ctypes.c_int, [ctypes.POINTER(_vp), ctypes.POINTER(_vp), ctypes.POINTER(_vp), _i32, _i64,
                                             _i32, _vp]),
    "equarx_dequantize": (ctypes.c_int, [_vp, _vp, _i64, _i32, _vp, _vp]),
    "equarx_reduce_stage": (ctypes.c_int, [_vp, _vp, _vp, _i64, _i32, _vp, _vp, _vp]),
    "equarx_reduce_quantized": (ctypes.c_int, [ctypes.POINTER(_vp), _i32, _i64, _i32, _vp, _vp, _sz, _vp, _vp, _vp]),
    "equarx_reduce_quantized_static": (ctypes.c_int, [ctypes.POINTER(_vp), _i32, _i64, _i32, _vp, _vp]),
    "equarx_reduce_quantized_fused_ends": (ctypes.c_int, [ctypes.POINTER(_vp), _i32, _i64, _i32, _vp, _vp, _sz, _vp]),
    "equarx_reduce_fused": (ctypes.c_int, [ctypes.POINTER(_vp), _i32, _i64, _i32, _vp, _vp, _vp, _vp]),
    "equarx_reduce_variant": (ctypes.c_int, [ctypes.POINTER(_vp), _i32, _i64, _i32, ctypes.c_uint32, _vp, _vp]),
    "equarx_reduce_variant_hops": (ctypes.c_int, [ctypes.POINTER(_vp), _i32, _i64, _i32, ctypes.c_uint32, _vp, _vp, _sz, _vp]),
    "equarx_variant_workspace_bytes": (_sz, [ctypes.c_uint32, _i32, _i64, _i32]),
    "equarx_reduce_flat": (ctypes.c_int, [_vp, ctypes.POINTER(_vp), ctypes.POINTER(_vp), _i32, _i64, _i32, _vp, _vp, _vp,
                                          _vp]),
    "equarx_quantize_strided": (ctypes.c_int, [_vp, _i64, _i32, _vp, _vp, _vp]),
    "equarx_dequantize_strided": (ctypes.c_int, [_vp, _vp, _i64, _i32, _vp, _vp]),
    "equarx_reduce_stage_strided": (ctypes.c_int, [_vp, _vp, _vp, _i64, _i32, _vp, _vp, _vp]),
    "equarx_reduce_quantized_strided": (ctypes.c_int, [ctypes.POINTER(_vp), _i32, _i64, _i32, _vp, _vp, _sz, _vp]),
    "equarx_reduce_fused_strided": (ctypes.c_int, [ctypes.POINTER(_vp), _i32, _i64, _i32, _vp, _vp]),
    "equarx_reduce_variant_strided": (ctypes.c_int, [ctypes.POINTER(_vp), _i32, _i64, _i32, ctypes.c_uint32, _vp, _vp]),
    "equarx_reduce_variant_hops_strided": (ctypes.c_int, [ctypes.POINTER(_vp), _i32, _i64, _i32, ctypes.c_uint32, _vp, _vp,
                                                          _sz, _vp]),
    "equarx_mx4_row_blocks": (_i64, [_i64]),
    "equarx_mx4_quantize": (ctypes.c_int, [_vp, _i64, _i64, _i64, _vp, _vp, _vp]),
    "equarx_mx4_dequantize": (ctypes.c_int, [_vp, _vp, _i64, _i64, _vp, _i64, _vp]),
    "equarx_mx4_product": (ctypes.c_int, [_vp, _vp, _vp, _vp, _i64, _i64, _i64, _vp, _i64, _vp, _sz, _vp]),
    "equarx_mx4_linear": (ctypes.c_int, [_vp, _i64, _vp, _vp, _i64, _i64, _i64, _vp, _i64, _vp, _sz, _vp]),
    "equarx_mx4_workspace_bytes": (_sz, [_i64, _i64, _i64]),
    "equarx_cache_write": (ctypes.c_int, [ctypes.POINTER(_CCache), _vp, _i64, _i64, _vp, _i64, _i64, _i64, _vp, _vp]),
    "equarx_cache_read": (ctypes.c_int, [ctypes.POINTER(_CCache), _vp, _i64, _vp, _vp, _i32, _i64, _i64, _vp, _vp, _vp]),
    "equarx_cache_attention": (ctypes.c_int, [ctypes.POINTER(_CCache), _vp, _i64, _i32, _i64, _i64, _vp, _vp, _i64, _vp, _i32,
                                              ctypes.c_float, _i32, _i64, ctypes.c_uint32, _i32, _vp, _vp, _vp, _sz, _vp]),
    "equarx_cache_attention_workspace_bytes": (_sz, [_i32, _i32, _i64, _i32, _i32, _i32, _i64]),
    "equarx_cache_attention_most_workspace_bytes": (_sz, [_i32, _i32, _i64, _i32, _i32, _i64]),
    "equarx_workspace_bytes": (_sz, [_i32, _i64, _i32]),
    "equarx_num_blocks": (_i64, [_i64, _i32]),
    "equarx_wire_row_codes": (_i64, [_i64]),
    "equarx_wire_row_scales": (_i64, [_i64, _i32]),
    "equarx_status_string": (ctypes.c_char_p, [ctypes.c_int]),
}
DEVTOOLS_SIGNATURES = {
    "equarx_calib_hop_traffic": (ctypes.c_int, [ctypes.POINTER(_vp), _i32, _i64, _i32, _vp, _vp, _vp, _vp, _vp]),
    "equarx_calib_copy": (ctypes.c_int, [_vp, _vp, _sz, _vp]),
    "equarx_calib_empty_launches": (ctypes.c_int, [_i32, _i32, _vp]),
    "equarx_calib_interleaved_chains": (ctypes.c_int, [ctypes.POINTER(_vp), _i32, _i32, _i64, _i32, ctypes.POINTER(_vp),
                                                       ctypes.POINTER(_vp), _sz, _i32, _vp]),
    "equarx_selftest_quotients": (ctypes.c_int, [ctypes.c_uint32, ctypes.c_uint64, _vp, _vp]),
    "equarx_selftest_rounding": (ctypes.c_int, [ctypes.c_uint32, ctypes.c_uint64, _vp, _vp]),
    "equarx_eval_quotients": (ctypes.c_int, [_vp, _i64, _vp, _vp, _vp]),
    "equarx_time_launch_span": (None, [_i32, _i32, _vp, _vp]),
    "equarx_time_next_launch": (None, [_vp, _vp]),
    "equarx_time_cancel": (None, []),
}


class EquarxError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = int(status)
        super().__init__(f"{where}: status {status} ({status_string(status)})")


def lib_path() -> str:
    return _build.LIB_PATH


def load() -> ctypes.CDLL:
    """Open libequarx.so (built in-tree by ``build.build()``); raises if it is not there."""
    global _lib, _native
    if _lib is None:
        path = lib_path()
        if not os.path.exists(path):
            raise RuntimeError(
                f"{path} is missing: build it first (python -m paper_2506_17615_amd.build); "
                "there is no fallback path")
        lib = ctypes.CDLL(path)
        for name, (res, args) in {**SIGNATURES, **DEVTOOLS_SIGNATURES}.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        native = _extension({name: ctypes.cast(getattr(lib, name), _vp).value for name in SIGNATURES})
        _lib, _native = lib, native
    return _lib


def status_string(status: int) -> str:
    return load().equarx_status_string(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != STATUS_OK:
        raise EquarxError(status, where)


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


def _need(t, dtype, count: int, what: str) -> None:
    """Host-side guard: a buffer handed to a kernel is a CUDA tensor of the right type, contiguous, long enough."""
    if count == 0:
        return
    if t is None or not t.is_cuda or t.dtype != dtype or not t.is_contiguous() or t.numel() < count:
        raise ValueError(f"{what}: need a contiguous CUDA {dtype} tensor of at least {count} elements")


def num_blocks(n: int, block: int) -> int:
    return int(load().equarx_num_blocks(n, block))


def workspace_bytes(P: int, n: int, block: int) -> int:
    return int(load().equarx_workspace_bytes(P, n, block))


def wire_row_codes(n: int) -> int:
    return int(load().equarx_wire_row_codes(n))


def wire_row_scales(n: int, block: int) -> int:
    return int(load().equarx_wire_row_scales(n, block))


def equarx_quantize(x_bf16: torch.Tensor, block: int, codes: torch.Tensor, scales: torch.Tensor) -> None:
    """codes[n] int8, scales[nb] fp32 <- Q_B(x_bf16[n])."""
    status = _native.equarx_quantize(x_bf16, block, codes, scales)
    if status >= 0:
        return _check(status, "equarx_quantize")
    n = x_bf16.numel()
    _need(x_bf16, torch.bfloat16, n, "x_bf16")
    _need(codes, torch.int8, n, "codes")
    _need(scales, torch.float32, num_blocks(n, block), "scales")
    _check(load().equarx_quantize(_ptr(x_bf16), x_bf16.numel(), block, _ptr(codes), _ptr(scales), _stream()),
           "equarx_quantize")


def equarx_quantize_batch(xs, block: int, codes_list, scales_list) -> None:
    """equarx_quantize on several bf16 tensors of equal length in one launch."""
    status = _native.equarx_quantize_batch(xs, block, codes_list, scales_list)
    if status >= 0:
        return _check(status, "equarx_quantize_batch")
    count = len(xs)
    if len(codes_list) != count or len(scales_list) != count:
        raise ValueError("xs, codes_list and scales_list differ in length")
    n = xs[0].numel() if count else 0
    nb = num_blocks(n, block) if count else 0
    for x, c, s in zip(xs, codes_list, scales_list):
        _need(x, torch.bfloat16, n, "x_bf16")
        if x.numel() != n:
            raise ValueError("tensors differ in length")
        _need(c, torch.int8, n, "codes")
        _need(s, torch.float32, nb, "scales")
    mk = lambda ts: (_vp * max(count, 1))(*[t.data_ptr() for t in ts])
    _check(load().equarx_quantize_batch(mk(xs), mk(codes_list), mk(scales_list), count, n, block, _stream()),
           "equarx_quantize_batch")


def equarx_dequantize(codes: torch.Tensor, scales: torch.Tensor, block: int, out_bf16: torch.Tensor) -> None:
    """out_bf16[n] <- bf16(codes * scales[block])."""
    status = _native.equarx_dequantize(codes, scales, block, out_bf16)
    if status >= 0:
        return _check(status, "equarx_dequantize")
    n = codes.numel()
    _need(codes, torch.int8, n, "codes")
    _need(scales, torch.float32, num_blocks(n, block), "scales")
    _need(out_bf16, torch.bfloat16, n, "out_bf16")
    _check(load().equarx_dequantize(_ptr(codes), _ptr(scales), codes.numel(), block, _ptr(out_bf16), _stream()),
           "equarx_dequantize")


def equarx_reduce_stage(codes_in, scales_in, local_bf16, block: int, codes_out, scales_out) -> None:
    """One hop: (codes_out, scales_out) <- Q_B(fma(codes_in, scales_in, local_bf16))."""
    status = _native.equarx_reduce_stage(codes_in, scales_in, local_bf16, block, codes_out, scales_out)
    if status >= 0:
        return _check(status, "equarx_reduce_stage")
    n = local_bf16.numel()
    nb = num_blocks(n, block)
    _need(local_bf16, torch.bfloat16, n, "local_bf16")
    _need(codes_in, torch.int8, n, "codes_in")
    _need(codes_out, torch.int8, n, "codes_out")
    _need(scales_in, torch.float32, nb, "scales_in")
    _need(scales_out, torch.float32, nb, "scales_out")
    _check(load().equarx_reduce_stage(_ptr(codes_in), _ptr(scales_in), _ptr(local_bf16), local_bf16.numel(), block,
                                      _ptr(codes_out), _ptr(scales_out), _stream()), "equarx_reduce_stage")


def equarx_reduce_quantized(partials, block: int, out_bf16, workspace=None, wire_codes=None, wire_scales=None) -> None:
    """The whole chain over the partials (sequence of bf16 tensors of equal length, chain order)."""
    status = _native.equarx_reduce_quantized(partials, block, out_bf16, workspace, wire_codes, wire_scales)
    if status >= 0:
        return _check(status, "equarx_reduce_quantized")
    P = len(partials)
    n = partials[0].numel() if P else 0
    for p in partials:
        _need(p, torch.bfloat16, n, "partial")
        if p.numel() != n:
            raise ValueError("partials differ in length")
    _need(out_bf16, torch.bfloat16, n, "out_bf16")
    if wire_codes is not None or wire_scales is not None:
        _need(wire_codes, torch.int8, P * wire_row_codes(n), "wire_codes")
        _need(wire_scales, torch.float32, P * wire_row_scales(n, block) if block in BLOCK_SIZES else 0, "wire_scales")
    if workspace is not None and not (workspace.is_cuda and workspace.is_contiguous()):
        raise ValueError("workspace: need a contiguous CUDA tensor")
    table = (_vp * max(P, 1))(*[p.data_ptr() for p in partials])
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load().equarx_reduce_quantized(table, P, n, block, _ptr(out_bf16), _ptr(workspace), ws_bytes,
                                          _ptr(wire_codes), _ptr(wire_scales), _stream()), "equarx_reduce_quantized")


STATIC_WORKSPACE_BYTES = 80 << 20


def equarx_reduce_quantized_static(partials, block: int, out_bf16) -> None:
    """equarx_reduce_quantized with the wire buffers in the library's static device array (allocates nothing)."""
    status = _native.equarx_reduce_quantized_static(partials, block, out_bf16)
    if status >= 0:
        return _check(status, "equarx_reduce_quantized_static")
    P = len(partials)
    n = partials[0].numel() if P else 0
    for p in partials:
        _need(p, torch.bfloat16, n, "partial")
        if p.numel() != n:
            raise ValueError("partials differ in length")
    _need(out_bf16, torch.bfloat16, n, "out_bf16")
    table = (_vp * max(P, 1))(*[p.data_ptr() for p in partials])
    _check(load().equarx_reduce_quantized_static(table, P, n, block, _ptr(out_bf16), _stream()),
           "equarx_reduce_quantized_static")


def equarx_reduce_quantized_fused_ends(partials, block: int, out_bf16, workspace=None) -> None:
    """The hop-by-hop chain with its first two and last two passes fused (P-1 launches, same bits)."""
    status = _native.equarx_reduce_quantized_fused_ends(partials, block, out_bf16, workspace)
    if status >= 0:
        return _check(status, "equarx_reduce_quantized_fused_ends")
    P = len(partials)
    n = partials[0].numel() if P else 0
    for p in partials:
        _need(p, torch.bfloat16, n, "partial")
        if p.numel() != n:
            raise ValueError("partials differ in length")
    _need(out_bf16, torch.bfloat16, n, "out_bf16")
    if workspace is not None and not (workspace.is_cuda and workspace.is_contiguous()):
        raise ValueError("workspace: need a contiguous CUDA tensor")
    table = (_vp * max(P, 1))(*[p.data_ptr() for p in partials])
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load().equarx_reduce_quantized_fused_ends(table, P, n, block, _ptr(out_bf16), _ptr(workspace), ws_bytes,
                                                     _stream()), "equarx_reduce_quantized_fused_ends")


def equarx_reduce_fused(partials, block: int, out_bf16, wire_codes=None, wire_scales=None) -> None:
    """The whole chain in one launch (same bits as equarx_reduce_quantized, no workspace)."""
    status = _native.equarx_reduce_fused(partials, block, out_bf16, wire_codes, wire_scales)
    if status >= 0:
        return _check(status, "equarx_reduce_fused")
    P = len(partials)
    n = partials[0].numel() if P else 0
    for p in partials:
        _need(p, torch.bfloat16, n, "partial")
        if p.numel() != n:
            raise ValueError("partials differ in length")
    _need(out_bf16, torch.bfloat16, n, "out_bf16")
    if wire_codes is not None or wire_scales is not None:
        _need(wire_codes, torch.int8, P * wire_row_codes(n), "wire_codes")
        _need(wire_scales, torch.float32, P * wire_row_scales(n, block) if block in BLOCK_SIZES else 0, "wire_scales")
    table = (_vp * max(P, 1))(*[p.data_ptr() for p in partials])
    _check(load().equarx_reduce_fused(table, P, n, block, _ptr(out_bf16), _ptr(wire_codes), _ptr(wire_scales),
                                      _stream()), "equarx_reduce_fused")


def equarx_reduce_variant(partials, block: int, flags: int, out_bf16) -> None:
    """A variant of the chain in one launch; flags: SEMI_LOOP | RS_UNQUANTIZED | AG_UNQUANTIZED | RING_ORDER."""
    status = _native.equarx_reduce_variant(partials, block, flags, out_bf16)
    if status >= 0:
        return _check(status, "equarx_reduce_variant")
    P = len(partials)
    n = partials[0].numel() if P else 0
    for p in partials:
        _need(p, torch.bfloat16, n, "partial")
        if p.numel() != n:
            raise ValueError("partials differ in length")
    _need(out_bf16, torch.bfloat16, n, "out_bf16")
    table = (_vp * max(P, 1))(*[p.data_ptr() for p in partials])
    _check(load().equarx_reduce_variant(table, P, n, block, flags, _ptr(out_bf16), _stream()), "equarx_reduce_variant")


def alloc_variant_workspace(flags: int, P: int, n: int, block: int) -> torch.Tensor:
    nbytes = int(load().equarx_variant_workspace_bytes(flags, P, n, block))
    return torch.empty(max(nbytes, 1), dtype=torch.uint8, device="cuda")


def equarx_reduce_variant_hops(partials, block: int, flags: int, out_bf16, workspace) -> None:
    """equarx_reduce_variant's full-loop / semi-loop forms hop by hop (one launch per hop, same bits)."""
    status = _native.equarx_reduce_variant_hops(partials, block, flags, out_bf16, workspace)
    if status >= 0:
        return _check(status, "equarx_reduce_variant_hops")
    P = len(partials)
    n = partials[0].numel() if P else 0
    for p in partials:
        _need(p, torch.bfloat16, n, "partial")
        if p.numel() != n:
            raise ValueError("partials differ in length")
    _need(out_bf16, torch.bfloat16, n, "out_bf16")
    if workspace is not None and not (workspace.is_cuda and workspace.is_contiguous()):
        raise ValueError("workspace: need a contiguous CUDA tensor")
    table = (_vp * max(P, 1))(*[p.data_ptr() for p in partials])
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load().equarx_reduce_variant_hops(table, P, n, block, flags, _ptr(out_bf16), _ptr(workspace), ws_bytes,
                                             _stream()), "equarx_reduce_variant_hops")


def equarx_reduce_flat(local_bf16, codes_list, scales_list, block: int, out_bf16=None, codes_out=None,
                       scales_out=None) -> None:
    """Flat one-shot reduce of a local bf16 shard and R received (codes, scales) pairs."""
    status = _native.equarx_reduce_flat(local_bf16, codes_list, scales_list, block, out_bf16, codes_out, scales_out)
    if status >= 0:
        return _check(status, "equarx_reduce_flat")
    n = local_bf16.numel()
    nb = num_blocks(n, block)
    R = len(codes_list)
    if len(scales_list) != R:
        raise ValueError("codes and scales lists differ in length")
    _need(local_bf16, torch.bfloat16, n, "local_bf16")
    for c, s in zip(codes_list, scales_list):
        _need(c, torch.int8, n, "codes")
        _need(s, torch.float32, nb, "scales")
    if out_bf16 is not None:
        _need(out_bf16, torch.bfloat16, n, "out_bf16")
    if codes_out is not None or scales_out is not None:
        _need(codes_out, torch.int8, n, "codes_out")
        _need(scales_out, torch.float32, nb, "scales_out")
    ctab = (_vp * max(R, 1))(*[c.data_ptr() for c in codes_list])
    stab = (_vp * max(R, 1))(*[s.data_ptr() for s in scales_list])
    _check(load().equarx_reduce_flat(_ptr(local_bf16), ctab, stab, R, n, block, _ptr(out_bf16), _ptr(codes_out),
                                     _ptr(scales_out), _stream()), "equarx_reduce_flat")


STRIDED_CHUNKS = (32, 64, 128)


def _strided_scales(n: int, chunks: int) -> int:
    return n // chunks if chunks in STRIDED_CHUNKS else 0


def equarx_quantize_strided(x_bf16, chunks: int, codes, scales) -> None:
    """Q with the strided block geometry: scale m*1024+j covers position j of every chunk of minishard m."""
    status = _native.equarx_quantize_strided(x_bf16, chunks, codes, scales)
    if status >= 0:
        return _check(status, "equarx_quantize_strided")
    n = x_bf16.numel()
    _need(x_bf16, torch.bfloat16, n, "x_bf16")
    _need(codes, torch.int8, n, "codes")
    _need(scales, torch.float32, _strided_scales(n, chunks), "scales")
    _check(load().equarx_quantize_strided(_ptr(x_bf16), n, chunks, _ptr(codes), _ptr(scales), _stream()),
           "equarx_quantize_strided")


def equarx_dequantize_strided(codes, scales, chunks: int, out_bf16) -> None:
    status = _native.equarx_dequantize_strided(codes, scales, chunks, out_bf16)
    if status >= 0:
        return _check(status, "equarx_dequantize_strided")
    n = codes.numel()
    _need(codes, torch.int8, n, "codes")
    _need(scales, torch.float32, _strided_scales(n, chunks), "scales")
    _need(out_bf16, torch.bfloat16, n, "out_bf16")
    _check(load().equarx_dequantize_strided(_ptr(codes), _ptr(scales), n, chunks, _ptr(out_bf16), _stream()),
           "equarx_dequantize_strided")


def equarx_reduce_stage_strided(codes_in, scales_in, local_bf16, chunks: int, codes_out, scales_out) -> None:
    status = _native.equarx_reduce_stage_strided(codes_in, scales_in, local_bf16, chunks, codes_out, scales_out)
    if status >= 0:
        return _check(status, "equarx_reduce_stage_strided")
    n = local_bf16.numel()
    ns = _strided_scales(n, chunks)
    _need(local_bf16, torch.bfloat16, n, "local_bf16")
    _need(codes_in, torch.int8, n, "codes_in")
    _need(codes_out, torch.int8, n, "codes_out")
    _need(scales_in, torch.float32, ns, "scales_in")
    _need(scales_out, torch.float32, ns, "scales_out")
    _check(load().equarx_reduce_stage_strided(_ptr(codes_in), _ptr(scales_in), _ptr(local_bf16), n, chunks,
                                              _ptr(codes_out), _ptr(scales_out), _stream()), "equarx_reduce_stage_strided")


def equarx_reduce_quantized_strided(partials, chunks: int, out_bf16, workspace) -> None:
    status = _native.equarx_reduce_quantized_strided(partials, chunks, out_bf16, workspace)
    if status >= 0:
        return _check(status, "equarx_reduce_quantized_strided")
    P = len(partials)
    n = partials[0].numel() if P else 0
    for p in partials:
        _need(p, torch.bfloat16, n, "partial")
        if p.numel() != n:
            raise ValueError("partials differ in length")
    _need(out_bf16, torch.bfloat16, n, "out_bf16")
    if workspace is not None and not (workspace.is_cuda and workspace.is_contiguous()):
        raise ValueError("workspace: need a contiguous CUDA tensor")
    table = (_vp * max(P, 1))(*[p.data_ptr() for p in partials])
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load().equarx_reduce_quantized_strided(table, P, n, chunks, _ptr(out_bf16), _ptr(workspace), ws_bytes,
                                                  _stream()), "equarx_reduce_quantized_strided")


def equarx_reduce_fused_strided(partials, chunks: int, out_bf16) -> None:
    """The strided chain in one launch (same bits as equarx_reduce_quantized_strided)."""
    status = _native.equarx_reduce_fused_strided(partials, chunks, out_bf16)
    if status >= 0:
        return _check(status, "equarx_reduce_fused_strided")
    P = len(partials)
    n = partials[0].numel() if P else 0
    for p in partials:
        _need(p, torch.bfloat16, n, "partial")
        if p.numel() != n:
            raise ValueError("partials differ in length")
    _need(out_bf16, torch.bfloat16, n, "out_bf16")
    table = (_vp * max(P, 1))(*[p.data_ptr() for p in partials])
    _check(load().equarx_reduce_fused_strided(table, P, n, chunks, _ptr(out_bf16), _stream()),
           "equarx_reduce_fused_strided")


def equarx_reduce_variant_strided(partials, chunks: int, flags: int, out_bf16) -> None:
    """Semi-loop / stage-knob flavours of the chain in the strided geometry, one launch."""
    status = _native.equarx_reduce_variant_strided(partials, chunks, flags, out_bf16)
    if status >= 0:
        return _check(status, "equarx_reduce_variant_strided")
    P = len(partials)
    n = partials[0].numel() if P else 0
    for p in partials:
        _need(p, torch.bfloat16, n, "partial")
        if p.numel() != n:
            raise ValueError("partials differ in length")
    _need(out_bf16, torch.bfloat16, n, "out_bf16")
    table = (_vp * max(P, 1))(*[p.data_ptr() for p in partials])
    _check(load().equarx_reduce_variant_strided(table, P, n, chunks, flags, _ptr(out_bf16), _stream()),
           "equarx_reduce_variant_strided")


def equarx_reduce_variant_hops_strided(partials, chunks: int, flags: int, out_bf16, workspace) -> None:
    """Full loop or semi-loop, all-gather quantized or not, hop by hop in the strided geometry."""
    status = _native.equarx_reduce_variant_hops_strided(partials, chunks, flags, out_bf16, workspace)
    if status >= 0:
        return _check(status, "equarx_reduce_variant_hops_strided")
    P = len(partials)
    n = partials[0].numel() if P else 0
    for p in partials:
        _need(p, torch.bfloat16, n, "partial")
        if p.numel() != n:
            raise ValueError("partials differ in length")
    _need(out_bf16, torch.bfloat16, n, "out_bf16")
    if not (workspace.is_cuda and workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous CUDA tensor")
    table = (_vp * max(P, 1))(*[p.data_ptr() for p in partials])
    _check(load().equarx_reduce_variant_hops_strided(table, P, n, chunks, flags, _ptr(out_bf16), _ptr(workspace),
                                                     workspace.numel() * workspace.element_size(), _stream()),
           "equarx_reduce_variant_hops_strided")


def mx4_row_blocks(cols: int) -> int:
    return int(load().equarx_mx4_row_blocks(cols))


def alloc_mx4(rows: int, cols: int, device="cuda"):
    """Buffers for the packed form of [rows, cols]: codes uint8 [rows, 16 * blocks], scales uint8 [rows, blocks]."""
    blocks = mx4_row_blocks(cols)
    return (torch.empty((rows, 16 * blocks), dtype=torch.uint8, device=device),
            torch.empty((rows, blocks), dtype=torch.uint8, device=device))


def alloc_mx4_workspace(M: int, N: int, K: int, device="cuda") -> torch.Tensor:
    """What equarx_mx4_linear and equarx_mx4_product need beside their operands."""
    return torch.empty(max(int(load().equarx_mx4_workspace_bytes(M, N, K)), 256), dtype=torch.uint8, device=device)


def _need_rows(t, dims: int, what: str):
    """A bf16 CUDA tensor of `dims` dimensions, the last one contiguous, and the strides of the others."""
    if t is None or not t.is_cuda or t.dtype != torch.bfloat16 or t.dim() != dims or (t.shape[-1] > 1 and t.stride(-1) != 1):
        raise ValueError(f"{what}: need a CUDA torch.bfloat16 tensor of {dims} dimensions, the last one contiguous")
    cols = t.shape[-1]
    head = t.stride(1) if dims == 3 and t.shape[1] > 1 else cols
    row = t.stride(0) if t.shape[0] > 1 else t.shape[1] * cols if dims == 3 else cols
    return row, head


def _need_packed(codes, scales, rows: int, cols: int, what: str) -> None:
    blocks = mx4_row_blocks(cols)
    for t, width in ((codes, 16 * blocks), (scales, blocks)):
        if t is None or not t.is_cuda or t.dtype != torch.uint8 or not t.is_contiguous() or tuple(t.shape) != (rows, width):
            raise ValueError(f"{what}: need contiguous CUDA torch.uint8 codes [{rows}, {16 * blocks}] and scales [{rows}, {blocks}]")


def _need_workspace(workspace) -> int:
    if workspace is None:
        return 0
    if not (workspace.is_cuda and workspace.is_contiguous()):
        raise ValueError("workspace: need a contiguous CUDA tensor")
    return workspace.numel() * workspace.element_size()


def equarx_mx4_quantize(x, codes, scales) -> None:
    """codes, scales <- the 4-bit microscaled form of bf16 x [rows, cols] (any row stride)."""
    status = _native.equarx_mx4_quantize(x, codes, scales)
    if status >= 0:
        return _check(status, "equarx_mx4_quantize")
    stride, _ = _need_rows(x, 2, "x_bf16")
    rows, cols = x.shape
    _need_packed(codes, scales, rows, cols, "packed x")
    _check(load().equarx_mx4_quantize(_ptr(x), rows, cols, stride, _ptr(codes), _ptr(scales), _stream()), "equarx_mx4_quantize")


def equarx_mx4_dequantize(codes, scales, out_bf16) -> None:
    """out_bf16 [rows, cols] (any row stride) <- the values that packed rows stand for."""
    status = _native.equarx_mx4_dequantize(codes, scales, out_bf16)
    if status >= 0:
        return _check(status, "equarx_mx4_dequantize")
    stride, _ = _need_rows(out_bf16, 2, "out_bf16")
    rows, cols = out_bf16.shape
    _need_packed(codes, scales, rows, cols, "packed rows")
    _check(load().equarx_mx4_dequantize(_ptr(codes), _ptr(scales), rows, cols, _ptr(out_bf16), stride, _stream()),
           "equarx_mx4_dequantize")


def equarx_mx4_product(x_codes, x_scales, w_codes, w_scales, K: int, out_bf16, workspace=None) -> None:
    """out_bf16 [M, N] <- x [M, K] w [N, K]^T, both packed."""
    status = _native.equarx_mx4_product(x_codes, x_scales, w_codes, w_scales, K, out_bf16, workspace)
    if status >= 0:
        return _check(status, "equarx_mx4_product")
    stride, _ = _need_rows(out_bf16, 2, "out_bf16")
    M, N = out_bf16.shape
    if not isinstance(K, int) or K < 0:
        raise ValueError("K: need an int that is not negative")
    _need_packed(x_codes, x_scales, M, K, "packed x")
    _need_packed(w_codes, w_scales, N, K, "packed w")
    nbytes = _need_workspace(workspace)
    _check(load().equarx_mx4_product(_ptr(x_codes), _ptr(x_scales), _ptr(w_codes), _ptr(w_scales), M, N, K, _ptr(out_bf16),
                                     stride, _ptr(workspace), nbytes, _stream()), "equarx_mx4_product")


def equarx_mx4_linear(x, w_codes, w_scales, out_bf16, workspace=None) -> None:
    """out_bf16 [M, N] <- x [M, K] w [N, K]^T with x bf16, quantized in the call: a row-parallel layer's partial sum."""
    status = _native.equarx_mx4_linear(x, w_codes, w_scales, out_bf16, workspace)
    if status >= 0:
        return _check(status, "equarx_mx4_linear")
    x_stride, _ = _need_rows(x, 2, "x_bf16")
    out_stride, _ = _need_rows(out_bf16, 2, "out_bf16")
    (M, K), N = x.shape, out_bf16.shape[1]
    if out_bf16.shape[0] != M:
        raise ValueError("x_bf16 and out_bf16 differ in rows")
    _need_packed(w_codes, w_scales, N, K, "packed w")
    nbytes = _need_workspace(workspace)
    _check(load().equarx_mx4_linear(_ptr(x), x_stride, _ptr(w_codes), _ptr(w_scales), M, N, K, _ptr(out_bf16), out_stride,
                                    _ptr(workspace), nbytes, _stream()), "equarx_mx4_linear")


class Cache(NamedTuple):
    """The buffers of a key/value cache: k_codes int8 [pages, heads, page, dim], k_scales fp32 [pages, heads, dim / block,
    page], v_codes int8 [pages, heads, page / 16, dim, 16], v_scales as k_scales."""
    k_codes: torch.Tensor
    k_scales: torch.Tensor
    v_codes: torch.Tensor
    v_scales: torch.Tensor


def alloc_cache(pages: int, heads: int, page: int, dim: int, block: int, device="cuda") -> Cache:
    """A cache that holds zeros."""
    zeros = lambda *shape, dtype: torch.zeros(shape, dtype=dtype, device=device)
    return Cache(zeros(pages, heads, page, dim, dtype=torch.int8), zeros(pages, heads, dim // block, page, dtype=torch.float32),
                 zeros(pages, heads, page // 16, dim, 16, dtype=torch.int8),
                 zeros(pages, heads, dim // block, page, dtype=torch.float32))


def _need_cache(cache):
    """The C structure of a Cache whose tensors have the shapes they should have."""
    if not isinstance(cache, (tuple, list)) or len(cache) != 4 or not all(isinstance(t, torch.Tensor) for t in cache):
        raise ValueError("cache: need the four tensors of a Cache")
    kc, ks, vc, vs = cache
    good = kc.dim() == 4 and ks.dim() == 4 and ks.shape[2] > 0 and kc.shape[3] % ks.shape[2] == 0
    if good:
        pages, heads, page, dim = kc.shape
        scales = (pages, heads, ks.shape[2], page)
        good = (tuple(ks.shape) == scales and tuple(vs.shape) == scales and page % 16 == 0
                and tuple(vc.shape) == (pages, heads, page // 16, dim, 16) and kc.numel() > 0)
    good = good and all(t.is_cuda and t.is_contiguous() and t.dtype == (torch.float32 if i % 2 else torch.int8)
                        for i, t in enumerate(cache))
    if not good:
        raise ValueError("cache: need contiguous CUDA tensors of the shapes and types that alloc_cache makes")
    return _CCache(_ptr(kc), _ptr(ks), _ptr(vc), _ptr(vs), pages, heads, page, dim, dim // ks.shape[2])


def _need_sequences(page_table, lengths) -> None:
    for t, what, dims in ((page_table, "page_table", 2), (lengths, "lengths", 1)):
        if t is None or not t.is_cuda or t.dtype != torch.int32 or not t.is_contiguous() or t.dim() != dims:
            raise ValueError(f"{what}: need a contiguous CUDA torch.int32 tensor of {dims} dimensions")
    if lengths.numel() != page_table.shape[0]:
        raise ValueError("page_table and lengths differ in sequences")


def equarx_cache_write(cache: Cache, k, v, slots) -> None:
    """Quantize k, v bf16 [tokens, heads, dim] (strided views welcome) into the slots int64 [tokens] of a cache."""
    status = _native.equarx_cache_write(cache, k, v, slots)
    if status >= 0:
        return _check(status, "equarx_cache_write")
    c = _need_cache(cache)
    strides = []
    for t, what in ((k, "k_bf16"), (v, "v_bf16")):
        strides.append(_need_rows(t, 3, what))
        if t.shape[0] != k.shape[0] or tuple(t.shape[1:]) != (c.heads, c.dim):
            raise ValueError(f"{what}: need [tokens, {c.heads}, {c.dim}]")
    _need(slots, torch.int64, k.shape[0], "slots")
    if slots.numel() != k.shape[0]:
        raise ValueError("one slot for every token")
    _check(load().equarx_cache_write(ctypes.byref(c), _ptr(k), *strides[0], _ptr(v), *strides[1], k.shape[0], _ptr(slots),
                                     _stream()), "equarx_cache_write")


def equarx_cache_read(cache: Cache, page_table, lengths, starts, k_out, v_out, max_length=None) -> None:
    """Sequences back as bf16: token t of sequence b to row starts[b] + t of k_out and v_out [rows, heads, dim]."""
    if max_length is None:
        try:
            max_length = page_table.shape[-1] * cache[0].shape[2]           # what the table can hold
        except (AttributeError, TypeError, IndexError):
            max_length = 0                                                  # no table or no cache: refused below
    status = _native.equarx_cache_read(cache, page_table, lengths, starts, k_out, v_out, max_length)
    if status >= 0:
        return _check(status, "equarx_cache_read")
    c = _need_cache(cache)
    _need_sequences(page_table, lengths)
    sequences, width = page_table.shape
    _need(starts, torch.int32, sequences, "starts")
    for t, what in ((k_out, "k_out"), (v_out, "v_out")):
        if (t is None or not t.is_cuda or t.dtype != torch.bfloat16 or not t.is_contiguous() or t.dim() != 3
                or tuple(t.shape) != (k_out.shape[0], c.heads, c.dim)):
            raise ValueError(f"{what}: need a contiguous CUDA torch.bfloat16 tensor [rows, {c.heads}, {c.dim}]")
    _check(load().equarx_cache_read(ctypes.byref(c), _ptr(page_table), width, _ptr(lengths), _ptr(starts), sequences, max_length,
                                    k_out.shape[0], _ptr(k_out), _ptr(v_out), _stream()), "equarx_cache_read")


def alloc_cache_attention_workspace(cache: Cache, q_rows: int, q_heads: int, sequences: int, max_queries, max_length: int,
                                    device="cuda") -> torch.Tensor:
    """For calls of these sizes; with max_queries None for all calls of up to so many rows, sequences and tokens, whose max_queries
    is at least their rows per sequence (a call of fewer sequences may need more than one of all)."""
    heads, dim = cache[0].shape[1], cache[0].shape[3]
    if max_queries is None:
        nbytes = load().equarx_cache_attention_most_workspace_bytes(heads, dim, q_rows, q_heads, sequences, max_length)
    else:
        nbytes = load().equarx_cache_attention_workspace_bytes(heads, dim, q_rows, q_heads, sequences, max_queries, max_length)
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def equarx_cache_attention(cache: Cache, q, q_starts, page_table, lengths, out, scale: float, max_queries: int, max_length: int,
                           causal: bool = True, window: int = 0, lse=None, workspace=None) -> None:
    """out [q_rows, q_heads, dim] <- softmax attention of q [q_rows, q_heads, dim] over cached sequences; sequence b has the
    query rows q_starts[b] .. q_starts[b + 1] - 1, the last of which stands at its last token."""
    status = _native.equarx_cache_attention(cache, q, q_starts, page_table, lengths, out, scale, max_queries, max_length, causal,
                                            window, lse, workspace)
    if status >= 0:
        return _check(status, "equarx_cache_attention")
    c = _need_cache(cache)
    row, head = _need_rows(q, 3, "q_bf16")
    q_rows, q_heads, dim = q.shape
    if dim != c.dim:
        raise ValueError(f"q_bf16: need heads of {c.dim} elements")
    _need_sequences(page_table, lengths)
    sequences, width = page_table.shape
    _need(q_starts, torch.int32, sequences + 1, "q_starts")
    if q_starts.numel() != sequences + 1:
        raise ValueError("q_starts: need one entry more than there are sequences")
    if out is None or not out.is_cuda or out.dtype != torch.bfloat16 or not out.is_contiguous() or out.shape != q.shape:
        raise ValueError("out: need a contiguous CUDA torch.bfloat16 tensor of q's shape")
    if lse is not None:
        _need(lse, torch.float32, q_rows * q_heads, "lse")
        if lse.numel() != q_rows * q_heads:
            raise ValueError("lse: need one entry for every row and head of q")
    nbytes = _need_workspace(workspace)
    _check(load().equarx_cache_attention(ctypes.byref(c), _ptr(q), q_rows, q_heads, row, head, _ptr(q_starts), _ptr(page_table),
                                         width, _ptr(lengths), sequences, float(scale), max_queries, max_length,
                                         1 if causal else 0, window, _ptr(out), _ptr(lse), _ptr(workspace), nbytes, _stream()),
           "equarx_cache_attention")


def equarx_calib_copy(src: torch.Tensor, dst: torch.Tensor) -> None:
    nbytes = src.numel() * src.element_size()
    if not (src.is_cuda and dst.is_cuda and src.is_contiguous() and dst.is_contiguous()
            and dst.numel() * dst.element_size() >= nbytes):
        raise ValueError("calib_copy: need contiguous CUDA tensors, dst at least as large as src")
    _check(load().equarx_calib_copy(_ptr(src), _ptr(dst), nbytes, _stream()), "equarx_calib_copy")


def equarx_calib_empty_launches(count: int, workgroups: int) -> None:
    """`count` back-to-back launches of a kernel that does nothing (`workgroups` workgroups each)."""
    _check(load().equarx_calib_empty_launches(count, workgroups, _stream()), "equarx_calib_empty_launches")


def equarx_calib_hop_traffic(partials, block: int, codes0, scales0, codes1, scales1) -> None:
    """The chain's P-1 hops as memory traffic only (XOR of what each launch read), ping-pong between two wires, or, if
    wire 1 is wire 0, rewriting it in place in the chain's order of tiles."""
    P = len(partials)
    n = partials[0].numel() if P else 0
    nb = num_blocks(n, block) if block in BLOCK_SIZES else 0
    for p in partials:
        _need(p, torch.bfloat16, n, "partial")
    for c, s in ((codes0, scales0), (codes1, scales1)):
        _need(c, torch.int8, n, "codes")
        _need(s, torch.float32, nb, "scales")
    table = (_vp * max(P, 1))(*[p.data_ptr() for p in partials])
    _check(load().equarx_calib_hop_traffic(table, P, n, block, _ptr(codes0), _ptr(scales0), _ptr(codes1),
                                           _ptr(scales1), _stream()), "equarx_calib_hop_traffic")


def equarx_calib_interleaved_chains(partial_sets, block: int, outs, workspaces, streaming: bool = False) -> None:
    """len(partial_sets) independent hop-by-hop chains, interleaved pass by pass (every wire read M-1 launches after
    it was written); chain m reduces partial_sets[m] into outs[m] using workspaces[m].  streaming: the wire is
    accessed with non-temporal hints, as the per-step entry points access it."""
    M = len(partial_sets)
    P = len(partial_sets[0]) if M else 0
    n = partial_sets[0][0].numel() if P else 0
    if len(outs) != M or len(workspaces) != M or any(len(ps) != P for ps in partial_sets):
        raise ValueError("one output, one workspace and P partials per chain")
    need = workspace_bytes(P, n, block) if P else 0
    for ps, o, w in zip(partial_sets, outs, workspaces):
        for p in ps:
            _need(p, torch.bfloat16, n, "partial")
            if p.numel() != n:
                raise ValueError("partials differ in length")
        _need(o, torch.bfloat16, n, "out_bf16")
        _need(w, torch.uint8, need, "workspace")
    flat = [p.data_ptr() for ps in partial_sets for p in ps]
    ptab = (_vp * max(len(flat), 1))(*flat)
    otab = (_vp * max(M, 1))(*[o.data_ptr() for o in outs])
    wtab = (_vp * max(M, 1))(*[w.data_ptr() for w in workspaces])
    _check(load().equarx_calib_interleaved_chains(ptab, M, P, n, block, otab, wtab, need, int(bool(streaming)), _stream()),
           "equarx_calib_interleaved_chains")


def equarx_time_launch_span(first: int, last: int, start_event, stop_event) -> None:
    """Raw hipEvent_t handles recorded before launch `first` and after launch `last` (from 0) of this thread's
    next call."""
    load().equarx_time_launch_span(first, last, start_event, stop_event)


def equarx_time_next_launch(start_event, stop_event) -> None:
    """start/stop: raw hipEvent_t handles (ints); the first launch of this thread's next call records its begin and
    end there."""
    load().equarx_time_next_launch(start_event, stop_event)


def equarx_time_cancel() -> None:
    load().equarx_time_cancel()


def equarx_selftest_quotients(first_bits: int, count: int, mismatches: torch.Tensor) -> None:
    """mismatches: CUDA int64[2], zeroed by the caller; receives the counts of differing scales / reciprocals."""
    _need(mismatches, torch.int64, 2, "mismatches")
    _check(load().equarx_selftest_quotients(first_bits, count, _ptr(mismatches), _stream()), "equarx_selftest_quotients")


def equarx_selftest_rounding(first_bits: int, count: int, mismatches: torch.Tensor) -> None:
    """mismatches: CUDA int64[1], zeroed by the caller; receives the number of |p| patterns whose codes differ."""
    _need(mismatches, torch.int64, 1, "mismatches")
    _check(load().equarx_selftest_rounding(first_bits, count, _ptr(mismatches), _stream()), "equarx_selftest_rounding")


def equarx_eval_quotients(absmax: torch.Tensor, scale: torch.Tensor, inv: torch.Tensor) -> None:
    n = absmax.numel()
    _need(absmax, torch.float32, n, "absmax")
    _need(scale, torch.float32, n, "scale")
    _need(inv, torch.float32, n, "inv")
    _check(load().equarx_eval_quotients(_ptr(absmax), n, _ptr(scale), _ptr(inv), _stream()), "equarx_eval_quotients")


def alloc_workspace(P: int, n: int, block: int, device="cuda") -> torch.Tensor:
    """Device buffer of the size the chain needs (torch is the allocator; the library never allocates)."""
    return torch.empty(max(workspace_bytes(P, n, block), 256), dtype=torch.uint8, device=device)
