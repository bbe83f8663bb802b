"""Thin ctypes binding of ``libloza_ssa.so``: argument marshalling only.

Every function has the name and the argument order of its C entry point (``include/loza_ssa.h``).
Tensors are torch tensors that already live on the GPU; nothing is computed here and there is no
fallback: if the shared library is missing, importing a symbol from it raises.
"""
from __future__ import annotations

import ctypes
import functools
import math
import os
from pathlib import Path

import torch

_PKG = Path(__file__).resolve().parent
# LOZA_SSA_LIB names another build of the same library (kernel experiments); default: the in-tree one
LIB_PATH = Path(os.environ["LOZA_SSA_LIB"]) if os.environ.get("LOZA_SSA_LIB") else _PKG / "libloza_ssa.so"
_lib = None

LOZA_OK = 0
LOZA_WINDOW_INF = (1 << 63) - 1

EXPORTS = (
    "loza_ssa_prefill", "loza_ssa_prefill_f32", "loza_ssa_decode",
    "loza_ssa_decode_workspace_bytes", "loza_ssa_decode_num_splits",
    "loza_ssa_live_ranges", "loza_ssa_live_pairs", "loza_status_str",
    "loza_ssa_prefill_blocks", "loza_ssa_prefill_blocks_f32", "loza_ssa_decode_blocks",
    "loza_ssa_live_ranges_blocks", "loza_ssa_live_pairs_blocks",
    "loza_ssa_decode_paged", "loza_ssa_decode_paged_blocks",
    "loza_ssa_prefill_calibration_blocks", "loza_ssa_calibration_workspace_bytes",
    "loza_ssa_extend", "loza_ssa_extend_blocks", "loza_ssa_extend_paged", "loza_ssa_extend_paged_blocks",
    "loza_ssa_extend_with_workspace", "loza_ssa_extend_workspace_bytes",
    "loza_ssa_backward", "loza_ssa_backward_blocks",
    "loza_ssa_backward_workspace_bytes", "loza_ssa_backward_workspace_bytes_blocks",
    "loza_ssa_backward_f32", "loza_ssa_backward_blocks_f32",
    "loza_ssa_decode_f32", "loza_ssa_decode_blocks_f32",
    "loza_ssa_calibration_alpha_grad", "loza_ssa_calibration_alpha_grad_workspace_bytes",
    "loza_ssa_decode_static",
    "loza_ssa_forward_kernel", "loza_ssa_decode_kernel", "loza_ssa_backward_split",
    "loza_ssa_step_tables", "loza_ssa_step_tables_held", "loza_ssa_rope", "loza_ssa_rope_f32", "loza_ssa_rope_append", "loza_ssa_rope_append_f32",
    "loza_ssa_rope_frequencies", "loza_ssa_extend_tree", "loza_ssa_extend_tree_workspace_bytes",
    "loza_ssa_extend_tree_kernel",
    "loza_ssa_verify_tree", "loza_ssa_verify_tree_workspace_bytes", "loza_ssa_keep_accepted",
)
KERNEL_TILES, KERNEL_ROWS, KERNEL_D128 = 1, 2, 3


class LozaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {loza_status_str(status)} ({status})")


def lib() -> ctypes.CDLL:
    """The loaded shared library (built beforehand by ``__graft_entry__.build()``)."""
    global _lib
    if _lib is None:
        if not LIB_PATH.exists():
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'`")
        L = ctypes.CDLL(str(LIB_PATH))
        vp, ci, i64, f32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
        f64 = ctypes.c_double
        L.loza_ssa_prefill.restype = ci
        L.loza_ssa_prefill.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, i64, ci, ci, i64, i64, f32, vp]
        L.loza_ssa_prefill_f32.restype = ci
        L.loza_ssa_prefill_f32.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, i64, ci, ci, i64, i64, f32, vp]
        L.loza_ssa_decode.restype = ci
        L.loza_ssa_decode.argtypes = [vp, vp, vp, vp, vp, vp, ci, ci, ci, i64, ci, ci, i64, i64, f32, vp, sz, vp]
        L.loza_ssa_decode_static.restype = ci
        L.loza_ssa_decode_static.argtypes = [vp, vp, vp, vp, vp, vp, ci, ci, ci, i64, ci, ci, i64, i64, f32, vp]
        L.loza_ssa_decode_workspace_bytes.restype = sz
        L.loza_ssa_decode_workspace_bytes.argtypes = [ci, ci, ci, i64, ci, i64, i64]
        L.loza_ssa_decode_num_splits.restype = ci
        L.loza_ssa_decode_num_splits.argtypes = [ci, ci, ci, i64, i64, i64]
        L.loza_ssa_live_ranges.restype = ci
        L.loza_ssa_live_ranges.argtypes = [i64, i64, i64, ctypes.POINTER(i64), ctypes.POINTER(i64), ctypes.POINTER(i64)]
        L.loza_ssa_live_pairs.restype = i64
        L.loza_ssa_live_pairs.argtypes = [i64, i64, i64]
        L.loza_ssa_prefill_blocks.restype = ci
        L.loza_ssa_prefill_blocks.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, i64, ci, ci, i64, i64, i64, f32, vp]
        L.loza_ssa_prefill_blocks_f32.restype = ci
        L.loza_ssa_prefill_blocks_f32.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, i64, ci, ci, i64, i64, i64, f32, vp]
        L.loza_ssa_decode_blocks.restype = ci
        L.loza_ssa_decode_blocks.argtypes = [vp, vp, vp, vp, vp, vp, ci, ci, ci, i64, ci, ci, i64, i64, i64, f32, vp, sz, vp]
        L.loza_ssa_live_ranges_blocks.restype = ci
        L.loza_ssa_live_ranges_blocks.argtypes = [i64, i64, i64, i64, ctypes.POINTER(i64), ctypes.POINTER(i64), ctypes.POINTER(i64)]
        L.loza_ssa_live_pairs_blocks.restype = i64
        L.loza_ssa_live_pairs_blocks.argtypes = [i64, i64, i64, i64]
        L.loza_ssa_decode_paged.restype = ci
        L.loza_ssa_decode_paged.argtypes = [vp, vp, vp, vp, vp, vp, vp, ci, ci, ci, i64, ci, ci, ci, ci, i64, i64, f32, vp, sz, vp]
        L.loza_ssa_decode_paged_blocks.restype = ci
        L.loza_ssa_decode_paged_blocks.argtypes = [vp, vp, vp, vp, vp, vp, vp, ci, ci, ci, i64, ci, ci, ci, ci, i64, i64, i64, f32, vp, sz, vp]
        L.loza_ssa_prefill_calibration_blocks.restype = ci
        L.loza_ssa_prefill_calibration_blocks.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, ci, ci, ci, i64, ci, ci,
                                                          i64, i64, i64, f32, f32, vp, sz, vp]
        L.loza_ssa_calibration_workspace_bytes.restype = sz
        L.loza_ssa_calibration_workspace_bytes.argtypes = [ci, ci, i64, ci]
        L.loza_ssa_extend.restype = ci
        L.loza_ssa_extend.argtypes = [vp, vp, vp, vp, vp, vp, ci, ci, ci, i64, ci, ci, ci, i64, i64, f32, vp]
        L.loza_ssa_extend_blocks.restype = ci
        L.loza_ssa_extend_blocks.argtypes = [vp, vp, vp, vp, vp, vp, ci, ci, ci, i64, ci, ci, ci, i64, i64, i64, f32, vp]
        L.loza_ssa_extend_paged.restype = ci
        L.loza_ssa_extend_paged.argtypes = [vp, vp, vp, vp, vp, vp, vp, ci, ci, ci, i64, ci, ci, ci, ci, ci, i64, i64, f32, vp]
        L.loza_ssa_extend_paged_blocks.restype = ci
        L.loza_ssa_extend_paged_blocks.argtypes = [vp, vp, vp, vp, vp, vp, vp, ci, ci, ci, i64, ci, ci, ci, ci, ci, i64, i64, i64, f32, vp]
        L.loza_ssa_extend_with_workspace.restype = ci
        L.loza_ssa_extend_with_workspace.argtypes = [vp] * 7 + [ci, ci, ci, i64, i64, ci, ci, ci, ci, ci, i64, i64, i64, f32, vp, sz, vp]
        L.loza_ssa_extend_workspace_bytes.restype = sz
        L.loza_ssa_extend_workspace_bytes.argtypes = [ci, ci, ci, i64, ci, ci, ci, i64, i64, i64]
        L.loza_ssa_backward.restype = ci
        L.loza_ssa_backward.argtypes = [vp] * 9 + [ci, ci, ci, i64, ci, ci, i64, i64, f32, vp, sz, vp]
        L.loza_ssa_backward_blocks.restype = ci
        L.loza_ssa_backward_blocks.argtypes = [vp] * 9 + [ci, ci, ci, i64, ci, ci, i64, i64, i64, f32, vp, sz, vp]
        L.loza_ssa_calibration_alpha_grad.restype = ci
        L.loza_ssa_calibration_alpha_grad.argtypes = [vp, vp, vp, vp, i64, vp, sz, vp]
        L.loza_ssa_calibration_alpha_grad_workspace_bytes.restype = sz
        L.loza_ssa_calibration_alpha_grad_workspace_bytes.argtypes = [i64]
        L.loza_ssa_decode_f32.restype = ci
        L.loza_ssa_decode_f32.argtypes = [vp, vp, vp, vp, vp, vp, ci, ci, ci, i64, ci, ci, i64, i64, f32, vp]
        L.loza_ssa_decode_blocks_f32.restype = ci
        L.loza_ssa_decode_blocks_f32.argtypes = [vp, vp, vp, vp, vp, vp, ci, ci, ci, i64, ci, ci, i64, i64, i64, f32, vp]
        L.loza_ssa_backward_f32.restype = ci
        L.loza_ssa_backward_f32.argtypes = [vp] * 9 + [ci, ci, ci, i64, ci, ci, i64, i64, f32, vp]
        L.loza_ssa_backward_blocks_f32.restype = ci
        L.loza_ssa_backward_blocks_f32.argtypes = [vp] * 9 + [ci, ci, ci, i64, ci, ci, i64, i64, i64, f32, vp]
        L.loza_ssa_backward_workspace_bytes.restype = sz
        L.loza_ssa_backward_workspace_bytes.argtypes = [ci, ci, ci, i64, ci, ci, i64, i64, ci]
        L.loza_ssa_backward_workspace_bytes_blocks.restype = sz
        L.loza_ssa_backward_workspace_bytes_blocks.argtypes = [ci, ci, ci, i64, ci, ci, i64, i64, i64, ci]
        L.loza_ssa_forward_kernel.restype = ci
        L.loza_ssa_forward_kernel.argtypes = [ci, ci, ci, i64, i64, ci, i64, i64, i64]
        L.loza_ssa_decode_kernel.restype = ci
        L.loza_ssa_decode_kernel.argtypes = [ci, ci, ci, i64, ci, i64, i64, i64, ctypes.POINTER(ci)]
        L.loza_ssa_backward_split.restype = ci
        L.loza_ssa_backward_split.argtypes = [ci, ci, ci, i64, ci, ci, i64, i64, i64, ci, ctypes.POINTER(ci), ctypes.POINTER(i64)]
        L.loza_ssa_step_tables.restype = ci
        L.loza_ssa_step_tables.argtypes = [vp] * 6 + [ci, ci, i64, i64, ci, ci] + [vp] * 7
        L.loza_ssa_step_tables_held.restype = ci
        L.loza_ssa_step_tables_held.argtypes = [vp] * 7 + [ci, ci, i64, i64, ci, ci] + [vp] * 8
        for name in ("loza_ssa_rope", "loza_ssa_rope_f32"):
            getattr(L, name).restype = ci
            getattr(L, name).argtypes = [vp] * 4 + [i64, ci, ci] + [i64] * 4 + [ci] * 4 + [f32, vp]
        for name in ("loza_ssa_rope_append", "loza_ssa_rope_append_f32"):
            getattr(L, name).restype = ci
            getattr(L, name).argtypes = [vp] * 9 + [i64] + [ci] * 5 + [i64] * 9 + [ci] * 4 + [f32, vp]
        L.loza_ssa_rope_frequencies.restype = ci
        L.loza_ssa_rope_frequencies.argtypes = [ci, f64, f64, i64, f64, f64, ctypes.POINTER(f64), ctypes.POINTER(f32)]
        L.loza_ssa_extend_tree.restype = ci
        L.loza_ssa_extend_tree.argtypes = [vp] * 9 + [ci, ci, ci, i64, i64, ci, ci, ci, ci, ci, i64, i64, i64, f32, vp, sz, vp]
        L.loza_ssa_extend_tree_workspace_bytes.restype = sz
        L.loza_ssa_extend_tree_workspace_bytes.argtypes = [ci, ci, ci, i64, ci, ci, ci, i64, i64, i64]
        L.loza_ssa_extend_tree_kernel.restype = ci
        L.loza_ssa_extend_tree_kernel.argtypes = [ci, ci, ci, i64, ci, ci, i64, i64, i64, ci, ctypes.POINTER(ci)]
        L.loza_ssa_verify_tree.restype = ci
        L.loza_ssa_verify_tree.argtypes = [vp] * 10 + [ci, ci, ci, vp, sz, vp]
        L.loza_ssa_verify_tree_workspace_bytes.restype = sz
        L.loza_ssa_verify_tree_workspace_bytes.argtypes = [ci, ci, ci]
        L.loza_ssa_keep_accepted.restype = ci
        L.loza_ssa_keep_accepted.argtypes = [vp] * 5 + [ci, ci, ci, i64, i64, i64, vp]
        # (of the HIP runtime that the library is linked with)
        L.hipThreadExchangeStreamCaptureMode.restype = ci
        L.hipThreadExchangeStreamCaptureMode.argtypes = [ctypes.POINTER(ci)]
        L.loza_status_str.restype = ctypes.c_char_p
        L.loza_status_str.argtypes = [ci]
        _lib = L
    return _lib


def _win(window) -> int:
    return LOZA_WINDOW_INF if window is None else min(int(window), LOZA_WINDOW_INF)


def _dev_ptr(t: torch.Tensor, dtype, name: str) -> int:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a tensor on the GPU")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


_STREAM_LEGACY, _STREAM_PER_THREAD = 1, 2   # HIP's handles for the default stream and for each thread's own
_CAPTURE_MODE_RELAXED = 2                    # hipStreamCaptureModeRelaxed


def _stream(stream) -> int:
    if stream is None:
        # torch.cuda.current_stream().cuda_stream without the object around it (2.8 us of a 10 us call)
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def loza_status_str(status: int) -> str:
    return lib().loza_status_str(int(status)).decode()


def loza_ssa_live_ranges(i: int, n_sink: int, window):
    """(sink_end, win_begin, win_end): live(i) = [0, sink_end) U [win_begin, win_end). Host only."""
    a, b, c = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64()
    rc = lib().loza_ssa_live_ranges(int(i), int(n_sink), _win(window), ctypes.byref(a), ctypes.byref(b), ctypes.byref(c))
    if rc != LOZA_OK:
        raise LozaError(rc, "loza_ssa_live_ranges")
    return a.value, b.value, c.value


def loza_ssa_live_pairs(S: int, n_sink: int, window) -> int:
    return int(lib().loza_ssa_live_pairs(int(S), int(n_sink), _win(window)))


def _prefill_common(fn_name, dtype, q, k, v, out, lse, pattern, scale, stream):
    B, S, Hq, d_qk = q.shape
    Hkv = k.shape[2]
    d_v = out.shape[3]
    if k.shape != (B, S, Hkv, d_qk) or out.shape != (B, S, Hq, d_v) or lse.shape != (B, Hq, S):
        raise ValueError("shape mismatch between q, k, out, lse")
    if v is not k and v.shape != (B, S, Hkv, d_v):
        raise ValueError("v must be [B, S, Hkv, d_v] (or the very tensor passed as k)")
    qp, kp = _dev_ptr(q, dtype, "q"), _dev_ptr(k, dtype, "k")
    vp = kp if v is k else _dev_ptr(v, dtype, "v")
    rc = getattr(lib(), fn_name)(qp, kp, vp, _dev_ptr(out, dtype, "out"), _dev_ptr(lse, torch.float32, "lse"),
                                 B, Hq, Hkv, S, d_qk, d_v, *pattern, float(scale), _stream(stream))
    if rc != LOZA_OK:
        raise LozaError(rc, fn_name)


def loza_ssa_prefill(q, k, v, out, lse, n_sink, window, scale, stream=None):
    """bf16 SSA prefill. q [B,S,Hq,d_qk], k [B,S,Hkv,d_qk], v [B,S,Hkv,d_v] or ``v is k`` (absorbed
    MLA: values are the first d_v columns of k), out [B,S,Hq,d_v] bf16, lse [B,Hq,S] fp32.
    ``window=None`` means infinity (full causal attention)."""
    _prefill_common("loza_ssa_prefill", torch.bfloat16, q, k, v, out, lse, (int(n_sink), _win(window)), scale, stream)


def loza_ssa_prefill_f32(q, k, v, out, lse, n_sink, window, scale, stream=None):
    """fp32 twin of :func:`loza_ssa_prefill`."""
    _prefill_common("loza_ssa_prefill_f32", torch.float32, q, k, v, out, lse, (int(n_sink), _win(window)), scale, stream)


def loza_ssa_prefill_blocks(q, k, v, out, lse, sink_blocks, local_blocks, block, scale, stream=None):
    """bf16 SSA prefill under the block-granular pattern (sink blocks, local blocks, block size)."""
    _prefill_common("loza_ssa_prefill_blocks", torch.bfloat16, q, k, v, out, lse,
                    (int(sink_blocks), _win(local_blocks), int(block)), scale, stream)


def loza_ssa_prefill_blocks_f32(q, k, v, out, lse, sink_blocks, local_blocks, block, scale, stream=None):
    """fp32 twin of :func:`loza_ssa_prefill_blocks`."""
    _prefill_common("loza_ssa_prefill_blocks_f32", torch.float32, q, k, v, out, lse,
                    (int(sink_blocks), _win(local_blocks), int(block)), scale, stream)


def loza_ssa_live_ranges_blocks(i: int, sink_blocks: int, local_blocks, block: int):
    """(sink_end, win_begin, win_end) of query i under the block-granular pattern. Host only."""
    a, b, c = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64()
    rc = lib().loza_ssa_live_ranges_blocks(int(i), int(sink_blocks), _win(local_blocks), int(block),
                                           ctypes.byref(a), ctypes.byref(b), ctypes.byref(c))
    if rc != LOZA_OK:
        raise LozaError(rc, "loza_ssa_live_ranges_blocks")
    return a.value, b.value, c.value


def loza_ssa_live_pairs_blocks(S: int, sink_blocks: int, local_blocks, block: int) -> int:
    return int(lib().loza_ssa_live_pairs_blocks(int(S), int(sink_blocks), _win(local_blocks), int(block)))


def loza_ssa_decode_num_splits(B, Hq, Hkv, S_max, n_sink, window) -> int:
    return int(lib().loza_ssa_decode_num_splits(B, Hq, Hkv, int(S_max), int(n_sink), _win(window)))


def _checked(value: int, where: str) -> int:
    if value < 0:
        raise LozaError(value, where)
    return value


def loza_ssa_forward_kernel(B, Hq, Hkv, n_queries, S, d_qk, sink, local, block=1) -> int:
    """Which kernel (KERNEL_...) a bf16 prefill or extend of these sizes runs. Host only, like the two below."""
    return _checked(lib().loza_ssa_forward_kernel(B, Hq, Hkv, int(n_queries), int(S), d_qk, int(sink), _win(local), int(block)),
                    "loza_ssa_forward_kernel")


def loza_ssa_decode_kernel(B, Hq, Hkv, S_max, d_qk, sink, local, block=1):
    """(kernel, key splits) of a bf16 decode."""
    n = ctypes.c_int()
    k = lib().loza_ssa_decode_kernel(B, Hq, Hkv, int(S_max), d_qk, int(sink), _win(local), int(block), ctypes.byref(n))
    return _checked(k, "loza_ssa_decode_kernel"), n.value


def loza_ssa_backward_split(B, Hq, Hkv, S, d_qk, d_v, sink, local, block=1, v_aliases_k=False):
    """(key tiles cut for balance, chunks of each, other work items) of a bf16 backward's dK/dV kernel."""
    n, w = ctypes.c_int(), ctypes.c_int64()
    t = lib().loza_ssa_backward_split(B, Hq, Hkv, int(S), d_qk, d_v, int(sink), _win(local), int(block), int(bool(v_aliases_k)),
                                      ctypes.byref(n), ctypes.byref(w))
    return _checked(t, "loza_ssa_backward_split"), n.value, w.value


def loza_ssa_decode_workspace_bytes(B, Hq, Hkv, S_max, d_v, n_sink, window) -> int:
    return int(lib().loza_ssa_decode_workspace_bytes(B, Hq, Hkv, int(S_max), d_v, int(n_sink), _win(window)))


def _decode_common(fn_name, q, kcache, vcache, seqlens, out, lse, pattern, scale, workspace, stream):
    """bf16 SSA decode. q [B,Hq,d_qk], kcache [B,S_max,Hkv,d_qk], vcache [B,S_max,Hkv,d_v] or
    ``vcache is kcache``, seqlens [B] int32 on the GPU, out [B,Hq,d_v] bf16, lse [B,Hq] fp32,
    workspace: uint8 GPU tensor of at least ``loza_ssa_decode_workspace_bytes`` bytes."""
    B, Hq, d_qk = q.shape
    _, S_max, Hkv, _ = kcache.shape
    d_v = out.shape[2]
    if kcache.shape != (B, S_max, Hkv, d_qk) or out.shape != (B, Hq, d_v) or lse.shape != (B, Hq) or seqlens.shape != (B,):
        raise ValueError("shape mismatch between q, kcache, seqlens, out, lse")
    if vcache is not kcache and vcache.shape != (B, S_max, Hkv, d_v):
        raise ValueError("vcache must be [B, S_max, Hkv, d_v] (or the very tensor passed as kcache)")
    bf = torch.bfloat16
    qp, kp = _dev_ptr(q, bf, "q"), _dev_ptr(kcache, bf, "kcache")
    vp = kp if vcache is kcache else _dev_ptr(vcache, bf, "vcache")
    wp = _dev_ptr(workspace, torch.uint8, "workspace")
    rc = getattr(lib(), fn_name)(qp, kp, vp, _dev_ptr(seqlens, torch.int32, "seqlens"), _dev_ptr(out, bf, "out"),
                                 _dev_ptr(lse, torch.float32, "lse"), B, Hq, Hkv, S_max, d_qk, d_v,
                                 *pattern, float(scale), wp, workspace.numel(), _stream(stream))
    if rc != LOZA_OK:
        raise LozaError(rc, fn_name)


def loza_ssa_decode(q, kcache, vcache, seqlens, out, lse, n_sink, window, scale, workspace, stream=None):
    """bf16 SSA decode (token-granular pattern); tensors as in :func:`_decode_common`."""
    _decode_common("loza_ssa_decode", q, kcache, vcache, seqlens, out, lse, (int(n_sink), _win(window)), scale,
                   workspace, stream)


LOZA_DECODE_STATIC_BYTES = 40 << 20


def loza_ssa_decode_static(q, kcache, vcache, seqlens, out, lse, n_sink, window, scale, stream=None):
    """:func:`loza_ssa_decode` without a workspace argument: the library's own static device buffer
    holds the partial results (sizes beyond ``LOZA_DECODE_STATIC_BYTES`` are rejected)."""
    B, Hq, d_qk = q.shape
    _, S_max, Hkv, _ = kcache.shape
    d_v = out.shape[2]
    if kcache.shape != (B, S_max, Hkv, d_qk) or out.shape != (B, Hq, d_v) or lse.shape != (B, Hq) or seqlens.shape != (B,):
        raise ValueError("shape mismatch between q, kcache, seqlens, out, lse")
    if vcache is not kcache and vcache.shape != (B, S_max, Hkv, d_v):
        raise ValueError("vcache must be [B, S_max, Hkv, d_v] (or the very tensor passed as kcache)")
    bf = torch.bfloat16
    qp, kp = _dev_ptr(q, bf, "q"), _dev_ptr(kcache, bf, "kcache")
    vp = kp if vcache is kcache else _dev_ptr(vcache, bf, "vcache")
    rc = lib().loza_ssa_decode_static(qp, kp, vp, _dev_ptr(seqlens, torch.int32, "seqlens"), _dev_ptr(out, bf, "out"),
                                      _dev_ptr(lse, torch.float32, "lse"), B, Hq, Hkv, S_max, d_qk, d_v,
                                      int(n_sink), _win(window), float(scale), _stream(stream))
    if rc != LOZA_OK:
        raise LozaError(rc, "loza_ssa_decode_static")


def loza_ssa_decode_blocks(q, kcache, vcache, seqlens, out, lse, sink_blocks, local_blocks, block, scale, workspace,
                           stream=None):
    """bf16 SSA decode under the block-granular pattern; the workspace is sized by
    ``loza_ssa_decode_workspace_bytes(..., sink_blocks * block, local_blocks * block)``."""
    _decode_common("loza_ssa_decode_blocks", q, kcache, vcache, seqlens, out, lse,
                   (int(sink_blocks), _win(local_blocks), int(block)), scale, workspace, stream)


def _decode_f32_common(fn_name, q, kcache, vcache, seqlens, out, lse, pattern, scale, stream):
    """fp32 SSA decode: the tensors of :func:`_decode_common` with float32 elements, no workspace."""
    B, Hq, d_qk = q.shape
    _, S_max, Hkv, _ = kcache.shape
    d_v = out.shape[2]
    if kcache.shape != (B, S_max, Hkv, d_qk) or out.shape != (B, Hq, d_v) or lse.shape != (B, Hq) or seqlens.shape != (B,):
        raise ValueError("shape mismatch between q, kcache, seqlens, out, lse")
    if vcache is not kcache and vcache.shape != (B, S_max, Hkv, d_v):
        raise ValueError("vcache must be [B, S_max, Hkv, d_v] (or the very tensor passed as kcache)")
    f32 = torch.float32
    qp, kp = _dev_ptr(q, f32, "q"), _dev_ptr(kcache, f32, "kcache")
    vp = kp if vcache is kcache else _dev_ptr(vcache, f32, "vcache")
    rc = getattr(lib(), fn_name)(qp, kp, vp, _dev_ptr(seqlens, torch.int32, "seqlens"), _dev_ptr(out, f32, "out"),
                                 _dev_ptr(lse, f32, "lse"), B, Hq, Hkv, S_max, d_qk, d_v, *pattern, float(scale), _stream(stream))
    if rc != LOZA_OK:
        raise LozaError(rc, fn_name)


def loza_ssa_decode_f32(q, kcache, vcache, seqlens, out, lse, n_sink, window, scale, stream=None):
    """fp32 twin of :func:`loza_ssa_decode` (no workspace)."""
    _decode_f32_common("loza_ssa_decode_f32", q, kcache, vcache, seqlens, out, lse, (int(n_sink), _win(window)), scale, stream)


def loza_ssa_decode_blocks_f32(q, kcache, vcache, seqlens, out, lse, sink_blocks, local_blocks, block, scale, stream=None):
    """fp32 twin of :func:`loza_ssa_decode_blocks` (no workspace)."""
    _decode_f32_common("loza_ssa_decode_blocks_f32", q, kcache, vcache, seqlens, out, lse,
                       (int(sink_blocks), _win(local_blocks), int(block)), scale, stream)


def _decode_paged_common(fn_name, q, k_pages, v_pages, block_table, seqlens, out, lse, pattern, scale, workspace, stream):
    """bf16 SSA decode against a paged cache. q [B,Hq,d_qk], k_pages [num_pages,page_size,Hkv,d_qk],
    v_pages [num_pages,page_size,Hkv,d_v] or ``v_pages is k_pages``, block_table [B,max_pages] int32 and
    seqlens [B] int32 on the GPU, out [B,Hq,d_v] bf16, lse [B,Hq] fp32, workspace uint8."""
    B, Hq, d_qk = q.shape
    num_pages, page_size, Hkv, _ = k_pages.shape
    d_v = out.shape[2]
    if k_pages.shape != (num_pages, page_size, Hkv, d_qk) or out.shape != (B, Hq, d_v) or lse.shape != (B, Hq) \
            or seqlens.shape != (B,) or block_table.dim() != 2 or block_table.shape[0] != B:
        raise ValueError("shape mismatch between q, k_pages, block_table, seqlens, out, lse")
    if v_pages is not k_pages and v_pages.shape != (num_pages, page_size, Hkv, d_v):
        raise ValueError("v_pages must be [num_pages, page_size, Hkv, d_v] (or the very tensor passed as k_pages)")
    bf = torch.bfloat16
    qp, kp = _dev_ptr(q, bf, "q"), _dev_ptr(k_pages, bf, "k_pages")
    vp = kp if v_pages is k_pages else _dev_ptr(v_pages, bf, "v_pages")
    rc = getattr(lib(), fn_name)(qp, kp, vp, _dev_ptr(block_table, torch.int32, "block_table"),
                                 _dev_ptr(seqlens, torch.int32, "seqlens"), _dev_ptr(out, bf, "out"),
                                 _dev_ptr(lse, torch.float32, "lse"), B, Hq, Hkv, num_pages, page_size,
                                 block_table.shape[1], d_qk, d_v, *pattern, float(scale),
                                 _dev_ptr(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(stream))
    if rc != LOZA_OK:
        raise LozaError(rc, fn_name)


def loza_ssa_decode_paged(q, k_pages, v_pages, block_table, seqlens, out, lse, n_sink, window, scale, workspace,
                          stream=None):
    """Paged-cache decode, token-granular pattern; tensors as in :func:`_decode_paged_common`."""
    _decode_paged_common("loza_ssa_decode_paged", q, k_pages, v_pages, block_table, seqlens, out, lse,
                         (int(n_sink), _win(window)), scale, workspace, stream)


def loza_ssa_decode_paged_blocks(q, k_pages, v_pages, block_table, seqlens, out, lse, sink_blocks, local_blocks, block,
                                 scale, workspace, stream=None):
    """Paged-cache decode, block-granular pattern."""
    _decode_paged_common("loza_ssa_decode_paged_blocks", q, k_pages, v_pages, block_table, seqlens, out, lse,
                         (int(sink_blocks), _win(local_blocks), int(block)), scale, workspace, stream)


def loza_ssa_calibration_workspace_bytes(B, Hq, S, d_v) -> int:
    return int(lib().loza_ssa_calibration_workspace_bytes(B, Hq, int(S), d_v))


def loza_ssa_prefill_calibration_blocks(q, k, v, out, out_full, out_sparse, lse_full, lse_sparse,
                                        sink_blocks, local_blocks, block, alpha, scale, workspace, stream=None):
    """Calibration forward: out = alpha * O_full + (1 - alpha) * O_sparse (bf16). ``out_full`` / ``out_sparse``
    may be None; lse_full, lse_sparse [B,Hq,S] fp32; workspace uint8 of ``loza_ssa_calibration_workspace_bytes``."""
    B, S, Hq, d_qk = q.shape
    Hkv = k.shape[2]
    d_v = out.shape[3]
    bf = torch.bfloat16
    if k.shape != (B, S, Hkv, d_qk) or out.shape != (B, S, Hq, d_v) or lse_full.shape != (B, Hq, S) or lse_sparse.shape != (B, Hq, S):
        raise ValueError("shape mismatch between q, k, out, lse_full, lse_sparse")
    for t in (out_full, out_sparse):
        if t is not None and t.shape != out.shape:
            raise ValueError("out_full / out_sparse must have the shape of out")
    if v is not k and v.shape != (B, S, Hkv, d_v):
        raise ValueError("v must be [B, S, Hkv, d_v] (or the very tensor passed as k)")
    qp, kp = _dev_ptr(q, bf, "q"), _dev_ptr(k, bf, "k")
    vp = kp if v is k else _dev_ptr(v, bf, "v")
    rc = lib().loza_ssa_prefill_calibration_blocks(
        qp, kp, vp, _dev_ptr(out, bf, "out"),
        None if out_full is None else _dev_ptr(out_full, bf, "out_full"),
        None if out_sparse is None else _dev_ptr(out_sparse, bf, "out_sparse"),
        _dev_ptr(lse_full, torch.float32, "lse_full"), _dev_ptr(lse_sparse, torch.float32, "lse_sparse"),
        B, Hq, Hkv, S, d_qk, d_v, int(sink_blocks), _win(local_blocks), int(block), float(alpha), float(scale),
        _dev_ptr(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(stream))
    if rc != LOZA_OK:
        raise LozaError(rc, "loza_ssa_prefill_calibration_blocks")


def loza_ssa_calibration_alpha_grad_workspace_bytes(n) -> int:
    return int(lib().loza_ssa_calibration_alpha_grad_workspace_bytes(int(n)))


def loza_ssa_calibration_alpha_grad(dout, out_full, out_sparse, dalpha, workspace, stream=None):
    """d(alpha) of the calibration blend: sum of dout * (out_full - out_sparse). Three bf16 GPU tensors of
    one shape, dalpha a float32 GPU tensor of one element, workspace uint8."""
    if out_full.shape != dout.shape or out_sparse.shape != dout.shape or dalpha.numel() != 1:
        raise ValueError("dout, out_full, out_sparse must share a shape; dalpha holds one element")
    bf = torch.bfloat16
    rc = lib().loza_ssa_calibration_alpha_grad(_dev_ptr(dout, bf, "dout"), _dev_ptr(out_full, bf, "out_full"),
                                               _dev_ptr(out_sparse, bf, "out_sparse"), _dev_ptr(dalpha, torch.float32, "dalpha"),
                                               dout.numel(), _dev_ptr(workspace, torch.uint8, "workspace"), workspace.numel(),
                                               _stream(stream))
    if rc != LOZA_OK:
        raise LozaError(rc, "loza_ssa_calibration_alpha_grad")


@functools.lru_cache(maxsize=1024)
def loza_ssa_extend_workspace_bytes(B, Hq, Hkv, S_max, q_len, d_qk, d_v, sink, local, block=1) -> int:
    """Bytes of scratch memory with which an extend of these sizes lets several workgroups share the keys of a query
    (0: it has no use for any). Host only."""
    return int(lib().loza_ssa_extend_workspace_bytes(B, Hq, Hkv, S_max, q_len, d_qk, d_v, sink, _win(local), block))


def _scratch(nbytes: int, stream):
    """Scratch memory for launches on `stream`, from torch's allocator and of that stream (given back when the caller
    drops it, it can only be handed out again behind those launches). None where there is none to be had: no memory
    left, a stream under capture, whose graph would keep the address of memory that is given back, or the per-thread
    stream, whose one handle names many streams."""
    if stream is not None and _stream(stream) != _stream(None):
        if not isinstance(stream, torch.cuda.Stream):
            handle = _stream(stream)
            if handle == _STREAM_PER_THREAD:
                return None
            # (torch takes a handle of 0 as none given, and makes a stream of its pool of it)
            stream = torch.cuda.default_stream() if handle in (0, _STREAM_LEGACY) else torch.cuda.ExternalStream(handle)
        with torch.cuda.stream(stream):
            return _scratch(nbytes, None)
    if torch.cuda.is_current_stream_capturing():
        return None
    # (an allocation that reaches the driver ends the captures of other threads, unless this thread says it may not matter)
    mode = ctypes.c_int(_CAPTURE_MODE_RELAXED)
    lib().hipThreadExchangeStreamCaptureMode(ctypes.byref(mode))
    try:
        return torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    except torch.OutOfMemoryError:
        return None
    finally:
        lib().hipThreadExchangeStreamCaptureMode(ctypes.byref(mode))


def _extend_call(fn_name, pointers, table, sizes, paging, S_max, q_len, d_qk, d_v, pattern, scale, workspace, stream):
    """The extend entry point of that name, or, where scratch memory helps and is there, the one that takes it."""
    B, Hq, Hkv = sizes
    blocks = pattern if len(pattern) == 3 else (*pattern, 1)
    need = loza_ssa_extend_workspace_bytes(B, Hq, Hkv, S_max, q_len, d_qk, d_v, *blocks)
    if need and workspace is None:
        workspace = _scratch(need, stream)
    if need and workspace is not None:
        rc = lib().loza_ssa_extend_with_workspace(*pointers[:3], table, *pointers[3:], B, Hq, Hkv, S_max, *(paging or (0, 0, 0)), q_len, d_qk, d_v,
                                                  *blocks, scale, _dev_ptr(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(stream))
    elif paging:
        rc = getattr(lib(), fn_name)(*pointers[:3], table, *pointers[3:], B, Hq, Hkv, *paging, q_len, d_qk, d_v, *pattern, scale, _stream(stream))
    else:
        rc = getattr(lib(), fn_name)(*pointers, B, Hq, Hkv, S_max, q_len, d_qk, d_v, *pattern, scale, _stream(stream))
    if rc != LOZA_OK:
        raise LozaError(rc, fn_name)


def _extend_common(fn_name, q, kcache, vcache, seqlens, out, lse, pattern, scale, workspace, stream):
    """bf16 SSA extend. q [B,q_len,Hq,d_qk], kcache [B,S_max,Hkv,d_qk], vcache [B,S_max,Hkv,d_v] or
    ``vcache is kcache``, seqlens [B] int32 on the GPU, out [B,q_len,Hq,d_v] bf16, lse [B,Hq,q_len] fp32.
    workspace: uint8 GPU tensor of at least ``loza_ssa_extend_workspace_bytes`` bytes, of its own for every call that may
    overlap another in time; without one, scratch memory comes from torch's allocator (which may have to give its cache
    back to find it) or, under capture and where there is none, the call does without: slower, and with other bits."""
    B, q_len, Hq, d_qk = q.shape
    _, S_max, Hkv, _ = kcache.shape
    d_v = out.shape[3]
    if kcache.shape != (B, S_max, Hkv, d_qk) or out.shape != (B, q_len, Hq, d_v) or lse.shape != (B, Hq, q_len) \
            or seqlens.shape != (B,):
        raise ValueError("shape mismatch between q, kcache, seqlens, out, lse")
    if vcache is not kcache and vcache.shape != (B, S_max, Hkv, d_v):
        raise ValueError("vcache must be [B, S_max, Hkv, d_v] (or the very tensor passed as kcache)")
    bf = torch.bfloat16
    qp, kp = _dev_ptr(q, bf, "q"), _dev_ptr(kcache, bf, "kcache")
    vp = kp if vcache is kcache else _dev_ptr(vcache, bf, "vcache")
    _extend_call(fn_name, (qp, kp, vp, _dev_ptr(seqlens, torch.int32, "seqlens"), _dev_ptr(out, bf, "out"), _dev_ptr(lse, torch.float32, "lse")),
                 None, (B, Hq, Hkv), None, S_max, q_len, d_qk, d_v, pattern, float(scale), workspace, stream)


def loza_ssa_extend(q, kcache, vcache, seqlens, out, lse, n_sink, window, scale, stream=None, workspace=None):
    """q_len new tokens per sequence against its cache, token-granular pattern (see :func:`_extend_common`)."""
    _extend_common("loza_ssa_extend", q, kcache, vcache, seqlens, out, lse, (int(n_sink), _win(window)), scale, workspace, stream)


def loza_ssa_extend_blocks(q, kcache, vcache, seqlens, out, lse, sink_blocks, local_blocks, block, scale, stream=None, workspace=None):
    """q_len new tokens per sequence against its cache, block-granular pattern."""
    _extend_common("loza_ssa_extend_blocks", q, kcache, vcache, seqlens, out, lse,
                   (int(sink_blocks), _win(local_blocks), int(block)), scale, workspace, stream)


def _extend_paged_common(fn_name, q, k_pages, v_pages, block_table, seqlens, out, lse, pattern, scale, workspace, stream):
    """bf16 SSA extend against a paged cache: q [B,q_len,Hq,d_qk], k_pages [num_pages,page_size,Hkv,d_qk],
    v_pages likewise with d_v (or ``v_pages is k_pages``), block_table [B,max_pages] int32, seqlens [B] int32,
    out [B,q_len,Hq,d_v] bf16, lse [B,Hq,q_len] fp32."""
    B, q_len, Hq, d_qk = q.shape
    num_pages, page_size, Hkv, _ = k_pages.shape
    d_v = out.shape[3]
    if k_pages.shape != (num_pages, page_size, Hkv, d_qk) or out.shape != (B, q_len, Hq, d_v) or lse.shape != (B, Hq, q_len) \
            or seqlens.shape != (B,) or block_table.dim() != 2 or block_table.shape[0] != B:
        raise ValueError("shape mismatch between q, k_pages, block_table, seqlens, out, lse")
    if v_pages is not k_pages and v_pages.shape != (num_pages, page_size, Hkv, d_v):
        raise ValueError("v_pages must be [num_pages, page_size, Hkv, d_v] (or the very tensor passed as k_pages)")
    bf = torch.bfloat16
    qp, kp = _dev_ptr(q, bf, "q"), _dev_ptr(k_pages, bf, "k_pages")
    vp = kp if v_pages is k_pages else _dev_ptr(v_pages, bf, "v_pages")
    max_pages = block_table.shape[1]
    _extend_call(fn_name, (qp, kp, vp, _dev_ptr(seqlens, torch.int32, "seqlens"), _dev_ptr(out, bf, "out"), _dev_ptr(lse, torch.float32, "lse")),
                 _dev_ptr(block_table, torch.int32, "block_table"), (B, Hq, Hkv), (num_pages, page_size, max_pages), max_pages * page_size,
                 q_len, d_qk, d_v, pattern, float(scale), workspace, stream)


def loza_ssa_extend_paged(q, k_pages, v_pages, block_table, seqlens, out, lse, n_sink, window, scale, stream=None, workspace=None):
    """Extend against a paged cache, token-granular pattern (see :func:`_extend_paged_common`)."""
    _extend_paged_common("loza_ssa_extend_paged", q, k_pages, v_pages, block_table, seqlens, out, lse,
                         (int(n_sink), _win(window)), scale, workspace, stream)


def loza_ssa_extend_paged_blocks(q, k_pages, v_pages, block_table, seqlens, out, lse, sink_blocks, local_blocks, block,
                                 scale, stream=None, workspace=None):
    """Extend against a paged cache, block-granular pattern."""
    _extend_paged_common("loza_ssa_extend_paged_blocks", q, k_pages, v_pages, block_table, seqlens, out, lse,
                         (int(sink_blocks), _win(local_blocks), int(block)), scale, workspace, stream)


def loza_ssa_backward_workspace_bytes(B, Hq, Hkv, S, d_qk, d_v, n_sink, window, v_aliases_k) -> int:
    return int(lib().loza_ssa_backward_workspace_bytes(B, Hq, Hkv, int(S), d_qk, d_v, int(n_sink), _win(window),
                                                       1 if v_aliases_k else 0))


def loza_ssa_backward_workspace_bytes_blocks(B, Hq, Hkv, S, d_qk, d_v, sink_blocks, local_blocks, block,
                                             v_aliases_k) -> int:
    return int(lib().loza_ssa_backward_workspace_bytes_blocks(B, Hq, Hkv, int(S), d_qk, d_v, int(sink_blocks),
                                                              _win(local_blocks), int(block), 1 if v_aliases_k else 0))


def _backward_common(fn_name, q, k, v, out, lse, dout, dq, dk, dv, pattern, scale, workspace, stream):
    """bf16 SSA backward. q, dq [B,S,Hq,d_qk]; k, dk [B,S,Hkv,d_qk]; v, dv [B,S,Hkv,d_v] (``v is k``:
    dk receives the gradient of the shared tensor, dv is None); out, dout [B,S,Hq,d_v] bf16; lse
    [B,Hq,S] fp32; workspace uint8 of at least ``loza_ssa_backward_workspace_bytes`` bytes."""
    B, S, Hq, d_qk = q.shape
    Hkv = k.shape[2]
    d_v = out.shape[3]
    if k.shape != (B, S, Hkv, d_qk) or out.shape != (B, S, Hq, d_v) or dout.shape != out.shape \
            or lse.shape != (B, Hq, S) or dq.shape != q.shape or dk.shape != k.shape:
        raise ValueError("shape mismatch between q, k, out, lse, dout, dq, dk")
    bf = torch.bfloat16
    kp = _dev_ptr(k, bf, "k")
    if v is k:
        vp, dvp = kp, None
    else:
        if v.shape != (B, S, Hkv, d_v) or dv is None or dv.shape != v.shape:
            raise ValueError("v and dv must be [B, S, Hkv, d_v] (or v the very tensor passed as k)")
        vp, dvp = _dev_ptr(v, bf, "v"), _dev_ptr(dv, bf, "dv")
    rc = getattr(lib(), fn_name)(_dev_ptr(q, bf, "q"), kp, vp, _dev_ptr(out, bf, "out"), _dev_ptr(lse, torch.float32, "lse"),
                                 _dev_ptr(dout, bf, "dout"), _dev_ptr(dq, bf, "dq"), _dev_ptr(dk, bf, "dk"), dvp,
                                 B, Hq, Hkv, S, d_qk, d_v, *pattern, float(scale),
                                 _dev_ptr(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(stream))
    if rc != LOZA_OK:
        raise LozaError(rc, fn_name)


def _backward_f32_common(fn_name, q, k, v, out, lse, dout, dq, dk, dv, pattern, scale, stream):
    """fp32 SSA backward: the tensors of :func:`_backward_common` with float32 elements, no workspace."""
    B, S, Hq, d_qk = q.shape
    Hkv = k.shape[2]
    d_v = out.shape[3]
    if k.shape != (B, S, Hkv, d_qk) or out.shape != (B, S, Hq, d_v) or dout.shape != out.shape \
            or lse.shape != (B, Hq, S) or dq.shape != q.shape or dk.shape != k.shape:
        raise ValueError("shape mismatch between q, k, out, lse, dout, dq, dk")
    f32 = torch.float32
    kp = _dev_ptr(k, f32, "k")
    if v is k:
        vp, dvp = kp, None
    else:
        if v.shape != (B, S, Hkv, d_v) or dv is None or dv.shape != v.shape:
            raise ValueError("v and dv must be [B, S, Hkv, d_v] (or v the very tensor passed as k)")
        vp, dvp = _dev_ptr(v, f32, "v"), _dev_ptr(dv, f32, "dv")
    rc = getattr(lib(), fn_name)(_dev_ptr(q, f32, "q"), kp, vp, _dev_ptr(out, f32, "out"), _dev_ptr(lse, f32, "lse"),
                                 _dev_ptr(dout, f32, "dout"), _dev_ptr(dq, f32, "dq"), _dev_ptr(dk, f32, "dk"), dvp,
                                 B, Hq, Hkv, S, d_qk, d_v, *pattern, float(scale), _stream(stream))
    if rc != LOZA_OK:
        raise LozaError(rc, fn_name)


def loza_ssa_backward_f32(q, k, v, out, lse, dout, dq, dk, dv, n_sink, window, scale, stream=None):
    """fp32 twin of :func:`loza_ssa_backward`."""
    _backward_f32_common("loza_ssa_backward_f32", q, k, v, out, lse, dout, dq, dk, dv, (int(n_sink), _win(window)), scale, stream)


def loza_ssa_backward_blocks_f32(q, k, v, out, lse, dout, dq, dk, dv, sink_blocks, local_blocks, block, scale, stream=None):
    """fp32 twin of :func:`loza_ssa_backward_blocks`."""
    _backward_f32_common("loza_ssa_backward_blocks_f32", q, k, v, out, lse, dout, dq, dk, dv,
                         (int(sink_blocks), _win(local_blocks), int(block)), scale, stream)


def loza_ssa_backward(q, k, v, out, lse, dout, dq, dk, dv, n_sink, window, scale, workspace, stream=None):
    """Gradients of :func:`loza_ssa_prefill` (token-granular pattern); tensors as in :func:`_backward_common`."""
    _backward_common("loza_ssa_backward", q, k, v, out, lse, dout, dq, dk, dv, (int(n_sink), _win(window)), scale,
                     workspace, stream)


def loza_ssa_backward_blocks(q, k, v, out, lse, dout, dq, dk, dv, sink_blocks, local_blocks, block, scale, workspace,
                             stream=None):
    """Gradients of :func:`loza_ssa_prefill_blocks` (block-granular pattern)."""
    _backward_common("loza_ssa_backward_blocks", q, k, v, out, lse, dout, dq, dk, dv,
                     (int(sink_blocks), _win(local_blocks), int(block)), scale, workspace, stream)


# ---- the step around the attention -------------------------------------------------------------------------

LOZA_TREE_MAX_NODES = 64


def _launch_device(t) -> int:
    """The current device, to which a launch goes (-2, which no tensor is on, where `t` is not on a GPU)."""
    return torch._C._cuda_getDevice() if isinstance(t, torch.Tensor) and t.is_cuda else -2


def _ptr(t, dtype, shape, name: str, device: int):
    """Address of a contiguous tensor of that type and shape (None: any) on that device; None for None. (One test of everything first: a
    dozen tensors looked at one property at a time are half the host's time of a call.)"""
    if t is None:
        return None
    if isinstance(t, torch.Tensor) and t.dtype is dtype and (shape is None or t.shape == shape) and t.get_device() == device and t.is_contiguous():
        return t.data_ptr()
    _dev_ptr(t, dtype, name)
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    raise ValueError(f"{name} is on device {t.get_device()}, the current one is {device}")


def _heads(t, dtype, shape, name: str, device: int):
    """(pointer, token stride, head stride) of a [T, H, d] tensor whose columns lie side by side; zeros for None."""
    if t is None:
        return None, 0, 0
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.get_device() == device:
        st, sh, sc = t.stride()
        if sc == 1 or shape[2] == 1:
            return t.data_ptr(), st, sh
        raise ValueError(f"the columns of {name} must lie side by side")
    _dev_ptr(t.contiguous() if isinstance(t, torch.Tensor) else t, dtype, name)
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    raise ValueError(f"{name} is on device {t.get_device()}, the current one is {device}")


def _call(fn_name, *args) -> None:
    rc = getattr(lib(), fn_name)(*args)
    if rc != LOZA_OK:
        raise LozaError(rc, fn_name)


def loza_ssa_step_tables(cache_lens, new_lens, parents, free_pages, free_count, block_table, num_pages, page_size,
                         granted, seqlens, positions, slots, masks, free_left, stream=None, held=None, held_after=None):
    """Block table entries, slots, positions and (``parents`` given: the tokens are trees) ancestor masks of a step. cache_lens, new_lens,
    granted, seqlens [B], parents (or None), positions, slots [B,n], block_table [B,max_pages], free_pages [F], free_count and
    free_left [1], all int32 on the GPU; masks [B,n] int64 (None without parents). ``block_table`` is extended in place. held, held_after [B]
    int32 (both or neither): pages that each request has before and after the call (``loza_ssa_step_tables_held``); a step whose rows are not
    all kept needs them, or its requests' spare pages are dealt out anew and lost."""
    dev, i32 = _launch_device(positions), torch.int32
    B, n = positions.shape
    rows, both, (num_free,), most = (B,), (B, n), free_pages.shape, block_table.shape[-1]
    if (parents is None) != (masks is None):
        raise ValueError("parents and masks must both be [B, n], or both None")
    if (held is None) != (held_after is None):
        raise ValueError("held and held_after must both be [B], or both None")
    if held is None:
        return _call("loza_ssa_step_tables", _ptr(cache_lens, i32, rows, "cache_lens", dev), _ptr(new_lens, i32, rows, "new_lens", dev),
                     _ptr(parents, i32, both, "parents", dev), _ptr(free_pages, i32, None, "free_pages", dev), _ptr(free_count, i32, (1,), "free_count", dev),
                     _ptr(block_table, i32, (B, most), "block_table", dev), B, n, num_free, int(num_pages), int(page_size), most,
                     _ptr(granted, i32, rows, "granted", dev), _ptr(seqlens, i32, rows, "seqlens", dev), _ptr(positions, i32, both, "positions", dev),
                     _ptr(slots, i32, both, "slots", dev), _ptr(masks, torch.int64, both, "masks", dev), _ptr(free_left, i32, (1,), "free_left", dev), _stream(stream))
    _call("loza_ssa_step_tables_held", _ptr(cache_lens, i32, rows, "cache_lens", dev), _ptr(new_lens, i32, rows, "new_lens", dev),
          _ptr(parents, i32, both, "parents", dev), _ptr(free_pages, i32, None, "free_pages", dev), _ptr(free_count, i32, (1,), "free_count", dev),
          _ptr(held, i32, rows, "held", dev), _ptr(block_table, i32, (B, most), "block_table", dev), B, n, num_free, int(num_pages), int(page_size), most,
          _ptr(granted, i32, rows, "granted", dev), _ptr(seqlens, i32, rows, "seqlens", dev), _ptr(positions, i32, both, "positions", dev),
          _ptr(slots, i32, both, "slots", dev), _ptr(masks, torch.int64, both, "masks", dev), _ptr(free_left, i32, (1,), "free_left", dev),
          _ptr(held_after, i32, rows, "held_after", dev), _stream(stream))


def loza_ssa_rope_frequencies(rot_dim, base, factor=1.0, original_context=0, slow_turns=1.0, fast_turns=32.0):
    """(freq, mscale): float64 CPU tensor [rot_dim / 2] of radians per position, and the scale of queries and keys. Host only."""
    freq, m = torch.empty(max(0, int(rot_dim)) // 2 or 1, dtype=torch.float64), ctypes.c_float()
    _call("loza_ssa_rope_frequencies", int(rot_dim), float(base), float(factor), int(original_context), float(slow_turns), float(fast_turns),
          ctypes.cast(freq.data_ptr(), ctypes.POINTER(ctypes.c_double)), ctypes.byref(m))
    return freq, m.value


def _rope(fn_name, dtype, x, positions, freq, out, rot_begin, interleaved, mscale, inverse, stream):
    dev, shape, (pairs,) = _launch_device(x), x.shape, freq.shape
    T, H, d = shape
    xp, xt, xh = _heads(x, dtype, shape, "x", dev)
    op, ot, oh = _heads(out, dtype, shape, "out", dev)
    _call(fn_name, xp, _ptr(positions, torch.int32, (T,), "positions", dev), _ptr(freq, torch.float64, None, "freq", dev), op, T, H, d, xt, xh, ot, oh,
          int(rot_begin), 2 * pairs, bool(interleaved), bool(inverse), float(mscale), _stream(stream))


def loza_ssa_rope(x, positions, freq, out, rot_begin, interleaved, mscale=1.0, inverse=False, stream=None):
    """Rotary positions: columns [rot_begin, rot_begin + 2 len(freq)) of x [T,H,d] bf16 into out (any token and head strides; ``out is x``: in
    place), the other columns copied. positions [T] int32 (negative: the row of out is left as it is), freq float64 on the GPU.
    ``inverse``: the gradient of x from that of out."""
    _rope("loza_ssa_rope", torch.bfloat16, x, positions, freq, out, rot_begin, interleaved, mscale, inverse, stream)


def loza_ssa_rope_f32(x, positions, freq, out, rot_begin, interleaved, mscale=1.0, inverse=False, stream=None):
    """fp32 twin of :func:`loza_ssa_rope`."""
    _rope("loza_ssa_rope_f32", torch.float32, x, positions, freq, out, rot_begin, interleaved, mscale, inverse, stream)


def _rope_append(fn_name, dtype, q, k, v, positions, slots, freq, q_out, k_rows, v_rows, q_rot_begin, k_rot_begin, interleaved, mscale, stream):
    dev, i32, (pairs,) = _launch_device(k), torch.int32, freq.shape
    T, Hkv, d_k = k.shape
    *lead, hk, dk = k_rows.shape
    if not lead or (hk, dk) != (Hkv, d_k):
        raise ValueError("k_rows must be [..., Hkv, d_k]")
    if (q is None) != (q_out is None) or (v is None) != (v_rows is None):
        raise ValueError("q and q_out go together, and so do v and v_rows")
    rows, Hq, d_q, d_v = math.prod(lead), 0, 0, 0
    if q is not None:
        _, Hq, d_q = q.shape
    if v is not None:
        d_v = v.shape[-1]
    qp, qt, qh = _heads(q, dtype, (T, Hq, d_q), "q", dev)
    op, ot, oh = _heads(q_out, dtype, (T, Hq, d_q), "q_out", dev)
    kp, kt, kh = _heads(k, dtype, (T, Hkv, d_k), "k", dev)
    vp, vt, vh = _heads(v, dtype, (T, Hkv, d_v), "v", dev)
    _call(fn_name, qp, kp, vp, _ptr(positions, i32, (T,), "positions", dev), _ptr(slots, i32, (T,), "slots", dev),
          _ptr(freq, torch.float64, None, "freq", dev), op, _ptr(k_rows, dtype, None, "k_rows", dev),
          _ptr(v_rows, dtype, (*lead, Hkv, d_v), "v_rows", dev), T, Hq, Hkv, d_q, d_k, d_v, qt, qh, ot, oh, kt, kh, vt, vh, rows,
          int(q_rot_begin), int(k_rot_begin), 2 * pairs, bool(interleaved), float(mscale), _stream(stream))


def loza_ssa_rope_append(q, k, v, positions, slots, freq, q_out, k_rows, v_rows, q_rot_begin, k_rot_begin, interleaved, mscale=1.0, stream=None):
    """Rotates q [T,Hq,d_q] into q_out (both may be None) and k [T,Hkv,d_k] into row slots[t] of k_rows [..., Hkv, d_k] (a paged or a
    contiguous cache), and copies v [T,Hkv,d_v] there (v and v_rows None: the values are part of the keys). bf16; positions, slots [T] int32, freq
    float64 on the GPU; q, q_out, k, v with any token and head strides."""
    _rope_append("loza_ssa_rope_append", torch.bfloat16, q, k, v, positions, slots, freq, q_out, k_rows, v_rows, q_rot_begin, k_rot_begin,
                 interleaved, mscale, stream)


def loza_ssa_rope_append_f32(q, k, v, positions, slots, freq, q_out, k_rows, v_rows, q_rot_begin, k_rot_begin, interleaved, mscale=1.0, stream=None):
    """fp32 twin of :func:`loza_ssa_rope_append`."""
    _rope_append("loza_ssa_rope_append_f32", torch.float32, q, k, v, positions, slots, freq, q_out, k_rows, v_rows, q_rot_begin, k_rot_begin,
                 interleaved, mscale, stream)


@functools.lru_cache(maxsize=1024)
def loza_ssa_extend_tree_workspace_bytes(B, Hq, Hkv, S_max, n, d_qk, d_v, sink, local, block=1) -> int:
    """Bytes of scratch memory with which :func:`loza_ssa_extend_tree` lets several workgroups share the keys of a query (0: it has no use
    for any). Host only."""
    return int(lib().loza_ssa_extend_tree_workspace_bytes(B, Hq, Hkv, S_max, n, d_qk, d_v, sink, _win(local), block))


def loza_ssa_extend_tree_kernel(B, Hq, Hkv, S_max, n, d_qk, sink, local, block=1, scratch=True):
    """(KERNEL_..., workgroups that share the keys of a row) of a tree call of these sizes. Host only."""
    k = ctypes.c_int()
    kernel = lib().loza_ssa_extend_tree_kernel(B, Hq, Hkv, int(S_max), n, d_qk, int(sink), _win(local), int(block), int(bool(scratch)), ctypes.byref(k))
    return _checked(kernel, "loza_ssa_extend_tree_kernel"), k.value


def loza_ssa_extend_tree(q, kcache, vcache, seqlens, tree_lens, masks, out, lse, sink_blocks, local_blocks, block, scale,
                         block_table=None, workspace=None, stream=None):
    """Attention of a tree of drafted tokens per sequence over a cache that holds their rows. q [B,n,Hq,d_qk], out [B,n,Hq,d_v] bf16, lse [B,Hq,n]
    fp32; kcache, vcache as for :func:`loza_ssa_extend`, or pages with ``block_table`` [B,max_pages]; seqlens (the nodes' rows included), tree_lens [B]
    int32, masks [B,n] int64 as :func:`loza_ssa_step_tables` makes them. block = 1: the pattern in tokens. workspace: as for the extends."""
    dev, bf, i32 = _launch_device(q), torch.bfloat16, torch.int32
    B, n, Hq, d_qk = q.shape
    lead, size, Hkv, d_k = kcache.shape
    d_v = out.shape[-1]
    if d_k != d_qk or (block_table is None and lead != B):
        raise ValueError("kcache must be [B, S_max, Hkv, d_qk], or pages [num_pages, page_size, Hkv, d_qk] with a block_table")
    paging = (0, 0, 0) if block_table is None else (lead, size, block_table.shape[-1])
    S_max = size if block_table is None else size * paging[2]
    pattern = (int(sink_blocks), _win(local_blocks), int(block))
    kp = _ptr(kcache, bf, None, "kcache", dev)
    args = (_ptr(q, bf, None, "q", dev), kp, kp if vcache is kcache else _ptr(vcache, bf, (lead, size, Hkv, d_v), "vcache", dev),
            _ptr(block_table, i32, (B, paging[2]), "block_table", dev), _ptr(seqlens, i32, (B,), "seqlens", dev), _ptr(tree_lens, i32, (B,), "tree_lens", dev),
            _ptr(masks, torch.int64, (B, n), "masks", dev), _ptr(out, bf, (B, n, Hq, d_v), "out", dev), _ptr(lse, torch.float32, (B, Hq, n), "lse", dev))
    if workspace is None:
        need = loza_ssa_extend_tree_workspace_bytes(B, Hq, Hkv, S_max, n, d_qk, d_v, *pattern)
        workspace = _scratch(need, stream) if need else None
    _call("loza_ssa_extend_tree", *args, B, Hq, Hkv, S_max, *paging, n, d_qk, d_v, *pattern, float(scale),
          _ptr(workspace, torch.uint8, None, "workspace", dev), 0 if workspace is None else workspace.numel(), _stream(stream))


def loza_ssa_verify_tree_workspace_bytes(B, n, V) -> int:
    return int(lib().loza_ssa_verify_tree_workspace_bytes(int(B), int(n), int(V)))


def loza_ssa_verify_tree(target, draft, tokens, parents, tree_lens, u_accept, u_next, path, path_lens, next_token, workspace, stream=None):
    """Which drafted nodes hold, and the token after them. target [B,n,V] float32 probabilities, draft likewise or None (drafts that are not random),
    tokens, parents, path [B,n], tree_lens, path_lens, next_token [B] int32, u_accept [B,n], u_next [B] float32, workspace uint8."""
    dev, f32, i32 = _launch_device(target), torch.float32, torch.int32
    B, n, V = target.shape
    rows, both = (B,), (B, n)
    _call("loza_ssa_verify_tree", _ptr(target, f32, None, "target", dev), _ptr(draft, f32, (B, n, V), "draft", dev), _ptr(tokens, i32, both, "tokens", dev),
          _ptr(parents, i32, both, "parents", dev), _ptr(tree_lens, i32, rows, "tree_lens", dev), _ptr(u_accept, f32, both, "u_accept", dev),
          _ptr(u_next, f32, rows, "u_next", dev), _ptr(path, i32, both, "path", dev), _ptr(path_lens, i32, rows, "path_lens", dev),
          _ptr(next_token, i32, rows, "next_token", dev), B, n, V, _ptr(workspace, torch.uint8, None, "workspace", dev), workspace.numel(), _stream(stream))


def loza_ssa_keep_accepted(k_rows, v_rows, slots, path, path_lens, stream=None):
    """Moves the rows of the accepted path: row slots[b, path[b, i]] of the cache becomes row slots[b, i]. k_rows [layers, ..., Hkv, d]: caches of one
    or more layers, any type, at least 4 dimensions, the first of them the layers, the last two a row; v_rows likewise or None."""
    dev, i32 = _launch_device(k_rows), torch.int32
    B, n = slots.shape
    layers, *lead, hk, dk = k_rows.shape
    if not lead or (v_rows is not None and v_rows.shape[:-2] != k_rows.shape[:-2]):
        raise ValueError("k_rows must be [layers, ..., Hkv, d], v_rows of the same layers and rows")
    v_bytes = 0 if v_rows is None else v_rows.shape[-2] * v_rows.shape[-1] * v_rows.element_size()
    _call("loza_ssa_keep_accepted", _ptr(k_rows, k_rows.dtype, None, "k_rows", dev), None if v_rows is None else _ptr(v_rows, v_rows.dtype, None, "v_rows", dev),
          _ptr(slots, i32, None, "slots", dev), _ptr(path, i32, (B, n), "path", dev), _ptr(path_lens, i32, (B,), "path_lens", dev), B, n, layers,
          math.prod(lead), hk * dk * k_rows.element_size(), v_bytes, _stream(stream))
