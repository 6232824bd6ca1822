"""ctypes binding of ``libmala.so`` (C ABI in ``include/mala.h``): argument marshalling only.

PyTorch is used for device memory and the current stream; every step of the attention path runs in
the library's kernels.  There is no CPU or eager fallback: if the library is missing or a call
fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import functools
import math
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIBPATH = os.path.join(_HERE, "libmala.so")
_lib = None

OP_FWD, OP_BWD, OP_DECODE = 0, 1, 2


class MalaError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {lib().mala_strerror(code).decode()} (code {code})")
        self.code = code


class _TIn(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("sb", ctypes.c_int64), ("sn", ctypes.c_int64), ("sh", ctypes.c_int64)]


class _TOut(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("sb", ctypes.c_int64), ("sn", ctypes.c_int64), ("sh", ctypes.c_int64)]


class _Stats(ctypes.Structure):
    _fields_ = [("retained_per_block", ctypes.c_void_p), ("tile_bitmask", ctypes.c_void_p),
                ("totals", ctypes.c_void_p)]


class _RelBias(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("sb", ctypes.c_int64), ("num_buckets", ctypes.c_int),
                ("max_distance", ctypes.c_int), ("bidirectional", ctypes.c_int)]


class _Rotary(ctypes.Structure):
    _fields_ = [("inv_freq", ctypes.c_void_p), ("rotary", ctypes.c_int), ("interleaved", ctypes.c_int),
                ("magnitude", ctypes.c_float)]


class _HeadNorm(ctypes.Structure):
    _fields_ = [("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("weights_fp32", ctypes.c_int),
                ("eps", ctypes.c_float)]


def lib():
    """Loads libmala.so (built in-tree by ``paper_2609_32712_b200.build``); fails loudly if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIBPATH):
            raise ImportError(f"{_LIBPATH} is missing: run `python -m paper_2609_32712_b200.build` (needs nvcc)")
        L = ctypes.CDLL(_LIBPATH)
        i, f, vp, sz = ctypes.c_int, ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t
        L.mala_fwd.argtypes = [_TIn, _TIn, _TIn, _TOut, vp, ctypes.POINTER(_Stats), i, i, i, i, i, i, f, f, vp, sz, vp]
        L.mala_bwd.argtypes = [_TIn, _TIn, _TIn, _TIn, _TIn, vp, _TOut, _TOut, _TOut, ctypes.POINTER(_Stats),
                               i, i, i, i, i, i, f, f, vp, sz, vp]
        L.mala_fwd_chunk.argtypes = [_TIn, _TIn, _TIn, _TOut, vp, ctypes.POINTER(_Stats), i, i, i, i, i, i, i, f, f, vp,
                                     sz, vp]
        L.mala_bwd_chunk.argtypes = [_TIn, _TIn, _TIn, _TIn, _TIn, vp, _TOut, _TOut, _TOut, ctypes.POINTER(_Stats),
                                     i, i, i, i, i, i, i, f, f, vp, sz, vp]
        L.mala_fwd_chunk.restype = i
        L.mala_bwd_chunk.restype = i
        L.mala_fwd_chunk_split.argtypes = [_TIn, _TIn, _TIn, _TOut, vp, ctypes.POINTER(_Stats), i, i, i, i, i, i, i, f, f,
                                           i, vp, sz, vp]
        L.mala_fwd_chunk_split.restype = i
        L.mala_fwd_varlen.argtypes = [_TIn, _TIn, _TIn, vp, _TOut, vp, ctypes.POINTER(_Stats), i, i, i, i, i, i, i, f, f,
                                      vp, sz, vp]
        L.mala_bwd_varlen.argtypes = [_TIn, _TIn, _TIn, _TIn, _TIn, vp, vp, _TOut, _TOut, _TOut, ctypes.POINTER(_Stats),
                                      i, i, i, i, i, i, i, f, f, vp, sz, vp]
        L.mala_fwd_varlen_prefix.argtypes = [_TIn, _TIn, _TIn, vp, vp, _TOut, vp, ctypes.POINTER(_Stats), i, i, i, i, i, i,
                                             i, i, i, f, f, vp, sz, vp]
        L.mala_fwd_varlen_prefix.restype = i
        L.mala_bwd_varlen_prefix.argtypes = [_TIn, _TIn, _TIn, _TIn, _TIn, vp, vp, vp, _TOut, _TOut, _TOut,
                                             ctypes.POINTER(_Stats), i, i, i, i, i, i, i, i, i, f, f, vp, sz, vp]
        L.mala_bwd_varlen_prefix.restype = i
        L.mala_fwd_paged.argtypes = [_TIn, _TIn, _TIn, vp, vp, vp, _TOut, vp, ctypes.POINTER(_Stats), i, i, i, i, i, i, i, i,
                                     i, i, f, f, vp, sz, vp]
        L.mala_fwd_paged.restype = i
        L.mala_fwd_varlen.restype = i
        L.mala_bwd_varlen.restype = i
        L.mala_decode.argtypes = [_TIn, _TIn, _TIn, _TOut, vp, ctypes.POINTER(_Stats), i, i, i, i, i, f, f, i, vp, sz, vp]
        L.mala_decode_multi.argtypes = [_TIn, _TIn, _TIn, _TOut, vp, ctypes.POINTER(_Stats), i, i, i, i, i, i, f, f, i,
                                        vp, sz, vp]
        L.mala_decode_multi.restype = i
        L.mala_decode_paged.argtypes = [_TIn, _TIn, _TIn, vp, vp, _TOut, vp, ctypes.POINTER(_Stats), i, i, i, i, i, i, i, i,
                                        f, f, i, vp, sz, vp]
        L.mala_decode_paged.restype = i
        L.mala_decode_fp8.argtypes = [_TIn, _TIn, _TIn, vp, vp, _TOut, vp, ctypes.POINTER(_Stats), i, i, i, i, i, f, f, i, vp,
                                      sz, vp]
        L.mala_decode_fp8.restype = i
        L.mala_decode_fp8_multi.argtypes = [_TIn, _TIn, _TIn, vp, vp, _TOut, vp, ctypes.POINTER(_Stats), i, i, i, i, i, i, f,
                                            f, i, vp, sz, vp]
        L.mala_decode_fp8_multi.restype = i
        L.mala_decode_fp8_paged.argtypes = [_TIn, _TIn, _TIn, vp, vp, vp, vp, _TOut, vp, ctypes.POINTER(_Stats),
                                            i, i, i, i, i, i, i, f, f, i, vp, sz, vp]
        L.mala_decode_fp8_paged.restype = i
        L.mala_decode_static.argtypes = [_TIn, _TIn, _TIn, _TOut, vp, i, i, i, i, i, f, f, i, vp]
        L.mala_decode_static.restype = i
        bp = ctypes.POINTER(_RelBias)
        L.mala_fwd_bias.argtypes = [_TIn, _TIn, _TIn, bp, _TOut, vp, ctypes.POINTER(_Stats), i, i, i, i, i, i, i, f, f, vp, sz, vp]
        L.mala_bwd_bias.argtypes = [_TIn, _TIn, _TIn, _TIn, _TIn, vp, bp, _TOut, _TOut, _TOut, vp, ctypes.c_int64,
                                    ctypes.POINTER(_Stats), i, i, i, i, i, i, i, f, f, vp, sz, vp]
        L.mala_fwd_varlen_bias.argtypes = [_TIn, _TIn, _TIn, vp, vp, bp, _TOut, vp, ctypes.POINTER(_Stats), i, i, i, i, i, i,
                                           i, i, i, f, f, vp, sz, vp]
        L.mala_bwd_varlen_bias.argtypes = [_TIn, _TIn, _TIn, _TIn, _TIn, vp, vp, vp, bp, _TOut, _TOut, _TOut, vp,
                                           ctypes.c_int64, ctypes.POINTER(_Stats), i, i, i, i, i, i, i, i, i, f, f, vp, sz, vp]
        L.mala_decode_paged_bias.argtypes = [_TIn, _TIn, _TIn, vp, vp, bp, _TOut, vp, ctypes.POINTER(_Stats), i, i, i, i, i, i,
                                             i, i, f, f, i, vp, sz, vp]
        L.mala_bias_workspace_bytes.argtypes = [i] * 11
        L.mala_bias_workspace_bytes.restype = sz
        for n in ("mala_fwd_bias", "mala_bwd_bias", "mala_fwd_varlen_bias", "mala_bwd_varlen_bias", "mala_decode_paged_bias"):
            getattr(L, n).restype = i
        L.mala_page_tables.argtypes = [vp] * 9 + [i] * 5 + [vp]
        L.mala_release_pages.argtypes = [vp] * 7 + [i] * 4 + [vp]
        L.mala_cache_write.argtypes = [_TIn, _TIn, vp, _TOut, _TOut, i, i, i, i, i, vp]
        L.mala_cache_write_fp8.argtypes = [_TIn, _TIn, vp, _TOut, _TOut, vp, vp, i, i, i, i, i, vp]
        for n in ("mala_page_tables", "mala_release_pages", "mala_cache_write", "mala_cache_write_fp8"):
            getattr(L, n).restype = i
        L.mala_page_tables_positions.argtypes = [vp] * 10 + [i] * 5 + [vp]
        L.mala_cache_read.argtypes = [_TIn, _TIn, vp, vp, _TOut, _TOut, vp] + [i] * 7 + [vp]
        L.mala_cache_read_fp8.argtypes = [_TIn, _TIn, vp, vp, vp, vp, _TOut, _TOut, vp] + [i] * 7 + [vp]
        L.mala_fwd_paged_fp8.argtypes = [_TIn, _TIn, _TIn, vp, vp, vp, vp, vp, _TOut, vp, ctypes.POINTER(_Stats)] + [i] * 11 + \
            [f, f, vp, sz, vp]
        L.mala_fwd_paged_fp8_split.argtypes = L.mala_fwd_paged_fp8.argtypes[:24] + [i] + L.mala_fwd_paged_fp8.argtypes[24:]
        L.mala_paged_fp8_workspace_bytes.argtypes = [i] * 4
        L.mala_paged_fp8_split_workspace_bytes.argtypes = [i] * 7
        L.mala_paged_fp8_suggest_splits.argtypes, L.mala_paged_fp8_suggest_splits.restype = [i] * 6, i
        rp, np_ = ctypes.POINTER(_Rotary), ctypes.POINTER(_HeadNorm)
        L.mala_rotary_fwd.argtypes = [_TIn, _TIn, vp, rp, np_, _TOut, _TOut] + [i] * 6 + [vp]
        L.mala_rotary_bwd.argtypes = [_TIn, _TIn, _TIn, _TIn, vp, rp, np_, _TOut, _TOut, vp, vp] + [i] * 6 + [vp, sz, vp]
        L.mala_rotary_fwd_varlen.argtypes = [_TIn, _TIn, vp, vp, rp, np_, _TOut, _TOut] + [i] * 6 + [vp]
        L.mala_rotary_bwd_varlen.argtypes = [_TIn, _TIn, _TIn, _TIn, vp, vp, rp, np_, _TOut, _TOut, vp, vp] + [i] * 6 + [vp, sz, vp]
        L.mala_rotary_write.argtypes = [_TIn, _TIn, _TIn, vp, vp, rp, np_, _TOut, _TOut, _TOut] + [i] * 6 + [vp]
        L.mala_rotary_write_fp8.argtypes = [_TIn, _TIn, _TIn, vp, vp, rp, np_, _TOut, _TOut, _TOut, vp, vp] + [i] * 6 + [vp]
        L.mala_rotary_workspace_bytes.argtypes = [i]
        for n in ("mala_paged_fp8_workspace_bytes", "mala_paged_fp8_split_workspace_bytes", "mala_rotary_workspace_bytes"):
            getattr(L, n).restype = sz
        for n in ("mala_page_tables_positions", "mala_cache_read", "mala_cache_read_fp8", "mala_fwd_paged_fp8", "mala_fwd_paged_fp8_split", "mala_rotary_fwd",
                  "mala_rotary_bwd", "mala_rotary_fwd_varlen", "mala_rotary_bwd_varlen", "mala_rotary_write", "mala_rotary_write_fp8"):
            getattr(L, n).restype = i
        L.mala_test_expire_wait.argtypes = [ctypes.c_longlong, vp]
        L.mala_test_expire_wait.restype = i
        L.mala_workspace_bytes.argtypes = [i, i, i, i, i, i, i]
        L.mala_workspace_bytes.restype = sz
        L.mala_tile_shape.argtypes = [i, i, ctypes.POINTER(i), ctypes.POINTER(i)]
        L.mala_decode_suggest_splits.argtypes = [i, i, i, i]
        L.mala_decode_suggest_splits.restype = i
        L.mala_device_status.argtypes = [ctypes.POINTER(i), i]
        L.mala_strerror.argtypes = [i]
        L.mala_strerror.restype = ctypes.c_char_p
        L.mala_version.restype = i
        for n in ("mala_fwd", "mala_bwd", "mala_decode", "mala_tile_shape", "mala_device_status"):
            getattr(L, n).restype = i
        _lib = L
    return _lib


_native_module = None


def _native():
    """The extension that marshals the rotary calls, the cache reads and prompts over an e4m3 cache (beside libmala.so; fails loudly if absent)."""
    global _native_module
    if _native_module is None:
        lib()                # (the library that it is linked with)
        try:
            from . import _native as module
        except ImportError as e:
            raise ImportError(f"{os.path.join(_HERE, '_native.so')}: run `python -m paper_2609_32712_b200.build` (needs g++)") from e
        _native_module = module
    return _native_module


def _done(r, what: str):
    """What a call of the extension gave: its outputs, or the code with which the library refused it."""
    if type(r) is int:
        raise MalaError(r, what)
    return r


# A decode step over a short cache takes about 10 us on the device, so what these helpers cost is what such a step waits
# for: strides read once, the stream's raw handle and new_empty took a step over 2000 keys from 24 to 16 us.
_BF16 = torch.bfloat16
_F32 = torch.float32


def _view(t: torch.Tensor, cls):
    s = t.stride()
    assert t.dtype is _BF16 and len(s) == 4 and s[3] == 1, "expects bf16 [B,N,H,d], last dim contiguous"
    return cls(t.data_ptr(), s[0], s[1], s[2])


# the current stream of the current device as a raw handle (torch.cuda.current_stream() builds a Stream object for it)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream() -> int:
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def tile_shape(op: int, d: int):
    bq, bk = ctypes.c_int(0), ctypes.c_int(0)
    rc = lib().mala_tile_shape(op, d, ctypes.byref(bq), ctypes.byref(bk))
    if rc != 0:
        raise MalaError(rc, "mala_tile_shape")
    return bq.value, bk.value


def decode_suggest_splits(B: int, Hkv: int, Nk: int, sm_count: int = 0) -> int:
    """mala_decode_suggest_splits: the smallest split count that still fills the SMs evenly."""
    rc = int(lib().mala_decode_suggest_splits(B, Hkv, Nk, sm_count))
    if rc < 0:
        raise MalaError(rc, "mala_decode_suggest_splits")
    return rc


def workspace_bytes(op: int, B: int, Hq: int, Hkv: int, N: int, d: int, num_splits: int = 0) -> int:
    return int(lib().mala_workspace_bytes(op, B, Hq, Hkv, N, d, num_splits))


def device_status(clear: bool = True) -> int:
    code = ctypes.c_int(0)
    rc = lib().mala_device_status(ctypes.byref(code), int(clear))
    if rc != 0:
        raise MalaError(rc, "mala_device_status")
    return code.value


def test_expire_wait(limit_cycles: int = 100000) -> None:
    """mala_test_expire_wait: makes one bounded device-side wait run out (test support)."""
    rc = lib().mala_test_expire_wait(limit_cycles, _stream())
    if rc != 0:
        raise MalaError(rc, "mala_test_expire_wait")


class Stats:
    """Device tensors for the optional telemetry of one call."""

    def __init__(self, retained_shape, words: int, device):
        self.retained = torch.zeros(retained_shape, dtype=torch.int32, device=device)
        self.bitmask = torch.zeros(tuple(retained_shape) + (words,), dtype=torch.int32, device=device)
        self.totals = torch.zeros(2, dtype=torch.int64, device=device)
        self.c = _Stats(self.retained.data_ptr(), self.bitmask.data_ptr(), self.totals.data_ptr())

    def mask(self, n_bits: int) -> torch.Tensor:
        """Boolean [..., n_bits] expansion of the bitmask (bit x of a row = tile x retained)."""
        w = self.bitmask.to(torch.int64) & 0xFFFFFFFF
        bits = (w.unsqueeze(-1) >> torch.arange(32, device=w.device)) & 1
        return bits.flatten(-2)[..., :n_bits].bool()


def _ws(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


def fwd(q, k, v, scale: float, tau: float, causal: bool = True, stats: bool = False, out=None, lse=None, ws=None):
    """mala_fwd: returns (o [B,N,Hq,d] bf16, lse [B,Hq,N] fp32, Stats or None)."""
    B, N, Hq, d = q.shape
    Hkv = k.shape[2]
    o = torch.empty_like(q) if out is None else out
    lse = q.new_empty((B, Hq, N), dtype=_F32) if lse is None else lse
    T = -(-N // 128)
    st = Stats((B, Hq, T), -(-T // 32), q.device) if stats else None
    ws = _ws(workspace_bytes(OP_FWD, B, Hq, Hkv, N, d), q.device) if ws is None else ws
    rc = lib().mala_fwd(_view(q, _TIn), _view(k, _TIn), _view(v, _TIn), _view(o, _TOut), lse.data_ptr(),
                        ctypes.byref(st.c) if st else None, B, Hq, Hkv, N, d, int(causal), scale, tau,
                        ws.data_ptr(), ws.numel(), _stream())
    if rc != 0:
        raise MalaError(rc, "mala_fwd")
    return o, lse, st


def bwd(q, k, v, o, do, lse, scale: float, tau: float, causal: bool = True, stats: bool = False, ws=None,
        dq=None, dk=None, dv=None):
    """mala_bwd: returns (dq, dk, dv, Stats or None)."""
    B, N, Hq, d = q.shape
    Hkv = k.shape[2]
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(v) if dv is None else dv
    T = -(-N // 128)
    st = Stats((B, Hq, T), -(-T // 32), q.device) if stats else None
    ws = _ws(workspace_bytes(OP_BWD, B, Hq, Hkv, N, d), q.device) if ws is None else ws
    rc = lib().mala_bwd(_view(q, _TIn), _view(k, _TIn), _view(v, _TIn), _view(o, _TIn), _view(do, _TIn),
                        lse.data_ptr(), _view(dq, _TOut), _view(dk, _TOut), _view(dv, _TOut),
                        ctypes.byref(st.c) if st else None, B, Hq, Hkv, N, d, int(causal), scale, tau,
                        ws.data_ptr(), ws.numel(), _stream())
    if rc != 0:
        raise MalaError(rc, "mala_bwd")
    return dq, dk, dv, st


def fwd_chunk(q, k, v, scale: float, tau: float, causal: bool = True, stats: bool = False, out=None, lse=None):
    """mala_fwd_chunk: q [B,Nq,Hq,d] against k, v [B,Nk,Hkv,d] (causal: the queries are the last Nq positions).
    Returns (o [B,Nq,Hq,d] bf16, lse [B,Hq,Nq] fp32, Stats or None); the telemetry's query blocks follow the key
    positions (block i = rows q with 128 i <= q + (Nk - Nq) % 128 < 128 (i + 1))."""
    B, Nq, Hq, d = q.shape
    Nk, Hkv = k.shape[1], k.shape[2]
    o = torch.empty_like(q) if out is None else out
    lse = q.new_empty((B, Hq, Nq), dtype=_F32) if lse is None else lse
    Tq, Tk = -(-(Nq + ((Nk - Nq) % 128 if causal else 0)) // 128), -(-Nk // 128)
    st = Stats((B, Hq, Tq), -(-Tk // 32), q.device) if stats else None
    rc = lib().mala_fwd_chunk(_view(q, _TIn), _view(k, _TIn), _view(v, _TIn), _view(o, _TOut), lse.data_ptr(),
                              ctypes.byref(st.c) if st else None, B, Hq, Hkv, Nq, Nk, d, int(causal), scale, tau,
                              None, 0, _stream())
    if rc != 0:
        raise MalaError(rc, "mala_fwd_chunk")
    return o, lse, st


def fwd_chunk_split(q, k, v, scale: float, tau: float, num_splits: int, causal: bool = True, stats: bool = False,
                    out=None, lse=None, ws=None):
    """mala_fwd_chunk_split: mala_fwd_chunk with the keys cut into num_splits ranges (split-local test, merged)."""
    B, Nq, Hq, d = q.shape
    Nk, Hkv = k.shape[1], k.shape[2]
    o = torch.empty_like(q) if out is None else out
    lse = q.new_empty((B, Hq, Nq), dtype=_F32) if lse is None else lse
    Tq, Tk = -(-(Nq + ((Nk - Nq) % 128 if causal else 0)) // 128), -(-Nk // 128)
    st = Stats((B, Hq, Tq), -(-Tk // 32), q.device) if stats else None
    ws = _ws(workspace_bytes(OP_FWD, B, Hq, Hkv, Nq, d, num_splits), q.device) if ws is None else ws
    rc = lib().mala_fwd_chunk_split(_view(q, _TIn), _view(k, _TIn), _view(v, _TIn), _view(o, _TOut), lse.data_ptr(),
                                    ctypes.byref(st.c) if st else None, B, Hq, Hkv, Nq, Nk, d, int(causal), scale, tau,
                                    num_splits, ws.data_ptr(), ws.numel(), _stream())
    if rc != 0:
        raise MalaError(rc, "mala_fwd_chunk_split")
    return o, lse, st


def bwd_chunk(q, k, v, o, do, lse, scale: float, tau: float, causal: bool = True, stats: bool = False, ws=None,
              dq=None, dk=None, dv=None):
    """mala_bwd_chunk: returns (dq [B,Nq,Hq,d], dk, dv [B,Nk,Hkv,d], Stats or None)."""
    B, Nq, Hq, d = q.shape
    Nk, Hkv = k.shape[1], k.shape[2]
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(v) if dv is None else dv
    shift = (Nk - Nq) % 128 if causal and Nk >= Nq else 0     # query blocks follow the positions
    Tq, Tk = -(-(Nq + shift) // 128), -(-Nk // 128)
    st = Stats((B, Hq, Tk), -(-Tq // 32), q.device) if stats else None
    ws = _ws(workspace_bytes(OP_BWD, B, Hq, Hkv, Nq + shift, d), q.device) if ws is None else ws
    rc = lib().mala_bwd_chunk(_view(q, _TIn), _view(k, _TIn), _view(v, _TIn), _view(o, _TIn), _view(do, _TIn),
                              lse.data_ptr(), _view(dq, _TOut), _view(dk, _TOut), _view(dv, _TOut),
                              ctypes.byref(st.c) if st else None, B, Hq, Hkv, Nq, Nk, d, int(causal), scale, tau,
                              ws.data_ptr(), ws.numel(), _stream())
    if rc != 0:
        raise MalaError(rc, "mala_bwd_chunk")
    return dq, dk, dv, st


def fwd_varlen(q, k, v, cu_seqlens, max_seqlen: int, scale: float, tau: float, causal: bool = True, stats: bool = False):
    """mala_fwd_varlen: q [1,total,Hq,d], k, v [1,total,Hkv,d] packed sequences; cu_seqlens int32 [B+1] on the device.
    Returns (o [1,total,Hq,d] bf16, lse [Hq,total] fp32, Stats or None)."""
    one, total, Hq, d = q.shape
    assert one == 1 and cu_seqlens.dtype == torch.int32 and cu_seqlens.is_contiguous()
    B, Hkv = cu_seqlens.numel() - 1, k.shape[2]
    o = torch.empty_like(q)
    lse = q.new_empty((Hq, total), dtype=_F32)
    T = -(-max_seqlen // 128)
    st = Stats((B, Hq, T), -(-T // 32), q.device) if stats else None
    rc = lib().mala_fwd_varlen(_view(q, _TIn), _view(k, _TIn), _view(v, _TIn), cu_seqlens.data_ptr(), _view(o, _TOut),
                               lse.data_ptr(), ctypes.byref(st.c) if st else None, B, Hq, Hkv, total, max_seqlen, d,
                               int(causal), scale, tau, None, 0, _stream())
    if rc != 0:
        raise MalaError(rc, "mala_fwd_varlen")
    return o, lse, st


def fwd_varlen_prefix(q, k, v, cu_seqlens_q, cu_seqlens_k, max_seqlen_q: int, max_seqlen_k: int, scale: float, tau: float,
                      causal: bool = True, stats: bool = False):
    """mala_fwd_varlen_prefix: packed q [1,total_q,Hq,d] against packed k, v [1,total_k,Hkv,d], every sequence with at
    least as many keys as queries.  Returns (o, lse [Hq,total_q], Stats or None)."""
    one, total_q, Hq, d = q.shape
    total_k, Hkv = k.shape[1], k.shape[2]
    B = cu_seqlens_q.numel() - 1
    o = torch.empty_like(q)
    lse = q.new_empty((Hq, total_q), dtype=_F32)
    Tq, Tk = -(-(max_seqlen_q + 127) // 128), -(-max_seqlen_k // 128)
    st = Stats((B, Hq, Tq), -(-Tk // 32), q.device) if stats else None
    rc = lib().mala_fwd_varlen_prefix(_view(q, _TIn), _view(k, _TIn), _view(v, _TIn), cu_seqlens_q.data_ptr(),
                                      cu_seqlens_k.data_ptr(), _view(o, _TOut), lse.data_ptr(),
                                      ctypes.byref(st.c) if st else None, B, Hq, Hkv, total_q, total_k, max_seqlen_q,
                                      max_seqlen_k, d, int(causal), scale, tau, None, 0, _stream())
    if rc != 0:
        raise MalaError(rc, "mala_fwd_varlen_prefix")
    return o, lse, st


def fwd_paged(q, kpages, vpages, cu_seqlens_q, block_table, seqlens_k, max_seqlen_q: int, scale: float, tau: float,
              causal: bool = True, stats: bool = False):
    """mala_fwd_paged: packed q [1,total_q,Hq,d] against keys / values in pages [num_pages, page_size, Hkv, d]
    (block_table int32 [B, max_pages], seqlens_k int32 [B]).  Returns (o, lse [Hq,total_q], Stats or None)."""
    one, total_q, Hq, d = q.shape
    num_pages, page_size, Hkv = kpages.shape[0], kpages.shape[1], kpages.shape[2]
    B, max_pages = block_table.shape
    o = torch.empty_like(q)
    lse = q.new_empty((Hq, total_q), dtype=_F32)
    Tq, Tk = -(-(max_seqlen_q + 127) // 128), -(-(max_pages * page_size) // 128)
    st = Stats((B, Hq, Tq), -(-Tk // 32), q.device) if stats else None
    rc = lib().mala_fwd_paged(_view(q, _TIn), _view(kpages, _TIn), _view(vpages, _TIn), cu_seqlens_q.data_ptr(),
                              block_table.data_ptr(), seqlens_k.data_ptr(), _view(o, _TOut), lse.data_ptr(),
                              ctypes.byref(st.c) if st else None, B, Hq, Hkv, total_q, max_seqlen_q, num_pages,
                              page_size, max_pages, d, int(causal), scale, tau, None, 0, _stream())
    if rc != 0:
        raise MalaError(rc, "mala_fwd_paged")
    return o, lse, st


def bwd_varlen(q, k, v, o, do, lse, cu_seqlens, max_seqlen: int, scale: float, tau: float, causal: bool = True,
               stats: bool = False, ws=None):
    """mala_bwd_varlen: returns (dq [1,total,Hq,d], dk, dv [1,total,Hkv,d], Stats or None)."""
    one, total, Hq, d = q.shape
    assert one == 1 and cu_seqlens.dtype == torch.int32 and cu_seqlens.is_contiguous()
    B, Hkv = cu_seqlens.numel() - 1, k.shape[2]
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    T = -(-max_seqlen // 128)
    st = Stats((B, Hq, T), -(-T // 32), q.device) if stats else None
    ws = _ws(workspace_bytes(OP_BWD, 1, Hq, Hkv, total + 128 * B, d), q.device) if ws is None else ws
    rc = lib().mala_bwd_varlen(_view(q, _TIn), _view(k, _TIn), _view(v, _TIn), _view(o, _TIn), _view(do, _TIn),
                               lse.data_ptr(), cu_seqlens.data_ptr(), _view(dq, _TOut), _view(dk, _TOut),
                               _view(dv, _TOut), ctypes.byref(st.c) if st else None, B, Hq, Hkv, total, max_seqlen, d,
                               int(causal), scale, tau, ws.data_ptr(), ws.numel(), _stream())
    if rc != 0:
        raise MalaError(rc, "mala_bwd_varlen")
    return dq, dk, dv, st


def bwd_varlen_prefix(q, k, v, o, do, lse, cu_seqlens_q, cu_seqlens_k, max_seqlen_q: int, max_seqlen_k: int,
                      scale: float, tau: float, causal: bool = True, stats: bool = False, ws=None):
    """mala_bwd_varlen_prefix: returns (dq [1,total_q,Hq,d], dk, dv [1,total_k,Hkv,d], Stats or None)."""
    one, total_q, Hq, d = q.shape
    total_k, Hkv = k.shape[1], k.shape[2]
    for cu in (cu_seqlens_q, cu_seqlens_k):
        assert cu.dtype == torch.int32 and cu.is_contiguous()
    B = cu_seqlens_q.numel() - 1
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    Tq, Tk = -(-(max_seqlen_q + 127) // 128), -(-max_seqlen_k // 128)
    st = Stats((B, Hq, Tk), -(-Tq // 32), q.device) if stats else None
    ws = _ws(workspace_bytes(OP_BWD, 1, Hq, Hkv, total_q + 384 * B, d), q.device) if ws is None else ws
    rc = lib().mala_bwd_varlen_prefix(_view(q, _TIn), _view(k, _TIn), _view(v, _TIn), _view(o, _TIn), _view(do, _TIn),
                                      lse.data_ptr(), cu_seqlens_q.data_ptr(), cu_seqlens_k.data_ptr(),
                                      _view(dq, _TOut), _view(dk, _TOut), _view(dv, _TOut),
                                      ctypes.byref(st.c) if st else None, B, Hq, Hkv, total_q, total_k, max_seqlen_q,
                                      max_seqlen_k, d, int(causal), scale, tau, ws.data_ptr(), ws.numel(), _stream())
    if rc != 0:
        raise MalaError(rc, "mala_bwd_varlen_prefix")
    return dq, dk, dv, st


def decode(q, kcache, vcache, scale: float, tau: float, num_splits: int, stats: bool = False, ws=None, out=None,
           want_lse: bool = True):
    """mala_decode: q [B,1,Hq,d]; returns (o [B,1,Hq,d] bf16, lse [B,Hq] fp32 or None, Stats or None)."""
    B, one, Hq, d = q.shape
    assert one == 1
    Nk, Hkv = kcache.shape[1], kcache.shape[2]
    o = torch.empty_like(q) if out is None else out
    lse = q.new_empty((B, Hq), dtype=_F32) if want_lse else None
    tps = -(-(-(-Nk // num_splits)) // 128)
    st = Stats((B, Hkv, num_splits), -(-tps // 32), q.device) if stats else None
    ws = _ws(workspace_bytes(OP_DECODE, B, Hq, Hkv, Nk, d, num_splits), q.device) if ws is None else ws
    rc = lib().mala_decode(_view(q, _TIn), _view(kcache, _TIn), _view(vcache, _TIn), _view(o, _TOut),
                           lse.data_ptr() if lse is not None else None, ctypes.byref(st.c) if st else None,
                           B, Hq, Hkv, Nk, d, scale, tau, num_splits, ws.data_ptr(), ws.numel(), _stream())
    if rc != 0:
        raise MalaError(rc, "mala_decode")
    return o, lse, st


def _view8(t: torch.Tensor):
    s = t.stride()
    assert t.dtype in (torch.uint8, torch.float8_e4m3fn) and len(s) == 4 and s[3] == 1, \
        "expects 8-bit [B,N,H,d], last dim contiguous"
    return _TIn(t.data_ptr(), s[0], s[1], s[2])


def decode_fp8(q, kcache8, vcache8, kscale, vscale, scale: float, tau: float, num_splits: int, stats: bool = False,
               ws=None, out=None, want_lse: bool = True):
    """mala_decode_fp8: q [B,1,Hq,d] bf16; kcache8, vcache8 e4m3 codes [B,Nk,Hkv,d] (uint8 or float8_e4m3fn);
    kscale, vscale fp32 [B,Hkv,ceil(Nk/128)].  Returns (o [B,1,Hq,d] bf16, lse [B,Hq] fp32 or None, Stats or None)."""
    B, one, Hq, d = q.shape
    assert one == 1
    Nk, Hkv = kcache8.shape[1], kcache8.shape[2]
    assert kscale.dtype == torch.float32 and kscale.is_contiguous() and tuple(kscale.shape) == (B, Hkv, -(-Nk // 128))
    assert vscale.dtype == torch.float32 and vscale.is_contiguous() and tuple(vscale.shape) == (B, Hkv, -(-Nk // 128))
    o = torch.empty_like(q) if out is None else out
    lse = q.new_empty((B, Hq), dtype=_F32) if want_lse else None
    tps = -(-(-(-Nk // num_splits)) // 128)
    st = Stats((B, Hkv, num_splits), -(-tps // 32), q.device) if stats else None
    ws = _ws(workspace_bytes(OP_DECODE, B, Hq, Hkv, Nk, 128, num_splits), q.device) if ws is None else ws
    rc = lib().mala_decode_fp8(_view(q, _TIn), _view8(kcache8), _view8(vcache8), kscale.data_ptr(), vscale.data_ptr(),
                               _view(o, _TOut), lse.data_ptr() if lse is not None else None,
                               ctypes.byref(st.c) if st else None, B, Hq, Hkv, Nk, d, scale, tau, num_splits,
                               ws.data_ptr(), ws.numel(), _stream())
    if rc != 0:
        raise MalaError(rc, "mala_decode_fp8")
    return o, lse, st


def decode_fp8_multi(q, kcache8, vcache8, kscale, vscale, scale: float, tau: float, num_splits: int, stats: bool = False,
                     ws=None, out=None, want_lse: bool = True):
    """mala_decode_fp8_multi: q [B,Sq,Hq,d] bf16, the Sq new tokens of each sequence (their keys / values are the last
    Sq positions of the caches); caches and scales as for decode_fp8.  Returns (o [B,Sq,Hq,d] bf16, lse [B,Sq,Hq]
    fp32 or None, Stats or None)."""
    B, Sq, Hq, d = q.shape
    Nk, Hkv = kcache8.shape[1], kcache8.shape[2]
    assert kscale.dtype == torch.float32 and kscale.is_contiguous() and tuple(kscale.shape) == (B, Hkv, -(-Nk // 128))
    assert vscale.dtype == torch.float32 and vscale.is_contiguous() and tuple(vscale.shape) == (B, Hkv, -(-Nk // 128))
    o = torch.empty_like(q) if out is None else out
    lse = q.new_empty((B, Sq, Hq), dtype=_F32) if want_lse else None
    tps = -(-(-(-Nk // num_splits)) // 128)
    st = Stats((B, Hkv, num_splits), -(-tps // 32), q.device) if stats else None
    ws = _ws(workspace_bytes(OP_DECODE, B * Sq, Hq, Hkv, Nk, 128, num_splits), q.device) if ws is None else ws
    rc = lib().mala_decode_fp8_multi(_view(q, _TIn), _view8(kcache8), _view8(vcache8), kscale.data_ptr(), vscale.data_ptr(),
                                     _view(o, _TOut), lse.data_ptr() if lse is not None else None,
                                     ctypes.byref(st.c) if st else None, B, Hq, Hkv, Nk, Sq, d, scale, tau, num_splits,
                                     ws.data_ptr(), ws.numel(), _stream())
    if rc != 0:
        raise MalaError(rc, "mala_decode_fp8_multi")
    return o, lse, st


def decode_fp8_paged(q, kpages8, vpages8, kscale, vscale, block_table, seqlens, scale: float, tau: float, num_splits: int,
                     stats: bool = False, ws=None, out=None, want_lse: bool = True):
    """mala_decode_fp8_paged: q [B,1,Hq,d] bf16; kpages8, vpages8 e4m3 codes [num_pages, page_size, Hkv, d];
    kscale, vscale fp32 [num_pages, Hkv, max(1, page_size/128)]; block_table int32 [B, max_pages_per_seq]; seqlens int32 [B] or
    None.  Returns (o [B,1,Hq,d] bf16, lse [B,Hq] fp32 or None, Stats or None)."""
    B, one, Hq, d = q.shape
    assert one == 1
    num_pages, page_size, Hkv = kpages8.shape[0], kpages8.shape[1], kpages8.shape[2]
    assert block_table.dtype == torch.int32 and block_table.is_contiguous() and block_table.shape[0] == B
    assert seqlens is None or (seqlens.dtype == torch.int32 and seqlens.is_contiguous() and seqlens.shape == (B,))
    for t in (kscale, vscale):
        assert t.dtype == torch.float32 and t.is_contiguous() and tuple(t.shape) == (num_pages, Hkv, max(1, page_size // 128))
    max_pages = block_table.shape[1]
    Nk = max_pages * page_size
    o = torch.empty_like(q) if out is None else out
    lse = q.new_empty((B, Hq), dtype=_F32) if want_lse else None
    tps = -(-(-(-Nk // num_splits)) // 128)
    st = Stats((B, Hkv, num_splits), -(-tps // 32), q.device) if stats else None
    ws = _ws(workspace_bytes(OP_DECODE, B, Hq, Hkv, Nk, 128, num_splits), q.device) if ws is None else ws
    rc = lib().mala_decode_fp8_paged(_view(q, _TIn), _view8(kpages8), _view8(vpages8), kscale.data_ptr(),
                                     vscale.data_ptr(), block_table.data_ptr(),
                                     seqlens.data_ptr() if seqlens is not None else None, _view(o, _TOut),
                                     lse.data_ptr() if lse is not None else None, ctypes.byref(st.c) if st else None,
                                     B, Hq, Hkv, num_pages, page_size, max_pages, d, scale, tau, num_splits,
                                     ws.data_ptr(), ws.numel(), _stream())
    if rc != 0:
        raise MalaError(rc, "mala_decode_fp8_paged")
    return o, lse, st


def decode_multi(q, kcache, vcache, scale: float, tau: float, num_splits: int, stats: bool = False, ws=None, out=None,
                 want_lse: bool = True):
    """mala_decode_multi: q [B,Sq,Hq,d], the Sq new tokens of each sequence (their keys / values are the last Sq
    positions of the caches).  Returns (o [B,Sq,Hq,d] bf16, lse [B,Sq,Hq] fp32 or None, Stats or None)."""
    B, Sq, Hq, d = q.shape
    Nk, Hkv = kcache.shape[1], kcache.shape[2]
    o = torch.empty_like(q) if out is None else out
    lse = q.new_empty((B, Sq, Hq), dtype=_F32) if want_lse else None
    tps = -(-(-(-Nk // num_splits)) // 128)
    st = Stats((B, Hkv, num_splits), -(-tps // 32), q.device) if stats else None
    ws = _ws(workspace_bytes(OP_DECODE, B * Sq, Hq, Hkv, Nk, d, num_splits), q.device) if ws is None else ws
    rc = lib().mala_decode_multi(_view(q, _TIn), _view(kcache, _TIn), _view(vcache, _TIn), _view(o, _TOut),
                                 lse.data_ptr() if lse is not None else None, ctypes.byref(st.c) if st else None,
                                 B, Hq, Hkv, Nk, Sq, d, scale, tau, num_splits, ws.data_ptr(), ws.numel(), _stream())
    if rc != 0:
        raise MalaError(rc, "mala_decode_multi")
    return o, lse, st


def decode_paged(q, kpages, vpages, block_table, seqlens, scale: float, tau: float, num_splits: int,
                 stats: bool = False, ws=None, out=None, want_lse: bool = True):
    """mala_decode_paged: q [B,Sq,Hq,d] (Sq new tokens per sequence); kpages, vpages [num_pages, page_size, Hkv, d];
    block_table int32 [B, max_pages_per_seq]; seqlens int32 [B] or None.
    Returns (o [B,Sq,Hq,d], lse [B,Hq] (Sq = 1) or [B,Sq,Hq] or None, Stats or None)."""
    B, Sq, Hq, d = q.shape
    num_pages, page_size, Hkv = kpages.shape[0], kpages.shape[1], kpages.shape[2]
    assert block_table.dtype == torch.int32 and block_table.is_contiguous() and block_table.shape[0] == B
    assert seqlens is None or (seqlens.dtype == torch.int32 and seqlens.is_contiguous() and seqlens.shape == (B,))
    max_pages = block_table.shape[1]
    Nk = max_pages * page_size
    o = torch.empty_like(q) if out is None else out
    lse = q.new_empty((B, Hq) if Sq == 1 else (B, Sq, Hq), dtype=_F32) if want_lse else None
    tps = -(-(-(-Nk // num_splits)) // 128)
    st = Stats((B, Hkv, num_splits), -(-tps // 32), q.device) if stats else None
    ws = _ws(workspace_bytes(OP_DECODE, B * Sq, Hq, Hkv, Nk, d, num_splits), q.device) if ws is None else ws
    rc = lib().mala_decode_paged(_view(q, _TIn), _view(kpages, _TIn), _view(vpages, _TIn), block_table.data_ptr(),
                                 seqlens.data_ptr() if seqlens is not None else None, _view(o, _TOut),
                                 lse.data_ptr() if lse is not None else None, ctypes.byref(st.c) if st else None,
                                 B, Hq, Hkv, num_pages, page_size, max_pages, Sq, d, scale, tau, num_splits,
                                 ws.data_ptr(), ws.numel(), _stream())
    if rc != 0:
        raise MalaError(rc, "mala_decode_paged")
    return o, lse, st


STATIC_SCRATCH_BYTES = 24 << 20


def decode_static(q, kcache, vcache, scale: float, tau: float, num_splits: int, out=None, want_lse: bool = True):
    """mala_decode_static: decode without any caller-provided scratch.

    For callers that cannot allocate device memory at the point of the call (a fixed memory plan, a plug-in
    that only receives its inputs and outputs, a path that must not touch the allocator).  The split partials
    live in a 24 MiB array inside the library image; calls on one device must not overlap on the GPU.  Only
    the output tensors are created here when the caller does not pass them.
    Returns (o [B,1,Hq,d] bf16, lse [B,Hq] fp32 or None)."""
    B, one, Hq, d = q.shape
    assert one == 1
    Nk, Hkv = kcache.shape[1], kcache.shape[2]
    o = torch.empty_like(q) if out is None else out
    lse = q.new_empty((B, Hq), dtype=_F32) if want_lse else None
    rc = lib().mala_decode_static(_view(q, _TIn), _view(kcache, _TIn), _view(vcache, _TIn), _view(o, _TOut),
                                  lse.data_ptr() if lse is not None else None, B, Hq, Hkv, Nk, d, scale, tau,
                                  num_splits, _stream())
    if rc != 0:
        raise MalaError(rc, "mala_decode_static")
    return o, lse


class RelativeBias:
    """A learned relative position bias: ``table`` bf16 [num_buckets, Hq] (heads contiguous), the bias of a score being
    ``table[bucket(key position - query position)][head]`` with the buckets of ``include/mala.h``."""

    def __init__(self, table: torch.Tensor, max_distance: int = 128, bidirectional: bool = False):
        assert table.dtype is _BF16 and table.dim() == 2 and (table.stride(1) == 1 or table.shape[1] == 1), \
            "expects a bf16 table [num_buckets, Hq], heads contiguous"
        self.table, self.max_distance, self.bidirectional = table, int(max_distance), bool(bidirectional)
        self.num_buckets, self.heads = table.shape
        self.c = _RelBias(table.data_ptr(), table.stride(0), self.num_buckets, self.max_distance, int(self.bidirectional))

    def _for(self, q):
        assert self.heads == q.shape[2] and self.table.device == q.device, "the table has a column per query head of q"
        self.c.table, self.c.sb = self.table.data_ptr(), self.table.stride(0)   # (a parameter's storage may have been replaced)
        return ctypes.byref(self.c)


def _here(*ts) -> int:
    """The current stream of the current device, on which all of ts have to lie (a kernel given another one's memory faults)."""
    dev = torch.cuda.current_device()
    for t in ts:
        assert t is None or t.get_device() == dev, "expects tensors on the current device"
    return torch.cuda.current_stream().cuda_stream if _raw_stream is None else _raw_stream(dev)


def bias_workspace_bytes(op: int, B: int, Hq: int, Hkv: int, Nq: int, Nk: int, d: int, bias: RelativeBias, total_q: int = 0,
                         num_splits: int = 0) -> int:
    return _bias_workspace_bytes(op, B, Hq, Hkv, Nq, Nk, total_q, d, num_splits, bias.num_buckets, bias.max_distance)


@functools.lru_cache(256)     # (a pure function of its arguments; the call into the library takes 1.4 us of a step's 25)
def _bias_workspace_bytes(*args) -> int:
    return int(lib().mala_bias_workspace_bytes(*args))


def fwd_bias(q, k, v, bias: RelativeBias, scale: float, tau: float, causal: bool = True, stats: bool = False, out=None,
             lse=None, ws=None):
    """mala_fwd_bias: fwd_chunk with a relative position bias.  q [B,Nq,Hq,d], k, v [B,Nk,Hkv,d]; the queries are the last Nq of
    the Nk positions.  Returns (o [B,Nq,Hq,d] bf16, lse [B,Hq,Nq] fp32, Stats or None)."""
    B, Nq, Hq, d = q.shape
    Nk, Hkv = k.shape[1], k.shape[2]
    assert k.shape == v.shape == (B, Nk, Hkv, d)
    o = torch.empty_like(q) if out is None else out
    lse = q.new_empty((B, Hq, Nq), dtype=_F32) if lse is None else lse
    Tq, Tk = -(-(Nq + ((Nk - Nq) % 128 if causal else 0)) // 128), -(-Nk // 128)
    assert o.shape == q.shape and lse.dtype is _F32 and lse.shape == (B, Hq, Nq) and lse.is_contiguous()
    st = Stats((B, Hq, Tq), -(-Tk // 32), q.device) if stats else None
    ws = _ws(bias_workspace_bytes(OP_FWD, B, Hq, Hkv, Nq, Nk, d, bias), q.device) if ws is None else ws
    rc = lib().mala_fwd_bias(_view(q, _TIn), _view(k, _TIn), _view(v, _TIn), bias._for(q), _view(o, _TOut), lse.data_ptr(),
                             ctypes.byref(st.c) if st else None, B, Hq, Hkv, Nq, Nk, d, int(causal), scale, tau,
                             ws.data_ptr(), ws.numel(), _here(q, k, v, o, lse, ws))
    if rc != 0:
        raise MalaError(rc, "mala_fwd_bias")
    return o, lse, st


def bwd_bias(q, k, v, o, do, lse, bias: RelativeBias, scale: float, tau: float, causal: bool = True, stats: bool = False,
             ws=None, dq=None, dk=None, dv=None):
    """mala_bwd_bias: returns (dq, dk, dv, dtable bf16 [num_buckets, Hq], Stats or None)."""
    B, Nq, Hq, d = q.shape
    Nk, Hkv = k.shape[1], k.shape[2]
    assert k.shape == v.shape == (B, Nk, Hkv, d) and q.shape == o.shape == do.shape
    assert lse.dtype is _F32 and lse.shape == (B, Hq, Nq) and lse.is_contiguous()
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(v) if dv is None else dv
    dtable = q.new_empty((bias.num_buckets, Hq))
    assert dq.shape == q.shape and dk.shape == dv.shape == k.shape
    Tq, Tk = -(-(Nq + ((Nk - Nq) % 128 if causal and Nk >= Nq else 0)) // 128), -(-Nk // 128)
    st = Stats((B, Hq, Tk), -(-Tq // 32), q.device) if stats else None
    ws = _ws(bias_workspace_bytes(OP_BWD, B, Hq, Hkv, Nq, Nk, d, bias), q.device) if ws is None else ws
    rc = lib().mala_bwd_bias(_view(q, _TIn), _view(k, _TIn), _view(v, _TIn), _view(o, _TIn), _view(do, _TIn), lse.data_ptr(),
                             bias._for(q), _view(dq, _TOut), _view(dk, _TOut), _view(dv, _TOut), dtable.data_ptr(), Hq,
                             ctypes.byref(st.c) if st else None, B, Hq, Hkv, Nq, Nk, d, int(causal), scale, tau,
                             ws.data_ptr(), ws.numel(), _here(q, k, v, o, do, lse, dq, dk, dv, ws))
    if rc != 0:
        raise MalaError(rc, "mala_bwd_bias")
    return dq, dk, dv, dtable, st


def fwd_varlen_bias(q, k, v, cu_seqlens_q, cu_seqlens_k, max_seqlen_q: int, max_seqlen_k: int, bias: RelativeBias,
                    scale: float, tau: float, causal: bool = True, stats: bool = False, ws=None):
    """mala_fwd_varlen_bias: packed q [1,total_q,Hq,d] against packed k, v [1,total_k,Hkv,d] (offsets int32 [B+1] on the
    device; the same tensor twice for self attention).  Returns (o, lse [Hq,total_q], Stats or None)."""
    one, total_q, Hq, d = q.shape
    total_k, Hkv = k.shape[1], k.shape[2]
    assert k.shape == v.shape == (1, total_k, Hkv, d)
    for cu in (cu_seqlens_q, cu_seqlens_k):
        assert one == 1 and cu.dtype == torch.int32 and cu.is_contiguous()
    B = cu_seqlens_q.numel() - 1
    assert cu_seqlens_k.numel() == B + 1
    o = torch.empty_like(q)
    lse = q.new_empty((Hq, total_q), dtype=_F32)
    Tq, Tk = -(-(max_seqlen_q + 127) // 128), -(-max_seqlen_k // 128)
    st = Stats((B, Hq, Tq), -(-Tk // 32), q.device) if stats else None
    ws = _ws(bias_workspace_bytes(OP_FWD, B, Hq, Hkv, max_seqlen_q, max_seqlen_k, d, bias), q.device) if ws is None else ws
    rc = lib().mala_fwd_varlen_bias(_view(q, _TIn), _view(k, _TIn), _view(v, _TIn), cu_seqlens_q.data_ptr(),
                                    cu_seqlens_k.data_ptr(), bias._for(q), _view(o, _TOut), lse.data_ptr(),
                                    ctypes.byref(st.c) if st else None, B, Hq, Hkv, total_q, total_k, max_seqlen_q,
                                    max_seqlen_k, d, int(causal), scale, tau, ws.data_ptr(), ws.numel(),
                                    _here(q, k, v, cu_seqlens_q, cu_seqlens_k, ws))
    if rc != 0:
        raise MalaError(rc, "mala_fwd_varlen_bias")
    return o, lse, st


def bwd_varlen_bias(q, k, v, o, do, lse, cu_seqlens_q, cu_seqlens_k, max_seqlen_q: int, max_seqlen_k: int, bias: RelativeBias,
                    scale: float, tau: float, causal: bool = True, stats: bool = False, ws=None):
    """mala_bwd_varlen_bias: returns (dq [1,total_q,Hq,d], dk, dv [1,total_k,Hkv,d], dtable bf16 [num_buckets, Hq], Stats or
    None)."""
    one, total_q, Hq, d = q.shape
    total_k, Hkv = k.shape[1], k.shape[2]
    assert k.shape == v.shape == (1, total_k, Hkv, d) and q.shape == o.shape == do.shape
    assert lse.dtype is _F32 and lse.shape == (Hq, total_q) and lse.is_contiguous()
    for cu in (cu_seqlens_q, cu_seqlens_k):
        assert one == 1 and cu.dtype == torch.int32 and cu.is_contiguous()
    B = cu_seqlens_q.numel() - 1
    assert cu_seqlens_k.numel() == B + 1
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    dtable = q.new_empty((bias.num_buckets, Hq))
    Tq, Tk = -(-(max_seqlen_q + 127) // 128), -(-max_seqlen_k // 128)
    st = Stats((B, Hq, Tk), -(-Tq // 32), q.device) if stats else None
    ws = _ws(bias_workspace_bytes(OP_BWD, B, Hq, Hkv, max_seqlen_q, max_seqlen_k, d, bias, total_q), q.device) if ws is None else ws
    rc = lib().mala_bwd_varlen_bias(_view(q, _TIn), _view(k, _TIn), _view(v, _TIn), _view(o, _TIn), _view(do, _TIn),
                                    lse.data_ptr(), cu_seqlens_q.data_ptr(), cu_seqlens_k.data_ptr(), bias._for(q),
                                    _view(dq, _TOut), _view(dk, _TOut), _view(dv, _TOut), dtable.data_ptr(), Hq,
                                    ctypes.byref(st.c) if st else None, B, Hq, Hkv, total_q, total_k, max_seqlen_q,
                                    max_seqlen_k, d, int(causal), scale, tau, ws.data_ptr(), ws.numel(),
                                    _here(q, k, v, o, do, lse, cu_seqlens_q, cu_seqlens_k, ws))
    if rc != 0:
        raise MalaError(rc, "mala_bwd_varlen_bias")
    return dq, dk, dv, dtable, st


def decode_paged_bias(q, kpages, vpages, block_table, seqlens, bias: RelativeBias, scale: float, tau: float, num_splits: int,
                      stats: bool = False, ws=None, out=None, want_lse: bool = True):
    """mala_decode_paged_bias: decode_paged with a relative position bias (a token's position is that of its own key)."""
    B, Sq, Hq, d = q.shape
    num_pages, page_size, Hkv = kpages.shape[0], kpages.shape[1], kpages.shape[2]
    assert block_table.dtype == torch.int32 and block_table.is_contiguous() and block_table.shape[0] == B
    assert seqlens is None or (seqlens.dtype == torch.int32 and seqlens.is_contiguous() and seqlens.shape == (B,))
    assert kpages.shape == vpages.shape and kpages.shape[3] == d
    max_pages = block_table.shape[1]
    Nk = max_pages * page_size
    o = torch.empty_like(q) if out is None else out
    assert o.shape == q.shape
    lse = q.new_empty((B, Hq) if Sq == 1 else (B, Sq, Hq), dtype=_F32) if want_lse else None
    tps = -(-(-(-Nk // num_splits)) // 128)
    st = Stats((B, Hkv, num_splits), -(-tps // 32), q.device) if stats else None
    if ws is None:
        ws = _ws(bias_workspace_bytes(OP_DECODE, B, Hq, Hkv, Sq, Nk, d, bias, num_splits=num_splits), q.device)
    rc = lib().mala_decode_paged_bias(_view(q, _TIn), _view(kpages, _TIn), _view(vpages, _TIn), block_table.data_ptr(),
                                      seqlens.data_ptr() if seqlens is not None else None, bias._for(q), _view(o, _TOut),
                                      lse.data_ptr() if lse is not None else None, ctypes.byref(st.c) if st else None,
                                      B, Hq, Hkv, num_pages, page_size, max_pages, Sq, d, scale, tau, num_splits,
                                      ws.data_ptr(), ws.numel(), _here(q, kpages, vpages, block_table, seqlens, o, ws))
    if rc != 0:
        raise MalaError(rc, "mala_decode_paged_bias")
    return o, lse, st


def _ints(*ts):
    for t in ts:
        assert t.dtype is torch.int32 and t.is_contiguous(), "expects contiguous int32 tensors"


def page_tables(seqlens, new_tokens, block_table, free_pages, free_count, page_size: int, rows: int, positions: bool = False):
    """mala_page_tables: pages for the new tokens of a serving step.  seqlens, new_tokens int32 [B]; block_table int32
    [B, max_pages_per_seq] (its new entries are written); free_pages int32 [num_pages], free_count int32 [1]; rows: how many
    slots to write (at least the sum of new_tokens for all of them).  Returns (cu_seqlens int32 [B+1], seqlens int32 [B],
    slots int64 [rows], free_count int32 [1]), and with positions the new tokens' positions int32 [rows] behind them."""
    _ints(seqlens, new_tokens, block_table, free_pages, free_count)
    B, max_pages = block_table.shape
    assert seqlens.shape == (B,) and new_tokens.shape == (B,) and free_count.shape == (1,)
    cu, lens, left = seqlens.new_empty(B + 1), seqlens.new_empty(B), seqlens.new_empty(1)
    slots = seqlens.new_empty(rows, dtype=torch.int64)
    if positions:
        pos = seqlens.new_empty(rows)
        rc = lib().mala_page_tables_positions(seqlens.data_ptr(), new_tokens.data_ptr(), block_table.data_ptr(), free_pages.data_ptr(),
                                              free_count.data_ptr(), cu.data_ptr(), lens.data_ptr(), slots.data_ptr(),
                                              pos.data_ptr(), left.data_ptr(), B, max_pages, page_size, free_pages.numel(), rows,
                                              _here(seqlens, new_tokens, block_table, free_pages, free_count))
        if rc != 0:
            raise MalaError(rc, "mala_page_tables_positions")
        return cu, lens, slots, left, pos
    rc = lib().mala_page_tables(seqlens.data_ptr(), new_tokens.data_ptr(), block_table.data_ptr(), free_pages.data_ptr(),
                                free_count.data_ptr(), cu.data_ptr(), lens.data_ptr(), slots.data_ptr(), left.data_ptr(), B,
                                max_pages, page_size, free_pages.numel(), rows,
                                _here(seqlens, new_tokens, block_table, free_pages, free_count))
    if rc != 0:
        raise MalaError(rc, "mala_page_tables")
    return cu, lens, slots, left


def release_pages(done, seqlens, block_table, free_pages, free_count, page_size: int):
    """mala_release_pages: the pages of the requests with done[b] (bool or uint8 [B]) go back to free_pages (written in
    place).  Returns (seqlens int32 [B], free_count int32 [1])."""
    _ints(seqlens, block_table, free_pages, free_count)
    B, max_pages = block_table.shape
    assert seqlens.shape == (B,) and free_count.shape == (1,) and done.shape == (B,)
    assert done.element_size() == 1 and done.is_contiguous()
    lens, left = seqlens.new_empty(B), seqlens.new_empty(1)
    rc = lib().mala_release_pages(done.data_ptr(), seqlens.data_ptr(), block_table.data_ptr(), free_pages.data_ptr(),
                                  free_count.data_ptr(), lens.data_ptr(), left.data_ptr(), B, max_pages, page_size,
                                  free_pages.numel(), _here(done, seqlens, block_table, free_pages, free_count))
    if rc != 0:
        raise MalaError(rc, "mala_release_pages")
    return lens, left


def _rows(t: torch.Tensor):
    s = t.stride()
    assert t.dtype is _BF16 and len(s) == 3 and s[2] == 1, "expects bf16 [rows,Hkv,d], last dim contiguous"
    return _TIn(t.data_ptr(), 0, s[0], s[1])


def cache_write(k, v, slots, kpages, vpages) -> None:
    """mala_cache_write: rows of k, v [rows,Hkv,d] to their slots (int64 [rows], negative: nowhere) of the bf16 pages
    [num_pages, page_size, Hkv, d]."""
    rows, Hkv, d = k.shape
    assert slots.dtype is torch.int64 and slots.is_contiguous() and slots.shape == (rows,) and v.shape == k.shape
    num_pages, page_size = kpages.shape[0], kpages.shape[1]
    assert kpages.shape == vpages.shape and kpages.shape[2:] == (Hkv, d)
    rc = lib().mala_cache_write(_rows(k), _rows(v), slots.data_ptr(), _view(kpages, _TOut), _view(vpages, _TOut), rows, Hkv,
                                num_pages, page_size, d, _here(k, v, slots, kpages, vpages))
    if rc != 0:
        raise MalaError(rc, "mala_cache_write")


def cache_write_fp8(k, v, slots, kpages8, vpages8, kscale, vscale) -> None:
    """mala_cache_write_fp8: the same into e4m3 pages (uint8 or float8_e4m3fn) with their scales, fp32
    [num_pages, Hkv, max(1, page_size/128)]."""
    rows, Hkv, d = k.shape
    assert slots.dtype is torch.int64 and slots.is_contiguous() and slots.shape == (rows,) and v.shape == k.shape
    num_pages, page_size = kpages8.shape[0], kpages8.shape[1]
    assert kpages8.shape == vpages8.shape and kpages8.shape[2:] == (Hkv, d)
    for t in (kscale, vscale):
        assert t.dtype is _F32 and t.is_contiguous() and tuple(t.shape) == (num_pages, Hkv, max(1, page_size // 128))
    kp, vp = _view8(kpages8), _view8(vpages8)
    rc = lib().mala_cache_write_fp8(_rows(k), _rows(v), slots.data_ptr(), _TOut(kp.p, kp.sb, kp.sn, kp.sh),
                                    _TOut(vp.p, vp.sb, vp.sn, vp.sh), kscale.data_ptr(), vscale.data_ptr(), rows, Hkv, num_pages,
                                    page_size, d, _here(k, v, slots, kpages8, vpages8, kscale, vscale))
    if rc != 0:
        raise MalaError(rc, "mala_cache_write_fp8")


def cache_read(kpages, vpages, block_table, seqlens, rows: int):
    """mala_cache_read: keys and values of the requests of block_table int32 [B, max_pages_per_seq] with seqlens int32 [B] tokens
    out of bf16 pages [num_pages, page_size, Hkv, d], packed.  rows: how many rows to make room for (at least the sum of the lengths for all
    of them).  Returns (k, v [1,rows,Hkv,d] bf16, cu_seqlens int32 [B+1]), as ``fwd_varlen_prefix`` takes them."""
    return _done(_native().cache_read(kpages, vpages, None, None, block_table, seqlens, rows), "mala_cache_read")


def cache_read_fp8(kpages8, vpages8, kscale, vscale, block_table, seqlens, rows: int):
    """mala_cache_read_fp8: the same out of e4m3 pages (uint8 or float8_e4m3fn) with their scales fp32
    [num_pages, Hkv, max(1, page_size/128)]."""
    assert kscale is not None and vscale is not None, "expects scales of keys and of values"
    return _done(_native().cache_read(kpages8, vpages8, kscale, vscale, block_table, seqlens, rows), "mala_cache_read_fp8")


def fwd_paged_fp8(q, kpages8, vpages8, kscale, vscale, cu_seqlens_q, block_table, seqlens_k, max_seqlen_q: int, total_k: int,
                  scale: float, tau: float, causal: bool = True, stats: bool = False, ws=None, num_splits: Optional[int] = None):
    """mala_fwd_paged_fp8(_split): ``fwd_paged`` over e4m3 pages with their scales; total_k: at least the sum of seqlens_k (room in the
    workspace).  num_splits: ranges that a sequence's keys are cut into, each with a skip test of its own (None: with tau 0, where that
    gives the same, and no ws of the caller's as many as the library suggests, else 1).  Returns (o, lse [Hq,total_q], Stats or None)."""
    st = None
    if stats:
        B, max_pages = block_table.shape
        Tk = -(-min(max_pages * kpages8.shape[1], total_k) // 128)
        st = Stats((B, q.shape[2], -(-(max_seqlen_q + 127) // 128)), -(-Tk // 32), q.device)
    o, lse = _done(_native().fwd_paged_fp8(q, kpages8, vpages8, kscale, vscale, cu_seqlens_q, block_table, seqlens_k, max_seqlen_q, total_k, scale, tau,
                                           causal, num_splits, ws, *((st.retained, st.bitmask, st.totals) if stats else (None, None, None))),
                   "mala_fwd_paged_fp8")
    return o, lse, st


def rotary_frequencies(rotary: int, base: float = 10000.0, scaling: Optional[str] = None, factor: float = 1.0, original: int = 8192,
                       fast: float = 32.0, slow: float = 1.0, low: float = 1.0, high: float = 4.0):
    """(radians per position of the ``rotary // 2`` pairs, float64 on the host; the magnitude) for ``Rotary``: base ** (-2 i / rotary),
    for contexts of ``factor`` times the ``original`` length

    - ``"linear"``: divided by factor;
    - ``"ntk"``: with the base raised to base * factor ** (rotary / (rotary - 2)), which divides the last pair's by factor;
    - ``"yarn"`` (Peng et al., 2023): pairs that make ``fast`` turns and more within the original length as they are, those below
      ``slow`` divided by factor, a ramp over the pairs between; magnitude 0.1 ln(factor) + 1;
    - ``"bands"``: by wavelength, those up to original / high as they are, beyond original / low divided by factor, blended between.
    """
    assert rotary >= 2 and rotary % 2 == 0 and base > 0 and factor > 0 and original > 0
    i = torch.arange(rotary // 2, dtype=torch.float64)
    f = base ** (-2 * i / rotary)
    if scaling is None:
        return f, 1.0
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "ntk":
        return (f if rotary == 2 else (base * factor ** (rotary / (rotary - 2))) ** (-2 * i / rotary)), 1.0
    if scaling == "yarn":
        at = [rotary * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base)) for turns in (fast, slow)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rotary - 1)
        ramp = ((i - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
        return f / factor * ramp + f * (1 - ramp), (0.1 * math.log(factor) + 1 if factor > 1 else 1.0)
    if scaling == "bands":
        keep = ((original * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
        return f / factor * (1 - keep) + f * keep, 1.0
    raise ValueError(f"unknown scaling {scaling!r}")


class Rotary:
    """Rotary positions: ``inv_freq`` (radians per position, one per pair of columns; kept as float64 on the device) for the first
    2 * len(inv_freq) columns of a head, paired as halves or, interleaved, as neighbours; ``magnitude`` scales the rotated columns."""

    def __init__(self, inv_freq: torch.Tensor, interleaved: bool = False, magnitude: float = 1.0, device=None):
        assert inv_freq.dim() == 1 and inv_freq.numel() >= 1 and inv_freq.is_floating_point(), "expects a frequency per pair of columns"
        if device is None and not inv_freq.is_cuda:
            device = "cuda"
        if device is not None or inv_freq.dtype is not torch.float64 or inv_freq.requires_grad or not inv_freq.is_contiguous():
            inv_freq = inv_freq.detach().to(device=device, dtype=torch.float64).contiguous()
        self.inv_freq = inv_freq
        self.rotary, self.interleaved, self.magnitude = 2 * inv_freq.numel(), bool(interleaved), float(magnitude)


class HeadNorm:
    """A root-mean-square norm of each head's row in front of its rotation: x / sqrt(mean(x^2) + eps) * weight, with weights [d] for
    queries and keys (bf16 or fp32, the same for both; None: 1)."""

    def __init__(self, q_weight: Optional[torch.Tensor], k_weight: Optional[torch.Tensor], eps: float = 1e-6):
        both = [w for w in (q_weight, k_weight) if w is not None]
        for w in both:
            assert w.dim() == 1 and w.is_contiguous() and w.dtype in (_BF16, _F32) and w.dtype == both[0].dtype and w.shape == both[0].shape, \
                "expects contiguous weights [d] of one type, bf16 or fp32"
        self.q_weight, self.k_weight, self.eps = q_weight, k_weight, float(eps)


def _rule(rot: Rotary, norm: Optional[HeadNorm]):
    if norm is None:
        return rot.inv_freq, rot.interleaved, rot.magnitude, None, None, None
    return rot.inv_freq, rot.interleaved, rot.magnitude, norm.eps, norm.q_weight, norm.k_weight


def rotary(q, k, rot: Rotary, positions=None, norm: Optional[HeadNorm] = None, q_out=None, k_out=None):
    """mala_rotary_fwd: rotary positions of q [B,Nq,Hq,d] and k [B,Nk,Hkv,d] (or None), bf16.  The queries are the last Nq of the Nk
    positions; positions int32 [B,Nk] (default 0 .. Nk - 1).  q_out, k_out may be q and k themselves.  Returns (q', k')."""
    return _done(_native().rotary(q, k, *_rule(rot, norm), positions, None, None, q_out, k_out), "mala_rotary_fwd")


def rotary_bwd(dq, dk, rot: Rotary, positions=None, norm: Optional[HeadNorm] = None, q=None, k=None, dq_out=None, dk_out=None,
               weights: bool = True):
    """mala_rotary_bwd: the gradients of q and k from those of rotary's outputs, dq and dk (or None); with a norm q and k as they went into it.
    dq_out, dk_out may be dq and dk themselves.  Returns (dq, dk, dq_weight, dk_weight), the weights' fp32 [d], None where there is
    none (or with weights false)."""
    return _done(_native().rotary_bwd(dq, dk, *_rule(rot, norm), positions, None, None, q, k, dq_out, dk_out, weights), "mala_rotary_bwd")


def rotary_varlen(q, k, cu_seqlens_q, cu_seqlens_k, rot: Rotary, norm: Optional[HeadNorm] = None, q_out=None, k_out=None):
    """mala_rotary_fwd_varlen: rotary on packed sequences, q [1,total_q,Hq,d], k [1,total_k,Hkv,d] (or None) with offsets int32 [B+1] on
    the device (the same tensor twice for self attention); positions count within a sequence's keys.  Returns (q', k')."""
    assert cu_seqlens_q is not None and cu_seqlens_k is not None, "expects the offsets of both"
    return _done(_native().rotary(q, k, *_rule(rot, norm), None, cu_seqlens_q, cu_seqlens_k, q_out, k_out), "mala_rotary_fwd_varlen")


def rotary_varlen_bwd(dq, dk, cu_seqlens_q, cu_seqlens_k, rot: Rotary, norm: Optional[HeadNorm] = None, q=None, k=None, dq_out=None,
                      dk_out=None, weights: bool = True):
    """mala_rotary_bwd_varlen: as rotary_bwd, on packed sequences."""
    assert cu_seqlens_q is not None and cu_seqlens_k is not None, "expects the offsets of both"
    return _done(_native().rotary_bwd(dq, dk, *_rule(rot, norm), None, cu_seqlens_q, cu_seqlens_k, q, k, dq_out, dk_out, weights),
                 "mala_rotary_bwd_varlen")


def rotary_write(q, k, v, positions, slots, kpages, vpages, rot: Rotary, norm: Optional[HeadNorm] = None, q_out=None):
    """mala_rotary_write: a serving step's rows q [rows,Hq,d], k, v [rows,Hkv,d] at positions int32 [rows]: k rotated into its slots
    (int64 [rows], negative: nowhere) of the bf16 pages [num_pages, page_size, Hkv, d], v into its own.  Returns q' (q_out may be q)."""
    return _done(_native().rotary_write(q, k, v, positions, slots, kpages, vpages, None, None, *_rule(rot, norm), q_out), "mala_rotary_write")


def rotary_write_fp8(q, k, v, positions, slots, kpages8, vpages8, kscale, vscale, rot: Rotary, norm: Optional[HeadNorm] = None,
                     q_out=None):
    """mala_rotary_write_fp8: the same into e4m3 pages (uint8 or float8_e4m3fn) with their scales (see ``cache_write_fp8``)."""
    assert kscale is not None and vscale is not None, "expects scales of keys and of values"
    return _done(_native().rotary_write(q, k, v, positions, slots, kpages8, vpages8, kscale, vscale, *_rule(rot, norm), q_out), "mala_rotary_write_fp8")
