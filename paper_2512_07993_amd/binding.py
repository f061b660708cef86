"""Thin ctypes binding of libskipkv.so: argument marshalling only.

Every function has the name and argument order of the C entry point in include/skipkv.h.
Tensors are torch tensors used purely as device-memory handles (data_ptr()); all work
runs in the library's HIP kernels on the current torch stream unless `stream` is given.
There is no fallback: if the library has not been built, loading raises.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional

import torch

F32, BF16 = 0, 1
OK, EINVAL, EBUDGET, ECAPACITY, EWORKSPACE, EHIP = 0, -1, -2, -3, -4, -5
DEV_BAD_OFFSETS, DEV_TOO_MANY_SENT, DEV_TIMEOUT, DEV_TOO_MANY_TOK, DEV_BAD_BLOCK_TABLE, DEV_BAD_BUDGET, DEV_BAD_SCORES = 1, 2, 4, 8, 16, 32, 64
DEV_BAD_LENGTHS, DEV_OUT_OF_BLOCKS = 128, 256
FLAG_FORCE_TWO_PASS = 1
PROFILE_SLOTS = 16

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libskipkv.so")
_lib = None


class CCache(C.Structure):
    _fields_ = [
        ("k", C.c_void_p), ("v", C.c_void_p),
        ("stride_layer", C.c_int64), ("stride_head", C.c_int64), ("stride_tok", C.c_int64),
        ("dtype", C.c_int32), ("n_layers", C.c_int32), ("n_kv_heads", C.c_int32),
        ("n_q_heads", C.c_int32), ("head_dim", C.c_int32), ("batch", C.c_int32),
        ("total_tokens", C.c_int32), ("total_sentences", C.c_int32),
        ("seq_off", C.c_void_p), ("sent_ptr", C.c_void_p), ("sent_off", C.c_void_p),
    ]


class CRanges(C.Structure):
    _fields_ = [("len", C.c_void_p), ("sent_cnt", C.c_void_p), ("sent_off", C.c_void_p)]


class CPaging(C.Structure):
    _fields_ = [("block_table", C.c_void_p), ("table_stride", C.c_int32), ("block_size", C.c_int32),
                ("n_blocks", C.c_int32), ("stride_block", C.c_int64)]


class CPages(C.Structure):
    _fields_ = [("block_table", C.c_void_p), ("n_held", C.c_void_p), ("free_list", C.c_void_p), ("n_free", C.c_void_p),
                ("batch", C.c_int32), ("table_stride", C.c_int32), ("block_size", C.c_int32), ("n_blocks", C.c_int32)]


class CQuantCache(C.Structure):
    _fields_ = [
        ("k", C.c_void_p), ("v", C.c_void_p), ("k_exp", C.c_void_p), ("v_exp", C.c_void_p),
        ("stride_layer", C.c_int64), ("stride_head", C.c_int64), ("stride_block", C.c_int64), ("stride_tok", C.c_int64),
        ("n_layers", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("batch", C.c_int32),
        ("block_size", C.c_int32), ("n_blocks", C.c_int32), ("table_stride", C.c_int32), ("block_table", C.c_void_p),
    ]


class CQueries(C.Structure):
    _fields_ = [
        ("q", C.c_void_p), ("out", C.c_void_p), ("lse", C.c_void_p),
        ("q_stride_tok", C.c_int64), ("q_stride_head", C.c_int64), ("out_stride_tok", C.c_int64), ("out_stride_head", C.c_int64),
        ("dtype", C.c_int32), ("n_q_heads", C.c_int32), ("total_q", C.c_int32), ("max_q", C.c_int32), ("max_len", C.c_int32),
        ("scale", C.c_float), ("q_off", C.c_void_p),
    ]


class CParams(C.Structure):
    _fields_ = [
        ("obs_window", C.c_int32), ("protect_window", C.c_int32),
        ("sigma", C.c_float), ("tau", C.c_float),
        ("budget", C.c_void_p), ("budget_scalar", C.c_int32), ("max_budget", C.c_int32),
        ("dev_status", C.c_void_p), ("profile", C.c_void_p),
        ("flags", C.c_uint32), ("spin_limit", C.c_int32),
    ]


def lib() -> C.CDLL:
    """Load libskipkv.so (built by paper_2512_07993_amd.build); raise if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(
                "libskipkv.so is not built: run `python -m paper_2512_07993_amd.build` "
                "(there is no CPU fallback)")
        L = C.CDLL(_LIB_PATH)
        vp, i32, sz, fl = C.c_void_p, C.c_int32, C.c_size_t, C.c_float
        cp, pp = C.POINTER(CCache), C.POINTER(CParams)
        L.skipkv_workspace_bytes.argtypes = [cp, pp, C.POINTER(sz)]
        L.skipkv_score.argtypes = [cp, pp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.skipkv_select.argtypes = [cp, pp, vp, vp, vp, vp, vp, vp, i32, vp]
        L.skipkv_compact.argtypes = [cp, vp, vp, i32, vp]
        L.skipkv_step.argtypes = [cp, pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, sz, vp]
        L.skipkv_step_static.argtypes = [cp, pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp]
        L.skipkv_select_tokens.argtypes = [cp, pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp]
        L.skipkv_redundancy_workspace_bytes.argtypes = [cp, C.POINTER(sz)]
        L.skipkv_token_redundancy.argtypes = [cp, vp, vp, sz, vp]
        L.skipkv_steer_add.argtypes = [vp, vp, vp, fl, vp, i32, i32, i32, vp]
        L.skipkv_similarity_workspace_bytes.argtypes = [cp, i32, C.POINTER(sz)]
        L.skipkv_sentence_similarity.argtypes = [cp, vp, i32, i32, vp, vp, sz, vp]
        L.skipkv_score_shared.argtypes = [cp, pp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.skipkv_steer_strength.argtypes = [vp, fl, fl, vp, i32, vp]
        rp = C.POINTER(CRanges)
        L.skipkv_ranges_workspace_bytes.argtypes = [cp, pp, C.POINTER(sz)]
        L.skipkv_ranges_append.argtypes = [cp, rp, vp, vp, vp, vp, vp]
        L.skipkv_token_redundancy_ranges.argtypes = [cp, rp, vp, vp, sz, vp]
        L.skipkv_score_ranges.argtypes = [cp, rp, pp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.skipkv_select_tokens_ranges.argtypes = [cp, rp, pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, sz, vp]
        L.skipkv_select_ranges.argtypes = [cp, rp, pp, vp, vp, vp, vp, vp, vp, i32, vp, sz, vp]
        L.skipkv_ranges_ids_select.argtypes = [cp, rp, i32, vp, vp, vp, vp]
        L.skipkv_ranges_ids_append.argtypes = [cp, vp, vp, vp, vp]
        L.skipkv_score_shared_ranges.argtypes = [cp, rp, vp, vp, pp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.skipkv_step_ranges.argtypes = [cp, rp, pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, sz, vp]
        gp = C.POINTER(CPaging)
        L.skipkv_paged_workspace_bytes.argtypes = [cp, gp, pp, C.POINTER(sz)]
        L.skipkv_step_paged.argtypes = [cp, gp, pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, sz, vp]
        L.skipkv_score_paged.argtypes = [cp, gp, pp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.skipkv_score_shared_paged.argtypes = [cp, gp, pp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.skipkv_compact_paged_workspace_bytes.argtypes = [cp, gp, i32, C.POINTER(sz)]
        L.skipkv_compact_paged.argtypes = [cp, gp, vp, vp, i32, vp, vp, sz, vp]
        L.skipkv_redundancy_paged_workspace_bytes.argtypes = [cp, gp, C.POINTER(sz)]
        L.skipkv_token_redundancy_paged.argtypes = [cp, gp, vp, vp, vp, sz, vp]
        L.skipkv_score_ranges_paged.argtypes = [cp, rp, gp, vp, vp, vp, pp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.skipkv_token_redundancy_ranges_paged.argtypes = [cp, rp, gp, vp, vp, vp, sz, vp]
        L.skipkv_ranges_paged_workspace_bytes.argtypes = [cp, gp, pp, C.POINTER(sz)]
        L.skipkv_step_ranges_paged.argtypes = [cp, rp, gp, pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, sz, vp]
        sp, qp, np_ = C.POINTER(CPages), C.POINTER(CQuantCache), C.POINTER(CQueries)
        L.skipkv_pages_workspace_bytes.argtypes = [sp, C.POINTER(sz)]
        L.skipkv_pages_update.argtypes = [sp, vp, i32, vp, i32, vp, vp, vp, sz, vp]
        L.skipkv_quant_store.argtypes = [qp, cp, i32, vp, vp, vp, vp]
        L.skipkv_quant_load.argtypes = [qp, cp, i32, vp, vp, vp, vp]
        L.skipkv_quant_attend_workspace_bytes.argtypes = [qp, np_, C.POINTER(sz)]
        L.skipkv_quant_attend.argtypes = [qp, i32, np_, vp, vp, vp, sz, vp]
        L.skipkv_profile_create.argtypes = [C.POINTER(vp)]
        L.skipkv_profile_read.argtypes = [vp, C.POINTER(i32), C.POINTER(C.c_char_p), C.POINTER(fl)]
        L.skipkv_profile_destroy.argtypes = [vp]
        L.skipkv_strerror.argtypes = [C.c_int]
        L.skipkv_strerror.restype = C.c_char_p
        L.skipkv_version.argtypes = []
        for name in ("skipkv_workspace_bytes", "skipkv_score", "skipkv_select", "skipkv_compact", "skipkv_step",
                     "skipkv_steer_add", "skipkv_redundancy_workspace_bytes", "skipkv_token_redundancy",
                     "skipkv_select_tokens", "skipkv_ranges_workspace_bytes", "skipkv_ranges_append", "skipkv_step_ranges",
                     "skipkv_similarity_workspace_bytes", "skipkv_sentence_similarity", "skipkv_score_shared", "skipkv_steer_strength",
                     "skipkv_paged_workspace_bytes", "skipkv_step_paged",
                     "skipkv_pages_workspace_bytes", "skipkv_pages_update", "skipkv_quant_store", "skipkv_quant_load",
                     "skipkv_quant_attend_workspace_bytes", "skipkv_quant_attend",
                     "skipkv_profile_create", "skipkv_profile_read", "skipkv_profile_destroy",
                     "skipkv_version"):
            getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


class SkipKVError(RuntimeError):
    def __init__(self, status: int):
        self.status = status
        super().__init__("libskipkv: %s (%d)" % (lib().skipkv_strerror(status).decode(), status))


def _check(status: int) -> None:
    if status != OK:
        raise SkipKVError(status)


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        # The handle itself once the device is in use: a Stream object and a look for devices at every call took
        # longer than the steering kernels do (the two calls of a steering step: 15.7 -> 9.6 us).
        if torch.cuda.is_initialized():
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        return torch.cuda.current_stream().cuda_stream if torch.cuda.is_available() else None
    return stream if isinstance(stream, int) else stream.cuda_stream


def _ints(t, device: int, optional=False) -> Optional[int]:
    """Address of a contiguous int32 tensor that lies on `device` (an index, -1: the host)."""
    if t is None and optional:
        return None
    assert t.dtype == torch.int32 and t.is_contiguous() and t.get_device() == device
    return t.data_ptr()


def _scratch(ws, device: int):
    """Address and bytes of a workspace without gaps that lies on `device`."""
    if ws is None:
        return None, 0
    assert ws.is_contiguous() and ws.get_device() == device, "the workspace has to be contiguous, on the device of the other tensors"
    return ws.data_ptr(), ws.numel() * ws.element_size()


def _status(t, device: int) -> Optional[int]:
    """Address of a status word: int32, on `device` or in pinned memory."""
    if t is None or isinstance(t, int):
        return t
    assert t.dtype == torch.int32 and (t.get_device() == device or t.is_pinned()), "the status word has to be int32, on the device of the other tensors"
    return t.data_ptr()


def _here(t) -> int:
    """Device of a tensor, which has to be the current one: a launch goes there."""
    device = t.get_device()
    if device < 0:  # (without a GPU the launch fails by itself)
        assert not torch.cuda.is_available(), "the tensors are in host memory"
    else:
        assert device == torch._C._cuda_getDevice(), "the tensors are on another device than the current one"
    return device


def dtype_code(t: torch.dtype) -> int:
    if t == torch.float32:
        return F32
    if t == torch.bfloat16:
        return BF16
    raise ValueError("unsupported dtype %s" % t)


@dataclass
class Cache:
    """Python mirror of skipkv_cache.  k, v: [L, Hk, T, D] tensors (any strides with D contiguous)."""
    k: torch.Tensor
    v: torch.Tensor
    n_q_heads: int
    seq_off: torch.Tensor      # int32 device [B+1]
    sent_ptr: torch.Tensor     # int32 device [B+1]
    sent_off: torch.Tensor     # int32 device [S_total + B]
    total_tokens: int
    total_sentences: int

    @property
    def batch(self) -> int:
        return int(self.seq_off.numel()) - 1

    def c(self) -> CCache:
        k = self.k
        assert k.dim() == 4 and k.stride(3) == 1 and self.v.stride() == k.stride() and self.v.shape == k.shape
        return CCache(k.data_ptr(), self.v.data_ptr(), k.stride(0), k.stride(1), k.stride(2), dtype_code(k.dtype),
                      k.shape[0], k.shape[1], self.n_q_heads, k.shape[3], self.batch,
                      self.total_tokens, self.total_sentences,
                      _ptr(self.seq_off), _ptr(self.sent_ptr), _ptr(self.sent_off))


@dataclass
class Params:
    """Python mirror of skipkv_params."""
    obs_window: int
    protect_window: int
    budget: "int | torch.Tensor"
    max_budget: int = -1
    sigma: float = 0.1
    tau: float = 0.95
    dev_status: Optional[torch.Tensor] = None
    profile: Optional[int] = None
    flags: int = 0
    spin_limit: int = 0

    def c(self) -> CParams:
        if isinstance(self.budget, int):
            bptr, bs = None, self.budget
            mb = self.budget if self.max_budget < 0 else self.max_budget
        else:
            bptr, bs, mb = self.budget.data_ptr(), 0, self.max_budget
        return CParams(self.obs_window, self.protect_window, self.sigma, self.tau, bptr, bs, mb,
                       _ptr(self.dev_status), self.profile, self.flags, self.spin_limit)


def skipkv_version() -> int:
    return lib().skipkv_version()


def skipkv_strerror(status: int) -> str:
    return lib().skipkv_strerror(status).decode()


def skipkv_workspace_bytes(cache: Cache, params: Params) -> int:
    out = C.c_size_t(0)
    _check(lib().skipkv_workspace_bytes(C.byref(cache.c()), C.byref(params.c()), C.byref(out)))
    return int(out.value)


def skipkv_score(cache: Cache, params: Params, q_obs, tok_redundancy, sent_score, sent_lambda, tok_importance,
                 ws, stream=None) -> None:
    _check(lib().skipkv_score(C.byref(cache.c()), C.byref(params.c()), _ptr(q_obs), _ptr(tok_redundancy),
                              _ptr(sent_score), _ptr(sent_lambda), _ptr(tok_importance), _ptr(ws),
                              ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream)))


def skipkv_select(cache: Cache, params: Params, sent_score, sent_keep, kept_idx, new_len, new_sent_off,
                  new_sent_cnt, kept_stride: int, stream=None) -> None:
    _check(lib().skipkv_select(C.byref(cache.c()), C.byref(params.c()), _ptr(sent_score), _ptr(sent_keep),
                               _ptr(kept_idx), _ptr(new_len), _ptr(new_sent_off), _ptr(new_sent_cnt),
                               kept_stride, _stream(stream)))


def skipkv_select_tokens(cache: Cache, params: Params, tok_importance, tok_redundancy, sent_lambda, tok_score,
                         tok_keep, kept_idx, new_len, new_sent_off, new_sent_cnt, kept_stride: int, stream=None) -> None:
    _check(lib().skipkv_select_tokens(C.byref(cache.c()), C.byref(params.c()), _ptr(tok_importance),
                                      _ptr(tok_redundancy), _ptr(sent_lambda), _ptr(tok_score), _ptr(tok_keep),
                                      _ptr(kept_idx), _ptr(new_len), _ptr(new_sent_off), _ptr(new_sent_cnt),
                                      kept_stride, _stream(stream)))


def skipkv_compact(cache: Cache, kept_idx, new_len, kept_stride: int, stream=None) -> None:
    _check(lib().skipkv_compact(C.byref(cache.c()), _ptr(kept_idx), _ptr(new_len), kept_stride, _stream(stream)))


def skipkv_step(cache: Cache, params: Params, q_obs, tok_redundancy, sent_score, sent_lambda, tok_importance,
                sent_keep, kept_idx, new_len, new_sent_off, new_sent_cnt, kept_stride: int, ws, stream=None) -> None:
    _check(lib().skipkv_step(C.byref(cache.c()), C.byref(params.c()), _ptr(q_obs), _ptr(tok_redundancy),
                             _ptr(sent_score), _ptr(sent_lambda), _ptr(tok_importance), _ptr(sent_keep),
                             _ptr(kept_idx), _ptr(new_len), _ptr(new_sent_off), _ptr(new_sent_cnt), kept_stride,
                             _ptr(ws), ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream)))


STATIC_WS_BYTES = 64 << 20  # SKIPKV_STATIC_WS_BYTES


def skipkv_step_static(cache: Cache, params: Params, q_obs, tok_redundancy, sent_score, sent_lambda, tok_importance,
                       sent_keep, kept_idx, new_len, new_sent_off, new_sent_cnt, kept_stride: int, stream=None) -> None:
    _check(lib().skipkv_step_static(C.byref(cache.c()), C.byref(params.c()), _ptr(q_obs), _ptr(tok_redundancy),
                                    _ptr(sent_score), _ptr(sent_lambda), _ptr(tok_importance), _ptr(sent_keep),
                                    _ptr(kept_idx), _ptr(new_len), _ptr(new_sent_off), _ptr(new_sent_cnt), kept_stride,
                                    _stream(stream)))


@dataclass
class Ranges:
    """Python mirror of skipkv_ranges: per-head lengths [L, Hk, B], sentence counts [L, Hk, B] and
    offsets [L, Hk, S_total + B] (int32 device tensors)."""
    len: torch.Tensor
    sent_cnt: torch.Tensor
    sent_off: torch.Tensor

    def c(self) -> CRanges:
        return CRanges(self.len.data_ptr(), self.sent_cnt.data_ptr(), self.sent_off.data_ptr())


def skipkv_ranges_workspace_bytes(cache: Cache, params: Params) -> int:
    out = C.c_size_t(0)
    _check(lib().skipkv_ranges_workspace_bytes(C.byref(cache.c()), C.byref(params.c()), C.byref(out)))
    return int(out.value)


def skipkv_ranges_append(cache: Cache, ranges: Ranges, n_new, bnd_ptr, bnd_off, dev_status=None, stream=None) -> None:
    _check(lib().skipkv_ranges_append(C.byref(cache.c()), C.byref(ranges.c()), _ptr(n_new), _ptr(bnd_ptr),
                                      _ptr(bnd_off), _ptr(dev_status), _stream(stream)))


def skipkv_step_ranges(cache: Cache, ranges: Ranges, params: Params, q_obs, tok_redundancy, sent_score, sent_lambda,
                       tok_importance, sent_keep, kept_idx, new_len, new_sent_off, new_sent_cnt, kept_stride: int, ws,
                       stream=None) -> None:
    _check(lib().skipkv_step_ranges(C.byref(cache.c()), C.byref(ranges.c()), C.byref(params.c()), _ptr(q_obs),
                                    _ptr(tok_redundancy), _ptr(sent_score), _ptr(sent_lambda), _ptr(tok_importance),
                                    _ptr(sent_keep), _ptr(kept_idx), _ptr(new_len), _ptr(new_sent_off),
                                    _ptr(new_sent_cnt), kept_stride, _ptr(ws),
                                    ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream)))


def _nbytes(ws) -> int:
    return ws.numel() * ws.element_size() if ws is not None else 0


def skipkv_token_redundancy_ranges(cache: Cache, ranges: Ranges, tok_redundancy, ws, stream=None) -> None:
    _check(lib().skipkv_token_redundancy_ranges(C.byref(cache.c()), C.byref(ranges.c()), _ptr(tok_redundancy), _ptr(ws),
                                                _nbytes(ws), _stream(stream)))


def skipkv_score_ranges(cache: Cache, ranges: Ranges, params: Params, q_obs, tok_redundancy, sent_score, sent_lambda,
                        tok_importance, ws, stream=None) -> None:
    _check(lib().skipkv_score_ranges(C.byref(cache.c()), C.byref(ranges.c()), C.byref(params.c()), _ptr(q_obs),
                                     _ptr(tok_redundancy), _ptr(sent_score), _ptr(sent_lambda), _ptr(tok_importance),
                                     _ptr(ws), _nbytes(ws), _stream(stream)))


def skipkv_select_tokens_ranges(cache: Cache, ranges: Ranges, params: Params, tok_importance, tok_redundancy, sent_lambda,
                                tok_score, tok_keep, kept_idx, new_len, new_sent_off, new_sent_cnt, kept_stride: int, ws,
                                stream=None) -> None:
    _check(lib().skipkv_select_tokens_ranges(C.byref(cache.c()), C.byref(ranges.c()), C.byref(params.c()),
                                             _ptr(tok_importance), _ptr(tok_redundancy), _ptr(sent_lambda), _ptr(tok_score),
                                             _ptr(tok_keep), _ptr(kept_idx), _ptr(new_len), _ptr(new_sent_off),
                                             _ptr(new_sent_cnt), kept_stride, _ptr(ws), _nbytes(ws), _stream(stream)))


def skipkv_select_ranges(cache: Cache, ranges: Ranges, params: Params, sent_score, sent_keep, kept_idx, new_len, new_sent_off,
                         new_sent_cnt, kept_stride: int, ws, stream=None) -> None:
    _check(lib().skipkv_select_ranges(C.byref(cache.c()), C.byref(ranges.c()), C.byref(params.c()), _ptr(sent_score),
                                      _ptr(sent_keep), _ptr(kept_idx), _ptr(new_len), _ptr(new_sent_off), _ptr(new_sent_cnt),
                                      kept_stride, _ptr(ws), _nbytes(ws), _stream(stream)))


def skipkv_ranges_ids_select(cache: Cache, ranges, protect_window: int, sent_keep, sent_id_in, sent_id_out, stream=None) -> None:
    _check(lib().skipkv_ranges_ids_select(C.byref(cache.c()), C.byref(ranges.c()) if ranges is not None else None,
                                          protect_window, _ptr(sent_keep), _ptr(sent_id_in), _ptr(sent_id_out),
                                          _stream(stream)))


def skipkv_ranges_ids_append(cache: Cache, old_cnt, new_cnt, sent_id, stream=None) -> None:
    _check(lib().skipkv_ranges_ids_append(C.byref(cache.c()), _ptr(old_cnt), _ptr(new_cnt), _ptr(sent_id), _stream(stream)))


def skipkv_score_shared_ranges(cache: Cache, ranges: Ranges, sent_id, lambda_ptr, params: Params, q_obs, tok_redundancy,
                               shared_lambda, sent_score, sent_lambda, tok_importance, ws, stream=None) -> None:
    _check(lib().skipkv_score_shared_ranges(C.byref(cache.c()), C.byref(ranges.c()), _ptr(sent_id), _ptr(lambda_ptr),
                                            C.byref(params.c()), _ptr(q_obs), _ptr(tok_redundancy), _ptr(shared_lambda),
                                            _ptr(sent_score), _ptr(sent_lambda), _ptr(tok_importance), _ptr(ws), _nbytes(ws),
                                            _stream(stream)))


@dataclass
class PagedCache:
    """Python mirror of skipkv_cache + skipkv_paging for pools laid out [L, blocks, slots, Hk, D]
    (any strides with D contiguous); seq_off numbers the logical tokens."""
    k: torch.Tensor
    v: torch.Tensor
    block_table: torch.Tensor  # int32 device [B, table_stride]
    n_q_heads: int
    seq_off: torch.Tensor
    sent_ptr: torch.Tensor
    sent_off: torch.Tensor
    total_tokens: int
    total_sentences: int

    def c(self) -> CCache:
        k = self.k
        assert k.dim() == 5 and k.stride(4) == 1 and self.v.stride() == k.stride() and self.v.shape == k.shape
        return CCache(k.data_ptr(), self.v.data_ptr(), k.stride(0), k.stride(3), k.stride(2), dtype_code(k.dtype),
                      k.shape[0], k.shape[3], self.n_q_heads, k.shape[4], int(self.seq_off.numel()) - 1,
                      self.total_tokens, self.total_sentences,
                      _ptr(self.seq_off), _ptr(self.sent_ptr), _ptr(self.sent_off))

    def paging(self) -> CPaging:
        bt = self.block_table
        assert bt.dim() == 2 and bt.dtype == torch.int32 and bt.stride(1) == 1
        return CPaging(bt.data_ptr(), bt.stride(0), self.k.shape[2], self.k.shape[1], self.k.stride(1))


def skipkv_paged_workspace_bytes(cache: PagedCache, params: Params) -> int:
    out = C.c_size_t(0)
    _check(lib().skipkv_paged_workspace_bytes(C.byref(cache.c()), C.byref(cache.paging()), C.byref(params.c()), C.byref(out)))
    return int(out.value)


def skipkv_step_paged(cache: PagedCache, params: Params, q_obs, tok_redundancy, sent_score, sent_lambda, tok_importance,
                      sent_keep, kept_idx, new_len, new_sent_off, new_sent_cnt, kept_stride: int, ws, stream=None) -> None:
    _check(lib().skipkv_step_paged(C.byref(cache.c()), C.byref(cache.paging()), C.byref(params.c()), _ptr(q_obs),
                                   _ptr(tok_redundancy), _ptr(sent_score), _ptr(sent_lambda), _ptr(tok_importance),
                                   _ptr(sent_keep), _ptr(kept_idx), _ptr(new_len), _ptr(new_sent_off),
                                   _ptr(new_sent_cnt), kept_stride, _ptr(ws),
                                   ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream)))


def skipkv_score_paged(cache: PagedCache, params: Params, q_obs, tok_redundancy, sent_score, sent_lambda, tok_importance,
                       ws, stream=None) -> None:
    _check(lib().skipkv_score_paged(C.byref(cache.c()), C.byref(cache.paging()), C.byref(params.c()), _ptr(q_obs),
                                    _ptr(tok_redundancy), _ptr(sent_score), _ptr(sent_lambda), _ptr(tok_importance),
                                    _ptr(ws), ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream)))


def skipkv_score_shared_paged(cache: PagedCache, params: Params, q_obs, tok_redundancy, shared_lambda, sent_score, sent_lambda,
                              tok_importance, ws, stream=None) -> None:
    _check(lib().skipkv_score_shared_paged(C.byref(cache.c()), C.byref(cache.paging()), C.byref(params.c()), _ptr(q_obs),
                                           _ptr(tok_redundancy), _ptr(shared_lambda), _ptr(sent_score), _ptr(sent_lambda),
                                           _ptr(tok_importance), _ptr(ws), _nbytes(ws), _stream(stream)))


def skipkv_compact_paged_workspace_bytes(cache: PagedCache, kept_stride: int) -> int:
    out = C.c_size_t(0)
    _check(lib().skipkv_compact_paged_workspace_bytes(C.byref(cache.c()), C.byref(cache.paging()), kept_stride, C.byref(out)))
    return int(out.value)


def skipkv_compact_paged(cache: PagedCache, kept_idx, new_len, kept_stride: int, dev_status, ws, stream=None) -> None:
    _check(lib().skipkv_compact_paged(C.byref(cache.c()), C.byref(cache.paging()), _ptr(kept_idx), _ptr(new_len),
                                      kept_stride, _ptr(dev_status), _ptr(ws),
                                      ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream)))


def skipkv_redundancy_paged_workspace_bytes(cache: PagedCache) -> int:
    out = C.c_size_t(0)
    _check(lib().skipkv_redundancy_paged_workspace_bytes(C.byref(cache.c()), C.byref(cache.paging()), C.byref(out)))
    return int(out.value)


def skipkv_token_redundancy_paged(cache: PagedCache, tok_redundancy, dev_status, ws, stream=None) -> None:
    _check(lib().skipkv_token_redundancy_paged(C.byref(cache.c()), C.byref(cache.paging()), _ptr(tok_redundancy),
                                               _ptr(dev_status), _ptr(ws),
                                               ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream)))


def skipkv_score_ranges_paged(cache: PagedCache, ranges: Ranges, sent_id, lambda_ptr, shared_lambda, params: Params, q_obs,
                              tok_redundancy, sent_score, sent_lambda, tok_importance, ws, stream=None) -> None:
    _check(lib().skipkv_score_ranges_paged(C.byref(cache.c()), C.byref(ranges.c()), C.byref(cache.paging()), _ptr(sent_id),
                                           _ptr(lambda_ptr), _ptr(shared_lambda), C.byref(params.c()), _ptr(q_obs),
                                           _ptr(tok_redundancy), _ptr(sent_score), _ptr(sent_lambda), _ptr(tok_importance),
                                           _ptr(ws), _nbytes(ws), _stream(stream)))


def skipkv_token_redundancy_ranges_paged(cache: PagedCache, ranges: Ranges, tok_redundancy, dev_status, ws, stream=None) -> None:
    _check(lib().skipkv_token_redundancy_ranges_paged(C.byref(cache.c()), C.byref(ranges.c()), C.byref(cache.paging()),
                                                      _ptr(tok_redundancy), _ptr(dev_status), _ptr(ws), _nbytes(ws),
                                                      _stream(stream)))


def skipkv_ranges_paged_workspace_bytes(cache: PagedCache, params: Params) -> int:
    out = C.c_size_t(0)
    _check(lib().skipkv_ranges_paged_workspace_bytes(C.byref(cache.c()), C.byref(cache.paging()), C.byref(params.c()),
                                                     C.byref(out)))
    return int(out.value)


def skipkv_step_ranges_paged(cache: PagedCache, ranges: Ranges, params: Params, q_obs, tok_redundancy, sent_score,
                             sent_lambda, tok_importance, sent_keep, kept_idx, new_len, new_sent_off, new_sent_cnt,
                             kept_stride: int, ws, stream=None) -> None:
    _check(lib().skipkv_step_ranges_paged(C.byref(cache.c()), C.byref(ranges.c()), C.byref(cache.paging()),
                                          C.byref(params.c()), _ptr(q_obs), _ptr(tok_redundancy), _ptr(sent_score),
                                          _ptr(sent_lambda), _ptr(tok_importance), _ptr(sent_keep), _ptr(kept_idx),
                                          _ptr(new_len), _ptr(new_sent_off), _ptr(new_sent_cnt), kept_stride, _ptr(ws),
                                          ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream)))


@dataclass
class Pages:
    """Python mirror of skipkv_pages: block_table [B, table_stride] (rows as far apart as they are wide), n_held [B],
    free_list [n_blocks] and n_free [1], int32 device tensors that skipkv_pages_update changes in place."""
    block_table: torch.Tensor
    n_held: torch.Tensor
    free_list: torch.Tensor
    n_free: torch.Tensor
    block_size: int

    def c(self) -> CPages:
        bt, device = self.block_table, self.block_table.get_device()
        # (the library takes a row's width for its pitch too: a view of some columns of a wider table would have it read and write the others)
        assert bt.dim() == 2 and bt.shape[0] == self.n_held.numel() and bt.is_contiguous(), "a block table's rows have to lie as far apart as they are wide"
        assert bt.dtype == torch.int32 and self.n_free.numel() >= 1
        return CPages(bt.data_ptr(), _ints(self.n_held, device), _ints(self.free_list, device), _ints(self.n_free, device),
                      bt.shape[0], bt.shape[1], self.block_size, self.free_list.numel())


def skipkv_pages_workspace_bytes(pages: Pages) -> int:
    out = C.c_size_t(0)
    _check(lib().skipkv_pages_workspace_bytes(C.byref(pages.c()), C.byref(out)))
    return int(out.value)


def skipkv_pages_update(pages: Pages, len, new_off, total_new: int, slot_map, ws, dev_status=None, stream=None) -> None:
    """len: [n_rows, B] (or [L, Hk, B]: n_rows = L * Hk); new_off: [B + 1] or None; slot_map: [n_rows, total_new] or None."""
    device, batch = _here(pages.block_table), pages.n_held.numel()
    assert len.shape[-1] == batch and (new_off is None or new_off.numel() == batch + 1)
    n_rows = len.numel() // max(batch, 1) if len.numel() else 1
    assert slot_map is None or slot_map.numel() == n_rows * total_new
    _check(lib().skipkv_pages_update(C.byref(pages.c()), _ints(len, device), n_rows, _ints(new_off, device, True), total_new,
                                     _ints(slot_map, device, True), _status(dev_status, device), *_scratch(ws, device), _stream(stream)))


_CODES = (torch.uint8, torch.float8_e4m3fn)


@dataclass
class QuantCache:
    """Python mirror of skipkv_quant_cache for pools laid out [L, blocks, slots, Hk, D] (any strides with D
    contiguous) of uint8 or float8_e4m3fn, scale bytes [L, Hk, blocks] and a block table [B, table_stride] (rows as far apart as
    they are wide)."""
    k: torch.Tensor
    v: torch.Tensor
    k_exp: torch.Tensor
    v_exp: torch.Tensor
    block_table: torch.Tensor

    def c(self) -> CQuantCache:
        # Strides and shapes once each: a look at a tensor's stride or size costs 0.2 us, and a call for one
        # token spends longer here than on the GPU (this structure 17.8 -> 9.6 us).
        k, v, ke, ve, bt = self.k, self.v, self.k_exp, self.v_exp, self.block_table
        st, sh = k.stride(), tuple(k.shape)
        assert len(sh) == 5 and st[4] == 1 and v.stride() == st and v.shape == sh
        assert k.dtype in _CODES and v.dtype in _CODES, "pools hold e4m3 codes: uint8 or float8_e4m3fn"
        L, blocks, slots, heads, dim = sh
        exps, device = (L, heads, blocks), k.get_device()
        assert v.get_device() == ke.get_device() == ve.get_device() == bt.get_device() == device
        assert ke.dtype == ve.dtype == torch.uint8 and ke.is_contiguous() and ve.is_contiguous() and ke.shape == exps and ve.shape == exps
        batch, wide = bt.shape
        assert bt.dtype == torch.int32 and bt.is_contiguous(), "a block table's rows have to lie as far apart as they are wide"
        return CQuantCache(k.data_ptr(), v.data_ptr(), ke.data_ptr(), ve.data_ptr(), st[0], st[3], st[1], st[2], L, heads, dim,
                           batch, slots, blocks, wide, bt.data_ptr())


@dataclass
class Queries:
    """Python mirror of skipkv_queries: q and out [total_q, Hq, D] (any strides with D contiguous), lse [total_q, Hq] fp32 or None."""
    q: torch.Tensor
    out: torch.Tensor
    q_off: torch.Tensor        # int32 device [B+1]
    max_q: int
    max_len: int
    scale: float
    lse: Optional[torch.Tensor] = None

    def c(self) -> CQueries:
        q, o, lse = self.q, self.out, self.lse
        qs, os_, sh = q.stride(), o.stride(), tuple(q.shape)
        assert len(sh) == 3 and o.shape == sh and o.get_device() == q.get_device() and o.dtype == q.dtype and qs[2] == 1 and os_[2] == 1
        assert lse is None or (lse.is_contiguous() and lse.dtype == torch.float32 and lse.shape == sh[:2]
                               and lse.get_device() == q.get_device())
        return CQueries(q.data_ptr(), o.data_ptr(), None if lse is None else lse.data_ptr(), qs[0], qs[1], os_[0], os_[1],
                        dtype_code(q.dtype), sh[1], sh[0], self.max_q, self.max_len, self.scale, _ints(self.q_off, q.get_device()))


def _quant_rows(call, qc: QuantCache, rows: Cache, first_layer: int, begin, end, dev_status, stream) -> None:
    device = _here(qc.k)
    assert rows.k.get_device() == device
    for t in (begin, end):
        assert t is None or t.numel() == rows.k.shape[0] * qc.k.shape[3] * qc.block_table.shape[0]
    _check(call(C.byref(qc.c()), C.byref(rows.c()), first_layer, _ints(begin, device, True), _ints(end, device, True),
                _status(dev_status, device), _stream(stream)))


def skipkv_quant_store(qc: QuantCache, rows: Cache, first_layer: int, begin, end, dev_status=None, stream=None) -> None:
    _quant_rows(lib().skipkv_quant_store, qc, rows, first_layer, begin, end, dev_status, stream)


def skipkv_quant_load(qc: QuantCache, rows: Cache, first_layer: int, begin, end, dev_status=None, stream=None) -> None:
    _quant_rows(lib().skipkv_quant_load, qc, rows, first_layer, begin, end, dev_status, stream)


def skipkv_quant_attend_workspace_bytes(qc: QuantCache, queries: Queries) -> int:
    out = C.c_size_t(0)
    _check(lib().skipkv_quant_attend_workspace_bytes(C.byref(qc.c()), C.byref(queries.c()), C.byref(out)))
    return int(out.value)


def skipkv_quant_attend(qc: QuantCache, layer: int, queries: Queries, len, ws, dev_status=None, stream=None) -> None:
    device = _here(qc.k)
    assert len.shape == (qc.k.shape[3], qc.block_table.shape[0]) and queries.q.get_device() == device
    assert queries.q_off.numel() == len.shape[1] + 1
    _check(lib().skipkv_quant_attend(C.byref(qc.c()), layer, C.byref(queries.c()), _ints(len, device),
                                     _status(dev_status, device), *_scratch(ws, device), _stream(stream)))


def skipkv_similarity_workspace_bytes(cache: Cache, d_model: int) -> int:
    out = C.c_size_t(0)
    _check(lib().skipkv_similarity_workspace_bytes(C.byref(cache.c()), d_model, C.byref(out)))
    return int(out.value)


def skipkv_sentence_similarity(cache: Cache, hidden, shared_lambda, ws, stream=None) -> None:
    assert hidden.dim() == 2 and hidden.is_contiguous()
    _check(lib().skipkv_sentence_similarity(C.byref(cache.c()), _ptr(hidden), hidden.shape[1], dtype_code(hidden.dtype),
                                            _ptr(shared_lambda), _ptr(ws),
                                            ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream)))


def skipkv_score_shared(cache: Cache, params: Params, q_obs, tok_redundancy, shared_lambda, sent_score, sent_lambda,
                        tok_importance, ws, stream=None) -> None:
    _check(lib().skipkv_score_shared(C.byref(cache.c()), C.byref(params.c()), _ptr(q_obs), _ptr(tok_redundancy),
                                     _ptr(shared_lambda), _ptr(sent_score), _ptr(sent_lambda), _ptr(tok_importance),
                                     _ptr(ws), ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream)))


def skipkv_redundancy_workspace_bytes(cache: Cache) -> int:
    out = C.c_size_t(0)
    _check(lib().skipkv_redundancy_workspace_bytes(C.byref(cache.c()), C.byref(out)))
    return int(out.value)


def skipkv_token_redundancy(cache: Cache, tok_redundancy, ws, stream=None) -> None:
    _check(lib().skipkv_token_redundancy(C.byref(cache.c()), _ptr(tok_redundancy), _ptr(ws),
                                         ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream)))


def skipkv_steer_add(hidden, vec, coef, coef_scalar: float, row_mask, stream=None) -> None:
    rows, d_model = hidden.shape
    assert hidden.is_contiguous() and vec.is_contiguous() and vec.dtype == hidden.dtype
    _check(lib().skipkv_steer_add(_ptr(hidden), _ptr(vec), _ptr(coef), float(coef_scalar), _ptr(row_mask),
                                  rows, d_model, dtype_code(hidden.dtype), _stream(stream)))


def skipkv_steer_strength(n_nonexec, alpha0: float, gamma: float, coef, stream=None) -> None:
    _check(lib().skipkv_steer_strength(_ptr(n_nonexec), float(alpha0), float(gamma), _ptr(coef), n_nonexec.numel(), _stream(stream)))


def skipkv_profile_create() -> int:
    out = C.c_void_p(0)
    _check(lib().skipkv_profile_create(C.byref(out)))
    return int(out.value)


def skipkv_profile_read(profile: int) -> "list[tuple[str, float]]":
    n = C.c_int32(0)
    names = (C.c_char_p * PROFILE_SLOTS)()
    ms = (C.c_float * PROFILE_SLOTS)()
    _check(lib().skipkv_profile_read(profile, C.byref(n), names, ms))
    return [(names[i].decode(), float(ms[i])) for i in range(n.value)]


def skipkv_profile_destroy(profile: int) -> None:
    _check(lib().skipkv_profile_destroy(profile))
