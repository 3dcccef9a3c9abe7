"""Thin ctypes binding of libskvq.so (include/skvq.h): argument marshalling only.

Every step of the path runs in the library's HIP kernels; PyTorch is used to own device
memory and to name the current stream.  There is no fallback: if the library has not been
built, importing a function from here raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libskvq.so")

SKVQ_OK = 0
SKVQ_ERR_INVALID_ARG, SKVQ_ERR_UNSUPPORTED, SKVQ_ERR_CAPACITY, SKVQ_ERR_STATE, SKVQ_ERR_HIP = -1, -2, -3, -4, -5
SKVQ_BITS_4, SKVQ_BITS_3, SKVQ_BITS_2, SKVQ_BITS_1P5 = 16, 8, 4, 3
SKVQ_MAX_SPLITS = 128
SKVQ_STATIC_MAX_ROWS = 64
HEAD_DIM = 128
BUFFER_NAMES = ("k_codes", "v_codes", "k_meta", "v_meta", "k_win", "v_win", "workspace")
PAGED_BUFFER_NAMES = ("pages", "k_rows", "v_rows", "workspace")
SKVQ_PAGED_BAD_COUNTS, SKVQ_PAGED_BAD_SLOT, SKVQ_PAGED_BAD_PAGE, SKVQ_PAGED_BAD_RANGE = 1, 2, 4, 8
DTYPES = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}   # skvq_dtype
ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3, "bands": 4}


class skvq_config(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("group_size", C.c_int32), ("k_bits", C.c_int32),
                ("v_bits", C.c_int32), ("window", C.c_int32), ("n_sink", C.c_int32),
                ("meta_format", C.c_int32), ("max_quant_tokens", C.c_int64),
                ("perm_k", C.c_void_p), ("perm_v", C.c_void_p), ("clip_k", C.c_void_p),
                ("clip_v", C.c_void_p), ("sm_scale", C.c_float), ("max_new_tokens", C.c_int32),
                ("group_bounds", C.c_void_p)]


class skvq_buffers(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in BUFFER_NAMES]


class skvq_rope_config(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("rotary_dim", C.c_int32), ("layout", C.c_int32), ("scaling", C.c_int32),
                ("base", C.c_double), ("factor", C.c_double), ("original_context", C.c_double), ("low", C.c_double),
                ("high", C.c_double), ("amplitude", C.c_double), ("frequencies", C.c_void_p)]


class skvq_rope_tensor(C.Structure):
    _fields_ = ([("x", C.c_void_p), ("y", C.c_void_p)]
                + [(n, C.c_int64) for n in ("x_batch", "x_token", "x_head", "y_batch", "y_token", "y_head")]
                + [("n_heads", C.c_int32)])


class skvq_paged_config(C.Structure):
    _fields_ = ([(n, C.c_int32) for n in ("n_q_heads", "n_kv_heads", "head_dim", "group_size", "k_bits", "v_bits", "window",
                                          "n_sink", "meta_format", "dtype", "page_size", "n_pages", "max_seqs", "max_tokens")]
                + [(n, C.c_void_p) for n in ("perm_k", "perm_v", "clip_k", "clip_v")] + [("sm_scale", C.c_float)])


class skvq_paged_buffers(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in PAGED_BUFFER_NAMES]


class skvq_batch(C.Structure):
    _fields_ = [("n_seqs", C.c_int32), ("n_tokens", C.c_int32), ("cu_tokens", C.c_void_p), ("seq_lens", C.c_void_p),
                ("page_table", C.c_void_p), ("table_stride", C.c_int32), ("slots", C.c_void_p), ("positions", C.c_void_p),
                ("first", C.c_void_p)]


_lib = None


def lib() -> C.CDLL:
    """The loaded library; raises if it has not been built (no fallback path exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2405_06219_amd.build`")
        L = C.CDLL(LIB_PATH)
        L.skvq_sizes.argtypes = [C.POINTER(skvq_config), C.POINTER(C.c_size_t)]
        L.skvq_validate_config.argtypes = [C.POINTER(skvq_config)]
        L.skvq_create.argtypes = [C.POINTER(skvq_config), C.POINTER(skvq_buffers), C.POINTER(C.c_void_p)]
        L.skvq_destroy.argtypes = [C.c_void_p]
        L.skvq_destroy.restype = None
        L.skvq_prefill_quantize.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]
        L.skvq_calibrate_channel_stats.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int64, C.c_void_p, C.c_void_p]
        L.skvq_calibrate_reorder.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p,
                                             C.c_void_p]
        L.skvq_decode_attention_multi.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
        L.skvq_set_clip.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.skvq_calibrate_clip.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int32,
                                          C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                          C.c_void_p]
        L.skvq_prefill_attention.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64,
                                             C.c_void_p, C.c_void_p, C.c_void_p]
        L.skvq_prefill_attention_quantize.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64,
                                                      C.c_void_p, C.c_void_p, C.c_void_p]
        L.skvq_quantize_append.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.skvq_prefill_quantize_filtered.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p,
                                                     C.c_void_p]
        L.skvq_quantize_append_filtered.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]
        L.skvq_decode_attention.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.skvq_decode_attention_static.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.skvq_append_decode_attention.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                                   C.c_void_p, C.c_void_p]
        L.skvq_get_state.argtypes = [C.c_void_p, C.POINTER(C.c_int64), C.POINTER(C.c_int64), C.POINTER(C.c_int32)]
        L.skvq_set_state.argtypes = [C.c_void_p, C.c_int64]
        L.skvq_set_num_splits.argtypes = [C.c_void_p, C.c_int32]
        L.skvq_read_yardstick.argtypes = [C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
        L.skvq_read_write_yardstick.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_int32, C.c_void_p]
        L.skvq_rope_create.argtypes = [C.POINTER(skvq_rope_config), C.POINTER(C.c_void_p)]
        L.skvq_rope_destroy.argtypes = [C.c_void_p]
        L.skvq_rope_destroy.restype = None
        L.skvq_rope_frequencies.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p]
        L.skvq_rope_apply.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int64,
                                      C.c_void_p, C.c_int64, C.c_int64, C.c_int32, C.c_void_p]
        L.skvq_paged_sizes.argtypes = [C.POINTER(skvq_paged_config), C.POINTER(C.c_size_t)]
        L.skvq_paged_validate_config.argtypes = [C.POINTER(skvq_paged_config)]
        L.skvq_paged_create.argtypes = [C.POINTER(skvq_paged_config), C.POINTER(skvq_paged_buffers), C.POINTER(C.c_void_p)]
        L.skvq_paged_destroy.argtypes = [C.c_void_p]
        L.skvq_paged_destroy.restype = None
        L.skvq_paged_append.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p,
                                        C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p]
        L.skvq_paged_read.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p]
        L.skvq_paged_attention.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64,
                                           C.c_void_p, C.c_void_p]
        L.skvq_paged_errors.argtypes = [C.c_void_p, C.POINTER(C.c_int32), C.c_void_p]
        L.skvq_paged_last_error.argtypes = [C.c_void_p]
        L.skvq_paged_last_error.restype = C.c_char_p
        L.skvq_status_string.argtypes = [C.c_int]
        L.skvq_status_string.restype = C.c_char_p
        L.skvq_last_error.argtypes = [C.c_void_p]
        L.skvq_last_error.restype = C.c_char_p
        _lib = L
    return _lib


class SkvqError(RuntimeError):
    def __init__(self, status: int, detail: str = ""):
        self.status = status
        text = lib().skvq_status_string(status).decode()
        super().__init__(f"skvq status {status} ({text}) {detail}".strip())


META_FORMATS = {"f32": 0, "f16": 1, "e4m3": 2}   # skvq_meta_format
META_DTYPES = {0: np.float32, 1: np.float16, 2: np.uint8}


def bits_enum(bits: float) -> int:
    return {4.0: SKVQ_BITS_4, 3.0: SKVQ_BITS_3, 2.0: SKVQ_BITS_2, 1.5: SKVQ_BITS_1P5}[float(bits)]


def make_config(batch, n_q_heads, n_kv_heads, group_size, v_bits, window, max_quant_tokens, perm_k, perm_v,
                clip_k, clip_v, sm_scale=0.0, k_bits=2.0, head_dim=HEAD_DIM, n_sink=0, meta="f32",
                group_bounds=None, max_new_tokens=0):
    """Returns (skvq_config, keepalive): the numpy arrays the config points to."""
    keep = [np.ascontiguousarray(perm_k, np.int32), np.ascontiguousarray(perm_v, np.int32),
            np.ascontiguousarray(clip_k, np.float32), np.ascontiguousarray(clip_v, np.float32)]
    if group_bounds is not None:      # [n_kv_heads][head_dim / group_size + 1]; one row serves every head
        gb = np.atleast_2d(np.asarray(group_bounds, np.int32))
        if gb.shape[0] == 1:
            gb = np.repeat(gb, n_kv_heads, axis=0)
        keep.append(np.ascontiguousarray(gb))
        if keep[4].shape != (n_kv_heads, head_dim // group_size + 1):
            raise ValueError("group_bounds needs head_dim / group_size + 1 entries per kv head")
    cfg = skvq_config(batch, n_q_heads, n_kv_heads, head_dim, group_size, bits_enum(k_bits), bits_enum(v_bits),
                      window, n_sink, META_FORMATS[meta], max_quant_tokens, keep[0].ctypes.data, keep[1].ctypes.data, keep[2].ctypes.data,
                      keep[3].ctypes.data, float(sm_scale), int(max_new_tokens),
                      keep[4].ctypes.data if group_bounds is not None else None)
    return cfg, keep


def skvq_sizes(cfg: skvq_config) -> list[int]:
    out = (C.c_size_t * 7)()
    rc = lib().skvq_sizes(C.byref(cfg), out)
    if rc != SKVQ_OK:
        raise SkvqError(rc)
    return [int(x) for x in out]


def skvq_calibrate_channel_stats(x: torch.Tensor, stream=None) -> np.ndarray:
    """(min, max) per (kv head, channel) of fp16 x [B][Hk][T][D] on the device -> float32 [Hk][D][2]."""
    b, hk, T, d = x.shape
    xp = _dev_ptr(x, torch.float16, (b, hk, T, HEAD_DIM))
    stats = np.zeros((hk, HEAD_DIM, 2), np.float32)
    rc = lib().skvq_calibrate_channel_stats(xp, b, hk, T, stats.ctypes.data, _stream_ptr(stream))
    if rc != SKVQ_OK:
        raise SkvqError(rc)
    return stats


def skvq_calibrate_reorder(stats: np.ndarray, group_size: int, granularity: int = 16, max_iter: int = 100):
    """KMeans channel reorder: returns (perm [Hk][D], bounds [Hk][D/G + 1])."""
    stats = np.ascontiguousarray(stats, np.float32)
    hk = stats.shape[0]
    perm = np.zeros((hk, HEAD_DIM), np.int32)
    bounds = np.zeros((hk, HEAD_DIM // group_size + 1), np.int32)
    rc = lib().skvq_calibrate_reorder(stats.ctypes.data, hk, group_size, granularity, max_iter, perm.ctypes.data,
                                      bounds.ctypes.data)
    if rc != SKVQ_OK:
        raise SkvqError(rc)
    return perm, bounds


def skvq_read_yardstick(src: torch.Tensor, sink: torch.Tensor, stream=None):
    """The library's read-only kernel over the bytes of `src` (a contiguous device tensor)."""
    rc = lib().skvq_read_yardstick(src.data_ptr(), src.numel() * src.element_size(), sink.data_ptr(), _stream_ptr(stream))
    if rc != SKVQ_OK:
        raise SkvqError(rc)


def skvq_read_write_yardstick(src: torch.Tensor, dst: torch.Tensor, ratio: int, stream=None):
    """The library's read/write kernel: reads ratio times the bytes of `dst` from `src` and fills `dst`
    (contiguous device tensors; `src` must hold at least that many bytes)."""
    nbytes = dst.numel() * dst.element_size()
    if src.numel() * src.element_size() < ratio * nbytes:
        raise SkvqError(SKVQ_ERR_INVALID_ARG)
    rc = lib().skvq_read_write_yardstick(src.data_ptr(), dst.data_ptr(), nbytes, ratio, _stream_ptr(stream))
    if rc != SKVQ_OK:
        raise SkvqError(rc)


def skvq_validate_config(cfg: skvq_config) -> int:
    return int(lib().skvq_validate_config(C.byref(cfg)))


def _stream_ptr(stream) -> int:
    if stream is None:
        # the current device's current stream, as torch.cuda.current_stream() names it, without the Stream
        # object (2.8 us a call, of 8 us that a short decode step takes)
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return int(stream.cuda_stream)


def _dev_ptr(t: torch.Tensor, dtype, shape) -> int:
    if not (t.shape == shape and t.dtype == dtype and t.is_cuda and t.is_contiguous()):
        raise ValueError(f"expected contiguous cuda {dtype} tensor of shape {tuple(shape)}, got {t.dtype} "
                         f"{tuple(t.shape)} on {t.device}")
    return t.data_ptr()


class SkvqCache:
    """One layer's cache: owns the device buffers (torch tensors) and the library handle."""

    def __init__(self, batch, n_q_heads, n_kv_heads, group_size, v_bits, window, max_quant_tokens, perm_k, perm_v,
                 clip_k, clip_v, sm_scale=0.0, k_bits=2.0, device="cuda:0", fill=None, n_sink=0,
                 meta="f32", group_bounds=None, max_new_tokens=0):
        self.cfg, self._keep = make_config(batch, n_q_heads, n_kv_heads, group_size, v_bits, window,
                                           max_quant_tokens, perm_k, perm_v, clip_k, clip_v, sm_scale, k_bits,
                                           n_sink=n_sink, meta=meta, group_bounds=group_bounds,
                                           max_new_tokens=max_new_tokens)
        self.shape = (batch, n_q_heads, n_kv_heads)
        self.window = window
        self.device = torch.device(device)
        self.sizes = skvq_sizes(self.cfg)
        self.buffers = {}
        for name, nbytes in zip(BUFFER_NAMES, self.sizes):
            t = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            if fill is not None:
                t.fill_(fill)
            self.buffers[name] = t
        self._bufs = skvq_buffers(*[self.buffers[n].data_ptr() for n in BUFFER_NAMES])
        handle = C.c_void_p()
        with torch.cuda.device(self.device):
            rc = lib().skvq_create(C.byref(self.cfg), C.byref(self._bufs), C.byref(handle))
        if rc != SKVQ_OK:
            raise SkvqError(rc)
        self._h = handle

    def close(self):
        if getattr(self, "_h", None):
            lib().skvq_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc):
        if rc != SKVQ_OK:
            raise SkvqError(rc, lib().skvq_last_error(self._h).decode())

    # ---- clip scales: Eq. 2's alpha, and its calibration by Eq. 3 ----
    def skvq_set_clip(self, clip_k: np.ndarray, clip_v: np.ndarray, stream=None):
        ck = np.ascontiguousarray(clip_k, np.float32)
        cv = np.ascontiguousarray(clip_v, np.float32)
        ng = HEAD_DIM // self.cfg.group_size
        if ck.shape != (self.shape[2], ng) or cv.shape != ck.shape:
            raise ValueError("clip scales must be [n_kv_heads][head_dim / group_size]")
        self._check(lib().skvq_set_clip(self._h, ck.ctypes.data, cv.ctypes.data, _stream_ptr(stream)))

    def skvq_calibrate_clip(self, k: torch.Tensor, v: torch.Tensor, q: torch.Tensor, o_ref: torch.Tensor,
                            alphas, stream=None):
        """Returns (clip_k, clip_v, loss) as numpy arrays [Hk][NG], [Hk][NG], [Hk]."""
        b, hq, hk = self.shape
        T, n = k.shape[2], q.shape[0]
        kp = _dev_ptr(k, torch.float16, (b, hk, T, HEAD_DIM))
        vp = _dev_ptr(v, torch.float16, (b, hk, T, HEAD_DIM))
        qp = _dev_ptr(q, torch.float16, (n, b, hq, HEAD_DIM))
        op = _dev_ptr(o_ref, torch.float32, (n, b, hq, HEAD_DIM))
        al = np.ascontiguousarray(alphas, np.float32)
        ng = HEAD_DIM // self.cfg.group_size
        ck, cv = np.zeros((hk, ng), np.float32), np.zeros((hk, ng), np.float32)
        loss = np.zeros(hk, np.float64)
        self._check(lib().skvq_calibrate_clip(self._h, kp, vp, T, qp, n, op, al.ctypes.data, al.size, ck.ctypes.data,
                                              cv.ctypes.data, loss.ctypes.data, _stream_ptr(stream)))
        return ck, cv, loss

    # ---- the hot-path calls, named as in the C ABI ----
    def skvq_prefill_attention(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                               out_f32: torch.Tensor | None = None, out_f16: torch.Tensor | None = None,
                               stream=None) -> torch.Tensor:
        b, hq, hk = self.shape
        T = q.shape[2]
        qp = _dev_ptr(q, torch.float16, (b, hq, T, HEAD_DIM))
        kp = _dev_ptr(k, torch.float16, (b, hk, T, HEAD_DIM))
        vp = _dev_ptr(v, torch.float16, (b, hk, T, HEAD_DIM))
        if out_f32 is None:
            out_f32 = torch.empty((b, hq, T, HEAD_DIM), dtype=torch.float32, device=self.device)
        op = _dev_ptr(out_f32, torch.float32, (b, hq, T, HEAD_DIM))
        o16 = _dev_ptr(out_f16, torch.float16, (b, hq, T, HEAD_DIM)) if out_f16 is not None else None
        self._check(lib().skvq_prefill_attention(self._h, qp, kp, vp, T, op, o16, _stream_ptr(stream)))
        return out_f32

    def skvq_prefill_attention_quantize(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                                        out_f32: torch.Tensor | None = None, out_f16: torch.Tensor | None = None,
                                        stream=None) -> torch.Tensor:
        b, hq, hk = self.shape
        T = q.shape[2]
        qp = _dev_ptr(q, torch.float16, (b, hq, T, HEAD_DIM))
        kp = _dev_ptr(k, torch.float16, (b, hk, T, HEAD_DIM))
        vp = _dev_ptr(v, torch.float16, (b, hk, T, HEAD_DIM))
        if out_f32 is None:
            out_f32 = torch.empty((b, hq, T, HEAD_DIM), dtype=torch.float32, device=self.device)
        op = _dev_ptr(out_f32, torch.float32, (b, hq, T, HEAD_DIM))
        o16 = _dev_ptr(out_f16, torch.float16, (b, hq, T, HEAD_DIM)) if out_f16 is not None else None
        self._check(lib().skvq_prefill_attention_quantize(self._h, qp, kp, vp, T, op, o16, _stream_ptr(stream)))
        return out_f32

    def skvq_prefill_quantize(self, k: torch.Tensor, v: torch.Tensor, stream=None):
        b, _, hk = self.shape
        T = k.shape[2]
        kp = _dev_ptr(k, torch.float16, (b, hk, T, HEAD_DIM))
        vp = _dev_ptr(v, torch.float16, (b, hk, T, HEAD_DIM))
        self._check(lib().skvq_prefill_quantize(self._h, kp, vp, T, _stream_ptr(stream)))

    def skvq_prefill_quantize_filtered(self, k: torch.Tensor, v: torch.Tensor, keep, stream=None):
        """keep: one entry per token older than the window (host array-like; nonzero = kept in fp16) or None."""
        b, _, hk = self.shape
        T = k.shape[2]
        kp = _dev_ptr(k, torch.float16, (b, hk, T, HEAD_DIM))
        vp = _dev_ptr(v, torch.float16, (b, hk, T, HEAD_DIM))
        mask = None
        if keep is not None:
            mask = np.ascontiguousarray(np.asarray(keep).astype(bool).astype(np.uint8))
            if mask.shape != (max(T - self.window, 0),):
                raise ValueError("keep must have one entry per token older than the window")
            if mask.size == 0:
                mask = np.zeros(1, np.uint8)
        self._check(lib().skvq_prefill_quantize_filtered(self._h, kp, vp, T, mask.ctypes.data if mask is not None else None,
                                                         _stream_ptr(stream)))

    def skvq_quantize_append_filtered(self, k_new: torch.Tensor, v_new: torch.Tensor, keep_leaving: bool, stream=None):
        b, _, hk = self.shape
        kp = _dev_ptr(k_new, torch.float16, (b, hk, HEAD_DIM))
        vp = _dev_ptr(v_new, torch.float16, (b, hk, HEAD_DIM))
        self._check(lib().skvq_quantize_append_filtered(self._h, kp, vp, 1 if keep_leaving else 0, _stream_ptr(stream)))

    def skvq_quantize_append(self, k_new: torch.Tensor, v_new: torch.Tensor, stream=None):
        b, _, hk = self.shape
        kp = _dev_ptr(k_new, torch.float16, (b, hk, HEAD_DIM))
        vp = _dev_ptr(v_new, torch.float16, (b, hk, HEAD_DIM))
        self._check(lib().skvq_quantize_append(self._h, kp, vp, _stream_ptr(stream)))

    def skvq_decode_attention(self, q: torch.Tensor, out_f32: torch.Tensor | None = None,
                              out_f16: torch.Tensor | None = None, stream=None) -> torch.Tensor:
        b, hq, _ = self.shape
        qp = _dev_ptr(q, torch.float16, (b, hq, HEAD_DIM))
        if out_f32 is None:
            out_f32 = torch.empty((b, hq, HEAD_DIM), dtype=torch.float32, device=self.device)
        op = _dev_ptr(out_f32, torch.float32, (b, hq, HEAD_DIM))
        hp = _dev_ptr(out_f16, torch.float16, (b, hq, HEAD_DIM)) if out_f16 is not None else None
        self._check(lib().skvq_decode_attention(self._h, qp, op, hp, _stream_ptr(stream)))
        return out_f32

    def skvq_decode_attention_static(self, q: torch.Tensor, out_f32: torch.Tensor, out_f16: torch.Tensor | None = None,
                                     stream=None) -> torch.Tensor:
        """The variant that allocates nothing: the caller passes the output tensor too."""
        b, hq, _ = self.shape
        qp = _dev_ptr(q, torch.float16, (b, hq, HEAD_DIM))
        op = _dev_ptr(out_f32, torch.float32, (b, hq, HEAD_DIM))
        hp = _dev_ptr(out_f16, torch.float16, (b, hq, HEAD_DIM)) if out_f16 is not None else None
        self._check(lib().skvq_decode_attention_static(self._h, qp, op, hp, _stream_ptr(stream)))
        return out_f32

    def skvq_append_decode_attention(self, k_new: torch.Tensor, v_new: torch.Tensor, q: torch.Tensor,
                                     out_f32: torch.Tensor | None = None, out_f16: torch.Tensor | None = None,
                                     stream=None) -> torch.Tensor:
        b, hq, hk = self.shape
        kp = _dev_ptr(k_new, torch.float16, (b, hk, HEAD_DIM))
        vp = _dev_ptr(v_new, torch.float16, (b, hk, HEAD_DIM))
        qp = _dev_ptr(q, torch.float16, (b, hq, HEAD_DIM))
        if out_f32 is None:
            out_f32 = torch.empty((b, hq, HEAD_DIM), dtype=torch.float32, device=self.device)
        op = _dev_ptr(out_f32, torch.float32, (b, hq, HEAD_DIM))
        hp = _dev_ptr(out_f16, torch.float16, (b, hq, HEAD_DIM)) if out_f16 is not None else None
        self._check(lib().skvq_append_decode_attention(self._h, kp, vp, qp, op, hp, _stream_ptr(stream)))
        return out_f32

    # ---- state ----
    def skvq_get_state(self):
        a, b, c = C.c_int64(), C.c_int64(), C.c_int32()
        self._check(lib().skvq_get_state(self._h, C.byref(a), C.byref(b), C.byref(c)))
        return a.value, b.value, c.value

    def skvq_set_state(self, n_tokens: int):
        self._check(lib().skvq_set_state(self._h, n_tokens))

    def skvq_set_num_splits(self, n: int):
        self._check(lib().skvq_set_num_splits(self._h, n))

    def skvq_decode_attention_multi(self, q: torch.Tensor, out_f32: torch.Tensor | None = None,
                                    out_f16: torch.Tensor | None = None, stream=None) -> torch.Tensor:
        """q [B][n_new][Hq][D]: the last n_new cached tokens' queries; returns fp32 [B][n_new][Hq][D]."""
        b, hq, _ = self.shape
        n_new = q.shape[1]
        qp = _dev_ptr(q, torch.float16, (b, n_new, hq, HEAD_DIM))
        if out_f32 is None:
            out_f32 = torch.empty((b, n_new, hq, HEAD_DIM), dtype=torch.float32, device=self.device)
        op = _dev_ptr(out_f32, torch.float32, (b, n_new, hq, HEAD_DIM))
        o16 = _dev_ptr(out_f16, torch.float16, (b, n_new, hq, HEAD_DIM)) if out_f16 is not None else None
        self._check(lib().skvq_decode_attention_multi(self._h, qp, n_new, op, o16, _stream_ptr(stream)))
        return out_f32

    # ---- views of the buffers for tests ----
    def host_arrays(self):
        """Buffers copied to the host with the shapes the format statement gives them."""
        b, _, hk = self.shape
        tcap = self.cfg.max_quant_tokens
        ng = HEAD_DIM // self.cfg.group_size
        vb = {SKVQ_BITS_1P5: 832, SKVQ_BITS_2: 1024, SKVQ_BITS_3: 1536, SKVQ_BITS_4: 2048}[self.cfg.v_bits]
        kb = {SKVQ_BITS_2: 32, SKVQ_BITS_3: 48, SKVQ_BITS_4: 64}[self.cfg.k_bits]
        torch.cuda.synchronize(self.device)
        raw = {n: self.buffers[n].cpu().numpy() for n in BUFFER_NAMES[:6]}
        return [raw["k_codes"].reshape(b, hk, tcap, kb),
                raw["v_codes"].reshape(b, hk, (tcap + 31) // 32, vb),
                raw["k_meta"].view(META_DTYPES[self.cfg.meta_format]).reshape(b, hk, tcap, ng, 2),
                raw["v_meta"].view(META_DTYPES[self.cfg.meta_format]).reshape(b, hk, tcap, ng, 2),
                raw["k_win"].view(np.uint16).reshape(b, hk, self.cfg.window + self.cfg.n_sink, HEAD_DIM),
                raw["v_win"].view(np.uint16).reshape(b, hk, self.cfg.window + self.cfg.n_sink, HEAD_DIM)]


# ---- rotary positions and the paged cache ------------------------------------------------------------------


_ROPE_SIDE = struct.Struct("@PPqqqqqqi4x").pack   # skvq_rope_tensor


def _stream_on(device: torch.device, stream) -> int:
    """The stream's handle; without one, the current stream of the tensors' device."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(device.index)
    return stream.cuda_stream


class SkvqRope:
    """Rotary positions: frequencies of the first rotary_dim channels of a head, as skvq_rope_config takes them."""

    def __init__(self, head_dim=HEAD_DIM, rotary_dim=None, layout="half", base=10000.0, scaling="none", factor=0.0,
                 original_context=0.0, low=0.0, high=0.0, amplitude=0.0, frequencies=None):
        rotary_dim = head_dim if rotary_dim is None else rotary_dim
        own = None
        if frequencies is not None:
            own = np.ascontiguousarray(frequencies, np.float64)
            if own.shape != (rotary_dim // 2,):
                raise ValueError("frequencies needs rotary_dim / 2 entries")
        cfg = skvq_rope_config(head_dim, rotary_dim, ROPE_LAYOUTS[layout], ROPE_SCALINGS[scaling], base, factor,
                               original_context, low, high, amplitude, own.ctypes.data if own is not None else None)
        handle = C.c_void_p()
        rc = lib().skvq_rope_create(C.byref(cfg), C.byref(handle))
        if rc != SKVQ_OK:
            raise SkvqError(rc)
        self._h, self.head_dim, self.rotary_dim = handle, head_dim, rotary_dim

    def __del__(self):
        try:
            if getattr(self, "_h", None):
                lib().skvq_rope_destroy(self._h)
                self._h = None
        except Exception:
            pass

    def skvq_rope_frequencies(self):
        """(radians per token of every pair, amplitude)."""
        f, a = np.zeros(self.rotary_dim // 2, np.float64), C.c_double()
        rc = lib().skvq_rope_frequencies(self._h, f.ctypes.data, C.addressof(a))
        if rc != SKVQ_OK:
            raise SkvqError(rc)
        return f, a.value

    def skvq_rope_apply(self, q: torch.Tensor, k: torch.Tensor | None = None, positions: torch.Tensor | None = None, start=0,
                        out_q: torch.Tensor | None = None, out_k: torch.Tensor | None = None, transpose=False, stream=None):
        """q, k [B][T][heads][head_dim] with any strides but the last dimension's; positions int32 [T] or [B][T], or
        None: start + t.  transpose: the gradient's way back.  Returns q's result, or (q's, k's); out_q / out_k may
        be q / k (in place)."""
        if q.dtype not in DTYPES:
            raise ValueError(f"rotary positions take fp16, bf16 and fp32 tensors, got {q.dtype}")
        if out_q is None:
            out_q = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        sides = self._side(q, out_q, q)
        if k is not None:
            if out_k is None:
                out_k = torch.empty(k.shape, dtype=k.dtype, device=k.device)
            sides += self._side(k, out_k, q)
        b, t = q.shape[:2]
        at, stride = None, 0
        if positions is not None:
            if positions.dtype != torch.int32 or positions.device != q.device or positions.shape not in ((t,), (b, t)) or (
                    t > 1 and positions.stride(-1) != 1):
                raise ValueError(f"positions must be int32 [{t}] or [{b}][{t}] on {q.device}")
            at, stride = positions.data_ptr(), positions.stride(0) if positions.dim() == 2 else 0
        device = q.device.index
        call = (self._h, sides, 1 if k is None else 2, DTYPES[q.dtype], b, t, at, stride, start, transpose,
                torch._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream)
        if device == torch._C._cuda_getDevice():
            rc = lib().skvq_rope_apply(*call)
        else:
            with torch.cuda.device(device):
                rc = lib().skvq_rope_apply(*call)
        if rc != SKVQ_OK:
            raise SkvqError(rc)
        return out_q if k is None else (out_q, out_k)

    def _side(self, x, y, q) -> bytes:
        """One skvq_rope_tensor (packed: a ctypes structure takes 2 us to fill)."""
        shape, sx, sy = x.shape, x.stride(), y.stride()
        if not (len(shape) == 4 and shape == y.shape and shape[:2] == q.shape[:2] and shape[3] == self.head_dim and x.is_cuda
                and x.dtype == y.dtype == q.dtype and x.device == y.device == q.device
                and (sx[3] == sy[3] == 1 or x.numel() == 0)):
            raise ValueError(f"expected {q.dtype} tensors [{q.shape[0]}][{q.shape[1]}][heads][{self.head_dim}] on {q.device}, channels "
                             f"contiguous, got {x.dtype} {tuple(x.shape)} on {x.device}, strides {sx}, and {y.dtype} "
                             f"{tuple(y.shape)} on {y.device}, strides {sy}")
        return _ROPE_SIDE(x.data_ptr(), y.data_ptr(), sx[0], sx[1], sx[2], sy[0], sy[1], sy[2], shape[2])


class SkvqBatch:
    """The sequences of a call (skvq_batch): int32 tensors on the cache's device, read when a call runs, so their contents
    may change between calls.  n_tokens: rows of the token tensors; None reads cu_tokens' last entry (and waits)."""

    def __init__(self, cu_tokens: torch.Tensor, seq_lens: torch.Tensor, page_table: torch.Tensor, slots=None, positions=None,
                 first=None, n_tokens=None):
        n = seq_lens.shape[0]
        if n_tokens is None:
            n_tokens = int(cu_tokens[-1])
        if page_table.dim() != 2 or page_table.shape[0] != n:
            raise ValueError("page_table must be [n_seqs][pages]")
        shapes = {"cu_tokens": (cu_tokens, (n + 1,)), "seq_lens": (seq_lens, (n,)), "page_table": (page_table, tuple(page_table.shape)),
                  "slots": (slots, (n,)), "positions": (positions, (n_tokens,)), "first": (first, (n,))}
        for name, (t, shape) in shapes.items():
            if t is not None and not (t.dtype == torch.int32 and t.is_cuda and t.device == seq_lens.device and t.is_contiguous()
                                      and tuple(t.shape) == shape):
                raise ValueError(f"{name} must be a contiguous int32 tensor of shape {shape} on {seq_lens.device}")
        self.tensors = [t for t, _ in shapes.values()]   # kept alive
        self.device, self.n_seqs, self.n_tokens = seq_lens.device, n, n_tokens

        def ptr(t):
            return t.data_ptr() if t is not None else None

        self.struct = skvq_batch(n, n_tokens, ptr(cu_tokens), ptr(seq_lens), ptr(page_table), page_table.shape[1], ptr(slots),
                                 ptr(positions), ptr(first))
        self.address = C.addressof(self.struct)


def make_paged_config(n_q_heads, n_kv_heads, group_size, window, page_size, n_pages, max_seqs, max_tokens, perm_k, perm_v,
                      clip_k, clip_v, sm_scale=0.0, k_bits=4.0, v_bits=4.0, head_dim=HEAD_DIM, n_sink=0, meta="f16",
                      dtype=torch.float16):
    """Returns (skvq_paged_config, keepalive): the numpy arrays the config points to."""
    keep = [np.ascontiguousarray(perm_k, np.int32), np.ascontiguousarray(perm_v, np.int32),
            np.ascontiguousarray(clip_k, np.float32), np.ascontiguousarray(clip_v, np.float32)]
    shapes = [(n_kv_heads, head_dim)] * 2 + [(n_kv_heads, head_dim // max(group_size, 1))] * 2
    if [a.shape for a in keep] != shapes:
        raise ValueError("perm must be [n_kv_heads][head_dim], clip [n_kv_heads][head_dim / group_size]")
    cfg = skvq_paged_config(n_q_heads, n_kv_heads, head_dim, group_size, bits_enum(k_bits), bits_enum(v_bits), window, n_sink,
                            META_FORMATS[meta], DTYPES[dtype], page_size, n_pages, max_seqs, max_tokens,
                            *[a.ctypes.data for a in keep], float(sm_scale))
    return cfg, keep


def skvq_paged_sizes(cfg: skvq_paged_config) -> list[int]:
    out = (C.c_size_t * 4)()
    rc = lib().skvq_paged_sizes(C.byref(cfg), out)
    if rc != SKVQ_OK:
        raise SkvqError(rc)
    return [int(x) for x in out]


def skvq_paged_validate_config(cfg: skvq_paged_config) -> int:
    return int(lib().skvq_paged_validate_config(C.byref(cfg)))


class SkvqPagedCache:
    """One layer's paged cache: owns the library handle and the device buffers (or adopts those of `buffers`, a dict of
    tensors under the names of skvq_paged_buffers; the others are allocated)."""

    def __init__(self, n_q_heads, n_kv_heads, group_size, window, page_size, n_pages, max_seqs, max_tokens, perm_k, perm_v,
                 clip_k, clip_v, sm_scale=0.0, k_bits=4.0, v_bits=4.0, n_sink=0, meta="f16", dtype=torch.float16,
                 device="cuda:0", buffers=None):
        self.cfg, self._keep = make_paged_config(n_q_heads, n_kv_heads, group_size, window, page_size, n_pages, max_seqs,
                                                 max_tokens, perm_k, perm_v, clip_k, clip_v, sm_scale, k_bits, v_bits,
                                                 n_sink=n_sink, meta=meta, dtype=dtype)
        self.heads, self.dtype = (n_q_heads, n_kv_heads), dtype
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.sizes = skvq_paged_sizes(self.cfg)
        self.buffers = {}
        for name, nbytes in zip(PAGED_BUFFER_NAMES, self.sizes):
            t = (buffers or {}).get(name)
            if t is None:
                t = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            elif t.device != self.device or not t.is_contiguous() or t.numel() * t.element_size() != nbytes:
                raise ValueError(f"buffer {name} must be a contiguous tensor of {nbytes} bytes on {self.device}")
            self.buffers[name] = t
        bufs = skvq_paged_buffers(*[self.buffers[n].data_ptr() for n in PAGED_BUFFER_NAMES])
        handle = C.c_void_p()
        with torch.cuda.device(self.device):
            rc = lib().skvq_paged_create(C.byref(self.cfg), C.byref(bufs), C.byref(handle))
        if rc != SKVQ_OK:
            raise SkvqError(rc)
        self._h = handle

    def close(self):
        if getattr(self, "_h", None):
            lib().skvq_paged_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc):
        if rc != SKVQ_OK:
            raise SkvqError(rc, lib().skvq_paged_last_error(self._h).decode())

    def _rows(self, t: torch.Tensor, n: int, heads: int) -> tuple[int, int]:
        """(address, elements between tokens) of rows [n][heads][D] whose heads lie one after the other."""
        stride = t.stride()
        if t.dtype != self.dtype or t.device != self.device or t.shape != (n, heads, HEAD_DIM) or (
                n and (stride[2] != 1 or (stride[1] != HEAD_DIM and heads > 1))):
            raise ValueError(f"expected {self.dtype} rows [{n}][{heads}][{HEAD_DIM}] on {self.device}, heads contiguous, got "
                             f"{t.dtype} {tuple(t.shape)} on {t.device}, strides {stride}")
        # (the stride of a dimension of one token says nothing)
        return t.data_ptr(), stride[0] if n > 1 else heads * HEAD_DIM

    def _batch(self, batch: SkvqBatch):
        if batch.device != self.device:
            raise ValueError(f"the batch is on {batch.device}, the cache on {self.device}")
        return batch.address, batch.n_tokens

    def _new(self, n: int, heads: int, dtype=None):
        return torch.empty((n, heads, HEAD_DIM), dtype=dtype or self.dtype, device=self.device)

    def skvq_paged_append(self, batch: SkvqBatch, k: torch.Tensor, v: torch.Tensor, rope: SkvqRope | None = None,
                          q: torch.Tensor | None = None, out_q: torch.Tensor | None = None, stream=None):
        """k, v [n_tokens][Hk][D]: the batch's new tokens.  With q [n_tokens][Hq][D] returns its rotated rows (in out_q,
        which may be q)."""
        bp, n = self._batch(batch)
        kp, vp = self._rows(k, n, self.heads[1]), self._rows(v, n, self.heads[1])
        qp = op = (None, 0)
        if q is not None:
            qp = self._rows(q, n, self.heads[0])
            out_q = self._new(n, self.heads[0]) if out_q is None else out_q
            op = self._rows(out_q, n, self.heads[0])
        self._check(lib().skvq_paged_append(self._h, rope._h if rope is not None else None, bp, *kp, *vp, *qp, *op,
                                            _stream_on(self.device, stream)))
        return out_q

    def skvq_paged_read(self, batch: SkvqBatch, out_k: torch.Tensor | None = None, out_v: torch.Tensor | None = None,
                        stream=None):
        """Cached tokens back as (k, v) [n_tokens][Hk][D]: batch.first's, or each sequence's last ones."""
        bp, n = self._batch(batch)
        out_k = self._new(n, self.heads[1]) if out_k is None else out_k
        out_v = self._new(n, self.heads[1]) if out_v is None else out_v
        self._check(lib().skvq_paged_read(self._h, bp, *self._rows(out_k, n, self.heads[1]), *self._rows(out_v, n, self.heads[1]),
                                          _stream_on(self.device, stream)))
        return out_k, out_v

    def skvq_paged_attention(self, batch: SkvqBatch, q: torch.Tensor, out: torch.Tensor | None = None,
                             out_f32: torch.Tensor | None = None, stream=None) -> torch.Tensor:
        """q [n_tokens][Hq][D]: returns out (allocated unless given; not written where only out_f32 is given)."""
        bp, n = self._batch(batch)
        qp = self._rows(q, n, self.heads[0])
        if out is None and out_f32 is None:
            out = self._new(n, self.heads[0])
        op = self._rows(out, n, self.heads[0]) if out is not None else (None, 0)
        fp = None
        if out_f32 is not None:
            fp = _dev_ptr(out_f32, torch.float32, (n, self.heads[0], HEAD_DIM))
        self._check(lib().skvq_paged_attention(self._h, bp, *qp, *op, fp, _stream_on(self.device, stream)))
        return out if out is not None else out_f32

    def skvq_paged_errors(self, stream=None) -> int:
        """Error bits (SKVQ_PAGED_BAD_*) that the device checks have set since the last call; waits for the stream."""
        bits = C.c_int32()
        self._check(lib().skvq_paged_errors(self._h, C.byref(bits), _stream_on(self.device, stream)))
        return bits.value
