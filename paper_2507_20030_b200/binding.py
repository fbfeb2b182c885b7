"""ctypes binding of libfaedkv.so: the same names as include/faedkv.h.

Argument marshalling only.  Every step of the path runs in the library's CUDA
kernels; there is no Python or CPU fallback -- if the library is missing or a
call fails, an exception is raised.

Device buffers are torch tensors (PyTorch is used for device memory and
streams only); their ``data_ptr()`` is what crosses the ABI.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# FAEDKV_LIBRARY selects another build of the same library (the checked build, lib/libfaedkv_debug.so)
LIB_PATH = os.environ.get("FAEDKV_LIBRARY") or os.path.join(_HERE, "lib", "libfaedkv.so")

F32, BF16 = 0, 1
PREFILL_AUTO, PREFILL_SIMT, PREFILL_UMMA, PREFILL_FFT = 0, 1, 2, 3
STATE_SUM, STATE_MEAN, STATE_ROTATING = 0, 1, 2
DECODE_AUTO, DECODE_SIMT, DECODE_UMMA, DECODE_FFT, DECODE_FFT_TWO_PASS = 0, 1, 2, 3, 4

EXPORTS = [
    "faedkv_create", "faedkv_destroy", "faedkv_last_error", "faedkv_plan", "faedkv_n_bins",
    "faedkv_get_bins", "faedkv_coef_bytes", "faedkv_mask_lowpass", "faedkv_mask_mixed",
    "faedkv_compress_prefill", "faedkv_append", "faedkv_reconstruct", "faedkv_decode_attn",
    "faedkv_append_decode_attn", "faedkv_chunk_range", "faedkv_ablation_bins", "faedkv_mask_from_scores", "faedkv_ablate",
    "faedkv_convert_state", "faedkv_window_bytes", "faedkv_prefill_windowed", "faedkv_step_windowed",
    "faedkv_reconstruct_windowed",
    "faedkv_device_status", "faedkv_launch_count", "faedkv_decode_attn_static",
    "faedkv_reset_device_status", "faedkv_test_hooks", "faedkv_debug_build", "faedkv_debug_word",
    "faedkv_pages_create", "faedkv_pages_destroy", "faedkv_pages_last_error", "faedkv_pages_bytes", "faedkv_pages_tables_bytes", "faedkv_pages_tables",
    "faedkv_pages_fork_bytes", "faedkv_pages_fork", "faedkv_pages_release_bytes", "faedkv_pages_release", "faedkv_pages_compact_bytes",
    "faedkv_pages_compact", "faedkv_pages_store", "faedkv_pages_attn_bytes", "faedkv_pages_attn", "faedkv_pages_attn_diff_bytes", "faedkv_pages_attn_diff",
    "faedkv_pages_attn_shared_bytes", "faedkv_pages_attn_shared",
    "faedkv_pages_load", "faedkv_pages_device_status",
    "faedkv_pages_reset_device_status", "faedkv_pages_launch_count", "faedkv_pages_test_hooks", "faedkv_pages_test_cluster", "faedkv_pages_debug_word",
]

STATIC_SCRATCH_BYTES = 8 << 20


class FaedkvError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"faedkv error {code}: {msg}")
        self.code = code


class Config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in (
        "n_layers", "n_kv_heads", "n_q_heads", "head_dim", "n_dft", "max_batch", "kv_dtype",
        "prefill_mode", "twiddle_terms", "decode_mode", "n_sink", "n_recent", "n_defer", "recon_engine")]


class PagesConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in (
        "n_kv_heads", "n_q_heads", "head_dim", "page_size", "n_pages", "max_pages", "max_batch", "kv_dtype")]


_lib = None
_vp = ctypes.c_void_p
_int = ctypes.c_int


def load() -> ctypes.CDLL:
    """Load the library (built by `python -m paper_2507_20030_b200.build`); fails loudly if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2507_20030_b200.build` "
            "(there is no fallback path)")
    lib = ctypes.CDLL(LIB_PATH)
    lib.faedkv_create.argtypes = [ctypes.POINTER(Config), ctypes.POINTER(_vp)]
    lib.faedkv_create.restype = _int
    lib.faedkv_destroy.argtypes = [_vp]
    lib.faedkv_destroy.restype = None
    lib.faedkv_last_error.argtypes = [_vp]
    lib.faedkv_last_error.restype = ctypes.c_char_p
    lib.faedkv_plan.argtypes = [_vp, _int, _vp, ctypes.POINTER(_int)]
    lib.faedkv_plan.restype = _int
    lib.faedkv_n_bins.argtypes = [_vp, _int]
    lib.faedkv_n_bins.restype = _int
    lib.faedkv_get_bins.argtypes = [_vp, _int, _vp]
    lib.faedkv_get_bins.restype = _int
    lib.faedkv_coef_bytes.argtypes = [_vp, _int, _int]
    lib.faedkv_coef_bytes.restype = ctypes.c_size_t
    lib.faedkv_mask_lowpass.argtypes = [_int, _int, _vp]
    lib.faedkv_mask_lowpass.restype = _int
    lib.faedkv_mask_mixed.argtypes = [_int, _int, _int, ctypes.c_uint64, _vp]
    lib.faedkv_mask_mixed.restype = _int
    lib.faedkv_compress_prefill.argtypes = [_vp, _int, _vp, _vp, _int, _int, _vp, _vp, _vp, _vp]
    lib.faedkv_compress_prefill.restype = _int
    lib.faedkv_append.argtypes = [_vp, _int, _vp, _vp, _int, _vp, _vp, _vp, _vp]
    lib.faedkv_append.restype = _int
    lib.faedkv_reconstruct.argtypes = [_vp, _int, _vp, _vp, _vp, _int, _int, _vp, _vp, _vp]
    lib.faedkv_reconstruct.restype = _int
    lib.faedkv_decode_attn.argtypes = [_vp, _int, _vp, _vp, _vp, _vp, _int, ctypes.c_float, _vp, _vp]
    lib.faedkv_decode_attn.restype = _int
    lib.faedkv_append_decode_attn.argtypes = [_vp, _int, _vp, _vp, _vp, _int, _vp, _vp, _vp, ctypes.c_float, _vp, _vp]
    lib.faedkv_append_decode_attn.restype = _int
    lib.faedkv_chunk_range.argtypes = [_int, _int, _int, ctypes.POINTER(_int), ctypes.POINTER(_int)]
    lib.faedkv_chunk_range.restype = _int
    lib.faedkv_ablation_bins.argtypes = [_int, _int, _int, _vp, _vp]
    lib.faedkv_ablation_bins.restype = _int
    lib.faedkv_mask_from_scores.argtypes = [_int, _int, _vp, ctypes.c_double, _vp, ctypes.POINTER(_int)]
    lib.faedkv_mask_from_scores.restype = _int
    lib.faedkv_ablate.argtypes = [_vp, _int, _vp, _vp, _int, _int, _vp, _vp, _vp, _vp, _vp, _vp, _vp]
    lib.faedkv_ablate.restype = _int
    lib.faedkv_convert_state.argtypes = [_vp, _int, _vp, _vp, _int, _int, _int, _vp, _vp]
    lib.faedkv_convert_state.restype = _int
    lib.faedkv_window_bytes.argtypes = [_vp, _int]
    lib.faedkv_window_bytes.restype = ctypes.c_size_t
    lib.faedkv_prefill_windowed.argtypes = [_vp, _int, _vp, _vp, _int, _int, _vp, _vp, _vp, _vp, _vp, _vp]
    lib.faedkv_prefill_windowed.restype = _int
    lib.faedkv_step_windowed.argtypes = [_vp, _int, _vp, _vp, _vp, _int, _vp, _vp, _vp, _vp, _vp, ctypes.c_float, _vp, _vp]
    lib.faedkv_step_windowed.restype = _int
    lib.faedkv_reconstruct_windowed.argtypes = [_vp, _int, _vp, _vp, _vp, _vp, _vp, _int, _int, _vp, _vp, _vp]
    lib.faedkv_reconstruct_windowed.restype = _int
    lib.faedkv_device_status.argtypes = [_vp, _vp]
    lib.faedkv_device_status.restype = _int
    lib.faedkv_decode_attn_static.argtypes = [_int, _int, _int, _int, _vp, _int, _vp, _vp, _vp, _vp, _int,
                                              ctypes.c_float, _vp, _vp, ctypes.c_char_p, ctypes.c_size_t]
    lib.faedkv_decode_attn_static.restype = _int
    lib.faedkv_launch_count.argtypes = [_vp]
    lib.faedkv_launch_count.restype = ctypes.c_ulonglong
    lib.faedkv_reset_device_status.argtypes = [_vp, _vp]
    lib.faedkv_reset_device_status.restype = _int
    lib.faedkv_test_hooks.argtypes = [_vp, ctypes.c_ulonglong, _int]
    lib.faedkv_test_hooks.restype = _int
    lib.faedkv_debug_build.argtypes = []
    lib.faedkv_debug_build.restype = _int
    lib.faedkv_debug_word.argtypes = [_vp, _vp]
    lib.faedkv_debug_word.restype = ctypes.c_longlong
    _ll = ctypes.c_longlong
    lib.faedkv_pages_create.argtypes = [ctypes.POINTER(PagesConfig), ctypes.POINTER(_vp)]
    lib.faedkv_pages_create.restype = _int
    lib.faedkv_pages_destroy.argtypes = [_vp]
    lib.faedkv_pages_destroy.restype = None
    lib.faedkv_pages_last_error.argtypes = [_vp]
    lib.faedkv_pages_last_error.restype = ctypes.c_char_p
    lib.faedkv_pages_bytes.argtypes = [_vp]
    lib.faedkv_pages_bytes.restype = ctypes.c_size_t
    lib.faedkv_pages_tables_bytes.argtypes = [_vp, _int, _int]
    lib.faedkv_pages_tables_bytes.restype = ctypes.c_size_t
    lib.faedkv_pages_tables.argtypes = [_vp, _vp, _vp, _int, _vp, _vp, _vp, _int, _vp, _vp, _vp, _vp, _vp, _vp]
    lib.faedkv_pages_tables.restype = _int
    lib.faedkv_pages_store.argtypes = [_vp, _vp, _vp, _ll, _vp, _int, _vp, _vp, _vp, _vp, _vp]
    lib.faedkv_pages_store.restype = _int
    lib.faedkv_pages_attn_bytes.argtypes = [_vp, _int, _int]
    lib.faedkv_pages_attn_bytes.restype = ctypes.c_size_t
    lib.faedkv_pages_attn.argtypes = [_vp, _vp, _ll, _vp, _int, _int, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_float, _vp, _vp,
                                      ctypes.c_size_t, _vp]
    lib.faedkv_pages_attn.restype = _int
    lib.faedkv_pages_attn_shared_bytes.argtypes = [_vp, _int, _int]
    lib.faedkv_pages_attn_shared_bytes.restype = ctypes.c_size_t
    lib.faedkv_pages_attn_shared.argtypes = [_vp, _vp, _ll, _vp, _vp, _int, _int, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_float, _vp, _vp,
                                             ctypes.c_size_t, _vp]
    lib.faedkv_pages_attn_shared.restype = _int
    lib.faedkv_pages_attn_diff_bytes.argtypes = [_vp, _int, _int]
    lib.faedkv_pages_attn_diff_bytes.restype = ctypes.c_size_t
    lib.faedkv_pages_attn_diff.argtypes = [_vp, _vp, _ll, _vp, _int, _int, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_float, _vp, _vp,
                                           ctypes.c_float, _vp, _vp, ctypes.c_size_t, _vp]
    lib.faedkv_pages_attn_diff.restype = _int
    lib.faedkv_pages_load.argtypes = [_vp, _vp, _vp, _int, _int, _vp, _vp, _vp, _vp, _vp, _vp, _vp]
    lib.faedkv_pages_load.restype = _int
    lib.faedkv_pages_fork_bytes.argtypes = [_vp, _int, _int]
    lib.faedkv_pages_fork_bytes.restype = ctypes.c_size_t
    lib.faedkv_pages_fork.argtypes = [_vp, _vp, _vp, _vp, _int, _int, *[_vp] * 11]
    lib.faedkv_pages_fork.restype = _int
    lib.faedkv_pages_release_bytes.argtypes = [_vp]
    lib.faedkv_pages_release_bytes.restype = ctypes.c_size_t
    lib.faedkv_pages_release.argtypes = [_vp, _vp, _vp, _int, *[_vp] * 7]
    lib.faedkv_pages_release.restype = _int
    lib.faedkv_pages_compact_bytes.argtypes = [_vp]
    lib.faedkv_pages_compact_bytes.restype = ctypes.c_size_t
    lib.faedkv_pages_compact.argtypes = [_vp, _vp, _int, *[_vp] * 11]
    lib.faedkv_pages_compact.restype = _int
    lib.faedkv_pages_device_status.argtypes = [_vp, _vp]
    lib.faedkv_pages_device_status.restype = _int
    lib.faedkv_pages_reset_device_status.argtypes = [_vp, _vp]
    lib.faedkv_pages_reset_device_status.restype = _int
    lib.faedkv_pages_test_hooks.argtypes = [_vp, ctypes.c_ulonglong, _int]
    lib.faedkv_pages_test_hooks.restype = _int
    lib.faedkv_pages_test_cluster.argtypes = [_vp, _int]
    lib.faedkv_pages_test_cluster.restype = _int
    lib.faedkv_pages_debug_word.argtypes = [_vp, _vp]
    lib.faedkv_pages_debug_word.restype = _ll
    lib.faedkv_pages_launch_count.argtypes = [_vp]
    lib.faedkv_pages_launch_count.restype = ctypes.c_ulonglong
    _lib = lib
    return lib


def mask_lowpass(n_dft: int, n_keep: int) -> np.ndarray:
    out = np.zeros(n_dft // 2 + 1, dtype=np.uint8)
    rc = load().faedkv_mask_lowpass(n_dft, n_keep, out.ctypes.data)
    if rc != 0:
        raise FaedkvError(rc, "faedkv_mask_lowpass rejected its arguments")
    return out


def mask_mixed(n_dft: int, n_keep: int, layer: int, seed: int) -> np.ndarray:
    out = np.zeros(n_dft // 2 + 1, dtype=np.uint8)
    rc = load().faedkv_mask_mixed(n_dft, n_keep, layer, seed, out.ctypes.data)
    if rc != 0:
        raise FaedkvError(rc, "faedkv_mask_mixed rejected its arguments")
    return out


def chunk_range(n_dft: int, n_chunks: int, chunk: int) -> tuple[int, int]:
    lo, hi = _int(0), _int(0)
    rc = load().faedkv_chunk_range(n_dft, n_chunks, chunk, ctypes.byref(lo), ctypes.byref(hi))
    if rc != 0:
        raise FaedkvError(rc, "faedkv_chunk_range rejected its arguments")
    return lo.value, hi.value


def ablation_bins(n_dft: int, lo: int, hi: int) -> tuple[np.ndarray, np.ndarray]:
    mask = np.zeros(n_dft // 2 + 1, dtype=np.uint8)
    gain = np.zeros(n_dft // 2 + 1, dtype=np.float32)
    rc = load().faedkv_ablation_bins(n_dft, lo, hi, mask.ctypes.data, gain.ctypes.data)
    if rc != 0:
        raise FaedkvError(rc, "faedkv_ablation_bins rejected its arguments")
    return mask, gain


def mask_from_scores(n_dft: int, n_chunks: int, delta, ratio: float) -> tuple[np.ndarray, int]:
    d = np.ascontiguousarray(delta, dtype=np.float64)
    if d.shape != (n_chunks,):
        raise ValueError("delta must have one entry per chunk")
    mask = np.zeros(n_dft // 2 + 1, dtype=np.uint8)
    n_keep = _int(0)
    rc = load().faedkv_mask_from_scores(n_dft, n_chunks, d.ctypes.data, float(ratio), mask.ctypes.data, ctypes.byref(n_keep))
    if rc != 0:
        raise FaedkvError(rc, "faedkv_mask_from_scores rejected its arguments")
    return mask, n_keep.value


def decode_attn_static(n_dft: int, n_kv_heads: int, n_q_heads: int, kv_dtype: int, bins, q, coefK, coefV,
                       t_len, out, scale: float = 0.0, stream=None) -> None:
    """faedkv_decode_attn_static: decode attention without a context and without any allocation.

    For callers that cannot allocate device memory where they need attention (inside a stream
    capture, under an external memory pool, in a plugin that only receives tensors).  `bins` is a
    device int32 tensor holding the layer's retained bins.  All intermediates live in a fixed
    array inside the library (STATIC_SCRATCH_BYTES); larger problems raise FaedkvError(-3).
    Calls share that array, so calls that overlap on the GPU must be serialised by the caller."""
    buf = ctypes.create_string_buffer(256)
    rc = load().faedkv_decode_attn_static(
        n_dft, n_kv_heads, n_q_heads, kv_dtype, _ptr(bins), int(bins.numel()), _ptr(q), _ptr(coefK),
        _ptr(coefV), _ptr(t_len), int(q.shape[0]), float(scale), _ptr(out), _stream(stream), buf, 256)
    if rc != 0:
        raise FaedkvError(rc, buf.value.decode())


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    assert t.is_contiguous(), "tensors crossing the ABI must be contiguous"
    return t.data_ptr()


def _stream(stream) -> int | None:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


@dataclass
class Context:
    """Owner of one faedkv_ctx; methods carry the names of the C calls without the prefix."""
    n_layers: int
    n_kv_heads: int
    n_q_heads: int
    n_dft: int
    max_batch: int
    kv_dtype: int = BF16
    head_dim: int = 128
    prefill_mode: int = PREFILL_AUTO
    twiddle_terms: int = 0
    decode_mode: int = DECODE_AUTO
    n_sink: int = 0
    n_recent: int = 0
    n_defer: int = 0
    recon_engine: int = 0

    def __post_init__(self):
        self._lib = load()
        cfg = Config(self.n_layers, self.n_kv_heads, self.n_q_heads, self.head_dim, self.n_dft,
                     self.max_batch, self.kv_dtype, self.prefill_mode, self.twiddle_terms, self.decode_mode,
                     self.n_sink, self.n_recent, self.n_defer, self.recon_engine)
        h = _vp()
        rc = self._lib.faedkv_create(ctypes.byref(cfg), ctypes.byref(h))
        if rc != 0:
            raise FaedkvError(rc, "faedkv_create failed")
        self._h = h

    # -- lifetime
    def close(self):
        if getattr(self, "_h", None):
            self._lib.faedkv_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc: int):
        if rc != 0:
            raise FaedkvError(rc, self._lib.faedkv_last_error(self._h).decode())

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.kv_dtype == BF16 else torch.float32

    # -- plan
    def plan(self, layer: int, bin_mask: np.ndarray) -> int:
        mask = np.ascontiguousarray(bin_mask, dtype=np.uint8)
        if mask.shape != (self.n_dft // 2 + 1,):
            raise ValueError("bin_mask must have length n_dft // 2 + 1")
        n = _int(0)
        self._check(self._lib.faedkv_plan(self._h, layer, mask.ctypes.data, ctypes.byref(n)))
        return n.value

    def n_bins(self, layer: int) -> int:
        m = self._lib.faedkv_n_bins(self._h, layer)
        if m < 0:
            raise FaedkvError(m, "layer not planned")
        return m

    def get_bins(self, layer: int) -> np.ndarray:
        out = np.zeros(self.n_bins(layer), dtype=np.int32)
        self._check(self._lib.faedkv_get_bins(self._h, layer, out.ctypes.data))
        return out

    def coef_bytes(self, layer: int, batch: int) -> int:
        return int(self._lib.faedkv_coef_bytes(self._h, layer, batch))

    def alloc_coef(self, layer: int, batch: int, device="cuda") -> torch.Tensor:
        """float32 [batch, n_kv_heads, 2, M, head_dim] (uninitialised)."""
        return torch.empty((batch, self.n_kv_heads, 2, self.n_bins(layer), self.head_dim),
                           dtype=torch.float32, device=device)

    # -- the four device calls
    def compress_prefill(self, layer, K, V, coefK, coefV, t_len, stream=None):
        batch, T = K.shape[0], K.shape[2]
        self._check(self._lib.faedkv_compress_prefill(
            self._h, layer, _ptr(K), _ptr(V), batch, T, _ptr(coefK), _ptr(coefV), _ptr(t_len),
            _stream(stream)))

    def append(self, layer, k_new, v_new, coefK, coefV, t_len, stream=None):
        batch = k_new.shape[0]
        self._check(self._lib.faedkv_append(
            self._h, layer, _ptr(k_new), _ptr(v_new), batch, _ptr(coefK), _ptr(coefV), _ptr(t_len),
            _stream(stream)))

    def reconstruct(self, layer, coefK, coefV, t_len, L, K_out, V_out, stream=None):
        batch = t_len.shape[0]
        self._check(self._lib.faedkv_reconstruct(
            self._h, layer, _ptr(coefK), _ptr(coefV), _ptr(t_len), batch, L, _ptr(K_out), _ptr(V_out),
            _stream(stream)))

    def decode_attn(self, layer, q, coefK, coefV, t_len, out, scale: float = 0.0, stream=None):
        batch = q.shape[0]
        self._check(self._lib.faedkv_decode_attn(
            self._h, layer, _ptr(q), _ptr(coefK), _ptr(coefV), _ptr(t_len), batch, float(scale),
            _ptr(out), _stream(stream)))

    def append_decode_attn(self, layer, k_new, v_new, q, coefK, coefV, t_len, out, scale: float = 0.0, stream=None):
        batch = q.shape[0]
        self._check(self._lib.faedkv_append_decode_attn(
            self._h, layer, _ptr(k_new), _ptr(v_new), _ptr(q), batch, _ptr(coefK), _ptr(coefV), _ptr(t_len),
            float(scale), _ptr(out), _stream(stream)))

    def ablate(self, layer, K, V, gain, wsK, wsV, ws_len, K_out, V_out, stream=None):
        batch, T = K.shape[0], K.shape[2]
        self._check(self._lib.faedkv_ablate(
            self._h, layer, _ptr(K), _ptr(V), batch, T, _ptr(gain), _ptr(wsK), _ptr(wsV), _ptr(ws_len),
            _ptr(K_out), _ptr(V_out), _stream(stream)))

    def convert_state(self, layer, coef_in, t_len, from_form, to_form, coef_out=None, stream=None):
        """Stationary sum <-> running mean <-> rotating frame; in place when coef_out is None."""
        coef_out = coef_in if coef_out is None else coef_out
        self._check(self._lib.faedkv_convert_state(
            self._h, layer, _ptr(coef_in), _ptr(t_len), t_len.shape[0], from_form, to_form, _ptr(coef_out),
            _stream(stream)))
        return coef_out

    # -- sink + recent window
    def alloc_window(self, batch: int, device="cuda") -> torch.Tensor:
        """[batch, n_kv_heads, n_sink + ring, head_dim] in the storage type (uninitialised); the ring has
        n_recent slots, or n_recent + n_defer with the block-deferred fold (n_defer >= 2)."""
        ring = self.n_recent + (self.n_defer if self.n_defer > 1 else 0)
        return torch.empty((batch, self.n_kv_heads, self.n_sink + ring, self.head_dim),
                           dtype=self.torch_dtype, device=device)

    def prefill_windowed(self, layer, K, V, coefK, coefV, winK, winV, t_len, stream=None):
        batch, T = K.shape[0], K.shape[2]
        self._check(self._lib.faedkv_prefill_windowed(
            self._h, layer, _ptr(K), _ptr(V), batch, T, _ptr(coefK), _ptr(coefV), _ptr(winK), _ptr(winV),
            _ptr(t_len), _stream(stream)))

    def step_windowed(self, layer, k_new, v_new, q, coefK, coefV, winK, winV, t_len, out, scale: float = 0.0, stream=None):
        batch = q.shape[0]
        self._check(self._lib.faedkv_step_windowed(
            self._h, layer, _ptr(k_new), _ptr(v_new), _ptr(q), batch, _ptr(coefK), _ptr(coefV), _ptr(winK),
            _ptr(winV), _ptr(t_len), float(scale), _ptr(out), _stream(stream)))

    def reconstruct_windowed(self, layer, coefK, coefV, winK, winV, t_len, L: int, K_out=None, V_out=None, stream=None):
        """[sink | reconstructed segment | tokens still in the time domain | zeros] as [batch, n_kv_heads, L, head_dim]."""
        batch = t_len.shape[0]
        shape = (batch, self.n_kv_heads, L, self.head_dim)
        if K_out is None:
            K_out = torch.empty(shape, dtype=self.torch_dtype, device=coefK.device)
        if V_out is None:
            V_out = torch.empty(shape, dtype=self.torch_dtype, device=coefK.device)
        self._check(self._lib.faedkv_reconstruct_windowed(
            self._h, layer, _ptr(coefK), _ptr(coefV), _ptr(winK), _ptr(winV), _ptr(t_len), batch, L, _ptr(K_out),
            _ptr(V_out), _stream(stream)))
        return K_out, V_out

    def launch_count(self) -> int:
        return int(self._lib.faedkv_launch_count(self._h))

    def device_status(self, stream=None) -> int:
        return int(self._lib.faedkv_device_status(self._h, _stream(stream)))

    def debug_word(self, stream=None) -> int:
        """faedkv_debug_word: first failed bounds check of the checked build since the last call (0: none)."""
        return int(self._lib.faedkv_debug_word(self._h, _stream(stream)))

    def reset_device_status(self, stream=None):
        self._check(self._lib.faedkv_reset_device_status(self._h, _stream(stream)))

    def test_hooks(self, wait_limit_ns: int = 0, withhold_step: int = 0):
        """faedkv_test_hooks: wait limit of the tensor-core prefill's bounded waits and the withheld-signal test."""
        self._check(self._lib.faedkv_test_hooks(self._h, int(wait_limit_ns), int(withhold_step)))


# the current stream's handle without building a Stream object (1 us a call)
_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda index: torch.cuda.current_stream(index).cuda_stream)


@dataclass
class Pages:
    """The paged 8-bit cache (faedkv_pages): methods carry the names of the C calls without the prefix.

    Shapes are checked here, since a wrong one would read or write past a tensor: a ValueError names the tensor.  Workspaces
    that a call needs are taken from PyTorch's allocator on the call's stream unless the caller passes one."""
    n_kv_heads: int
    n_q_heads: int
    page_size: int
    n_pages: int
    max_pages: int
    max_batch: int
    kv_dtype: int = BF16
    head_dim: int = 128

    def __post_init__(self):
        self._lib = load()
        cfg = PagesConfig(self.n_kv_heads, self.n_q_heads, self.head_dim, self.page_size, self.n_pages, self.max_pages,
                          self.max_batch, self.kv_dtype)
        h = _vp()
        rc = self._lib.faedkv_pages_create(ctypes.byref(cfg), ctypes.byref(h))
        if rc != 0:
            raise FaedkvError(rc, "faedkv_pages_create failed")
        self._h = h
        self.device = torch.device("cuda", torch.cuda.current_device())
        self._shapes()

    # -- lifetime
    def close(self):
        if getattr(self, "_h", None):
            self._lib.faedkv_pages_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc: int):
        if rc != 0:
            raise FaedkvError(rc, self._lib.faedkv_pages_last_error(self._h).decode())

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.kv_dtype == BF16 else torch.float32

    def _shapes(self):
        """What the checks compare with, worked out once: a decode step's calls are short enough for it to show."""
        self._index = -1 if self.device.type == "cpu" else self.device.index
        self._dtype = torch.bfloat16 if self.kv_dtype == BF16 else torch.float32
        self._scale_shape = (self.n_pages, self.n_kv_heads)
        self._code_shape = (*self._scale_shape, self.page_size, self.head_dim)
        self._pool_shape = (self.n_pages,)
        self._attn_bytes = {}

    def _refuse(self, name, t, dtype, shape):
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {shape} on {self.device}, got {t.dtype} {tuple(t.shape)} "
                         f"with strides {t.stride()} on {t.device}")

    def _need(self, name, t, dtype, shape):
        if t.dtype is not dtype or t.shape != shape or t.get_device() != self._index or not t.is_contiguous():
            self._refuse(name, t, dtype, shape)
        return t.data_ptr()

    def _rows(self, name, t, heads):
        """Token rows [n_tokens, heads, head_dim], contiguous from the head on: pointer, tokens, row stride in elements."""
        if t.dtype is not self._dtype or t.get_device() != self._index:
            raise ValueError(f"{name} must be {self._dtype} on {self.device}, got {t.dtype} on {t.device}")
        shape = t.shape
        if len(shape) != 3 or shape[1] != heads or shape[2] != self.head_dim:
            raise ValueError(f"{name} must have shape [n_tokens, {heads}, {self.head_dim}], got {tuple(shape)}")
        n, row = shape[0], heads * self.head_dim
        if t.is_contiguous():
            return t.data_ptr(), n, row
        st = t.stride()
        if (heads > 1 and st[1] != self.head_dim) or st[2] != 1 or (n > 1 and st[0] < row):
            raise ValueError(f"{name}: heads and channels must be contiguous within a token row, strides {st}")
        return t.data_ptr(), n, (st[0] if n > 1 else row)

    def _cache(self, k_pages, v_pages, k_scale, v_scale):
        need, f8, f32 = self._need, torch.float8_e4m3fn, torch.float32
        return (need("k_pages", k_pages, f8, self._code_shape), need("v_pages", v_pages, f8, self._code_shape),
                need("k_scale", k_scale, f32, self._scale_shape), need("v_scale", v_scale, f32, self._scale_shape))

    def _workspace(self, ws, nbytes, stream):
        if ws is not None:
            if not ws.is_contiguous() or ws.get_device() != self._index or ws.numel() * ws.element_size() < nbytes:
                raise ValueError(f"ws must be a contiguous tensor of at least {nbytes} bytes on {self.device}")
            return ws
        return self._empty(nbytes, torch.uint8, stream)

    def _empty(self, shape, dtype, stream):
        """Memory of the call's stream: the allocator may hand out again what the current stream is still working on."""
        if stream is None:
            return torch.empty(shape, dtype=dtype, device=self.device)
        s = torch.cuda.ExternalStream(stream, device=self.device) if isinstance(stream, int) else stream
        with torch.cuda.stream(s):
            return torch.empty(shape, dtype=dtype, device=self.device)

    def _on(self, stream):
        """The stream's handle; by default the current stream of the handle's device."""
        if stream is None:
            return _current_raw_stream(self._index)
        return stream if isinstance(stream, int) else stream.cuda_stream

    def alloc(self):
        """k_pages, v_pages (torch.float8_e4m3fn [n_pages, n_kv_heads, page_size, head_dim]), k_scale, v_scale (float32
        [n_pages, n_kv_heads]), all uninitialised."""
        codes = [torch.empty(self._code_shape, dtype=torch.float8_e4m3fn, device=self.device) for _ in range(2)]
        scales = [torch.empty(self._scale_shape, dtype=torch.float32, device=self.device) for _ in range(2)]
        return (*codes, *scales)

    # -- the calls
    def tables(self, t_len, n_new, table, free_pages, n_free, q_start, kv_len, slots, n_free_out, ws=None, stream=None):
        batch, i32, need = t_len.shape[0], torch.int32, self._need
        per_seq, one, n_tokens = (batch,), (1,), slots.numel()
        args = (need("t_len", t_len, i32, per_seq), need("n_new", n_new, i32, per_seq), batch,
                need("table", table, i32, (batch, self.max_pages)), need("free_pages", free_pages, i32, self._pool_shape),
                need("n_free", n_free, i32, one), n_tokens, need("q_start", q_start, i32, (batch + 1,)),
                need("kv_len", kv_len, i32, per_seq), need("slots", slots, i32, (n_tokens,)), need("n_free_out", n_free_out, i32, one))
        nbytes = self._lib.faedkv_pages_tables_bytes(self._h, batch, n_tokens)
        w = self._workspace(ws, nbytes, stream) if nbytes else None
        self._check(self._lib.faedkv_pages_tables(self._h, *args, None if w is None else w.data_ptr(), self._on(stream)))

    def store(self, k_new, v_new, slots, k_pages, v_pages, k_scale, v_scale, stream=None):
        k, n, ld = self._rows("k_new", k_new, self.n_kv_heads)
        v, nv, ldv = self._rows("v_new", v_new, self.n_kv_heads)
        if nv != n or ldv != ld:
            raise ValueError(f"k_new and v_new must have the same tokens and row stride, got {n}, {nv} tokens, strides {ld}, {ldv}")
        s = self._need("slots", slots, torch.int32, (n,))
        self._check(self._lib.faedkv_pages_store(self._h, k, v, ld, s, n, *self._cache(k_pages, v_pages, k_scale, v_scale),
                                                 self._on(stream)))

    def _bytes(self, call, *counts):
        """A workspace's size, a function of the handle's configuration and the counts alone, so it is asked for once."""
        key = (call, counts)
        size = self._attn_bytes.get(key)
        if size is None:
            if len(self._attn_bytes) > 4096:
                self._attn_bytes.clear()
            size = self._attn_bytes[key] = getattr(self._lib, call)(self._h, *counts)
        return size

    def attn_bytes(self, batch: int, n_tokens: int) -> int:
        """Workspace of attn()."""
        return self._bytes("faedkv_pages_attn_bytes", batch, n_tokens)

    def attn_shared_bytes(self, batch: int, n_groups: int) -> int:
        """Workspace of attn_shared()."""
        return self._bytes("faedkv_pages_attn_shared_bytes", batch, n_groups)

    def attn_diff_bytes(self, batch: int, n_tokens: int) -> int:
        """Workspace of attn_diff()."""
        return self._bytes("faedkv_pages_attn_diff_bytes", batch, n_tokens)

    def attn(self, q, kv_len, table, k_pages, v_pages, k_scale, v_scale, out, q_start=None, scale: float = 0.0, ws=None, stream=None):
        batch, i32, need = kv_len.shape[0], torch.int32, self._need
        qp, n, ld = self._rows("q", q, self.n_q_heads)
        o = need("out", out, self._dtype, (n, self.n_q_heads, self.head_dim))
        st = None if q_start is None else need("q_start", q_start, i32, (batch + 1,))
        kv = need("kv_len", kv_len, i32, (batch,))
        tb = need("table", table, i32, (batch, self.max_pages))
        cache = self._cache(k_pages, v_pages, k_scale, v_scale)
        nbytes = self.attn_bytes(batch, n)
        w = self._workspace(ws, nbytes, stream)
        self._check(self._lib.faedkv_pages_attn(self._h, qp, ld, st, n, batch, kv, tb, *cache, scale, o, w.data_ptr(), nbytes,
                                                self._on(stream)))

    def attn_shared(self, q, kv_len, table, group_start, shared_len, k_pages, v_pages, k_scale, v_scale, out, scale: float = 0.0, ws=None,
                    stream=None):
        """attn() of one new token of every row, where the rows of a group hold their first shared_len[g] tokens in the same pages."""
        batch, groups, i32, need = kv_len.shape[0], shared_len.shape[0], torch.int32, self._need
        qp, n, ld = self._rows("q", q, self.n_q_heads)
        if n != batch:
            raise ValueError(f"q must have one token for each of {batch} rows, got {n}")
        o = need("out", out, self._dtype, (n, self.n_q_heads, self.head_dim))
        kv = need("kv_len", kv_len, i32, (batch,))
        tb = need("table", table, i32, (batch, self.max_pages))
        gs, sl = need("group_start", group_start, i32, (groups + 1,)), need("shared_len", shared_len, i32, (groups,))
        cache = self._cache(k_pages, v_pages, k_scale, v_scale)
        nbytes = self.attn_shared_bytes(batch, groups)
        w = self._workspace(ws, nbytes, stream)
        self._check(self._lib.faedkv_pages_attn_shared(self._h, qp, ld, gs, sl, groups, batch, kv, tb, *cache, scale, o, w.data_ptr(), nbytes,
                                                       self._on(stream)))

    def attn_diff(self, q, kv_len, table, k_pages, v_pages, k_scale, v_scale, lam, out, q_start=None, gain=None, eps: float = 0.0,
                  scale: float = 0.0, ws=None, stream=None):
        """Differential attention: softmax over the first 64 channels minus lam times softmax over the last 64, normalised where a gain
        is given."""
        batch, i32, f32, need = kv_len.shape[0], torch.int32, torch.float32, self._need
        qp, n, ld = self._rows("q", q, self.n_q_heads)
        o = need("out", out, self._dtype, (n, self.n_q_heads, self.head_dim))
        st = None if q_start is None else need("q_start", q_start, i32, (batch + 1,))
        kv = need("kv_len", kv_len, i32, (batch,))
        tb = need("table", table, i32, (batch, self.max_pages))
        lm = need("lam", lam, f32, (self.n_q_heads,))
        gn = None if gain is None else need("gain", gain, f32, (self.head_dim,))
        cache = self._cache(k_pages, v_pages, k_scale, v_scale)
        nbytes = self.attn_diff_bytes(batch, n)
        w = self._workspace(ws, nbytes, stream)
        self._check(self._lib.faedkv_pages_attn_diff(self._h, qp, ld, st, n, batch, kv, tb, *cache, scale, lm, gn, eps, o, w.data_ptr(),
                                                     nbytes, self._on(stream)))

    def load(self, kv_len, table, k_pages, v_pages, k_scale, v_scale, L: int, K_out=None, V_out=None, stream=None):
        """K, V rows [batch, n_kv_heads, L, head_dim], zero behind each sequence's end.  What is not given is allocated on the call's
        stream.  Without k_pages and k_scale, or without v_pages and v_scale (None), only the other one is read back."""
        batch, need = kv_len.shape[0], self._need
        shape = (batch, self.n_kv_heads, L, self.head_dim)
        kv = need("kv_len", kv_len, torch.int32, (batch,))
        tb = need("table", table, torch.int32, (batch, self.max_pages))
        out, ptrs = [], []
        for which, codes, scale, rows in (("k", k_pages, k_scale, K_out), ("v", v_pages, v_scale, V_out)):
            if codes is None and scale is None and rows is None:
                out.append(None)
                ptrs.append((None, None, None))
                continue
            if codes is None or scale is None:
                raise ValueError(f"{which}_pages and {which}_scale go together" + ("" if rows is None else f", and with {which.upper()}_out"))
            c = need(which + "_pages", codes, torch.float8_e4m3fn, self._code_shape)
            s = need(which + "_scale", scale, torch.float32, self._scale_shape)
            if rows is None:
                rows = self._empty(shape, self.torch_dtype, stream)
            out.append(rows)
            ptrs.append((c, s, need(which.upper() + "_out", rows, self._dtype, shape)))
        (kc, ks, ko), (vc, vs, vo) = ptrs
        if kc is None and vc is None:
            raise ValueError("neither K nor V to read back")
        self._check(self._lib.faedkv_pages_load(self._h, kv, tb, batch, L, kc, vc, ks, vs, ko, vo, self._on(stream)))
        return tuple(out)

    # -- pages that several requests share
    def fork(self, src, dst, kv_len, table, free_pages, n_free, n_free_out, k_pages, v_pages, k_scale, v_scale, length=None, ws=None,
             stream=None):
        """Rows dst begin as copies of the first `length` tokens (all of them without it) of rows src; kv_len and table in place."""
        n, batch, i32, need = src.numel(), kv_len.shape[0], torch.int32, self._need
        args = (need("src", src, i32, (n,)), need("dst", dst, i32, (n,)), None if length is None else need("length", length, i32, (n,)), n, batch,
                need("kv_len", kv_len, i32, (batch,)), need("table", table, i32, (batch, self.max_pages)),
                need("free_pages", free_pages, i32, self._pool_shape), need("n_free", n_free, i32, (1,)),
                need("n_free_out", n_free_out, i32, (1,)), *self._cache(k_pages, v_pages, k_scale, v_scale))
        nbytes = self._bytes("faedkv_pages_fork_bytes", batch, n)
        w = self._workspace(ws, nbytes, stream) if nbytes else None
        self._check(self._lib.faedkv_pages_fork(self._h, *args, None if w is None else w.data_ptr(), self._on(stream)))

    def release(self, t_len, n_new, table, free_pages, n_free, kv_len, n_free_out, ws=None, stream=None):
        """Requests with n_new < 0 give back the pages that no other request names."""
        batch, i32, need = t_len.shape[0], torch.int32, self._need
        args = (need("t_len", t_len, i32, (batch,)), need("n_new", n_new, i32, (batch,)), batch,
                need("table", table, i32, (batch, self.max_pages)), need("free_pages", free_pages, i32, self._pool_shape),
                need("n_free", n_free, i32, (1,)), need("kv_len", kv_len, i32, (batch,)), need("n_free_out", n_free_out, i32, (1,)))
        w = self._workspace(ws, self._bytes("faedkv_pages_release_bytes"), stream)
        self._check(self._lib.faedkv_pages_release(self._h, *args, w.data_ptr(), self._on(stream)))

    def compact(self, kv_len, table, table_out, free_pages, n_free, new_id, k_pages, v_pages, k_scale, v_scale, ws=None, stream=None):
        """The pages in use to the front of the pool; free_pages, n_free and new_id are written, table_out may be table."""
        batch, i32, need = kv_len.shape[0], torch.int32, self._need
        rows = (batch, self.max_pages)
        args = (need("kv_len", kv_len, i32, (batch,)), batch, need("table", table, i32, rows), need("table_out", table_out, i32, rows),
                need("free_pages", free_pages, i32, self._pool_shape), need("n_free", n_free, i32, (1,)),
                need("new_id", new_id, i32, self._pool_shape), *self._cache(k_pages, v_pages, k_scale, v_scale))
        w = self._workspace(ws, self._bytes("faedkv_pages_compact_bytes"), stream)
        self._check(self._lib.faedkv_pages_compact(self._h, *args, w.data_ptr(), self._on(stream)))

    def launch_count(self) -> int:
        return int(self._lib.faedkv_pages_launch_count(self._h))

    def device_status(self, stream=None) -> int:
        return int(self._lib.faedkv_pages_device_status(self._h, self._on(stream)))

    def reset_device_status(self, stream=None):
        self._check(self._lib.faedkv_pages_reset_device_status(self._h, self._on(stream)))

    def test_hooks(self, wait_limit_ns: int = 0, withhold_tile: int = 0):
        """faedkv_pages_test_hooks: wait limit of the attention's bounded waits and the withheld-signal test."""
        self._check(self._lib.faedkv_pages_test_hooks(self._h, int(wait_limit_ns), int(withhold_tile)))

    def test_cluster(self, most: int = 0):
        """faedkv_pages_test_cluster: release and compact with clusters of eight CTAs."""
        self._check(self._lib.faedkv_pages_test_cluster(self._h, int(most)))

    def debug_word(self, stream=None) -> int:
        return int(self._lib.faedkv_pages_debug_word(self._h, self._on(stream)))
