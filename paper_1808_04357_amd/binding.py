"""ctypes binding of librgc.so -- argument marshalling only.

Names follow include/rgc.h (and include/rgc_diag.h for the diagnostics).  Tensors are anything with ``data_ptr()`` / ``numel()``
(PyTorch-ROCm tensors on the GPU); streams are raw ``hipStream_t`` values
(``torch.cuda.current_stream().cuda_stream``), ``None`` = the null stream.
"""
from __future__ import annotations

import ctypes
import os
from typing import List, Optional, Sequence

RGC_OK = 0
RGC_EINVAL = -1
RGC_ENOMEM = -2
RGC_EHIP = -3
RGC_EINTERNAL = -4
RGC_NO_MOMENTUM_MASK = 0x1
RGC_NO_HINTS = 0x2
RGC_NESTEROV = 0x4
RGC_OVERWRITE = 0x10
RGC_ADD_TO_DST = 0x20
RGC_VALIDATE = 0x40
RGC_ONE_VALUE = 0x80
RGC_SELECT_LARGEST = 0x100
RGC_SELECT_SMALLEST = 0x200
RGC_THRESHOLD_SEARCH = 0x400
RGC_STATUS_INDEX_RANGE = 0x1
RGC_STATUS_INDEX_ORDER = 0x2
RGC_F32 = 0
RGC_BF16 = 1
RGC_F16 = 2
RGC_TOP_MAX = 128
RGC_RECURRENCE_CHUNK = 256
RGC_SCAN_CHUNK = 32
RGC_SCAN_STATES_MAX = 64
RGC_TAPS_MAX = 8

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "librgc.so")

EXPORTS = ["rgc_create", "rgc_destroy", "rgc_k_for_density", "rgc_compress_layers",
           "rgc_compress_layers_scaled", "rgc_clip_coefficient", "rgc_message_means", "rgc_message_means_noalloc",
           "rgc_compress_layers_threshold",
           "rgc_token_logprobs", "rgc_token_logprobs_backward", "rgc_distill_loss", "rgc_gated_recurrence",
           "rgc_gated_recurrence_backward",
           "rgc_embed_tokens", "rgc_embed_tokens_backward", "rgc_causal_convolution", "rgc_causal_convolution_backward",
           "rgc_selective_scan", "rgc_selective_scan_backward",
           "rgc_decompress_accumulate", "rgc_reset_hints", "rgc_poison_hints", "rgc_limit_optional_scratch", "rgc_limit_looks", "rgc_selftest",
           "rgc_last_paths", "rgc_last_stats", "rgc_last_error", "rgc_decompress_status", "rgc_profile_enable", "rgc_profile_read", "rgc_stream_yardstick", "rgc_strerror"]


class RgcError(RuntimeError):
    def __init__(self, status: int, text: str):
        super().__init__("rgc status %d: %s" % (status, text))
        self.status = status


class rgc_layer(ctypes.Structure):
    _fields_ = [("grad", ctypes.c_void_p), ("residual", ctypes.c_void_p), ("momentum", ctypes.c_void_p),
                ("n", ctypes.c_int64), ("k", ctypes.c_int32), ("out_idx", ctypes.c_void_p),
                ("out_val", ctypes.c_void_p), ("out_count", ctypes.c_void_p)]


class rgc_msg(ctypes.Structure):
    _fields_ = [("idx", ctypes.c_void_p), ("val", ctypes.c_void_p), ("count", ctypes.c_int32)]


class rgc_token_scores(ctypes.Structure):
    _fields_ = [("logits", ctypes.c_void_p), ("row_stride", ctypes.c_int64), ("rows", ctypes.c_int64),
                ("vocab", ctypes.c_int32), ("dtype", ctypes.c_int32), ("targets", ctypes.c_void_p),
                ("temperature", ctypes.c_float), ("top", ctypes.c_int32), ("logprob", ctypes.c_void_p),
                ("entropy", ctypes.c_void_p), ("stats", ctypes.c_void_p), ("top_idx", ctypes.c_void_p),
                ("top_logprob", ctypes.c_void_p)]


class rgc_distill(ctypes.Structure):
    _fields_ = [("logits", ctypes.c_void_p), ("row_stride", ctypes.c_int64), ("rows", ctypes.c_int64),
                ("vocab", ctypes.c_int32), ("dtype", ctypes.c_int32), ("teacher_idx", ctypes.c_void_p),
                ("teacher_logits", ctypes.c_void_p), ("k", ctypes.c_int32), ("targets", ctypes.c_void_p),
                ("temperature", ctypes.c_float), ("soft_weight", ctypes.c_float), ("label_weight", ctypes.c_float),
                ("grad_loss", ctypes.c_void_p), ("loss", ctypes.c_void_p), ("grad_logits", ctypes.c_void_p),
                ("grad_row_stride", ctypes.c_int64)]


class rgc_sequence(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch_stride", ctypes.c_int64), ("step_stride", ctypes.c_int64)]


class rgc_recurrence(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("steps", ctypes.c_int64), ("width", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("x", rgc_sequence), ("gate", rgc_sequence), ("out_gate", rgc_sequence), ("y", rgc_sequence),
                ("lengths", ctypes.c_void_p), ("resets", ctypes.c_void_p), ("h0", ctypes.c_void_p),
                ("h_last", ctypes.c_void_p), ("states", ctypes.c_void_p)]


class rgc_recurrence_grads(ctypes.Structure):
    _fields_ = [("dy", rgc_sequence), ("dx", rgc_sequence), ("dgate", rgc_sequence), ("dout_gate", rgc_sequence),
                ("dh_last", ctypes.c_void_p), ("dh0", ctypes.c_void_p)]


class rgc_embedding(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("table_stride", ctypes.c_int64), ("vocab", ctypes.c_int32), ("width", ctypes.c_int32),
                ("table_dtype", ctypes.c_int32), ("dtype", ctypes.c_int32), ("tokens", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("scale", ctypes.c_float), ("out", ctypes.c_void_p), ("out_stride", ctypes.c_int64)]


class rgc_convolution(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("steps", ctypes.c_int64), ("width", ctypes.c_int32), ("taps", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("silu", ctypes.c_int32), ("x", rgc_sequence), ("y", rgc_sequence), ("weight", ctypes.c_void_p), ("bias", ctypes.c_void_p),
                ("lengths", ctypes.c_void_p), ("resets", ctypes.c_void_p), ("before", ctypes.c_void_p), ("last", ctypes.c_void_p)]


class rgc_convolution_grads(ctypes.Structure):
    _fields_ = [("dy", rgc_sequence), ("dx", rgc_sequence), ("dweight", ctypes.c_void_p), ("dbias", ctypes.c_void_p), ("dlast", ctypes.c_void_p),
                ("dbefore", ctypes.c_void_p)]


class rgc_scan(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("steps", ctypes.c_int64), ("width", ctypes.c_int32), ("states", ctypes.c_int32), ("groups", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("softplus", ctypes.c_int32), ("x", rgc_sequence), ("delta", rgc_sequence), ("gate", rgc_sequence), ("b", rgc_sequence),
                ("c", rgc_sequence), ("y", rgc_sequence), ("a", ctypes.c_void_p), ("d", ctypes.c_void_p), ("delta_bias", ctypes.c_void_p), ("lengths", ctypes.c_void_p),
                ("resets", ctypes.c_void_p), ("h0", ctypes.c_void_p), ("h_last", ctypes.c_void_p), ("kept", ctypes.c_void_p)]


class rgc_scan_grads(ctypes.Structure):
    _fields_ = [("dy", rgc_sequence), ("dx", rgc_sequence), ("ddelta", rgc_sequence), ("dgate", rgc_sequence), ("db", rgc_sequence), ("dc", rgc_sequence),
                ("da", ctypes.c_void_p), ("dd", ctypes.c_void_p), ("ddelta_bias", ctypes.c_void_p), ("dh_last", ctypes.c_void_p), ("dh0", ctypes.c_void_p)]


_lib = None


def library_path() -> str:
    return _LIB_PATH


def load_library() -> ctypes.CDLL:
    """Load librgc.so; raises if it has not been built (there is no fallback path)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError("librgc.so is not built: run `python -m paper_1808_04357_amd.build` "
                           "(or __graft_entry__.build()) first; there is no CPU fallback")
    # The tensors handed to the library are PyTorch's, so both must talk to ONE HIP runtime: PyTorch's
    # wheel brings its own libamdhip64.so.7, and whichever copy of that soname is mapped first serves the
    # whole process.  Loaded before torch, librgc.so would bind to the system copy and see no device.
    import torch  # noqa: F401
    L = ctypes.CDLL(_LIB_PATH)
    L.rgc_create.restype = ctypes.c_int
    L.rgc_create.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_int, ctypes.c_int64, ctypes.c_int32]
    L.rgc_destroy.restype = ctypes.c_int
    L.rgc_destroy.argtypes = [ctypes.c_void_p]
    L.rgc_k_for_density.restype = ctypes.c_int32
    L.rgc_k_for_density.argtypes = [ctypes.c_int64, ctypes.c_uint32]
    L.rgc_compress_layers.restype = ctypes.c_int
    L.rgc_compress_layers.argtypes = [ctypes.c_void_p, ctypes.POINTER(rgc_layer), ctypes.c_int32,
                                      ctypes.c_float, ctypes.c_uint32, ctypes.c_void_p]
    L.rgc_compress_layers_scaled.restype = ctypes.c_int
    L.rgc_compress_layers_scaled.argtypes = [ctypes.c_void_p, ctypes.POINTER(rgc_layer), ctypes.c_int32,
                                             ctypes.c_float, ctypes.c_void_p, ctypes.c_uint32, ctypes.c_void_p]
    L.rgc_compress_layers_threshold.restype = ctypes.c_int
    L.rgc_compress_layers_threshold.argtypes = [ctypes.c_void_p, ctypes.POINTER(rgc_layer), ctypes.c_int32,
                                                ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                                ctypes.c_uint32, ctypes.c_void_p]
    L.rgc_message_means.restype = ctypes.c_int
    L.rgc_message_means.argtypes = [ctypes.c_void_p, ctypes.POINTER(rgc_layer), ctypes.c_int32, ctypes.c_void_p,
                                    ctypes.c_void_p]
    L.rgc_message_means_noalloc.restype = ctypes.c_int
    L.rgc_message_means_noalloc.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.POINTER(ctypes.c_void_p),
                                            ctypes.POINTER(ctypes.c_int32), ctypes.c_int32, ctypes.c_void_p,
                                            ctypes.c_void_p]
    L.rgc_clip_coefficient.restype = ctypes.c_int
    L.rgc_clip_coefficient.argtypes = [ctypes.c_void_p, ctypes.POINTER(rgc_layer), ctypes.c_int32, ctypes.c_float,
                                       ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p]
    L.rgc_decompress_accumulate.restype = ctypes.c_int
    L.rgc_decompress_accumulate.argtypes = [ctypes.c_void_p, ctypes.POINTER(rgc_msg), ctypes.c_int32,
                                            ctypes.c_int32, ctypes.POINTER(ctypes.c_void_p),
                                            ctypes.POINTER(ctypes.c_int64), ctypes.c_float,
                                            ctypes.c_uint32, ctypes.c_void_p]
    L.rgc_token_logprobs.restype = ctypes.c_int
    L.rgc_token_logprobs.argtypes = [ctypes.c_void_p, ctypes.POINTER(rgc_token_scores), ctypes.c_void_p]
    L.rgc_token_logprobs_backward.restype = ctypes.c_int
    L.rgc_token_logprobs_backward.argtypes = [ctypes.c_void_p, ctypes.POINTER(rgc_token_scores), ctypes.c_void_p,
                                              ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p]
    L.rgc_distill_loss.restype = ctypes.c_int
    L.rgc_distill_loss.argtypes = [ctypes.c_void_p, ctypes.POINTER(rgc_distill), ctypes.c_void_p]
    L.rgc_gated_recurrence.restype = ctypes.c_int
    L.rgc_gated_recurrence.argtypes = [ctypes.c_void_p, ctypes.POINTER(rgc_recurrence), ctypes.c_void_p]
    L.rgc_gated_recurrence_backward.restype = ctypes.c_int
    L.rgc_gated_recurrence_backward.argtypes = [ctypes.c_void_p, ctypes.POINTER(rgc_recurrence),
                                                ctypes.POINTER(rgc_recurrence_grads), ctypes.c_void_p]
    L.rgc_embed_tokens.restype = ctypes.c_int
    L.rgc_embed_tokens.argtypes = [ctypes.c_void_p, ctypes.POINTER(rgc_embedding), ctypes.c_void_p]
    L.rgc_embed_tokens_backward.restype = ctypes.c_int
    L.rgc_embed_tokens_backward.argtypes = [ctypes.c_void_p, ctypes.POINTER(rgc_embedding), ctypes.c_void_p, ctypes.c_int64,
                                            ctypes.c_void_p, ctypes.c_uint32, ctypes.c_void_p]
    L.rgc_causal_convolution.restype = ctypes.c_int
    L.rgc_causal_convolution.argtypes = [ctypes.c_void_p, ctypes.POINTER(rgc_convolution), ctypes.c_void_p]
    L.rgc_causal_convolution_backward.restype = ctypes.c_int
    L.rgc_causal_convolution_backward.argtypes = [ctypes.c_void_p, ctypes.POINTER(rgc_convolution), ctypes.POINTER(rgc_convolution_grads), ctypes.c_void_p]
    L.rgc_selective_scan.restype = ctypes.c_int
    L.rgc_selective_scan.argtypes = [ctypes.c_void_p, ctypes.POINTER(rgc_scan), ctypes.c_void_p]
    L.rgc_selective_scan_backward.restype = ctypes.c_int
    L.rgc_selective_scan_backward.argtypes = [ctypes.c_void_p, ctypes.POINTER(rgc_scan), ctypes.POINTER(rgc_scan_grads), ctypes.c_void_p]
    L.rgc_reset_hints.restype = ctypes.c_int
    L.rgc_reset_hints.argtypes = [ctypes.c_void_p]
    L.rgc_limit_looks.restype = ctypes.c_int
    L.rgc_limit_looks.argtypes = [ctypes.c_void_p, ctypes.c_int32]
    L.rgc_limit_optional_scratch.restype = ctypes.c_int
    L.rgc_limit_optional_scratch.argtypes = [ctypes.c_void_p, ctypes.c_int64]
    L.rgc_poison_hints.restype = ctypes.c_int
    L.rgc_poison_hints.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p]
    L.rgc_selftest.restype = ctypes.c_int
    L.rgc_selftest.argtypes = [ctypes.c_void_p, ctypes.c_void_p]
    L.rgc_last_paths.restype = ctypes.c_int
    L.rgc_last_paths.argtypes = [ctypes.c_void_p, ctypes.POINTER(ctypes.c_int32), ctypes.c_int32, ctypes.c_void_p]
    L.rgc_last_error.restype = ctypes.c_int
    L.rgc_last_error.argtypes = [ctypes.c_void_p, ctypes.c_void_p]
    L.rgc_last_stats.restype = ctypes.c_int
    L.rgc_last_stats.argtypes = [ctypes.c_void_p, ctypes.POINTER(ctypes.c_int64), ctypes.c_int32, ctypes.c_void_p]
    L.rgc_decompress_status.restype = ctypes.c_int
    L.rgc_decompress_status.argtypes = [ctypes.c_void_p, ctypes.POINTER(ctypes.c_uint32), ctypes.c_void_p]
    L.rgc_profile_enable.restype = ctypes.c_int
    L.rgc_profile_enable.argtypes = [ctypes.c_void_p, ctypes.c_int]
    L.rgc_profile_read.restype = ctypes.c_int
    L.rgc_profile_read.argtypes = [ctypes.c_void_p, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64)]
    L.rgc_stream_yardstick.restype = ctypes.c_int
    L.rgc_stream_yardstick.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_float,
                                       ctypes.c_int, ctypes.c_void_p]
    L.rgc_strerror.restype = ctypes.c_char_p
    L.rgc_strerror.argtypes = [ctypes.c_int]
    _lib = L
    return L


def _check(status: int) -> None:
    if status != RGC_OK:
        raise RgcError(status, load_library().rgc_strerror(status).decode())


def _stream(stream) -> ctypes.c_void_p:
    if stream is None:
        return ctypes.c_void_p(0)
    return ctypes.c_void_p(int(getattr(stream, "cuda_stream", stream)))


def _ptr(t) -> Optional[int]:
    return None if t is None else int(t.data_ptr())


def rgc_k_for_density(n: int, density_ppm: int = 1000) -> int:
    return int(load_library().rgc_k_for_density(int(n), int(density_ppm)))


class Context:
    """Owns an ``rgc_ctx`` (scratch + speed hints) on one device."""

    def __init__(self, max_total_elems: int, max_layers: int, device_id: int = 0):
        self._lib = load_library()
        self._h = ctypes.c_void_p(0)
        _check(self._lib.rgc_create(ctypes.byref(self._h), int(device_id), int(max_total_elems), int(max_layers)))

    @property
    def handle(self) -> ctypes.c_void_p:
        return self._h

    def close(self) -> None:
        if self._h:
            self._lib.rgc_destroy(self._h)
            self._h = ctypes.c_void_p(0)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def reset_hints(self) -> None:
        _check(self._lib.rgc_reset_hints(self._h))

    def limit_optional_scratch(self, max_bytes: int) -> None:
        _check(self._lib.rgc_limit_optional_scratch(self._h, int(max_bytes)))

    def limit_looks(self, looks: int) -> None:
        _check(self._lib.rgc_limit_looks(self._h, int(looks)))

    def poison_hints(self, mode: int, stream=None) -> None:
        _check(self._lib.rgc_poison_hints(self._h, int(mode), _stream(stream)))

    def selftest(self, stream=None) -> None:
        _check(self._lib.rgc_selftest(self._h, _stream(stream)))

    def profile_enable(self, enable: bool) -> None:
        _check(self._lib.rgc_profile_enable(self._h, 1 if enable else 0))

    def profile_read(self):
        """-> (ms[4]: accumulate, phases, decompress table, decompress tiles; calls[2])."""
        ms = (ctypes.c_double * 4)()
        calls = (ctypes.c_int64 * 2)()
        _check(self._lib.rgc_profile_read(self._h, ms, calls))
        return list(ms), list(calls)

    def last_stats(self, num_layers: int, stream=None) -> List[List[int]]:
        """-> per layer [path, candidates, exactly ranked candidates, threshold key, hint misses so far]."""
        out = (ctypes.c_int64 * (5 * num_layers))()
        _check(self._lib.rgc_last_stats(self._h, out, int(num_layers), _stream(stream)))
        return [list(out[5 * l:5 * l + 5]) for l in range(num_layers)]

    def decompress_status(self, stream=None) -> int:
        """OR of the RGC_STATUS_* bits found by the RGC_VALIDATE checks so far (waits for the stream; clears the word)."""
        out = ctypes.c_uint32(0)
        _check(self._lib.rgc_decompress_status(self._h, ctypes.byref(out), _stream(stream)))
        return int(out.value)

    def last_error(self, stream=None) -> None:
        """Raises RgcError(RGC_EINTERNAL) if a kernel has reported an internal inconsistency (waits for the stream)."""
        _check(self._lib.rgc_last_error(self._h, _stream(stream)))

    def last_paths(self, num_layers: int, stream=None) -> List[int]:
        out = (ctypes.c_int32 * num_layers)()
        _check(self._lib.rgc_last_paths(self._h, out, int(num_layers), _stream(stream)))
        return list(out)


class LayerList:
    """A host ``rgc_layer[]`` built once from tensors (keeps them alive)."""

    def __init__(self, grads: Sequence, residuals: Sequence, ks: Sequence[int], out_idx: Sequence,
                 out_val: Sequence, out_count, momenta: Optional[Sequence] = None):
        L = len(grads)
        self.num_layers = L
        self._keep = (grads, residuals, ks, out_idx, out_val, out_count, momenta)
        self.array = (rgc_layer * L)()
        base = int(out_count.data_ptr())
        for l in range(L):
            a = self.array[l]
            a.grad = _ptr(grads[l])
            a.residual = _ptr(residuals[l])
            a.momentum = _ptr(momenta[l]) if momenta is not None else None
            a.n = int(grads[l].numel())
            a.k = int(ks[l])
            a.out_idx = _ptr(out_idx[l])
            a.out_val = _ptr(out_val[l])
            a.out_count = base + 4 * l


class MessageList:
    """Host ``rgc_msg[workers][layers]`` plus the dense pointer / size arrays."""

    def __init__(self, idx: Sequence[Sequence], val: Sequence[Sequence], dense: Sequence):
        N = len(idx)
        L = len(dense)
        self.num_workers, self.num_layers = N, L
        self._keep = (idx, val, dense)
        self.msgs = (rgc_msg * max(N * L, 1))()
        for w in range(N):
            for l in range(L):
                m = self.msgs[w * L + l]
                c = int(idx[w][l].numel())
                m.idx = _ptr(idx[w][l]) if c else None
                m.val = _ptr(val[w][l]) if c else None
                m.count = c
        self.dense = (ctypes.c_void_p * L)(*[int(d.data_ptr()) for d in dense])
        self.n = (ctypes.c_int64 * L)(*[int(d.numel()) for d in dense])


def rgc_compress_layers(ctx: Context, layers: LayerList, momentum: float = 0.0, flags: int = 0,
                        stream=None) -> None:
    _check(load_library().rgc_compress_layers(ctx.handle, layers.array, layers.num_layers,
                                              float(momentum), int(flags), _stream(stream)))


def rgc_compress_layers_scaled(ctx: Context, layers: LayerList, momentum: float = 0.0, grad_scale=None,
                               flags: int = 0, stream=None) -> None:
    """grad_scale: a one-element float32 device tensor (or None)."""
    _check(load_library().rgc_compress_layers_scaled(ctx.handle, layers.array, layers.num_layers,
                                                     float(momentum), _ptr(grad_scale), int(flags), _stream(stream)))


def rgc_compress_layers_threshold(ctx: Context, layers: LayerList, momentum: float, thresholds, nnz=None,
                                  flags: int = 0, stream=None, grad_scale=None) -> None:
    """thresholds: float32 device tensor of num_layers elements (written with RGC_THRESHOLD_SEARCH, read
    otherwise); nnz: int32 device tensor of num_layers elements or None; grad_scale: a one-element float32
    device tensor or None.  The layers' out_idx / out_val hold 2 * k entries."""
    _check(load_library().rgc_compress_layers_threshold(ctx.handle, layers.array, layers.num_layers, float(momentum),
                                                        _ptr(grad_scale) if grad_scale is not None else None,
                                                        _ptr(thresholds), _ptr(nnz) if nnz is not None else None,
                                                        int(flags), _stream(stream)))


def rgc_message_means(ctx: Context, layers: LayerList, means, stream=None) -> None:
    """means: a float32 device tensor of num_layers elements that receives each layer's average value."""
    _check(load_library().rgc_message_means(ctx.handle, layers.array, layers.num_layers, _ptr(means), _stream(stream)))


RGC_NOALLOC_MAX_LAYERS = 64


def rgc_message_means_noalloc(values: Sequence, counts, capacity: Sequence[int], means, stream=None) -> None:
    """values: one float32 device tensor per message; counts: an int32 device tensor holding their length
    words, one per message; capacity: how many values each buffer holds; means: float32 device tensor."""
    L = len(values)
    vp = (ctypes.c_void_p * max(L, 1))(*[int(v.data_ptr()) for v in values])
    base = int(counts.data_ptr())
    cp = (ctypes.c_void_p * max(L, 1))(*[base + 4 * l for l in range(L)])
    cap = (ctypes.c_int32 * max(L, 1))(*[int(c) for c in capacity])
    _check(load_library().rgc_message_means_noalloc(vp, cp, cap, L, _ptr(means), _stream(stream)))


def rgc_stream_yardstick(grad, residual, velocity, momentum: float, reverse: bool = False, stream=None) -> None:
    """grad, residual, velocity: float32 device tensors of one length; residual and velocity are updated in place."""
    _check(load_library().rgc_stream_yardstick(_ptr(grad), _ptr(residual), _ptr(velocity), int(grad.numel()),
                                               float(momentum), int(bool(reverse)), _stream(stream)))


def rgc_clip_coefficient(ctx: Context, layers: LayerList, max_norm: float, num_workers: int, coefficient,
                         stream=None) -> None:
    """coefficient: a one-element float32 device tensor that receives the clipping coefficient."""
    _check(load_library().rgc_clip_coefficient(ctx.handle, layers.array, layers.num_layers, float(max_norm),
                                               int(num_workers), _ptr(coefficient), _stream(stream)))


def rgc_decompress_accumulate(ctx: Context, msgs: MessageList, scale: float,
                              flags: int = RGC_OVERWRITE, stream=None) -> None:
    _check(load_library().rgc_decompress_accumulate(ctx.handle, msgs.msgs, msgs.num_workers,
                                                    msgs.num_layers, msgs.dense, msgs.n,
                                                    float(scale), int(flags), _stream(stream)))


# ---------------------------------------------------------------- the language model's operators

_DTYPES = {"torch.float32": RGC_F32, "torch.bfloat16": RGC_BF16, "torch.float16": RGC_F16}


def _require(ok: bool, text: str) -> None:
    """What the library cannot see from a pointer: shapes, types, strides."""
    if not ok:
        raise RgcError(RGC_EINVAL, text)


def _plain(t, name: str, shape, dtype: str, like) -> Optional[int]:
    """A contiguous tensor of that shape and type on `like`'s device, or None."""
    if t is None:
        return None
    _require(tuple(t.shape) == tuple(shape), "%s: shape %s expected, got %s" % (name, tuple(shape), tuple(t.shape)))
    _require(str(t.dtype) == "torch." + dtype, "%s: %s expected, got %s" % (name, dtype, t.dtype))
    _require(t.is_contiguous(), "%s: must be contiguous" % name)
    _require(t.device == like.device, "%s: on %s, the others on %s" % (name, t.device, like.device))
    return _ptr(t)


def _rows(t, name: str, like=None) -> int:
    """Row stride of a [rows, vocab] tensor whose rows are contiguous."""
    _require(t.dim() == 2 and str(t.dtype) in _DTYPES, "%s: a [rows, vocab] tensor of float32, bfloat16 or float16 expected" % name)
    _require(t.shape[1] >= 1 and (t.shape[1] == 1 or t.stride(1) == 1), "%s: the vocabulary must be contiguous" % name)
    if like is not None:
        _require(t.shape == like.shape and t.dtype == like.dtype and t.device == like.device,
                 "%s: shape, type and device of the logits expected" % name)
    return int(t.stride(0)) if t.shape[0] > 1 else max(int(t.stride(0)), int(t.shape[1]))


class TokenScores:
    """A host ``rgc_token_scores`` built once from tensors (keeps them alive).  logits: [rows, vocab], rows strided as they
    may be; targets: int32 [rows] or None; outputs (each may be None): float32 logprob [rows], entropy [rows], stats [rows, 2];
    top_idx int32 [rows, top] and top_logprob float32 [rows, top] together."""

    def __init__(self, logits, targets=None, logprob=None, entropy=None, top_idx=None, top_logprob=None, stats=None,
                 temperature: float = 1.0):
        a = self.desc = rgc_token_scores()
        a.row_stride = _rows(logits, "logits")
        rows, vocab = (int(n) for n in logits.shape)
        a.logits, a.rows, a.vocab, a.dtype = _ptr(logits), rows, vocab, _DTYPES[str(logits.dtype)]
        a.targets = _plain(targets, "targets", (rows,), "int32", logits)
        a.temperature = float(temperature)
        _require((top_idx is None) == (top_logprob is None), "top_idx and top_logprob come together")
        _require(top_idx is None or top_idx.dim() == 2, "top_idx: a [rows, top] tensor expected")
        a.top = 0 if top_idx is None else int(top_idx.shape[1])
        a.logprob = _plain(logprob, "logprob", (rows,), "float32", logits)
        a.entropy = _plain(entropy, "entropy", (rows,), "float32", logits)
        a.stats = _plain(stats, "stats", (rows, 2), "float32", logits)
        a.top_idx = _plain(top_idx, "top_idx", (rows, a.top), "int32", logits)
        a.top_logprob = _plain(top_logprob, "top_logprob", (rows, a.top), "float32", logits)
        self.logits = logits
        self._keep = (logits, targets, logprob, entropy, stats, top_idx, top_logprob)
        self._ref = ctypes.byref(a)


class Distillation:
    """A host ``rgc_distill`` built once from tensors (keeps them alive).  logits: [rows, vocab]; teacher_idx: int32 [rows, k];
    teacher_logits: float32 [rows, k]; targets: int32 [rows] or None; grad_loss, loss: float32 [rows] or None; grad_logits: like
    the logits (or the logits themselves) or None."""

    def __init__(self, logits, teacher_idx, teacher_logits, targets=None, loss=None, grad_loss=None, grad_logits=None,
                 temperature: float = 1.0, soft_weight: float = 1.0, label_weight: float = 0.0):
        a = self.desc = rgc_distill()
        a.row_stride = _rows(logits, "logits")
        rows, vocab = (int(n) for n in logits.shape)
        a.logits, a.rows, a.vocab, a.dtype = _ptr(logits), rows, vocab, _DTYPES[str(logits.dtype)]
        _require(teacher_idx.dim() == 2, "teacher_idx: a [rows, k] tensor expected")
        a.k = int(teacher_idx.shape[1])
        a.teacher_idx = _plain(teacher_idx, "teacher_idx", (rows, a.k), "int32", logits)
        a.teacher_logits = _plain(teacher_logits, "teacher_logits", (rows, a.k), "float32", logits)
        a.targets = _plain(targets, "targets", (rows,), "int32", logits)
        a.temperature, a.soft_weight, a.label_weight = float(temperature), float(soft_weight), float(label_weight)
        a.grad_loss = _plain(grad_loss, "grad_loss", (rows,), "float32", logits)
        a.loss = _plain(loss, "loss", (rows,), "float32", logits)
        if grad_logits is not None:
            a.grad_row_stride = _rows(grad_logits, "grad_logits", logits)
            a.grad_logits = _ptr(grad_logits)
        self._keep = (logits, teacher_idx, teacher_logits, targets, loss, grad_loss, grad_logits)
        self._ref = ctypes.byref(a)


def _sequence(t, name: str, like=None) -> rgc_sequence:
    """A [batch, steps, width] tensor whose channels are contiguous; other layouts come as transposed views."""
    if t is None:
        return rgc_sequence()
    _require(t.dim() == 3 and str(t.dtype) in _DTYPES, "%s: a [batch, steps, width] tensor of float32, bfloat16 or float16 expected" % name)
    _require(t.shape[2] >= 1 and (t.shape[2] == 1 or t.stride(2) == 1), "%s: the channels must be contiguous" % name)
    if like is not None:
        _require(t.shape == like.shape and t.dtype == like.dtype and t.device == like.device,
                 "%s: shape, type and device of x expected" % name)
    return rgc_sequence(_ptr(t), int(t.stride(0)), int(t.stride(1)))


class Recurrence:
    """A host ``rgc_recurrence`` built once from tensors (keeps them alive).  x, gate, y, out_gate (or None): [batch, steps, width]
    of one type, the first two dimensions strided as they may be; lengths: int32 [batch] or None; resets: uint8 or bool
    [batch, steps] or None; h0, h_last: float32 [batch, width] or None; states: float32
    [batch, ceil(steps / RGC_RECURRENCE_CHUNK), width], needed for the backward call."""

    def __init__(self, x, gate, y, out_gate=None, lengths=None, resets=None, h0=None, h_last=None, states=None):
        a = self.desc = rgc_recurrence()
        a.x = _sequence(x, "x")
        a.gate, a.y, a.out_gate = _sequence(gate, "gate", x), _sequence(y, "y", x), _sequence(out_gate, "out_gate", x)
        batch, steps, width = (int(n) for n in x.shape)
        a.batch, a.steps, a.width, a.dtype = batch, steps, width, _DTYPES[str(x.dtype)]
        a.lengths = _plain(lengths, "lengths", (batch,), "int32", x)
        a.resets = _plain(resets, "resets", (batch, steps), "bool" if str(getattr(resets, "dtype", "")) == "torch.bool" else "uint8", x)
        a.h0 = _plain(h0, "h0", (batch, width), "float32", x)
        a.h_last = _plain(h_last, "h_last", (batch, width), "float32", x)
        a.states = _plain(states, "states", (batch, -(-steps // RGC_RECURRENCE_CHUNK), width), "float32", x)
        self.x, self.has_out_gate = x, out_gate is not None
        self._keep = (x, gate, y, out_gate, lengths, resets, h0, h_last, states)
        self._ref = ctypes.byref(a)


class RecurrenceGrads:
    """A host ``rgc_recurrence_grads`` for a Recurrence (keeps the tensors alive).  dy, dx, dgate, dout_gate: like x; dh_last,
    dh0: float32 [batch, width] or None."""

    def __init__(self, recurrence: Recurrence, dy, dx, dgate, dout_gate=None, dh_last=None, dh0=None):
        x = recurrence.x
        _require(recurrence.has_out_gate == (dout_gate is not None), "dout_gate comes with an out_gate")
        a = self.desc = rgc_recurrence_grads()
        a.dy, a.dx, a.dgate = _sequence(dy, "dy", x), _sequence(dx, "dx", x), _sequence(dgate, "dgate", x)
        a.dout_gate = _sequence(dout_gate, "dout_gate", x)
        a.dh_last = _plain(dh_last, "dh_last", (x.shape[0], x.shape[2]), "float32", x)
        a.dh0 = _plain(dh0, "dh0", (x.shape[0], x.shape[2]), "float32", x)
        self._keep = (recurrence, dy, dx, dgate, dout_gate, dh_last, dh0)
        self._ref = ctypes.byref(a)


def rgc_token_logprobs(ctx: Context, scores: TokenScores, stream=None) -> None:
    _check(load_library().rgc_token_logprobs(ctx.handle, scores._ref, _stream(stream)))


def rgc_token_logprobs_backward(ctx: Context, scores: TokenScores, grad_logits, grad_logprob=None, grad_entropy=None,
                                stream=None) -> None:
    """grad_logits: like the logits, or the logits themselves; grad_logprob, grad_entropy: float32 [rows] or None."""
    stride, rows = _rows(grad_logits, "grad_logits", scores.logits), (scores.desc.rows,)
    _check(load_library().rgc_token_logprobs_backward(ctx.handle, scores._ref,
                                                      _plain(grad_logprob, "grad_logprob", rows, "float32", grad_logits),
                                                      _plain(grad_entropy, "grad_entropy", rows, "float32", grad_logits),
                                                      _ptr(grad_logits), stride, _stream(stream)))


def rgc_distill_loss(ctx: Context, distillation: Distillation, stream=None) -> None:
    _check(load_library().rgc_distill_loss(ctx.handle, distillation._ref, _stream(stream)))


def rgc_gated_recurrence(ctx: Context, recurrence: Recurrence, stream=None) -> None:
    _check(load_library().rgc_gated_recurrence(ctx.handle, recurrence._ref, _stream(stream)))


def rgc_gated_recurrence_backward(ctx: Context, recurrence: Recurrence, grads: RecurrenceGrads, stream=None) -> None:
    _check(load_library().rgc_gated_recurrence_backward(ctx.handle, recurrence._ref, grads._ref, _stream(stream)))


def _table(t, name: str) -> int:
    """Row stride of a [rows, width] tensor whose channels are contiguous."""
    _require(t.dim() == 2 and str(t.dtype) in _DTYPES, "%s: a [rows, width] tensor of float32, bfloat16 or float16 expected" % name)
    _require(t.shape[1] >= 1 and (t.shape[1] == 1 or t.stride(1) == 1), "%s: the channels must be contiguous" % name)
    return int(t.stride(0)) if t.shape[0] > 1 else max(int(t.stride(0)), int(t.shape[1]))


class Embedding:
    """A host ``rgc_embedding`` built once from tensors (keeps them alive).  table: [vocab, width], rows strided as they may be; tokens: int32
    [rows]; out: [rows, width] of any of the three types, rows strided as they may be."""

    def __init__(self, table, tokens, out, scale: float = 1.0):
        a = self.desc = rgc_embedding()
        a.table_stride, a.out_stride = _table(table, "table"), _table(out, "out")
        rows, width = (int(n) for n in out.shape)
        _require(int(table.shape[1]) == width and table.device == out.device, "out: width and device of the table expected")
        a.table, a.vocab, a.width, a.table_dtype = _ptr(table), int(table.shape[0]), width, _DTYPES[str(table.dtype)]
        a.out, a.rows, a.dtype = _ptr(out), rows, _DTYPES[str(out.dtype)]
        a.tokens = _plain(tokens, "tokens", (rows,), "int32", table)
        a.scale = float(scale)
        self.table, self.out = table, out
        self._keep = (table, tokens, out)
        self._ref = ctypes.byref(a)


def rgc_embed_tokens(ctx: Context, embedding: Embedding, stream=None) -> None:
    _check(load_library().rgc_embed_tokens(ctx.handle, embedding._ref, _stream(stream)))


def rgc_embed_tokens_backward(ctx: Context, embedding: Embedding, dout, dtable, flags: int = RGC_OVERWRITE, stream=None) -> None:
    """dout: like the embedding's out; dtable: float32 [vocab, width]."""
    stride, out = _table(dout, "dout"), embedding.out
    _require(dout.shape == out.shape and dout.dtype == out.dtype and dout.device == out.device, "dout: shape, type and device of out expected")
    to = _plain(dtable, "dtable", (embedding.desc.vocab, embedding.desc.width), "float32", out)
    _check(load_library().rgc_embed_tokens_backward(ctx.handle, embedding._ref, _ptr(dout), stride, to, int(flags), _stream(stream)))


def _resets(t, shape, like) -> Optional[int]:
    return _plain(t, "resets", shape, "bool" if str(getattr(t, "dtype", "")) == "torch.bool" else "uint8", like)


class Convolution:
    """A host ``rgc_convolution`` built once from tensors (keeps them alive).  x, y: [batch, steps, width] of one type, the first two dimensions strided
    as they may be; weight: float32 [width, taps]; bias: float32 [width] or None; lengths: int32 [batch] or None; resets: uint8 or bool
    [batch, steps] or None; before, last: [batch, taps - 1, width] of x's type or None."""

    def __init__(self, x, weight, y, bias=None, silu: bool = False, lengths=None, resets=None, before=None, last=None):
        a = self.desc = rgc_convolution()
        a.x, a.y = _sequence(x, "x"), _sequence(y, "y", x)
        batch, steps, width = (int(n) for n in x.shape)
        _require(weight.dim() == 2, "weight: a [width, taps] tensor expected")
        a.batch, a.steps, a.width, a.taps, a.dtype, a.silu = batch, steps, width, int(weight.shape[1]), _DTYPES[str(x.dtype)], int(bool(silu))
        a.weight, a.bias = _plain(weight, "weight", (width, a.taps), "float32", x), _plain(bias, "bias", (width,), "float32", x)
        a.lengths, a.resets = _plain(lengths, "lengths", (batch,), "int32", x), _resets(resets, (batch, steps), x)
        self.kept, kind = (batch, a.taps - 1, width), str(x.dtype)[len("torch."):]
        a.before, a.last = _plain(before, "before", self.kept, kind, x), _plain(last, "last", self.kept, kind, x)
        self.x, self.kind = x, kind
        self._keep = (x, weight, y, bias, lengths, resets, before, last)
        self._ref = ctypes.byref(a)


class ConvolutionGrads:
    """A host ``rgc_convolution_grads`` for a Convolution (keeps the tensors alive).  dy, dx: like x; dweight: float32 [width, taps]; dbias: float32 [width]
    or None; dlast, dbefore: [batch, taps - 1, width] of x's type or None.  A Convolution whose last is its before has no gradients: they need before as the call read it."""

    def __init__(self, convolution: Convolution, dy, dx, dweight, dbias=None, dlast=None, dbefore=None):
        x, a = convolution.x, rgc_convolution_grads()
        self.desc = a
        a.dy, a.dx = _sequence(dy, "dy", x), _sequence(dx, "dx", x)
        a.dweight = _plain(dweight, "dweight", (x.shape[2], convolution.desc.taps), "float32", x)
        a.dbias = _plain(dbias, "dbias", (x.shape[2],), "float32", x)
        a.dlast = _plain(dlast, "dlast", convolution.kept, convolution.kind, x)
        a.dbefore = _plain(dbefore, "dbefore", convolution.kept, convolution.kind, x)
        self._keep = (convolution, dy, dx, dweight, dbias, dlast, dbefore)
        self._ref = ctypes.byref(a)


def rgc_causal_convolution(ctx: Context, convolution: Convolution, stream=None) -> None:
    _check(load_library().rgc_causal_convolution(ctx.handle, convolution._ref, _stream(stream)))


def rgc_causal_convolution_backward(ctx: Context, convolution: Convolution, grads: ConvolutionGrads, stream=None) -> None:
    _check(load_library().rgc_causal_convolution_backward(ctx.handle, convolution._ref, grads._ref, _stream(stream)))


def _group_sequence(t, name: str, x, channels: int) -> rgc_sequence:
    """A [batch, steps, channels] tensor of x's type."""
    s = _sequence(t, name)
    _require(tuple(t.shape) == tuple(x.shape[:2]) + (channels,) and t.dtype == x.dtype and t.device == x.device,
             "%s: a [batch, steps, %d] tensor of x's type on its device expected" % (name, channels))
    return s


class Scan:
    """A host ``rgc_scan`` built once from tensors (keeps them alive).  x, delta, y, gate (or None): [batch, steps, width] of one type; b, c: [batch, steps, groups * N] of that
    type; the first two dimensions strided as they may be.  a: float32 [width, N]; d, delta_bias: float32 [width] or None; lengths: int32 [batch] or None; resets: uint8 or bool
    [batch, steps] or None; h0, h_last: float32 [batch, width, N] or None; states: float32 [batch, ceil(steps / RGC_SCAN_CHUNK), width, N], needed for the backward call."""

    def __init__(self, x, delta, a, b, c, y, groups: int = 1, d=None, gate=None, delta_bias=None, softplus: bool = False, lengths=None, resets=None, h0=None, h_last=None,
                 states=None):
        s = self.desc = rgc_scan()
        s.x = _sequence(x, "x")
        s.delta, s.y, s.gate = _sequence(delta, "delta", x), _sequence(y, "y", x), _sequence(gate, "gate", x)
        batch, steps, width = (int(n) for n in x.shape)
        _require(a.dim() == 2, "a: a [width, states] tensor expected")
        n = int(a.shape[1])
        _require(int(groups) >= 1 and width % int(groups) == 0, "groups: the width must be a multiple of them")
        s.batch, s.steps, s.width, s.states, s.groups, s.dtype, s.softplus = batch, steps, width, n, int(groups), _DTYPES[str(x.dtype)], int(bool(softplus))
        self.channels, self.x, self.has_gate, self.state_shape = int(groups) * n, x, gate is not None, (batch, width, n)
        s.b, s.c = _group_sequence(b, "b", x, self.channels), _group_sequence(c, "c", x, self.channels)
        s.a, s.d, s.delta_bias = _plain(a, "a", (width, n), "float32", x), _plain(d, "d", (width,), "float32", x), _plain(delta_bias, "delta_bias", (width,), "float32", x)
        s.lengths, s.resets = _plain(lengths, "lengths", (batch,), "int32", x), _resets(resets, (batch, steps), x)
        s.h0, s.h_last = _plain(h0, "h0", self.state_shape, "float32", x), _plain(h_last, "h_last", self.state_shape, "float32", x)
        s.kept = _plain(states, "states", (batch, -(-steps // RGC_SCAN_CHUNK), width, n), "float32", x)
        self._keep = (x, delta, a, b, c, y, d, gate, delta_bias, lengths, resets, h0, h_last, states)
        self._ref = ctypes.byref(s)


class ScanGrads:
    """A host ``rgc_scan_grads`` for a Scan (keeps the tensors alive).  dy, dx, ddelta, dgate (with a gate): like x; db, dc: like b and c; da: float32 [width, N]; dd, ddelta_bias:
    float32 [width] or None; dh_last, dh0: float32 [batch, width, N] or None."""

    def __init__(self, scan: Scan, dy, dx, ddelta, da, db, dc, dd=None, dgate=None, ddelta_bias=None, dh_last=None, dh0=None):
        x, g = scan.x, rgc_scan_grads()
        self.desc = g
        _require(scan.has_gate == (dgate is not None), "dgate comes with a gate")
        width, n = int(x.shape[2]), scan.desc.states
        g.dy, g.dx, g.ddelta, g.dgate = _sequence(dy, "dy", x), _sequence(dx, "dx", x), _sequence(ddelta, "ddelta", x), _sequence(dgate, "dgate", x)
        g.db, g.dc = _group_sequence(db, "db", x, scan.channels), _group_sequence(dc, "dc", x, scan.channels)
        g.da, g.dd, g.ddelta_bias = _plain(da, "da", (width, n), "float32", x), _plain(dd, "dd", (width,), "float32", x), _plain(ddelta_bias, "ddelta_bias", (width,), "float32", x)
        g.dh_last, g.dh0 = _plain(dh_last, "dh_last", scan.state_shape, "float32", x), _plain(dh0, "dh0", scan.state_shape, "float32", x)
        self._keep = (scan, dy, dx, ddelta, da, db, dc, dd, dgate, ddelta_bias, dh_last, dh0)
        self._ref = ctypes.byref(g)


def rgc_selective_scan(ctx: Context, scan: Scan, stream=None) -> None:
    _check(load_library().rgc_selective_scan(ctx.handle, scan._ref, _stream(stream)))


def rgc_selective_scan_backward(ctx: Context, scan: Scan, grads: ScanGrads, stream=None) -> None:
    _check(load_library().rgc_selective_scan_backward(ctx.handle, scan._ref, grads._ref, _stream(stream)))
