"""Python binding of the gfx950 sparse-FFN decode library (``liblsffn.so``).

Argument marshalling only: every step of the decode path runs in the HIP
kernels behind the C ABI of ``include/ls_ffn.h`` (class ``Ffn``) and of
``include/ls_ops.h`` (class ``Ops``: the decoder layer's operators around the
FFN).  Function names mirror the C entry points.  PyTorch supplies device memory and the stream.

The library is loaded from this package directory.  There is no fallback: if
it has not been built, every call raises ``RuntimeError``.
"""
from __future__ import annotations

import atexit
import ctypes
import os
import weakref

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblsffn.so")

LS_OK, LS_E_INVAL, LS_E_NOMEM, LS_E_DEVICE, LS_E_STATE, LS_E_UNSUPPORTED, LS_E_CAPACITY = range(7)
STATUS_NAMES = {0: "LS_OK", 1: "LS_E_INVAL", 2: "LS_E_NOMEM", 3: "LS_E_DEVICE", 4: "LS_E_STATE",
                5: "LS_E_UNSUPPORTED", 6: "LS_E_CAPACITY"}
LS_F32, LS_F16, LS_BF16, LS_I8 = 0, 1, 2, 3
LS_ACT_REGLU, LS_ACT_SWIGLU_THRESH = 0, 1
LS_WEIGHTS_HBM, LS_WEIGHTS_HOST = 0, 1
LS_SEL_TOPK, LS_SEL_THRESHOLD = 0, 1
LS_PREFETCH_NONE, LS_PREFETCH_ONESHOT, LS_PREFETCH_REFINE = 0, 1, 2
LS_ROPE_HALF, LS_ROPE_PAIR = 0, 1

EXPORTS = ("ls_ffn_create", "ls_ffn_set_layer", "ls_ffn_destroy", "ls_predict", "ls_select_blocks",
           "ls_sparse_ffn_step", "ls_sparse_ffn_step_static", "ls_stream_weights", "ls_decode_step_streamed", "ls_decode_step",
           "ls_set_hash_predictor", "ls_hash_predict",
           "ls_debug_last_activations", "ls_set_kernel_timing", "ls_kernel_timing",
           "ls_configure", "ls_ffn_sync", "ls_debug_decode_trace", "ls_debug_phase_trace",
           "ls_debug_stages_done", "ls_measure_read_bandwidth", "ls_build_digest", "ls_last_error")
# entry points of ls_ops.h
OPS_EXPORTS = ("ls_ops_create", "ls_ops_destroy", "ls_ops_sync", "ls_ops_last_error", "ls_norm_residual", "ls_linear_i8",
               "ls_kv_append", "ls_attend")
(LS_CFG_DECODE_PATH, LS_CFG_SPEC_BLOCKS, LS_CFG_TRACE_WG, LS_CFG_COOPERATIVE, LS_CFG_BATCH_MFMA, LS_CFG_ZERO_SKIP,
 LS_CFG_STREAM_SYNC, LS_CFG_STAGE_WAIT_US) = range(8)
LS_SYNC_EVENTS, LS_SYNC_FLAGS, LS_SYNC_HOST = range(3)
PHASES = ("layer_start", "input_ready", "scores_published", "all_scores", "acts_gathered",
          "exact_ranked", "slot_map", "misses_done", "partials_ready", "output_published",
          "prefetch_issued", "partials_done", "next_list_ranked", "early_gateup_done",
          "worker_start", "worker_acts_seen")
(LS_K_PRENORM, LS_K_PRED_P1, LS_K_PRED_P2, LS_K_SELECT, LS_K_GATEUP, LS_K_DOWN, LS_K_DECODE,
 LS_K_HASH, LS_K_STAGE) = range(9)


class LsFfnDesc(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("d_model", ctypes.c_int32),
                ("d_ff", ctypes.c_int32), ("block", ctypes.c_int32), ("rank", ctypes.c_int32),
                ("max_batch", ctypes.c_int32), ("dtype", ctypes.c_int), ("act", ctypes.c_int),
                ("residency", ctypes.c_int), ("prenorm_rms", ctypes.c_int32),
                ("hbm_cache_bytes", ctypes.c_uint64), ("stream", ctypes.c_void_p),
                ("debug_flags", ctypes.c_uint32)]


class LsLayerWeights(ctypes.Structure):
    _fields_ = [("w_gate", ctypes.c_void_p), ("w_up", ctypes.c_void_p),
                ("w_down", ctypes.c_void_p), ("b_gate", ctypes.c_void_p),
                ("p1", ctypes.c_void_p), ("p2", ctypes.c_void_p), ("threshold", ctypes.c_float)]


class LsStreamStats(ctypes.Structure):
    _fields_ = [("hits", ctypes.c_int64), ("misses", ctypes.c_int64), ("bytes", ctypes.c_int64),
                ("evictions", ctypes.c_int64)]


class LsHashWeights(ctypes.Structure):
    _fields_ = [("w1", ctypes.c_void_p), ("w_bin", ctypes.c_void_p), ("tables", ctypes.c_void_p),
                ("head", ctypes.c_void_p)]


class LsStreamReport(ctypes.Structure):
    _fields_ = [("final_bytes", ctypes.c_int64), ("copied_bytes", ctypes.c_int64),
                ("late_bytes", ctypes.c_int64), ("spec_bytes", ctypes.c_int64),
                ("wasted_bytes", ctypes.c_int64)]


class LsOpsDesc(ctypes.Structure):
    _fields_ = [("workspace_bytes", ctypes.c_uint64), ("stream", ctypes.c_void_p), ("debug_flags", ctypes.c_uint32)]


class LsNormArgs(ctypes.Structure):
    _fields_ = [("n_tokens", ctypes.c_int32), ("d", ctypes.c_int32), ("dtype", ctypes.c_int), ("post_norm", ctypes.c_int32),
                ("pre_norm", ctypes.c_int32), ("x_scale", ctypes.c_float), ("y_scale", ctypes.c_float), ("eps", ctypes.c_float),
                ("x", ctypes.c_void_p), ("x_stride", ctypes.c_int64), ("y", ctypes.c_void_p), ("y_stride", ctypes.c_int64),
                ("gate", ctypes.c_void_p), ("gate_stride", ctypes.c_int64), ("post_weight", ctypes.c_void_p),
                ("pre_weight", ctypes.c_void_p), ("x_out", ctypes.c_void_p), ("x_out_stride", ctypes.c_int64),
                ("h", ctypes.c_void_p), ("h_stride", ctypes.c_int64)]


class LsLinearI8Args(ctypes.Structure):
    _fields_ = [("n_tokens", ctypes.c_int32), ("k", ctypes.c_int32), ("n", ctypes.c_int32), ("x_type", ctypes.c_int),
                ("out_type", ctypes.c_int), ("x", ctypes.c_void_p), ("x_stride", ctypes.c_int64), ("x_scale", ctypes.c_void_p),
                ("w", ctypes.c_void_p), ("w_stride", ctypes.c_int64), ("w_scale", ctypes.c_void_p), ("bias", ctypes.c_void_p),
                ("out", ctypes.c_void_p), ("out_stride", ctypes.c_int64)]


class LsKvCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("dtype", ctypes.c_int), ("n_pages", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64)]


class LsAppendArgs(ctypes.Structure):
    _fields_ = [("n_tokens", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("rot_dim", ctypes.c_int32), ("n_pos", ctypes.c_int32),
                ("style", ctypes.c_int), ("k", ctypes.c_void_p), ("k_token_stride", ctypes.c_int64), ("k_head_stride", ctypes.c_int64),
                ("v", ctypes.c_void_p), ("v_token_stride", ctypes.c_int64), ("v_head_stride", ctypes.c_int64),
                ("q", ctypes.c_void_p), ("q_token_stride", ctypes.c_int64), ("q_head_stride", ctypes.c_int64),
                ("q_out", ctypes.c_void_p), ("q_out_token_stride", ctypes.c_int64), ("q_out_head_stride", ctypes.c_int64),
                ("positions", ctypes.c_void_p), ("slots", ctypes.c_void_p), ("cos_sin", ctypes.c_void_p)]


class LsAttendArgs(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("n_q", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("prefix_len", ctypes.c_int32),
                ("max_len", ctypes.c_int32), ("scale", ctypes.c_float), ("q", ctypes.c_void_p), ("q_token_stride", ctypes.c_int64),
                ("q_head_stride", ctypes.c_int64), ("out", ctypes.c_void_p), ("out_token_stride", ctypes.c_int64),
                ("out_head_stride", ctypes.c_int64), ("prefix_pages", ctypes.c_void_p), ("pages", ctypes.c_void_p),
                ("pages_stride", ctypes.c_int64), ("lens", ctypes.c_void_p)]


class LsError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


_lib = None


def load():
    """Load ``liblsffn.so`` (no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"HIP library not built: {LIB_PATH} is missing (run __graft_entry__.build())")
    lib = ctypes.CDLL(LIB_PATH)
    from . import build as _build
    lib.ls_build_digest.argtypes = []
    lib.ls_build_digest.restype = ctypes.c_char_p
    built = lib.ls_build_digest().decode()
    want = _build.source_digest()
    if built != want:
        raise RuntimeError(f"{LIB_PATH} was built from other sources (digest {built[:12]}, sources "
                           f"{want[:12]}): rebuild it (__graft_entry__.build())")
    P, I32, I64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    lib.ls_ffn_create.argtypes = [ctypes.POINTER(LsFfnDesc), ctypes.POINTER(ctypes.c_void_p)]
    lib.ls_ffn_set_layer.argtypes = [P, I32, ctypes.POINTER(LsLayerWeights)]
    lib.ls_ffn_destroy.argtypes = [P]
    lib.ls_predict.argtypes = [P, I32, P, I32, P]
    lib.ls_select_blocks.argtypes = [P, P, I32, ctypes.c_int, I32, ctypes.c_float, I32, I32, P, P]
    lib.ls_sparse_ffn_step.argtypes = [P, I32, P, I32, P, P, I32, I32, P]
    lib.ls_sparse_ffn_step_static.argtypes = [P, I32, P, I32, P, P, I32, I32, P]
    lib.ls_stream_weights.argtypes = [P, I32, P, I32, I32, ctypes.POINTER(LsStreamStats)]
    lib.ls_decode_step.argtypes = [P, P, I32, I32]
    lib.ls_decode_step_streamed.argtypes = [P, P, I32, I32, I32, I32, ctypes.POINTER(LsStreamReport)]
    lib.ls_set_hash_predictor.argtypes = [P, I32, ctypes.POINTER(LsHashWeights)]
    lib.ls_hash_predict.argtypes = [P, I32, P, I32, P]
    lib.ls_debug_last_activations.argtypes = [P, P, I64, ctypes.POINTER(I64)]
    lib.ls_set_kernel_timing.argtypes = [P, I32]
    lib.ls_kernel_timing.argtypes = [P, I32, I32, ctypes.POINTER(ctypes.c_double),
                                     ctypes.POINTER(I64)]
    lib.ls_configure.argtypes = [P, I32, I64]
    lib.ls_ffn_sync.argtypes = [P]
    lib.ls_debug_decode_trace.argtypes = [P, I32, P, P]
    lib.ls_debug_phase_trace.argtypes = [P, P, I64, ctypes.POINTER(I64)]
    lib.ls_measure_read_bandwidth.argtypes = [P, P, I64, I32, ctypes.POINTER(ctypes.c_double),
                                              ctypes.POINTER(ctypes.c_double)]
    lib.ls_last_error.argtypes = [P]
    lib.ls_last_error.restype = ctypes.c_char_p
    lib.ls_ops_create.argtypes = [ctypes.POINTER(LsOpsDesc), ctypes.POINTER(ctypes.c_void_p)]
    lib.ls_ops_destroy.argtypes = [P]
    lib.ls_ops_sync.argtypes = [P]
    lib.ls_ops_last_error.argtypes = [P]
    lib.ls_norm_residual.argtypes = [P, ctypes.POINTER(LsNormArgs)]
    lib.ls_linear_i8.argtypes = [P, ctypes.POINTER(LsLinearI8Args)]
    lib.ls_kv_append.argtypes = [P, ctypes.POINTER(LsKvCache), ctypes.POINTER(LsAppendArgs)]
    lib.ls_attend.argtypes = [P, ctypes.POINTER(LsKvCache), ctypes.POINTER(LsAttendArgs)]
    for name in OPS_EXPORTS:
        getattr(lib, name).restype = ctypes.c_char_p if name == "ls_ops_last_error" else ctypes.c_int
    for name in EXPORTS:
        if name not in ("ls_last_error", "ls_build_digest"):
            getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def _check(lib, ctx, status: int):
    if status != LS_OK:
        msg = lib.ls_last_error(ctx)
        raise LsError(status, msg.decode() if msg else "")


def _ptr(t) -> int | None:
    """Device pointer of a torch tensor (or None)."""
    return None if t is None else t.data_ptr()


def _host_ptr(a):
    return None if a is None else np.ascontiguousarray(a).ctypes.data


_live = weakref.WeakSet()


@atexit.register
def _close_all():
    """Destroy every context still open at interpreter exit, while the HIP runtime is alive:
    objects left to the garbage collector would otherwise be released during interpreter
    teardown, after the runtime's own exit handlers may have run."""
    for f in list(_live):
        try:
            f.close()
        except Exception:
            pass


class Ffn:
    """One library context.  Methods mirror the C entry points one to one."""

    def __init__(self, *, n_layers, d_model, d_ff, block, rank, max_batch=1, dtype=LS_F16,
                 act=LS_ACT_REGLU, residency=LS_WEIGHTS_HBM, prenorm_rms=1, hbm_cache_bytes=0,
                 stream=None):
        self.lib = load()
        import torch
        if stream is None:
            stream = torch.cuda.current_stream()
        self.torch_stream = stream
        desc = LsFfnDesc(n_layers, d_model, d_ff, block, rank, max_batch, dtype, act, residency,
                         prenorm_rms, hbm_cache_bytes, ctypes.c_void_p(stream.cuda_stream), 0)
        h = ctypes.c_void_p()
        st = self.lib.ls_ffn_create(ctypes.byref(desc), ctypes.byref(h))
        _check(self.lib, None, st)
        self.ctx = h
        self.n_layers, self.d_model, self.d_ff, self.block, self.rank = (n_layers, d_model, d_ff,
                                                                          block, rank)
        self.n_blk = d_ff // block
        self.max_batch = max_batch
        _live.add(self)

    def close(self):
        if getattr(self, "ctx", None):
            self.lib.ls_ffn_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def ls_ffn_set_layer(self, layer: int, w) -> None:
        """w: object with gate, up, down, bias, p1, p2 (host arrays in storage type), threshold."""
        arrs = [np.ascontiguousarray(a) if a is not None else None
                for a in (w.gate, w.up, w.down, w.bias, w.p1, w.p2)]
        lw = LsLayerWeights(*[_host_ptr(a) for a in arrs], float(getattr(w, "threshold", 0.0)))
        _check(self.lib, self.ctx, self.lib.ls_ffn_set_layer(self.ctx, layer, ctypes.byref(lw)))

    def ls_predict(self, layer: int, x, B: int, scores) -> None:
        _check(self.lib, self.ctx, self.lib.ls_predict(self.ctx, layer, _ptr(x), B, _ptr(scores)))

    def ls_select_blocks(self, scores, B: int, mode: int, k: int, tau: float, union_batch: int,
                         cap: int, idx, count) -> None:
        _check(self.lib, self.ctx, self.lib.ls_select_blocks(self.ctx, _ptr(scores), B, mode, k, tau,
                                                             union_batch, cap, _ptr(idx),
                                                             _ptr(count)))

    def ls_sparse_ffn_step(self, layer: int, x_in, B: int, idx, count, begin: int, end: int,
                           x_acc) -> None:
        _check(self.lib, self.ctx, self.lib.ls_sparse_ffn_step(self.ctx, layer, _ptr(x_in), B,
                                                               _ptr(idx), _ptr(count), begin, end,
                                                               _ptr(x_acc)))

    def ls_sparse_ffn_step_static(self, layer: int, x_in, B: int, idx, count, begin: int, end: int,
                                  x_acc) -> None:
        _check(self.lib, self.ctx, self.lib.ls_sparse_ffn_step_static(self.ctx, layer, _ptr(x_in), B,
                                                                      _ptr(idx), _ptr(count), begin, end,
                                                                      _ptr(x_acc)))

    def ls_stream_weights(self, layer: int, idx_host, n_stages: int = 1) -> LsStreamStats:
        a = np.ascontiguousarray(idx_host, dtype=np.int32)
        stats = LsStreamStats()
        _check(self.lib, self.ctx, self.lib.ls_stream_weights(self.ctx, layer, a.ctypes.data,
                                                              int(a.size), n_stages,
                                                              ctypes.byref(stats)))
        return stats

    def ls_set_hash_predictor(self, layer: int, hw) -> None:
        """hw: .w1 fp32 [d, 8], .w_bin uint32 [4, 8, 8], .tables uint32 [4, 256, 8], .head uint8 [256, n_blk]"""
        arrs = [np.ascontiguousarray(hw.w1, np.float32), np.ascontiguousarray(hw.w_bin, np.uint32),
                np.ascontiguousarray(hw.tables, np.uint32), np.ascontiguousarray(hw.head, np.uint8)]
        if arrs[0].shape != (self.d_model, 8) or arrs[1].shape != (4, 8, 8) or \
                arrs[2].shape != (4, 256, 8) or arrs[3].shape != (256, self.d_ff // self.block):
            raise ValueError("hashing predictor arrays have the wrong shapes")
        w = LsHashWeights(*[a.ctypes.data for a in arrs])
        _check(self.lib, self.ctx, self.lib.ls_set_hash_predictor(self.ctx, layer, ctypes.byref(w)))

    def ls_hash_predict(self, layer: int, x, B: int, scores) -> None:
        _check(self.lib, self.ctx, self.lib.ls_hash_predict(self.ctx, layer, _ptr(x), B, _ptr(scores)))

    def ls_decode_step_streamed(self, x, k: int, n_stages: int, mode: int, k_spec: int = 0
                                ) -> LsStreamReport:
        rep = LsStreamReport()
        _check(self.lib, self.ctx, self.lib.ls_decode_step_streamed(self.ctx, _ptr(x), k, n_stages,
                                                                    mode, k_spec, ctypes.byref(rep)))
        return rep

    def ls_decode_step(self, x, B: int, k: int) -> None:
        _check(self.lib, self.ctx, self.lib.ls_decode_step(self.ctx, _ptr(x), B, k))

    def ls_configure(self, key: int, value: int) -> None:
        _check(self.lib, self.ctx, self.lib.ls_configure(self.ctx, key, int(value)))

    def ls_debug_decode_trace(self, layer: int, x_in=None, scores=None) -> None:
        _check(self.lib, self.ctx, self.lib.ls_debug_decode_trace(self.ctx, layer, _ptr(x_in),
                                                                  _ptr(scores)))

    def ls_debug_phase_trace(self):
        """Phase timestamps [n_layers, 16] (100 MHz ticks) of the traced workgroup (see PHASES)."""
        out = np.zeros((self.n_layers, len(PHASES)), np.int64)
        n = ctypes.c_int64()
        _check(self.lib, self.ctx, self.lib.ls_debug_phase_trace(self.ctx, out.ctypes.data, out.size,
                                                                 ctypes.byref(n)))
        return out

    def ls_debug_stages_done(self, layer: int) -> int:
        """Stages of the layer's latest flagged request whose done word carries its tag."""
        n = ctypes.c_int32()
        _check(self.lib, self.ctx, self.lib.ls_debug_stages_done(self.ctx, layer, ctypes.byref(n)))
        return n.value

    def ls_ffn_sync(self) -> None:
        _check(self.lib, self.ctx, self.lib.ls_ffn_sync(self.ctx))

    def ls_set_kernel_timing(self, enable: bool, kernels=None) -> None:
        """enable: bracket launches with HIP events; kernels: the LS_K_* ids to bracket
        (default: every kernel)."""
        mask = 0
        if enable:
            mask = 1 if kernels is None else sum(1 << int(k) for k in set(kernels) if int(k) != LS_K_PRENORM)
            if mask == 0:
                raise ValueError("no launching kernel id given")
        _check(self.lib, self.ctx, self.lib.ls_set_kernel_timing(self.ctx, mask))

    def ls_kernel_timing(self, kernel: int, reset: bool = False):
        """(total milliseconds, launches) of one kernel id since the last reset."""
        ms, n = ctypes.c_double(), ctypes.c_int64()
        _check(self.lib, self.ctx, self.lib.ls_kernel_timing(self.ctx, kernel, int(reset),
                                                             ctypes.byref(ms), ctypes.byref(n)))
        return ms.value, n.value

    def ls_measure_read_bandwidth(self, buf, reps: int = 10):
        """(best, median) GB/s of a streaming-read kernel over the device tensor buf."""
        best, med = ctypes.c_double(), ctypes.c_double()
        nbytes = buf.numel() * buf.element_size()
        _check(self.lib, self.ctx, self.lib.ls_measure_read_bandwidth(self.ctx, _ptr(buf), nbytes, reps,
                                                                      ctypes.byref(best), ctypes.byref(med)))
        return best.value, med.value

    def ls_debug_last_activations(self, dst) -> int:
        n = ctypes.c_int64()
        _check(self.lib, self.ctx, self.lib.ls_debug_last_activations(self.ctx, _ptr(dst),
                                                                      dst.numel(), ctypes.byref(n)))
        return n.value


def _dtype(t, what: str, allowed) -> int:
    """Library type of a tensor's elements."""
    import torch
    ls = {torch.float32: LS_F32, torch.float16: LS_F16, torch.bfloat16: LS_BF16, torch.int8: LS_I8}.get(t.dtype)
    if ls not in allowed:
        raise ValueError(f"{what} has type {t.dtype}")
    return ls


def _strides(t, shape, what: str):
    """Element strides of a device tensor of the given shape, 0 where a dimension has one entry
    (and 1, not counted, for the last: it must be contiguous)."""
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if not t.is_cuda:
        raise ValueError(f"{what} is not on the GPU")
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{what} is not contiguous in its last dimension")
    return [t.stride(i) if t.shape[i] > 1 else 0 for i in range(t.dim() - 1)]


class Ops:
    """The decoder layer's operators around the FFN (``ls_ops.h``) on one stream.  Methods mirror
    the C entry points; sizes, strides and types are those of the tensors they are given."""

    def __init__(self, *, workspace_bytes=0, stream=None):
        self.lib = load()
        import torch
        if stream is None:
            stream = torch.cuda.current_stream()
        self.torch_stream = stream
        h = ctypes.c_void_p()
        desc = LsOpsDesc(workspace_bytes, ctypes.c_void_p(stream.cuda_stream), 0)
        self.ctx = None
        self._check(self.lib.ls_ops_create(ctypes.byref(desc), ctypes.byref(h)))
        self.ctx = h
        _live.add(self)

    def _check(self, status: int) -> None:
        if status != LS_OK:
            msg = self.lib.ls_ops_last_error(self.ctx)
            raise LsError(status, msg.decode() if msg else "")

    def close(self):
        if getattr(self, "ctx", None):
            self.lib.ls_ops_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def ls_ops_sync(self) -> None:
        self._check(self.lib.ls_ops_sync(self.ctx))

    def ls_norm_residual(self, x, *, y=None, gate=None, post_norm=False, post_weight=None, pre_norm=False, pre_weight=None,
                         x_scale=1.0, y_scale=1.0, eps=1e-6, x_out=None, h=None) -> None:
        """x, x_out: fp32 [T, d]; y, h: [T, d]; gate: [d] or [T, d]; the weights: [d]."""
        T, d = x.shape
        _dtype(x, "x", (LS_F32,))
        (xs,) = _strides(x, (T, d), "x")
        rest = [(t, n) for t, n in ((y, "y"), (h, "h"), (gate, "gate"), (post_weight, "post_weight"), (pre_weight, "pre_weight"))
                if t is not None]
        dt = _dtype(rest[0][0], rest[0][1], (LS_F32, LS_F16, LS_BF16)) if rest else LS_F32
        for t, n in rest:
            _dtype(t, n, (dt,))
        ys = _strides(y, (T, d), "y")[0] if y is not None else 0
        hs = _strides(h, (T, d), "h")[0] if h is not None else 0
        gs = 0
        if gate is not None:
            gs = _strides(gate, (T, d), "gate")[0] if gate.dim() == 2 else 0 * len(_strides(gate, (d,), "gate"))
        for t, n in ((post_weight, "post_weight"), (pre_weight, "pre_weight")):
            if t is not None:
                _strides(t, (d,), n)
        os_ = 0
        if x_out is not None:
            _dtype(x_out, "x_out", (LS_F32,))
            (os_,) = _strides(x_out, (T, d), "x_out")
        a = LsNormArgs(T, d, dt, int(post_norm), int(pre_norm), x_scale, y_scale, eps, _ptr(x), xs, _ptr(y), ys, _ptr(gate), gs,
                       _ptr(post_weight), _ptr(pre_weight), _ptr(x_out), os_, _ptr(h), hs)
        self._check(self.lib.ls_norm_residual(self.ctx, ctypes.byref(a)))

    def ls_linear_i8(self, x, w, w_scale, out, *, x_scale=None, bias=None) -> None:
        """x: [T, k] int8 with x_scale fp32 [T], or floating; w: int8 [n, k]; w_scale, bias: fp32 [n]; out: [T, n]."""
        T, k = x.shape
        n = w.shape[0]
        xt = _dtype(x, "x", (LS_I8, LS_F32, LS_F16, LS_BF16))
        _dtype(w, "w", (LS_I8,))
        ot = _dtype(out, "out", (LS_F32, LS_F16, LS_BF16))
        (xs,), (ws,), (os_,) = _strides(x, (T, k), "x"), _strides(w, (n, k), "w"), _strides(out, (T, n), "out")
        for t, shape, what in ((w_scale, (n,), "w_scale"), (bias, (n,), "bias"), (x_scale, (T,), "x_scale")):
            if t is not None:
                _dtype(t, what, (LS_F32,))
                _strides(t, shape, what)
        a = LsLinearI8Args(T, k, n, xt, ot, _ptr(x), xs, _ptr(x_scale), _ptr(w), ws, _ptr(w_scale), _ptr(bias), _ptr(out), os_)
        self._check(self.lib.ls_linear_i8(self.ctx, ctypes.byref(a)))

    @staticmethod
    def _cache(k_cache, v_cache) -> LsKvCache:
        """k_cache, v_cache: [n_pages, n_kv_heads, page_size, head_dim], of the same strides in any order."""
        dt = _dtype(k_cache, "k_cache", (LS_F32, LS_F16, LS_BF16))
        _dtype(v_cache, "v_cache", (dt,))
        s = _strides(k_cache, k_cache.shape, "k_cache")
        if _strides(v_cache, k_cache.shape, "v_cache") != s:
            raise ValueError("k_cache and v_cache have different strides")
        n, kv, page, d = k_cache.shape
        return LsKvCache(_ptr(k_cache), _ptr(v_cache), dt, n, page, kv, d, *s)

    def ls_kv_append(self, k_cache, v_cache, k, v, positions, slots, cos_sin, *, q=None, q_out=None, style=LS_ROPE_HALF) -> None:
        """k, v: [T, n_kv_heads, head_dim]; q, q_out: [T, n_heads, head_dim]; positions, slots: int32 [T];
        cos_sin: fp32 [n_pos, rot_dim], or None (with positions None) for a plain append."""
        import torch
        c = self._cache(k_cache, v_cache)
        T = k.shape[0]
        shape = (T, c.n_kv_heads, c.head_dim)
        for t, what in ((k, "k"), (v, "v"), (q, "q"), (q_out, "q_out")):
            if t is not None:
                _dtype(t, what, (c.dtype,))
        heads = 0 if q is None else q.shape[1]
        qs, qos = [0, 0], [0, 0]
        if q is not None:
            qs = _strides(q, (T, heads, c.head_dim), "q")
        if q_out is not None:
            qos = _strides(q_out, (T, heads, c.head_dim), "q_out")
        for t, what in ((positions, "positions"), (slots, "slots")):
            if t is not None and (t.dtype != torch.int32 or _strides(t, (T,), what)):
                raise ValueError(f"{what} must be int32")
        n_pos = rot = 0
        if cos_sin is not None:
            n_pos, rot = cos_sin.shape
            _dtype(cos_sin, "cos_sin", (LS_F32,))
            if not cos_sin.is_contiguous():
                raise ValueError("cos_sin is not contiguous")
            _strides(cos_sin, (n_pos, rot), "cos_sin")
        a = LsAppendArgs(T, heads, rot, n_pos, style, _ptr(k), *_strides(k, shape, "k"), _ptr(v), *_strides(v, shape, "v"),
                         _ptr(q), *qs, _ptr(q_out), *qos, _ptr(positions), _ptr(slots), _ptr(cos_sin))
        self._check(self.lib.ls_kv_append(self.ctx, ctypes.byref(c), ctypes.byref(a)))

    def ls_attend(self, q, k_cache, v_cache, pages, lens, out, *, max_len, scale, n_q=1, prefix_pages=None, prefix_len=0) -> None:
        """q, out: [n_seqs * n_q, n_heads, head_dim]; pages: int32 [n_seqs, pages of a sequence]; lens: int32 [n_seqs];
        prefix_pages: int32 [pages of the prefix]; max_len: a bound of lens that the caller knows."""
        import torch
        c = self._cache(k_cache, v_cache)
        T, heads, _ = q.shape
        n_seqs = lens.shape[0]
        _dtype(q, "q", (c.dtype,))
        _dtype(out, "out", (c.dtype,))
        if T != n_seqs * n_q:
            raise ValueError(f"q has {T} tokens, expected {n_seqs} sequences of {n_q}")
        qs, os_ = _strides(q, (T, heads, c.head_dim), "q"), _strides(out, (T, heads, c.head_dim), "out")
        for t, what in ((pages, "pages"), (lens, "lens"), (prefix_pages, "prefix_pages")):
            if t is not None and (t.dtype != torch.int32 or not t.is_cuda or (t.numel() > 0 and t.stride(-1) != 1)):
                raise ValueError(f"{what} must be int32 on the GPU, contiguous in its last dimension")
        if prefix_len > 0 and (prefix_pages is None or prefix_pages.numel() * c.page_size < prefix_len):
            raise ValueError("prefix_pages hold fewer than prefix_len keys")
        stride = 0
        if pages is not None:
            if pages.dim() != 2 or pages.shape[0] != n_seqs:
                raise ValueError("pages must have a row for each sequence")
            if pages.shape[1] * c.page_size < max_len:
                raise ValueError("pages hold fewer than max_len keys")
            stride = pages.stride(0) if n_seqs > 1 else pages.shape[1]
        a = LsAttendArgs(n_seqs, n_q, heads, prefix_len, max_len, scale, _ptr(q), *qs, _ptr(out), *os_, _ptr(prefix_pages),
                         _ptr(pages), stride, _ptr(lens))
        self._check(self.lib.ls_attend(self.ctx, ctypes.byref(c), ctypes.byref(a)))
