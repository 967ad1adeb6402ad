"""ctypes binding with the same names as include/dc.h."""
from __future__ import annotations

import ctypes as C
import os
from array import array
from typing import List, Optional, Sequence

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG, "libdc.so")
_lib = None

DC_MAX_CONV, DC_MAX_UP, DC_MAX_RES = 32, 4, 4
PIPE = {"conv": 1, "flow": 2, "vocoder": 3, "token2wav": 4}
PREC = {"f32": 0, "bf16": 1}
STATUS = {0: "DC_OK", 1: "DC_ERR_ARG", 2: "DC_ERR_CONFIG", 3: "DC_ERR_FRAMES", 4: "DC_ERR_OOM",
          5: "DC_ERR_CUDA", 6: "DC_ERR_TIMEOUT", 7: "DC_ERR_STATE"}

EXPORTS = ["dc_weights_count", "dc_create", "dc_destroy", "dc_stream_open", "dc_stream_reset",
           "dc_stream_close", "dc_decode_chunk", "dc_decode_batch", "dc_decode_chunk_host",
           "dc_stream_carry_info", "dc_get_counters", "dc_status_str", "dc_last_error",
           "dc_decode_batch_host", "dc_profile_begin", "dc_profile_end", "dc_conv_stack_noalloc",
           "dc_selftest_bounded_wait", "dc_stream_snapshot", "dc_stream_restore", "dc_snapshot_free",
           "dc_decode_wavefront", "dc_decode_wavefront_batch", "dc_stream_check_guards", "dc_test_fail_allocation", "dc_test_wavefront_form", "dc_measure_fp32_peak",
           "dc_cache_open", "dc_cache_close", "dc_cache_check", "dc_cache_append", "dc_cache_attend", "dc_sample_tokens"]


class dc_config(C.Structure):
    _fields_ = [("size", C.c_uint32), ("pipeline", C.c_int32), ("precision", C.c_int32),
                ("hidden", C.c_int32), ("n_conv", C.c_int32), ("dilations", C.c_int32 * DC_MAX_CONV),
                ("n_attn", C.c_int32), ("n_heads", C.c_int32), ("head_dim", C.c_int32),
                ("kv_cap", C.c_int32), ("n_steps", C.c_int32), ("f_chunk", C.c_int32),
                ("mel_dim", C.c_int32), ("n_up", C.c_int32), ("up_strides", C.c_int32 * DC_MAX_UP),
                ("up_channels", C.c_int32 * (DC_MAX_UP + 1)), ("n_res", C.c_int32),
                ("res_dilations", C.c_int32 * DC_MAX_RES), ("n_fft", C.c_int32), ("hop", C.c_int32),
                ("rms_eps", C.c_float), ("logmag_clamp", C.c_float), ("max_batch", C.c_int32),
                ("f_prompt", C.c_int32), ("f_lookahead", C.c_int32), ("noise_seed_lo", C.c_uint32), ("noise_seed_hi", C.c_uint32),
                ("cfg_scale", C.c_float), ("max_wave_frames", C.c_int32), ("options", C.c_uint32),
                ("excitation_std", C.c_float), ("excitation_seed_lo", C.c_uint32), ("excitation_seed_hi", C.c_uint32)]


class dc_cache_config(C.Structure):
    _fields_ = [("size", C.c_uint32), ("dtype", C.c_int32), ("n_sessions", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("n_sink", C.c_int32), ("window", C.c_int32), ("ring_rows", C.c_int32)]


class dc_token_batch(C.Structure):
    _fields_ = [("size", C.c_uint32), ("n_seqs", C.c_int32), ("n_tokens", C.c_int32), ("max_tokens", C.c_int32),
                ("sessions_dev", C.c_void_p), ("cu_tokens_dev", C.c_void_p), ("start_dev", C.c_void_p)]


class dc_qk_norm(C.Structure):
    _fields_ = [("size", C.c_uint32), ("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("eps", C.c_float),
                ("q_gain_dev", C.c_void_p), ("k_gain_dev", C.c_void_p), ("inv_freq_dev", C.c_void_p)]


class dc_sample_rules(C.Structure):
    _fields_ = [("size", C.c_uint32), ("temperature_dev", C.c_void_p), ("top_k_dev", C.c_void_p), ("top_p_dev", C.c_void_p), ("min_p_dev", C.c_void_p)]


class DCError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = load_library().dc_last_error().decode()
        super().__init__(f"{where}: {STATUS.get(status, status)} {msg}")


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """Loads libdc.so; raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(f"{_LIB_PATH} is missing: run `python -m paper_2609_35115_b200.build`")
    lib = C.CDLL(_LIB_PATH)
    vp, cp = C.c_void_p, C.POINTER
    lib.dc_weights_count.restype = C.c_size_t
    lib.dc_weights_count.argtypes = [cp(dc_config)]
    lib.dc_create.argtypes = [vp, C.c_size_t, cp(dc_config), cp(vp)]
    lib.dc_destroy.argtypes = [vp]
    lib.dc_stream_open.argtypes = [vp, cp(vp)]
    lib.dc_stream_reset.argtypes = [vp, vp]
    lib.dc_stream_snapshot.argtypes = [vp, cp(vp), vp]
    lib.dc_stream_restore.argtypes = [vp, vp, vp]
    lib.dc_snapshot_free.argtypes = [vp]
    lib.dc_stream_close.argtypes = [vp]
    lib.dc_decode_chunk.argtypes = [vp, vp, C.c_int, vp, cp(C.c_int), vp]
    lib.dc_decode_batch.argtypes = [vp, C.c_int, cp(vp), cp(vp), cp(C.c_int), cp(vp), vp]
    lib.dc_decode_wavefront.argtypes = [vp, vp, C.c_longlong, vp, cp(C.c_longlong), vp]
    lib.dc_decode_wavefront_batch.argtypes = [vp, C.c_int, cp(vp), cp(vp), cp(C.c_longlong), cp(vp), vp]
    lib.dc_decode_chunk_host.argtypes = [vp, vp, C.c_int, vp, cp(C.c_int), vp]
    lib.dc_decode_batch_host.argtypes = [vp, C.c_int, cp(vp), cp(vp), cp(C.c_int), cp(vp), vp]
    lib.dc_profile_begin.argtypes = [vp, C.c_int]
    lib.dc_profile_end.argtypes = [vp, cp(C.c_double), cp(C.c_uint64)]
    lib.dc_conv_stack_noalloc.argtypes = [vp, C.c_int, C.c_int, cp(C.c_int), vp, C.c_int, vp, vp]
    lib.dc_selftest_bounded_wait.argtypes = [C.c_int]
    lib.dc_stream_check_guards.argtypes = [vp, cp(C.c_int)]
    lib.dc_test_fail_allocation.argtypes = [C.c_int]
    lib.dc_test_wavefront_form.argtypes = [vp, cp(C.c_int), cp(C.c_uint64)]
    lib.dc_measure_fp32_peak.argtypes = [cp(C.c_double)]
    lib.dc_stream_carry_info.argtypes = [vp, cp(C.c_uint64), C.c_int, cp(C.c_int)]
    lib.dc_sample_tokens.argtypes = [vp, C.c_int, C.c_int, C.c_int, C.c_longlong, cp(dc_sample_rules), vp, vp, vp, vp]
    lib.dc_get_counters.argtypes = [vp, cp(C.c_uint64)]
    lib.dc_cache_open.argtypes = [cp(dc_cache_config), vp, vp, cp(vp)]
    lib.dc_cache_close.argtypes = [vp]
    lib.dc_cache_check.argtypes = [vp]
    lib.dc_cache_append.argtypes = [vp, vp, vp, vp, C.c_longlong, vp, C.c_longlong, vp]     # (structures by address: the objects below keep them)
    lib.dc_cache_attend.argtypes = [vp, vp, vp, C.c_longlong, C.c_float, vp, C.c_longlong, vp]
    lib.dc_status_str.restype = C.c_char_p
    lib.dc_status_str.argtypes = [C.c_int]
    lib.dc_last_error.restype = C.c_char_p
    lib.dc_last_error.argtypes = []
    for fn in EXPORTS:
        if fn not in ("dc_weights_count", "dc_status_str", "dc_last_error"):
            getattr(lib, fn).restype = C.c_int
    _lib = lib
    return lib


OPT_NO_GRAPH, OPT_NO_PDL, OPT_NO_ZEROCOPY, OPT_SERIAL_TAILS, OPT_ROUNDED_NORM, OPT_GUARD_ZONES = 1, 2, 4, 8, 16, 32
OPT_CTA_PAIRS = 64
OPT_SKIP_CONV_GEMM, OPT_SKIP_ATTENTION, OPT_EMPTY_KERNELS = 1 << 16, 1 << 17, 1 << 18     # measurement only: outputs are meaningless


def make_config(cfg, max_batch: int = 1, max_wave_frames: int = 0, options: int = 0) -> dc_config:
    """dc_workloads.DCConfig (or any object with the same attributes) -> dc_config."""
    c = dc_config()
    c.size = C.sizeof(dc_config)
    c.pipeline = PIPE[cfg.pipeline]
    c.precision = PREC[cfg.precision]
    c.hidden = cfg.hidden
    c.n_conv = len(cfg.dilations)
    for i, d in enumerate(cfg.dilations):
        c.dilations[i] = d
    c.n_attn, c.n_heads, c.head_dim, c.kv_cap = cfg.n_attn_layers, cfg.n_heads, cfg.head_dim, cfg.kv_cap
    c.n_steps, c.f_chunk, c.mel_dim = cfg.n_steps, cfg.f_chunk, cfg.mel_dim
    if cfg.pipeline in ("vocoder", "token2wav"):
        c.n_up = len(cfg.up_strides)
        for i, s in enumerate(cfg.up_strides):
            c.up_strides[i] = s
        for i, ch in enumerate(cfg.up_channels):
            c.up_channels[i] = ch
        c.n_res = len(cfg.res_dilations)
        for i, d in enumerate(cfg.res_dilations):
            c.res_dilations[i] = d
        c.n_fft, c.hop = cfg.n_fft, cfg.hop
    c.rms_eps, c.logmag_clamp = cfg.rms_eps, cfg.logmag_clamp
    c.max_batch = max_batch
    c.max_wave_frames = max_wave_frames
    c.options = options
    c.excitation_std = float(getattr(cfg, "excitation_std", 0.0))
    eseed = int(getattr(cfg, "excitation_seed", 0))
    c.excitation_seed_lo, c.excitation_seed_hi = eseed & 0xFFFFFFFF, (eseed >> 32) & 0xFFFFFFFF
    c.cfg_scale = float(getattr(cfg, "cfg_scale", 0.0))
    c.f_prompt = int(getattr(cfg, "f_prompt", 0))
    c.f_lookahead = int(getattr(cfg, "f_lookahead", 0))
    seed = int(getattr(cfg, "noise_seed", 0))
    c.noise_seed_lo, c.noise_seed_hi = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    return c


def _check(status: int, where: str):
    if status != 0:
        raise DCError(status, where)


def _cuda_stream_handle(stream) -> Optional[int]:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    return stream if isinstance(stream, int) else stream.cuda_stream


def _result(shape, dtype, device, stream):
    """Memory for what a call returns: the current stream's, or that of the stream it is given, which writes it; the current stream may then be
    using it when it is dropped."""
    import torch
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    here = torch.cuda.current_stream(device)
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=device) if stream else torch.cuda.default_stream(device)
    with torch.cuda.stream(stream):
        out = torch.empty(shape, dtype=dtype, device=device)
    if stream.cuda_stream != here.cuda_stream:
        out.record_stream(here)
    return out


class Snapshot:
    def __init__(self, lib, handle):
        self.lib, self.handle = lib, handle

    def free(self):
        if self.handle:
            _check(self.lib.dc_snapshot_free(self.handle), "dc_snapshot_free")
            self.handle = None


class Model:
    """dc_create / dc_destroy."""

    def __init__(self, cfg, weights: np.ndarray, max_batch: int = 1, max_wave_frames: int = 0, options: int = 0):
        self.lib = load_library()
        self.cfg = cfg
        self.c_cfg = make_config(cfg, max_batch, max_wave_frames, options)
        w = np.ascontiguousarray(weights, dtype=np.float32)
        self.handle = C.c_void_p()
        _check(self.lib.dc_create(w.ctypes.data, w.size, C.byref(self.c_cfg), C.byref(self.handle)), "dc_create")
        self.out_per_frame = cfg.out_per_frame
        self.in_dim = cfg.in_dim

    def weights_count(self) -> int:
        return self.lib.dc_weights_count(C.byref(self.c_cfg))

    def open_stream(self) -> "Stream":
        return Stream(self)

    def counters(self) -> List[int]:
        out = (C.c_uint64 * 8)()
        _check(self.lib.dc_get_counters(self.handle, out), "dc_get_counters")
        return list(out)

    def profile_begin(self, max_launches: int = 1 << 16):
        _check(self.lib.dc_profile_begin(self.handle, max_launches), "dc_profile_begin")

    def profile_end(self):
        """Returns ({class: ms}, {class: launches}) summed since profile_begin."""
        ms = (C.c_double * 8)()
        n = (C.c_uint64 * 8)()
        _check(self.lib.dc_profile_end(self.handle, ms, n), "dc_profile_end")
        names = ["gemm_conv", "gemm_proj", "attention", "rmsnorm", "prep", "tapconv_f32", "head_istft_f32"]
        pairs = bool(self.c_cfg.options & OPT_CTA_PAIRS)      # class 7 is one or the other
        names += ["gemm_pair", "flow_cluster"] if pairs else ["flow_cluster", "gemm_pair"]
        return ({k: ms[i] if i < 8 else 0.0 for i, k in enumerate(names)}, {k: n[i] if i < 8 else 0 for i, k in enumerate(names)})

    def wavefront_form(self):
        """dc_test_wavefront_form: (clusters resident, wavefront passes with one slot per cluster so far)."""
        n, passes = C.c_int(0), C.c_uint64(0)
        _check(self.lib.dc_test_wavefront_form(self.handle, C.byref(n), C.byref(passes)), "dc_test_wavefront_form")
        return n.value, passes.value

    def destroy(self):
        if self.handle:
            _check(self.lib.dc_destroy(self.handle), "dc_destroy")
            self.handle = C.c_void_p()


class Stream:
    """dc_stream_open / dc_decode_chunk / dc_stream_reset / dc_stream_close."""

    def __init__(self, model: Model):
        self.model = model
        self.lib = model.lib
        self.handle = C.c_void_p()
        _check(self.lib.dc_stream_open(model.handle, C.byref(self.handle)), "dc_stream_open")
        self.address = self.handle.value or 0    # the handle as a plain number: batch calls make an array of them

    def decode_chunk(self, feats, out=None, stream=None):
        """feats: CUDA float32 tensor [T, in_dim]; returns a CUDA float32 tensor."""
        import torch
        assert feats.is_cuda and feats.dtype == torch.float32 and feats.is_contiguous()
        T = feats.shape[0]
        if out is None:
            n = max(T, 0) * self.model.out_per_frame
            out = _result((max(n, 1),), torch.float32, feats.device, stream)
        n_out = C.c_int(0)
        st = self.lib.dc_decode_chunk(self.handle, feats.data_ptr(), T, out.data_ptr(), C.byref(n_out),
                                      _cuda_stream_handle(stream))
        _check(st, "dc_decode_chunk")
        res = out[: n_out.value]
        if self.model.cfg.pipeline not in ("vocoder", "token2wav"):
            res = res.view(-1, self.model.out_per_frame)      # committed frames (fewer than T when the call carried look-ahead frames)
        return res

    def decode_wavefront(self, feats, out=None, stream=None):
        """dc_decode_wavefront: feats is a CUDA float32 tensor [n_frames, in_dim] holding all the stream's
        remaining input; returns what the chunk-by-chunk calls would have returned, concatenated."""
        import torch
        assert feats.is_cuda and feats.dtype == torch.float32 and feats.is_contiguous()
        n = feats.shape[0]
        if out is None:
            out = _result((n * self.model.out_per_frame,), torch.float32, feats.device, stream)
        n_out = C.c_longlong(0)
        st = self.lib.dc_decode_wavefront(self.handle, feats.data_ptr(), n, out.data_ptr(), C.byref(n_out),
                                          _cuda_stream_handle(stream))
        _check(st, "dc_decode_wavefront")
        res = out[: n_out.value]
        if self.model.cfg.pipeline not in ("vocoder", "token2wav"):
            res = res.view(-1, self.model.out_per_frame)
        return res

    def decode_chunk_host(self, feats_host, out_host, stream=None) -> int:
        """feats_host / out_host: CPU float32 tensors (pinned for true async copies)."""
        T = feats_host.shape[0]
        n_out = C.c_int(0)
        st = self.lib.dc_decode_chunk_host(self.handle, feats_host.data_ptr(), T, out_host.data_ptr(),
                                           C.byref(n_out), _cuda_stream_handle(stream))
        _check(st, "dc_decode_chunk_host")
        return n_out.value

    def decode_raw(self, feats_ptr: int, T: int, out_ptr: int, stream=None) -> int:
        """Unchecked pass-through (used by the error-path tests)."""
        n_out = C.c_int(0)
        return self.lib.dc_decode_chunk(self.handle, feats_ptr, T, out_ptr, C.byref(n_out),
                                        _cuda_stream_handle(stream))

    def carry_info(self):
        buf = (C.c_uint64 * 256)()
        n = C.c_int(0)
        _check(self.lib.dc_stream_carry_info(self.handle, buf, 128, C.byref(n)), "dc_stream_carry_info")
        return [(buf[2 * i], buf[2 * i + 1]) for i in range(min(n.value, 128))]

    def snapshot(self, stream=None) -> "Snapshot":
        """Device-side copy of every carry of the stream plus its clocks (dc_stream_snapshot)."""
        h = C.c_void_p()
        _check(self.lib.dc_stream_snapshot(self.handle, C.byref(h), _cuda_stream_handle(stream)), "dc_stream_snapshot")
        return Snapshot(self.lib, h)

    def restore(self, snap: "Snapshot", stream=None):
        """Writes a snapshot back in place (of this stream or of another stream of the same model)."""
        _check(self.lib.dc_stream_restore(self.handle, snap.handle, _cuda_stream_handle(stream)), "dc_stream_restore")

    def check_guards(self) -> int:
        """dc_stream_check_guards: returns the number of damaged guard zones (0 = intact); raises on other errors."""
        n = C.c_int(0)
        st = self.lib.dc_stream_check_guards(self.handle, C.byref(n))
        if st not in (0, 7):
            _check(st, "dc_stream_check_guards")
        return n.value

    def reset(self, stream=None):
        _check(self.lib.dc_stream_reset(self.handle, _cuda_stream_handle(stream)), "dc_stream_reset")

    def close(self):
        if self.handle:
            _check(self.lib.dc_stream_close(self.handle), "dc_stream_close")
            self.handle, self.address = C.c_void_p(), 0


def _ptr_array(items, n):
    """Pointers of n chunks: a list of tensors, or one contiguous tensor [n, T, width] (fast path)."""
    if hasattr(items, "data_ptr"):
        assert items.is_contiguous() and items.shape[0] == n
        stride = items.stride(0) * items.element_size()
        ptrs = items.data_ptr() + stride * np.arange(n, dtype=np.uint64)
        return (C.c_void_p * n).from_buffer_copy(ptrs.astype(np.uint64).tobytes()), items.shape[1]
    return (C.c_void_p * n)(*[t.data_ptr() for t in items]), None


def _batch_args(model: Model, streams: Sequence[Stream], feats, outs):
    n = len(streams)
    hs = (C.c_void_p * n).from_buffer(array("Q", [s.address for s in streams]))
    fp, T = _ptr_array(feats, n)
    op, _ = _ptr_array(outs, n)
    nf = (C.c_int * n)(*([T] * n if T is not None else [f.shape[0] for f in feats]))
    return n, hs, fp, nf, op


def decode_batch_host(model: Model, streams: Sequence[Stream], feats_host, outs_host, stream=None):
    """dc_decode_batch_host: feats_host / outs_host are lists of CPU float32 tensors, or single contiguous
    CPU tensors [n_streams, T, width] (one chunk per stream)."""
    n, hs, fp, nf, op = _batch_args(model, streams, feats_host, outs_host)
    _check(model.lib.dc_decode_batch_host(model.handle, n, hs, fp, nf, op, _cuda_stream_handle(stream)),
           "dc_decode_batch_host")


def decode_batch(model: Model, streams: Sequence[Stream], feats, outs, stream=None):
    """dc_decode_batch: one chunk for each stream; feats / outs are lists of CUDA float32 tensors
    ([T_i, in_dim] / [T_i, out]) or single contiguous CUDA tensors [n_streams, T, width]."""
    n, hs, fp, nf, op = _batch_args(model, streams, feats, outs)
    _check(model.lib.dc_decode_batch(model.handle, n, hs, fp, nf, op, _cuda_stream_handle(stream)),
           "dc_decode_batch")


def decode_wavefront_batch(model: Model, streams: Sequence[Stream], feats, outs=None, stream=None):
    """dc_decode_wavefront_batch: feats[i] is a CUDA float32 tensor [n_frames_i, in_dim] with all of stream i's
    remaining input; returns the list of outputs (allocated here unless given)."""
    import torch
    n = len(streams)
    if outs is None:
        outs = [_result((f.shape[0] * model.out_per_frame,), torch.float32, f.device, stream) for f in feats]
    for f in feats:
        assert f.is_cuda and f.dtype == torch.float32 and f.is_contiguous()
    hs = (C.c_void_p * n)(*[s.handle for s in streams])
    fp = (C.c_void_p * n)(*[f.data_ptr() for f in feats])
    nf = (C.c_longlong * n)(*[f.shape[0] for f in feats])
    op = (C.c_void_p * n)(*[o.data_ptr() for o in outs])
    _check(model.lib.dc_decode_wavefront_batch(model.handle, n, hs, fp, nf, op, _cuda_stream_handle(stream)),
           "dc_decode_wavefront_batch")
    if model.cfg.pipeline not in ("vocoder", "token2wav"):
        outs = [o.view(-1, model.out_per_frame) for o in outs]
    return outs


def measure_fp32_peak() -> float:
    """dc_measure_fp32_peak: measured FP32 multiply-add throughput of the current device in TFLOP/s."""
    v = C.c_double(0.0)
    _check(load_library().dc_measure_fp32_peak(C.byref(v)), "dc_measure_fp32_peak")
    return v.value


def fail_allocation(nth: int) -> None:
    """dc_test_fail_allocation: the nth device allocation of the calling thread from now on fails (0 disarms)."""
    _check(load_library().dc_test_fail_allocation(nth), "dc_test_fail_allocation")


def selftest_bounded_wait(max_polls: int = 1000) -> int:
    """dc_selftest_bounded_wait: returns the dc_status (6 = DC_ERR_TIMEOUT is the expected outcome)."""
    return load_library().dc_selftest_bounded_wait(max_polls)


NOALLOC_SCRATCH_FLOATS = 1 << 19


def conv_stack_noalloc(weights_dev, hidden: int, dilations: Sequence[int], x, y, stream=None) -> int:
    """dc_conv_stack_noalloc: the conv residual stack over one whole sequence, for callers that
    must not allocate device memory.  weights_dev, x, y are CUDA float32 tensors the caller owns;
    returns the dc_status (0 = DC_OK) so that refusals can be inspected."""
    lib = load_library()
    d = (C.c_int * len(dilations))(*dilations)
    return lib.dc_conv_stack_noalloc(weights_dev.data_ptr(), hidden, len(dilations), d, x.data_ptr(),
                                     x.shape[0], y.data_ptr(), _cuda_stream_handle(stream))


# ---- the token step ------------------------------------------------------------------------------------------------------


def _dtype_code(t) -> int:
    import torch
    try:
        return {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}[t.dtype]
    except KeyError:
        raise TypeError(f"{t.dtype} is not served: float32, bfloat16 or float16") from None


def _vector(name, t, dtype, n=None, index=None):
    """Checks a small device array that a call reads or writes; returns its address (None: none)."""
    if t is None:
        return None
    at = t.get_device()      # (-1: not on a CUDA device)
    if t.dtype is dtype and at >= 0 and (index is None or at == index) and t.dim() == 1 and t.is_contiguous() and (n is None or t.numel() == n):
        return t.data_ptr()
    raise ValueError(f"{name}: a contiguous vector of {'' if n is None else f'{n} '}{dtype} on the call's CUDA device is wanted, not {tuple(t.shape)} {t.dtype} on {t.device}")


class TokenBatch:
    """dc_token_batch: the sequences of a call.  start (and sessions, cu_tokens) are CUDA int32 vectors that the program may rewrite in
    place between calls or graph replays; the object keeps references to them.  With cu_tokens, n_tokens is the number of rows of the call's
    matrices and max_tokens the most that one sequence brings (a sequence that brings more is left out)."""

    def __init__(self, sessions, start, cu_tokens=None, n_tokens: Optional[int] = None, max_tokens: Optional[int] = None):
        import torch
        if cu_tokens is not None and (n_tokens is None or max_tokens is None):
            raise ValueError("n_tokens and max_tokens are needed with cu_tokens")
        self.index, n = start.get_device(), start.shape[0]
        self._kept = (sessions, start, cu_tokens)
        self.c = c = dc_token_batch()
        c.size, c.n_seqs, c.max_tokens = C.sizeof(dc_token_batch), n, 1 if max_tokens is None else max_tokens
        c.n_tokens = n if n_tokens is None else n_tokens
        c.start_dev = _vector("start", start, torch.int32, n)
        c.sessions_dev = _vector("sessions", sessions, torch.int32, n, self.index)
        c.cu_tokens_dev = _vector("cu_tokens", cu_tokens, torch.int32, n + 1, self.index)
        self.n_tokens, self.address = c.n_tokens, C.addressof(c)


class QKNorm:
    """dc_qk_norm: gains [head_dim] and rotation frequencies [rot_dim / 2], CUDA float32 vectors that the object keeps."""

    def __init__(self, q_gain, k_gain, inv_freq=None, eps: float = 1e-6, interleaved: bool = False):
        import torch
        self.index, self.head_dim = q_gain.get_device(), q_gain.shape[0]
        self._kept = (q_gain, k_gain, inv_freq)
        self.c = c = dc_qk_norm()
        c.size, c.eps, c.interleaved = C.sizeof(dc_qk_norm), eps, int(interleaved)
        c.q_gain_dev = _vector("q_gain", q_gain, torch.float32)
        c.k_gain_dev = _vector("k_gain", k_gain, torch.float32, self.head_dim, self.index)
        c.rot_dim = 0 if inv_freq is None else 2 * inv_freq.shape[0]
        c.inv_freq_dev = _vector("inv_freq", inv_freq, torch.float32, None, self.index)
        self.address = C.addressof(c)


class TokenCache:
    """dc_cache_open / dc_cache_append / dc_cache_attend: keys and values of many sessions with a sliding window and
    first tokens that stay, in the caller's tensors k and v [sessions, kv_heads, n_sink + ring_rows, head_dim] (bf16 or fp16)."""

    def __init__(self, k, v, n_heads: int, n_sink: int = 0, window: Optional[int] = None):
        self.handle = C.c_void_p()
        for name, t in (("k", k), ("v", v)):
            if not t.is_cuda or t.dim() != 4 or not t.is_contiguous() or t.shape != k.shape or t.dtype != k.dtype or t.device != k.device:
                raise ValueError(f"{name}: a contiguous CUDA tensor [sessions, kv_heads, rows, head_dim] is wanted, k and v alike")
        self.lib, self.k, self.v, self.device, self.dtype, self._index = load_library(), k, v, k.device, k.dtype, k.get_device()
        self._append, self._attend = self.lib.dc_cache_append, self.lib.dc_cache_attend
        c = dc_cache_config()
        c.size, c.dtype, c.n_heads, c.n_sink = C.sizeof(dc_cache_config), _dtype_code(k), n_heads, n_sink
        c.n_sessions, c.n_kv_heads, rows, c.head_dim = k.shape
        c.ring_rows = rows - n_sink
        c.window = c.ring_rows if window is None else window
        self.c_cfg, self.head_dim, self.scale = c, c.head_dim, c.head_dim ** -0.5
        self._q_width, self._qkv_width = n_heads * c.head_dim, (n_heads + 2 * c.n_kv_heads) * c.head_dim
        with _on(self.device):
            _check(self.lib.dc_cache_open(C.byref(c), k.data_ptr(), v.data_ptr(), C.byref(self.handle)), "dc_cache_open")
        self._h = self.handle.value

    def _rows(self, name, t, width, n):
        """Checks a matrix of the call ([n, width] or [n, heads, head_dim], rows any stride apart); returns (address, stride).  (The checks are a good
        part of a single token's call: few and cheap ones.)"""
        st, d = t.stride(), self.head_dim
        if t.dtype is self.dtype and t.get_device() == self._index and (
                (len(st) == 3 and t.shape == (n, width // d, d) and st[1] == d and st[2] == 1) or (len(st) == 2 and t.shape == (n, width) and st[1] == 1)):
            return t.data_ptr(), st[0] if n > 1 else (max(st[0], width) + 7) & ~7      # (one row: any multiple of 8 will do)
        raise ValueError(f"{name}: {n} rows of {width} {self.dtype} values on {self.device} are wanted, not {tuple(t.shape)} (strides {st}) {t.dtype} on {t.device}")

    def append(self, qkv, batch: TokenBatch, norm: QKNorm, q=None, stream=None):
        """dc_cache_append: qkv is [n_tokens, (heads + 2 kv_heads) * head_dim]; returns the normalised, rotated queries
        [n_tokens, heads, head_dim] (in q if given; qkv's own query columns may be given)."""
        n = batch.n_tokens
        if q is None:
            q = _result((n, self.c_cfg.n_heads, self.head_dim), self.dtype, self.device, stream)
        if batch.index != self._index or norm.index != self._index or norm.head_dim != self.head_dim:
            raise ValueError("the batch and the norm belong to another device or head_dim than the cache")
        x, xs = self._rows("qkv", qkv, self._qkv_width, n)
        y, ys = self._rows("q", q, self._q_width, n)
        st = self._append(self._h, batch.address, norm.address, x, xs, y, ys, _raw_stream(self._index) if stream is None else _cuda_stream_handle(stream))
        if st:
            raise DCError(st, "dc_cache_append")
        return q

    def attend(self, q, batch: TokenBatch, out=None, scale: Optional[float] = None, stream=None):
        """dc_cache_attend: q is [n_tokens, heads, head_dim] (or [n_tokens, heads * head_dim]); returns the outputs, in the shape of q."""
        n = batch.n_tokens
        if out is None:
            out = _result(q.shape, self.dtype, self.device, stream)
        if batch.index != self._index:
            raise ValueError("the batch belongs to another device than the cache")
        x, xs = self._rows("q", q, self._q_width, n)
        y, ys = self._rows("out", out, self._q_width, n)
        st = self._attend(self._h, batch.address, x, xs, self.scale if scale is None else scale, y, ys, _raw_stream(self._index) if stream is None else _cuda_stream_handle(stream))
        if st:
            raise DCError(st, "dc_cache_attend")
        return out

    def check(self):
        """dc_cache_check: waits for the device; raises if a bounded device-side wait of an attention call has given up."""
        with _on(self.device):
            _check(self.lib.dc_cache_check(self._h), "dc_cache_check")

    def close(self):
        if self.handle:
            _check(self.lib.dc_cache_close(self.handle), "dc_cache_close")
            self.handle, self._h = C.c_void_p(), None

    def __del__(self):
        try:
            self.close()
        except Exception:      # (the interpreter, or the context, is going)
            pass


def sample_tokens(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, tokens=None, probs=None, stream=None):
    """dc_sample_tokens: the next token of every row of logits [rows, vocab] (float32, bfloat16 or float16, rows any stride apart) from the random numbers
    u [rows] in [0, 1).  The rules are CUDA vectors [rows] (float32; top_k int32) or None: off.  Returns the tokens (int32 [rows], in `tokens` if given);
    probs, if given, receives each token's share of the kept mass.  The logits' device has to be the current one."""
    import torch
    if logits.dim() != 2 or not logits.is_cuda or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError(f"logits: CUDA rows [rows, vocab] are wanted, not {tuple(logits.shape)}")
    n, vocab = logits.shape
    f32, i32, at, stride = torch.float32, torch.int32, logits.get_device(), logits.stride(0)
    if torch.cuda.current_device() != at:      # (the library launches on the current device)
        raise ValueError(f"logits: they are on device {at}, the current device is {torch.cuda.current_device()}")
    if tokens is None:
        tokens = _result((n,), i32, logits.device, stream)
    r = dc_sample_rules(_RULES_SIZE, _vector("temperature", temperature, f32, n, at), _vector("top_k", top_k, i32, n, at), _vector("top_p", top_p, f32, n, at),
                        _vector("min_p", min_p, f32, n, at))
    st = load_library().dc_sample_tokens(logits.data_ptr(), _dtype_code(logits), n, vocab, stride if n > 1 else max(stride, vocab), C.byref(r), _vector("u", u, f32, n, at),
                                         _vector("tokens", tokens, i32, n, at), _vector("probs", probs, f32, n, at), _raw_stream(at) if stream is None else _cuda_stream_handle(stream))
    if st:
        raise DCError(st, "dc_sample_tokens")
    return tokens


_RULES_SIZE = C.sizeof(dc_sample_rules)


def _on(device):
    import torch
    return torch.cuda.device(device)


def _raw_stream(index: int) -> int:
    """The current stream of a device (which need not be the current device): the tensors' own."""
    global _raw_stream
    import torch
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
    return _raw_stream(index)
