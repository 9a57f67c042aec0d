"""Thin ctypes binding of libsali (include/sali.h): argument marshalling only.

PyTorch supplies device memory (`tensor.data_ptr()`) and streams
(`torch.cuda.current_stream().cuda_stream`); every step of the method runs in
the library's HIP kernels.  There is no CPU fallback: a missing library or a
non-zero return code raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import numpy as np
import torch   # imported before the library is loaded so that both share one HIP runtime

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libsali.so")
_lib = None

TOKENS = 576
MAX_BATCH = 16          # SALI_MAX_BATCH
TIER_FP16, TIER_INT8, TIER_INT4, TIER_PRUNE = 0, 1, 2, 3
FAULT_OVERFLOW, FAULT_NONFINITE, FAULT_NAN_SCORE, FAULT_NO_DATA, FAULT_PAGE, FAULT_BATCH = 1, 2, 4, 8, 16, 32
STORE_16, STORE_INT8, STORE_INT4 = 0, 1, 2


class SaliError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {error_string(code)} ({code})")
        self.code = code


class sali_config(C.Structure):
    _fields_ = [
        ("src_h", C.c_int32), ("src_w", C.c_int32), ("grid", C.c_int32),
        ("flow_levels", C.c_int32), ("flow_iters", C.c_int32),
        ("tau_t", C.c_float), ("theta_r", C.c_float),
        ("canny_lo", C.c_int32), ("canny_hi", C.c_int32),
        ("tier_mode", C.c_int32),
        ("tau_high", C.c_float), ("tau_med", C.c_float), ("tau_low", C.c_float),
        ("k_fp16", C.c_int32), ("k_int8", C.c_int32), ("k_int4", C.c_int32),
        ("n_layers", C.c_int32), ("n_heads", C.c_int32), ("head_dim", C.c_int32), ("group", C.c_int32),
        ("cap_fp16", C.c_int64), ("cap_int8", C.c_int64), ("cap_int4", C.c_int64),
        ("max_frames", C.c_int32), ("budget_tokens", C.c_int32), ("tiles_per_frame", C.c_int32), ("adapt_rate_q8", C.c_int32),
    ]


class sali_gate(C.Structure):
    _fields_ = [("n_static", C.c_int32), ("r_frame", C.c_float), ("redundant", C.c_int32), ("reserved", C.c_int32)]


class sali_frame_row(C.Structure):
    _fields_ = [("frame_id", C.c_int32), ("src", C.c_int32), ("stored", C.c_int32),
                ("base16", C.c_int32), ("base8", C.c_int32), ("base4", C.c_int32),
                ("n16", C.c_int32), ("n8", C.c_int32), ("n4", C.c_int32), ("n_pruned", C.c_int32),
                ("reserved", C.c_int32 * 2)]

    def as_tuple(self):
        return (self.frame_id, self.src, self.stored, self.base16, self.base8, self.base4,
                self.n16, self.n8, self.n4, self.n_pruned)


class sali_pool_layout(C.Structure):
    _fields_ = [("off_fp16", C.c_uint64), ("off_codes8", C.c_uint64), ("off_scale8", C.c_uint64),
                ("off_codes4", C.c_uint64), ("off_scale4", C.c_uint64), ("off_zero4", C.c_uint64),
                ("total_bytes", C.c_uint64)]


class sali_pages_config(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("n_kv_heads", C.c_int32), ("n_heads", C.c_int32), ("head_dim", C.c_int32),
                ("page_tokens", C.c_int32), ("n_pages", C.c_int32), ("dtype", C.c_int32), ("store", C.c_int32)]


class sali_page_batch(C.Structure):
    _fields_ = [("d_start", C.c_void_p), ("d_length", C.c_void_p), ("d_table", C.c_void_p), ("n_seqs", C.c_int32), ("table_width", C.c_int32),
                ("n_tokens", C.c_int32), ("max_q", C.c_int32), ("max_kv", C.c_int32), ("reserved", C.c_int32)]


class sali_rows(C.Structure):
    _fields_ = [("d", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


EXPORTS = {
    "sali_workspace_bytes": (C.c_int, [C.POINTER(sali_config), C.POINTER(C.c_size_t), C.POINTER(C.c_size_t),
                                       C.POINTER(C.c_size_t)]),
    "sali_pool_offsets": (C.c_int, [C.POINTER(sali_config), C.POINTER(sali_pool_layout)]),
    "sali_create": (C.c_int, [C.POINTER(sali_config), C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(C.c_void_p)]),
    "sali_destroy": (None, [C.c_void_p]),
    "sali_reset": (C.c_int, [C.c_void_p, C.c_void_p]),
    "sali_set_gate_thresholds": (C.c_int, [C.c_void_p, C.c_float, C.c_float]),
    "sali_set_tier_params": (C.c_int, [C.c_void_p, C.c_int32, C.c_float, C.c_float, C.c_float, C.c_int32, C.c_int32,
                                       C.c_int32]),
    "sali_flow_score": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                  C.c_void_p]),
    "sali_saliency_pool": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "sali_kv_compress": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]),
    "sali_kv_decompress": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]),
    "sali_step": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]),
    "sali_analyze": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]),
    "sali_analyze_batch": (C.c_int, [C.c_void_p, C.POINTER(C.c_void_p), C.c_int32, C.c_int32, C.c_void_p]),
    "sali_store": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]),
    "sali_store_batch": (C.c_int, [C.c_void_p, C.POINTER(C.c_void_p), C.c_int32, C.c_int32, C.c_void_p]),
    "sali_kv_decompress_batch": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.POINTER(C.c_void_p), C.c_void_p,
                                           C.c_void_p]),
    "sali_step_batch": (C.c_int, [C.c_void_p, C.POINTER(C.c_void_p), C.POINTER(C.c_void_p), C.c_int32, C.c_int32,
                                  C.c_void_p]),
    "sali_attend_decode": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_int32, C.c_float, C.c_void_p,
                                     C.c_void_p, C.c_void_p]),
    "sali_attend_decode_gqa": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_float,
                                         C.c_void_p, C.c_void_p, C.c_void_p]),
    "sali_attend_decode_static": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_int32, C.c_float,
                                            C.c_void_p, C.c_void_p, C.c_void_p]),
    "sali_step_pipelined": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p,
                                      C.c_void_p]),
    "sali_read_frame_table": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p]),
    "sali_read_frame_tiers": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]),
    "sali_read_last_step": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "sali_read_analysis": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "sali_set_profile_events": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p]),
    "sali_get_status": (C.c_int, [C.c_void_p, C.POINTER(C.c_uint32), C.c_void_p]),
    "sali_error_string": (C.c_char_p, [C.c_int]),
    "sali_pages_bytes": (C.c_int, [C.POINTER(sali_pages_config), C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]),
    "sali_pages_create": (C.c_int, [C.POINTER(sali_pages_config), C.c_void_p, C.c_void_p, C.POINTER(C.c_void_p)]),
    "sali_pages_destroy": (None, [C.c_void_p]),
    "sali_pages_append": (C.c_int, [C.c_void_p, C.c_int32, C.POINTER(sali_page_batch), C.POINTER(sali_rows), C.POINTER(sali_rows), C.c_void_p]),
    "sali_pages_read": (C.c_int, [C.c_void_p, C.c_int32, C.POINTER(sali_page_batch), C.POINTER(sali_rows), C.POINTER(sali_rows), C.c_void_p]),
    "sali_pages_attend": (C.c_int, [C.c_void_p, C.c_int32, C.POINTER(sali_page_batch), C.POINTER(sali_rows), C.c_float, C.c_int32, C.c_int32,
                                    C.c_void_p, C.c_void_p, C.POINTER(sali_rows), C.c_void_p, C.c_void_p]),
    "sali_pages_get_status": (C.c_int, [C.c_void_p, C.POINTER(C.c_uint32), C.c_void_p]),
}


def load_library():
    """Load libsali.so (built by `python -m paper_2602_14236_amd.build`); raises if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(f"{_LIB_PATH} is missing: run `python -m paper_2602_14236_amd.build` first "
                              "(there is no CPU fallback)")
        lib = C.CDLL(_LIB_PATH)
        for name, (res, args) in EXPORTS.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


def library_path() -> str:
    return _LIB_PATH


def error_string(code: int) -> str:
    return load_library().sali_error_string(code).decode()


def _check(code: int, what: str):
    if code != 0:
        raise SaliError(code, what)


def _stream() -> int:
    """Handle of the current device's current stream, without a Stream object made for it (of the 13 us that a
    small attention call took in Python and ctypes, that and pointer objects were five)."""
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _ptr_array(tensors):
    """Host array of device pointers (the batched entry points read it before they return)."""
    return (C.c_void_p * len(tensors))(*[t.data_ptr() for t in tensors])


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()          # ctypes makes the pointer from the declared type


def make_config(src_h, src_w, *, flow_levels=3, flow_iters=3, tau_t=0.5, theta_r=0.90, canny_lo=50, canny_hi=100,
                tier_mode=0, tau_high=0.30, tau_med=0.15, tau_low=0.03, k_fp16=0, k_int8=0, k_int4=0,
                n_layers=1, n_heads=32, cap_fp16=0, cap_int8=0, cap_int4=0, max_frames=1,
                budget_tokens=0, tiles_per_frame=1, adapt_rate_q8=0) -> sali_config:
    return sali_config(src_h, src_w, 24, flow_levels, flow_iters, tau_t, theta_r, canny_lo, canny_hi, tier_mode,
                       tau_high, tau_med, tau_low, k_fp16, k_int8, k_int4, n_layers, n_heads, 128, 32,
                       cap_fp16, cap_int8, cap_int4, max_frames, budget_tokens, tiles_per_frame, adapt_rate_q8)


def workspace_bytes(cfg: sali_config):
    a, b, c = C.c_size_t(), C.c_size_t(), C.c_size_t()
    _check(load_library().sali_workspace_bytes(C.byref(cfg), C.byref(a), C.byref(b), C.byref(c)),
           "sali_workspace_bytes")
    return a.value, b.value, c.value


def pool_offsets(cfg: sali_config) -> sali_pool_layout:
    out = sali_pool_layout()
    _check(load_library().sali_pool_offsets(C.byref(cfg), C.byref(out)), "sali_pool_offsets")
    return out


class SaliContext:
    """Owns the three torch device buffers a context works in and forwards the C calls."""

    def __init__(self, cfg: sali_config, device="cuda:0"):
        self.lib = load_library()
        self.cfg = cfg
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise ValueError("libsali runs on the GPU only")
        sb, pb, tb = workspace_bytes(cfg)
        with torch.cuda.device(self.device):
            self.scratch = torch.empty(sb, dtype=torch.uint8, device=self.device)
            self.pools = torch.empty(pb, dtype=torch.uint8, device=self.device)
            self.tables = torch.zeros(tb, dtype=torch.uint8, device=self.device)
            torch.cuda.synchronize(self.device)
            h = C.c_void_p()
            _check(self.lib.sali_create(C.byref(cfg), _ptr(self.scratch), _ptr(self.pools), _ptr(self.tables),
                                        C.byref(h)), "sali_create")
        self.handle = h
        self.layout = pool_offsets(cfg)
        self.n_planes = cfg.n_layers * 2 * cfg.n_heads

    def close(self):
        if getattr(self, "handle", None):
            torch.cuda.synchronize(self.device)
            self.lib.sali_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- the C calls -------------------------------------------------------------------------
    def reset(self):
        _check(self.lib.sali_reset(self.handle, _stream()), "sali_reset")

    def set_gate_thresholds(self, tau_t: float, theta_r: float):
        _check(self.lib.sali_set_gate_thresholds(self.handle, tau_t, theta_r), "sali_set_gate_thresholds")

    def set_tier_params(self, tier_mode, tau_high=0.30, tau_med=0.15, tau_low=0.03, k_fp16=0, k_int8=0, k_int4=0):
        _check(self.lib.sali_set_tier_params(self.handle, tier_mode, tau_high, tau_med, tau_low, k_fp16, k_int8,
                                             k_int4), "sali_set_tier_params")

    def flow_score(self, prev_rgb, cur_rgb, flow_uv, patch_motion, gate_out):
        _check(self.lib.sali_flow_score(self.handle, _ptr(prev_rgb), _ptr(cur_rgb), _ptr(flow_uv),
                                        _ptr(patch_motion), _ptr(gate_out), _stream()), "sali_flow_score")

    def saliency_pool(self, rgb, salmap, scores):
        _check(self.lib.sali_saliency_pool(self.handle, _ptr(rgb), _ptr(salmap), _ptr(scores), _stream()),
               "sali_saliency_pool")

    def kv_compress(self, kv, scores, frame_id: int):
        _check(self.lib.sali_kv_compress(self.handle, _ptr(kv), _ptr(scores), frame_id, _stream()),
               "sali_kv_compress")

    def kv_decompress(self, frame_id: int, out, valid=None):
        _check(self.lib.sali_kv_decompress(self.handle, frame_id, _ptr(out), _ptr(valid), _stream()),
               "sali_kv_decompress")

    def step(self, rgb, kv, frame_id: int):
        _check(self.lib.sali_step(self.handle, _ptr(rgb), _ptr(kv), frame_id, _stream()), "sali_step")

    def analyze(self, rgb, frame_id: int, stream: Optional[torch.cuda.Stream] = None):
        s = _stream() if stream is None else stream.cuda_stream
        _check(self.lib.sali_analyze(self.handle, _ptr(rgb), frame_id, s), "sali_analyze")

    def analyze_batch(self, rgb_frames, first_frame_id: int, stream: Optional[torch.cuda.Stream] = None):
        s = _stream() if stream is None else stream.cuda_stream
        _check(self.lib.sali_analyze_batch(self.handle, _ptr_array(rgb_frames), first_frame_id, len(rgb_frames), s),
               "sali_analyze_batch")

    def attend_decode(self, layer: int, q, frame_lo: int, frame_hi: int, softmax_scale: float, out, lse=None,
                      stream: Optional[torch.cuda.Stream] = None):
        s = _stream() if stream is None else stream.cuda_stream
        _check(self.lib.sali_attend_decode(self.handle, layer, _ptr(q), frame_lo, frame_hi, softmax_scale, _ptr(out),
                                           _ptr(lse), s), "sali_attend_decode")

    def attend_decode_static(self, layer: int, q, frame_lo: int, frame_hi: int, softmax_scale: float, out, lse=None,
                             stream: Optional[torch.cuda.Stream] = None):
        s = _stream() if stream is None else stream.cuda_stream
        _check(self.lib.sali_attend_decode_static(self.handle, layer, _ptr(q), frame_lo, frame_hi, softmax_scale,
                                                  _ptr(out), _ptr(lse), s), "sali_attend_decode_static")

    def attend_decode_gqa(self, layer: int, q, q_per_kv: int, frame_lo: int, frame_hi: int, softmax_scale: float, out,
                          lse=None, stream: Optional[torch.cuda.Stream] = None):
        s = _stream() if stream is None else stream.cuda_stream
        _check(self.lib.sali_attend_decode_gqa(self.handle, layer, _ptr(q), q_per_kv, frame_lo, frame_hi, softmax_scale,
                                               _ptr(out), _ptr(lse), s), "sali_attend_decode_gqa")

    def store_batch(self, kv_frames, first_frame_id: int, stream: Optional[torch.cuda.Stream] = None):
        s = _stream() if stream is None else stream.cuda_stream
        _check(self.lib.sali_store_batch(self.handle, _ptr_array(kv_frames), first_frame_id, len(kv_frames), s),
               "sali_store_batch")

    def kv_decompress_batch(self, first_frame_id: int, out_frames, valid=None,
                            stream: Optional[torch.cuda.Stream] = None):
        s = _stream() if stream is None else stream.cuda_stream
        _check(self.lib.sali_kv_decompress_batch(self.handle, first_frame_id, len(out_frames), _ptr_array(out_frames),
                                                 _ptr(valid), s), "sali_kv_decompress_batch")

    def step_batch(self, rgb_frames, kv_frames, first_frame_id: int, stream: Optional[torch.cuda.Stream] = None):
        s = _stream() if stream is None else stream.cuda_stream
        assert len(rgb_frames) == len(kv_frames)
        _check(self.lib.sali_step_batch(self.handle, _ptr_array(rgb_frames), _ptr_array(kv_frames), first_frame_id,
                                        len(rgb_frames), s), "sali_step_batch")

    def store(self, kv, frame_id: int, stream: Optional[torch.cuda.Stream] = None):
        s = _stream() if stream is None else stream.cuda_stream
        _check(self.lib.sali_store(self.handle, _ptr(kv), frame_id, s), "sali_store")

    def step_pipelined(self, rgb_next, next_frame_id: int, kv, frame_id: int, image_stream: torch.cuda.Stream,
                       kv_stream: torch.cuda.Stream):
        _check(self.lib.sali_step_pipelined(self.handle, _ptr(rgb_next), next_frame_id, _ptr(kv), frame_id,
                                            image_stream.cuda_stream, kv_stream.cuda_stream), "sali_step_pipelined")

    def read_frame_table(self, first=0, count=None):
        count = self.cfg.max_frames - first if count is None else count
        rows = (sali_frame_row * count)()
        _check(self.lib.sali_read_frame_table(self.handle, rows, first, count, _stream()), "sali_read_frame_table")
        return list(rows)

    def read_frame_tiers(self, frame_id: int):
        tier = np.empty(TOKENS, dtype=np.uint8)
        slot = np.empty(TOKENS, dtype=np.uint16)
        _check(self.lib.sali_read_frame_tiers(self.handle, frame_id, tier.ctypes.data_as(C.c_void_p),
                                              slot.ctypes.data_as(C.c_void_p), _stream()), "sali_read_frame_tiers")
        return tier, slot

    def read_last_step(self):
        dp = np.empty(TOKENS, dtype=np.float32)
        sc = np.empty(TOKENS, dtype=np.float32)
        g = sali_gate()
        _check(self.lib.sali_read_last_step(self.handle, dp.ctypes.data_as(C.c_void_p), C.byref(g),
                                            sc.ctypes.data_as(C.c_void_p), _stream()), "sali_read_last_step")
        return dp, g, sc

    def read_analysis(self, frame_id: int):
        """(Delta P [576], gate, scores [576]) of one of the most recently analysed frames."""
        dp = np.empty(TOKENS, dtype=np.float32)
        sc = np.empty(TOKENS, dtype=np.float32)
        g = sali_gate()
        _check(self.lib.sali_read_analysis(self.handle, frame_id, dp.ctypes.data_as(C.c_void_p), C.byref(g),
                                           sc.ctypes.data_as(C.c_void_p), _stream()), "sali_read_analysis")
        return dp, g, sc

    def set_profile_events(self, which: int, start: Optional[torch.cuda.Event], stop: Optional[torch.cuda.Event]):
        """Arm a pair of torch events (created with enable_timing=True and already recorded once, so that
        their HIP handles exist) around the next pack (0) / unpack (1) kernel."""
        a = None if start is None else C.c_void_p(start.cuda_event)
        b = None if stop is None else C.c_void_p(stop.cuda_event)
        _check(self.lib.sali_set_profile_events(self.handle, which, a, b), "sali_set_profile_events")

    def get_status(self) -> int:
        f = C.c_uint32()
        _check(self.lib.sali_get_status(self.handle, C.byref(f), _stream()), "sali_get_status")
        return f.value

    # ---- views of the pool buffer (for inspection; the layout is part of the ABI) ----------------
    def pool_views_flat(self):
        """The six pool arrays as they lie in memory: [cap * n_planes, row], frame-major (a stored frame
        with base b and n rows owns rows [b * P, (b + n) * P), plane p of it rows [b * P + p * n, ...))."""
        c, L, P = self.cfg, self.layout, self.n_planes
        d, g = c.head_dim, c.head_dim // c.group
        # one typed view of the buffer per type and one strided view of it per array (slicing and reshaping each
        # array by itself took 22 us, half of the smallest compress and read-back)
        as_u8, as_i8, as_f16, as_f32 = (self.pools, self.pools.view(torch.int8), self.pools.view(torch.float16),
                                        self.pools.view(torch.float32))

        def view(base, size, off, rows, row):
            return base.as_strided((rows, row), (row, 1), base.storage_offset() + off // size)

        n16, n8, n4 = P * c.cap_fp16, P * c.cap_int8, P * c.cap_int4
        return {
            "fp16": view(as_f16, 2, L.off_fp16, n16, d),
            "codes8": view(as_i8, 1, L.off_codes8, n8, d),
            "scale8": view(as_f32, 4, L.off_scale8, n8, g),
            "codes4": view(as_u8, 1, L.off_codes4, n4, d // 2),
            "scale4": view(as_f32, 4, L.off_scale4, n4, g),
            "zero4": view(as_f16, 2, L.off_zero4, n4, g),
        }

    def pool_views(self, planes=None):
        """Copies of the pools regrouped per plane, [n_planes (or len(planes)), rows used, row], the
        rows of a plane in the order of the frame table (what a plain [plane][cap][row] cache would
        hold): for inspection and tests.  Synchronises the device."""
        torch.cuda.synchronize(self.device)
        P = self.n_planes
        flat = self.pool_views_flat()
        rows = [r for r in self.read_frame_table(0, self.cfg.max_frames) if r.stored]
        which = {"fp16": ("base16", "n16"), "codes8": ("base8", "n8"), "scale8": ("base8", "n8"),
                 "codes4": ("base4", "n4"), "scale4": ("base4", "n4"), "zero4": ("base4", "n4")}
        sel = slice(None) if planes is None else torch.as_tensor(list(planes), device=self.device)
        n_sel = P if planes is None else len(planes)
        out = {}
        for k, a in flat.items():
            fb, fn = which[k]
            used = max([getattr(r, fb) + getattr(r, fn) for r in rows], default=0)
            t = torch.zeros((n_sel, used, a.shape[1]), dtype=a.dtype, device=a.device)
            for r in rows:
                b, n = getattr(r, fb), getattr(r, fn)
                if n > 0:
                    t[:, b:b + n] = a[b * P:(b + n) * P].view(P, n, a.shape[1])[sel]
            out[k] = t
        return out


# ---- paged cache of text tokens ------------------------------------------------------------------
_PAGE_DTYPES = {torch.float16: 0, torch.bfloat16: 1}
_PAGE_STORES = {"16": STORE_16, "int8": STORE_INT8, "int4": STORE_INT4}


def make_pages_config(*, n_layers=1, n_kv_heads, n_heads, head_dim=128, page_tokens=64, n_pages, dtype=torch.float16, store="16") -> sali_pages_config:
    """dtype: torch.float16 or torch.bfloat16; store: "16", "int8" or "int4" (what the pages hold)."""
    if dtype not in _PAGE_DTYPES:
        raise ValueError(f"pages hold float16 or bfloat16 tokens, not {dtype}")
    if store not in _PAGE_STORES:
        raise ValueError(f"store is one of {sorted(_PAGE_STORES)}, not {store!r}")
    return sali_pages_config(n_layers, n_kv_heads, n_heads, head_dim, page_tokens, n_pages, _PAGE_DTYPES[dtype], _PAGE_STORES[store])


def pages_bytes(cfg: sali_pages_config):
    """(bytes of the pool, bytes of the scratch)"""
    a, b = C.c_size_t(), C.c_size_t()
    _check(load_library().sali_pages_bytes(C.byref(cfg), C.byref(a), C.byref(b)), "sali_pages_bytes")
    return a.value, b.value


class PageBatch:
    """The sequences of a step, for all layers: int32 tensors start [n + 1], length [n] and table [n, width] on one GPU, as sali_page_batch has
    them.  `tokens` is the number of rows of the per-token arrays; max_q (if not given, tokens) and max_kv bound the new tokens and the tokens of a
    sequence.  Attention chooses its kernels by them: a batch of single tokens without max_q=1 is taken for one that may hold a long sequence,
    which is three more launches a call (48 of them 7 to 9 us).  The tensors are read when a call's kernels run: a captured call takes what they hold at its replay."""

    def __init__(self, start: torch.Tensor, length: torch.Tensor, table: torch.Tensor, tokens: int, *, max_q: Optional[int] = None, max_kv: int):
        for name, t, dims in (("start", start, 1), ("length", length, 1), ("table", table, 2)):
            if t.dtype != torch.int32 or t.dim() != dims or not t.is_contiguous():
                raise ValueError(f"{name}: contiguous int32 tensor of {dims} dimension(s) expected, got {t.dtype} {tuple(t.shape)}")
            if t.device != length.device:
                raise ValueError("start, length and table lie on different devices")
        n = length.shape[0]
        if start.shape[0] != n + 1 or table.shape[0] != n:
            raise ValueError(f"{n} lengths need {n + 1} starts and {n} rows of the table, got {start.shape[0]} and {table.shape[0]}")
        self.tensors = (start, length, table)
        self.tokens = tokens
        self.device, self.index = length.device, length.get_device()
        self.c = sali_page_batch(start.data_ptr(), length.data_ptr(), table.data_ptr(), n, table.shape[1], tokens, tokens if max_q is None else max_q,
                                 max_kv, 0)


class SaliPages:
    """Owns the pool (or works in the caller's) and the scratch of a paged cache and forwards the C calls.  Per-token tensors are [tokens, heads,
    head_dim] with values side by side; tokens and heads may be strided (slices of one projection's output).  Where another GPU is the current one,
    a call makes the pages' current for itself: the default stream's handle is the same on every GPU, and means the current one's."""

    def __init__(self, cfg: sali_pages_config, device="cuda:0", pool: Optional[torch.Tensor] = None):
        self.lib = load_library()
        self.cfg = cfg
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise ValueError("libsali runs on the GPU only")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        pool_bytes, scratch_bytes = pages_bytes(cfg)
        if pool is not None and (not pool.is_contiguous() or pool.numel() * pool.element_size() < pool_bytes or pool.device != self.device):
            raise ValueError(f"pool: {pool_bytes} contiguous bytes on {self.device} expected, got {pool.numel() * pool.element_size()} on {pool.device}")
        self.dtype = torch.bfloat16 if cfg.dtype else torch.float16
        self.n_heads, self.n_kv_heads, self.head_dim = cfg.n_heads, cfg.n_kv_heads, cfg.head_dim
        self.handle = None
        with torch.cuda.device(self.device):
            self.pool = torch.empty(pool_bytes, dtype=torch.uint8, device=self.device) if pool is None else pool
            self.scratch = torch.empty(scratch_bytes, dtype=torch.uint8, device=self.device)
            self.index = self.device.index
            h = C.c_void_p()
            _check(self.lib.sali_pages_create(C.byref(cfg), _ptr(self.pool), _ptr(self.scratch), C.byref(h)), "sali_pages_create")
        self.handle = h

    def close(self):
        if getattr(self, "handle", None):
            torch.cuda.synchronize(self.device)
            self.lib.sali_pages_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _rows(self, t: torch.Tensor, batch: PageBatch, heads: int, name: str) -> sali_rows:
        token, head, one = t.stride() if t.dim() == 3 else (0, 0, 0)
        if t.dtype is not self.dtype or t.shape != (batch.tokens, heads, self.head_dim) or one != 1 or t.get_device() != self.index:
            raise ValueError(f"{name}: {self.dtype} [{batch.tokens}, {heads}, {self.head_dim}] on {self.device} with its last dimension side by "
                             f"side expected, got {t.dtype} {tuple(t.shape)} on {t.device} with strides {t.stride()}")
        return sali_rows(t.data_ptr(), token, head)

    def _call(self, batch: PageBatch, stream: Optional[torch.cuda.Stream]) -> int:
        """The stream of a call on `batch`: the pages' GPU's current one, if none is given."""
        if batch.index != self.index:
            raise ValueError(f"the batch lies on {batch.device}, the pages on {self.device}")
        if stream is None:
            return torch._C._cuda_getCurrentRawStream(self.index)
        if stream.device_index != self.index:
            raise ValueError(f"the stream is of {stream.device}, the pages lie on {self.device}")
        return stream.cuda_stream

    def _dense(self, t: Optional[torch.Tensor], shape, name: str):
        if t is None:
            return None
        if t.dtype is not torch.float32 or t.shape != shape or not t.is_contiguous() or t.get_device() != self.index:
            raise ValueError(f"{name}: contiguous float32 {list(shape)} on {self.device} expected, got {t.dtype} {tuple(t.shape)} on {t.device}")
        return t.data_ptr()

    def append(self, layer: int, batch: PageBatch, k: torch.Tensor, v: torch.Tensor, stream: Optional[torch.cuda.Stream] = None):
        """Store the K/V rows of the batch's new tokens, [tokens, n_kv_heads, head_dim]."""
        if torch._C._cuda_getDevice() != self.index:
            with torch.cuda.device(self.index):
                return self.append(layer, batch, k, v, stream)
        n = self.n_kv_heads
        _check(self.lib.sali_pages_append(self.handle, layer, batch.c, self._rows(k, batch, n, "k"), self._rows(v, batch, n, "v"),
                                          self._call(batch, stream)), "sali_pages_append")

    def read(self, layer: int, batch: PageBatch, k_out: torch.Tensor, v_out: torch.Tensor, stream: Optional[torch.cuda.Stream] = None):
        """The rows of the batch's new tokens as the pages hold them."""
        if torch._C._cuda_getDevice() != self.index:
            with torch.cuda.device(self.index):
                return self.read(layer, batch, k_out, v_out, stream)
        n = self.n_kv_heads
        _check(self.lib.sali_pages_read(self.handle, layer, batch.c, self._rows(k_out, batch, n, "k_out"), self._rows(v_out, batch, n, "v_out"),
                                        self._call(batch, stream)), "sali_pages_read")

    def attend(self, layer: int, batch: PageBatch, q: torch.Tensor, softmax_scale: float, out: torch.Tensor, lse: Optional[torch.Tensor] = None, *,
               window: int = 0, sinks: int = 0, prior: Optional[torch.Tensor] = None, prior_lse: Optional[torch.Tensor] = None,
               stream: Optional[torch.cuda.Stream] = None):
        """Causal attention of the batch's new tokens over the pages: q, out [tokens, n_heads, head_dim], lse [tokens, n_heads] in fp32.  prior and
        prior_lse (fp32): attention of the same queries over other keys, joined with this one."""
        if torch._C._cuda_getDevice() != self.index:
            with torch.cuda.device(self.index):
                return self.attend(layer, batch, q, softmax_scale, out, lse, window=window, sinks=sinks, prior=prior, prior_lse=prior_lse, stream=stream)
        n, d = self.n_heads, self.head_dim
        _check(self.lib.sali_pages_attend(self.handle, layer, batch.c, self._rows(q, batch, n, "q"), softmax_scale, window, sinks,
                                          self._dense(prior, (batch.tokens, n, d), "prior"), self._dense(prior_lse, (batch.tokens, n), "prior_lse"),
                                          self._rows(out, batch, n, "out"), self._dense(lse, (batch.tokens, n), "lse"),
                                          self._call(batch, stream)), "sali_pages_attend")

    def get_status(self) -> int:
        if torch._C._cuda_getDevice() != self.index:
            with torch.cuda.device(self.index):
                return self.get_status()
        f = C.c_uint32()
        _check(self.lib.sali_pages_get_status(self.handle, C.byref(f), torch._C._cuda_getCurrentRawStream(self.index)), "sali_pages_get_status")
        return f.value
