"""ctypes binding of libkperf.so -- same names as the C ABI in include/kperf.h.

Argument marshalling only.  Tensors must live on the GPU (device pointers are
passed through unchanged); `stream` defaults to torch's current stream.
"""
from __future__ import annotations

import ctypes
import os
import struct

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libkperf.so")

KP_OK = 0
KP_ERR_INVALID_ARG = -1
KP_ERR_UNSUPPORTED_SHAPE = -2
KP_ERR_TRACE_TOO_SMALL = -3
KP_ERR_BAD_TRACE = -4
KP_ERR_HIP = -5

KP_FLAG_FLUSH = 1
KP_MASK_FLUSH = 1 << 31
KP_MASK_WAVE_GROUP = 1 << 30  # one record stream per group of four waves
KP_MASK_PHASES = 1 << 29      # 256x256x64 GEMM: the stages of a K step one after the other, 5 regions
KP_MASK_REALTIME = 1 << 28    # records carry the constant-rate 100 MHz clock
KP_MASK_COLLAB = 1 << 27      # all lanes store a record; hardware ids of the waves in the workgroup header
KP_MASK_UNFENCED = 1 << 26    # with KP_MASK_PHASES and no region: the staged K step without scheduling fences
KP_FLAG_REALTIME = 2
KP_FLAG_HW_IDS = 4
KP_BF16, KP_FP16, KP_FP32 = 0, 1, 2
KP_CACHE_SAME, KP_CACHE_E4M3 = 0, 1
KP_MOVE_RUN = 128  # moves of a group of kp_cache_move that may be any


class KperfError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"libkperf status {status}: {message}")
        self.status = status


class kp_trace_hdr(ctypes.Structure):
    _fields_ = [
        ("magic", ctypes.c_uint32), ("version", ctypes.c_uint32), ("n_wg", ctypes.c_uint32),
        ("waves_per_wg", ctypes.c_uint32), ("n_regions", ctypes.c_uint32), ("cap_wave", ctypes.c_uint32),
        ("rec_cost", ctypes.c_uint32), ("flags", ctypes.c_uint32), ("pad", ctypes.c_uint32 * 8),
    ]


class kp_heads(ctypes.Structure):
    _fields_ = [("at", ctypes.c_void_p), ("seq", ctypes.c_int64), ("head", ctypes.c_int64), ("token", ctypes.c_int64)]


class kp_cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_exp", ctypes.c_void_p), ("v_exp", ctypes.c_void_p),
                ("n_pages", ctypes.c_int), ("Hkv", ctypes.c_int), ("page", ctypes.c_int), ("D", ctypes.c_int),
                ("type", ctypes.c_int), ("cache_type", ctypes.c_int)]


class kp_turns(ctypes.Structure):
    _fields_ = [("at", ctypes.c_void_p), ("axis_step", ctypes.c_int64), ("seq_step", ctypes.c_int64), ("freq", ctypes.c_void_p),
                ("axis", ctypes.c_void_p), ("pairs", ctypes.c_int), ("axes", ctypes.c_int), ("adjacent", ctypes.c_int)]


_lib = None


def lib() -> ctypes.CDLL:
    """Load libkperf.so; raises if it has not been built (no fallback path exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(
                f"{LIB_PATH} is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'`"
            )
        # The caller's device buffers come from torch, which ships its own copy of the HIP runtime.
        # That copy has to be the first one in the process: if this library pulled in the system's
        # runtime before torch loaded its own, the two would not share a device context and every
        # launch from here would fail with "no ROCm-capable device".
        try:
            import torch  # noqa: F401
        except ImportError:
            pass
        L = ctypes.CDLL(LIB_PATH)
        vp, sz, ci, u32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_uint32
        L.kp_last_error.restype = ctypes.c_char_p
        L.kp_last_error.argtypes = []
        L.kp_trace_bytes.restype = sz
        L.kp_trace_bytes.argtypes = [ci, ci, ci]
        L.kp_stats_bytes.restype = sz
        L.kp_stats_bytes.argtypes = [ci, ci, ci]
        L.kp_trace_reduce.restype = ci
        L.kp_trace_reduce.argtypes = [vp, sz, vp, vp]
        L.kp_trace_reduce_hdr.restype = ci
        L.kp_trace_reduce_hdr.argtypes = [vp, sz, ctypes.POINTER(kp_trace_hdr), vp, vp]
        L.kp_trace_reduce_hdr_events.restype = ci
        L.kp_trace_reduce_hdr_events.argtypes = [vp, sz, ctypes.POINTER(kp_trace_hdr), vp, vp, vp, vp]
        L.kp_trace_reduce_steps.restype = ci
        L.kp_trace_reduce_steps.argtypes = [vp, sz, ctypes.POINTER(kp_trace_hdr), vp, ci, vp]
        L.kp_pairs_bytes.restype = sz
        L.kp_pairs_bytes.argtypes = [ci, ci, ci]
        L.kp_trace_pairs.restype = ci
        L.kp_trace_pairs.argtypes = [vp, sz, vp, vp]
        L.kp_trace_pairs_hdr.restype = ci
        L.kp_trace_pairs_hdr.argtypes = [vp, sz, ctypes.POINTER(kp_trace_hdr), vp, vp]
        L.kp_waits_bytes.restype = sz
        L.kp_waits_bytes.argtypes = [ci, ci, ci]
        L.kp_trace_waits.restype = ci
        L.kp_trace_waits.argtypes = [vp, sz, vp, vp]
        L.kp_trace_waits_hdr.restype = ci
        L.kp_trace_waits_hdr.argtypes = [vp, sz, ctypes.POINTER(kp_trace_hdr), vp, vp]
        L.kp_stages_bytes.restype = sz
        L.kp_stages_bytes.argtypes = [ci, ci, ci]
        L.kp_pairs_stages.restype = ci
        L.kp_pairs_stages.argtypes = [vp, ci, ci, ci, ci, ci, vp, vp]
        L.kp_critical_bytes.restype = sz
        L.kp_critical_bytes.argtypes = [ci, ci]
        L.kp_stages_critical.restype = ci
        L.kp_stages_critical.argtypes = [vp, ci, ci, ci, vp, vp]
        L.kp_set_rec_cost.restype = None
        L.kp_set_rec_cost.argtypes = [u32]
        L.kp_get_rec_cost.restype = u32
        L.kp_get_rec_cost.argtypes = []
        _optional(L)
        _lib = L
    return _lib


def _optional(L):
    vp, sz, ci, u32, fl = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_uint32, ctypes.c_float
    ip = ctypes.POINTER(ctypes.c_int)
    hp = cp = tp = vp  # kp_heads, kp_cache and kp_turns: their bytes, or byref of a structure
    sigs = {
        "kp_attn_window": [hp, hp, hp, hp, vp, ci, ci, ci, ci, ci, ci, ci, ci, ci, fl, vp, sz, u32, vp, sz, vp],
        "kp_attn_window_launch_shape": [ci] * 8 + [ip] * 3,
        "kp_attn_paged_launch_shape": [ci] * 9 + [ip] * 3,
        "kp_attn_window_grad": [hp, hp, hp, hp, vp, hp, hp, hp, hp, ci, ci, ci, ci, ci, ci, ci, ci, ci, fl, vp, sz, vp],
        "kp_cache_write": [hp, hp, vp, ci, cp, vp],
        "kp_cache_read": [cp, vp, ci, vp, ci, ci, hp, hp, vp],
        "kp_attn_paged": [hp, cp, vp, ci, vp, vp, hp, vp, ci, ci, ci, ci, ci, fl, vp, sz, u32, vp, sz, vp],
        "kp_attn_tree": [hp, cp, vp, ci, vp, vp, vp, ci, vp, hp, vp, ci, ci, ci, ci, ci, fl, vp, sz, u32, vp, sz, vp],
        "kp_attn_tree_launch_shape": [ci] * 10 + [ip] * 3,
        "kp_cache_move": [vp, vp, ci, vp, ci, cp, vp],
        "kp_norm_rotate": [hp, hp, vp, vp, ci, fl, tp, hp, hp, ci, ci, ci, ci, ci, ci, vp],
        "kp_norm_rotate_grad": [hp, hp, vp, vp, ci, fl, tp, hp, hp, hp, hp, vp, vp, ci, ci, ci, ci, ci, ci, vp, sz, vp],
        "kp_norm_rotate_write": [hp, hp, hp, vp, vp, ci, fl, tp, hp, vp, ci, ci, cp, vp],
        "kp_gemm_launch_shape": [ci, ci, ci, ip, ip, ip],
        "kp_gemm_instrumented": [vp, vp, vp, ci, ci, ci, u32, vp, sz, vp],
        "kp_attn_launch_shape": [ci, ci, ci, ci, ip, ip, ip],
        "kp_attn_instrumented": [vp, vp, vp, vp, ci, ci, ci, ci, ci, fl, u32, vp, sz, vp],
        "kp_calibrate": [ctypes.POINTER(u32), ci, ci, ci, ci, vp, sz, vp],
    }
    for name, args in sigs.items():
        if hasattr(L, name):
            f = getattr(L, name)
            f.restype = ci
            f.argtypes = args
    for name, n in (("kp_attn_window_bytes", 8), ("kp_attn_window_grad_bytes", 8), ("kp_attn_paged_bytes", 9), ("kp_attn_tree_bytes", 10),
                    ("kp_norm_rotate_grad_bytes", 5)):
        if hasattr(L, name):
            getattr(L, name).restype = sz
            getattr(L, name).argtypes = [ci] * n


def _check(status: int):
    if status != KP_OK:
        raise KperfError(status, kp_last_error())


def _ptr(t) -> int:
    if t is None:
        return 0
    if not t.is_cuda:
        raise ValueError("libkperf takes device memory: tensor must be on the GPU")
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return t.data_ptr()


_current_stream = None  # () -> hipStream_t of torch's current stream
_raw_stream = None  # the same, of a GPU by its number (where torch offers it)


def _stream_lookup():
    import torch

    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is None:  # (not part of torch's public interface)
        return lambda: torch.cuda.current_stream().cuda_stream
    torch.cuda.init()
    global _raw_stream
    _raw_stream = raw
    device = torch.cuda.current_device
    return lambda: raw(device())


_current_device = None  # torch.cuda.current_device


def _stream_at(stream, t) -> int:
    """The stream of a call on tensor t, which has to be on the current GPU."""
    global _current_device
    if _current_device is None:
        import torch

        torch.cuda.init()
        _current_device = torch.cuda.current_device
    device = _current_device()
    if t.get_device() != device:
        raise ValueError(f"tensor on {t.device}, but the current GPU is {device}")
    if stream is None and _raw_stream is not None:
        return _raw_stream(device)
    return _stream(stream)


def _stream(stream) -> int:
    global _current_stream
    if stream is None:
        # The handle itself: building a torch.cuda.Stream object around it took 2.8 of the 6.9 us that a call
        # spent on the host, which is what the smallest calls are bound by (0.2 us this way).
        if _current_stream is None:
            _current_stream = _stream_lookup()
        return _current_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def kp_last_error() -> str:
    return lib().kp_last_error().decode()


def kp_trace_bytes(n_wg: int, waves_per_wg: int, cap_per_wg: int) -> int:
    return lib().kp_trace_bytes(n_wg, waves_per_wg, cap_per_wg)


def kp_stats_bytes(n_wg: int, waves_per_wg: int, n_regions: int) -> int:
    return lib().kp_stats_bytes(n_wg, waves_per_wg, n_regions)


def kp_set_rec_cost(ticks: int) -> None:
    lib().kp_set_rec_cost(int(ticks))


def kp_get_rec_cost() -> int:
    return int(lib().kp_get_rec_cost())


def kp_trace_reduce(raw, n: int, out_stats, stream=None) -> None:
    _check(lib().kp_trace_reduce(_ptr(raw), n, _ptr(out_stats), _stream(stream)))


def make_hdr(n_wg: int, waves_per_wg: int, n_regions: int, cap_wave: int, rec_cost: int = 0,
             flags: int = 0) -> kp_trace_hdr:
    h = kp_trace_hdr()
    h.magic, h.version = 0x4652504B, 1
    h.n_wg, h.waves_per_wg, h.n_regions, h.cap_wave = n_wg, waves_per_wg, n_regions, cap_wave
    h.rec_cost, h.flags = rec_cost, flags
    return h


def kp_trace_reduce_hdr(raw, n: int, hdr_host: kp_trace_hdr, out_stats, stream=None) -> None:
    _check(lib().kp_trace_reduce_hdr(_ptr(raw), n, ctypes.byref(hdr_host), _ptr(out_stats), _stream(stream)))


def kp_trace_reduce_hdr_events(raw, n: int, hdr_host: kp_trace_hdr, out_stats, main_begin, main_end, stream=None) -> None:
    """main_begin, main_end: torch.cuda.Event objects with timing enabled that have been recorded before (an
    event's handle exists from its first record on), raw hipEvent_t handles as int, or None."""
    def handle(ev):
        if ev is None or isinstance(ev, int):
            return ev
        h = ev.cuda_event
        if not h:
            raise ValueError("record the event once before passing it: it has no handle yet")
        return h
    _check(lib().kp_trace_reduce_hdr_events(_ptr(raw), n, ctypes.byref(hdr_host), _ptr(out_stats), _stream(stream),
                                            handle(main_begin), handle(main_end)))


def kp_trace_reduce_steps(raw, n: int, hdr_host: kp_trace_hdr, out_stats, last_step: int, stream=None) -> None:
    _check(lib().kp_trace_reduce_steps(_ptr(raw), n, ctypes.byref(hdr_host), _ptr(out_stats), last_step,
                                       _stream(stream)))


def kp_pairs_bytes(n_wg: int, waves_per_wg: int, cap_per_wg: int) -> int:
    return lib().kp_pairs_bytes(n_wg, waves_per_wg, cap_per_wg)


def kp_trace_pairs(raw, n: int, out_pairs, stream=None) -> None:
    _check(lib().kp_trace_pairs(_ptr(raw), n, _ptr(out_pairs), _stream(stream)))


def kp_trace_pairs_hdr(raw, n: int, hdr_host: kp_trace_hdr, out_pairs, stream=None) -> None:
    _check(lib().kp_trace_pairs_hdr(_ptr(raw), n, ctypes.byref(hdr_host), _ptr(out_pairs), _stream(stream)))


PAIR_ROW_DTYPE = [("start", "<u4"), ("dur", "<u4"), ("iter", "<u4"), ("region", "<u4")]


def parse_pairs(buf, n_wg: int, waves_per_wg: int, cap_per_wg: int):
    """Split a pairs block (host bytes: numpy array or CPU tensor) into (count[n_wg, waves],
    rows[n_wg, waves, cap_wave // 2]); only the first count[wg, wave] rows of a wave are meaningful."""
    import numpy as np

    b = np.ascontiguousarray(buf.cpu().numpy() if hasattr(buf, "numpy") else buf).view(np.uint8)
    n_seg, half = n_wg * waves_per_wg, cap_per_wg // waves_per_wg // 2
    head = ((n_seg + 3) // 4) * 16
    count = b[: 4 * n_seg].view("<u4").reshape(n_wg, waves_per_wg)
    rows = b[head : head + 16 * n_seg * half].view(np.dtype(PAIR_ROW_DTYPE)).reshape(n_wg, waves_per_wg, half)
    return count, rows


def kp_waits_bytes(n_wg: int, waves_per_wg: int, n_regions: int) -> int:
    return lib().kp_waits_bytes(n_wg, waves_per_wg, n_regions)


def kp_trace_waits(raw, n: int, out_waits, stream=None) -> None:
    _check(lib().kp_trace_waits(_ptr(raw), n, _ptr(out_waits), _stream(stream)))


def kp_trace_waits_hdr(raw, n: int, hdr_host: kp_trace_hdr, out_waits, stream=None) -> None:
    _check(lib().kp_trace_waits_hdr(_ptr(raw), n, ctypes.byref(hdr_host), _ptr(out_waits), _stream(stream)))


WAITS_HEADER_FIELDS = ("n_waits", "n_uncovered", "n_async", None, None, None, None, None,
                       "n_wg", "waves_per_wg", "n_regions", "cap_wave", "rec_cost", None, None, None)


def parse_waits(buf) -> dict:
    """Split a waits block (bytes on the host: numpy uint8 array or CPU tensor) into fields."""
    if hasattr(buf, "numpy"):
        buf = buf.cpu().numpy()
    b = np.ascontiguousarray(buf).view(np.uint8)
    hdr = b[:128].view("<u8")
    out = {k: int(hdr[i]) for i, k in enumerate(WAITS_HEADER_FIELDS) if k}
    n_wg, W, R = out["n_wg"], out["waves_per_wg"], out["n_regions"]
    pos = 128
    out["hist"] = b[pos : pos + 8 * 64 * R].view("<u8").reshape(R, 64)
    pos += 8 * 64 * R
    for name in ("cnt", "sum", "min", "max", "uncovered", "async_cnt", "async_sum"):
        out[name] = b[pos : pos + 8 * R].view("<u8")
        pos += 8 * R
    out["per"] = b[pos : pos + 16 * n_wg * W * R].view(WAVE_REGION_DTYPE).reshape(n_wg, W, R)
    return out


def kp_stages_bytes(n_wg: int, n_regions: int, max_iter: int) -> int:
    return lib().kp_stages_bytes(n_wg, n_regions, max_iter)


def kp_pairs_stages(pairs, n_wg: int, waves_per_wg: int, cap_per_wg: int, n_regions: int, max_iter: int,
                    out_stages, stream=None) -> None:
    _check(lib().kp_pairs_stages(_ptr(pairs), n_wg, waves_per_wg, cap_per_wg, n_regions, max_iter,
                                 _ptr(out_stages), _stream(stream)))


STAGE_ROW_DTYPE = [("max_dur", "<u4"), ("min_start", "<u4"), ("max_end", "<u4"), ("n_waves", "<u4")]
PATH_ROW_DTYPE = [("n_stages", "<u4"), ("last_stage", "<u4"), ("first_start", "<u4"), ("last_end", "<u4"),
                  ("sum_latency", "<u8"), ("bubbles", "<u8")]


def kp_critical_bytes(n_wg: int, n_regions: int) -> int:
    return int(lib().kp_critical_bytes(n_wg, n_regions))


def kp_stages_critical(stages, n_wg: int, n_regions: int, max_iter: int, out_paths, stream=None) -> None:
    _check(lib().kp_stages_critical(_ptr(stages), n_wg, n_regions, max_iter, _ptr(out_paths), _stream(stream)))


def parse_critical(buf, n_wg: int, n_regions: int):
    """Split a critical-path block (host bytes) into (header dict, per-region array[R, 2], rows[n_wg])."""
    b = np.ascontiguousarray(buf.cpu().numpy() if hasattr(buf, "numpy") else buf).view(np.uint8)
    h = b[:64].view("<u8")
    hdr = {"n_wg": int(h[0]), "n_regions": int(h[1]), "max_iter": int(h[2]), "n_paths": int(h[3]),
           "n_path_stages": int(h[4]), "sum_latency": int(h[5]), "sum_bubbles": int(h[6])}
    per_region = b[64 : 64 + 16 * n_regions].view("<u8").reshape(n_regions, 2)
    rows = b[64 + 16 * n_regions : 64 + 16 * n_regions + 32 * n_wg].view(np.dtype(PATH_ROW_DTYPE))
    return hdr, per_region, rows


def parse_stages(buf, n_wg: int, n_regions: int, max_iter: int):
    """Split a stage block (host bytes) into (header dict, table[n_wg, n_regions, max_iter])."""
    b = np.ascontiguousarray(buf.cpu().numpy() if hasattr(buf, "numpy") else buf).view(np.uint8)
    h = b[:32].view("<u8")
    hdr = {"n_rows": int(h[0]), "n_clipped": int(h[1]), "n_bad_region": int(h[2])}
    tab = b[32 : 32 + 16 * n_wg * n_regions * max_iter].view(np.dtype(STAGE_ROW_DTYPE)).reshape(n_wg, n_regions, max_iter)
    return hdr, tab


def kp_gemm_launch_shape(M: int, N: int, K: int) -> tuple[int, int, int]:
    a, b, c = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
    _check(lib().kp_gemm_launch_shape(M, N, K, ctypes.byref(a), ctypes.byref(b), ctypes.byref(c)))
    return a.value, b.value, c.value


def kp_gemm_instrumented(A, B, C, M: int, N: int, K: int, region_mask: int, trace_buf, trace_cap: int,
                         stream=None) -> None:
    _check(lib().kp_gemm_instrumented(_ptr(A), _ptr(B), _ptr(C), M, N, K, region_mask & 0xFFFFFFFF,
                                      _ptr(trace_buf), trace_cap, _stream(stream)))


def kp_attn_launch_shape(B: int, H: int, S: int, D: int) -> tuple[int, int, int]:
    a, b, c = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
    _check(lib().kp_attn_launch_shape(B, H, S, D, ctypes.byref(a), ctypes.byref(b), ctypes.byref(c)))
    return a.value, b.value, c.value


def kp_attn_instrumented(Q, K, V, O, B: int, H: int, S: int, D: int, causal: bool, scale: float,
                         region_mask: int, trace_buf, trace_cap: int, stream=None) -> None:
    _check(lib().kp_attn_instrumented(_ptr(Q), _ptr(K), _ptr(V), _ptr(O), B, H, S, D, int(bool(causal)),
                                      float(scale), region_mask & 0xFFFFFFFF, _ptr(trace_buf), trace_cap,
                                      _stream(stream)))


def kp_calibrate(cycles, n_wg: int, waves: int, mode: int, trace_buf, trace_cap: int, stream=None) -> None:
    arr = (ctypes.c_uint32 * len(cycles))(*[int(c) for c in cycles])
    _check(lib().kp_calibrate(arr, len(cycles), n_wg, waves, mode, _ptr(trace_buf), trace_cap, _stream(stream)))


# ---- attention with windows, caches and gradients --------------------------------------------------
# Tensors of heads keep their strides: [B, H, S, D] in any order in memory with D innermost (a transposed view of
# [B, S, H, D], a slice of a fused projection), or [T, H, D] where there is no batch.


_names = {}  # torch's types by the names below, filled in by the first call


def _types() -> dict:
    global _names
    if not _names:
        import torch

        names = {n: getattr(torch, n) for n in ("float32", "uint8", "int32", "int64", "float8_e4m3fn", "bfloat16")}
        names.update({torch.bfloat16: KP_BF16, torch.float16: KP_FP16})
        _names = names  # (whole: another thread may be looking)
    return _names


def _type_code(dtype) -> int:
    code = (_names or _types()).get(dtype)
    if code is None:
        raise ValueError(f"tensors must be bfloat16 or float16, not {dtype}")
    return code


# The bytes of a kp_heads and of a kp_cache: the smallest calls are bound by what the host spends on them, and packing is
# faster than building ctypes structures (kp_cache_write 6.6 us a call, 7.0 with structures; 3.3 of it are the launch).
_pack_heads, _pack_cache = struct.Struct("Pqqq").pack, struct.Struct("PPPPiiiiii").pack


def _heads(name: str, t, shape, dtype) -> bytes:
    """kp_heads of a [B, H, S, D] or [T, H, D] tensor of a shape (None: its own is the one that counts)."""
    if not t.is_cuda:
        raise ValueError("libkperf takes device memory: tensor must be on the GPU")
    if t.dtype is not dtype or (shape is not None and t.shape != shape):
        raise ValueError(f"{name} must be {'' if shape is None else str(list(shape)) + ' '}of {dtype}, not {list(t.shape)} of {t.dtype}")
    st = t.stride()
    if st[-1] != 1:
        raise ValueError(f"the last dimension of {name} must be contiguous")
    if len(st) == 4:
        return _pack_heads(t.data_ptr(), st[0], st[1], st[2])
    return _pack_heads(t.data_ptr(), 0, st[1], st[0])


def _flat(name: str, t, dtype, shape=None):
    """Device pointer of a contiguous tensor of a type and (where given) a shape."""
    if t.dtype is not dtype or (shape is not None and t.shape != shape):
        raise ValueError(f"{name} must be {'' if shape is None else str(list(shape)) + ' '}of {dtype}, not {list(t.shape)} of {t.dtype}")
    return t.data_ptr() if t.is_cuda and t.is_contiguous() else _ptr(t)


def _workspace(workspace) -> tuple[int, int]:
    return (0, 0) if workspace is None else (_ptr(workspace), workspace.numel() * workspace.element_size())


def _window_sizes(q, k):
    B, Hq, Sq, D = q.shape
    return B, Hq, k.shape[1], Sq, k.shape[2], D


def kp_attn_window_bytes(q, k, window: int, sinks: int) -> int:
    """Bytes of workspace that kp_attn_window takes for q [B, Hq, Sq, D] and k [B, Hkv, Sk, D]."""
    return int(lib().kp_attn_window_bytes(*_window_sizes(q, k), window, sinks))


def _shape_of(call, *sizes) -> tuple[int, int, int]:
    a, b, c = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
    _check(call(*sizes, ctypes.byref(a), ctypes.byref(b), ctypes.byref(c)))
    return a.value, b.value, c.value


def kp_attn_window_launch_shape(q, k, window: int, sinks: int) -> tuple[int, int, int]:
    """Workgroups, waves per workgroup and regions of a recording of kp_attn_window."""
    return _shape_of(lib().kp_attn_window_launch_shape, *_window_sizes(q, k), window, sinks)


def kp_attn_window(q, k, v, o, lse, window: int, sinks: int, scale: float, workspace=None, region_mask: int = 0,
                   trace_buf=None, trace_cap: int = 0, stream=None) -> None:
    """o = softmax(scale q k^T over the visible keys) v; q, o [B, Hq, Sq, D], k, v [B, Hkv, Sk, D] (any strides with D
    innermost), lse [B, Hq, Sq] float32 or None.  A token at position p = Sk - Sq + i sees keys j <= p with p - j < window
    (window 0: all) or j < sinks."""
    dtype, kv = q.dtype, k.shape
    B, Hq, Hkv, Sq, Sk, D = _window_sizes(q, k)
    ws, n = _workspace(workspace)
    _check(lib().kp_attn_window(
        _heads("q", q, q.shape, dtype), _heads("k", k, (B, Hkv, Sk, D), dtype), _heads("v", v, kv, dtype),
        _heads("o", o, q.shape, dtype), 0 if lse is None else _flat("lse", lse, (_names or _types())["float32"], (B, Hq, Sq)),
        B, Hq, Hkv, Sq, Sk, D, _type_code(dtype), window, sinks, scale, ws, n, region_mask & 0xFFFFFFFF, _ptr(trace_buf),
        trace_cap, _stream(stream)))


def kp_attn_window_grad_bytes(q, k, window: int, sinks: int) -> int:
    return int(lib().kp_attn_window_grad_bytes(*_window_sizes(q, k), window, sinks))


def kp_attn_window_grad(q, k, v, o, lse, d_o, dq, dk, dv, window: int, sinks: int, scale: float, workspace,
                        stream=None) -> None:
    """Gradients dq, dk, dv of kp_attn_window from its o and lse and the gradient d_o of o."""
    dtype, qs, ks = q.dtype, q.shape, k.shape
    B, Hq, Hkv, Sq, Sk, D = _window_sizes(q, k)
    ws, n = _workspace(workspace)
    _check(lib().kp_attn_window_grad(
        _heads("q", q, qs, dtype), _heads("k", k, (B, Hkv, Sk, D), dtype), _heads("v", v, ks, dtype),
        _heads("o", o, qs, dtype), _flat("lse", lse, (_names or _types())["float32"], (B, Hq, Sq)), _heads("d_o", d_o, qs, dtype),
        _heads("dq", dq, qs, dtype), _heads("dk", dk, ks, dtype), _heads("dv", dv, ks, dtype),
        B, Hq, Hkv, Sq, Sk, D, _type_code(dtype), window, sinks, scale, ws, n, _stream(stream)))


def _cache_of(k_cache, v_cache, k_exp, v_exp, dtype) -> bytes:
    """kp_cache of two halves [n_pages, Hkv, page, D]: of `dtype`, or float8_e4m3fn with exponent bytes."""
    code, kind, shape = _type_code(dtype), k_cache.dtype, k_cache.shape
    n_pages, Hkv, page, D = shape
    e4m3 = kind is _names["float8_e4m3fn"]
    if (not e4m3 and kind is not dtype) or v_cache.dtype is not kind or v_cache.shape != shape:
        raise ValueError(f"the cache's halves must be alike and of {dtype} or float8_e4m3fn, not {list(k_cache.shape)} of {kind} "
                         f"and {list(v_cache.shape)} of {v_cache.dtype}")
    if not (k_cache.is_cuda and v_cache.is_cuda and k_cache.is_contiguous() and v_cache.is_contiguous()):
        _ptr(k_cache), _ptr(v_cache)  # (one of them raises)
    if not e4m3:
        return _pack_cache(k_cache.data_ptr(), v_cache.data_ptr(), 0, 0, n_pages, Hkv, page, D, code, 0)
    rows, byte = shape[:3], _names["uint8"]
    return _pack_cache(k_cache.data_ptr(), v_cache.data_ptr(), _flat("k_exp", k_exp, byte, rows), _flat("v_exp", v_exp, byte, rows),
                       n_pages, Hkv, page, D, code, 1)


def kp_cache_write(k, v, slots, k_cache, v_cache, k_exp=None, v_exp=None, stream=None) -> None:
    """New rows k, v [T, Hkv, D] into slots [T] int64 (negative: skipped; each named at most once) of the cache [n_pages, Hkv, page, D], as they are
    or, into a float8_e4m3fn cache with exponents [n_pages, Hkv, page] uint8, quantised row by row."""
    T, (_, Hkv, _, D) = k.shape[0], k_cache.shape
    _check(lib().kp_cache_write(_heads("k", k, (T, Hkv, D), k.dtype), _heads("v", v, (T, Hkv, D), k.dtype),
                                _flat("slots", slots, (_names or _types())["int64"], (T,)), T,
                                _cache_of(k_cache, v_cache, k_exp, v_exp, k.dtype), _stream(stream)))


def kp_cache_read(k_cache, v_cache, k_exp, v_exp, block_table, starts, k, v, stream=None) -> None:
    """Whole sequences out of the cache: key t of sequence s (block_table [n, width] int32) goes to row starts[s] + t of
    k, v [T, Hkv, D], up to starts[s + 1] (starts [n + 1] int32)."""
    T, (_, Hkv, _, D) = k.shape[0], k_cache.shape
    n, width = block_table.shape
    _check(lib().kp_cache_read(_cache_of(k_cache, v_cache, k_exp, v_exp, k.dtype),
                               _flat("block_table", block_table, (_names or _types())["int32"]), width,
                               _flat("starts", starts, (_names or _types())["int32"], (n + 1,)), n, T,
                               _heads("k", k, (T, Hkv, D), k.dtype), _heads("v", v, (T, Hkv, D), k.dtype), _stream(stream)))


def kp_cache_move(source, target, starts, k_cache, v_cache, k_exp=None, v_exp=None, stream=None) -> None:
    """Rows of slots source [N] int64 to slots target [N] int64 of the cache, all heads, keys and values.  starts None: no slot is
    in both; else int32 [n + 1]: groups of moves, each in order (see the header for what groups of more than KP_MOVE_RUN may
    hold)."""
    i64, N = (_names or _types())["int64"], source.shape[0]
    # (what the codes of an e4m3 cache are read as does not matter here)
    kind = k_cache.dtype if k_cache.dtype is not _names["float8_e4m3fn"] else _names["bfloat16"]
    _check(lib().kp_cache_move(_flat("source", source, i64, (N,)), _flat("target", target, i64, (N,)), N,
                               0 if starts is None else _flat("starts", starts, _names["int32"]), 0 if starts is None else starts.shape[0] - 1,
                               _cache_of(k_cache, v_cache, k_exp, v_exp, kind), _stream_at(stream, source)))


def kp_attn_paged_bytes(q, k_cache, block_table, window: int, sinks: int) -> int:
    """Bytes of workspace that kp_attn_paged takes for q [T, Hq, D]."""
    T, Hq, D = q.shape
    n, width = block_table.shape
    return int(lib().kp_attn_paged_bytes(T, n, Hq, k_cache.shape[1], D, width, k_cache.shape[2], window, sinks))


def kp_attn_paged_launch_shape(q, k_cache, block_table, window: int, sinks: int) -> tuple[int, int, int]:
    """Workgroups, waves per workgroup and regions of a recording of kp_attn_paged."""
    T, Hq, D = q.shape
    n, width = block_table.shape
    return _shape_of(lib().kp_attn_paged_launch_shape, T, n, Hq, k_cache.shape[1], D, width, k_cache.shape[2], window, sinks)


def kp_attn_paged(q, k_cache, v_cache, k_exp, v_exp, block_table, lens, starts, o, lse, window: int, sinks: int,
                  scale: float, workspace=None, region_mask: int = 0, trace_buf=None, trace_cap: int = 0,
                  stream=None) -> None:
    """Attention of new tokens q [T, Hq, D] over a cache that holds them: sequence s has the tokens starts[s] ..
    starts[s + 1] - 1 and lens[s] keys, found through block_table [n, width] int32; o [T, Hq, D], lse [Hq, T] or None."""
    T, Hq, D = q.shape
    n, width = block_table.shape
    if D != k_cache.shape[3]:
        raise ValueError("q and the cache must have the same D")
    ws, nbytes = _workspace(workspace)
    _check(lib().kp_attn_paged(
        _heads("q", q, q.shape, q.dtype), _cache_of(k_cache, v_cache, k_exp, v_exp, q.dtype),
        _flat("block_table", block_table, (_names or _types())["int32"]), width, _flat("lens", lens, (_names or _types())["int32"], (n,)),
        _flat("starts", starts, (_names or _types())["int32"], (n + 1,)), _heads("o", o, q.shape, q.dtype),
        0 if lse is None else _flat("lse", lse, (_names or _types())["float32"], (Hq, T)), T, n, Hq, window, sinks, scale, ws, nbytes,
        region_mask & 0xFFFFFFFF, _ptr(trace_buf), trace_cap, _stream(stream)))


def _cache_type(k_cache) -> int:
    return KP_CACHE_E4M3 if k_cache.dtype is (_names or _types())["float8_e4m3fn"] else KP_CACHE_SAME


def kp_attn_tree_bytes(q, k_cache, block_table, window: int, sinks: int) -> int:
    """Bytes of workspace that kp_attn_tree takes for q [T, Hq, D]."""
    T, Hq, D = q.shape
    n, width = block_table.shape
    return int(lib().kp_attn_tree_bytes(T, n, Hq, k_cache.shape[1], D, width, k_cache.shape[2], _cache_type(k_cache), window, sinks))


def kp_attn_tree_launch_shape(q, k_cache, block_table, window: int, sinks: int) -> tuple[int, int, int]:
    """Workgroups, waves per workgroup and regions of a recording of kp_attn_tree."""
    T, Hq, D = q.shape
    n, width = block_table.shape
    return _shape_of(lib().kp_attn_tree_launch_shape, T, n, Hq, k_cache.shape[1], D, width, k_cache.shape[2], _cache_type(k_cache), window, sinks)


def kp_attn_tree(q, k_cache, v_cache, k_exp, v_exp, block_table, lens, starts, seen, depth, o, lse, window: int, sinks: int,
                 scale: float, workspace=None, region_mask: int = 0, trace_buf=None, trace_cap: int = 0, stream=None) -> None:
    """Attention of drafted tokens q [T, Hq, D] over a cache that holds them as the last of each sequence's keys: as kp_attn_paged, but
    that a token sees the drafted ones that its bits seen [T, words] int64 name (bit j % 64 of word j / 64: drafted token j of its
    sequence; None: none), and the context from position lens - drafted + depth; depth [T] int32 or None."""
    T, Hq, D = q.shape
    n, width = block_table.shape
    if D != k_cache.shape[3]:
        raise ValueError("q and the cache must have the same D")
    names = _names or _types()
    i32 = names["int32"]
    ws, nbytes = _workspace(workspace)
    words = 0 if seen is None else seen.shape[1]
    _check(lib().kp_attn_tree(
        _heads("q", q, q.shape, q.dtype), _cache_of(k_cache, v_cache, k_exp, v_exp, q.dtype), _flat("block_table", block_table, i32), width,
        _flat("lens", lens, i32, (n,)), _flat("starts", starts, i32, (n + 1,)), 0 if seen is None else _flat("seen", seen, names["int64"], (T, words)), words,
        0 if depth is None else _flat("depth", depth, i32, (T,)), _heads("o", o, q.shape, q.dtype),
        0 if lse is None else _flat("lse", lse, names["float32"], (Hq, T)), T, n, Hq, window, sinks, scale, ws, nbytes,
        region_mask & 0xFFFFFFFF, _ptr(trace_buf), trace_cap, _stream_at(stream, q)))


# ---- queries and keys normed and turned ----------------------------------------------------------------
# positions: int32, of each token, [S] (or [T]) if all sequences share them, [B, S], or with an axis in front, [axes, S] for a
# batch without a dimension of its own and [axes, B, S] for one with it; any strides with the last dimension contiguous.


_pack_turns = struct.Struct("PqqPPiiixxxx").pack


def _turns(positions, freq, axis, adjacent, batch, tokens):
    """kp_turns of the tensors above; batch: number of sequences, or None for a batch without a dimension of its own."""
    if freq is None:
        return None
    names = _names or _types()
    shape, steps, pairs = positions.shape, positions.stride(), freq.shape[0]
    front = 2 if batch is None else 3  # dimensions, with that of the axes
    n = len(shape)
    if positions.dtype is not names["int32"] or not positions.is_cuda or not 0 < n <= front or shape[-1] != tokens or (tokens > 1 and steps[-1] != 1):
        raise ValueError(f"positions must be int32 on the GPU, {tokens} for each sequence, contiguous, not {list(shape)} of {positions.dtype}")
    if batch is not None and n >= 2 and shape[-2] != batch:
        raise ValueError(f"positions must be [S], [B, S] or [axes, B, S] with B = {batch}, not {list(shape)}")
    axes, axis_step = (shape[0], steps[0]) if n == front else (1, 0)
    return _pack_turns(positions.data_ptr(), axis_step, steps[-2] if batch is not None and n >= 2 else 0, _flat("freq", freq, names["float32"], (pairs,)),
                       0 if axis is None else _flat("axis", axis, names["uint8"], (pairs,)), pairs, axes, 1 if adjacent else 0)


def _norms(q_weight, k_weight, D, dtype):
    """Device pointers of the norms' weights (0: none) and their type."""
    code = _type_code(dtype)
    if q_weight is None and k_weight is None:
        return 0, 0, code
    kind = (k_weight if q_weight is None else q_weight).dtype
    if kind is not dtype:
        if kind is not _names["float32"]:
            raise ValueError(f"weights must both be float32 or both {dtype}, not {kind}")
        code = KP_FP32
    return 0 if q_weight is None else _flat("q_weight", q_weight, kind, (D,)), 0 if k_weight is None else _flat("k_weight", k_weight, kind, (D,)), code


def _two(q, k):
    """Of queries and keys, either of which may be None: number of sequences (None: [T, H, D]), both shapes, heads, tokens, D and
    type."""
    some = k if q is None else q
    if some is None:
        raise ValueError("queries or keys are needed")
    shape = some.shape
    if len(shape) == 4:
        B, H, S, D = shape
    else:
        S, H, D = shape
        B = None
    if q is None:
        return B, None, shape, 0, H, S, D, some.dtype
    if k is None:
        return B, shape, None, H, 0, S, D, some.dtype
    other = k.shape
    if len(other) != len(shape) or other[0] != shape[0] or other[2:] != shape[2:]:
        raise ValueError(f"keys must have the queries' sequences, tokens and D, not {list(other)} to {list(shape)}")
    return B, shape, other, H, other[1], S, D, some.dtype


def kp_norm_rotate(q, k, q_weight, k_weight, eps: float, positions, freq, axis, adjacent: bool, q_out, k_out, stream=None) -> None:
    """Heads of q and k ([B, H, S, D], or [T, H, D] where there is no batch) normed by their root mean square with weights [D]
    (None: not normed), their pairs turned by position * freq[pair]; freq float32 [pairs] (None: not turned), axis uint8
    [pairs] or None.  q and q_out, or k and k_out, may be None; outputs may be the inputs."""
    B, qs, ks, Hq, Hk, S, D, dtype = _two(q, k)
    qw, kw, kind = _norms(q_weight, k_weight, D, dtype)
    _check(lib().kp_norm_rotate(
        None if q is None else _heads("q", q, None, dtype), None if k is None else _heads("k", k, None, dtype), qw, kw, kind, eps,
        _turns(positions, freq, axis, adjacent, B, S), None if q is None else _heads("q_out", q_out, qs, dtype),
        None if k is None else _heads("k_out", k_out, ks, dtype), 1 if B is None else B, Hq, Hk, S, D, _names[dtype],
        _stream_at(stream, k if q is None else q)))


def kp_norm_rotate_grad_bytes(q, k) -> int:
    """Bytes of workspace that kp_norm_rotate_grad takes for q and k (either may be None)."""
    B, _, _, Hq, Hk, S, D, _ = _two(q, k)
    return int(lib().kp_norm_rotate_grad_bytes(1 if B is None else B, Hq, Hk, S, D))


def kp_norm_rotate_grad(q, k, q_weight, k_weight, eps: float, positions, freq, axis, adjacent: bool, d_q_out, d_k_out, dq, dk,
                        dq_weight=None, dk_weight=None, workspace=None, stream=None) -> None:
    """Gradient of kp_norm_rotate: dq, dk from d_q_out, d_k_out and the q, k that were normed (not looked at without weights), and
    dq_weight, dk_weight [D] float32 where there are weights."""
    B, qs, ks, Hq, Hk, S, D, dtype = _two(d_q_out, d_k_out)
    qw, kw, kind = _norms(q_weight, k_weight, D, dtype)
    f32 = _names["float32"]
    ws, n = _workspace(workspace)
    some = lambda name, t, shape: None if shape is None else _heads(name, t, shape, dtype)  # noqa: E731
    _check(lib().kp_norm_rotate_grad(
        some("q", q, qs if qw else None), some("k", k, ks if kw else None), qw, kw, kind, eps, _turns(positions, freq, axis, adjacent, B, S),
        some("d_q_out", d_q_out, qs), some("d_k_out", d_k_out, ks), some("dq", dq, qs), some("dk", dk, ks),
        _flat("dq_weight", dq_weight, f32, (D,)) if qw else 0, _flat("dk_weight", dk_weight, f32, (D,)) if kw else 0,
        1 if B is None else B, Hq, Hk, S, D, _names[dtype], ws, n, _stream_at(stream, d_k_out if d_q_out is None else d_q_out)))


def kp_norm_rotate_write(q, k, v, q_weight, k_weight, eps: float, positions, freq, axis, adjacent: bool, q_out, slots, k_cache, v_cache,
                         k_exp=None, v_exp=None, stream=None) -> None:
    """kp_norm_rotate of new tokens q [T, Hq, D] (or None) and k [T, Hkv, D], queries to q_out, keys and the values v to slots [T] of the
    cache as kp_cache_write puts them there."""
    T, (_, Hkv, _, D), dtype = k.shape[0], k_cache.shape, k.dtype
    Hq = 0 if q is None else q.shape[1]
    queries, keys = (T, Hq, D), (T, Hkv, D)
    qw, kw, kind = _norms(q_weight, k_weight, D, dtype)
    _check(lib().kp_norm_rotate_write(
        None if q is None else _heads("q", q, queries, dtype), _heads("k", k, keys, dtype), _heads("v", v, keys, dtype), qw, kw, kind, eps,
        _turns(positions, freq, axis, adjacent, None, T), None if q is None else _heads("q_out", q_out, queries, dtype),
        _flat("slots", slots, _names["int64"], (T,)), T, Hq, _cache_of(k_cache, v_cache, k_exp, v_exp, dtype), _stream_at(stream, k)))


# ---- views of the statistics block (layout documented in include/kperf.h) ------------------------

STATS_HEADER_FIELDS = (
    "n_slots_valid", "n_pairs", "n_orphan_start", "n_orphan_end", "n_invalid", "n_dropped",
    "n_disorder", "n_span_overflow_wgs", "n_nonmonotonic", "n_overlap_wgs", "status",
    "n_wg", "waves_per_wg", "n_regions", "cap_wave", "reserved",
)
WAVE_REGION_DTYPE = np.dtype([("sum", "<u8"), ("n", "<u4"), ("max", "<u4")])


def parse_stats(buf) -> dict:
    """Split a statistics block (bytes on the host: numpy uint8 array or CPU tensor) into fields."""
    if hasattr(buf, "numpy"):
        buf = buf.cpu().numpy()
    b = np.ascontiguousarray(buf).view(np.uint8)
    hdr = b[:128].view("<u8")
    out = {k: int(hdr[i]) for i, k in enumerate(STATS_HEADER_FIELDS)}
    n_wg, W, R = out["n_wg"], out["waves_per_wg"], out["n_regions"]
    pos = 128
    for name, count, dt, shape in (
        ("hist", 64 * R, "<u8", (R, 64)), ("cnt", R, "<u8", (R,)), ("sum", R, "<u8", (R,)),
        ("min", R, "<u8", (R,)), ("max", R, "<u8", (R,)), ("U", R, "<u8", (R,)),
        ("O", R * R, "<u8", (R, R)), ("F", R * R, "<f8", (R, R)),
    ):
        out[name] = b[pos : pos + 8 * count].view(dt).reshape(shape)
        pos += 8 * count
    out["per"] = b[pos : pos + 16 * n_wg * W * R].view(WAVE_REGION_DTYPE).reshape(n_wg, W, R)
    return out
