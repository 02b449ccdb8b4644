"""ctypes binding of libdsla.so: same entry-point names as include/dsla.h, argument
marshalling only.  Tensors are torch tensors on the GPU; their data pointers and the
current torch HIP stream are handed to the library.  No computation happens here, and
there is no fallback: if the library is missing, loading raises.

The calls of a serving loop go through _marshal.so, the same in native code; arguments that
it does not take (it then returns None) go the way written out here, and so do all where it is
not built, or not for this interpreter, PyTorch and header.
"""
from __future__ import annotations

import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(HERE, "libdsla.so")
_lib = None
_torch = None   # torch._C once the library is loaded


class _General:
    """In the place of _marshal: leaves every call to the general way."""
    decode = decode_slots = prefill = prefill_varlen = attention_decode = attention_prefill = project = staticmethod(lambda *a: None)
    residual_norm = head_norm = quantize = project_fp8 = decode
    cache_extend = cache_fork = cache_truncate = cache_accept = cache_compact = qk_rope = attention_paged = decode


_native = _General   # _marshal once the library is loaded, where it can be used

DSLA_F32, DSLA_BF16, DSLA_E4M3 = 0, 1, 2
DSLA_SCALE_F32, DSLA_SCALE_E8M0 = 0, 1
DSLA_ACT_NONE, DSLA_ACT_SIGMOID, DSLA_ACT_SILU = 0, 1, 2
KERNEL_NAMES = ("state_init", "prefill_segment_state", "prefill_segment_scan", "prefill_chunk_loop", "decode",
                "prefill_segment_list", "attention_entropy", "attention_decode", "decode_multi", "attention_prefill", "project",
                "cache", "qk_rope", "attention_paged", "residual_norm", "head_norm", "quantize", "project_fp8")
EXPORTS = ("dsla_state_init", "dsla_prefill_workspace_bytes", "dsla_prefill", "dsla_prefill_static_ws", "dsla_decode",
           "dsla_prefill_varlen_workspace_bytes", "dsla_prefill_varlen", "dsla_decode_slots",
           "dsla_decode_multi", "dsla_prefill_multi_workspace_bytes", "dsla_prefill_multi",
           "dsla_attention_entropy_workspace_bytes", "dsla_attention_entropy",
           "dsla_attention_decode_workspace_bytes", "dsla_attention_decode", "dsla_attention_prefill", "dsla_project",
           "dsla_residual_norm", "dsla_head_norm", "dsla_quantize", "dsla_project_fp8",
           "dsla_cache_workspace_bytes", "dsla_cache_init", "dsla_cache_extend", "dsla_cache_fork", "dsla_cache_truncate",
           "dsla_cache_accept", "dsla_cache_compact", "dsla_qk_rope", "dsla_attention_paged_workspace_bytes", "dsla_attention_paged",
           "dsla_rank_layers", "dsla_max_conversion_rate", "dsla_kv_cache_bytes", "dsla_conversion_plan",
           "dsla_status_string", "dsla_last_hip_error", "dsla_profile_enable", "dsla_profile_collect")


class DslaDesc(ctypes.Structure):
    """Mirror of `dsla_desc` in include/dsla.h."""
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("d_k", ctypes.c_int32), ("d_v", ctypes.c_int32),
                ("chunk", ctypes.c_int32), ("segments", ctypes.c_int32), ("io_dtype", ctypes.c_int32),
                ("gate_dtype", ctypes.c_int32), ("gate_mode", ctypes.c_int32), ("zero_init", ctypes.c_int32),
                ("tau", ctypes.c_float), ("gamma", ctypes.c_float), ("scale", ctypes.c_float),
                ("gamma_per_head", ctypes.c_void_p), ("status", ctypes.c_void_p)]


class DslaMulti(ctypes.Structure):
    """Mirror of `dsla_multi` in include/dsla.h."""
    _fields_ = [("n_states", ctypes.c_int32), ("H_kv", ctypes.c_int32), ("g_alpha", ctypes.POINTER(ctypes.c_void_p)),
                ("g_beta", ctypes.POINTER(ctypes.c_void_p)), ("S", ctypes.POINTER(ctypes.c_void_p)),
                ("weights", ctypes.POINTER(ctypes.c_float)), ("weights_per_head", ctypes.c_void_p)]


class DslaCache(ctypes.Structure):
    """Mirror of `dsla_cache` in include/dsla.h."""
    _fields_ = [("n_pages", ctypes.c_int32), ("page", ctypes.c_int32), ("H_kv", ctypes.c_int32), ("d", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("n_seqs", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("table", ctypes.c_void_p), ("lens", ctypes.c_void_p),
                ("refs", ctypes.c_void_p), ("status", ctypes.c_void_p)]


class DslaBatch(ctypes.Structure):
    """Mirror of `dsla_batch` in include/dsla.h."""
    _fields_ = [("B", ctypes.c_int32), ("max_n", ctypes.c_int32), ("total", ctypes.c_int64), ("cu", ctypes.c_void_p), ("row", ctypes.c_void_p),
                ("start", ctypes.c_void_p)]


class DslaRope(ctypes.Structure):
    """Mirror of `dsla_rope` in include/dsla.h."""
    _fields_ = [("H", ctypes.c_int32), ("H_kv", ctypes.c_int32), ("d", ctypes.c_int32), ("io_dtype", ctypes.c_int32), ("rot_dim", ctypes.c_int32),
                ("interleaved", ctypes.c_int32), ("eps", ctypes.c_float), ("inv_freq", ctypes.c_void_p), ("q_weight", ctypes.c_void_p),
                ("k_weight", ctypes.c_void_p), ("offsets", ctypes.c_void_p)]


class DslaNorm(ctypes.Structure):
    """Mirror of `dsla_norm` in include/dsla.h."""
    _fields_ = [("D", ctypes.c_int32), ("x_dtype", ctypes.c_int32), ("y_dtype", ctypes.c_int32), ("h_dtype", ctypes.c_int32),
                ("scale_type", ctypes.c_int32), ("gate_act", ctypes.c_int32), ("eps", ctypes.c_float), ("residual_scale", ctypes.c_float),
                ("post_weight", ctypes.c_void_p), ("pre_weight", ctypes.c_void_p)]


class DslaHeads(ctypes.Structure):
    """Mirror of `dsla_heads` in include/dsla.h."""
    _fields_ = [("H", ctypes.c_int32), ("d", ctypes.c_int32), ("io_dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32),
                ("scale_type", ctypes.c_int32), ("gate_act", ctypes.c_int32), ("eps", ctypes.c_float), ("weight", ctypes.c_void_p)]


class DslaError(RuntimeError):
    def __init__(self, status: int, text: str):
        super().__init__(f"dsla status {status}: {text}")
        self.status = status


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """Loads libdsla.so (built by paper_2506_09316_amd/build.py).  Raises if it is absent."""
    global _lib, _torch, _native
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise FileNotFoundError(f"{_LIB_PATH} is not built; run `python -m paper_2506_09316_amd.build` "
                                "(or __graft_entry__.build())")
    # PyTorch ships its own copy of the HIP runtime.  Whichever copy is loaded first serves the whole process, and
    # tensors and kernels must live in the same one: load PyTorch's before the library pulls in the system's.
    try:
        from torch import _C as _torch
    except ImportError:
        pass
    lib = ctypes.CDLL(_LIB_PATH)
    vp, dp = ctypes.c_void_p, ctypes.POINTER(DslaDesc)
    lib.dsla_state_init.argtypes = [dp, vp, vp, vp]
    lib.dsla_state_init.restype = ctypes.c_int
    lib.dsla_prefill_workspace_bytes.argtypes = [dp, ctypes.c_int64]
    lib.dsla_prefill_workspace_bytes.restype = ctypes.c_size_t
    lib.dsla_prefill.argtypes = [dp, ctypes.c_int64] + [vp] * 9 + [ctypes.c_size_t, vp]
    lib.dsla_prefill.restype = ctypes.c_int
    lib.dsla_prefill_static_ws.argtypes = [dp, ctypes.c_int64] + [vp] * 9
    lib.dsla_prefill_static_ws.restype = ctypes.c_int
    lib.dsla_decode.argtypes = [dp] + [vp] * 9
    lib.dsla_decode.restype = ctypes.c_int
    lib.dsla_prefill_varlen_workspace_bytes.argtypes = [dp, ctypes.c_int64, ctypes.c_int64]
    lib.dsla_prefill_varlen_workspace_bytes.restype = ctypes.c_size_t
    lib.dsla_prefill_varlen.argtypes = [dp, ctypes.c_int64, ctypes.c_int64] + [vp] * 12 + [ctypes.c_size_t, vp]
    lib.dsla_prefill_varlen.restype = ctypes.c_int
    lib.dsla_decode_slots.argtypes = [dp] + [vp] * 11
    lib.dsla_decode_slots.restype = ctypes.c_int
    mp = ctypes.POINTER(DslaMulti)
    lib.dsla_decode_multi.argtypes = [dp, mp] + [vp] * 5
    lib.dsla_decode_multi.restype = ctypes.c_int
    lib.dsla_prefill_multi_workspace_bytes.argtypes = [dp, mp, ctypes.c_int64]
    lib.dsla_prefill_multi_workspace_bytes.restype = ctypes.c_size_t
    lib.dsla_prefill_multi.argtypes = [dp, mp, ctypes.c_int64] + [vp] * 5 + [ctypes.c_size_t, vp]
    lib.dsla_prefill_multi.restype = ctypes.c_int
    lib.dsla_attention_entropy_workspace_bytes.argtypes = [ctypes.c_int32] * 3 + [ctypes.c_int64]
    lib.dsla_attention_entropy_workspace_bytes.restype = ctypes.c_size_t
    lib.dsla_attention_entropy.argtypes = ([ctypes.c_int32] * 3 + [ctypes.c_int64, ctypes.c_int32, ctypes.c_float]
                                           + [vp] * 4 + [ctypes.c_size_t, vp])
    lib.dsla_attention_entropy.restype = ctypes.c_int
    lib.dsla_attention_decode_workspace_bytes.argtypes = [ctypes.c_int32] * 3 + [ctypes.c_int64]
    lib.dsla_attention_decode_workspace_bytes.restype = ctypes.c_size_t
    lib.dsla_attention_decode.argtypes = ([ctypes.c_int32] * 3 + [ctypes.c_int64, ctypes.c_int32, ctypes.c_float]
                                          + [vp] * 6 + [ctypes.c_size_t, vp])
    lib.dsla_attention_decode.restype = ctypes.c_int
    lib.dsla_project.argtypes = [ctypes.c_int64] + [ctypes.c_int32] * 3 + [vp] * 3 + [ctypes.POINTER(ctypes.c_void_p), vp]
    lib.dsla_project.restype = ctypes.c_int
    lib.dsla_residual_norm.argtypes = [ctypes.POINTER(DslaNorm), ctypes.c_int64] + [vp] * 7
    lib.dsla_residual_norm.restype = ctypes.c_int
    lib.dsla_head_norm.argtypes = [ctypes.POINTER(DslaHeads), ctypes.c_int64] + [vp] * 5
    lib.dsla_head_norm.restype = ctypes.c_int
    lib.dsla_quantize.argtypes = [ctypes.c_int64] + [ctypes.c_int32] * 4 + [vp] * 4
    lib.dsla_quantize.restype = ctypes.c_int
    lib.dsla_project_fp8.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(ctypes.c_int32), ctypes.c_int32] + [vp] * 5 + [
        ctypes.c_int32, ctypes.POINTER(ctypes.c_void_p), vp]
    lib.dsla_project_fp8.restype = ctypes.c_int
    lib.dsla_attention_prefill.argtypes = [ctypes.c_int32] * 3 + [ctypes.c_int64, ctypes.c_int32, ctypes.c_float] + [vp] * 5
    lib.dsla_attention_prefill.restype = ctypes.c_int
    cp, bp, pools = ctypes.POINTER(DslaCache), ctypes.POINTER(DslaBatch), [ctypes.c_int32, ctypes.POINTER(ctypes.c_void_p)]
    scratch = [vp, ctypes.c_size_t, vp]
    lib.dsla_cache_workspace_bytes.argtypes = [cp, ctypes.c_int32]
    lib.dsla_cache_workspace_bytes.restype = ctypes.c_size_t
    lib.dsla_cache_init.argtypes = [cp, vp]
    lib.dsla_cache_init.restype = ctypes.c_int
    lib.dsla_cache_extend.argtypes = [cp, bp, *pools, *scratch]
    lib.dsla_cache_extend.restype = ctypes.c_int
    lib.dsla_cache_fork.argtypes = [cp, vp, vp]
    lib.dsla_cache_fork.restype = ctypes.c_int
    lib.dsla_cache_truncate.argtypes = [cp, vp, vp]
    lib.dsla_cache_truncate.restype = ctypes.c_int
    lib.dsla_cache_accept.argtypes = [cp, bp, vp, vp, *pools, *scratch]
    lib.dsla_cache_accept.restype = ctypes.c_int
    lib.dsla_cache_compact.argtypes = [cp, vp, *pools, *scratch]
    lib.dsla_cache_compact.restype = ctypes.c_int
    lib.dsla_qk_rope.argtypes = [ctypes.POINTER(DslaRope), ctypes.c_int64] + [vp] * 5 + [cp, bp] + [vp] * 3
    lib.dsla_qk_rope.restype = ctypes.c_int
    lib.dsla_attention_paged_workspace_bytes.argtypes = [cp, bp, ctypes.c_int32, ctypes.c_int64]
    lib.dsla_attention_paged_workspace_bytes.restype = ctypes.c_size_t
    lib.dsla_attention_paged.argtypes = [cp, bp, ctypes.c_int32, ctypes.c_int64, ctypes.c_float] + [vp] * 5 + scratch
    lib.dsla_attention_paged.restype = ctypes.c_int
    lib.dsla_rank_layers.argtypes = [ctypes.c_int32, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_int32)]
    lib.dsla_rank_layers.restype = ctypes.c_int
    lib.dsla_max_conversion_rate.argtypes = [ctypes.c_int64]
    lib.dsla_max_conversion_rate.restype = ctypes.c_float
    lib.dsla_kv_cache_bytes.argtypes = [ctypes.c_int32, ctypes.c_int64, ctypes.c_int64] + [ctypes.c_int32] * 3
    lib.dsla_kv_cache_bytes.restype = ctypes.c_int64
    lib.dsla_conversion_plan.argtypes = ([ctypes.c_int32, ctypes.POINTER(ctypes.c_int32)] + [ctypes.c_int64] * 4
                                         + [ctypes.c_float, ctypes.POINTER(ctypes.c_uint8), ctypes.POINTER(ctypes.c_int32),
                                            ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_int32)])
    lib.dsla_conversion_plan.restype = ctypes.c_int
    lib.dsla_status_string.argtypes = [ctypes.c_int]
    lib.dsla_status_string.restype = ctypes.c_char_p
    lib.dsla_last_hip_error.argtypes = []
    lib.dsla_last_hip_error.restype = ctypes.c_char_p
    lib.dsla_profile_enable.argtypes = [ctypes.c_int, ctypes.c_int]
    lib.dsla_profile_enable.restype = ctypes.c_int
    lib.dsla_profile_collect.argtypes = [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64)]
    lib.dsla_profile_collect.restype = ctypes.c_int
    if _torch is not None:
        _native = _load_native(lib)
    _lib = lib
    return lib


def _load_native(lib):
    import torch
    try:
        from . import _marshal
        from .build import marshal_stamp
        built_for, here = getattr(_marshal, "built_for", "another version"), marshal_stamp()
        if built_for != here:
            raise ImportError(f"_marshal.so was built for {built_for}, this is {here}")
        torch_calls = _torch._cuda_getDevice, _torch._cuda_getCurrentRawStream   # (a PyTorch without GPUs has none)
    except (ImportError, AttributeError, OSError) as e:
        import warnings
        warnings.warn(f"the calls go through ctypes, at 2 us more each on the host ({e}); `python -m paper_2506_09316_amd.build` builds the native ones",
                      RuntimeWarning, stacklevel=3)
        return _General
    entries = (lib.dsla_decode, lib.dsla_decode_slots, lib.dsla_prefill, lib.dsla_prefill_varlen, lib.dsla_attention_decode,
               lib.dsla_attention_prefill, lib.dsla_project, lib.dsla_cache_extend, lib.dsla_cache_fork, lib.dsla_cache_truncate, lib.dsla_cache_accept,
               lib.dsla_cache_compact, lib.dsla_qk_rope, lib.dsla_attention_paged, lib.dsla_residual_norm, lib.dsla_head_norm, lib.dsla_quantize, lib.dsla_project_fp8)
    _marshal.bind(*torch_calls, torch.nn.Parameter, DslaDesc, DslaCache, DslaBatch, DslaRope, DslaNorm, DslaHeads, *[ctypes.cast(f, ctypes.c_void_p).value for f in entries])
    return _marshal


def _check(status: int):
    if status != 0:
        lib = load_library()
        text = lib.dsla_status_string(status).decode()
        if status == 5:
            text += ": " + lib.dsla_last_hip_error().decode()
        raise DslaError(status, text)


def _dtype_code(t):
    import torch
    if t.dtype == torch.bfloat16:
        return DSLA_BF16
    if t.dtype == torch.float32:
        return DSLA_F32
    raise TypeError(f"unsupported dtype {t.dtype}")


def _ptr(t):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "tensors must be contiguous GPU tensors"
    return t.data_ptr()


def _stream():
    """Handle of torch's current stream on its current device.  torch.cuda.current_stream() builds a Stream object: 3.0 us
    against 0.2, in a decode call of one sequence that took 8.8 us on the host for 4 us on the GPU (5.4 this way, 3.5 through _marshal)."""
    return _torch._cuda_getCurrentRawStream(_torch._cuda_getDevice())


def make_desc(B, H, d_k, d_v, *, io_dtype, gate_dtype, gamma=0.5, scale=1.0, chunk=0, segments=0,
              gamma_per_head=None, gate_mode=0, tau=16.0, zero_init=False, status=None) -> DslaDesc:
    """status: optional int32 GPU tensor of one element (the caller keeps it alive)."""
    gp = ctypes.c_void_p(gamma_per_head.data_ptr()) if gamma_per_head is not None else None
    sp = ctypes.c_void_p(status.data_ptr()) if status is not None else None
    return DslaDesc(int(B), int(H), int(d_k), int(d_v), int(chunk), int(segments), int(io_dtype), int(gate_dtype),
                    int(gate_mode), int(bool(zero_init)), float(tau), float(gamma), float(scale), gp, sp)


def dsla_state_init(desc: DslaDesc, S1, S2):
    """Zero both states (include/dsla.h: dsla_state_init)."""
    _check(load_library().dsla_state_init(ctypes.byref(desc), _ptr(S1), _ptr(S2), _stream()))


def dsla_prefill_workspace_bytes(desc: DslaDesc, T: int) -> int:
    return int(load_library().dsla_prefill_workspace_bytes(ctypes.byref(desc), int(T)))


def dsla_prefill(desc: DslaDesc, T, q, k, v, g1, g2, S1, S2, o, workspace=None):
    """Chunked prefill over T tokens (include/dsla.h: dsla_prefill).  `workspace` is a uint8 GPU
    tensor of at least dsla_prefill_workspace_bytes(desc, T) bytes, or None when that is zero."""
    lib = _lib or load_library()
    status = _native.prefill(desc, T, q, k, v, g1, g2, S1, S2, o, workspace)
    if status is not None:
        return _check(status)
    wbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib.dsla_prefill(ctypes.byref(desc), int(T), _ptr(q), _ptr(k), _ptr(v), _ptr(g1), _ptr(g2),
                                       _ptr(S1), _ptr(S2), _ptr(o), _ptr(workspace), wbytes, _stream()))


def dsla_prefill_static_ws(desc: DslaDesc, T, q, k, v, g1, g2, S1, S2, o):
    """dsla_prefill on the library's built-in scratch buffer (include/dsla.h: dsla_prefill_static_ws)."""
    _check(load_library().dsla_prefill_static_ws(ctypes.byref(desc), int(T), _ptr(q), _ptr(k), _ptr(v), _ptr(g1),
                                                 _ptr(g2), _ptr(S1), _ptr(S2), _ptr(o), _stream()))


def dsla_decode(desc: DslaDesc, q, k, v, g1, g2, S1, S2, o):
    """One fused decode step (include/dsla.h: dsla_decode)."""
    lib = _lib or load_library()
    status = _native.decode(desc, q, k, v, g1, g2, S1, S2, o)
    if status is not None:
        return _check(status)
    _check(lib.dsla_decode(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(g1), _ptr(g2),
                                      _ptr(S1), _ptr(S2), _ptr(o), _stream()))


def dsla_prefill_varlen_workspace_bytes(desc: DslaDesc, total_T: int, max_T: int) -> int:
    return int(load_library().dsla_prefill_varlen_workspace_bytes(ctypes.byref(desc), int(total_T), int(max_T)))


def dsla_prefill_varlen(desc: DslaDesc, total_T, max_T, cu_seqlens, state_slot, q, k, v, g1, g2, S1, S2, o,
                        workspace=None, seq_index=None):
    """Prefill of packed sequences (include/dsla.h: dsla_prefill_varlen).  cu_seqlens: int32 GPU tensor;
    state_slot, seq_index: int32 GPU tensors [B] or None."""
    lib = _lib or load_library()
    status = _native.prefill_varlen(desc, total_T, max_T, cu_seqlens, seq_index, state_slot, q, k, v, g1, g2, S1, S2, o, workspace)
    if status is not None:
        return _check(status)
    wbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib.dsla_prefill_varlen(ctypes.byref(desc), int(total_T), int(max_T), _ptr(cu_seqlens),
                                              _ptr(seq_index), _ptr(state_slot), _ptr(q), _ptr(k), _ptr(v), _ptr(g1), _ptr(g2),
                                              _ptr(S1), _ptr(S2), _ptr(o), _ptr(workspace), wbytes, _stream()))


def dsla_decode_slots(desc: DslaDesc, q, k, v, g1, g2, state_slot, S1, S2, o, row_index=None):
    """One decode step on states picked from a pool (include/dsla.h: dsla_decode_slots)."""
    lib = _lib or load_library()
    status = _native.decode_slots(desc, q, k, v, g1, g2, row_index, state_slot, S1, S2, o)
    if status is not None:
        return _check(status)
    _check(lib.dsla_decode_slots(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(g1), _ptr(g2),
                                            _ptr(row_index), _ptr(state_slot), _ptr(S1), _ptr(S2), _ptr(o), _stream()))


def make_multi(g_alpha, S, weights, *, g_beta=None, H_kv=0, weights_per_head=None) -> DslaMulti:
    """dsla_multi from lists of GPU tensors (one per state).  The returned structure keeps the host arrays it
    points to, and the tensors themselves, alive (attribute _keep)."""
    n = len(g_alpha)
    assert len(S) == n and len(weights) == n and (g_beta is None or len(g_beta) == n)
    ga = (ctypes.c_void_p * n)(*[t.data_ptr() for t in g_alpha])
    gb = None
    if g_beta is not None:
        gb = (ctypes.c_void_p * n)(*[(t.data_ptr() if t is not None else None) for t in g_beta])
    Sp = (ctypes.c_void_p * n)(*[t.data_ptr() for t in S])
    w = (ctypes.c_float * n)(*[float(x) for x in weights])
    wph = ctypes.c_void_p(weights_per_head.data_ptr()) if weights_per_head is not None else None
    m = DslaMulti(n, int(H_kv), ctypes.cast(ga, ctypes.POINTER(ctypes.c_void_p)),
                  ctypes.cast(gb, ctypes.POINTER(ctypes.c_void_p)) if gb is not None else None,
                  ctypes.cast(Sp, ctypes.POINTER(ctypes.c_void_p)), ctypes.cast(w, ctypes.POINTER(ctypes.c_float)), wph)
    m._keep = (ga, gb, Sp, w, list(g_alpha), list(g_beta) if g_beta is not None else None, list(S), weights_per_head)
    return m


def dsla_decode_multi(desc: DslaDesc, multi: DslaMulti, q, k, v, o):
    """One decode step of a layer with N states (include/dsla.h: dsla_decode_multi)."""
    _check(load_library().dsla_decode_multi(ctypes.byref(desc), ctypes.byref(multi), _ptr(q), _ptr(k), _ptr(v), _ptr(o),
                                            _stream()))


def dsla_prefill_multi_workspace_bytes(desc: DslaDesc, multi: DslaMulti, T: int) -> int:
    return int(load_library().dsla_prefill_multi_workspace_bytes(ctypes.byref(desc), ctypes.byref(multi), int(T)))


def dsla_prefill_multi(desc: DslaDesc, multi: DslaMulti, T, q, k, v, o, workspace=None):
    """Prefill of a layer with N states (include/dsla.h: dsla_prefill_multi)."""
    wbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load_library().dsla_prefill_multi(ctypes.byref(desc), ctypes.byref(multi), int(T), _ptr(q), _ptr(k), _ptr(v),
                                             _ptr(o), _ptr(workspace), wbytes, _stream()))


def dsla_attention_entropy_workspace_bytes(B: int, H: int, d: int, T: int) -> int:
    return int(load_library().dsla_attention_entropy_workspace_bytes(int(B), int(H), int(d), int(T)))


def dsla_attention_entropy(q_last, k, entropy, scale: float, workspace=None):
    """Entropy of the final query's attention row (include/dsla.h: dsla_attention_entropy).
    q_last [B,H,d], k [B,T,H,d] (bf16 or fp32 GPU tensors), entropy [B,H] fp32, written."""
    B, T, H, d = k.shape
    wbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load_library().dsla_attention_entropy(int(B), int(H), int(d), int(T), _dtype_code(k), float(scale),
                                                 _ptr(q_last), _ptr(k), _ptr(entropy), _ptr(workspace), wbytes,
                                                 _stream()))


def dsla_attention_decode_workspace_bytes(B: int, H: int, d: int, T: int) -> int:
    return int(load_library().dsla_attention_decode_workspace_bytes(int(B), int(H), int(d), int(T)))


def dsla_attention_decode(q, k, v, o, scale: float, workspace=None, seq_lens=None):
    """Single-query softmax attention over cached keys and values (include/dsla.h: dsla_attention_decode).
    q, o [B,H,d]; k, v [B,T,H,d] (all bf16 or all fp32 GPU tensors); seq_lens: int32 GPU tensor [B] or None."""
    lib = _lib or load_library()
    status = _native.attention_decode(q, k, v, o, scale, workspace, seq_lens)
    if status is not None:
        return _check(status)
    B, T, H, d = k.shape
    wbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib.dsla_attention_decode(int(B), int(H), int(d), int(T), _dtype_code(k), float(scale),
                                                _ptr(q), _ptr(k), _ptr(v), _ptr(seq_lens), _ptr(o), _ptr(workspace), wbytes,
                                                _stream()))


def dsla_project(x, W, outs, bias=None):
    """The projections in front of a layer as one GEMM (include/dsla.h: dsla_project).  x [M,K] bf16; W [n_out*width,K]
    bf16; outs: list of n_out bf16 GPU tensors of M*width elements each; bias: fp32 GPU tensor [n_out*width] or None."""
    lib = _lib or load_library()
    status = _native.project(x, W, outs, bias)
    if status is not None:
        return _check(status)
    M, K = x.shape
    n_out = len(outs)
    width = W.shape[0] // n_out
    assert W.shape == (n_out * width, K) and all(t.numel() == M * width for t in outs)
    po = (ctypes.c_void_p * n_out)(*[t.data_ptr() for t in outs])
    for t in outs:
        assert t.is_cuda and t.is_contiguous()
    _check(lib.dsla_project(int(M), int(K), n_out, int(width), _ptr(x), _ptr(W), _ptr(bias), po, _stream()))


def dsla_attention_prefill(q, k, v, o, scale: float):
    """Causal softmax attention over a prompt (include/dsla.h: dsla_attention_prefill).  q, k, v, o: [B,T,H,d] bf16."""
    lib = _lib or load_library()
    status = _native.attention_prefill(q, k, v, o, scale)
    if status is not None:
        return _check(status)
    B, T, H, d = q.shape
    _check(lib.dsla_attention_prefill(int(B), int(H), int(d), int(T), _dtype_code(q), float(scale), _ptr(q),
                                                 _ptr(k), _ptr(v), _ptr(o), _stream()))


def _here(t, dtype, numel=None, optional=False):
    """Pointer of a contiguous tensor on the current device, of that type and number of elements."""
    if t is None:
        if optional:
            return None
        raise ValueError("a required tensor is None")
    p = _ptr(t)
    if t.dtype != dtype:
        raise TypeError(f"{t.dtype} in the place of {dtype}")
    if numel is not None and t.numel() != numel:
        raise ValueError(f"{t.numel()} elements in the place of {numel}")
    if t.get_device() != _torch._cuda_getDevice():
        raise ValueError(f"a tensor of device {t.get_device()}, and the current one is {_torch._cuda_getDevice()}")
    return p


def _same_device(*structures):
    """Structures are for the device that their tensors are on."""
    here = _torch._cuda_getDevice()
    for x in structures:
        if getattr(x, "device", here) != here:
            raise ValueError(f"a structure for device {x.device}, and the current one is {here}")


def _io_dtype(code):
    import torch
    return torch.bfloat16 if code == DSLA_BF16 else torch.float32


def make_cache(table, lens, refs, *, page, H_kv, d, dtype, status=None) -> DslaCache:
    """dsla_cache from int32 GPU tensors: table [n_seqs, max_pages], lens [n_seqs], refs [n_pages], status [1] or None.  dtype:
    DSLA_F32 or DSLA_BF16, the type of the pools.  The structure keeps the tensors alive."""
    import torch
    load_library()
    n_seqs, max_pages = table.shape
    c = DslaCache(int(refs.numel()), int(page), int(H_kv), int(d), int(dtype), int(n_seqs), int(max_pages), _here(table, torch.int32),
                  _here(lens, torch.int32, n_seqs), _here(refs, torch.int32), _here(status, torch.int32, 1, optional=True))
    c._keep, c.device = (table, lens, refs, status), table.get_device()
    return c


def make_batch(start, total, *, cu=None, row=None, max_n=1) -> DslaBatch:
    """dsla_batch from int32 GPU tensors: start [B], cu [B + 1] or None (one token each), row [B] or None.  max_n: an upper bound of the
    tokens of an entry.  The structure keeps the tensors alive."""
    import torch
    load_library()
    B = start.numel()
    x = DslaBatch(int(B), int(max_n), int(total), _here(cu, torch.int32, B + 1, optional=True), _here(row, torch.int32, B, optional=True),
                  _here(start, torch.int32))
    x._keep, x.device = (start, cu, row), start.get_device()
    return x


class Pools:
    """The pools of a cache as the calls take them; keeps the tensors alive."""

    def __init__(self, tensors):
        self.tensors = list(tensors)
        for t in self.tensors:
            _here(t, t.dtype)
        self.array = (ctypes.c_void_p * max(1, len(self.tensors)))(*[t.data_ptr() for t in self.tensors])
        if self.tensors:
            self.device = _torch._cuda_getDevice()
        self.address, self.sizes = ctypes.addressof(self.array), {(t.numel(), t.dtype) for t in self.tensors}

    def of(self, cache: DslaCache):
        """Number and array, for a cache that they are pools of."""
        want = {(cache.n_pages * cache.H_kv * cache.page * cache.d, _io_dtype(cache.dtype))}
        if not self.sizes <= want:
            raise ValueError(f"pools of {self.sizes}, the cache's are of {want}")
        return len(self.tensors), self.array


def make_pools(tensors) -> Pools:
    """From a list of GPU tensors [n_pages, H_kv, page, d]: keys and values of every layer that shares a cache's table."""
    load_library()
    return Pools(tensors)


def _scratch(workspace):
    return (None, 0) if workspace is None else (_here(workspace, workspace.dtype), workspace.numel() * workspace.element_size())


def dsla_cache_workspace_bytes(cache: DslaCache, B: int) -> int:
    return int(load_library().dsla_cache_workspace_bytes(ctypes.byref(cache), int(B)))


def dsla_cache_init(cache: DslaCache):
    """All pages free, all sequences empty (include/dsla.h: dsla_cache_init)."""
    lib = _lib or load_library()
    _same_device(cache)
    _check(lib.dsla_cache_init(ctypes.byref(cache), _stream()))


def dsla_cache_extend(cache: DslaCache, batch: DslaBatch, pools: Pools, workspace):
    """Room for the tokens of every entry at the end of its sequence (include/dsla.h: dsla_cache_extend)."""
    lib, (n, array) = _lib or load_library(), pools.of(cache)
    _same_device(cache, batch, pools)
    status = _native.cache_extend(cache, batch, n, pools.address, workspace)
    if status is not None:
        return _check(status)
    _check(lib.dsla_cache_extend(ctypes.byref(cache), ctypes.byref(batch), n, array, *_scratch(workspace), _stream()))


def dsla_cache_fork(cache: DslaCache, parent):
    """Sequences that share the pages of others (include/dsla.h: dsla_cache_fork).  parent: int32 GPU tensor [n_seqs]."""
    lib = _lib or load_library()
    _same_device(cache)
    status = _native.cache_fork(cache, parent)
    if status is not None:
        return _check(status)
    import torch
    _check(lib.dsla_cache_fork(ctypes.byref(cache), _here(parent, torch.int32, cache.n_seqs), _stream()))


def dsla_cache_truncate(cache: DslaCache, new_lens):
    """Sequences cut to their first tokens, or ended (include/dsla.h: dsla_cache_truncate).  new_lens: int32 GPU tensor [n_seqs]."""
    lib = _lib or load_library()
    _same_device(cache)
    status = _native.cache_truncate(cache, new_lens)
    if status is not None:
        return _check(status)
    import torch
    _check(lib.dsla_cache_truncate(ctypes.byref(cache), _here(new_lens, torch.int32, cache.n_seqs), _stream()))


def dsla_cache_accept(cache: DslaCache, batch: DslaBatch, path, n_accepted, pools: Pools, workspace):
    """Keeps the accepted tokens of every entry (include/dsla.h: dsla_cache_accept).  path: int32 GPU tensor [total], n_accepted [B]."""
    lib, (n, array) = _lib or load_library(), pools.of(cache)
    _same_device(cache, batch, pools)
    status = _native.cache_accept(cache, batch, path, n_accepted, n, pools.address, workspace)
    if status is not None:
        return _check(status)
    import torch
    _check(lib.dsla_cache_accept(ctypes.byref(cache), ctypes.byref(batch), _here(path, torch.int32, batch.total), _here(n_accepted, torch.int32, batch.B),
                                 n, array, *_scratch(workspace), _stream()))


def dsla_cache_compact(cache: DslaCache, n_live, pools: Pools, workspace):
    """Pages in use to the front of the pools (include/dsla.h: dsla_cache_compact).  n_live: int32 GPU tensor [1], written."""
    lib, (n, array) = _lib or load_library(), pools.of(cache)
    _same_device(cache, pools)
    status = _native.cache_compact(cache, n_live, n, pools.address, workspace)
    if status is not None:
        return _check(status)
    import torch
    _check(lib.dsla_cache_compact(ctypes.byref(cache), _here(n_live, torch.int32, 1), n, array, *_scratch(workspace), _stream()))


def make_rope(H, H_kv, d, *, io_dtype, inv_freq=None, interleaved=False, q_weight=None, k_weight=None, eps=1e-6, offsets=None) -> DslaRope:
    """dsla_rope: inv_freq fp32 GPU tensor [rot_dim / 2] or None (nothing rotated), q_weight and k_weight fp32 [d] or None (no norm), offsets
    int32 [total] or None.  The structure keeps the tensors alive."""
    import torch
    load_library()
    r = DslaRope(int(H), int(H_kv), int(d), int(io_dtype), 0 if inv_freq is None else 2 * inv_freq.numel(), int(bool(interleaved)), float(eps),
                 _here(inv_freq, torch.float32, optional=True), _here(q_weight, torch.float32, d, optional=True),
                 _here(k_weight, torch.float32, d, optional=True), _here(offsets, torch.int32, optional=True))
    r._keep = (inv_freq, q_weight, k_weight, offsets)
    if any(t is not None for t in r._keep):
        r.device = _torch._cuda_getDevice()
    return r


def dsla_qk_rope(rope: DslaRope, q, k, v, q_out, k_out=None, cache: DslaCache = None, batch: DslaBatch = None, k_pages=None, v_pages=None):
    """Norm and rotation of q and k, keys and values into their pages (include/dsla.h: dsla_qk_rope).  q, q_out [total, H, d];
    k, v, k_out [total, H_kv, d]; k_pages, v_pages [n_pages, H_kv, page, d]."""
    lib, total = _lib or load_library(), q.shape[0]
    if rope.offsets and rope._keep[3].numel() != total:
        raise ValueError(f"{rope._keep[3].numel()} offsets for {total} tokens")
    _same_device(rope, cache, batch)
    status = _native.qk_rope(rope, total, q, k, v, q_out, k_out, cache, batch, k_pages, v_pages)
    if status is not None:
        return _check(status)
    dtype, nq, nk = _io_dtype(rope.io_dtype), total * rope.H * rope.d, total * rope.H_kv * rope.d
    pool = None if cache is None else cache.n_pages * cache.H_kv * cache.page * cache.d
    _check(lib.dsla_qk_rope(ctypes.byref(rope), int(total), _here(q, dtype, nq), _here(k, dtype, nk), _here(v, dtype, nk, optional=True),
                            _here(q_out, dtype, nq), _here(k_out, dtype, nk, optional=True),
                            None if cache is None else ctypes.byref(cache), None if batch is None else ctypes.byref(batch),
                            _here(k_pages, dtype, pool, optional=True), _here(v_pages, dtype, pool, optional=True), _stream()))


def dsla_attention_paged_workspace_bytes(cache: DslaCache, batch: DslaBatch, H: int, max_len: int) -> int:
    return int(load_library().dsla_attention_paged_workspace_bytes(ctypes.byref(cache), ctypes.byref(batch), int(H), int(max_len)))


def dsla_attention_paged(cache: DslaCache, batch: DslaBatch, q, k_pages, v_pages, o, scale: float, max_len: int, tree=None, workspace=None):
    """Attention of the last tokens of every sequence over a paged cache (include/dsla.h: dsla_attention_paged).  q, o [total, H, d];
    k_pages, v_pages [n_pages, H_kv, page, d]; tree: int64 GPU tensor [total] (its bits) or None."""
    lib = _lib or load_library()
    _same_device(cache, batch)
    status = _native.attention_paged(cache, batch, q, k_pages, v_pages, o, scale, max_len, tree, workspace)
    if status is not None:
        return _check(status)
    import torch
    dtype, pool = _io_dtype(cache.dtype), cache.n_pages * cache.H_kv * cache.page * cache.d
    H, n = q.shape[1], batch.total * q.shape[1] * cache.d
    _check(lib.dsla_attention_paged(ctypes.byref(cache), ctypes.byref(batch), int(H), int(max_len), float(scale), _here(q, dtype, n),
                                               _here(k_pages, dtype, pool), _here(v_pages, dtype, pool),
                                               _here(tree, torch.int64, batch.total, optional=True), _here(o, dtype, n), *_scratch(workspace), _stream()))


def scale_pitch(cols: int) -> int:
    """Scales of a row of an e4m3 tensor (include/dsla.h: DSLA_SCALE_PITCH)."""
    return (int(cols) + 511) // 512 * 4


def _result_dtype(code):
    import torch
    return torch.float8_e4m3fn if code == DSLA_E4M3 else _io_dtype(code)


def _scale_dtype(code):
    import torch
    return torch.float8_e8m0fnu if code == DSLA_SCALE_E8M0 else torch.float32


def _scale_code(t):
    import torch
    if t.dtype not in (torch.float32, torch.float8_e8m0fnu):
        raise TypeError(f"scales of {t.dtype}")
    return DSLA_SCALE_F32 if t.dtype == torch.float32 else DSLA_SCALE_E8M0


def make_norm(D, *, x_dtype, y_dtype, h_dtype, scale_type=DSLA_SCALE_E8M0, gate_act=DSLA_ACT_NONE, eps=1e-6, residual_scale=1.0, post_weight=None,
              pre_weight=None) -> DslaNorm:
    """dsla_norm: post_weight, pre_weight fp32 GPU tensors [D] or None (no norm).  The structure keeps the tensors alive."""
    import torch
    load_library()
    n = DslaNorm(int(D), int(x_dtype), int(y_dtype), int(h_dtype), int(scale_type), int(gate_act), float(eps), float(residual_scale),
                 _here(post_weight, torch.float32, D, optional=True), _here(pre_weight, torch.float32, D, optional=True))
    n._keep = (post_weight, pre_weight)
    if any(t is not None for t in n._keep):
        n.device = _torch._cuda_getDevice()
    return n


def dsla_residual_norm(norm: DslaNorm, x, y, x_out, h, gate=None, h_scale=None):
    """Residual, gate, scale and norms of a block's border (include/dsla.h: dsla_residual_norm).  x, x_out, y, gate, h: [rows, D]; y, x_out or h,
    gate may be None.  h e4m3: h_scale [rows, scale_pitch(D)], float32 or float8_e8m0fnu."""
    lib = _lib or load_library()
    _same_device(norm)
    status = _native.residual_norm(norm, x, y, gate, x_out, h, h_scale)
    if status is not None:
        return _check(status)
    n, D = x.numel(), max(1, norm.D)
    rows = n // D
    _check(lib.dsla_residual_norm(ctypes.byref(norm), rows, _here(x, _io_dtype(norm.x_dtype), rows * D), _here(y, _io_dtype(norm.y_dtype), n, optional=True),
                                  _here(gate, _io_dtype(norm.y_dtype), n, optional=True), _here(x_out, _io_dtype(norm.x_dtype), n, optional=True),
                                  _here(h, _result_dtype(norm.h_dtype), n, optional=True),
                                  _here(h_scale, _scale_dtype(norm.scale_type), rows * scale_pitch(D), optional=True), _stream()))


def make_head_norm(H, d, *, io_dtype, out_dtype, scale_type=DSLA_SCALE_E8M0, gate_act=DSLA_ACT_SILU, eps=1e-6, weight=None) -> DslaHeads:
    """dsla_heads: weight fp32 GPU tensor [d] or None (no norm).  The structure keeps the tensor alive."""
    import torch
    load_library()
    x = DslaHeads(int(H), int(d), int(io_dtype), int(out_dtype), int(scale_type), int(gate_act), float(eps), _here(weight, torch.float32, d, optional=True))
    x._keep = (weight,)
    if weight is not None:
        x.device = _torch._cuda_getDevice()
    return x


def dsla_head_norm(heads: DslaHeads, o, out, gate=None, out_scale=None):
    """Norm and gate of every head (include/dsla.h: dsla_head_norm).  o, gate [rows, H, d]; out [rows, H * d]; out e4m3: out_scale [rows,
    scale_pitch(H * d)], float32 or float8_e8m0fnu."""
    lib = _lib or load_library()
    _same_device(heads)
    status = _native.head_norm(heads, o, gate, out, out_scale)
    if status is not None:
        return _check(status)
    n, W = o.numel(), max(1, heads.H * heads.d)
    rows = n // W
    _check(lib.dsla_head_norm(ctypes.byref(heads), rows, _here(o, _io_dtype(heads.io_dtype), rows * W), _here(gate, _io_dtype(heads.io_dtype), n, optional=True),
                              _here(out, _result_dtype(heads.out_dtype), n), _here(out_scale, _scale_dtype(heads.scale_type), rows * scale_pitch(W), optional=True),
                              _stream()))


def dsla_quantize(x, q, scale, block_rows: int = 1):
    """e4m3 values with block scales (include/dsla.h: dsla_quantize).  x [rows, cols] bf16 or fp32, q the same in float8_e4m3fn, scale [rows or
    ceil(rows / 128), scale_pitch(cols)] float32 or float8_e8m0fnu.  block_rows: 1 or 128."""
    lib = _lib or load_library()
    status = _native.quantize(x, q, scale, block_rows)
    if status is not None:
        return _check(status)
    import torch
    rows, cols = x.shape
    n = -(-rows // max(1, int(block_rows))) * scale_pitch(cols)
    _check(lib.dsla_quantize(int(rows), int(cols), _dtype_code(x), int(block_rows), _scale_code(scale), _here(x, x.dtype),
                             _here(q, torch.float8_e4m3fn, rows * cols), _here(scale, scale.dtype, n), _stream()))


def dsla_project_fp8(x, x_scale, W, W_scale, outs, bias=None):
    """The projections as one product of e4m3 operands with block scales (include/dsla.h: dsla_project_fp8).  x [M, K], W [sum of widths, K]
    float8_e4m3fn, their scales as dsla_quantize leaves them; outs: list of bf16 or fp32 GPU tensors [M, width]; bias: fp32 GPU tensor or None."""
    lib = _lib or load_library()
    status = _native.project_fp8(x, x_scale, W, W_scale, outs, bias)
    if status is not None:
        return _check(status)
    import torch
    M, K = x.shape
    if not outs:
        raise ValueError("no outputs")
    dtype = outs[0].dtype
    if any(t.dim() != 2 or t.shape[0] != M or t.shape[1] > 1 << 24 for t in outs):
        raise ValueError("outputs are [M, width], of up to 2^24 columns")
    n_out, code, widths = len(outs), _dtype_code(outs[0]), [t.shape[1] for t in outs]
    N = sum(widths)
    if W.dim() != 2 or W.shape[1] != K:
        raise ValueError(f"weights of {tuple(W.shape)} for rows of {K}")
    P = scale_pitch(K)
    po = (ctypes.c_void_p * n_out)(*[_here(t, dtype) for t in outs])
    _check(lib.dsla_project_fp8(int(M), int(K), n_out, (ctypes.c_int32 * n_out)(*widths), _scale_code(x_scale), _here(x, torch.float8_e4m3fn),
                                _here(x_scale, x_scale.dtype, M * P), _here(W, torch.float8_e4m3fn, N * K),
                                _here(W_scale, x_scale.dtype, sum(-(-w // 128) for w in widths) * P), _here(bias, torch.float32, N, optional=True),
                                code, po, _stream()))


PLAN_REASONS = ("no pressure", "memory relief", "quality limit", "all converted")


def dsla_rank_layers(sensitivity) -> list:
    """Layer indices in ascending order of sensitivity (include/dsla.h: dsla_rank_layers)."""
    n = len(sensitivity)
    s = (ctypes.c_float * n)(*[float(x) for x in sensitivity])
    order = (ctypes.c_int32 * n)()
    _check(load_library().dsla_rank_layers(n, s, order))
    return list(order)


def dsla_max_conversion_rate(prompt_len: int) -> float:
    return float(load_library().dsla_max_conversion_rate(int(prompt_len)))


def dsla_kv_cache_bytes(n_layers, batch, context, heads, d_head, bytes_per_element) -> int:
    return int(load_library().dsla_kv_cache_bytes(int(n_layers), int(batch), int(context), int(heads), int(d_head),
                                                  int(bytes_per_element)))


def dsla_conversion_plan(order, memory_used, memory_threshold, kv_bytes_per_layer, state_bytes_per_layer, max_rate):
    """Returns (converted layer indices in conversion order, memory use afterwards, reason text)
    (include/dsla.h: dsla_conversion_plan)."""
    n = len(order)
    o = (ctypes.c_int32 * n)(*[int(x) for x in order])
    conv = (ctypes.c_uint8 * n)()
    cnt, after, why = ctypes.c_int32(), ctypes.c_int64(), ctypes.c_int32()
    _check(load_library().dsla_conversion_plan(n, o, int(memory_used), int(memory_threshold), int(kv_bytes_per_layer),
                                               int(state_bytes_per_layer), float(max_rate), conv, ctypes.byref(cnt),
                                               ctypes.byref(after), ctypes.byref(why)))
    layers = [l for l in order if conv[l]]
    assert len(layers) == cnt.value
    return layers, int(after.value), PLAN_REASONS[why.value]


def profile_enable(enable: bool, max_records: int = 4096):
    _check(load_library().dsla_profile_enable(1 if enable else 0, int(max_records)))


def profile_collect() -> dict:
    """Returns {kernel name: (total milliseconds, launches)} since the last collect."""
    n = len(KERNEL_NAMES)
    ms = (ctypes.c_double * n)()
    cnt = (ctypes.c_int64 * n)()
    _check(load_library().dsla_profile_collect(ms, cnt))
    return {KERNEL_NAMES[i]: (float(ms[i]), int(cnt[i])) for i in range(n)}
