"""Thin ctypes binding over liblaser.so: argument marshalling only.

Every function has the name of the C entry point it calls (include/laser.h).
Tensors are PyTorch device tensors used purely as owners of HBM allocations; the
current torch stream is handed to the library. There is no fallback: if the
shared library is missing or an entry point reports an error, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblaser.so")

LASER_F32, LASER_BF16 = 0, 1
STA_AUTO, STA_GENERIC, STA_MFMA, STA_STREAM, STA_MFMA_CACHED = 0, 1, 2, 3, 4
GSTA_AUTO, GSTA_GENERIC, GSTA_TILED, GSTA_SPLIT, GSTA_ONE = 0, 1, 2, 3, 4
FFN_AUTO, FFN_GENERIC, FFN_MFMA = 0, 1, 2
PROJECT_AUTO, PROJECT_GENERIC, PROJECT_MFMA = 0, 1, 2
ROTARY_HALF, ROTARY_INTERLEAVED = 0, 1
ROTARY_NONE, ROTARY_LINEAR, ROTARY_BASE, ROTARY_PARTS = 0, 1, 2, 3

EXPORTS = [
    "laser_sta_forward", "laser_sta_forward_variant", "laser_sta_forward_heads", "laser_sta_forward_softmax", "laser_sta_forward_ragged",
    "laser_gsta_forward_ragged", "laser_forward_ragged", "laser_multires_forward_ragged",
    "laser_segment_ffn_forward_ragged", "laser_gsta_forward", "laser_gsta_forward_variant",
    "laser_forward", "laser_forward_fused", "laser_forward_fused_work_bytes", "laser_multires_forward", "laser_forward_multires", "laser_gsta_forward_multires",
    "laser_sta_kernel_name",
    "laser_gsta_kernel_name", "laser_segment_ffn_forward", "laser_segment_ffn_forward_variant", "laser_ffn_gsta_forward", "laser_ffn_gsta_forward_multires",
    "laser_gsta_kernel_name_layers", "laser_project_q_forward", "laser_project_q_forward_variant",
    "laser_project_kv_forward", "laser_project_kv_forward_variant", "laser_fold_query_weights",
    "laser_project_heads_forward", "laser_sta_folded_forward", "laser_sta_backward", "laser_sta_backward_bf16", "laser_sta_backward_static", "laser_sta_backward_work_bytes", "laser_gsta_backward",
    "laser_gsta_backward_work_bytes",
    "laser_history_attention_forward", "laser_history_attention_backward", "laser_history_attention_backward_work_bytes",
    "laser_cache_append", "laser_cache_attention_forward", "laser_cache_attention_work_bytes", "laser_cache_weights", "laser_cache_evict",
    "laser_rotary_frequencies", "laser_rotary_forward", "laser_rotary_backward",
    "laser_cache8_append", "laser_cache8_attention_forward", "laser_cache8_attention_work_bytes",
    "laser_pages_work_bytes", "laser_pages_grow", "laser_pages_fork", "laser_pages_free", "laser_pages_compact", "laser_pages_copy",
    "laser_status_string", "laser_version",
]


class LaserError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {status_string(code)} (status {code})")


_lib = None


def load_library() -> ctypes.CDLL:
    """dlopen liblaser.so (built by paper_2602_11562_amd.build) and declare the prototypes."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2602_11562_amd.build` "
                          "(there is no CPU or PyTorch fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    lib.forward_address = ctypes.cast(lib.laser_forward, ctypes.c_void_p).value
    vp, ip, i32, f32 = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_float
    lib.laser_sta_forward.argtypes = [vp, vp, vp, ip, i32, i32, i32, i32, i32, i32, f32, i32, vp, ip, vp]
    lib.laser_sta_forward_variant.argtypes = lib.laser_sta_forward.argtypes + [i32]
    lib.laser_sta_forward_heads.argtypes = [vp, vp, vp, ip, i32, i32, i32, i32, i32, i32, f32, i32, i32, vp, ip, vp, i32]
    lib.laser_sta_forward_heads.restype = i32
    lib.laser_sta_forward_softmax.argtypes = lib.laser_sta_forward_heads.argtypes
    lib.laser_sta_forward_softmax.restype = i32
    lib.laser_gsta_forward.argtypes = [vp, vp, vp, vp, vp, ip, i32, i32, i32, i32, i32, i32, i32, vp, vp]
    lib.laser_gsta_forward_variant.argtypes = lib.laser_gsta_forward.argtypes + [i32]
    lib.laser_forward.argtypes = [vp, vp, vp, vp, vp, vp, vp, ip, i32, i32, i32, i32, i32, i32, f32, i32, i32,
                                  vp, ip, vp, vp]
    lib.laser_forward_fused.argtypes = [vp, vp, vp, vp, vp, vp, vp, ip, i32, i32, i32, i32, i32, i32, f32, i32,
                                        ip, vp, vp, ctypes.c_size_t, vp]
    lib.laser_forward_fused.restype = i32
    lib.laser_forward_fused_work_bytes.argtypes = [i32, i32, i32, i32, i32, i32, i32]
    lib.laser_forward_fused_work_bytes.restype = ctypes.c_size_t
    for name in ("laser_sta_forward", "laser_sta_forward_variant", "laser_gsta_forward",
                 "laser_gsta_forward_variant", "laser_forward", "laser_version"):
        getattr(lib, name).restype = i32
    lib.laser_multires_forward.argtypes = [vp, ip, i32, i32, i32, i32, i32, i32, i32, vp, vp, vp]
    lib.laser_multires_forward.restype = i32
    lib.laser_forward_multires.argtypes = lib.laser_forward.argtypes[:-1] + [i32, vp, vp, vp]
    lib.laser_forward_multires.restype = i32
    lib.laser_gsta_forward_multires.argtypes = lib.laser_gsta_forward.argtypes[:-1] + [i32, vp, vp, vp]
    lib.laser_gsta_forward_multires.restype = i32
    fp = ctypes.c_void_p
    lib.laser_segment_ffn_forward.argtypes = [vp, ip, vp, fp, vp, fp, fp, fp, i32, i32, i32, i32, i32, i32, f32, i32,
                                              vp, vp]
    lib.laser_segment_ffn_forward.restype = i32
    lib.laser_segment_ffn_forward_variant.argtypes = lib.laser_segment_ffn_forward.argtypes + [i32]
    lib.laser_segment_ffn_forward_variant.restype = i32
    lib.laser_ffn_gsta_forward.argtypes = [vp, vp, vp, vp, vp, ip, vp, fp, vp, fp, fp, fp, i32, i32, i32, i32, i32, i32,
                                           i32, f32, i32, vp, vp, vp]
    lib.laser_ffn_gsta_forward.restype = i32
    lib.laser_ffn_gsta_forward_multires.argtypes = lib.laser_ffn_gsta_forward.argtypes[:-1] + [i32, vp, vp, vp]
    lib.laser_ffn_gsta_forward_multires.restype = i32
    lib.laser_project_q_forward.argtypes = [vp, vp, i32, i32, i32, i32, i32, vp, vp]
    lib.laser_project_q_forward_variant.argtypes = lib.laser_project_q_forward.argtypes + [i32]
    lib.laser_project_kv_forward.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, vp, vp]
    lib.laser_project_kv_forward_variant.argtypes = lib.laser_project_kv_forward.argtypes + [i32]
    for name in ("laser_project_q_forward", "laser_project_q_forward_variant", "laser_project_kv_forward",
                 "laser_project_kv_forward_variant"):
        getattr(lib, name).restype = i32
    lib.laser_fold_query_weights.argtypes = [vp, vp, i32, i32, i32, i32, vp, vp]
    lib.laser_project_heads_forward.argtypes = [vp, vp, i32, i32, i32, i32, i32, i32, vp, vp, i32]
    lib.laser_sta_folded_forward.argtypes = [vp, vp, vp, vp, ip, i32, i32, i32, i32, i32, i32, f32, i32, i32,
                                             vp, vp, vp, ip, vp]
    for name in ("laser_fold_query_weights", "laser_project_heads_forward", "laser_sta_folded_forward"):
        getattr(lib, name).restype = i32
    lib.laser_sta_forward_ragged.argtypes = [vp, vp, vp, ip, ip, i32, i32, i32, i32, i32, i32, i32, f32, i32, vp, ip, vp]
    lib.laser_gsta_forward_ragged.argtypes = [vp, vp, vp, vp, vp, ip, ip, i32, i32, i32, i32, i32, i32, i32, i32, vp, vp]
    lib.laser_forward_ragged.argtypes = [vp, vp, vp, vp, vp, vp, vp, ip, ip, i32, i32, i32, i32, i32, i32, i32, f32,
                                         i32, i32, vp, ip, vp, vp]
    lib.laser_multires_forward_ragged.argtypes = [vp, ip, ip, i32, i32, i32, i32, i32, i32, i32, i32, vp, vp, vp]
    lib.laser_segment_ffn_forward_ragged.argtypes = [vp, ip, ip, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32,
                                                     i32, f32, i32, vp, vp]
    for name in ("laser_sta_forward_ragged", "laser_gsta_forward_ragged", "laser_forward_ragged",
                 "laser_multires_forward_ragged", "laser_segment_ffn_forward_ragged"):
        getattr(lib, name).restype = i32
    lib.laser_sta_backward_work_bytes.argtypes = [i32, i32, i32, i32, i32]
    lib.laser_sta_backward_work_bytes.restype = ctypes.c_size_t
    lib.laser_sta_backward.argtypes = [vp, vp, vp, ip, vp, i32, i32, i32, i32, i32, i32, f32, i32, vp, vp, vp, vp,
                                       ctypes.c_size_t, vp]
    lib.laser_sta_backward.restype = i32
    lib.laser_sta_backward_bf16.argtypes = [vp, vp, vp, ip, vp, i32, i32, i32, i32, i32, i32, f32, vp, vp, vp, vp,
                                            ctypes.c_size_t, vp]
    lib.laser_sta_backward_bf16.restype = i32
    lib.laser_sta_backward_static.argtypes = [vp, vp, vp, ip, vp, i32, i32, i32, i32, i32, i32, f32, i32, vp, vp, vp, vp]
    lib.laser_sta_backward_static.restype = i32
    lib.laser_gsta_backward_work_bytes.argtypes = [i32, i32, i32, i32]
    lib.laser_gsta_backward_work_bytes.restype = ctypes.c_size_t
    lib.laser_gsta_backward.argtypes = [vp, vp, vp, vp, vp, ip, vp, i32, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp,
                                        vp, ctypes.c_size_t, vp]
    lib.laser_gsta_backward.restype = i32
    i64, sz = ctypes.c_int64, ctypes.c_size_t
    rows3 = [vp, i64, vp, i64, vp, i64]
    lib.laser_history_attention_forward.argtypes = rows3 + [ip] + [i32] * 6 + [f32, i32, vp, vp, vp]
    lib.laser_history_attention_backward.argtypes = rows3 + [vp, vp, vp, ip] + [i32] * 6 + [f32, i32] + rows3 + [vp, sz, vp]
    lib.laser_cache_append.argtypes = [vp, i64, vp, i64, vp, vp, ip, ip, ip] + [i32] * 9 + [i32, vp, vp]
    lib.laser_cache_attention_forward.argtypes = [vp, i64, vp, vp, ip, ip, ip] + [i32] * 10 + [f32, i32, i32, vp, vp, vp, sz, vp]
    lib.laser_cache_weights.argtypes = [vp, i64, vp, vp, ip, ip, ip] + [i32] * 10 + [f32, i32, i32, i32, vp, vp]
    lib.laser_cache_evict.argtypes = [vp, vp, vp, ip, ip, ip] + [i32] * 11 + [ip, ip, vp]
    for name in ("laser_history_attention_forward", "laser_history_attention_backward", "laser_cache_append",
                 "laser_cache_attention_forward", "laser_cache_weights", "laser_cache_evict"):
        getattr(lib, name).restype = i32
    lib.laser_history_attention_backward_work_bytes.argtypes = [i32] * 7
    lib.laser_cache_attention_work_bytes.argtypes = [i32] * 8
    f64 = ctypes.c_double
    lib.laser_rotary_frequencies.argtypes = [i32, f64, i32, f64, f64, f64, f64, vp, vp]
    lib.laser_rotary_forward.argtypes = [vp, i64, vp, i64, ip, vp] + [i32] * 6 + [f32, i32, vp, i64, vp, i64, vp]
    lib.laser_rotary_backward.argtypes = lib.laser_rotary_forward.argtypes
    lib.laser_cache8_append.argtypes = [vp, i64, vp, i64, vp, vp, vp, vp, ip, ip, ip] + [i32] * 11 + [vp]
    lib.laser_cache8_attention_forward.argtypes = ([vp, i64, vp, vp, vp, vp, ip, ip, ip] + [i32] * 11 +
                                                   [f32, i32, i32, vp, vp, vp, sz, vp])
    lib.laser_pages_copy.argtypes = [vp, vp, i32, ip, ip, i32, i32, vp]
    lib.laser_pages_grow.argtypes = [ip, ip, ip, ip, i32, i32, i32, i32, ip, vp, sz, vp]
    lib.laser_pages_fork.argtypes = [vp, vp, i32, ip, ip, ip, ip] + [i32] * 6 + [ip, ip, ip, vp, sz, vp]
    lib.laser_pages_free.argtypes = [ip, ip, ip, ip, i32, i32, i32, i32, vp]
    lib.laser_pages_compact.argtypes = [vp, vp, i32, ip, ip, ip, i32, i32, i32, i32, ip, ip, ip, vp, sz, vp]
    for name in ("laser_rotary_frequencies", "laser_rotary_forward", "laser_rotary_backward", "laser_cache8_append",
                 "laser_cache8_attention_forward", "laser_pages_copy", "laser_pages_grow", "laser_pages_fork", "laser_pages_free",
                 "laser_pages_compact"):
        getattr(lib, name).restype = i32
    lib.laser_cache8_attention_work_bytes.argtypes = [i32] * 8
    lib.laser_pages_work_bytes.argtypes = [i32] * 2
    for name in ("laser_history_attention_backward_work_bytes", "laser_cache_attention_work_bytes",
                 "laser_cache8_attention_work_bytes", "laser_pages_work_bytes"):
        getattr(lib, name).restype = sz
    lib.laser_sta_kernel_name.argtypes = [i32, i32, i32, i32, i32]
    lib.laser_sta_kernel_name.restype = ctypes.c_char_p
    lib.laser_gsta_kernel_name.argtypes = [i32, i32, i32, i32]
    lib.laser_gsta_kernel_name.restype = ctypes.c_char_p
    lib.laser_gsta_kernel_name_layers.argtypes = [i32, i32, i32, i32, i32]
    lib.laser_gsta_kernel_name_layers.restype = ctypes.c_char_p
    lib.laser_status_string.argtypes = [i32]
    lib.laser_status_string.restype = ctypes.c_char_p
    _lib = lib
    return lib


def status_string(code: int) -> str:
    return load_library().laser_status_string(int(code)).decode()


def laser_version() -> int:
    return int(load_library().laser_version())


def laser_sta_kernel_name(C: int, d_q: int, d: int, w: int, dt: int) -> str:
    return load_library().laser_sta_kernel_name(C, d_q, d, w, dt).decode()


def laser_gsta_kernel_name(C: int, S: int, d: int, dt: int, M: int = 1) -> str:
    return load_library().laser_gsta_kernel_name_layers(C, S, d, M, dt).decode()


# ----------------------------------------------------------------------------- tensor marshalling
# A small request is a few microseconds of kernels: what every call does here is kept to attribute reads (the torch module is
# looked up once, the stream's handle is read without building a Stream object, 3.0 -> 0.3 us), and laser_forward, the call of single
# requests, is handed over in native code where every output is given and every tensor is a plain contiguous device tensor (16
# candidates, L = 1024, 8 us of kernels: passes in a row 10.5 -> 8.5 us). Without outputs, and at every other entry point, the host part
# is the one below.
_torch_module = None
_fast_module = None     # None: not looked for yet; False: not there, or not of this torch


def torch_stamp() -> str:
    """The torch and the Python that laser_fast.so, which reads their objects through inlined accessors, has to be built against."""
    import sysconfig
    torch = _torch()
    return f"{torch.__version__} {getattr(torch.version, 'git_version', '')} {sysconfig.get_config_var('SOABI')}"


def _fast():
    """The native marshalling (csrc/binding_fast.cpp), or False: its calls then go the way of every other."""
    global _fast_module
    if _fast_module is None:
        import importlib
        _torch()     # (its libraries are the module's)
        try:
            found = importlib.import_module(".laser_fast", __package__)
            _fast_module = found if getattr(found, "stamp", None) == torch_stamp() else False
        except ImportError:
            _fast_module = False
    return _fast_module


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _dt(t) -> int:
    torch = _torch()
    if t.dtype == torch.float32:
        return LASER_F32
    if t.dtype == torch.bfloat16:
        return LASER_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _ptr(t, name: str, dtype=None) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must live in device memory")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is not None:
        return stream.cuda_stream or None
    core = _torch()._C     # handle of the current device's current stream
    try:
        return core._cuda_getCurrentRawStream(core._cuda_getDevice()) or None
    except AttributeError:     # a torch without these two, which are not of its documented interface
        return _torch().cuda.current_stream().cuda_stream or None


def _check(code: int, where: str) -> None:
    if code != 0:
        raise LaserError(code, where)


def laser_sta_forward(q, k, v, lens, w: int, gamma: float, seg_out=None, seg_cnt=None, stream=None,
                      variant: int = STA_AUTO, want_cnt: bool = True, heads: int = 1, softmax: bool = False):
    """q [U,C,d_q], k [U,L,d_q], v [U,L,d], lens int32 [U] or None -> (H' [U,C,S,d], cnt [U,S] or None).
    heads > 1 calls laser_sta_forward_heads (head h owns the h-th run of columns of q, k, v and H'); softmax=True
    calls laser_sta_forward_softmax (softmax over a segment's valid items instead of sigmoid gates)."""
    torch = _torch()
    U, C, d_q = q.shape
    L, d = v.shape[1], v.shape[2]
    if k.shape != (U, L, d_q) or v.shape[0] != U:
        raise ValueError("q, k, v shapes disagree")
    if k.dtype != q.dtype or v.dtype != q.dtype:
        raise TypeError("q, k, v must share a dtype")
    S = -(-L // w)
    if seg_out is None:
        seg_out = torch.empty((U, C, S, d), dtype=q.dtype, device=q.device)
    elif tuple(seg_out.shape) != (U, C, S, d) or seg_out.dtype != q.dtype:
        raise ValueError("seg_out must be [U,C,S,d] in the input dtype")
    if seg_cnt is None and want_cnt:
        seg_cnt = torch.empty((U, S), dtype=torch.int32, device=q.device)
    if lens is not None and tuple(lens.shape) != (U,):
        raise ValueError("lens must be [U]")
    if softmax or int(heads) != 1:
        fn = load_library().laser_sta_forward_softmax if softmax else load_library().laser_sta_forward_heads
        code = fn(
            _ptr(q, "q"), _ptr(k, "k"), _ptr(v, "v"), _ptr(lens, "lens", torch.int32), U, C, L, d_q, d, int(w),
            float(gamma), int(heads), _dt(q), _ptr(seg_out, "seg_out"), _ptr(seg_cnt, "seg_cnt", torch.int32),
            _stream(stream), int(variant))
        _check(code, "laser_sta_forward_softmax" if softmax else "laser_sta_forward_heads")
        return seg_out, seg_cnt
    code = load_library().laser_sta_forward_variant(
        _ptr(q, "q"), _ptr(k, "k"), _ptr(v, "v"), _ptr(lens, "lens", torch.int32), U, C, L, d_q, d, int(w),
        float(gamma), _dt(q), _ptr(seg_out, "seg_out"), _ptr(seg_cnt, "seg_cnt", torch.int32), _stream(stream),
        int(variant))
    _check(code, "laser_sta_forward")
    return seg_out, seg_cnt


def laser_gsta_forward(seg, t0, wq, wk, wv, lens, L: int, w: int, z_out=None, stream=None,
                       variant: int = GSTA_AUTO):
    """seg [U,C,S,d], t0 [U,C,d], w* [M,d,d], lens int32 [U] or None -> z [U,C,d] fp32."""
    torch = _torch()
    U, C, S, d = seg.shape
    M = wq.shape[0]
    if S != -(-L // w):
        raise ValueError("seg.shape[2] must be ceil(L / w)")
    if tuple(t0.shape) != (U, C, d) or any(tuple(x.shape) != (M, d, d) for x in (wq, wk, wv)):
        raise ValueError("t0 / weight shapes disagree with seg")
    if any(x.dtype != seg.dtype for x in (t0, wq, wk, wv)):
        raise TypeError("seg, t0 and the weights must share a dtype")
    if z_out is None:
        z_out = torch.empty((U, C, d), dtype=torch.float32, device=seg.device)
    code = load_library().laser_gsta_forward_variant(
        _ptr(seg, "seg"), _ptr(t0, "t0"), _ptr(wq, "wq"), _ptr(wk, "wk"), _ptr(wv, "wv"),
        _ptr(lens, "lens", torch.int32), U, C, int(L), d, int(w), M, _dt(seg), _ptr(z_out, "z_out", torch.float32),
        _stream(stream), int(variant))
    _check(code, "laser_gsta_forward")
    return z_out


def laser_segment_ffn_forward(seg, lens, w1, b1, w2, b2, ln_g, ln_b, L: int, w: int, eps: float = 1e-5, seg_out=None,
                              stream=None, variant: int = FFN_AUTO):
    """seg [U,C,S,d] -> LN(FFN(seg) + seg) [U,C,S,d] (same dtype); w1 [d,d_ff], w2 [d_ff,d] in seg's dtype, the rest fp32.
    seg_out may be seg itself."""
    torch = _torch()
    U, C, S, d = seg.shape
    d_ff = w1.shape[1]
    if S != -(-L // w):
        raise ValueError("seg.shape[2] must be ceil(L / w)")
    if tuple(w1.shape) != (d, d_ff) or tuple(w2.shape) != (d_ff, d):
        raise ValueError("w1 must be [d, d_ff] and w2 [d_ff, d]")
    if tuple(b1.shape) != (d_ff,) or any(tuple(x.shape) != (d,) for x in (b2, ln_g, ln_b)):
        raise ValueError("b1 must be [d_ff]; b2, ln_g, ln_b must be [d]")
    if w1.dtype != seg.dtype or w2.dtype != seg.dtype:
        raise TypeError("w1 and w2 must have the dtype of seg")
    if seg_out is None:
        seg_out = torch.empty_like(seg)
    code = load_library().laser_segment_ffn_forward_variant(
        _ptr(seg, "seg"), _ptr(lens, "lens", torch.int32), _ptr(w1, "w1"), _ptr(b1, "b1", torch.float32),
        _ptr(w2, "w2"), _ptr(b2, "b2", torch.float32), _ptr(ln_g, "ln_g", torch.float32),
        _ptr(ln_b, "ln_b", torch.float32), U, C, int(L), d, d_ff, int(w), float(eps), _dt(seg),
        _ptr(seg_out, "seg_out", seg.dtype), _stream(stream), int(variant))
    _check(code, "laser_segment_ffn_forward")
    return seg_out


def laser_project_q_forward(t, w_q, q_out=None, stream=None, variant: int = PROJECT_AUTO):
    """Q = t W_q: t [U,C,d_in], w_q [d_in,d_q] (same dtype) -> [U,C,d_q]."""
    torch = _torch()
    U, C, d_in = t.shape
    if w_q.dim() != 2 or w_q.shape[0] != d_in:
        raise ValueError("w_q must be [d_in, d_q]")
    if w_q.dtype != t.dtype:
        raise TypeError("w_q must have the dtype of t")
    d_q = w_q.shape[1]
    if q_out is None:
        q_out = torch.empty((U, C, d_q), dtype=t.dtype, device=t.device)
    elif tuple(q_out.shape) != (U, C, d_q):
        raise ValueError("q_out must be [U, C, d_q]")
    code = load_library().laser_project_q_forward_variant(
        _ptr(t, "t"), _ptr(w_q, "w_q"), U, C, d_in, d_q, _dt(t), _ptr(q_out, "q_out", t.dtype), _stream(stream),
        int(variant))
    _check(code, "laser_project_q_forward")
    return q_out


def laser_project_kv_forward(h, w_k, w_v, k_out=None, v_out=None, stream=None, variant: int = PROJECT_AUTO):
    """K = H W_k, V = H W_v from one pass over h [U,L,d_in]: w_k [d_in,d_q], w_v [d_in,d] -> ([U,L,d_q], [U,L,d])."""
    torch = _torch()
    U, L, d_in = h.shape
    if w_k.dim() != 2 or w_v.dim() != 2 or w_k.shape[0] != d_in or w_v.shape[0] != d_in:
        raise ValueError("w_k must be [d_in, d_q] and w_v [d_in, d]")
    if w_k.dtype != h.dtype or w_v.dtype != h.dtype:
        raise TypeError("w_k and w_v must have the dtype of h")
    d_q, d = w_k.shape[1], w_v.shape[1]
    if k_out is None:
        k_out = torch.empty((U, L, d_q), dtype=h.dtype, device=h.device)
    elif tuple(k_out.shape) != (U, L, d_q):
        raise ValueError("k_out must be [U, L, d_q]")
    if v_out is None:
        v_out = torch.empty((U, L, d), dtype=h.dtype, device=h.device)
    elif tuple(v_out.shape) != (U, L, d):
        raise ValueError("v_out must be [U, L, d]")
    code = load_library().laser_project_kv_forward_variant(
        _ptr(h, "h"), _ptr(w_k, "w_k"), _ptr(w_v, "w_v"), U, L, d_in, d_q, d, _dt(h), _ptr(k_out, "k_out", h.dtype),
        _ptr(v_out, "v_out", h.dtype), _stream(stream), int(variant))
    _check(code, "laser_project_kv_forward")
    return k_out, v_out


def laser_forward_ragged(q, k, v, t0, wq, wk, wv, lens, cand_off, c_max: int, w: int, gamma: float, seg_out=None,
                         seg_cnt=None, z_out=None, stream=None, want_cnt: bool = True, stage: str = "both"):
    """Packed pairs: q [P,d_q], t0 [P,d] with cand_off int32 [U+1] (device) -> (H' [P,S,d], cnt [U,S], z [P,d] fp32).
    stage = "sta" runs STA only (t0 and the weights may be None, z is None), "gsta" runs GSTA only on seg_out."""
    torch = _torch()
    U, L = k.shape[0], k.shape[1]
    P = q.shape[0] if q is not None else seg_out.shape[0]
    d = v.shape[2]
    S = -(-L // w)
    if tuple(cand_off.shape) != (U + 1,):
        raise ValueError("cand_off must be [U + 1]")
    dev, tdt = k.device, k.dtype
    if seg_out is None:
        seg_out = torch.empty((P, S, d), dtype=tdt, device=dev)
    if seg_cnt is None and want_cnt and stage != "gsta":
        seg_cnt = torch.empty((U, S), dtype=torch.int32, device=dev)
    if z_out is None and stage != "sta":
        z_out = torch.empty((P, d), dtype=torch.float32, device=dev)
    lib = load_library()
    common = (_ptr(lens, "lens", torch.int32), _ptr(cand_off, "cand_off", torch.int32), U, int(c_max), P, L)
    if stage == "sta":
        code = lib.laser_sta_forward_ragged(_ptr(q, "q"), _ptr(k, "k"), _ptr(v, "v"), *common, q.shape[1], d, int(w),
                                            float(gamma), _dt(k), _ptr(seg_out, "seg_out", tdt),
                                            _ptr(seg_cnt, "seg_cnt", torch.int32), _stream(stream))
    elif stage == "gsta":
        code = lib.laser_gsta_forward_ragged(_ptr(seg_out, "seg_out"), _ptr(t0, "t0"), _ptr(wq, "wq"), _ptr(wk, "wk"),
                                             _ptr(wv, "wv"), *common, d, int(w), wq.shape[0], _dt(k),
                                             _ptr(z_out, "z_out", torch.float32), _stream(stream))
    else:
        code = lib.laser_forward_ragged(_ptr(q, "q"), _ptr(k, "k"), _ptr(v, "v"), _ptr(t0, "t0"), _ptr(wq, "wq"),
                                        _ptr(wk, "wk"), _ptr(wv, "wv"), *common, q.shape[1], d, int(w), float(gamma),
                                        wq.shape[0], _dt(k), _ptr(seg_out, "seg_out", tdt),
                                        _ptr(seg_cnt, "seg_cnt", torch.int32), _ptr(z_out, "z_out", torch.float32),
                                        _stream(stream))
    _check(code, "laser_forward_ragged")
    return seg_out, seg_cnt, z_out


def laser_sta_backward(q, k, v, lens, dseg, w: int, gamma: float, dq_out=None, dk_out=None, dv_out=None, work=None,
                       stream=None, grads_bf16: bool = False):
    """Gradients of STA: dseg = dL/dH' [U,C,S,d] (dtype of q) -> (dq [U,C,d_q], dk [U,L,d_q], dv [U,L,d]) in fp32;
    with grads_bf16 (bf16 inputs) dk and dv come back in bf16 (laser_sta_backward_bf16)."""
    torch = _torch()
    U, C, d_q = q.shape
    L, d = v.shape[1], v.shape[2]
    S = -(-L // w)
    if tuple(k.shape) != (U, L, d_q) or tuple(v.shape) != (U, L, d) or tuple(dseg.shape) != (U, C, S, d):
        raise ValueError("q, k, v, dseg shapes disagree")
    if any(x.dtype != q.dtype for x in (k, v, dseg)):
        raise TypeError("q, k, v and dseg must share a dtype")
    f32 = dict(dtype=torch.float32, device=q.device)
    dq_out = torch.empty((U, C, d_q), **f32) if dq_out is None else dq_out
    gkw = dict(dtype=torch.bfloat16, device=q.device) if grads_bf16 else f32
    dk_out = torch.empty((U, L, d_q), **gkw) if dk_out is None else dk_out
    dv_out = torch.empty((U, L, d), **gkw) if dv_out is None else dv_out
    lib = load_library()
    need = lib.laser_sta_backward_work_bytes(U, C, L, d_q, int(w))
    if work is None:
        work = torch.empty(max(need, 16), dtype=torch.uint8, device=q.device)
    if grads_bf16:
        if q.dtype != torch.bfloat16:
            raise TypeError("grads_bf16 needs bf16 inputs")
        code = lib.laser_sta_backward_bf16(_ptr(q, "q"), _ptr(k, "k"), _ptr(v, "v"), _ptr(lens, "lens", torch.int32),
                                           _ptr(dseg, "dseg"), U, C, L, d_q, d, int(w), float(gamma),
                                           _ptr(dq_out, "dq_out", torch.float32),
                                           _ptr(dk_out, "dk_out", torch.bfloat16),
                                           _ptr(dv_out, "dv_out", torch.bfloat16), _ptr(work, "work"),
                                           work.numel() * work.element_size(), _stream(stream))
        _check(code, "laser_sta_backward_bf16")
        return dq_out, dk_out, dv_out
    code = lib.laser_sta_backward(_ptr(q, "q"), _ptr(k, "k"), _ptr(v, "v"), _ptr(lens, "lens", torch.int32),
                                  _ptr(dseg, "dseg"), U, C, L, d_q, d, int(w), float(gamma), _dt(q),
                                  _ptr(dq_out, "dq_out", torch.float32), _ptr(dk_out, "dk_out", torch.float32),
                                  _ptr(dv_out, "dv_out", torch.float32), _ptr(work, "work"),
                                  work.numel() * work.element_size(), _stream(stream))
    _check(code, "laser_sta_backward")
    return dq_out, dk_out, dv_out


STATIC_SCRATCH_BYTES = 8 << 20     # LASER_STATIC_SCRATCH_BYTES of include/laser.h


def laser_sta_backward_static(q, k, v, lens, dseg, w: int, gamma: float, dq_out, dk_out, dv_out, stream=None):
    """laser_sta_backward with the library's own fixed scratch: the call allocates nothing, so the three outputs
    [U,C,d_q], [U,L,d_q], [U,L,d] (fp32) are the caller's."""
    torch = _torch()
    U, C, d_q = q.shape
    L, d = v.shape[1], v.shape[2]
    S = -(-L // w)
    if tuple(k.shape) != (U, L, d_q) or tuple(v.shape) != (U, L, d) or tuple(dseg.shape) != (U, C, S, d):
        raise ValueError("q, k, v, dseg shapes disagree")
    if tuple(dq_out.shape) != (U, C, d_q) or tuple(dk_out.shape) != (U, L, d_q) or tuple(dv_out.shape) != (U, L, d):
        raise ValueError("output shapes disagree with the inputs")
    if any(x.dtype != q.dtype for x in (k, v, dseg)):
        raise TypeError("q, k, v and dseg must share a dtype")
    code = load_library().laser_sta_backward_static(
        _ptr(q, "q"), _ptr(k, "k"), _ptr(v, "v"), _ptr(lens, "lens", torch.int32), _ptr(dseg, "dseg"), U, C, L, d_q, d,
        int(w), float(gamma), _dt(q), _ptr(dq_out, "dq_out", torch.float32), _ptr(dk_out, "dk_out", torch.float32),
        _ptr(dv_out, "dv_out", torch.float32), _stream(stream))
    _check(code, "laser_sta_backward_static")
    return dq_out, dk_out, dv_out


def laser_gsta_backward(seg, t0, wq, wk, wv, lens, dz, L: int, w: int, work=None, stream=None):
    """Gradients of GSTA from dz [U,C,d] fp32: (dseg [U,C,S,d] in seg's dtype, dt0 [U,C,d], dwq, dwk, dwv [M,d,d] fp32)."""
    torch = _torch()
    U, C, S, d = seg.shape
    M = wq.shape[0]
    if S != -(-L // w) or tuple(dz.shape) != (U, C, d) or tuple(t0.shape) != (U, C, d):
        raise ValueError("seg, t0, dz shapes disagree")
    f32 = dict(dtype=torch.float32, device=seg.device)
    dseg = torch.empty_like(seg)
    dt0 = torch.empty((U, C, d), **f32)
    dwq, dwk, dwv = (torch.empty((M, d, d), **f32) for _ in range(3))
    lib = load_library()
    need = lib.laser_gsta_backward_work_bytes(U, C, d, M)
    if work is None:
        work = torch.empty(max(need, 16), dtype=torch.uint8, device=seg.device)
    code = lib.laser_gsta_backward(_ptr(seg, "seg"), _ptr(t0, "t0"), _ptr(wq, "wq"), _ptr(wk, "wk"), _ptr(wv, "wv"),
                                   _ptr(lens, "lens", torch.int32), _ptr(dz, "dz", torch.float32), U, C, int(L), d,
                                   int(w), M, _dt(seg), _ptr(dseg, "dseg"), _ptr(dt0, "dt0"), _ptr(dwq, "dwq"),
                                   _ptr(dwk, "dwk"), _ptr(dwv, "dwv"), _ptr(work, "work"),
                                   work.numel() * work.element_size(), _stream(stream))
    _check(code, "laser_gsta_backward")
    return dseg, dt0, dwq, dwk, dwv


def laser_multires_forward_ragged(seg, lens, cand_off, c_max: int, L: int, w: int, r: int, stream=None):
    """Packed pairs: seg [P,S,d] with cand_off [U+1] -> (pool [P,d], recent [P,r,d] or None)."""
    torch = _torch()
    P, S, d = seg.shape
    U = cand_off.shape[0] - 1
    pool = torch.empty((P, d), dtype=seg.dtype, device=seg.device)
    recent = torch.empty((P, r, d), dtype=seg.dtype, device=seg.device) if r > 0 else None
    code = load_library().laser_multires_forward_ragged(
        _ptr(seg, "seg"), _ptr(lens, "lens", torch.int32), _ptr(cand_off, "cand_off", torch.int32), U, int(c_max), P,
        int(L), d, int(w), int(r), _dt(seg), _ptr(pool, "pool"), _ptr(recent, "recent"), _stream(stream))
    _check(code, "laser_multires_forward_ragged")
    return pool, recent


def laser_segment_ffn_forward_ragged(seg, lens, cand_off, c_max: int, w1, b1, w2, b2, ln_g, ln_b, L: int, w: int,
                                     eps: float = 1e-5, seg_out=None, stream=None):
    """Packed pairs: seg [P,S,d] with cand_off [U+1] -> LN(FFN(seg) + seg) [P,S,d]; seg_out may be seg."""
    torch = _torch()
    P, S, d = seg.shape
    U = cand_off.shape[0] - 1
    if seg_out is None:
        seg_out = torch.empty_like(seg)
    code = load_library().laser_segment_ffn_forward_ragged(
        _ptr(seg, "seg"), _ptr(lens, "lens", torch.int32), _ptr(cand_off, "cand_off", torch.int32), _ptr(w1, "w1"),
        _ptr(b1, "b1", torch.float32), _ptr(w2, "w2"), _ptr(b2, "b2", torch.float32), _ptr(ln_g, "ln_g", torch.float32),
        _ptr(ln_b, "ln_b", torch.float32), U, int(c_max), P, int(L), d, w1.shape[1], int(w), float(eps), _dt(seg),
        _ptr(seg_out, "seg_out", seg.dtype), _stream(stream))
    _check(code, "laser_segment_ffn_forward_ragged")
    return seg_out


def laser_fold_query_weights(w_q, w_k, heads: int = 1, a_out=None, stream=None):
    """A = [W_q,h W_k,h^T for every head] : w_q, w_k [d_in, d_q] -> [d_in, heads * d_in] (same dtype)."""
    torch = _torch()
    d_in, d_q = w_q.shape
    if tuple(w_k.shape) != (d_in, d_q) or w_k.dtype != w_q.dtype:
        raise ValueError("w_q and w_k must both be [d_in, d_q] in one dtype")
    if a_out is None:
        a_out = torch.empty((d_in, heads * d_in), dtype=w_q.dtype, device=w_q.device)
    code = load_library().laser_fold_query_weights(_ptr(w_q, "w_q"), _ptr(w_k, "w_k"), d_in, d_q, int(heads), _dt(w_q),
                                                   _ptr(a_out, "a_out", w_q.dtype), _stream(stream))
    _check(code, "laser_fold_query_weights")
    return a_out


def laser_project_heads_forward(x, w_v, y=None, stream=None, variant: int = PROJECT_AUTO):
    """x [P, heads, S, d_in], w_v [d_in, d] -> y [P, S, d]: head h's columns of w_v applied to x[:, h]."""
    torch = _torch()
    P, heads, S, d_in = x.shape
    if w_v.dim() != 2 or w_v.shape[0] != d_in or w_v.dtype != x.dtype:
        raise ValueError("w_v must be [d_in, d] in the dtype of x")
    d = w_v.shape[1]
    if y is None:
        y = torch.empty((P, S, d), dtype=x.dtype, device=x.device)
    elif tuple(y.shape) != (P, S, d):
        raise ValueError("y must be [P, S, d]")
    code = load_library().laser_project_heads_forward(_ptr(x, "x"), _ptr(w_v, "w_v"), P, S, d_in, d, heads, _dt(x),
                                                      _ptr(y, "y", x.dtype), _stream(stream), int(variant))
    _check(code, "laser_project_heads_forward")
    return y


def laser_sta_folded_forward(t, h, a_fold, w_v, lens, w: int, gamma: float, heads: int = 1, qf_work=None, g_work=None,
                             seg_out=None, seg_cnt=None, stream=None, want_cnt: bool = True):
    """Raw embeddings t [U,C,d_in], h [U,L,d_in] -> (H' [U,C,S,d], cnt [U,S] or None) without forming K and V.
    a_fold comes from laser_fold_query_weights. Pass your own work buffers (qf_work [U,C*heads,d_in],
    g_work [U,C*heads,S,d_in]) to reuse them across calls; otherwise they are allocated here, by torch."""
    torch = _torch()
    U, C, d_in = t.shape
    L = h.shape[1]
    d = w_v.shape[1]
    S = -(-L // w)
    if tuple(h.shape) != (U, L, d_in) or tuple(a_fold.shape) != (d_in, heads * d_in) or w_v.shape[0] != d_in:
        raise ValueError("t, h, a_fold, w_v shapes disagree")
    if any(x.dtype != t.dtype for x in (h, a_fold, w_v)):
        raise TypeError("t, h, a_fold and w_v must share a dtype")
    if qf_work is None:
        qf_work = torch.empty((U, C * heads, d_in), dtype=t.dtype, device=t.device)
    if g_work is None:
        g_work = torch.empty((U, C * heads, S, d_in), dtype=t.dtype, device=t.device)
    if seg_out is None:
        seg_out = torch.empty((U, C, S, d), dtype=t.dtype, device=t.device)
    if seg_cnt is None and want_cnt:
        seg_cnt = torch.empty((U, S), dtype=torch.int32, device=t.device)
    if tuple(qf_work.shape) != (U, C * heads, d_in) or tuple(g_work.shape) != (U, C * heads, S, d_in) or \
            tuple(seg_out.shape) != (U, C, S, d):
        raise ValueError("work / output buffer shapes disagree")
    code = load_library().laser_sta_folded_forward(
        _ptr(t, "t"), _ptr(h, "h"), _ptr(a_fold, "a_fold"), _ptr(w_v, "w_v"), _ptr(lens, "lens", torch.int32), U, C, L,
        d_in, d, int(w), float(gamma), int(heads), _dt(t), _ptr(qf_work, "qf_work", t.dtype),
        _ptr(g_work, "g_work", t.dtype), _ptr(seg_out, "seg_out", t.dtype), _ptr(seg_cnt, "seg_cnt", torch.int32),
        _stream(stream))
    _check(code, "laser_sta_folded_forward")
    return seg_out, seg_cnt


def laser_forward_multires(q, k, v, t0, wq, wk, wv, lens, w: int, gamma: float, r: int, seg_out=None, seg_cnt=None,
                           z_out=None, pool_out=None, recent_out=None, stream=None):
    """The whole path with all three views. Returns (H', cnt, z fp32, pool [U,C,d], recent [U,C,r,d] or None)."""
    torch = _torch()
    U, C, d_q = q.shape
    L, d = v.shape[1], v.shape[2]
    M = wq.shape[0]
    S = -(-L // w)
    if any(x.dtype != q.dtype for x in (k, v, t0, wq, wk, wv)):
        raise TypeError("all inputs must share a dtype")
    if seg_out is None:
        seg_out = torch.empty((U, C, S, d), dtype=q.dtype, device=q.device)
    if seg_cnt is None:
        seg_cnt = torch.empty((U, S), dtype=torch.int32, device=q.device)
    if z_out is None:
        z_out = torch.empty((U, C, d), dtype=torch.float32, device=q.device)
    if pool_out is None:
        pool_out = torch.empty((U, C, d), dtype=q.dtype, device=q.device)
    if recent_out is None and r > 0:
        recent_out = torch.empty((U, C, r, d), dtype=q.dtype, device=q.device)
    for name, x in (("seg_out", seg_out), ("pool_out", pool_out), ("recent_out", recent_out)):
        if x is not None and x.dtype != q.dtype:
            raise TypeError(f"{name} must have the dtype of the inputs")
    code = load_library().laser_forward_multires(
        _ptr(q, "q"), _ptr(k, "k"), _ptr(v, "v"), _ptr(t0, "t0"), _ptr(wq, "wq"), _ptr(wk, "wk"), _ptr(wv, "wv"),
        _ptr(lens, "lens", torch.int32), U, C, L, d_q, d, int(w), float(gamma), M, _dt(q), _ptr(seg_out, "seg_out"),
        _ptr(seg_cnt, "seg_cnt", torch.int32), _ptr(z_out, "z_out", torch.float32), int(r),
        _ptr(pool_out, "pool_out"), _ptr(recent_out, "recent_out"), _stream(stream))
    _check(code, "laser_forward_multires")
    return seg_out, seg_cnt, z_out, pool_out, recent_out


def laser_gsta_forward_multires(seg, t0, wq, wk, wv, lens, L: int, w: int, r: int, z_out=None, pool_out=None,
                                recent_out=None, stream=None):
    """GSTA and the two other views from a stored H' [U,C,S,d]. Returns (z fp32 [U,C,d], pool [U,C,d], recent
    [U,C,r,d] or None)."""
    torch = _torch()
    U, C, S, d = seg.shape
    M = wq.shape[0]
    if S != -(-L // w):
        raise ValueError("seg.shape[2] must be ceil(L / w)")
    if any(x.dtype != seg.dtype for x in (t0, wq, wk, wv)):
        raise TypeError("all inputs must share a dtype")
    if z_out is None:
        z_out = torch.empty((U, C, d), dtype=torch.float32, device=seg.device)
    if pool_out is None:
        pool_out = torch.empty((U, C, d), dtype=seg.dtype, device=seg.device)
    if recent_out is None and r > 0:
        recent_out = torch.empty((U, C, r, d), dtype=seg.dtype, device=seg.device)
    for name, x in (("pool_out", pool_out), ("recent_out", recent_out)):
        if x is not None and x.dtype != seg.dtype:
            raise TypeError(f"{name} must have the dtype of seg")
    code = load_library().laser_gsta_forward_multires(
        _ptr(seg, "seg"), _ptr(t0, "t0"), _ptr(wq, "wq"), _ptr(wk, "wk"), _ptr(wv, "wv"),
        _ptr(lens, "lens", torch.int32), U, C, int(L), d, int(w), M, _dt(seg), _ptr(z_out, "z_out", torch.float32),
        int(r), _ptr(pool_out, "pool_out"), _ptr(recent_out, "recent_out"), _stream(stream))
    _check(code, "laser_gsta_forward_multires")
    return z_out, pool_out, recent_out


def laser_ffn_gsta_forward(seg, t0, wq, wk, wv, lens, w1, b1, w2, b2, ln_g, ln_b, L: int, w: int, eps: float = 1e-5,
                           seg_out=None, z_out=None, stream=None, want_seg: bool = True, r: Optional[int] = None,
                           pool_out=None, recent_out=None):
    """seg [U,C,S,d] -> (s = LN(FFN(seg) + seg) [U,C,S,d] or None, z = GSTA(t0; s) [U,C,d] fp32). want_seg=False
    passes a null seg_out (s is not written); seg_out may be seg itself. With r (an int >= 0) the call is
    laser_ffn_gsta_forward_multires and returns (s or None, z, pool [U,C,d], recent [U,C,r,d] or None)."""
    torch = _torch()
    U, C, S, d = seg.shape
    d_ff = w1.shape[1]
    M = wq.shape[0]
    if S != -(-L // w):
        raise ValueError("seg.shape[2] must be ceil(L / w)")
    if tuple(w1.shape) != (d, d_ff) or tuple(w2.shape) != (d_ff, d):
        raise ValueError("w1 must be [d, d_ff] and w2 [d_ff, d]")
    if tuple(b1.shape) != (d_ff,) or any(tuple(x.shape) != (d,) for x in (b2, ln_g, ln_b)):
        raise ValueError("b1 must be [d_ff]; b2, ln_g, ln_b must be [d]")
    if tuple(t0.shape) != (U, C, d) or any(tuple(x.shape) != (M, d, d) for x in (wq, wk, wv)):
        raise ValueError("t0 / weight shapes disagree with seg")
    if any(x.dtype != seg.dtype for x in (t0, wq, wk, wv, w1, w2)):
        raise TypeError("seg, t0 and the weight matrices must share a dtype")
    if seg_out is None and want_seg:
        seg_out = torch.empty_like(seg)
    if z_out is None:
        z_out = torch.empty((U, C, d), dtype=torch.float32, device=seg.device)
    if r is not None:
        if pool_out is None:
            pool_out = torch.empty((U, C, d), dtype=seg.dtype, device=seg.device)
        if recent_out is None and r > 0:
            recent_out = torch.empty((U, C, r, d), dtype=seg.dtype, device=seg.device)
        code = load_library().laser_ffn_gsta_forward_multires(
            _ptr(seg, "seg"), _ptr(t0, "t0"), _ptr(wq, "wq"), _ptr(wk, "wk"), _ptr(wv, "wv"),
            _ptr(lens, "lens", torch.int32), _ptr(w1, "w1"), _ptr(b1, "b1", torch.float32), _ptr(w2, "w2"),
            _ptr(b2, "b2", torch.float32), _ptr(ln_g, "ln_g", torch.float32), _ptr(ln_b, "ln_b", torch.float32), U, C,
            int(L), d, d_ff, int(w), M, float(eps), _dt(seg), _ptr(seg_out, "seg_out", seg.dtype),
            _ptr(z_out, "z_out", torch.float32), int(r), _ptr(pool_out, "pool_out", seg.dtype),
            _ptr(recent_out, "recent_out", seg.dtype), _stream(stream))
        _check(code, "laser_ffn_gsta_forward_multires")
        return seg_out, z_out, pool_out, recent_out
    code = load_library().laser_ffn_gsta_forward(
        _ptr(seg, "seg"), _ptr(t0, "t0"), _ptr(wq, "wq"), _ptr(wk, "wk"), _ptr(wv, "wv"),
        _ptr(lens, "lens", torch.int32), _ptr(w1, "w1"), _ptr(b1, "b1", torch.float32), _ptr(w2, "w2"),
        _ptr(b2, "b2", torch.float32), _ptr(ln_g, "ln_g", torch.float32), _ptr(ln_b, "ln_b", torch.float32), U, C,
        int(L), d, d_ff, int(w), M, float(eps), _dt(seg), _ptr(seg_out, "seg_out", seg.dtype),
        _ptr(z_out, "z_out", torch.float32), _stream(stream))
    _check(code, "laser_ffn_gsta_forward")
    return seg_out, z_out


def laser_multires_forward(seg, lens, L: int, w: int, r: int, pool_out=None, recent_out=None, stream=None,
                           want_pool: bool = True):
    """seg [U,C,S,d], lens int32 [U] or None -> (pool [U,C,d] or None, recent [U,C,r,d] or None), dtype of seg."""
    torch = _torch()
    U, C, S, d = seg.shape
    if S != -(-L // w):
        raise ValueError("seg.shape[2] must be ceil(L / w)")
    if pool_out is None and want_pool:
        pool_out = torch.empty((U, C, d), dtype=seg.dtype, device=seg.device)
    if recent_out is None and r > 0:
        recent_out = torch.empty((U, C, r, d), dtype=seg.dtype, device=seg.device)
    for name, x in (("pool_out", pool_out), ("recent_out", recent_out)):
        if x is not None and x.dtype != seg.dtype:
            raise TypeError(f"{name} must have the dtype of seg")
    code = load_library().laser_multires_forward(
        _ptr(seg, "seg"), _ptr(lens, "lens", torch.int32), U, C, int(L), d, int(w), int(r), _dt(seg),
        _ptr(pool_out, "pool_out"), _ptr(recent_out, "recent_out"), _stream(stream))
    _check(code, "laser_multires_forward")
    return pool_out, recent_out


def laser_forward_fused(q, k, v, t0, wq, wk, wv, lens, w: int, gamma: float, seg_cnt=None, z_out=None, work=None,
                        stream=None, want_cnt: bool = True, use_work: bool = True):
    """The whole path with one GSTA layer and H' never stored. Returns (cnt [U,S] or None, z [U,C,d] fp32).
    work: device scratch for the partial results of the runs of a history (allocated here when None and use_work);
    use_work=False passes NULL, i.e. one run per user."""
    torch = _torch()
    U, C, d_q = q.shape
    L, d = v.shape[1], v.shape[2]
    S = -(-L // w)
    if tuple(wq.shape[-2:]) != (d, d) or wq.numel() != d * d:
        raise ValueError("one layer: wq, wk, wv must hold d x d elements")
    if seg_cnt is None and want_cnt:
        seg_cnt = torch.empty((U, S), dtype=torch.int32, device=q.device)
    if z_out is None:
        z_out = torch.empty((U, C, d), dtype=torch.float32, device=q.device)
    if any(x.dtype != q.dtype for x in (k, v, t0, wq, wk, wv)):
        raise TypeError("all inputs must share a dtype")
    lib = load_library()
    if work is None and use_work:
        need = lib.laser_forward_fused_work_bytes(U, C, L, d_q, d, int(w), _dt(q))
        if need:
            work = torch.empty(need, dtype=torch.uint8, device=q.device)
    code = lib.laser_forward_fused(
        _ptr(q, "q"), _ptr(k, "k"), _ptr(v, "v"), _ptr(t0, "t0"), _ptr(wq, "wq"), _ptr(wk, "wk"), _ptr(wv, "wv"),
        _ptr(lens, "lens", torch.int32), U, C, L, d_q, d, int(w), float(gamma), _dt(q),
        _ptr(seg_cnt, "seg_cnt", torch.int32), _ptr(z_out, "z_out", torch.float32), _ptr(work, "work"),
        0 if work is None else work.numel() * work.element_size(), _stream(stream))
    _check(code, "laser_forward_fused")
    return seg_cnt, z_out


def laser_forward(q, k, v, t0, wq, wk, wv, lens, w: int, gamma: float, seg_out=None, seg_cnt=None, z_out=None,
                  stream=None, want_cnt: bool = True, want_seg: bool = True):
    """The whole path. Returns (H' [U,C,S,d], cnt [U,S] or None, z [U,C,d] fp32); with want_seg=False seg_out is passed
    as NULL (H' is never stored: the fused kernels, one layer only) and None comes back in its place."""
    torch = _torch()
    if q.is_cuda and seg_out is not None and z_out is not None and (seg_cnt is not None or not want_cnt):
        fast = _fast()
        code = fast.forward(load_library().forward_address, q, k, v, t0, wq, wk, wv, lens, w, gamma, seg_out, seg_cnt, z_out,
                            _stream(stream)) if fast else None
        if code is not None:
            _check(code, "laser_forward")
            return seg_out, seg_cnt, z_out
    U, C, d_q = q.shape
    L, d = v.shape[1], v.shape[2]
    M = wq.shape[0]
    S = -(-L // w)
    if seg_out is None and want_seg:
        seg_out = torch.empty((U, C, S, d), dtype=q.dtype, device=q.device)
    if seg_cnt is None and want_cnt:
        seg_cnt = torch.empty((U, S), dtype=torch.int32, device=q.device)
    if z_out is None:
        z_out = torch.empty((U, C, d), dtype=torch.float32, device=q.device)
    dt = q.dtype
    if k.dtype != dt or v.dtype != dt or t0.dtype != dt or wq.dtype != dt or wk.dtype != dt or wv.dtype != dt or \
            (seg_out is not None and seg_out.dtype != dt):
        raise TypeError("all inputs and seg_out must share a dtype")
    code = load_library().laser_forward(
        _ptr(q, "q"), _ptr(k, "k"), _ptr(v, "v"), _ptr(t0, "t0"), _ptr(wq, "wq"), _ptr(wk, "wk"), _ptr(wv, "wv"),
        _ptr(lens, "lens", torch.int32), U, C, L, d_q, d, int(w), float(gamma), M, _dt(q), _ptr(seg_out, "seg_out"),
        _ptr(seg_cnt, "seg_cnt", torch.int32), _ptr(z_out, "z_out", torch.float32), _stream(stream))
    _check(code, "laser_forward")
    return seg_out, seg_cnt, z_out


# ----------------------------------------------------------------------------- attention among a history's items
# (A small call is a few microseconds of kernels. On the current stream, with every output given, it is handed over in native code;
# any other form goes by Python, which reads each attribute of a tensor once and puts names together for errors only. Measured, by
# Python and so: four heads over 60 items in fp32 8.8 and 6.3 us a call, append, attention and weights of one item 31.8 and 20.9.)
_ADDRESS: dict = {}     # of the entry points, for the native part


def _native(name: str, *args):
    """The call handed over by native code: its status, or None where it is not of the ordinary form."""
    fast = _fast()
    if not fast:
        return None
    entry = _ADDRESS.get(name)
    if entry is None:
        fn = getattr(load_library(), "laser_" + {"history_forward": "history_attention_forward", "history_backward":
                     "history_attention_backward", "cache_attention": "cache_attention_forward", "cache8_attention":
                     "cache8_attention_forward"}.get(name, name))
        entry = _ADDRESS[name] = (getattr(fast, name.replace("rotary_backward", "rotary_forward")), ctypes.cast(fn, ctypes.c_void_p).value)
    core = _torch()._C
    return entry[0](entry[1], core._cuda_getDevice(), *args, _stream(None))


def _one_device(names: str, *tensors) -> int:
    """The index of the device that all of the given tensors live on."""
    index = tensors[0].get_device()
    for t in tensors:
        if t is not None and (t.get_device() != index or index < 0):
            for name, x in zip(names.split(), tensors):
                if x is not None and x.get_device() < 0:
                    raise ValueError(f"{name} must live in device memory")
            raise ValueError(f"{names} must live on one device")
    return index


def _there(index: int, stream, call):
    """call() with the device, and the stream where one is given, current: kernels run there, and what is allocated belongs there."""
    torch = _torch()
    if stream is None and torch._C._cuda_getDevice() == index:
        return call()
    if stream is not None and stream.device_index != index:
        raise ValueError(f"the stream is of device {stream.device_index}, the tensors are on {index}")
    with torch.cuda.device(index):
        if stream is None:
            return call()
        with torch.cuda.stream(stream):
            return call()


def _pitch(t, name: str, shape) -> int:
    """Elements between the tokens of a [tokens, heads, D] tensor of this shape whose heads lie side by side; tokens may be apart."""
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    n, heads, D = shape
    tokens, head, column = t.stride()
    if (column != 1 and D > 1) or (head != D and heads > 1):
        raise ValueError(f"the heads of {name} must lie side by side within a token")
    return tokens if n > 1 else heads * D


def _flat(t, name: str, shape, dtype) -> int:
    """Pointer of a contiguous tensor of this shape and type."""
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _heads_of(t, name: str):
    if t.dim() != 3:
        raise ValueError(f"{name} must be [tokens, heads, D]")
    return t.shape


def _parts_of(off) -> int:
    if off.dim() != 1 or off.shape[0] < 2:
        raise ValueError("off must be [N + 1]")
    return off.shape[0] - 1


def laser_history_attention_forward(q, k, v, off, L_max: int, gamma: float, o_out=None, lse_out=None, stream=None):
    """Causal attention over packed sequences: q [T,H,D], k, v [T,H_kv,D] (column blocks of one tensor will do), off int32 [N+1],
    L_max at least the longest sequence -> (o [T,H,D], lse [T,H] fp32). Rows of no sequence are not written."""
    if stream is None and o_out is not None and lse_out is not None and q.is_cuda:
        code = _native("history_forward", q, k, v, off, L_max, gamma, o_out, lse_out)
        if code is not None:
            _check(code, "laser_history_attention_forward")
            return o_out, lse_out
    torch = _torch()
    index = _one_device("q k v off o_out lse_out", q, k, v, off, o_out, lse_out)
    shape, dtype = _heads_of(q, "q"), q.dtype
    T, H, D = shape
    kv = (T, _heads_of(k, "k")[1], D)
    if k.dtype != dtype or v.dtype != dtype:
        raise TypeError("q, k, v must share a dtype")

    def call():
        o = torch.empty_like(q, memory_format=torch.contiguous_format) if o_out is None else o_out
        lse = torch.empty((T, H), dtype=torch.float32, device=q.device) if lse_out is None else lse_out
        N = _parts_of(off)
        _check(load_library().laser_history_attention_forward(
            q.data_ptr(), _pitch(q, "q", shape), k.data_ptr(), _pitch(k, "k", kv), v.data_ptr(), _pitch(v, "v", kv),
            _flat(off, "off", (N + 1,), torch.int32), N, T, int(L_max), H, kv[1], D, float(gamma), _dt(q),
            _flat(o, "o_out", shape, dtype), _flat(lse, "lse_out", (T, H), torch.float32), _stream(stream)),
            "laser_history_attention_forward")
        return o, lse

    return _there(index, stream, call)


def laser_history_attention_backward_work_bytes(N: int, T: int, L_max: int, H: int, H_kv: int, D: int, dt: int) -> int:
    return load_library().laser_history_attention_backward_work_bytes(N, T, L_max, H, H_kv, D, dt)


def laser_history_attention_backward(q, k, v, o, lse, d_o, off, L_max: int, gamma: float, dq_out=None, dk_out=None,
                                     dv_out=None, work=None, stream=None):
    """Gradients of laser_history_attention_forward: o [T,H,D], lse [T,H] as it returned them, d_o [T,H,D] ->
    (dq [T,H,D], dk [T,H_kv,D], dv [T,H_kv,D]) in the dtype of q. The outputs may be column blocks of one tensor."""
    if stream is None and work is not None and dq_out is not None and dk_out is not None and dv_out is not None and q.is_cuda:
        code = _native("history_backward", q, k, v, o, lse, d_o, off, L_max, gamma, dq_out, dk_out, dv_out, work)
        if code is not None:
            _check(code, "laser_history_attention_backward")
            return dq_out, dk_out, dv_out
    torch = _torch()
    index = _one_device("q k v o lse d_o off dq_out dk_out dv_out work", q, k, v, o, lse, d_o, off, dq_out, dk_out, dv_out, work)
    shape, dtype = _heads_of(q, "q"), q.dtype
    T, H, D = shape
    kv = (T, _heads_of(k, "k")[1], D)
    if k.dtype != dtype or v.dtype != dtype or any(x is not None and x.dtype != dtype for x in (dq_out, dk_out, dv_out)):
        raise TypeError("q, k, v and the gradients must share a dtype")

    def call():
        N, lib = _parts_of(off), load_library()
        dq = torch.empty(shape, dtype=dtype, device=q.device) if dq_out is None else dq_out
        dk = torch.empty(kv, dtype=dtype, device=q.device) if dk_out is None else dk_out
        dv = torch.empty(kv, dtype=dtype, device=q.device) if dv_out is None else dv_out
        room = work
        if room is None:
            need = lib.laser_history_attention_backward_work_bytes(N, T, int(L_max), H, kv[1], D, _dt(q))
            room = torch.empty(max(need, 16), dtype=torch.uint8, device=q.device)
        _check(lib.laser_history_attention_backward(
            q.data_ptr(), _pitch(q, "q", shape), k.data_ptr(), _pitch(k, "k", kv), v.data_ptr(), _pitch(v, "v", kv),
            _flat(o, "o", shape, dtype), _flat(lse, "lse", (T, H), torch.float32), _flat(d_o, "d_o", shape, dtype),
            _flat(off, "off", (N + 1,), torch.int32), N, T, int(L_max), H, kv[1], D, float(gamma), _dt(q),
            dq.data_ptr(), _pitch(dq, "dq_out", shape), dk.data_ptr(), _pitch(dk, "dk_out", kv), dv.data_ptr(),
            _pitch(dv, "dv_out", kv), _ptr(room, "work"), room.numel() * room.element_size(), _stream(stream)),
            "laser_history_attention_backward")
        return dq, dk, dv

    return _there(index, stream, call)


def _cache_of(k_cache, v_cache, pages, lens):
    """(P, H_kv, page, D, U, max_pages) of a paged cache and its table, and the pointers of all four."""
    i32 = _torch().int32
    if k_cache.dim() != 4 or pages.dim() != 2:
        raise ValueError("k_cache and v_cache must be [P, H_kv, page, D], pages [U, max_pages]")
    shape, table = k_cache.shape, pages.shape
    k = _flat(k_cache, "k_cache", shape, k_cache.dtype)
    v = k if v_cache is k_cache else _flat(v_cache, "v_cache", shape, k_cache.dtype)
    return (*shape, *table), k, v, _flat(pages, "pages", table, i32), _flat(lens, "lens", (table[0],), i32)


def laser_cache_append(k, v, k_cache, v_cache, off, pages, lens, C_max: int, L_max: int, weight=None, stream=None):
    """New keys and values [T,H_kv,D], packed by off int32 [U+1] (at most C_max a user), become the last items of each user's
    lens [U] in k_cache, v_cache [P,H_kv,page,D]; pages int32 [U,max_pages]. weight [P,page]: their places are set to 0."""
    if stream is None and k.is_cuda:
        code = _native("cache_append", k, v, k_cache, v_cache, off, pages, lens, C_max, L_max, weight)
        if code is not None:
            _check(code, "laser_cache_append")
            return
    torch = _torch()
    index = _one_device("k v k_cache v_cache off pages lens weight", k, v, k_cache, v_cache, off, pages, lens, weight)
    (P, Hkv, page, D, U, max_pages), kc, vc, table, held = _cache_of(k_cache, v_cache, pages, lens)
    shape = (_heads_of(k, "k")[0], Hkv, D)
    if k.dtype != k_cache.dtype or v.dtype != k_cache.dtype:
        raise TypeError("k, v must have the dtype of the cache")

    def call():
        _check(load_library().laser_cache_append(
            k.data_ptr(), _pitch(k, "k", shape), v.data_ptr(), _pitch(v, "v", shape), kc, vc,
            _flat(off, "off", (U + 1,), torch.int32), table, held, U, shape[0], int(C_max), P, page, max_pages, int(L_max), Hkv, D,
            _dt(k_cache), None if weight is None else _flat(weight, "weight", (P, page), torch.float32), _stream(stream)),
            "laser_cache_append")

    _there(index, stream, call)


def laser_cache_attention_work_bytes(U: int, T: int, C_max: int, L_max: int, H: int, H_kv: int, D: int, dt: int) -> int:
    return load_library().laser_cache_attention_work_bytes(U, T, C_max, L_max, H, H_kv, D, dt)


def laser_cache_attention_forward(q, k_cache, v_cache, off, pages, lens, C_max: int, L_max: int, gamma: float,
                                  causal: bool = True, o_out=None, lse_out=None, work=None, stream=None):
    """Queries [T,H,D], packed by off int32 [U+1] (at most C_max a user), over each user's cached items -> (o [T,H,D], lse [T,H]).
    causal: the queries are those of the cache's last items, each sees the items up to its own; otherwise (candidates) all."""
    if stream is None and o_out is not None and lse_out is not None and work is not None and q.is_cuda:
        code = _native("cache_attention", q, k_cache, v_cache, off, pages, lens, C_max, L_max, gamma, causal, o_out, lse_out, work)
        if code is not None:
            _check(code, "laser_cache_attention_forward")
            return o_out, lse_out
    torch = _torch()
    index = _one_device("q k_cache v_cache off pages lens o_out lse_out work", q, k_cache, v_cache, off, pages, lens, o_out, lse_out,
                        work)
    (P, Hkv, page, D, U, max_pages), kc, vc, table, held = _cache_of(k_cache, v_cache, pages, lens)
    T, H, _ = _heads_of(q, "q")
    shape, dtype = (T, H, D), q.dtype
    if dtype != k_cache.dtype:
        raise TypeError("q must have the dtype of the cache")

    def call():
        lib = load_library()
        o = torch.empty(shape, dtype=dtype, device=q.device) if o_out is None else o_out
        lse = torch.empty((T, H), dtype=torch.float32, device=q.device) if lse_out is None else lse_out
        room = work
        if room is None:
            need = lib.laser_cache_attention_work_bytes(U, T, int(C_max), int(L_max), H, Hkv, D, _dt(q))
            room = torch.empty(max(need, 16), dtype=torch.uint8, device=q.device)
        _check(lib.laser_cache_attention_forward(
            q.data_ptr(), _pitch(q, "q", shape), kc, vc, _flat(off, "off", (U + 1,), torch.int32), table, held, U, T, int(C_max), P,
            page, max_pages, int(L_max), H, Hkv, D, float(gamma), 1 if causal else 0, _dt(q), _flat(o, "o_out", shape, dtype),
            _flat(lse, "lse_out", (T, H), torch.float32), _ptr(room, "work"), room.numel() * room.element_size(), _stream(stream)),
            "laser_cache_attention_forward")
        return o, lse

    return _there(index, stream, call)


def laser_cache_weights(q, lse, k_cache, off, pages, lens, C_max: int, L_max: int, gamma: float, weight, causal: bool = True,
                        add: bool = True, stream=None):
    """What each cached item received from the queries of laser_cache_attention_forward, summed over queries and heads, into
    weight [P,page] fp32 (add: onto what stands there). lse [T,H] as that call returned it. Returns weight."""
    if stream is None and q.is_cuda:
        code = _native("cache_weights", q, lse, k_cache, off, pages, lens, C_max, L_max, gamma, weight, causal, add)
        if code is not None:
            _check(code, "laser_cache_weights")
            return weight
    torch = _torch()
    index = _one_device("q lse k_cache off pages lens weight", q, lse, k_cache, off, pages, lens, weight)
    (P, Hkv, page, D, U, max_pages), kc, _, table, held = _cache_of(k_cache, k_cache, pages, lens)
    T, H, _ = _heads_of(q, "q")
    if q.dtype != k_cache.dtype:
        raise TypeError("q must have the dtype of the cache")

    def call():
        _check(load_library().laser_cache_weights(
            q.data_ptr(), _pitch(q, "q", (T, H, D)), _flat(lse, "lse", (T, H), torch.float32), kc,
            _flat(off, "off", (U + 1,), torch.int32), table, held, U, T, int(C_max), P, page, max_pages, int(L_max), H, Hkv, D,
            float(gamma), 1 if causal else 0, 1 if add else 0, _dt(q), _flat(weight, "weight", (P, page), torch.float32),
            _stream(stream)), "laser_cache_weights")
        return weight

    return _there(index, stream, call)


def laser_cache_evict(k_cache, v_cache, weight, pages, lens, pages_out, budget: int, recent: int, L_max: int, lens_out=None,
                      kept_out=None, stream=None):
    """Each user keeps the `recent` last of its items and the heaviest others by weight [P,page], `budget` in all; they move, in
    order and with their weights, into the pages of pages_out int32 [U,max_pages_out] -> (lens [U], kept [U,budget], the old
    places, -1 behind the last)."""
    if stream is None and lens_out is not None and kept_out is not None and k_cache.is_cuda:
        code = _native("cache_evict", k_cache, v_cache, weight, pages, lens, pages_out, budget, recent, L_max, lens_out, kept_out)
        if code is not None:
            _check(code, "laser_cache_evict")
            return lens_out, kept_out
    torch = _torch()
    index = _one_device("k_cache v_cache weight pages lens pages_out lens_out kept_out", k_cache, v_cache, weight, pages, lens,
                        pages_out, lens_out, kept_out)
    (P, Hkv, page, D, U, max_pages), kc, vc, table, held = _cache_of(k_cache, v_cache, pages, lens)
    budget, i32 = int(budget), torch.int32
    if pages_out.dim() != 2 or pages_out.shape[0] != U:
        raise ValueError("pages_out must be [U, max_pages_out]")

    def call():
        left = torch.empty((U,), dtype=i32, device=lens.device) if lens_out is None else lens_out
        kept = torch.empty((U, max(budget, 0)), dtype=i32, device=lens.device) if kept_out is None else kept_out
        _check(load_library().laser_cache_evict(
            kc, vc, _flat(weight, "weight", (P, page), torch.float32), table, held, _flat(pages_out, "pages_out", pages_out.shape, i32),
            U, P, page, max_pages, pages_out.shape[1], int(L_max), budget, int(recent), Hkv, D, _dt(k_cache),
            _flat(left, "lens_out", (U,), i32), _flat(kept, "kept_out", (U, max(budget, 0)), i32), _stream(stream)),
            "laser_cache_evict")
        return left, kept

    return _there(index, stream, call)


def laser_rotary_frequencies(R: int, base: float = 10000.0, scaling: int = ROTARY_NONE, factor: float = 1.0, length: float = 4096.0,
                             low: float = 1.0, high: float = 32.0, freq_out=None, device=None, stream=None):
    """Angles that a position adds to each of the R / 2 pairs, fp64 [R / 2]; scaling: for contexts `factor` times as long as those of
    training (ROTARY_LINEAR, ROTARY_BASE, ROTARY_PARTS, which looks at the turns within `length` between low and high)."""
    torch = _torch()
    if freq_out is None:
        device = torch.device("cuda" if device is None else device)
        index = torch.cuda.current_device() if device.index is None else device.index
    else:
        index = _one_device("freq_out", freq_out)

    def call():
        freq = torch.empty(max(int(R) // 2, 1), dtype=torch.float64, device=f"cuda:{index}") if freq_out is None else freq_out
        _check(load_library().laser_rotary_frequencies(int(R), float(base), int(scaling), float(factor), float(length), float(low),
                                                       float(high), _flat(freq, "freq_out", (int(R) // 2,), torch.float64),
                                                       _stream(stream)), "laser_rotary_frequencies")
        return freq

    return _there(index, stream, call)


def _rotary(name: str, q, k, pos, freq, layout, scale, q_out, k_out, stream, names):
    if stream is None and q_out is not None and (k is None) == (k_out is None) and q.is_cuda:
        code = _native(name, q, k, pos, freq, layout, scale, q_out, k_out)
        if code is not None:
            _check(code, "laser_" + name)
            return q_out, k_out
    torch = _torch()
    index = _one_device(names, q, k, pos, freq, q_out, k_out)
    words = names.split()
    shape, dtype = _heads_of(q, words[0]), q.dtype
    T, H, D = shape
    kv = None if k is None else (T, _heads_of(k, words[1])[1], D)
    if any(x is not None and x.dtype != dtype for x in (k, q_out, k_out)):
        raise TypeError(f"{words[0]}, {words[1]} and the outputs must share a dtype")
    if k is None and k_out is not None:
        raise ValueError(f"{words[5]} without {words[1]}")
    if freq.dim() != 1:
        raise ValueError("freq must be [R / 2]")

    def call():
        y = torch.empty(shape, dtype=dtype, device=q.device) if q_out is None else q_out
        z = k_out if k is None or k_out is not None else torch.empty(kv, dtype=dtype, device=q.device)
        keys = (None, 0) if k is None else (k.data_ptr(), _pitch(k, words[1], kv))
        _check(getattr(load_library(), "laser_" + name)(
            q.data_ptr(), _pitch(q, words[0], shape), *keys, _flat(pos, "pos", (T,), torch.int32),
            _flat(freq, "freq", freq.shape, torch.float64), T, H, 0 if k is None else kv[1], D, 2 * freq.shape[0], int(layout),
            float(scale), _dt(q), y.data_ptr(), _pitch(y, words[4], shape), None if k is None else z.data_ptr(),
            0 if k is None else _pitch(z, words[5], kv), _stream(stream)), "laser_" + name)
        return y, z

    return _there(index, stream, call)


def laser_rotary_forward(q, k, pos, freq, layout: int = ROTARY_HALF, scale: float = 1.0, q_out=None, k_out=None, stream=None):
    """Queries [T,H,D] and keys [T,H_kv,D] (or None) turned by their positions int32 [T] (negative: the row is left out), pair i by pos *
    freq[i], fp64 [R / 2] -> (q, k). The outputs may be the inputs, or column blocks of one tensor."""
    return _rotary("rotary_forward", q, k, pos, freq, layout, scale, q_out, k_out, stream, "q k pos freq q_out k_out")


def laser_rotary_backward(d_q, d_k, pos, freq, layout: int = ROTARY_HALF, scale: float = 1.0, dq_out=None, dk_out=None, stream=None):
    """Gradients of laser_rotary_forward: of its results -> of its queries and keys."""
    return _rotary("rotary_backward", d_q, d_k, pos, freq, layout, scale, dq_out, dk_out, stream,
                   "d_q d_k pos freq dq_out dk_out")


def _cache8_of(k_cache, v_cache, k_scale, v_scale, pages, lens):
    """(P, H_kv, page, D, U, max_pages), block, and the pointers of all six."""
    torch = _torch()
    if k_cache.dtype not in (torch.float8_e4m3fn, torch.uint8):
        raise TypeError(f"k_cache must be {torch.float8_e4m3fn}, got {k_cache.dtype}")
    sizes, kc, vc, table, held = _cache_of(k_cache, v_cache, pages, lens)
    P, Hkv, page = sizes[:3]
    if k_scale.dim() != 3 or k_scale.shape[:2] != (P, Hkv) or k_scale.shape[2] < 1 or page % k_scale.shape[2]:
        raise ValueError(f"k_scale must be [{P}, {Hkv}, {page} / block], got {list(k_scale.shape)}")
    scales = [_flat(x, name, k_scale.shape, torch.float32) for x, name in ((k_scale, "k_scale"), (v_scale, "v_scale"))]
    return sizes, page // k_scale.shape[2], (kc, vc, *scales), table, held


def laser_cache8_append(k, v, k_cache, v_cache, k_scale, v_scale, off, pages, lens, C_max: int, L_max: int, stream=None):
    """As laser_cache_append into a cache of 8-bit blocks: k_cache, v_cache float8_e4m3fn [P,H_kv,page,D], whose items are their numbers
    times k_scale, v_scale fp32 [P,H_kv,page/block], powers of two that grow where new items ask for it."""
    if stream is None and k.is_cuda:
        code = _native("cache8_append", k, v, k_cache, v_cache, k_scale, v_scale, off, pages, lens, C_max, L_max)
        if code is not None:
            _check(code, "laser_cache8_append")
            return
    torch = _torch()
    index = _one_device("k v k_cache v_cache k_scale v_scale off pages lens", k, v, k_cache, v_cache, k_scale, v_scale, off, pages, lens)
    (P, Hkv, page, D, U, max_pages), block, held, table, n = _cache8_of(k_cache, v_cache, k_scale, v_scale, pages, lens)
    shape = (_heads_of(k, "k")[0], Hkv, D)
    if v.dtype != k.dtype:
        raise TypeError("k, v must share a dtype")

    def call():
        _check(load_library().laser_cache8_append(
            k.data_ptr(), _pitch(k, "k", shape), v.data_ptr(), _pitch(v, "v", shape), *held, _flat(off, "off", (U + 1,), torch.int32),
            table, n, U, shape[0], int(C_max), P, page, block, max_pages, int(L_max), Hkv, D, _dt(k), _stream(stream)),
            "laser_cache8_append")

    _there(index, stream, call)


def laser_cache8_attention_work_bytes(U: int, T: int, C_max: int, L_max: int, H: int, H_kv: int, D: int, dt: int) -> int:
    return load_library().laser_cache8_attention_work_bytes(U, T, C_max, L_max, H, H_kv, D, dt)


def laser_cache8_attention_forward(q, k_cache, v_cache, k_scale, v_scale, off, pages, lens, C_max: int, L_max: int, gamma: float,
                                   causal: bool = True, o_out=None, lse_out=None, work=None, stream=None):
    """As laser_cache_attention_forward over a cache of 8-bit blocks (laser_cache8_append); queries in fp32 or bf16."""
    if stream is None and o_out is not None and lse_out is not None and work is not None and q.is_cuda:
        code = _native("cache8_attention", q, k_cache, v_cache, k_scale, v_scale, off, pages, lens, C_max, L_max, gamma, causal, o_out,
                       lse_out, work)
        if code is not None:
            _check(code, "laser_cache8_attention_forward")
            return o_out, lse_out
    torch = _torch()
    index = _one_device("q k_cache v_cache k_scale v_scale off pages lens o_out lse_out work", q, k_cache, v_cache, k_scale, v_scale, off,
                        pages, lens, o_out, lse_out, work)
    (P, Hkv, page, D, U, max_pages), block, held, table, n = _cache8_of(k_cache, v_cache, k_scale, v_scale, pages, lens)
    T, H, _ = _heads_of(q, "q")
    shape, dtype = (T, H, D), q.dtype

    def call():
        lib = load_library()
        o = torch.empty(shape, dtype=dtype, device=q.device) if o_out is None else o_out
        lse = torch.empty((T, H), dtype=torch.float32, device=q.device) if lse_out is None else lse_out
        room = work
        if room is None:
            need = lib.laser_cache8_attention_work_bytes(U, T, int(C_max), int(L_max), H, Hkv, D, _dt(q))
            room = torch.empty(max(need, 16), dtype=torch.uint8, device=q.device)
        _check(lib.laser_cache8_attention_forward(
            q.data_ptr(), _pitch(q, "q", shape), *held, _flat(off, "off", (U + 1,), torch.int32), table, n, U, T, int(C_max), P, page,
            block, max_pages, int(L_max), H, Hkv, D, float(gamma), 1 if causal else 0, _dt(q), _flat(o, "o_out", shape, dtype),
            _flat(lse, "lse_out", (T, H), torch.float32), _ptr(room, "work"), room.numel() * room.element_size(), _stream(stream)),
            "laser_cache8_attention_forward")
        return o, lse

    return _there(index, stream, call)


def laser_pages_work_bytes(U: int, P: int) -> int:
    """Scratch of the calls below for U users (of the larger side) and a pool of P pages."""
    return load_library().laser_pages_work_bytes(U, P)


def _parts_of_page(parts, P: int):
    """(host array of pointers, host array of bytes a page, how many) of tensors [P, ...]."""
    n = len(parts)
    at, size = (ctypes.c_void_p * max(n, 1))(), (ctypes.c_int64 * max(n, 1))()
    for i, t in enumerate(parts):
        if t.dim() < 1 or t.shape[0] != P:
            raise ValueError(f"parts[{i}] must be [{P}, ...], got {list(t.shape)}")
        at[i], size[i] = _ptr(t, f"parts[{i}]"), t.numel() // max(P, 1) * t.element_size()
    return at, size, n


def _page_tables(pages, lens, refs, device_of):
    """(index of the device, U, max_pages, P, pointers of pages, lens and refs)"""
    i32 = _torch().int32
    if pages.dim() != 2 or refs.dim() != 1:
        raise ValueError("pages must be [U, max_pages], refs [P]")
    index = _one_device(*device_of)
    U, max_pages = pages.shape
    return (index, U, max_pages, refs.shape[0], _flat(pages, "pages", pages.shape, i32), _flat(lens, "lens", (U,), i32),
            _flat(refs, "refs", refs.shape, i32))


def _page_work(work, U: int, P: int, like):
    torch = _torch()
    if work is None:
        work = torch.empty(max(load_library().laser_pages_work_bytes(U, P), 16), dtype=torch.uint8, device=like.device)
    return _ptr(work, "work"), work.numel() * work.element_size(), work


def _names(parts) -> str:
    return " ".join(f"parts[{i}]" for i in range(len(parts)))


def laser_pages_grow(pages, lens, off, refs, page: int, missing_out=None, work=None, stream=None):
    """lens int32 [U] grow by the rows that off int32 [U+1] packs, and the tables pages int32 [U,max_pages] get fresh pages of `page` items for
    them, the lowest free ones of the pool (refs int32 [P]: how many tables name a page). Returns missing [1], the pages that there were none for."""
    if stream is None and missing_out is not None and work is not None and pages.is_cuda:
        code = _native("pages_grow", pages, lens, off, refs, page, missing_out, work)
        if code is not None:
            _check(code, "laser_pages_grow")
            return missing_out
    torch = _torch()
    index, U, max_pages, P, table, n, counts = _page_tables(
        pages, lens, refs, ("pages lens off refs missing_out work", pages, lens, off, refs, missing_out, work))

    def call():
        missing = torch.empty(1, dtype=torch.int32, device=pages.device) if missing_out is None else missing_out
        room, size, keep = _page_work(work, U, P, pages)
        _check(load_library().laser_pages_grow(table, n, _flat(off, "off", (U + 1,), torch.int32), counts, U, P, int(page), max_pages,
                                               _flat(missing, "missing_out", (1,), torch.int32), room, size, _stream(stream)),
               "laser_pages_grow")
        return missing

    return _there(index, stream, call)


def laser_pages_fork(parts, pages, lens, source, refs, page: int, max_pages_out: Optional[int] = None, pages_out=None, lens_out=None,
                     missing_out=None, work=None, stream=None):
    """New tables whose history v is that of user source[v], int32 [V]: whole pages are shared, a partly filled last one is copied, in
    every one of the parts [P, ...], into a fresh page -> (pages_out [V,max_pages_out], lens_out [V])."""
    if (stream is None and max_pages_out is None and pages_out is not None and lens_out is not None and missing_out is not None and
            work is not None and pages.is_cuda):
        code = _native("pages_fork", parts, pages, lens, source, refs, page, pages_out, lens_out, missing_out, work)
        if code is not None:
            _check(code, "laser_pages_fork")
            return pages_out, lens_out
    torch = _torch()
    index, U, max_pages, P, table, n, counts = _page_tables(
        pages, lens, refs, ("pages lens source refs pages_out lens_out missing_out work " + _names(parts), pages, lens, source, refs, pages_out,
                            lens_out, missing_out, work, *parts))
    if source.dim() != 1 or source.shape[0] < 1:
        raise ValueError("source must be [V]")
    if pages_out is not None and pages_out.dim() != 2:
        raise ValueError("pages_out must be [V, max_pages_out]")
    V, i32 = source.shape[0], torch.int32
    most = int(max_pages_out) if max_pages_out is not None else max_pages if pages_out is None else pages_out.shape[1]

    def call():
        to = torch.empty((V, most), dtype=i32, device=pages.device) if pages_out is None else pages_out
        left = torch.empty((V,), dtype=i32, device=pages.device) if lens_out is None else lens_out
        missing = torch.empty(1, dtype=i32, device=pages.device) if missing_out is None else missing_out
        room, size, keep = _page_work(work, max(U, V), P, pages)
        _check(load_library().laser_pages_fork(
            *_parts_of_page(parts, P), table, n, _flat(source, "source", (V,), i32), counts, U, V, P, int(page), max_pages, most,
            _flat(to, "pages_out", (V, most), i32), _flat(left, "lens_out", (V,), i32), _flat(missing, "missing_out", (1,), i32), room,
            size, _stream(stream)), "laser_pages_fork")
        return to, left

    return _there(index, stream, call)


def laser_pages_free(pages, lens, gone, refs, page: int, stream=None):
    """Users with gone int32 [U] != 0 (None: all) give their pages back and have no items any more."""
    if stream is None and pages.is_cuda:
        code = _native("pages_free", pages, lens, gone, refs, page)
        if code is not None:
            _check(code, "laser_pages_free")
            return
    torch = _torch()
    index, U, max_pages, P, table, n, counts = _page_tables(pages, lens, refs, ("pages lens gone refs", pages, lens, gone, refs))

    def call():
        _check(load_library().laser_pages_free(table, n, None if gone is None else _flat(gone, "gone", (U,), torch.int32), counts, U, P,
                                               int(page), max_pages, _stream(stream)), "laser_pages_free")

    _there(index, stream, call)


def laser_pages_compact(parts, pages, lens, refs, page: int, pages_out=None, refs_out=None, in_use_out=None, work=None, stream=None):
    """The pages in use become the first ones of the pool, in every one of the parts [P, ...] -> (pages [U,max_pages] and refs [P] with the
    new numbers, in_use [1])."""
    if stream is None and pages_out is not None and refs_out is not None and in_use_out is not None and work is not None and pages.is_cuda:
        code = _native("pages_compact", parts, pages, lens, refs, page, pages_out, refs_out, in_use_out, work)
        if code is not None:
            _check(code, "laser_pages_compact")
            return pages_out, refs_out, in_use_out
    torch = _torch()
    index, U, max_pages, P, table, n, counts = _page_tables(
        pages, lens, refs, ("pages lens refs pages_out refs_out in_use_out work " + _names(parts), pages, lens, refs, pages_out, refs_out,
                            in_use_out, work, *parts))
    i32 = torch.int32

    def call():
        to = torch.empty_like(pages) if pages_out is None else pages_out
        counts_to = torch.empty_like(refs) if refs_out is None else refs_out
        used = torch.empty(1, dtype=i32, device=pages.device) if in_use_out is None else in_use_out
        room, size, keep = _page_work(work, U, P, pages)
        _check(load_library().laser_pages_compact(
            *_parts_of_page(parts, P), table, n, counts, U, P, int(page), max_pages, _flat(to, "pages_out", (U, max_pages), i32),
            _flat(counts_to, "refs_out", (P,), i32), _flat(used, "in_use_out", (1,), i32), room, size, _stream(stream)),
            "laser_pages_compact")
        return to, counts_to, used

    return _there(index, stream, call)


def laser_pages_copy(parts, source, target, stream=None):
    """Page target[i] becomes a copy of page source[i], int32 [n], in every one of the parts [P, ...]."""
    torch = _torch()
    if len(parts) == 0:
        raise ValueError("there must be parts to copy")
    index = _one_device("source target " + _names(parts), source, target, *parts)
    if source.dim() != 1 or source.shape[0] < 1:
        raise ValueError("source must be [n]")

    def call():
        n, P, i32 = source.shape[0], parts[0].shape[0], torch.int32
        _check(load_library().laser_pages_copy(*_parts_of_page(parts, P), _flat(source, "source", (n,), i32),
                                               _flat(target, "target", (n,), i32), n, P, _stream(stream)), "laser_pages_copy")

    _there(index, stream, call)
