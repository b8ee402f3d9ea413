"""ctypes binding of libvidkv.so: same names as the C ABI, argument marshalling only.

Every step of the path runs in the library's HIP kernels; this module checks
tensor dtype / device / contiguity, takes data pointers and the current
stream, and turns a non-zero status into an exception.  If the library has not
been built the first call raises: there is no fallback.  The calls that are made
once per layer go through vidkv_marshal.so (csrc/marshal.cpp), which does the same
natively for plain tensors that pass the checks and leaves everything else to
this module; where it is missing or was built for another Python or torch, this
module takes every call.
"""
from __future__ import annotations

import ctypes as C
import logging
import math
import os
import sys

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libvidkv.so")

OK, EINVAL, ESHAPE, ENOSPACE, EHIP = 0, 1, 2, 3, 4


ABI_VERSION = 3          # VIDKV_ABI_VERSION of include/vidkv.h that this binding was written for


class VidkvParams(C.Structure):
    _fields_ = [
        ("n_layers", C.c_int32), ("batch", C.c_int32), ("n_kv_heads", C.c_int32),
        ("n_q_heads", C.c_int32), ("head_dim", C.c_int32), ("group", C.c_int32),
        ("t_quant", C.c_int32), ("n_anom", C.c_int32), ("use_fft", C.c_int32),
        ("n_salient", C.c_int32), ("gamma", C.c_float), ("softmax_scale", C.c_float),
        ("t_capacity", C.c_int32), ("salient_bits", C.c_int32), ("channel_metric", C.c_int32),
    ]


class VidkvView(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride_batch", C.c_int64), ("stride_head", C.c_int64),
                ("stride_token", C.c_int64), ("dtype", C.c_int32)]


ROTARY_PAIRS = 128       # VIDKV_ROTARY_PAIRS


class VidkvRotary(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("rot_dim", C.c_int32), ("adjacent", C.c_int32), ("n_axes", C.c_int32),
                ("axis", C.c_uint8 * ROTARY_PAIRS), ("turn", C.c_uint64 * ROTARY_PAIRS)]


CODE_INT8, CODE_E4M3 = 0, 1


class VidkvCache8(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("batch", C.c_int32), ("n_kv_heads", C.c_int32), ("n_q_heads", C.c_int32),
                ("head_dim", C.c_int32), ("capacity", C.c_int32), ("code", C.c_int32), ("softmax_scale", C.c_float)]


class VidkvRows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride_batch", C.c_int64), ("stride_row", C.c_int64), ("dtype", C.c_int32)]


TREE_NODES, TREE_VOCAB = 256, 1 << 22    # VIDKV_TREE_NODES, VIDKV_TREE_VOCAB


class VidkvSideStream(C.Structure):
    _fields_ = [("hip_stream", C.c_void_p), ("fork_event", C.c_void_p), ("join_event", C.c_void_p)]


class SideStream:
    """A torch stream and two events for the calls that take a vidkv_side_stream.

    Owned by the caller: keep it alive as long as work enqueued with it may run."""

    def __init__(self, device="cuda:0"):
        import torch
        with torch.cuda.device(device):
            self.stream = torch.cuda.Stream(device=device)          # default priority
            self.fork = torch.cuda.Event(enable_timing=False)
            self.join = torch.cuda.Event(enable_timing=False)
            # torch creates the event handle lazily, at the first record
            self.fork.record(self.stream)
            self.join.record(self.stream)
        self.c = VidkvSideStream(self.stream.cuda_stream, self.fork.cuda_event, self.join.cuda_event)


def _side(side):
    return None if side is None else C.byref(side.c)


class VidkvError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


_lib = _native = None


def lib() -> C.CDLL:
    """Load the shared library (once).  Raises if it is not built."""
    global _lib, _native
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2503_16257_amd.build`")
        # PyTorch ships its own HIP runtime; it must be in the process before this library is
        # loaded, so that both resolve to that one copy.  Loaded the other way round the
        # library registers its kernels with a second runtime, and every launch on a torch
        # stream fails.
        import torch
        L = C.CDLL(LIB_PATH)
        PP = C.POINTER(VidkvParams)
        vp, sz, i32 = C.c_void_p, C.c_size_t, C.c_int32
        L.vidkv_packed_keys_bytes.argtypes = [PP]
        L.vidkv_packed_keys_bytes.restype = sz
        L.vidkv_packed_values_bytes.argtypes = [PP]
        L.vidkv_packed_values_bytes.restype = sz
        L.vidkv_workspace_bytes.argtypes = [PP, C.c_int]
        L.vidkv_workspace_bytes.restype = sz
        L.vidkv_quantize_keys.argtypes = [PP, vp, vp, sz, vp, sz, vp]
        L.vidkv_quantize_keys.restype = C.c_int
        L.vidkv_quantize_values.argtypes = [PP, vp, vp, vp, vp, sz, vp, sz, vp]
        L.vidkv_quantize_values.restype = C.c_int
        SP = C.POINTER(VidkvSideStream)
        L.vidkv_quantize_kv.argtypes = [PP, vp, vp, vp, vp, vp, sz, vp, sz, vp, sz, vp, SP]
        L.vidkv_quantize_kv.restype = C.c_int
        L.vidkv_flush_residual.argtypes = [PP, i32, vp, vp, i32, i32, vp, sz, vp, sz, vp]
        L.vidkv_flush_residual.restype = C.c_int
        L.vidkv_saliency_workspace_bytes.argtypes = [i32, i32]
        L.vidkv_saliency_workspace_bytes.restype = sz
        L.vidkv_saliency_scores.argtypes = [vp, vp, i32, i32, i32, i32, vp, vp, sz, vp]
        L.vidkv_saliency_scores.restype = C.c_int
        L.vidkv_decode_attention.argtypes = [PP, i32, vp, vp, vp, vp, vp, i32, vp, vp, vp, sz, vp, SP]
        L.vidkv_decode_attention.restype = C.c_int
        L.vidkv_decode_attention_noalloc.argtypes = [PP, i32, vp, vp, vp, vp, vp, i32, vp, vp, vp]
        L.vidkv_decode_attention_noalloc.restype = C.c_int
        u32 = C.c_uint32
        L.vidkv_quantize_keys_stages.argtypes = [PP, vp, vp, sz, vp, sz, u32, vp]
        L.vidkv_quantize_keys_stages.restype = C.c_int
        L.vidkv_quantize_values_stages.argtypes = [PP, vp, vp, vp, vp, sz, vp, sz, u32, vp]
        L.vidkv_quantize_values_stages.restype = C.c_int
        L.vidkv_decode_attention_stages.argtypes = [PP, i32, vp, vp, vp, vp, vp, i32, vp, vp, vp,
                                                    sz, u32, vp, SP]
        L.vidkv_decode_attention_stages.restype = C.c_int
        L.vidkv_calib_copy.argtypes = [vp, vp, sz, vp]
        L.vidkv_calib_copy.restype = C.c_int
        VP, RP, CP, f64 = C.POINTER(VidkvView), C.POINTER(VidkvRotary), C.POINTER(VidkvCache8), C.c_double
        L.vidkv_rotary_init.argtypes = [RP, i32, i32, i32, i32, C.POINTER(i32), f64, C.POINTER(f64)]
        L.vidkv_rotary_init.restype = C.c_int
        L.vidkv_rotary_apply.argtypes = [RP, i32, i32, i32, vp, i32, VP, VP, i32, VP, VP, vp]
        L.vidkv_rotary_apply.restype = C.c_int
        L.vidkv_cache8_bytes.argtypes = [CP]
        L.vidkv_cache8_bytes.restype = sz
        L.vidkv_cache8_workspace_bytes.argtypes = [CP, i32]
        L.vidkv_cache8_workspace_bytes.restype = sz
        L.vidkv_cache8_write.argtypes = [CP, i32, i32, VP, VP, vp, vp, RP, vp, vp, sz, vp]
        L.vidkv_cache8_write.restype = C.c_int
        L.vidkv_cache8_read.argtypes = [CP, i32, i32, vp, vp, sz, VP, VP, vp]
        L.vidkv_cache8_read.restype = C.c_int
        L.vidkv_cache8_attention.argtypes = [CP, i32, i32, i32, VP, vp, sz, vp, vp, VP, vp, sz, vp]
        L.vidkv_cache8_attention.restype = C.c_int
        WP, i64 = C.POINTER(VidkvRows), C.c_int64
        L.vidkv_tree_masks.argtypes = [i32, i32, vp, vp, vp, i32, vp, vp, vp]
        L.vidkv_tree_masks.restype = C.c_int
        L.vidkv_cache8_tree_attention.argtypes = [CP, i32, i32, VP, VP, VP, vp, vp, sz, vp, vp, VP, vp, sz, vp]
        L.vidkv_cache8_tree_attention.restype = C.c_int
        L.vidkv_tree_verify_workspace_bytes.argtypes = [i32, i32, i32]
        L.vidkv_tree_verify_workspace_bytes.restype = sz
        L.vidkv_tree_verify.argtypes = [i32, i32, i32, WP, WP, i32, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.vidkv_tree_verify.restype = C.c_int
        L.vidkv_cache8_append_path.argtypes = [CP, i32, VP, i64, VP, i64, vp, vp, vp, vp, sz, vp]
        L.vidkv_cache8_append_path.restype = C.c_int
        L.vidkv_status_string.argtypes = [C.c_int]
        L.vidkv_status_string.restype = C.c_char_p
        L.vidkv_abi_version.argtypes = []
        L.vidkv_abi_version.restype = C.c_int
        _bind_torch(torch)
        _native = _load_native(L)
        _lib = L
    return _lib


def native_tag() -> str:
    """What a build of the native call layer belongs to: it reads CPython's and torch's structures."""
    import torch
    return f"{sys.implementation.cache_tag} torch {torch.__version__}"


def _load_native(L):
    """The native call layer, or None: then every call takes the Python path."""
    try:
        from . import vidkv_marshal as m
        built_for = getattr(m, "built_for", None)
        if built_for != native_tag():
            raise ImportError(f"it was built for {built_for}, this is {native_tag()}")
    except ImportError as e:
        logging.getLogger(__name__).warning(
            "vidkv_marshal.so is not used (%s): each call costs a few us more on the host; build it with "
            "`python -m paper_2503_16257_amd.build`", e)
        return None
    m.bind(*(C.cast(f, C.c_void_p).value for f in (
        L.vidkv_decode_attention, L.vidkv_decode_attention_noalloc, L.vidkv_flush_residual)),
        VidkvParams, VidkvSideStream)
    m.bind8(*(C.cast(f, C.c_void_p).value for f in (
        L.vidkv_rotary_apply, L.vidkv_cache8_write, L.vidkv_cache8_read, L.vidkv_cache8_attention)),
        VidkvRotary, VidkvCache8)
    m.bind_tree(*(C.cast(f, C.c_void_p).value for f in (
        L.vidkv_tree_masks, L.vidkv_cache8_tree_attention, L.vidkv_tree_verify, L.vidkv_cache8_append_path)))
    return m


def make_params(n_layers, batch, n_kv_heads, n_q_heads, t_quant, n_anom, n_salient,
                gamma=0.7, softmax_scale=None, head_dim=128, group=32, use_fft=1,
                t_capacity=0, salient_bits=0, channel_metric=0) -> VidkvParams:
    if softmax_scale is None:
        softmax_scale = 1.0 / math.sqrt(head_dim)
    return VidkvParams(n_layers, batch, n_kv_heads, n_q_heads, head_dim, group, t_quant, n_anom,
                       use_fft, n_salient, gamma, softmax_scale, t_capacity, salient_bits, channel_metric)


def status_string(status: int) -> str:
    return lib().vidkv_status_string(status).decode()


def abi_version() -> int:
    return lib().vidkv_abi_version()


def packed_keys_bytes(p: VidkvParams) -> int:
    return lib().vidkv_packed_keys_bytes(C.byref(p))


def packed_values_bytes(p: VidkvParams) -> int:
    return lib().vidkv_packed_values_bytes(C.byref(p))


def workspace_bytes(p: VidkvParams, which: int) -> int:
    return lib().vidkv_workspace_bytes(C.byref(p), which)


# A decode call marshals ten arguments and a flush eight, once per layer: natively where the arguments are
# plain (host time with and without, in turn in one process: 6.9 against 9.0 us a decode call, 3.5 against 5.7 a flush, in
# another 7.8 against 10.0 and 4.2 against 5.8; the launches are 3 us each), and what follows is kept to a few
# attribute reads per tensor.  torch's names are looked up once, with the library.
_Tensor = _f16 = _u8 = _f32 = _i32 = _i64 = _raw_stream = _cur_device = None
_dtypes = {}             # of views: torch's to vidkv_dtype


def _bind_torch(torch) -> None:
    global _Tensor, _f16, _u8, _f32, _i32, _i64, _raw_stream, _cur_device
    _f16, _u8, _f32, _i32, _i64 = torch.float16, torch.uint8, torch.float32, torch.int32, torch.int64
    _dtypes.update({torch.float16: 0, torch.bfloat16: 1, torch.float32: 2})
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    _cur_device = torch.cuda.current_device
    _Tensor = torch.Tensor


def _ptr(t, dtype=None, name="tensor"):
    """Device pointer of a contiguous CUDA tensor (None -> NULL)."""
    if t is None:
        return None
    if not isinstance(t, _Tensor) or not t.is_cuda:
        raise TypeError(f"{name}: expected a CUDA tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    if dtype is not None and t.dtype is not dtype:
        raise TypeError(f"{name}: expected dtype {dtype}, got {t.dtype}")
    return t.data_ptr()


def _nbytes(t) -> int:
    return t.nbytes


def _stream(stream):
    """Handle of a torch stream, of the current device's current one for None."""
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None:
        return _raw_stream(_cur_device())
    import torch
    return torch.cuda.current_stream().cuda_stream


def _check(status: int, where: str):
    if status != OK:
        raise VidkvError(status, where)


def quantize_keys(p: VidkvParams, K, packed_K, workspace, stream=None, stages=None) -> None:
    """vidkv_quantize_keys: K [L,B,Hkv,Tq,128] fp16 -> packed_K (uint8 buffer).
    With `stages` (bit mask) calls vidkv_quantize_keys_stages instead."""
    L = _lib or lib()
    a = [C.byref(p), _ptr(K, _f16, "K"), _ptr(packed_K, _u8, "packed_K"),
         _nbytes(packed_K), _ptr(workspace, _u8, "workspace"), _nbytes(workspace)]
    if stages is None:
        _check(L.vidkv_quantize_keys(*a, _stream(stream)), "vidkv_quantize_keys")
    else:
        _check(L.vidkv_quantize_keys_stages(*a, stages, _stream(stream)),
               "vidkv_quantize_keys_stages")


def quantize_values(p: VidkvParams, V, packed_V, workspace, saliency=None, salient_idx=None,
                    stream=None, stages=None) -> None:
    """vidkv_quantize_values: V fp16 (+ scores [B,Tq] f32 or indices [B,n_s] i32) -> packed_V."""
    L = _lib or lib()
    a = [C.byref(p), _ptr(V, _f16, "V"), _ptr(saliency, _f32, "saliency"),
         _ptr(salient_idx, _i32, "salient_idx"), _ptr(packed_V, _u8, "packed_V"),
         _nbytes(packed_V), _ptr(workspace, _u8, "workspace"), _nbytes(workspace)]
    if stages is None:
        _check(L.vidkv_quantize_values(*a, _stream(stream)), "vidkv_quantize_values")
    else:
        _check(L.vidkv_quantize_values_stages(*a, stages, _stream(stream)),
               "vidkv_quantize_values_stages")


def decode_attention(p: VidkvParams, layer: int, q, packed_K, packed_V, out, workspace,
                     K_tail=None, V_tail=None, tail_capacity: int = 0, tail_len=None,
                     stream=None, stages=None, side=None) -> None:
    """vidkv_decode_attention: one decode step of one layer -> out [B,Hq,128] fp16.
    `side`: a SideStream or None: not used, the call runs in line either way."""
    L = _lib or lib()
    if stages is None and _native is not None:
        st = _native.decode_attention(p, layer, q, packed_K, packed_V, K_tail, V_tail, tail_capacity, tail_len, out,
                                      workspace, _stream, stream, None if side is None else side.c)
        if st is not None:
            if st != OK:
                raise VidkvError(st, "vidkv_decode_attention")
            return
    a = [C.byref(p), layer, _ptr(q, _f16, "q"), _ptr(packed_K, _u8, "packed_K"),
         _ptr(packed_V, _u8, "packed_V"), _ptr(K_tail, _f16, "K_tail"),
         _ptr(V_tail, _f16, "V_tail"), tail_capacity, _ptr(tail_len, _i32, "tail_len"),
         _ptr(out, _f16, "out"), _ptr(workspace, _u8, "workspace"),
         _nbytes(workspace)]
    if stages is None:
        _check(L.vidkv_decode_attention(*a, _stream(stream), _side(side)), "vidkv_decode_attention")
    else:
        _check(L.vidkv_decode_attention_stages(*a, stages, _stream(stream), _side(side)),
               "vidkv_decode_attention_stages")


NOALLOC_SCRATCH_BYTES = 16 << 20     # VIDKV_NOALLOC_SCRATCH_BYTES of include/vidkv.h


def decode_attention_noalloc(p: VidkvParams, layer: int, q, packed_K, packed_V, out, K_tail=None,
                             V_tail=None, tail_capacity: int = 0, tail_len=None, stream=None) -> None:
    """vidkv_decode_attention_noalloc: the decode step without a workspace argument."""
    L = _lib or lib()
    if _native is not None:
        st = _native.decode_attention_noalloc(p, layer, q, packed_K, packed_V, K_tail, V_tail, tail_capacity, tail_len, out,
                                              _stream, stream)
        if st is not None:
            return _check(st, "vidkv_decode_attention_noalloc")
    _check(L.vidkv_decode_attention_noalloc(
        C.byref(p), layer, _ptr(q, _f16, "q"), _ptr(packed_K, _u8, "packed_K"),
        _ptr(packed_V, _u8, "packed_V"), _ptr(K_tail, _f16, "K_tail"),
        _ptr(V_tail, _f16, "V_tail"), tail_capacity, _ptr(tail_len, _i32, "tail_len"),
        _ptr(out, _f16, "out"), _stream(stream)), "vidkv_decode_attention_noalloc")


def quantize_kv(p: VidkvParams, K, V, packed_K, packed_V, workspace, saliency=None,
                salient_idx=None, stream=None, side=None) -> None:
    """vidkv_quantize_kv: both tensors of the same tokens in one call.
    `side`: a SideStream for the protected-token selection, or None (in line)."""
    L = _lib or lib()
    _check(L.vidkv_quantize_kv(
        C.byref(p), _ptr(K, _f16, "K"), _ptr(V, _f16, "V"),
        _ptr(saliency, _f32, "saliency"), _ptr(salient_idx, _i32, "salient_idx"),
        _ptr(packed_K, _u8, "packed_K"), _nbytes(packed_K),
        _ptr(packed_V, _u8, "packed_V"), _nbytes(packed_V),
        _ptr(workspace, _u8, "workspace"), _nbytes(workspace), _stream(stream), _side(side)),
        "vidkv_quantize_kv")


def flush_residual(p: VidkvParams, layer: int, K_tail, V_tail, tail_capacity: int, n_flush: int,
                   packed_K, packed_V, stream=None) -> None:
    """vidkv_flush_residual: code the first n_flush residual tokens of one layer and append them."""
    L = _lib or lib()
    if _native is not None:
        st = _native.flush_residual(p, layer, K_tail, V_tail, tail_capacity, n_flush, packed_K, packed_V, _stream, stream)
        if st is not None:
            return _check(st, "vidkv_flush_residual")
    _check(L.vidkv_flush_residual(
        C.byref(p), layer, _ptr(K_tail, _f16, "K_tail"), _ptr(V_tail, _f16, "V_tail"),
        tail_capacity, n_flush, _ptr(packed_K, _u8, "packed_K"), _nbytes(packed_K),
        _ptr(packed_V, _u8, "packed_V"), _nbytes(packed_V), _stream(stream)),
        "vidkv_flush_residual")


def saliency_workspace_bytes(batch: int, hidden_dim: int) -> int:
    return lib().vidkv_saliency_workspace_bytes(batch, hidden_dim)


def saliency_scores(X_v, X_t, scores, workspace, stream=None) -> None:
    """vidkv_saliency_scores: X_v [B,Tv,d] fp16, X_t [B,Nt,d] fp16 -> scores [B,Tv] f32."""
    L = _lib or lib()
    B, Tv, d = X_v.shape
    assert X_t.shape[0] == B and X_t.shape[2] == d and tuple(scores.shape) == (B, Tv)
    _check(L.vidkv_saliency_scores(
        _ptr(X_v, _f16, "X_v"), _ptr(X_t, _f16, "X_t"), B, Tv, X_t.shape[1], d,
        _ptr(scores, _f32, "scores"), _ptr(workspace, _u8, "workspace"),
        _nbytes(workspace), _stream(stream)), "vidkv_saliency_scores")


# ---- rotary positions and the 8-bit cache: views [B, heads, tokens, channels] with strides of their own ----

def _here(t, name):
    if t.device.index != _cur_device():
        raise ValueError(f"{name}: is on {t.device}, the current device is cuda:{_cur_device()}")


def _arg(t, dtype, name, shape=None):
    """_ptr of a tensor on the current device (None -> NULL), of `shape` if given."""
    p = _ptr(t, dtype, name)
    if t is not None:
        _here(t, name)
        if shape is not None and tuple(t.shape) != shape:
            raise ValueError(f"{name}: expected shape {shape}, got {tuple(t.shape)}")
    return p


def _view(t, name, shape, written=False):
    """A tensor of any strides whose channels lie next to each other, as a VidkvView (None -> NULL)."""
    if t is None:
        return None
    if not isinstance(t, _Tensor) or not t.is_cuda:
        raise TypeError(f"{name}: expected a CUDA tensor")
    _here(t, name)
    code = _dtypes.get(t.dtype)
    if code is None:
        raise TypeError(f"{name}: expected float16, bfloat16 or float32, got {t.dtype}")
    if tuple(t.shape) != shape:
        raise ValueError(f"{name}: expected shape {shape}, got {tuple(t.shape)}")
    b, h, n, c = t.stride()
    if c != 1:
        raise ValueError(f"{name}: the channels of a token must lie next to each other")
    # the stride of an axis of one is never used, and torch leaves what it likes there
    b, h, n = (b if shape[0] > 1 else 0), (h if shape[1] > 1 else 0), (n if shape[2] > 1 else 0)
    if written and 0 not in shape:
        extent = shape[3]                      # (axes that nest: any further one steps over what the nearer ones span)
        for st, size in sorted((abs(st), size) for st, size in ((b, shape[0]), (h, shape[1]), (n, shape[2])) if size > 1):
            if st < extent:
                raise ValueError(f"{name}: is written to, and its elements overlap")
            extent += st * (size - 1)
    return VidkvView(t.data_ptr(), b, h, n, code)


def _ref(v):
    return None if v is None else C.byref(v)


def make_rotary(sections, theta: float = 10000.0, head_dim: int = 128, rot_dim=None, adjacent: bool = False,
                freq=None) -> VidkvRotary:
    """vidkv_rotary_init: `sections` pairs of each axis (time, height, width: e.g. 16, 24, 24), frequencies
    theta^(-2i / rot_dim) or `freq` (radians a position, one for each pair)."""
    rot_dim = head_dim if rot_dim is None else rot_dim
    sec = (C.c_int32 * max(len(sections), 1))(*sections)
    fr = None
    if freq is not None:
        if len(freq) != rot_dim // 2:
            raise ValueError(f"freq: expected {rot_dim // 2} numbers, got {len(freq)}")
        fr = (C.c_double * len(freq))(*(float(f) for f in freq))
    r = VidkvRotary()
    _check((_lib or lib()).vidkv_rotary_init(C.byref(r), head_dim, rot_dim, int(adjacent), len(sections), sec, theta, fr),
           "vidkv_rotary_init")
    return r


def rotary(rot: VidkvRotary, positions, q, q_out, k=None, k_out=None, inverse: bool = False, stream=None) -> None:
    """vidkv_rotary_apply: q [B,Hq,n,d] (and k [B,Hk,n,d]) turned by their positions [n_axes,B,n] int32 into q_out, k_out
    (which may be q and k themselves).  `inverse`: turned back; of gradients, the backward pass.  q or k may be None."""
    L = _lib or lib()
    if _native is not None:
        st = _native.rotary(rot, positions, q, q_out, k, k_out, inverse, _stream, stream)
        if st is not None:
            return _check(st, "vidkv_rotary_apply")
    x = q if q is not None else k
    if x is None:
        raise ValueError("rotary: neither q nor k")
    B, n = (x.shape[0], x.shape[2]) if x.dim() == 4 else (-1, -1)
    d = rot.head_dim
    hq, hk = (0 if t is None or t.dim() != 4 else t.shape[1] for t in (q, k))
    v = [_view(q, "q", (B, hq, n, d)), _view(q_out if q is not None else None, "q_out", (B, hq, n, d), True),
         _view(k, "k", (B, hk, n, d)), _view(k_out if k is not None else None, "k_out", (B, hk, n, d), True)]
    pos = _arg(positions, _i32, "positions", (rot.n_axes, B, n))
    if B * n == 0 or hq + hk == 0:
        return
    _check(L.vidkv_rotary_apply(C.byref(rot), int(inverse), B, n, pos, hq, _ref(v[0]), _ref(v[1]), hk, _ref(v[2]),
                                _ref(v[3]), _stream(stream)), "vidkv_rotary_apply")


def make_cache8(n_layers, batch, n_kv_heads, n_q_heads, capacity, code=CODE_INT8, softmax_scale=None,
                head_dim=128) -> VidkvCache8:
    if softmax_scale is None:
        softmax_scale = 1.0 / math.sqrt(head_dim)
    return VidkvCache8(n_layers, batch, n_kv_heads, n_q_heads, head_dim, capacity, code, softmax_scale)


def cache8_bytes(p: VidkvCache8) -> int:
    return lib().vidkv_cache8_bytes(C.byref(p))


def cache8_workspace_bytes(p: VidkvCache8, n_query: int) -> int:
    return lib().vidkv_cache8_workspace_bytes(C.byref(p), n_query)


def cache8_write(p: VidkvCache8, layer: int, cache, K, V, start, count=None, rotary=None, positions=None,
                 stream=None) -> None:
    """vidkv_cache8_write: K, V [B,Hkv,n,128] fp16 / bf16 coded as tokens start[b].. (int32 [B]) of each sequence, the
    first count[b] of them; with a VidkvRotary and positions [n_axes,B,n] the keys are turned on the way."""
    L = _lib or lib()
    if _native is not None:
        st = _native.cache8_write(p, layer, cache, K, V, start, count, rotary, positions, _stream, stream)
        if st is not None:
            return _check(st, "vidkv_cache8_write")
    n = K.shape[2] if isinstance(K, _Tensor) and K.dim() == 4 else -1
    shape = (p.batch, p.n_kv_heads, n, 128)
    vk, vv = _view(K, "K", shape), _view(V, "V", shape)
    if rotary is not None and positions is None or rotary is None and positions is not None:
        raise ValueError("cache8_write: rotary and positions come together")
    pos = None if rotary is None else _arg(positions, _i32, "positions", (rotary.n_axes, p.batch, n))
    a = [_arg(start, _i32, "start", (p.batch,)), _arg(count, _i32, "count", (p.batch,)), _ref(rotary), pos,
         _arg(cache, _u8, "cache"), _nbytes(cache), _stream(stream)]
    if n == 0:
        return
    _check(L.vidkv_cache8_write(C.byref(p), layer, n, _ref(vk), _ref(vv), *a), "vidkv_cache8_write")


def cache8_read(p: VidkvCache8, layer: int, cache, start, K, V=None, stream=None) -> None:
    """vidkv_cache8_read: tokens start[b].. (int32 [B]) as values into K, V [B,Hkv,n,128] (fp16, bf16 or fp32; either
    may be None)."""
    L = _lib or lib()
    if _native is not None:
        st = _native.cache8_read(p, layer, cache, start, K, V, _stream, stream)
        if st is not None:
            return _check(st, "vidkv_cache8_read")
    x = K if K is not None else V
    n = x.shape[2] if isinstance(x, _Tensor) and x.dim() == 4 else -1
    shape = (p.batch, p.n_kv_heads, n, 128)
    vk, vv = _view(K, "K", shape, True), _view(V, "V", shape, True)
    a = [_arg(start, _i32, "start", (p.batch,)), _arg(cache, _u8, "cache"), _nbytes(cache)]
    if n == 0:
        return
    _check(L.vidkv_cache8_read(C.byref(p), layer, n, *a, _ref(vk), _ref(vv), _stream(stream)), "vidkv_cache8_read")


def cache8_attention(p: VidkvCache8, layer: int, cache, q, out, length, workspace, q_count=None, causal: bool = True,
                     stream=None) -> None:
    """vidkv_cache8_attention: queries q [B,Hq,n,128], the last tokens of each sequence, over its first length[b] (int32
    [B]) tokens of the cache -> out; q_count[b]: how many of them there are (None: all n)."""
    L = _lib or lib()
    if _native is not None:
        st = _native.cache8_attention(p, layer, cache, q, out, length, workspace, q_count, causal, _stream, stream)
        if st is not None:
            return _check(st, "vidkv_cache8_attention")
    n = q.shape[2] if isinstance(q, _Tensor) and q.dim() == 4 else -1
    shape = (p.batch, p.n_q_heads, n, 128)
    vq, vo = _view(q, "q", shape), _view(out, "out", shape, True)
    a = [_arg(cache, _u8, "cache"), _nbytes(cache), _arg(length, _i32, "length", (p.batch,)),
         _arg(q_count, _i32, "q_count", (p.batch,)), _ref(vo), _arg(workspace, _u8, "workspace"), _nbytes(workspace)]
    if n == 0:
        return
    _check(L.vidkv_cache8_attention(C.byref(p), layer, n, int(causal), _ref(vq), *a, _stream(stream)),
           "vidkv_cache8_attention")


# ---- trees of drafted tokens: node 0 is the last token that was sampled, node i > 0 is drafted behind parents[b][i] < i ----

def _nodes(t, name):
    """Batch and nodes of an int32 [B, n] tensor."""
    if not isinstance(t, _Tensor) or t.dim() != 2:
        raise ValueError(f"{name}: expected a tensor [batch, nodes]")
    return t.shape[0], t.shape[1]


def tree_masks(parents, masks, base=None, positions=None, count=None, stream=None) -> None:
    """vidkv_tree_masks: parents [B,n] int32 -> masks [B,n,ceil(n/64)] int64, the nodes that each node sees as bits, and, with
    base [B] int32, positions [n_axes,B,n] int32.  parents None: chains, of the masks' sizes.  count[b]: nodes that there are
    (None: all n)."""
    L = _lib or lib()
    if _native is not None:
        st = _native.tree_masks(parents, masks, base, positions, count, _stream, stream)
        if st is not None:
            return _check(st, "vidkv_tree_masks")
    if not isinstance(masks, _Tensor) or masks.dim() != 3:
        raise ValueError("masks: expected a tensor [batch, nodes, words]")
    B, n = masks.shape[0], masks.shape[1]
    if (base is None) != (positions is None):
        raise ValueError("tree_masks: base and positions come together")
    axes = 0
    if positions is not None:
        axes = positions.shape[0] if isinstance(positions, _Tensor) and positions.dim() == 3 else -1
    a = [_arg(parents, _i32, "parents", (B, n)), _arg(count, _i32, "count", (B,)),
         _arg(masks, _i64, "masks", (B, n, (n + 63) // 64)), axes, _arg(base, _i32, "base", (B,)),
         _arg(positions, _i32, "positions", (axes, B, n))]
    if B == 0:
        return
    _check(L.vidkv_tree_masks(B, n, *a, _stream(stream)), "vidkv_tree_masks")


def cache8_tree_attention(p: VidkvCache8, layer: int, cache, q, K, V, masks, out, length, workspace, count=None,
                          stream=None) -> None:
    """vidkv_cache8_tree_attention: the nodes' queries q [B,Hq,n,128] over the first length[b] tokens of the cache and the
    nodes of K, V [B,Hkv,n,128] that masks [B,n,words] int64 has for each -> out.  The workspace is that of
    cache8_attention (cache8_workspace_bytes(p, n))."""
    L = _lib or lib()
    if _native is not None:
        st = _native.cache8_tree_attention(p, layer, cache, q, K, V, masks, out, length, workspace, count, _stream, stream)
        if st is not None:
            return _check(st, "vidkv_cache8_tree_attention")
    n = q.shape[2] if isinstance(q, _Tensor) and q.dim() == 4 else -1
    shape, kv = (p.batch, p.n_q_heads, n, 128), (p.batch, p.n_kv_heads, n, 128)
    vq, vk, vv, vo = _view(q, "q", shape), _view(K, "K", kv), _view(V, "V", kv), _view(out, "out", shape, True)
    _check(L.vidkv_cache8_tree_attention(
        C.byref(p), layer, n, _ref(vq), _ref(vk), _ref(vv), _arg(masks, _i64, "masks", (p.batch, n, (n + 63) // 64)),
        _arg(cache, _u8, "cache"), _nbytes(cache), _arg(length, _i32, "length", (p.batch,)),
        _arg(count, _i32, "count", (p.batch,)), _ref(vo), _arg(workspace, _u8, "workspace"), _nbytes(workspace),
        _stream(stream)), "vidkv_cache8_tree_attention")


def tree_verify_workspace_bytes(batch: int, n_nodes: int, vocab: int) -> int:
    return lib().vidkv_tree_verify_workspace_bytes(batch, n_nodes, vocab)


def _rows(t, name, shape):
    """Rows of probabilities [B, n, vocab] of any strides, entries next to each other, as a VidkvRows (None -> NULL)."""
    if t is None:
        return None
    if not isinstance(t, _Tensor) or not t.is_cuda:
        raise TypeError(f"{name}: expected a CUDA tensor")
    _here(t, name)
    code = _dtypes.get(t.dtype)
    if code is None:
        raise TypeError(f"{name}: expected float16, bfloat16 or float32, got {t.dtype}")
    if tuple(t.shape) != shape:
        raise ValueError(f"{name}: expected shape {shape}, got {tuple(t.shape)}")
    b, r, c = t.stride()
    if c != 1 and shape[2] > 1:
        raise ValueError(f"{name}: the entries of a row must lie next to each other")
    return VidkvRows(t.data_ptr(), b if shape[0] > 1 else 0, r if shape[1] > 1 else 0, code)


def tree_verify(target, tokens, uniform, path, accepted, next_token, workspace, draft=None, parents=None, count=None,
                distinct: bool = False, stream=None) -> None:
    """vidkv_tree_verify: target [B,n,vocab] probabilities (float32, float16, bfloat16) behind each node, tokens [B,n] int32,
    uniform [B,n] float32 in [0, 1) -> path [B,n] (nodes that stand, then -1), accepted [B] (how many), next_token [B], all int32.
    draft [B,n,vocab]: what the children of each node were drawn from, with `distinct` without putting back; None: they are no
    random ones.  parents None: chains.  Rows sum to one: with `distinct` a nearly certain draft's rows are better passed in float32 and
    divided by their sums (vidkv.h says what others are off by)."""
    L = _lib or lib()
    if _native is not None:
        st = _native.tree_verify(target, tokens, uniform, path, accepted, next_token, workspace, draft, parents, count, distinct,
                                 _stream, stream)
        if st is not None:
            return _check(st, "vidkv_tree_verify")
    B, n = _nodes(tokens, "tokens")
    V = target.shape[2] if isinstance(target, _Tensor) and target.dim() == 3 else -1
    t, d = _rows(target, "target", (B, n, V)), _rows(draft, "draft", (B, n, V))
    a = [_arg(tokens, _i32, "tokens", (B, n)), _arg(parents, _i32, "parents", (B, n)), _arg(count, _i32, "count", (B,)),
         _arg(uniform, _f32, "uniform", (B, n)), _arg(path, _i32, "path", (B, n)), _arg(accepted, _i32, "accepted", (B,)),
         _arg(next_token, _i32, "next_token", (B,)), _arg(workspace, _u8, "workspace"), _nbytes(workspace)]
    if B == 0:
        return
    _check(L.vidkv_tree_verify(B, n, V, _ref(t), _ref(d), int(distinct), *a, _stream(stream)), "vidkv_tree_verify")


def cache8_append_path(p: VidkvCache8, cache, K, V, path, accepted, start, stream=None) -> None:
    """vidkv_cache8_append_path: of K, V [n_layers,B,Hkv,n,128] fp16 / bf16 the nodes path[b][:accepted[b]] coded as tokens
    start[b].. of every layer."""
    L = _lib or lib()
    if _native is not None:
        st = _native.cache8_append_path(p, cache, K, V, path, accepted, start, _stream, stream)
        if st is not None:
            return _check(st, "vidkv_cache8_append_path")
    B, n = _nodes(path, "path")
    v, layer = [], []
    for t, name in ((K, "K"), (V, "V")):
        if not isinstance(t, _Tensor) or t.dim() != 5 or t.shape[0] != p.n_layers:
            raise ValueError(f"{name}: expected a tensor [{p.n_layers}, batch, heads, nodes, 128]")
        v.append(_view(t[0], name, (p.batch, p.n_kv_heads, n, 128)))
        layer.append(t.stride(0) if p.n_layers > 1 else 0)
    _check(L.vidkv_cache8_append_path(
        C.byref(p), n, _ref(v[0]), layer[0], _ref(v[1]), layer[1], _arg(path, _i32, "path", (p.batch, n)),
        _arg(accepted, _i32, "accepted", (p.batch,)), _arg(start, _i32, "start", (p.batch,)), _arg(cache, _u8, "cache"),
        _nbytes(cache), _stream(stream)), "vidkv_cache8_append_path")


def calib_copy(dst, src, stream=None) -> None:
    L = _lib or lib()
    _check(L.vidkv_calib_copy(_ptr(dst, None, "dst"), _ptr(src, None, "src"), _nbytes(src),
                                  _stream(stream)), "vidkv_calib_copy")


def alloc_bytes(nbytes: int, device="cuda:0"):
    """A 256-byte-aligned uint8 device buffer (torch's allocator aligns to 512)."""
    import torch
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)
