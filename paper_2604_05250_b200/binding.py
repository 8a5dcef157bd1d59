"""Thin ctypes binding of ``include/dualdiff.h``: argument marshalling only.

Every function takes torch tensors (device memory for the plain calls, pinned
host memory for the ``*_host`` calls), passes their data pointers and sizes
through the C ABI, and raises ``DualDiffError`` on a non-zero status.  There is
no Python or CPU implementation behind these names: if ``libdualdiff.so`` is
missing the first call raises.
"""
from __future__ import annotations

import contextlib
import ctypes
import importlib.util
import os
from typing import NamedTuple

import torch
from torch import Tensor

from .build import host_path

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdualdiff.so")

DD_OK, DD_ERR_INVALID_ARG, DD_ERR_UNSUPPORTED, DD_ERR_CUDA, DD_ERR_TIMEOUT = 0, -1, -2, -3, -4
DD_MODE_TRUST, DD_MODE_KL, DD_MODE_CONF = 0, 1, 2
DD_FLAG_PROBABILISTIC, DD_FLAG_EMIT_DRAFTER = 0x100, 0x200
DD_LAYOUT_BHND, DD_LAYOUT_BNHD = 0, 1

# every symbol include/dualdiff.h declares
EXPORTS = (
    "dd_bidir_attention", "dd_block_attention", "dd_verify", "dd_unmask", "dd_bidir_attention_host", "dd_verify_host", "dd_verify_static",
    "dd_verify_workspace_bytes", "dd_attention_status", "dd_verify_status", "dd_launch_count", "dd_release",
    "dd_status_string", "dd_last_cuda_error", "dd_version", "dd_debug_set_max_ctas", "dd_clear_status", "dd_debug_expire_wait", "dd_lm_head_verify",
    "dd_qk_norm_rope", "dd_cache_append", "dd_cached_attention", "dd_cached_attention_workspace_bytes",
)


class _Rotation(ctypes.Structure):
    _fields_ = [("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p), ("positions", ctypes.c_int), ("dims", ctypes.c_int),
                ("interleaved", ctypes.c_int)]


class _Strides(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("token", ctypes.c_int64), ("head", ctypes.c_int64)]


class _Cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("page_table", ctypes.c_void_p), ("num_pages", ctypes.c_int), ("max_pages", ctypes.c_int), ("page_size", ctypes.c_int),
                ("heads", ctypes.c_int), ("D", ctypes.c_int)]


class Cache(NamedTuple):
    """The pools of a paged 8-bit cache of one layer (dd_cache): k, v torch.float8_e4m3fn [num_pages, heads, page_size, D],
    k_scale, v_scale torch.float32 [num_pages, heads].  new_cache() makes one; pages are the caller's to give out.  The calls take a
    plain tuple of the four tensors as well."""
    k: Tensor
    v: Tensor
    k_scale: Tensor
    v_scale: Tensor


class DualDiffError(RuntimeError):
    def __init__(self, status: int, text: str):
        super().__init__(f"dualdiff status {status}: {text}")
        self.status = status


_lib = None


def lib() -> ctypes.CDLL:
    """Loads libdualdiff.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        _lib = load(LIB_PATH)
    return _lib


class use_library:
    """Context manager: the wrappers below call the library at `path` (for instance the
    bounds-checked build) instead of libdualdiff.so until the block ends."""

    def __init__(self, path):
        self.path = path

    def __enter__(self):
        global _lib
        self.saved = _lib
        _lib = load(self.path)
        return _lib

    def __exit__(self, *exc):
        global _lib
        _lib = self.saved
        return False


def load(path) -> ctypes.CDLL:
    """Loads one build of the library and declares its entry points."""
    if True:
        if not os.path.exists(path):
            raise RuntimeError(
                f"{path} is missing: build it with `python -m paper_2604_05250_b200.build`; "
                "there is no fallback implementation")
        L = ctypes.CDLL(path)
        vp, i32, f32, u64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_uint64
        attn = [vp, vp, vp, vp, i32, i32, i32, i32, f32, vp]
        ver = [vp, vp, vp, vp, i32, f32, i32, u64, vp, vp, vp, i32, i32, i32, vp]
        L.dd_bidir_attention.argtypes = attn
        L.dd_bidir_attention_host.argtypes = attn
        L.dd_block_attention.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, i32, vp, i32, f32, vp]
        L.dd_block_attention.restype = i32
        L.dd_verify.argtypes = ver
        L.dd_verify_host.argtypes = ver
        L.dd_verify_static.argtypes = ver
        L.dd_unmask.argtypes = [vp, vp, vp, f32, i32, vp, vp, vp, i32, i32, i32, vp]
        L.dd_unmask.restype = i32
        L.dd_verify_static.restype = i32
        for name in ("dd_bidir_attention", "dd_bidir_attention_host", "dd_verify", "dd_verify_host",
                     "dd_attention_status", "dd_verify_status", "dd_release", "dd_version"):
            getattr(L, name).restype = i32
        L.dd_attention_status.argtypes = []
        L.dd_verify_status.argtypes = []
        L.dd_release.argtypes = []
        L.dd_version.argtypes = []
        L.dd_verify_workspace_bytes.argtypes = [i32, i32, i32]
        L.dd_verify_workspace_bytes.restype = ctypes.c_size_t
        L.dd_launch_count.argtypes = []
        L.dd_launch_count.restype = u64
        L.dd_lm_head_verify.argtypes = [vp, vp, vp, vp, vp, vp, i32, f32, i32, u64, vp, vp, vp, i32, i32, i32, i32, vp]
        L.dd_lm_head_verify.restype = i32
        L.dd_qk_norm_rope.argtypes = [vp, vp, i32, vp, vp, i32, vp, vp, f32, vp, vp, vp, vp, i32, i32, i32, i32, vp]
        L.dd_cache_append.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, f32, vp, i32, i32, vp]
        L.dd_cached_attention.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, i32, f32, vp, ctypes.c_size_t, vp]
        L.dd_cached_attention_workspace_bytes.argtypes = [i32, i32, i32, vp]
        L.dd_cached_attention_workspace_bytes.restype = ctypes.c_size_t
        for name in ("dd_qk_norm_rope", "dd_cache_append", "dd_cached_attention"):
            getattr(L, name).restype = i32
        L.dd_clear_status.argtypes = []
        L.dd_clear_status.restype = i32
        L.dd_debug_expire_wait.argtypes = [i32, vp]
        L.dd_debug_expire_wait.restype = i32
        L.dd_debug_set_max_ctas.argtypes = [i32]
        L.dd_debug_set_max_ctas.restype = i32
        L.dd_status_string.argtypes = [i32]
        L.dd_status_string.restype = ctypes.c_char_p
        L.dd_last_cuda_error.argtypes = []
        L.dd_last_cuda_error.restype = ctypes.c_char_p
    return L


_fast = None        # the native form of the wrappers below (csrc/host_call.cpp); None: the Python form serves every call


def load_native():
    """Loads the native form if it has been built for this Python and torch; build.build() calls it again."""
    global _fast
    path = host_path()
    if _fast is None and os.path.exists(path):
        name = __package__ + "._host_call"
        spec = importlib.util.spec_from_file_location(name, path)
        try:
            module = importlib.util.module_from_spec(spec)
            spec.loader.exec_module(module)
        except ImportError:
            return
        _fast = module


load_native()


def _addresses(L):
    """Addresses of the entry points that _fast calls, looked up once per library."""
    try:
        return L._dd_addresses
    except AttributeError:
        L._dd_addresses = {name: ctypes.cast(getattr(L, name), ctypes.c_void_p).value
                           for name in ("dd_bidir_attention", "dd_block_attention", "dd_verify", "dd_verify_static", "dd_unmask",
                                        "dd_qk_norm_rope", "dd_cache_append", "dd_cached_attention",
                                        "dd_cached_attention_workspace_bytes")}
        return L._dd_addresses


def _check(status: int):
    if status != DD_OK:
        L = lib()
        text = L.dd_status_string(status).decode()
        if status == DD_ERR_CUDA:
            text += ": " + L.dd_last_cuda_error().decode()
        raise DualDiffError(status, text)


# A call on small tensors is bound by what happens here, so the wrappers below check all tensors in one
# expression and only go through _require, which words the error, when something is wrong; addresses and
# the stream are passed as plain integers, and outputs are made like an input of the same shape.
# (dd_verify on the tiny workload, host side of a call: 23.2 us at first, 12.9 so; attention 14.9 and 8.3.)
# Calls on device tensors on the current stream go through _fast, which does the same natively (5.7 us, the
# launch itself included) and returns None for whatever it does not take, so that every error is worded here.

_BF16, _I32, _U8, _F32 = torch.bfloat16, torch.int32, torch.uint8, torch.float32
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream_ptr(stream):
    """The given stream, or the current stream of the current device, as an integer."""
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None or _device is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_device())


def _made_on(stream):
    """Within this, outputs are made as memory of the stream that the call runs on, as torch's own operators make theirs: the current
    stream's may still be read there.  (Whoever reads an output on another stream says so to torch, with Tensor.record_stream.)"""
    if stream is None:
        return contextlib.nullcontext()
    # (anything with a cuda_stream will do: another library's stream)
    return torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(stream.cuda_stream))


def _ptr(t):
    return None if t is None else t.data_ptr()


def _fits(t, dtype, shape, cuda):
    return isinstance(t, Tensor) and t.dtype is dtype and t.shape == shape and t.is_cuda is cuda and t.is_contiguous()


def _require(t, dtype, shape, cuda, name):
    if not isinstance(t, Tensor):
        raise TypeError(f"{name}: expected a torch.Tensor")
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{name}: expected contiguous {dtype} of shape {tuple(shape)}, "
                         f"got {t.dtype} {tuple(t.shape)}")
    if t.is_cuda != cuda:
        raise ValueError(f"{name}: expected a {'device' if cuda else 'host'} tensor")


def bidir_attention(q, k, v, out=None, scale=None, stream=None, host=False):
    """dd_bidir_attention (dd_bidir_attention_host if host=True).

    q, k, v: [B,H,N,D] torch.bfloat16.  Returns out (allocated if None)."""
    if _fast is not None and stream is None and not host:
        r = _fast.attention(_addresses(_lib or lib())["dd_bidir_attention"], q, k, v, out, scale)
        if r is not None:
            if type(r) is int:
                _check(r)
            return r
    shape = q.shape
    B, H, N, D = shape
    cuda = not host
    if not (_fits(q, _BF16, shape, cuda) and _fits(k, _BF16, shape, cuda) and _fits(v, _BF16, shape, cuda)):
        for name, t in (("q", q), ("k", k), ("v", v)):
            _require(t, _BF16, (B, H, N, D), cuda, name)
    if out is None:
        with _made_on(stream):
            out = torch.empty_like(q)
    elif not _fits(out, _BF16, shape, cuda):
        _require(out, _BF16, (B, H, N, D), cuda, "out")
    if scale is None:
        scale = float(D) ** -0.5
    L = _lib or lib()
    fn = L.dd_bidir_attention_host if host else L.dd_bidir_attention
    status = fn(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), B, H, N, D, float(scale), _stream_ptr(stream))
    if status:
        _check(status)
    return out


def block_attention(q, k, v, kv_len=None, layout="bhnd", out=None, scale=None, stream=None):
    """dd_block_attention: a block of Nq queries over Nkv stored keys and values.

    layout "bhnd": q [B,H,Nq,D], k, v [B,H,Nkv,D]; "bnhd": q [B,Nq,H,D], k, v [B,Nkv,H,D];
    torch.bfloat16 device tensors.  kv_len: int32 [B] device tensor (valid keys per sequence)
    or None.  Returns out (allocated if None), in the layout of q."""
    if _fast is not None and stream is None and (layout == "bhnd" or layout == "bnhd"):
        r = _fast.block(_addresses(_lib or lib())["dd_block_attention"], q, k, v, kv_len,
                        DD_LAYOUT_BHND if layout == "bhnd" else DD_LAYOUT_BNHD, out, scale)
        if r is not None:
            if type(r) is int:
                _check(r)
            return r
    shape = q.shape
    if layout == "bhnd":
        B, H, Nq, D = shape
        Nkv = k.shape[2]
        kshape = (B, H, Nkv, D)
    elif layout == "bnhd":
        B, Nq, H, D = shape
        Nkv = k.shape[1]
        kshape = (B, Nkv, H, D)
    else:
        raise ValueError("layout: 'bhnd' or 'bnhd'")
    if not (_fits(q, _BF16, shape, True) and _fits(k, _BF16, kshape, True) and _fits(v, _BF16, kshape, True)):
        _require(q, _BF16, tuple(shape), True, "q")
        _require(k, _BF16, kshape, True, "k")
        _require(v, _BF16, kshape, True, "v")
    if kv_len is not None and not _fits(kv_len, _I32, (B,), True):
        _require(kv_len, _I32, (B,), True, "kv_len")
    if out is None:
        with _made_on(stream):
            out = torch.empty_like(q)
    elif not _fits(out, _BF16, shape, True):
        _require(out, _BF16, tuple(shape), True, "out")
    if scale is None:
        scale = float(D) ** -0.5
    status = (_lib or lib()).dd_block_attention(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), B, H, Nq, Nkv, D, _ptr(kv_len),
        DD_LAYOUT_BHND if layout == "bhnd" else DD_LAYOUT_BNHD, float(scale), _stream_ptr(stream))
    if status:
        _check(status)
    return out


def _decision_inputs(tokens, mask_flags, shape, cuda):
    if not (_fits(tokens, _I32, shape, cuda) and _fits(mask_flags, _U8, shape, cuda)):
        _require(tokens, _I32, shape, cuda, "tokens")
        _require(mask_flags, _U8, shape, cuda, "mask_flags")


def _decision_outputs(out_tokens, out_mask, out_score, want_score, tokens, mask_flags, like, shape, host, score_name, stream):
    """The three outputs of shape [B,P]: made where they are None (on the call's stream), checked where they are given."""
    cuda = not host
    near = cuda and tokens.device == like.device and mask_flags.device == like.device

    def make(source, dtype):
        with _made_on(stream):
            return torch.empty_like(source, dtype=dtype) if near else torch.empty(shape, dtype=dtype, device=like.device, pin_memory=host)

    if out_tokens is None:
        out_tokens = make(tokens, _I32)
    elif not _fits(out_tokens, _I32, shape, cuda):
        _require(out_tokens, _I32, shape, cuda, "out_tokens")
    if out_mask is None:
        out_mask = make(mask_flags, _U8)
    elif not _fits(out_mask, _U8, shape, cuda):
        _require(out_mask, _U8, shape, cuda, "out_mask")
    if out_score is None:
        if want_score:
            out_score = make(tokens, _F32)
    elif not _fits(out_score, _F32, shape, cuda):
        _require(out_score, _F32, shape, cuda, score_name)
    return out_tokens, out_mask, out_score


def verify(drafter_logits, verifier_logits, tokens, mask_flags, mode, tau, k, seed,
           out_tokens=None, out_mask=None, out_score=None, want_score=True, stream=None, host=False,
           static_scratch=False):
    """dd_verify (dd_verify_host if host=True; dd_verify_static, the variant that allocates
    nothing, if static_scratch=True and every output tensor is passed in).

    Returns (out_tokens int32 [B,P], out_mask uint8 [B,P], out_score float32 [B,P] or None)."""
    if _fast is not None and stream is None and not host:
        r = _fast.verify(_addresses(_lib or lib())["dd_verify_static" if static_scratch else "dd_verify"], drafter_logits,
                         verifier_logits, tokens, mask_flags, mode, tau, k, seed, out_tokens, out_mask, out_score, want_score)
        if r is not None:
            if type(r) is int:
                _check(r)
            return r
    B, P, V = full = verifier_logits.shape
    cuda = not host
    if not _fits(verifier_logits, _BF16, full, cuda):
        _require(verifier_logits, _BF16, (B, P, V), cuda, "verifier_logits")
    if drafter_logits is not None and not _fits(drafter_logits, _BF16, full, cuda):
        _require(drafter_logits, _BF16, (B, P, V), cuda, "drafter_logits")
    shape = (B, P)
    _decision_inputs(tokens, mask_flags, shape, cuda)
    out_tokens, out_mask, out_score = _decision_outputs(out_tokens, out_mask, out_score, want_score, tokens, mask_flags,
                                                        verifier_logits, shape, host, "out_score", stream)
    L = _lib or lib()
    fn = L.dd_verify_host if host else (L.dd_verify_static if static_scratch else L.dd_verify)
    status = fn(_ptr(drafter_logits), verifier_logits.data_ptr(), tokens.data_ptr(), mask_flags.data_ptr(),
                int(mode), float(tau), int(k), int(seed) & 0xFFFFFFFFFFFFFFFF,
                out_tokens.data_ptr(), out_mask.data_ptr(), _ptr(out_score), B, P, V, _stream_ptr(stream))
    if status:
        _check(status)
    return out_tokens, out_mask, out_score


def lm_head_verify(drafter_hidden, drafter_weight, verifier_hidden, verifier_weight, tokens, mask_flags,
                   mode, tau, k, seed, out_tokens=None, out_mask=None, out_score=None, stream=None):
    """dd_lm_head_verify: the language-model heads fused with the verification algorithm.

    verifier_hidden [B,P,K], verifier_weight [V,K]: torch.bfloat16 device tensors; drafter_hidden,
    drafter_weight: the same shapes, or None in the modes that need the verifier only.
    Returns (out_tokens int32 [B,P], out_mask uint8 [B,P], out_score float32 [B,P])."""
    B, P, K = verifier_hidden.shape
    V = verifier_weight.shape[0]
    if drafter_hidden is not None:
        _require(drafter_hidden, _BF16, (B, P, K), True, "drafter_hidden")
    if drafter_weight is not None:
        _require(drafter_weight, _BF16, (V, K), True, "drafter_weight")
    _require(verifier_hidden, _BF16, (B, P, K), True, "verifier_hidden")
    _require(verifier_weight, _BF16, (V, K), True, "verifier_weight")
    shape = (B, P)
    _decision_inputs(tokens, mask_flags, shape, True)
    out_tokens, out_mask, out_score = _decision_outputs(out_tokens, out_mask, out_score, True, tokens, mask_flags,
                                                        verifier_hidden, shape, False, "out_score", stream)
    status = (_lib or lib()).dd_lm_head_verify(
        _ptr(drafter_hidden), _ptr(drafter_weight), verifier_hidden.data_ptr(), verifier_weight.data_ptr(),
        tokens.data_ptr(), mask_flags.data_ptr(), int(mode), float(tau), int(k), int(seed) & 0xFFFFFFFFFFFFFFFF,
        out_tokens.data_ptr(), out_mask.data_ptr(), out_score.data_ptr(), B, P, K, V, _stream_ptr(stream))
    if status:
        _check(status)
    return out_tokens, out_mask, out_score


def unmask(logits, tokens, mask_flags, tau, k, out_tokens=None, out_mask=None, out_conf=None, stream=None):
    """dd_unmask: one confidence-based unmasking step on logits [B,P,V] (device tensors).

    Returns (out_tokens int32 [B,P], out_mask uint8 [B,P] with 1 = still masked, out_conf float32 [B,P])."""
    if _fast is not None and stream is None:
        r = _fast.unmask(_addresses(_lib or lib())["dd_unmask"], logits, tokens, mask_flags, tau, k, out_tokens, out_mask, out_conf)
        if r is not None:
            if type(r) is int:
                _check(r)
            return r
    B, P, V = full = logits.shape
    if not _fits(logits, _BF16, full, True):
        _require(logits, _BF16, (B, P, V), True, "logits")
    shape = (B, P)
    _decision_inputs(tokens, mask_flags, shape, True)
    out_tokens, out_mask, out_conf = _decision_outputs(out_tokens, out_mask, out_conf, True, tokens, mask_flags,
                                                       logits, shape, False, "out_conf", stream)
    status = (_lib or lib()).dd_unmask(logits.data_ptr(), tokens.data_ptr(), mask_flags.data_ptr(), float(tau), int(k),
                                       out_tokens.data_ptr(), out_mask.data_ptr(), out_conf.data_ptr(), B, P, V,
                                       _stream_ptr(stream))
    if status:
        _check(status)
    return out_tokens, out_mask, out_conf


_E4M3 = torch.float8_e4m3fn


def _require_rows(t, shape, name):
    """bf16 [B,N,H,D] on the device, D contiguous, any other strides."""
    if not isinstance(t, Tensor):
        raise TypeError(f"{name}: expected a torch.Tensor")
    if t.dtype != _BF16 or tuple(t.shape) != tuple(shape) or (t.shape[-1] > 1 and t.stride(-1) != 1):
        raise ValueError(f"{name}: expected {_BF16} of shape {tuple(shape)} with contiguous rows, got {t.dtype} {tuple(t.shape)} "
                         f"with strides {tuple(t.stride())}")
    if not t.is_cuda:
        raise ValueError(f"{name}: expected a device tensor")


def _one_device(like, **tensors):
    for name, t in tensors.items():
        if t is not None and t.device != like.device:
            raise ValueError(f"{name}: on {t.device}, expected {like.device}")


def _device_of(like, stream):
    """The tensors' device is the current one within this context; a stream that is given has to be of that device, if it says of which it is."""
    if stream is not None and getattr(stream, "device", like.device) != like.device:
        raise ValueError(f"stream: on {stream.device}, the tensors are on {like.device}")
    return torch.cuda.device(like.device)


def _row_strides(t, head_major=False):
    # a dimension of size 1 has no stride worth the name
    s = [t.stride(i) if t.shape[i] > 1 else 0 for i in range(3)]
    return _Strides(s[0], s[2], s[1]) if head_major else _Strides(s[0], s[1], s[2])


def _rotation(cos, sin, interleaved, like):
    if (cos is None) != (sin is None):
        raise ValueError("cos, sin: both or neither")
    if cos is None:
        return None
    if cos.dim() != 2:
        raise ValueError("cos: expected [positions, dims / 2]")
    _require(cos, _F32, cos.shape, True, "cos")
    _require(sin, _F32, cos.shape, True, "sin")
    _one_device(like, cos=cos, sin=sin)
    return _Rotation(cos.data_ptr(), sin.data_ptr(), cos.shape[0], 2 * cos.shape[1], int(bool(interleaved)))


def _cache_view(cache, page_table, B, like):
    if not isinstance(cache, tuple) or len(cache) != 4:
        raise TypeError("cache: expected a Cache (k, v, k_scale, v_scale)")
    cache = Cache(*cache)
    if not isinstance(cache.k, Tensor):
        raise TypeError("cache.k: expected a torch.Tensor")
    if cache.k.dim() != 4:
        raise ValueError(f"cache.k: expected [num_pages, heads, page_size, D], got {tuple(cache.k.shape)}")
    num_pages, heads, page, D = shape = tuple(cache.k.shape)
    _require(cache.k, _E4M3, shape, True, "cache.k")
    _require(cache.v, _E4M3, shape, True, "cache.v")
    _require(cache.k_scale, _F32, (num_pages, heads), True, "cache.k_scale")
    _require(cache.v_scale, _F32, (num_pages, heads), True, "cache.v_scale")
    if not isinstance(page_table, Tensor) or page_table.dim() != 2:
        raise ValueError("page_table: expected [B, max_pages]")
    _require(page_table, _I32, (B, page_table.shape[1]), True, "page_table")
    _one_device(like, **{"cache.k": cache.k, "cache.v": cache.v, "cache.k_scale": cache.k_scale, "cache.v_scale": cache.v_scale,
                         "page_table": page_table})
    return _Cache(cache.k.data_ptr(), cache.v.data_ptr(), cache.k_scale.data_ptr(), cache.v_scale.data_ptr(), page_table.data_ptr(),
                  num_pages, page_table.shape[1], page, heads, D)


def _lengths(t, B, name, like):
    if t is not None:
        _require(t, _I32, (B,), True, name)
        _one_device(like, **{name: t})
    return _ptr(t)


def _weight(t, D, name, like):
    if t is not None:
        _require(t, _BF16, (D,), True, name)
        _one_device(like, **{name: t})
    return _ptr(t)


def new_cache(num_pages, heads, page_size, D, device="cuda"):
    """An empty Cache: zero bytes under scales of 1."""
    shape = (num_pages, heads, page_size, D)
    return Cache(torch.zeros(shape, dtype=torch.uint8, device=device).view(_E4M3), torch.zeros(shape, dtype=torch.uint8, device=device).view(_E4M3),
                 torch.ones(num_pages, heads, device=device), torch.ones(num_pages, heads, device=device))


def qk_norm_rope(q, k=None, q_weight=None, k_weight=None, eps=1e-6, cos=None, sin=None, start=None, interleaved=False,
                 layout="bnhd", out_q=None, out_k=None, stream=None):
    """dd_qk_norm_rope: norms of queries and keys for each head, and their rotation by position.

    q [B,N,H,D], k [B,N,Hkv,D] (or None): torch.bfloat16 device tensors with contiguous rows (views of a projection).
    q_weight, k_weight: bfloat16 [D] or None (no norm).  cos, sin: float32 [positions, dims / 2] or None (no rotation);
    row i of sequence b stands at position start[b] + i (start: int32 [B], None: 0).  layout: of the outputs, "bnhd" or "bhnd".
    Returns (out_q, out_k), contiguous; out_k is None without k."""
    if layout not in ("bnhd", "bhnd"):
        raise ValueError("layout: 'bhnd' or 'bnhd'")
    code = DD_LAYOUT_BNHD if layout == "bnhd" else DD_LAYOUT_BHND
    if _fast is not None and stream is None:
        r = _fast.norm_rope(_addresses(_lib or lib())["dd_qk_norm_rope"], q, k, q_weight, k_weight, eps, cos, sin, start, interleaved, code,
                            out_q, out_k)
        if r is not None:
            if type(r) is int:
                _check(r)
            return r
    B, N, H, D = q.shape
    _require_rows(q, (B, N, H, D), "q")
    Hkv = 0
    if k is not None:
        Hkv = k.shape[2] if k.dim() == 4 else 0
        _require_rows(k, (B, N, Hkv, D), "k")
        _one_device(q, k=k)
    wq, wk = _weight(q_weight, D, "q_weight", q), _weight(k_weight, D, "k_weight", q)
    rotation = _rotation(cos, sin, interleaved, q)
    st = _lengths(start, B, "start", q)

    def output(given, heads, name):
        shape = (B, N, heads, D) if layout == "bnhd" else (B, heads, N, D)
        if given is None:
            return torch.empty(shape, dtype=_BF16, device=q.device)
        _require(given, _BF16, shape, True, name)
        _one_device(q, **{name: given})
        return given

    if k is None and out_k is not None:
        raise ValueError("out_k: given without k")
    with _device_of(q, stream), _made_on(stream):
        out_q = output(out_q, H, "out_q")
        if k is not None:
            out_k = output(out_k, Hkv, "out_k")
        status = (_lib or lib()).dd_qk_norm_rope(
            q.data_ptr(), ctypes.byref(_row_strides(q)), H, _ptr(k), None if k is None else ctypes.byref(_row_strides(k)), Hkv, wq, wk,
            float(eps), None if rotation is None else ctypes.byref(rotation), st, out_q.data_ptr(), _ptr(out_k), B, N, D, code,
            _stream_ptr(stream))
    if status:
        _check(status)
    return out_q, out_k


def cache_append(k, v, cache, page_table, start, count=None, kv_len=None, k_weight=None, eps=1e-6, cos=None, sin=None,
                 interleaved=False, stream=None):
    """dd_cache_append: new keys (normed with k_weight, rotated by cos, sin) and values into a paged 8-bit cache, in place.

    k, v [B,N,heads,D]: torch.bfloat16 device tensors with contiguous rows.  cache: a Cache; page_table: int32 [B, max_pages];
    start: int32 [B], the position of each sequence's first new token; count: int32 [B], how many of the N are new (None: all);
    kv_len: int32 [B], how many tokens each sequence holds before the call (None: start): those that are not among the new
    positions stay.  Returns cache."""
    if _fast is not None and stream is None:
        r = _fast.append(_addresses(_lib or lib())["dd_cache_append"], k, v, cache, page_table, start, count, kv_len, k_weight, eps, cos, sin,
                         interleaved)
        if r is not None:
            if type(r) is int:
                _check(r)
            return r
    B, N, heads, D = k.shape
    view = _cache_view(cache, page_table, B, k)
    _require_rows(k, (B, N, view.heads, view.D), "k")
    _require_rows(v, (B, N, view.heads, view.D), "v")
    _one_device(k, v=v)
    if start is None:
        raise TypeError("start: expected a torch.Tensor")
    weight = _weight(k_weight, D, "k_weight", k)
    rotation = _rotation(cos, sin, interleaved, k)
    st, n, held = _lengths(start, B, "start", k), _lengths(count, B, "count", k), _lengths(kv_len, B, "kv_len", k)
    with _device_of(k, stream):
        status = (_lib or lib()).dd_cache_append(
            k.data_ptr(), ctypes.byref(_row_strides(k)), v.data_ptr(), ctypes.byref(_row_strides(v)), ctypes.byref(view), st, n, held, weight,
            float(eps), None if rotation is None else ctypes.byref(rotation), B, N, _stream_ptr(stream))
    if status:
        _check(status)
    return cache


def cached_attention(q, cache, page_table, kv_len, layout="bnhd", out=None, scale=None, stream=None):
    """dd_cached_attention: queries over a paged 8-bit cache; query heads may share key heads.

    layout "bnhd": q [B,Nq,H,D]; "bhnd": q [B,H,Nq,D]; torch.bfloat16 device tensor with contiguous rows.  cache: a Cache, of whose
    heads H is a multiple; page_table: int32 [B, max_pages]; kv_len: int32 [B], the tokens of each sequence.
    Returns out (allocated if None), in the layout of q.  The workspace is taken from torch's allocator for each call, on the stream
    that the call runs on."""
    if layout not in ("bnhd", "bhnd"):
        raise ValueError("layout: 'bhnd' or 'bnhd'")
    head_major = layout == "bhnd"
    if _fast is not None and stream is None:
        at = _addresses(_lib or lib())
        r = _fast.cached(at["dd_cached_attention"], at["dd_cached_attention_workspace_bytes"], q, cache, page_table, kv_len,
                         DD_LAYOUT_BHND if head_major else DD_LAYOUT_BNHD, scale, out)
        if r is not None:
            if type(r) is int:
                _check(r)
            return r
    B, Nq, H, D = q.shape
    if head_major:
        Nq, H = H, Nq
    view = _cache_view(cache, page_table, B, q)
    if D != view.D:
        raise ValueError(f"q: heads of {D}, the cache's are of {view.D}")
    _require_rows(q, q.shape, "q")
    if kv_len is None:
        raise TypeError("kv_len: expected a torch.Tensor")
    lens = _lengths(kv_len, B, "kv_len", q)
    if out is not None:
        _require_rows(out, q.shape, "out")
        _one_device(q, out=out)
        if any(n > 1 and s == 0 for n, s in zip(out.shape, out.stride())):
            raise ValueError("out: rows that share memory")
    if scale is None:
        scale = float(D) ** -0.5
    L = _lib or lib()
    with _device_of(q, stream), _made_on(stream):                # (the workspace too)
        if out is None:
            out = torch.empty(q.shape, dtype=_BF16, device=q.device)
        need = L.dd_cached_attention_workspace_bytes(B, H, Nq, ctypes.byref(view))
        work = torch.empty(max(need, 16), dtype=_U8, device=q.device)
        status = L.dd_cached_attention(
            q.data_ptr(), ctypes.byref(_row_strides(q, head_major)), ctypes.byref(view), lens, out.data_ptr(),
            ctypes.byref(_row_strides(out, head_major)), B, H, Nq, float(scale), work.data_ptr(), need, _stream_ptr(stream))
    if status:
        _check(status)
    return out


def attention_status() -> int:
    return int(lib().dd_attention_status())


def verify_status() -> int:
    return int(lib().dd_verify_status())


def launch_count() -> int:
    return int(lib().dd_launch_count())


def debug_set_max_ctas(n: int):
    """Test hook: cap the grid of the streaming verify kernel (0 = no cap)."""
    _check(lib().dd_debug_set_max_ctas(int(n)))


def clear_status():
    """Re-arms the kernels' health words on the current device after a recorded timeout."""
    _check(lib().dd_clear_status())


def debug_expire_wait(which: int, stream=None):
    """Test hook: records an expired wait for the attention kernel (0) or dd_verify (1)."""
    _check(lib().dd_debug_expire_wait(int(which), _stream_ptr(stream)))


def release():
    _check(lib().dd_release())


def version() -> int:
    return int(lib().dd_version())


def verify_workspace_bytes(B, P, V) -> int:
    return int(lib().dd_verify_workspace_bytes(B, P, V))
