"""ctypes binding of the operators that read a KV cache and make it smaller (``include/dynakv.h``): attention over a window and its backward,
the cache in 4 bits, eviction.  Same conventions as ``train.py``: torch CUDA (ROCm) tensors in, the current stream, ``LmheadError`` on a
negative status; a tensor of the wrong type or shape, or on another device than the current one, raises ``ValueError`` before the call.
Nothing is computed here.

Queries, keys, values and outputs are 4-D tensors [sequence, slot, head, channel] with any strides that the descriptor names: a cache that
keeps each head's tokens together is passed as its ``transpose(1, 2)``.
"""
from __future__ import annotations

import ctypes as C
import math

import torch

from .binding import LmheadError, _check, load_library
from .train import _DTYPES, _TORCH, _arg, _bad, _device, _refuse, _stream

EVICT_PLANES = 4


class AttnLayout(C.Structure):
    _fields_ = [("seq", C.c_int64), ("slot", C.c_int64), ("head", C.c_int64)]


class AttnDesc(C.Structure):
    _sizes = None
    _fields_ = [
        ("B", C.c_int32), ("Tq", C.c_int32), ("Tk", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("D", C.c_int32),
        ("window", C.c_int32), ("sinks", C.c_int32), ("dtype", C.c_int32), ("scale", C.c_float), ("flags", C.c_uint32),
        ("reserved", C.c_int32), ("q", AttnLayout), ("k", AttnLayout), ("v", AttnLayout), ("o", AttnLayout),
    ]


class EvictDesc(C.Structure):
    _fields_ = [
        ("B", C.c_int32), ("T", C.c_int32), ("Hkv", C.c_int32), ("keep", C.c_int32), ("sinks", C.c_int32), ("recent", C.c_int32),
        ("flags", C.c_int32), ("reserved", C.c_int32),
    ]


class _Plane(C.Structure):
    _fields_ = [("data", C.c_void_p), ("seq", C.c_int64), ("slot", C.c_int64), ("head", C.c_int64), ("bytes", C.c_int64)]


_ready = None


def _lib():
    global _ready
    if _ready is None:
        lib = load_library()
        vp, i32, f32, sz = C.c_void_p, C.c_int32, C.c_float, C.c_size_t
        ap, ep, pp = C.POINTER(AttnDesc), C.POINTER(EvictDesc), C.POINTER(_Plane)
        lib.attn_validate_desc.restype = C.c_int
        lib.attn_validate_desc.argtypes = [ap]
        lib.attn_workspace_bytes.restype = sz
        lib.attn_workspace_bytes.argtypes = [ap]
        lib.attn_fwd.restype = C.c_int
        lib.attn_fwd.argtypes = [ap, vp, vp, vp, vp, vp, vp, vp, vp, f32, vp, sz, vp]
        lib.attn_bwd_workspace_bytes.restype = sz
        lib.attn_bwd_workspace_bytes.argtypes = [ap]
        lib.attn_bwd.restype = C.c_int
        lib.attn_bwd.argtypes = [ap, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.kv4_store.restype = C.c_int
        lib.kv4_store.argtypes = [ap, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.kv4_attn.restype = C.c_int
        lib.kv4_attn.argtypes = [ap, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, f32, vp, sz, vp]
        lib.evict_validate_desc.restype = C.c_int
        lib.evict_validate_desc.argtypes = [ep]
        lib.evict_workspace_bytes.restype = sz
        lib.evict_workspace_bytes.argtypes = [ep]
        lib.cache_evict.restype = C.c_int
        lib.cache_evict.argtypes = [ep, pp, i32, vp, vp, vp, vp, vp, sz, vp]
        _ready = lib
    return _ready


# ---- attention ------------------------------------------------------------------------------------------------------


def attn_layout(t):
    """Strides (sequence, slot, head) of a [B, T, H, D] tensor.  Those of dimensions with one element can be anything in torch: they are
    taken as if the dimension had more, dense behind the others."""
    if t.dim() != 4:
        raise ValueError(f"[sequence, slot, head, channel] expected, got {tuple(t.shape)}")
    s, n = list(t.stride()[:3]), t.shape
    span = max([n[3]] + [abs(s[i]) * n[i] for i in range(3) if n[i] > 1])
    return tuple(s[i] if n[i] > 1 else (n[3] if i == 1 else span) for i in range(3))


def make_attn_desc(B, Tq, Tk, Hq, Hkv, D, dtype, window=0, sinks=0, scale=None, q=None, k=None, v=None, o=None) -> AttnDesc:
    """Layouts are (sequence, slot, head) strides in elements; by default tensors are dense [B, T, H, D].  scale: default D ** -0.5."""
    def layout(x, T, H):
        return AttnLayout(*((T * H * D, H * D, D) if x is None else x))
    return AttnDesc(B=B, Tq=Tq, Tk=Tk, Hq=Hq, Hkv=Hkv, D=D, window=window, sinks=sinks, dtype=_DTYPES.get(dtype, dtype),
                    scale=(D ** -0.5 if D > 0 else 1.0) if scale is None else scale, flags=0, reserved=0,
                    q=layout(q, Tq, Hq), k=layout(k, Tk, Hkv), v=layout(v, Tk, Hkv), o=layout(o, Tq, Hq))


def attn_validate_desc(desc: AttnDesc) -> int:
    return int(_lib().attn_validate_desc(C.byref(desc)))


def attn_workspace_bytes(desc: AttnDesc) -> int:
    return int(_lib().attn_workspace_bytes(C.byref(desc)))


def attn_bwd_workspace_bytes(desc: AttnDesc) -> int:
    return int(_lib().attn_bwd_workspace_bytes(C.byref(desc)))


def _merges(n, want):
    """Whether dimensions `n` are those of `want`, some of them neighbours taken together: dense tensors of either are the same memory."""
    at = 0
    for size in n:
        have = 1
        while have < size and at < len(want):
            have *= want[at]
            at += 1
        if have != size:
            return False
    return all(x == 1 for x in want[at:])


def _block(t, name, dtype, n, want, device):
    """Device pointer of a dense tensor of the sizes `want` (`n` elements), of one that has more where that moves nothing of what is used (more sequences
    do not, more slots would move every head but the first), or of a flat buffer with room for them; None for None."""
    if t is None:
        return None
    if t.dtype is dtype and t.get_device() == device and t.is_contiguous():
        sizes = t.shape
        if sizes == want:
            return t.data_ptr()
        inner = min(len(sizes), len(want)) - 1      # dimensions behind the first one, which may be larger
        if t.numel() >= n and inner >= 0 and sizes[len(sizes) - inner:] == want[len(want) - inner:] or t.numel() == n and _merges(sizes, want):
            return t.data_ptr()
        if (len(sizes) == len(want) and all(a >= b for a, b in zip(sizes, want))
                and all(a == math.prod(want[i + 1:]) or want[i] == 1 for i, a in enumerate(t.stride()))):
            return t.data_ptr()
    return _refuse(t, name, dtype, device, f"{tuple(want)} contiguous expected, got {tuple(t.shape)}")


class _Heads:
    """What a [B, T, H, D] tensor of a call has to be."""

    def __init__(self, B, T, H, D, x):
        self.shape, self.strides, self.n = torch.Size((B, T, H, D)), (x.seq, x.slot, x.head, 1), B * T * H * D
        dense = (T * H * D, H * D, D)
        self.dense = all(a == b or n == 1 for a, b, n in zip(self.strides, dense, self.shape))


class _Sizes:
    """What the checks of a descriptor's tensors compare with, made once for its contents.  Nothing here refers to the descriptor: a copy of it
    has these too."""

    def __init__(self, desc, raw):
        self.raw, d = raw, desc
        self.status = int(_lib().attn_validate_desc(C.byref(desc)))
        if self.status:
            return
        self.dtype, self.B = _TORCH[d.dtype], d.B
        B, Tq, Tk, Hq, Hkv, D = d.B, d.Tq, d.Tk, d.Hq, d.Hkv, d.D
        self.q, self.o = _Heads(B, Tq, Hq, D, d.q), _Heads(B, Tq, Hq, D, d.o)
        self.k, self.v = _Heads(B, Tk, Hkv, D, d.k), _Heads(B, Tk, Hkv, D, d.v)
        self.k_new, self.v_new = _Heads(B, Tq, Hkv, D, d.k), _Heads(B, Tq, Hkv, D, d.v)      # rows for a cache in 4 bits
        rows = B * Hkv * Tk
        self.lse, self.weight, self.codes, self.scales = B * Hq * Tq, rows, rows * (D // 2), rows * (D // 32)
        self.lse_shape, self.weight_shape = torch.Size((B, Hq, Tq)), torch.Size((B, Hkv, Tk))
        self.codes_shape, self.scales_shape = torch.Size((B, Hkv, Tk, D // 2)), torch.Size((B, Hkv, Tk, D // 32))
        self.odd = D % 32 != 0      # no cache in 4 bits has such rows, and the library refuses them


def _sizes(desc, where):
    """The descriptor's own refusal comes first: the checks of tensors rely on its sizes."""
    raw = bytes(desc)
    sizes = desc._sizes
    if sizes is None or sizes.raw != raw:
        sizes = desc._sizes = _Sizes(desc, raw)
    if sizes.status:
        raise LmheadError(sizes.status, where)
    return sizes


def _heads(t, name, s, want, device):
    """Device pointer of a [B, T, H, D] tensor with the shape and strides that are wanted (it may have more of each), or of a dense buffer where
    they are dense."""
    if t.dtype is s.dtype and t.get_device() == device:
        n = t.shape
        if want.dense and t.is_contiguous() and (n == want.shape or t.numel() == want.n and _merges(n, want.shape)):
            return t.data_ptr()
        st = t.stride()
        if n == want.shape and st == want.strides:
            return t.data_ptr()
        if len(n) == 4 and all(a >= b for a, b in zip(n, want.shape)) and all(a == b or c == 1 for a, b, c in zip(st, want.strides, want.shape)):
            return t.data_ptr()
        _bad(name, f"{tuple(want.shape)} with strides {want.strides} expected, got {tuple(n)} with {tuple(st)}")
    return _refuse(t, name, s.dtype, device, "")


def attn_fwd(desc, q, k, v, len_q, len_k, out, lse, weight, decay, ws) -> None:
    """len_q, len_k: int32[B], or None where every slot is valid; lse, weight: or None."""
    s, dev, i32, f32 = _sizes(desc, "attn_fwd"), _device(), torch.int32, torch.float32
    rc = _lib().attn_fwd(
        C.byref(desc), _heads(q, "q", s, s.q, dev), _heads(k, "k", s, s.k, dev), _heads(v, "v", s, s.v, dev), _arg(len_q, "len_q", i32, s.B, dev),
        _arg(len_k, "len_k", i32, s.B, dev), _heads(out, "out", s, s.o, dev), _block(lse, "lse", f32, s.lse, s.lse_shape, dev),
        _block(weight, "weight", f32, s.weight, s.weight_shape, dev), decay, _arg(ws, "ws", torch.uint8, 0, dev), ws.numel(), _stream(dev))
    _check(rc, "attn_fwd")


def attn_bwd(desc, q, k, v, len_q, len_k, out, lse, g_out, dq, dk, dv, ws) -> None:
    s, dev, i32 = _sizes(desc, "attn_bwd"), _device(), torch.int32
    rc = _lib().attn_bwd(
        C.byref(desc), _heads(q, "q", s, s.q, dev), _heads(k, "k", s, s.k, dev), _heads(v, "v", s, s.v, dev), _arg(len_q, "len_q", i32, s.B, dev),
        _arg(len_k, "len_k", i32, s.B, dev), _heads(out, "out", s, s.o, dev), _block(lse, "lse", torch.float32, s.lse, s.lse_shape, dev),
        _heads(g_out, "g_out", s, s.o, dev), _heads(dq, "dq", s, s.q, dev), _heads(dk, "dk", s, s.k, dev), _heads(dv, "dv", s, s.v, dev),
        _arg(ws, "ws", torch.uint8, 0, dev), ws.numel(), _stream(dev))
    _check(rc, "attn_bwd")


# ---- the cache in 4 bits --------------------------------------------------------------------------------------------


def _cache(s, k_codes, k_scales, v_codes, v_scales, dev):
    u8 = torch.uint8
    return (_block(k_codes, "k_codes", u8, s.codes, s.codes_shape, dev), _block(k_scales, "k_scales", u8, s.scales, s.scales_shape, dev),
            _block(v_codes, "v_codes", u8, s.codes, s.codes_shape, dev), _block(v_scales, "v_scales", u8, s.scales, s.scales_shape, dev))


def kv4_store(desc, k, v, len_q, len_k, k_codes, k_scales, v_codes, v_scales, ws) -> None:
    """k, v: the new tokens' rows, [B, Tq, Hkv, D]."""
    s, dev, i32 = _sizes(desc, "kv4_store"), _device(), torch.int32
    if s.odd:
        raise LmheadError(-2, "kv4_store")
    rc = _lib().kv4_store(
        C.byref(desc), _heads(k, "k", s, s.k_new, dev), _heads(v, "v", s, s.v_new, dev), _arg(len_q, "len_q", i32, s.B, dev),
        _arg(len_k, "len_k", i32, s.B, dev), *_cache(s, k_codes, k_scales, v_codes, v_scales, dev), _arg(ws, "ws", torch.uint8, 0, dev),
        ws.numel(), _stream(dev))
    _check(rc, "kv4_store")


def kv4_attn(desc, q, k_codes, k_scales, v_codes, v_scales, len_q, len_k, out, lse, weight, decay, ws) -> None:
    s, dev, i32, f32 = _sizes(desc, "kv4_attn"), _device(), torch.int32, torch.float32
    if s.odd:
        raise LmheadError(-2, "kv4_attn")
    rc = _lib().kv4_attn(
        C.byref(desc), _heads(q, "q", s, s.q, dev), *_cache(s, k_codes, k_scales, v_codes, v_scales, dev), _arg(len_q, "len_q", i32, s.B, dev),
        _arg(len_k, "len_k", i32, s.B, dev), _heads(out, "out", s, s.o, dev), _block(lse, "lse", f32, s.lse, s.lse_shape, dev),
        _block(weight, "weight", f32, s.weight, s.weight_shape, dev), decay, _arg(ws, "ws", torch.uint8, 0, dev), ws.numel(), _stream(dev))
    _check(rc, "kv4_attn")


# ---- eviction -------------------------------------------------------------------------------------------------------


def make_evict_desc(B, T, Hkv, keep, sinks=0, recent=0) -> EvictDesc:
    return EvictDesc(B=B, T=T, Hkv=Hkv, keep=keep, sinks=sinks, recent=recent, flags=0, reserved=0)


def evict_validate_desc(desc: EvictDesc) -> int:
    return int(_lib().evict_validate_desc(C.byref(desc)))


def evict_workspace_bytes(desc: EvictDesc) -> int:
    return int(_lib().evict_workspace_bytes(C.byref(desc)))


class CachePlanes:
    """The tensors of a cache, [sequence, slot, head, channel] each with any strides, as cache_evict takes them.  It holds on to them."""

    def __init__(self, tensors):
        self.tensors = [t.detach() for t in tensors]
        self.array = (_Plane * max(len(self.tensors), 1))()
        self.device = None
        for i, t in enumerate(self.tensors):
            name = f"plane {i}"
            if not t.is_cuda:
                _bad(name, "device tensor expected")
            if t.dim() != 4 or t.stride(3) != 1 and t.shape[3] != 1:
                _bad(name, "[sequence, slot, head, channel] with dense channels expected")
            if self.device is None:
                self.device = t.get_device()
            elif t.get_device() != self.device:
                _bad(name, f"on cuda:{t.get_device()}, others on cuda:{self.device}")
            seq, slot, head = (x * t.element_size() for x in attn_layout(t))
            self.array[i] = _Plane(t.data_ptr() or None, seq, slot, head, t.shape[3] * t.element_size())
        self.storages = [t.untyped_storage() for t in self.tensors]
        self.addresses = [s.data_ptr() for s in self.storages]

    def __len__(self):
        return len(self.tensors)


def make_cache_planes(tensors) -> CachePlanes:
    return CachePlanes(tensors)


def cache_evict(desc, planes: CachePlanes, weight, lens, lens_out, kept, ws) -> None:
    """lens: int32[B], or None where every slot is valid."""
    rc = _lib().evict_validate_desc(C.byref(desc))
    if rc != 0:
        raise LmheadError(rc, "cache_evict")
    lib, dev, i32 = _lib(), _device(), torch.int32
    if planes.device is not None and planes.device != dev:
        _bad("planes", f"on cuda:{planes.device}, the current device is cuda:{dev}")
    for i, t in enumerate(planes.tensors):
        if t.shape[0] < desc.B or t.shape[1] < desc.T or t.shape[2] < desc.Hkv:
            _bad(f"plane {i}", f"[{desc.B}, {desc.T}, {desc.Hkv}, .] expected, got {tuple(t.shape)}")
        if planes.storages[i].data_ptr() != planes.addresses[i]:
            _bad(f"plane {i}", "its storage was resized after the list was made")
    rows = desc.B * desc.Hkv
    rc = lib.cache_evict(
        C.byref(desc), planes.array, len(planes),
        _block(weight, "weight", torch.float32, rows * desc.T, torch.Size((desc.B, desc.Hkv, desc.T)), dev),
        _arg(lens, "lens", i32, desc.B, dev), _arg(lens_out, "lens_out", i32, desc.B, dev),
        _block(kept, "kept", i32, rows * desc.keep, torch.Size((desc.B, desc.Hkv, desc.keep)), dev), _arg(ws, "ws", torch.uint8, 0, dev),
        ws.numel(), _stream(dev))
    _check(rc, "cache_evict")
