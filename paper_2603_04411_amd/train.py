"""ctypes binding of the operators around the head in a training step (``include/lmhead.h``): preference loss, embedding lookup and its
gradient, gradient norm and clipping.  Same conventions as ``binding.py``: torch CUDA (ROCm) tensors in, the current stream,
``LmheadError`` on a negative status; a tensor of the wrong type, too small, not contiguous or on another device than the current one raises
``ValueError`` before the call.  Nothing is computed here.
"""
from __future__ import annotations

import ctypes as C

import torch

from .binding import FLAG_ACCUM_DW, LMHEAD_BF16, LMHEAD_F32, LmheadError, _check, load_library

_DTYPES = {"bf16": LMHEAD_BF16, "f32": LMHEAD_F32}
_TORCH = {LMHEAD_BF16: torch.bfloat16, LMHEAD_F32: torch.float32}
_CODES = {torch.bfloat16: LMHEAD_BF16, torch.float32: LMHEAD_F32}


class PreferenceParams(C.Structure):
    _fields_ = [
        ("loss", C.c_int32), ("pairs", C.c_int32), ("mean", C.c_int32), ("weights", C.c_int32),
        ("beta", C.c_float), ("margin", C.c_float), ("margin_scale", C.c_float), ("smoothing", C.c_float),
        ("nll_coef", C.c_float), ("reserved", C.c_int32),
    ]


class EmbedDesc(C.Structure):
    _fields_ = [
        ("R", C.c_int32), ("T", C.c_int32), ("d", C.c_int32), ("V", C.c_int32),
        ("dtype", C.c_int32), ("rows", C.c_int32), ("flags", C.c_uint32), ("reserved", C.c_int32),
        ("ldW", C.c_int64), ("ldX", C.c_int64),
    ]


class _Tensor(C.Structure):
    _fields_ = [("data", C.c_void_p), ("n", C.c_int64), ("dtype", C.c_int32), ("reserved", C.c_int32)]


_ready = None


def _lib():
    global _ready
    if _ready is None:
        lib = load_library()
        vp, i32, f32, sz = C.c_void_p, C.c_int32, C.c_float, C.c_size_t
        pp, ep, tp = C.POINTER(PreferenceParams), C.POINTER(EmbedDesc), C.POINTER(_Tensor)
        lib.preference_workspace_bytes.restype = sz
        lib.preference_workspace_bytes.argtypes = [i32, i32, i32]
        lib.preference_loss.restype = C.c_int
        lib.preference_loss.argtypes = [pp, vp, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, sz, vp]
        lib.embed_validate_desc.restype = C.c_int
        lib.embed_validate_desc.argtypes = [ep]
        lib.embed_workspace_bytes.restype = sz
        lib.embed_workspace_bytes.argtypes = [ep]
        lib.embed_fwd.restype = C.c_int
        lib.embed_fwd.argtypes = [ep, vp, vp, vp, f32, vp, vp, sz, vp]
        lib.embed_bwd.restype = C.c_int
        lib.embed_bwd.argtypes = [ep, vp, vp, vp, f32, vp, vp, sz, vp]
        lib.grad_workspace_bytes.restype = sz
        lib.grad_workspace_bytes.argtypes = []
        lib.grad_norm.restype = C.c_int
        lib.grad_norm.argtypes = [tp, i32, vp, vp, sz, vp]
        lib.grad_clip.restype = C.c_int
        lib.grad_clip.argtypes = [tp, tp, i32, f32, f32, vp, vp, sz, vp]
        _ready = lib
    return _ready


def _bad(name, what):
    raise ValueError(f"{name}: {what}")


def _refuse(t, name, dtype, device, rest):
    if not t.is_cuda:
        _bad(name, "device tensor expected")
    if t.dtype is not dtype:
        _bad(name, f"{dtype} expected, got {t.dtype}")
    if t.get_device() != device:
        _bad(name, f"on cuda:{t.get_device()}, the current device is cuda:{device}")
    _bad(name, rest)


def _arg(t, name, dtype, n, device):
    """Device pointer of a dense tensor of at least `n` elements; None for None."""
    if t is None:
        return None
    if t.dtype is dtype and t.get_device() == device and t.numel() >= n and t.is_contiguous():
        return t.data_ptr()
    return _refuse(t, name, dtype, device, f"{n} contiguous elements expected")


def _rows(t, name, dtype, rows, d, ld, device):
    """Device pointer of a [rows x d] matrix with row stride `ld`: a 2-D view with these strides, or a dense buffer that holds it."""
    if t is None or t.dim() != 2 or t.is_contiguous() and ld == t.shape[1]:
        return _arg(t, name, dtype, (rows - 1) * ld + d, device)
    if (t.dtype is dtype and t.get_device() == device and t.shape[0] >= rows and t.shape[1] >= d and t.stride(1) == 1
            and (t.stride(0) == ld or rows == 1)):
        return t.data_ptr()
    return _refuse(t, name, dtype, device, f"[{rows} x {d}] with row stride {ld} expected")


def _device():
    return torch.cuda.current_device()


def _stream(device):
    """The current stream's handle.  (torch.cuda.current_stream() makes an object of it: 2.9 us of a call of 10.)"""
    return torch._C._cuda_getCurrentRawStream(device) or None


# ---- preference loss ------------------------------------------------------------------------------------------------


def make_preference(loss="logistic", pairs="all", mean=False, weights="prompt", beta=0.1, margin=0.0, margin_scale=0.0, smoothing=0.0,
                    nll_coef=0.0) -> PreferenceParams:
    """loss: "logistic" | "hinge" | "squared"; pairs: "all" | "extremes"; weights: "prompt" | "pair" (or the ABI's numbers)."""
    return PreferenceParams(
        loss={"logistic": 0, "hinge": 1, "squared": 2}.get(loss, loss), pairs={"all": 0, "extremes": 1}.get(pairs, pairs),
        mean=int(mean), weights={"prompt": 0, "pair": 1}.get(weights, weights), beta=beta, margin=margin, margin_scale=margin_scale,
        smoothing=smoothing, nll_coef=nll_coef, reserved=0)


def preference_workspace_bytes(P: int, G: int, T: int) -> int:
    return int(_lib().preference_workspace_bytes(P, G, T))


def preference_loss(params, logp, logp_ref, reward, lens, P, G, T, loss, g_logp, ratio, stats, ws) -> None:
    if P < 0 or G < 0 or T < 0:      # as an int32 of the call it might not be
        raise LmheadError(-2, "preference_loss")
    lib, dev, f32 = _lib(), _device(), torch.float32
    R, N = P * G, P * G * T
    rc = lib.preference_loss(
        C.byref(params), _arg(logp, "logp", f32, N, dev), _arg(logp_ref, "logp_ref", f32, N, dev), _arg(reward, "reward", f32, R, dev),
        _arg(lens, "lens", torch.int32, R, dev), P, G, T, _arg(loss, "loss", f32, 1, dev), _arg(g_logp, "g_logp", f32, N, dev),
        _arg(ratio, "ratio", f32, R, dev), _arg(stats, "stats", f32, 4, dev), _arg(ws, "ws", torch.uint8, 0, dev), ws.numel(), _stream(dev))
    _check(rc, "preference_loss")


# ---- embedding ------------------------------------------------------------------------------------------------------


def make_embed_desc(R, T, d, V, dtype, rows=None, ldW=None, ldX=None, flags=0) -> EmbedDesc:
    """dtype: storage type of W; rows: of the rows that are written or whose gradient is given (default: the same)."""
    code = _DTYPES.get(dtype, dtype)
    return EmbedDesc(R=R, T=T, d=d, V=V, dtype=code, rows=code if rows is None else _DTYPES.get(rows, rows), flags=flags, reserved=0,
                     ldW=d if ldW is None else ldW, ldX=d if ldX is None else ldX)


def embed_validate_desc(desc: EmbedDesc) -> int:
    return int(_lib().embed_validate_desc(C.byref(desc)))


def embed_workspace_bytes(desc: EmbedDesc) -> int:
    return int(_lib().embed_workspace_bytes(C.byref(desc)))


def embed_fwd(desc, W, tok, lens, scale, X, ws) -> None:
    """lens: int32[R], or None where every slot is valid."""
    lib, dev, N = _lib(), _device(), desc.R * desc.T
    rc = lib.embed_fwd(
        C.byref(desc), _rows(W, "W", _TORCH.get(desc.dtype), desc.V, desc.d, desc.ldW, dev), _arg(tok, "tok", torch.int32, N, dev),
        _arg(lens, "lens", torch.int32, desc.R, dev), scale, _rows(X, "X", _TORCH.get(desc.rows), N, desc.d, desc.ldX, dev),
        _arg(ws, "ws", torch.uint8, 0, dev), ws.numel(), _stream(dev))
    _check(rc, "embed_fwd")


def embed_bwd(desc, gX, tok, lens, scale, dW, ws) -> None:
    lib, dev, N = _lib(), _device(), desc.R * desc.T
    rc = lib.embed_bwd(
        C.byref(desc), _rows(gX, "gX", _TORCH.get(desc.rows), N, desc.d, desc.ldX, dev), _arg(tok, "tok", torch.int32, N, dev),
        _arg(lens, "lens", torch.int32, desc.R, dev), scale, _arg(dW, "dW", torch.float32, desc.V * desc.d, dev),
        _arg(ws, "ws", torch.uint8, 0, dev), ws.numel(), _stream(dev))
    _check(rc, "embed_bwd")


# ---- gradient norm and clipping -------------------------------------------------------------------------------------


class GradList:
    """The tensors of a call to grad_norm or grad_clip, as the ABI takes them.  Buffers that stay the same from step to step need one
    list.  It holds on to the memory that the tensors had when it was made: a tensor that is given other memory later (``set_``,
    assigning ``data``) needs a new list.  Resizing a tensor or its storage frees that memory; a call with the list then raises
    ``ValueError``."""

    def __init__(self, tensors):
        self.tensors = [t.detach() for t in tensors]
        self.array = (_Tensor * max(len(self.tensors), 1))()
        self.device = None
        found = {}              # by the address that the list relies on: the storage, and the first tensor in it
        for i, t in enumerate(self.tensors):
            name = f"gradient {i}"
            if not t.is_cuda:
                _bad(name, "device tensor expected")
            if t.dtype not in _CODES:
                _bad(name, f"float32 or bfloat16 expected, got {t.dtype}")
            if not t.is_contiguous():
                _bad(name, "contiguous tensor expected")
            if self.device is None:
                self.device = t.get_device()
            elif t.get_device() != self.device:
                _bad(name, f"on cuda:{t.get_device()}, others on cuda:{self.device}")
            self.array[i] = _Tensor(t.data_ptr() or None, t.numel(), _CODES[t.dtype], 0)
            if t.numel():
                storage = t.untyped_storage()
                found.setdefault(storage.data_ptr(), (storage, i))
        self.addresses, self.storages, self.first = list(found), [s for s, _ in found.values()], [i for _, i in found.values()]

    def __len__(self):
        return len(self.tensors)


def make_grad_list(tensors) -> GradList:
    return GradList(tensors)


def _list(g, device):
    if g is None:
        return None
    if g.device is not None and g.device != device:
        _bad("gradients", f"on cuda:{g.device}, the current device is cuda:{device}")
    now = list(map(torch.UntypedStorage.data_ptr, g.storages))      # 0.07 us each
    if now != g.addresses:
        i = next(i for i, a, b in zip(g.first, now, g.addresses) if a != b)
        _bad(f"gradient {i}", "its storage was resized after the list was made")
    return g.array


def grad_workspace_bytes() -> int:
    return int(_lib().grad_workspace_bytes())


def grad_norm(grads: GradList, norm, ws) -> None:
    lib, dev = _lib(), _device()
    rc = lib.grad_norm(_list(grads, dev), len(grads), _arg(norm, "norm", torch.float32, 1, dev), _arg(ws, "ws", torch.uint8, 0, dev),
                       ws.numel(), _stream(dev))
    _check(rc, "grad_norm")


def grad_clip(grads: GradList, outs, max_norm, eps, norm, ws) -> None:
    """outs: GradList of the same sizes, or None: in place."""
    lib, dev = _lib(), _device()
    if outs is not None and len(outs) != len(grads):
        raise ValueError("one output per gradient")
    rc = lib.grad_clip(_list(grads, dev), _list(outs, dev), len(grads), max_norm, eps, _arg(norm, "norm", torch.float32, 2, dev),
                       _arg(ws, "ws", torch.uint8, 0, dev), ws.numel(), _stream(dev))
    _check(rc, "grad_clip")
