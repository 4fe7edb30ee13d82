"""Host side of attention, the 4-bit cache and eviction: argument validation returns the documented codes before anything is launched, the binding
refuses tensors that are not what the call needs."""
import ctypes as C
import os

import pytest

import paper_2603_04411_amd as L
from paper_2603_04411_amd import attention as B

P_ = 0x10000   # never dereferenced: every call below has to fail in host-side validation


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(L.library_path()):
        from paper_2603_04411_amd.build import build_library
        build_library()
    return B._lib()


def test_structures_match_the_c_layout():
    assert C.sizeof(B.AttnLayout) == 24 and C.sizeof(B.AttnDesc) == 48 + 4 * 24 and B.AttnDesc.q.offset == 48 and B.AttnDesc.scale.offset == 36
    assert C.sizeof(B.EvictDesc) == 32 and C.sizeof(B._Plane) == 40


BASE = dict(B=2, Tq=5, Tk=40, Hq=8, Hkv=2, D=64, dtype="bf16")


def addresses(n):
    return [P_ + 0x1000 * i for i in range(n)]


def fwd(lib, d, over=None, null=None, nbytes=1 << 60, decay=1.0):
    p = addresses(9)      # q k v len_q len_k out lse weight ws
    for i, x in (over or {}).items():
        p[i] = x
    if null is not None:
        p[null] = None
    return lib.attn_fwd(C.byref(d) if d else None, *p[:8], decay, p[8], nbytes, None)


def bwd(lib, d, over=None, null=None, nbytes=1 << 60):
    p = addresses(12)     # q k v len_q len_k out lse g dq dk dv ws
    for i, x in (over or {}).items():
        p[i] = x
    if null is not None:
        p[null] = None
    return lib.attn_bwd(C.byref(d), *p, nbytes, None)


def store(lib, d, over=None, null=None, nbytes=1 << 60):
    p = addresses(9)      # k v len_q len_k and the cache, ws
    for i, x in (over or {}).items():
        p[i] = x
    if null is not None:
        p[null] = None
    return lib.kv4_store(C.byref(d), *p, nbytes, None)


def attend4(lib, d, over=None, null=None, nbytes=1 << 60, decay=1.0):
    p = addresses(11)     # q, the cache, len_q len_k out lse weight ws
    for i, x in (over or {}).items():
        p[i] = x
    if null is not None:
        p[null] = None
    return lib.kv4_attn(C.byref(d), *p[:10], decay, p[10], nbytes, None)


CHANGES = [
    (dict(B=0), -2), (dict(B=65536), -2), (dict(Tq=0), -2), (dict(Tk=0), -2), (dict(Hq=0), -2), (dict(Hkv=0), -2), (dict(Hq=9), -2), (dict(Hq=1026), -2),
    (dict(D=0), -2), (dict(D=60), -2), (dict(D=136), -2), (dict(window=-1), -2), (dict(sinks=-1), -2), (dict(scale=0.0), -2), (dict(scale=-1.0), -2),
    (dict(scale=float("nan")), -2), (dict(scale=float("inf")), -2), (dict(scale=3e38), -2), (dict(dtype=2), -3), (dict(Tk=1 << 30), -2),
    (dict(Tq=1 << 21), -2), (dict(q=(-64, 64, 64)), -2), (dict(q=(1 << 41, 512, 64)), -2), (dict(q=(2560, 32, 64)), -2), (dict(k=(5120, 1 << 23, 64)), -2),
    (dict(v=(5120, 132, 64)), -4), (dict(q=(2564, 512, 64)), -4), (dict(o=(2560, 512, 68)), -4),
    (dict(o=(2560, 512, 0)), -2), (dict(o=(0, 512, 64)), -2), (dict(o=(512, 512, 64)), -2), (dict(B=65535, Hkv=8, Tk=1 << 20, Tq=1), -2),
]


def test_descriptor_refusals(lib):
    ok = L.make_attn_desc(**BASE)
    assert L.attn_validate_desc(ok) == 0 and lib.attn_validate_desc(None) == -1
    assert L.attn_workspace_bytes(ok) >= 256 and L.attn_bwd_workspace_bytes(ok) >= 256
    for change, code in CHANGES:
        d = L.make_attn_desc(**{**BASE, **change})
        assert L.attn_validate_desc(d) == code, change
        assert L.attn_workspace_bytes(d) == 0 and L.attn_bwd_workspace_bytes(d) == 0
        assert fwd(lib, d) == code and bwd(lib, d) == code and store(lib, d) == code and attend4(lib, d) == code, change
    for field, code in (("flags", -3), ("reserved", -2)):
        d = L.make_attn_desc(**BASE)
        setattr(d, field, 1)
        assert L.attn_validate_desc(d) == code
    # what inputs may be: heads or sequences that share their keys; 16 bytes of fp32
    assert L.attn_validate_desc(L.make_attn_desc(**{**BASE, "k": (0, 128, 0), "v": (0, 128, 0)})) == 0
    assert L.attn_validate_desc(L.make_attn_desc(**{**BASE, "dtype": "f32", "q": (2580, 516, 64)})) == 0
    assert L.attn_validate_desc(L.make_attn_desc(**{**BASE, "window": (1 << 31) - 1, "sinks": (1 << 31) - 1})) == 0
    # but gradients of shared keys would lie upon each other
    assert bwd(lib, L.make_attn_desc(**{**BASE, "k": (0, 128, 64)})) == -2
    assert bwd(lib, L.make_attn_desc(**{**BASE, "q": (2560, 512, 0)})) == -2


def test_call_refusals(lib):
    d = L.make_attn_desc(**BASE)
    need, more = L.attn_workspace_bytes(d), L.attn_bwd_workspace_bytes(d)
    for call, optional, ws, least in ((fwd, (3, 4, 6, 7), 8, need), (bwd, (3, 4), 11, more), (store, (2, 3), 8, 256), (attend4, (5, 6, 8, 9), 10, need)):
        for i in range(ws + 1):
            if i not in optional:
                assert call(lib, d, null=i) == -1, (call, i)
        assert call(lib, d, nbytes=least - 1) == -5 and call(lib, d, over={ws: P_ + 0x20010}) == -4
    for i in (0, 1, 2, 5):
        assert fwd(lib, d, over={i: P_ + 0x20008}) == -4
    for i in (0, 1, 2, 5, 7, 8, 9, 10):
        assert bwd(lib, d, over={i: P_ + 0x20008}) == -4
    for i in (0, 1, 4, 6):
        assert store(lib, d, over={i: P_ + 0x20008}) == -4
    for i in (5, 7):
        assert store(lib, d, over={i: P_ + 0x20002}) == -4
    # one address twice
    for i, j in ((5, 0), (5, 1), (5, 2), (7, 6), (6, 5), (7, 3), (8, 5)):
        assert fwd(lib, d, over={i: addresses(9)[j]}) == -2, (i, j)
    for i, j in ((8, 0), (9, 1), (10, 2), (8, 9), (9, 10), (8, 7), (10, 5)):
        assert bwd(lib, d, over={i: addresses(12)[j]}) == -2, (i, j)
    for decay in (-0.5, float("nan"), float("inf")):
        assert fwd(lib, d, decay=decay) == -2 and attend4(lib, d, decay=decay) == -2
    for D in (8, 40, 72):
        e = L.make_attn_desc(**{**BASE, "D": D})
        assert L.attn_validate_desc(e) == 0 and store(lib, e) == -2 and attend4(lib, e) == -2


def evict(lib, d, planes, count=None, null=None, over=None, nbytes=256):
    p = addresses(5)      # weight len len_out kept ws
    for i, x in (over or {}).items():
        p[i] = x
    if null is not None:
        p[null] = None
    return lib.cache_evict(C.byref(d) if d else None, planes, len(planes) if planes and count is None else count or 0, *p, nbytes, None)


def planes(*each):
    a = (B._Plane * len(each))()
    for i, (data, seq, slot, head, n) in enumerate(each):
        a[i] = B._Plane(data, seq, slot, head, n)
    return a


def test_eviction_refusals(lib):
    ok = L.make_evict_desc(2, 40, 3, 10, sinks=4, recent=6)
    assert L.evict_validate_desc(ok) == 0 and L.evict_workspace_bytes(ok) == 256 and lib.evict_validate_desc(None) == -1
    for change in (dict(B=0), dict(B=65536), dict(T=0), dict(Hkv=0), dict(Hkv=1025), dict(keep=0), dict(keep=41), dict(sinks=-1), dict(recent=-1), dict(recent=7),
                   dict(sinks=11, recent=0), dict(sinks=(1 << 31) - 1), dict(T=1 << 30)):
        d = L.make_evict_desc(**{**dict(B=2, T=40, Hkv=3, keep=10, sinks=4, recent=6), **change})
        assert L.evict_validate_desc(d) == -2 and L.evict_workspace_bytes(d) == 0, change
    for field, code in (("flags", -3), ("reserved", -2)):
        d = L.make_evict_desc(2, 40, 3, 10)
        setattr(d, field, 1)
        assert L.evict_validate_desc(d) == code
    A, Z = 0x100000, 0x200000
    row = (40 * 3 * 64, 3 * 64, 64, 64)
    assert evict(lib, None, planes((A, *row))) == -1 and evict(lib, ok, None, 1) == -1
    for i in (0, 2, 3, 4):
        assert evict(lib, ok, planes((A, *row)), null=i) == -1
    assert evict(lib, ok, planes((None, *row))) == -1
    assert evict(lib, ok, planes((A, *row)), count=5) == -2 and evict(lib, ok, planes((A, *row)), count=-1) == -2
    assert evict(lib, ok, planes((A, *row), (A, *row))) == -2                    # twice the same memory
    for i, j in ((2, 1), (3, 0), (0, 1)):
        assert evict(lib, ok, planes((A, *row)), over={i: addresses(5)[j]}) == -2
    assert evict(lib, ok, planes((A, *row)), over={3: A}) == -2
    for r, code in (((40 * 3 * 64, 3 * 64, 64, 62), -4), ((40 * 3 * 64, 3 * 64, 66, 64), -4), ((40 * 3 * 64, 3 * 64, 64, 0), -2), ((40 * 3 * 64, 3 * 64, 64, 8192), -2),
                    ((40 * 3 * 64, 3 * 64, 32, 64), -2), ((40 * 3 * 64, 64, 64, 64), -2), ((0, 3 * 64, 64, 64), -2), ((-4, 3 * 64, 64, 64), -2)):
        assert evict(lib, ok, planes((A, *row), (Z, *r))) == code, r
    assert evict(lib, ok, planes((A + 2, *row))) == -4 and evict(lib, ok, planes((A, *row)), over={4: P_ + 0x9008}) == -4
    assert evict(lib, ok, planes((A, *row)), nbytes=255) == -5


def test_binding_refuses_tensors_before_the_call(lib):
    import torch
    q = torch.zeros(2, 5, 8, 64, dtype=torch.bfloat16)
    k = torch.zeros(2, 40, 2, 64, dtype=torch.bfloat16)
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    with pytest.raises(L.LmheadError) as e:      # the descriptor's refusal comes first, whatever the tensors
        L.attn_fwd(L.make_attn_desc(**{**BASE, "Tq": -1}), q, k, k, None, None, q, None, None, 1.0, ws)
    assert e.value.code == -2
    with pytest.raises(ValueError, match="plane 0: device tensor expected"):
        L.make_cache_planes([k])


def test_a_descriptor_that_changes_is_looked_at_again(lib):
    d = L.make_attn_desc(**BASE)
    assert B._sizes(d, "x").weight == 2 * 2 * 40
    d.Tk = 50
    assert B._sizes(d, "x").weight == 2 * 2 * 50
    d.D = 63
    with pytest.raises(L.LmheadError):
        B._sizes(d, "x")


def test_layouts_of_views():
    import torch
    t = torch.zeros(3, 7, 4, 16)
    assert L.attn_layout(t) == (448, 64, 16) and L.attn_layout(t.transpose(1, 2)) == (448, 16, 64)
    assert L.attn_layout(t[:, :, :1]) == (448, 64, 1344) and L.attn_layout(t[:1]) == (448, 64, 16)
    assert L.attn_layout(t[:, :1]) == (448, 16, 16) and L.attn_layout(t[:, :, :1].expand(3, 7, 5, 16)) == (448, 64, 0)
    with pytest.raises(ValueError):
        L.attn_layout(t[0])


def test_workspaces_do_not_grow_with_shorter_calls_of_a_step(lib):
    """A decoding loop sizes its workspace for the longest cache."""
    last = 0
    for Tk in (1, 31, 64, 100, 1000, 4096, 20000, 131072):
        n = L.attn_workspace_bytes(L.make_attn_desc(4, 1, Tk, 32, 8, 128, "bf16"))
        assert n >= last
        last = n
