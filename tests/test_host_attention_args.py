"""What the attention binding hands to the library, on the CPU: the calls run against a stand-in for the library that records its arguments."""
import copy
import ctypes as C
import os
from types import SimpleNamespace

import pytest

import paper_2603_04411_amd as L
from paper_2603_04411_amd import attention as B


@pytest.fixture
def calls(monkeypatch):
    """The calls that reached the library, as (name, the descriptor's contents, other arguments).  Host tensors count as the device's."""
    if not os.path.exists(L.library_path()):
        from paper_2603_04411_amd.build import build_library
        build_library()
    seen, lib = [], B._lib()

    def record(name):
        def call(ref, *rest):
            seen.append((name, bytes(ref._obj), rest))
            return 0
        return call
    stand_in = SimpleNamespace(attn_validate_desc=lib.attn_validate_desc, evict_validate_desc=lib.evict_validate_desc,
                               **{n: record(n) for n in ("attn_fwd", "attn_bwd", "kv4_store", "kv4_attn", "cache_evict")})
    monkeypatch.setattr(B, "_lib", lambda: stand_in)
    monkeypatch.setattr(B, "_device", lambda: -1)      # what a host tensor's get_device() says
    monkeypatch.setattr(B, "_stream", lambda device: None)
    return seen


Bn, Tq, Tk, Hq, Hkv, D = 2, 5, 40, 8, 2, 64


def tensors(Tk=Tk):
    import torch
    bf, f32, u8 = torch.bfloat16, torch.float32, torch.uint8
    t = dict(q=torch.zeros(Bn, Tq, Hq, D, dtype=bf), k=torch.zeros(Bn, Tk, Hkv, D, dtype=bf),
             lse=torch.zeros(Bn, Hq, Tq, dtype=f32), weight=torch.zeros(Bn, Hkv, Tk, dtype=f32), ws=torch.zeros(64, dtype=u8),
             codes=torch.zeros(Bn, Hkv, Tk, D // 2, dtype=u8), scales=torch.zeros(Bn, Hkv, Tk, D // 32, dtype=u8))
    return SimpleNamespace(**t)


def call_all(d, t):
    cache = (t.codes, t.scales, t.codes, t.scales)
    L.attn_fwd(d, t.q, t.k, t.k, None, None, t.q, t.lse, t.weight, 1.0, t.ws)
    L.attn_bwd(d, t.q, t.k, t.k, None, None, t.q, t.lse, t.q, t.q, t.k, t.k, t.ws)
    L.kv4_store(d, t.k[:, :Tq], t.k[:, :Tq], None, None, *cache, t.ws)
    L.kv4_attn(d, t.q, *cache, None, None, t.q, t.lse, t.weight, 1.0, t.ws)


@pytest.mark.parametrize("copied", [copy.copy, copy.deepcopy], ids=["copy", "deepcopy"])
def test_a_copied_descriptor_is_the_one_that_is_passed(calls, copied):
    """A descriptor made from one that was used: what is checked and what the library gets are its own contents, whatever becomes of the first."""
    first = L.make_attn_desc(Bn, Tq, Tk, Hq, Hkv, D, "bf16")
    call_all(first, tensors())
    second = copied(first)
    first.Tk = 4000
    calls.clear()
    call_all(second, tensors())
    assert [n for n, *_ in calls] == ["attn_fwd", "attn_bwd", "kv4_store", "kv4_attn"]
    for name, raw, _ in calls:
        assert B.AttnDesc.from_buffer_copy(raw).Tk == Tk and raw == bytes(second), name
    with pytest.raises(ValueError):      # the first one is held against its new contents
        L.attn_fwd(first, *(getattr(tensors(), x) for x in ("q", "k", "k")), None, None, tensors().q, None, None, 1.0, tensors().ws)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,Tq,Tk,Hq,Hkv", [(1, 1 << 20, 33280, 1024, 1), (1, 1 << 20, 65000, 1024, 1), (1, 1 << 20, 16384, 1024, 1), (2, 1 << 20, 12800, 1024, 2),
                                            (1, 1 << 20, 25600, 1024, 1), (3, 4096, 4096, 28, 4), (1, 1, 1, 1, 1), (1, 1 << 20, 1 << 25, 1, 1)])
def test_backward_workspaces_of_the_largest_calls(B, Tq, Tk, Hq, Hkv, dtype):
    """What is cut of dk and dv is counted in 64 bits: a call with many tiles and few blocks of keys has as many workgroups as are resident."""
    d = L.make_attn_desc(B, Tq, Tk, Hq, Hkv, 8, dtype)
    assert L.attn_validate_desc(d) == 0
    lse, before, parts = 4 * B * Hq * Tq, 8 * (B * ((Tk + 127) // 128) + 1), 2 * 512 * 128 * 2 * 64 * 4     # at most 512 workgroups, two parts each
    assert 256 + lse <= L.attn_bwd_workspace_bytes(d) <= 256 + lse + before + parts + 3 * 256
    assert L.attn_workspace_bytes(d) >= 256 + lse
