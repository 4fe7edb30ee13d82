"""What the attention binding hands to the library, on the CPU: the calls run against a stand-in for the library that records its arguments."""
import copy
import ctypes as C
import os
import subprocess
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
@pytest.mark.parametrize("B,Tq,Tk,Hq,Hkv", [(1, 1 << 20, 33280, 1024, 1), (1, 1 << 20, 65000, 1024, 1), (1, 1 << 20, 16384, 1024, 1),
                                            (2, 1 << 20, 12800, 1024, 2), (1, 1 << 20, 25600, 1024, 1), (3, 4096, 4096, 28, 4), (1, 1, 1, 1, 1), (1, 1 << 20, 1 << 25, 1, 1)])
def test_backward_workspaces_of_the_largest_calls(B, Tq, Tk, Hq, Hkv, dtype):
    """What is cut of dk and dv is counted in 64 bits: a call with many tiles and few blocks of keys has as many workgroups as are resident."""
    d = L.make_attn_desc(B, Tq, Tk, Hq, Hkv, 8, dtype)
    assert L.attn_validate_desc(d) == 0
    lse, before, parts = 4 * B * Hq * Tq, 8 * (B * ((Tk + 127) // 128) + 1), 2 * 512 * 128 * 2 * 64 * 4     # at most 512 workgroups, two parts each
    assert 256 + lse <= L.attn_bwd_workspace_bytes(d) <= 256 + lse + before + parts + 3 * 256
    assert L.attn_workspace_bytes(d) >= 256 + lse


def test_tensors_with_more_slots_than_the_descriptor_are_refused(calls):
    """A head's rows begin at a multiple of the descriptor's slots: in a tensor with more of them every head but the first would be read and written
    at another head's place.  (The tensors hold more than the call needs, so no access would leave them.)"""
    import torch
    d, t, wide = L.make_attn_desc(Bn, Tq, Tk, Hq, Hkv, D, "bf16"), tensors(), tensors(2 * Tk)
    more_lse = torch.zeros(Bn, Hq, 2 * Tq)

    def fwd(lse=t.lse, weight=t.weight, q=t.q, k=t.k):
        L.attn_fwd(d, q, k, t.k, None, None, t.q, lse, weight, 1.0, t.ws)

    def store(codes=t.codes, scales=t.scales):
        L.kv4_store(d, t.k[:, :Tq], t.k[:, :Tq], None, None, codes, scales, t.codes, t.scales, t.ws)

    def attend(codes=t.codes, scales=t.scales, weight=t.weight):
        L.kv4_attn(d, t.q, t.codes, t.scales, codes, scales, None, None, t.q, t.lse, weight, 1.0, t.ws)
    fwd(), store(), attend()
    assert len(calls) == 3
    calls.clear()
    for refused in (lambda: fwd(lse=more_lse), lambda: fwd(weight=wide.weight), lambda: store(codes=wide.codes), lambda: store(scales=wide.scales),
                    lambda: attend(codes=wide.codes), lambda: attend(scales=wide.scales), lambda: attend(weight=wide.weight),
                    lambda: fwd(weight=wide.weight[:, :, :Tk]), lambda: fwd(weight=wide.weight.view(Bn * Hkv, 2 * Tk)),
                    lambda: L.attn_bwd(d, t.q, t.k, t.k, None, None, t.q, more_lse, t.q, t.q, t.k, t.k, t.ws),
                    # as many elements, in another order
                    lambda: fwd(weight=torch.zeros(Bn, Tk, Hkv)), lambda: fwd(q=torch.zeros(Bn, Hq, Tq, D, dtype=torch.bfloat16)),
                    lambda: fwd(k=torch.zeros(Bn * Hkv, Tk, D, dtype=torch.bfloat16)), lambda: store(codes=torch.zeros(Bn, Tk, Hkv, D // 2, dtype=torch.uint8)),
                    # too few
                    lambda: fwd(weight=t.weight[:1]), lambda: fwd(lse=t.lse[:, :4].contiguous()), lambda: fwd(weight=t.weight.flatten()[1:])):
        with pytest.raises(ValueError):
            refused()
    odd = L.make_attn_desc(Bn, Tq, Tk, Hq, Hkv, 40, "bf16")      # no cache has such rows
    for call in (lambda: L.kv4_store(odd, t.k, t.k, None, None, t.codes, t.scales, t.codes, t.scales, t.ws),
                 lambda: L.kv4_attn(odd, t.q, t.codes, t.scales, t.codes, t.scales, None, None, t.q, None, None, 1.0, t.ws)):
        with pytest.raises(L.LmheadError) as e:
            call()
        assert e.value.code == -2
    # more sequences, flat buffers and merged dimensions mean the same memory
    for weight in (torch.zeros(Bn + 1, Hkv, Tk), torch.zeros(Bn * Hkv * Tk + 5), t.weight.view(Bn * Hkv, Tk), t.weight.view(Bn, Hkv * Tk), t.weight[None],
                   t.weight.flatten(), torch.zeros(Bn * Hkv + 1, Tk), torch.zeros(2, Bn, Hkv, Tk), torch.zeros(3, 1, Bn * Hkv, Tk)[:1]):
        fwd(weight=weight)
        assert calls[-1][2][7] == weight.data_ptr()
    for q in (t.q.view(Bn, Tq, Hq * D), t.q.view(Bn * Tq, Hq, D), t.q.flatten(), t.q.view(1, Bn * Tq, Hq, D), torch.zeros(Bn + 1, Tq, Hq, D, dtype=torch.bfloat16)):
        fwd(q=q)
        assert calls[-1][2][0] == q.data_ptr()
    # of one head of one sequence all slots that are used come first
    one = L.make_attn_desc(1, 1, Tk, 1, 1, D, "bf16")
    q, k, weight, ws = t.q[:1, :1, :1], t.k[:1, :, :1].contiguous(), torch.zeros(1, 1, 3 * Tk), t.ws
    L.attn_fwd(one, q, k, k, None, None, q, None, weight, 1.0, ws)
    assert calls[-1][2][7] == weight.data_ptr()


def test_eviction_refuses_weights_and_slots_of_other_shapes(calls):
    import torch
    keep = 10
    d, i32 = L.make_evict_desc(Bn, Tk, Hkv, keep), dict(dtype=torch.int32)
    t, wide = tensors(), tensors(2 * Tk)
    planes = SimpleNamespace(tensors=[], storages=[], addresses=[], device=None, array=None)
    planes = type("Planes", (), dict(vars(planes), __len__=lambda self: 1))()
    lens, kept = torch.zeros(Bn, **i32), torch.zeros(Bn, Hkv, keep, **i32)

    def evict(weight=t.weight, kept=kept):
        L.cache_evict(d, planes, weight, None, lens, kept, t.ws)
    evict()
    for weight in (torch.zeros(Bn + 1, Hkv, Tk), t.weight.flatten(), t.weight.view(Bn * Hkv, Tk)):
        evict(weight)
    evict(kept=kept.flatten())
    n = len(calls)
    for change in (dict(weight=wide.weight), dict(weight=torch.zeros(Bn, Tk, Hkv)), dict(kept=torch.zeros(Bn, Hkv, keep + 1, **i32)),
                   dict(kept=torch.zeros(Bn, keep, Hkv, **i32)), dict(kept=kept[:1])):
        with pytest.raises(ValueError):
            evict(**change)
    assert len(calls) == n


# ---- tensors that share memory (pointers are never dereferenced: every call here is refused) ----

FAR = 1 << 24


def _raw(name, d, shift):
    """The call with its pointers FAR apart but for argument `at`, which begins `by` bytes from argument `to`."""
    at, to, by = shift
    n = {"attn_fwd": 9, "attn_bwd": 12, "kv4_store": 9, "kv4_attn": 11}[name]
    p = [FAR * (i + 1) for i in range(n)]
    p[at] = p[to] + by
    rest = (C.c_size_t(1 << 30), None)
    if name in ("attn_fwd", "kv4_attn"):
        return getattr(B._lib(), name)(C.byref(d), *p[:-1], 1.0, p[-1], *rest)
    return getattr(B._lib(), name)(C.byref(d), *p, *rest)


ARGS = {
    "attn_fwd": ("q k v len_q len_k out lse weight ws", "out lse weight ws"), "attn_bwd": ("q k v len_q len_k out lse g dq dk dv ws", "dq dk dv ws"),
    "kv4_store": ("k v len_q len_k k_codes k_scales v_codes v_scales ws", "k_codes k_scales v_codes v_scales ws"),
    "kv4_attn": ("q k_codes k_scales v_codes v_scales len_q len_k out lse weight ws", "out lse weight ws"),
}


@pytest.mark.parametrize("name", ARGS)
def test_outputs_that_share_memory_are_refused(name):
    """Every output against every other tensor of the call: at the same place, 256 bytes behind its beginning, and the other way round."""
    names, outputs = (x.split() for x in ARGS[name])
    d = L.make_attn_desc(128, 40, 40, Hq, Hkv, 64, "bf16")      # every tensor takes 512 bytes at least
    for o in outputs:
        for i, x in enumerate(names):
            if x == o:
                continue
            assert _raw(name, d, (names.index(o), i, 0)) == -2, (o, x)
            for first, second in ((o, x), (x, o)):
                if (name, second) != ("kv4_store", "ws"):      # its header is all that is used
                    assert _raw(name, d, (names.index(first), names.index(second), 256)) == -2, (first, second)


def test_a_dense_output_among_the_rows_of_a_tensor_with_gaps():
    """lse (2560 bytes) in the gap of 3 KB behind each slot of q is the caller's; where it reaches into a row the call is refused."""
    d = L.make_attn_desc(Bn, 40, 40, Hq, Hkv, 64, "bf16", q=(40 * 2048, 2048, 64))      # a slot's 1 KB, then nothing for 3 KB
    row, slot = Hq * 64 * 2, 4096
    names = ARGS["attn_fwd"][0].split()
    assert 4 * Bn * Hq * 40 == 2560
    for by in (row - 16, slot - 2560 + 16, 7 * slot - 1024, 79 * slot, 79 * slot + row - 16):
        assert _raw("attn_fwd", d, (names.index("lse"), names.index("q"), by)) == -2, by


def test_eviction_refuses_planes_that_share_memory():
    d = L.make_evict_desc(2, 40, 3, 10)
    row, lib = (40 * 3 * 64, 3 * 64, 64, 64), B._lib()

    def evict(shift, plane=(FAR * 8, FAR * 9)):
        p = [FAR * (i + 1) for i in range(5)]      # weight len len_out kept ws
        for at, x in shift.items():
            p[at] = x
        a = (B._Plane * 2)()
        for i, x in enumerate(plane):
            a[i] = B._Plane(x, *row)
        return lib.cache_evict(C.byref(d), a, 2, *p, 256, None)
    size = 2 * 40 * 3 * 64
    assert evict({}, (FAR * 8, FAR * 8 + size - 4)) == -2 and evict({}, (FAR * 8 + 64, FAR * 8)) == -2
    for at, n in ((0, 2 * 3 * 40 * 4), (2, 8), (3, 2 * 3 * 10 * 4), (4, 256)):
        assert evict({at: FAR * 8 + size - 256}) == -2 and evict({at: FAR * 9}) == -2, at
    assert evict({3: FAR + 2 * 3 * 40 * 4 - 4}) == -2 and evict({2: FAR * 4 + 4}) == -2 and evict({2: FAR * 2 + 4}) == -2 and evict({0: FAR * 5 - 4}) == -2


def test_overlaps_byte_by_byte(tmp_path):
    exe = tmp_path / "regions_check"
    source = os.path.join(os.path.dirname(os.path.abspath(__file__)), "host", "regions_check.cpp")
    subprocess.run(["g++", "-O2", "-std=c++17", "-o", str(exe), source], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and "bad=0" in r.stdout, r.stdout + r.stderr
