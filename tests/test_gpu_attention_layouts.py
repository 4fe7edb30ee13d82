"""Tensors of an attention call side by side in one buffer: neighbours that share no memory are taken, whatever lies between their rows."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("order", ["slot", "head"])
def test_all_tensors_in_one_buffer(dtype, order):
    """q, k, v, out, its gradient and the three gradients as heads of one tensor, lse and weight in a gap of it: the bits of a call on tensors of their own."""
    import torch
    import paper_2603_04411_amd as L
    B, T, Hq, Hkv, D = 2, 70, 4, 2, 64
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    heads = dict(q=Hq, k=Hkv, v=Hkv, out=Hq, g=Hq, dq=Hq, dk=Hkv, dv=Hkv)
    many = sum(heads.values()) + 4      # the last ones: the gap
    big = torch.zeros((B, T, many, D) if order == "slot" else (B, many, T, D), dtype=tdt, device="cuda")
    whole = big if order == "slot" else big.transpose(1, 2)
    views, at = {}, 0
    for n, h in heads.items():
        views[n] = whole[:, :, at:at + h]
        at += h
    gen = torch.Generator(device="cuda").manual_seed(3)
    for n in "qkvg":
        views[n].copy_(torch.randn(views[n].shape, device="cuda", generator=gen))
    own = {n: x.clone(memory_format=torch.contiguous_format) for n, x in views.items()}
    lens = torch.tensor([70, 33], dtype=torch.int32, device="cuda")
    results = []
    for t in (views, own):
        lay = {n: L.attn_layout(x) for n, x in t.items()}
        d = L.make_attn_desc(B, T, T, Hq, Hkv, D, dtype, window=40, sinks=2, q=lay["q"], k=lay["k"], v=lay["v"], o=lay["out"])
        lse, weight = torch.zeros(B, Hq, T, device="cuda"), torch.zeros(B, Hkv, T, device="cuda")
        if t is views and order == "head":      # the gap of a sequence is [4, T, D]: room for both
            flat = big[0, -4:].flatten().view(torch.float32)
            lse, weight = flat[:lse.numel()].view(lse.shape), flat[lse.numel():lse.numel() + weight.numel()].view(weight.shape)
        ws = torch.empty(max(L.attn_workspace_bytes(d), L.attn_bwd_workspace_bytes(d)), dtype=torch.uint8, device="cuda")
        L.attn_fwd(d, t["q"], t["k"], t["v"], lens, lens, t["out"], lse, weight, 0.0, ws)
        L.attn_bwd(d, t["q"], t["k"], t["v"], lens, lens, t["out"], lse, t["g"], t["dq"], t["dk"], t["dv"], ws)
        assert L.lmhead_check(ws) == 0
        results.append([t[n].clone() for n in ("out", "dq", "dk", "dv")] + [lse.clone(), weight[:, :, :33].clone()])
        ev = L.make_evict_desc(B, T, Hkv, 20, 2, 5)
        i32 = dict(dtype=torch.int32, device="cuda")
        left, kept = torch.empty(B, **i32), torch.empty(B, Hkv, 20, **i32)
        L.cache_evict(ev, L.make_cache_planes([t["k"], t["v"]]), weight, lens, left, kept, ws)
        results[-1] += [t[n][:, :20].clone() for n in "kv"] + [kept]
    assert all(torch.equal(x, y) for x, y in zip(*results))


def test_tensors_that_share_memory_are_refused():
    """In the binding's own terms: an output behind the beginning of an input, of a workspace or of another output."""
    import torch
    import paper_2603_04411_amd as L
    B, T, H, D = 2, 40, 4, 64
    d = L.make_attn_desc(B, T, T, H, H, D, "bf16")
    n = B * T * H * D
    buf = torch.zeros(8 * n, dtype=torch.bfloat16, device="cuda")
    q, k, v, out = (buf[i * n:(i + 1) * n].view(B, T, H, D) for i in range(4))
    need = L.attn_workspace_bytes(d)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    lse = torch.zeros(B, H, T, device="cuda")
    L.attn_fwd(d, q, k, v, None, None, out, lse, None, 0.0, ws)
    over = buf[n // 2:n // 2 + n].view(B, T, H, D)
    inner = out.flatten()[-2 * lse.numel():].view(torch.float32).view(lse.shape)
    tail = ws[need - 4 * lse.numel():].view(torch.float32).view(lse.shape)
    for change in (dict(out=over), dict(lse=inner), dict(lse=tail), dict(weight=lse)):
        a = dict(q=q, k=k, v=v, len_q=None, len_k=None, out=out, lse=lse, weight=None, decay=0.0, ws=ws)
        a.update(change)
        with pytest.raises(L.LmheadError) as e:
            L.attn_fwd(d, *a.values())
        assert e.value.code == -2
