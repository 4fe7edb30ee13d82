"""Attention, the 4-bit cache and eviction as a program uses them: one after the other over one cache, behind the compression of keys, in graphs that are
replayed, on other streams, with layouts that share memory or pass 32 bits; gradients against difference quotients."""
import numpy as np
import pytest

from oracle import attention_oracle as A
from tests.attention_cases import bounds, holds
from tests.test_gpu_attention import Problem, check_fwd, np64
from tests.test_gpu_kv_cache import Cache4

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_eviction_and_decoding_in_four_bits(dtype):
    """A padded batch's prompt with the keys' weights, the cache made smaller by them, what is left stored in 4 bits, then tokens one by one from a
    replayed graph that also moves the lengths on."""
    import torch
    import paper_2603_04411_amd as L
    B, T, Hq, Hkv, D, keep, sinks, recent, room, steps = 2, 90, 4, 2, 64, 48, 4, 16, 64, 5
    p = Problem(B, T, T, Hq, Hkv, D, dtype, len_q=[90, 37], len_k=[90, 37], seed=5)
    check_fwd(p, decay=0.0)
    weight, k, v = (np64(t).copy() for t in (p.weight, p.k, p.v))
    ev = L.make_evict_desc(B, T, Hkv, keep, sinks, recent)
    i32 = dict(dtype=torch.int32, device="cuda")
    lens, kept = torch.full((B,), -7, **i32), torch.full((B, Hkv, keep), -7, **i32)
    ws = torch.empty(L.evict_workspace_bytes(ev), dtype=torch.uint8, device="cuda")
    L.cache_evict(ev, L.make_cache_planes([p.k, p.v]), p.weight, p.len_k, lens, kept, ws)
    assert L.lmhead_check(ws) == 0 and lens.tolist() == [48, 37]
    for b, h in ((b, h) for b in range(B) for h in range(Hkv)):
        n = int(lens[b])
        want = A.evict(weight[b, h], int(p.lk[b]), keep, sinks, recent)
        assert kept[b, h, :n].tolist() == want
        for got, old in ((p.k, k), (p.v, v)):
            assert np.array_equal(np64(got)[b, :n, h], old[b, want, h])
        assert np.array_equal(np64(p.weight)[b, h, :n], weight[b, h, want])

    cache = [torch.full((B, Hkv, room, w), 255, dtype=torch.uint8, device="cuda") for w in (D // 2, D // 32) * 2]
    fill = L.make_attn_desc(B, keep, room, Hq, Hkv, D, dtype, k=L.attn_layout(p.k), v=L.attn_layout(p.v))
    ws4 = torch.empty(L.attn_workspace_bytes(fill), dtype=torch.uint8, device="cuda")
    L.kv4_store(fill, p.k, p.v, lens, lens, *cache, ws4)
    rng = np.random.default_rng(11)
    rows = [torch.from_numpy(rng.standard_normal((steps, B, 1, H, D))).to(p.tdt).cuda() for H in (Hq, Hkv, Hkv)]
    q, kn, vn = (torch.empty_like(x[0]) for x in rows)
    out, lse = torch.empty_like(q), torch.empty(B, Hq, 1, device="cuda")
    w4 = torch.zeros(B, Hkv, room, device="cuda")
    w4[:, :, :keep] = p.weight[:, :, :keep]
    for b in range(B):
        w4[b, :, int(lens[b]):] = 0
    step = L.make_attn_desc(B, 1, room, Hq, Hkv, D, dtype, k=L.attn_layout(kn), v=L.attn_layout(vn))      # of the rows that are stored
    ws1 = torch.empty(L.attn_workspace_bytes(step), dtype=torch.uint8, device="cuda")

    def token():
        lens.add_(1)
        L.kv4_store(step, kn, vn, None, lens, *cache, ws1)
        L.kv4_attn(step, q, *cache, None, lens, out, lse, w4, 0.5, ws1)

    graph = None
    for s in range(steps):
        for x, r in zip((q, kn, vn), rows):
            x.copy_(r[s])
        n0, w0 = lens.tolist(), np64(w4).copy()
        if s == 1:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                token()
        if graph is None:
            token()
        else:
            graph.replay()
        assert L.lmhead_check(ws1) == 0 and lens.tolist() == [n + 1 for n in n0]
        host = [x.cpu().numpy() for x in cache]
        K, V = (A.values4(host[i], host[i + 1]).transpose(0, 2, 1, 3) for i in (0, 2))
        for b in range(B):
            for got, new in ((host[0:2], rows[1]), (host[2:4], rows[2])):
                c, e = A.quantise4(np64(new[s, b, 0]))
                assert np.array_equal(got[0][b, :, n0[b]], c) and np.array_equal(got[1][b, :, n0[b]], e)
        K, V = np.where(np.isnan(K), 0, K), np.where(np.isnan(V), 0, V)      # slots behind the end
        want, bound = bounds(np64(rows[0][s]), K, V, [1, 1], lens.tolist(), float(np.float32(D ** -0.5)), 0, 0, dtype)
        holds(np64(out), want["out"], bound["out"], "out")
        holds(np64(lse), want["lse"], bound["lse"], "lse")
        for b in range(B):
            n = int(lens[b])
            total = 0.5 * w0[b, :, :n] + want["weight"][b, :, :n]
            holds(np64(w4)[b, :, :n], total, bound["weight"][b, :, :n] + 2.0 ** -22 * total, "weight")


def test_attention_over_reconstructed_keys():
    """Keys and values that went through the learned compression, read as two heads of 128."""
    import torch
    import paper_2603_04411_amd as L
    import workloads.dynakv as kv
    from tests.harness import KvProblem
    B, T, Hkv, D = 3, 70, 2, 128
    cfg = kv.KV_CONFIGS[1].scaled(n=B * T, d=Hkv * D)
    kp = KvProblem(cfg, kv.kv_inputs(cfg))
    xt, k, m, xhat = kp.gate(cfg.tau)
    off, packed = kp.store(xt, k)
    x = kp.reconstruct(packed, int(off[-1].item()), off, k).view(B, T, Hkv, D)
    assert kp.check() == 0
    dtype = "bf16" if x.dtype == torch.bfloat16 else "f32"
    q = torch.from_numpy(np.random.default_rng(2).standard_normal((B, 1, 8, D))).to(x.dtype).cuda()
    v = x.flip(1).contiguous()
    lk = torch.tensor([70, 1, 33], dtype=torch.int32, device="cuda")
    desc = L.make_attn_desc(B, 1, T, 8, Hkv, D, dtype, window=40, sinks=2)
    out, ws = torch.empty_like(q), torch.empty(L.attn_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    L.attn_fwd(desc, q, x, v, None, lk, out, None, None, 1.0, ws)
    want, bound = bounds(np64(q), np64(x), np64(v), [1] * B, lk.tolist(), float(np.float32(D ** -0.5)), 40, 2, dtype)
    holds(np64(out), want["out"], bound["out"], "out")


@pytest.mark.parametrize("case", [dict(B=2, Tq=70, Tk=200, Hq=4, Hkv=2, D=64, window=50, sinks=3, len_q=[70, 9], len_k=[200, 100]),
                                  dict(B=1, Tq=700, Tk=700, Hq=2, Hkv=1, D=128),
                                  dict(B=2, Tq=1, Tk=5000, Hq=8, Hkv=2, D=128, len_k=[5000, 77])], ids=["few", "long", "decode"])
def test_graphs_that_share_a_workspace(case):
    """Forward and backward in a graph each, over one workspace, replayed with other inputs and eager calls between."""
    import torch
    p = Problem(seed=3, **case)
    L = p.L
    ws = torch.empty(max(L.attn_workspace_bytes(p.desc), L.attn_bwd_workspace_bytes(p.desc)), dtype=torch.uint8, device="cuda")
    grads = [torch.empty_like(x) for x in (p.q, p.k, p.v)]

    def fwd():
        L.attn_fwd(p.desc, p.q, p.k, p.v, p.len_q, p.len_k, p.out, p.lse, p.weight, 0.25, ws)

    def bwd():
        L.attn_bwd(p.desc, p.q, p.k, p.v, p.len_q, p.len_k, p.out, p.lse, p.g, *grads, ws)

    def same(x, y):
        return torch.equal(torch.nan_to_num(x, nan=123.0), torch.nan_to_num(y, nan=123.0))

    fwd(), bwd()
    graphs = []
    for f in (fwd, bwd):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            f()
        graphs.append(g)
    w0 = p.weight.clone()
    for n in range(4):
        p.q.mul_(-1.0 if n % 2 else 0.5)
        p.weight.copy_(w0)
        graphs[0].replay(), graphs[1].replay()
        assert L.lmhead_check(ws) == 0
        got = [x.clone() for x in (p.out, p.lse, p.weight, *grads)]
        p.weight.copy_(w0)
        for x in (p.out, p.lse, *grads):
            x.fill_(9.0)
        fwd(), bwd()
        torch.cuda.synchronize()
        assert all(same(x, y) for x, y in zip(got, (p.out, p.lse, p.weight, *grads))), n


def test_eviction_in_a_graph():
    import torch
    import paper_2603_04411_amd as L
    B, T, H, keep = 2, 500, 3, 100
    gen = torch.Generator(device="cuda").manual_seed(1)
    k0, v0 = (torch.randn(B, T, H, 72, device="cuda", generator=gen) for _ in range(2))
    w0 = torch.rand(B, H, T, device="cuda", generator=gen)
    k, v, w = k0.clone(), v0.clone(), w0.clone()
    ev = L.make_evict_desc(B, T, H, keep, 3, 20)
    i32 = dict(dtype=torch.int32, device="cuda")
    lens, lens_out, kept = torch.tensor([500, 333], **i32), torch.empty(B, **i32), torch.empty(B, H, keep, **i32)
    ws, planes = torch.empty(L.evict_workspace_bytes(ev), dtype=torch.uint8, device="cuda"), L.make_cache_planes([k, v])
    L.cache_evict(ev, planes, w, lens, lens_out, kept, ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.cache_evict(ev, planes, w, lens, lens_out, kept, ws)
    for n in range(4):
        w0 = w0.roll(37 * n, 2).contiguous()
        k.copy_(k0), v.copy_(v0), w.copy_(w0), kept.fill_(-1), lens_out.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        assert lens_out.tolist() == [keep, keep]
        for b, h in ((b, h) for b in range(B) for h in range(H)):
            want = A.evict(w0[b, h].cpu().numpy(), int(lens[b]), keep, 3, 20)
            assert kept[b, h].tolist() == want
            assert torch.equal(k[b, :keep, h], k0[b, want, h]) and torch.equal(v[b, :keep, h], v0[b, want, h]) and torch.equal(w[b, h, :keep], w0[b, h, want])


def test_the_current_stream_is_used():
    """Inputs made on a side stream behind long work, read there; two calls at once with a workspace each."""
    import torch
    ps = [Problem(2, 60, 300, 4, 2, 64, seed=s, len_q=[60, 20], len_k=[300, 200]) for s in (1, 2)]
    kept = [[x.clone() for x in (p.q, p.k, p.v)] for p in ps]
    want = []
    for p in ps:
        p.fwd(weight=False)
        want.append((p.out.clone(), p.lse.clone()))
        for x in (p.q, p.k, p.v, p.out):
            x.fill_(1.0)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ps]
    big = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    for p, s, x in zip(ps, streams, kept):
        with torch.cuda.stream(s):
            for _ in range(10):
                big @ big
            for a, b in zip((p.q, p.k, p.v), x):
                a.copy_(b)
            p.fwd(weight=False)
    for p, s, (out, lse) in zip(ps, streams, want):
        s.synchronize()
        assert all(torch.equal(p.out[b, :n], out[b, :n]) for b, n in enumerate(p.lq)) and torch.equal(p.lse, lse)


def test_heads_and_sequences_that_share_memory():
    """Keys of one head, or of one sequence, read by all; keys that are the values too; keys and values side by side in one tensor."""
    import torch
    import paper_2603_04411_amd as L
    rng = np.random.default_rng(7)
    B, Tq, Tk, H, D = 2, 40, 150, 3, 64
    q = torch.from_numpy(rng.standard_normal((B, Tq, H, D))).bfloat16().cuda()
    kv = torch.from_numpy(rng.standard_normal((B, Tk, 2 * H, D))).bfloat16().cuda()
    pairs = [(kv[:, :, :1].expand(B, Tk, H, D),) * 2, (kv[:1, :, :H].expand(B, Tk, H, D), kv[:, :, H:]), (kv[:, :, ::2], kv[:, :, 1::2]),
             (kv[:, :, :H], kv[:, :, :H])]
    for k, v in pairs:
        got = []
        for kk, vv in ((k, v), (k.contiguous(), v.contiguous())):
            lay = [tuple(x.stride()[:3]) for x in (kk, vv)]
            desc = L.make_attn_desc(B, Tq, Tk, H, H, D, "bf16", k=lay[0], v=lay[1])
            out, w = torch.empty_like(q), torch.zeros(B, H, Tk, device="cuda")
            ws = torch.empty(L.attn_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
            L.attn_fwd(desc, q, kk, vv, None, None, out, None, w, 0.0, ws)
            got.append((out, w))
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
        want, bound = bounds(np64(q), np64(k), np64(v), [Tq] * B, [Tk] * B, float(np.float32(D ** -0.5)), 0, 0, "bf16")
        holds(np64(got[0][0]), want["out"], bound["out"], "out")


@pytest.mark.parametrize("Tq", [1, 70])
def test_offsets_past_32_bits(Tq):
    """Slots 16 MB apart, heads more than 4 GiB apart: forward, backward and eviction against the same call on dense copies, bit for bit."""
    import torch
    import paper_2603_04411_amd as L
    B, Tk, H, D, slot = 1, 300, 2, 64, 8_000_000
    head = slot * Tk + 64
    big = torch.empty(head * H, dtype=torch.bfloat16, device="cuda")       # 9.6 GB
    gen = torch.Generator(device="cuda").manual_seed(1)

    def make(T, at):
        t = big[at:].as_strided((B, T, H, D), (2 * head, slot, head, 1))
        return t, torch.randn(B, T, H, D, device="cuda", generator=gen).bfloat16()
    views, dense = zip(*(make(T, 128 * i) for i, T in enumerate((Tq, Tk, Tk, Tq, Tq, Tq, Tk, Tk))))
    for x, y in zip(views, dense):
        x.copy_(y)
    lay = [(2 * head, slot, head)] * 4
    results = []
    for (q, k, v, g, out, dq, dk, dv), l in ((views, lay), ([x.clone() for x in dense], [None] * 4)):
        desc = L.make_attn_desc(B, Tq, Tk, 2, 2, D, "bf16", q=l[0], k=l[1], v=l[2], o=l[3])
        lse = torch.empty(B, 2, Tq, device="cuda")
        w = torch.zeros(B, H, Tk, device="cuda")
        ws = torch.empty(max(L.attn_workspace_bytes(desc), L.attn_bwd_workspace_bytes(desc)), dtype=torch.uint8, device="cuda")
        L.attn_fwd(desc, q, k, v, None, None, out, lse, w, 0.0, ws)
        L.attn_bwd(desc, q, k, v, None, None, out, lse, g, dq, dk, dv, ws)
        ev = L.make_evict_desc(B, Tk, H, 100, 2, 10)
        i32 = dict(dtype=torch.int32, device="cuda")
        n, kept = torch.empty(B, **i32), torch.empty(B, H, 100, **i32)
        L.cache_evict(ev, L.make_cache_planes([k, v]), w, None, n, kept, ws)
        assert L.lmhead_check(ws) == 0
        results.append([x.contiguous() for x in (out, lse, dq, dk, dv, w, n, kept, k, v)])
    for i, (x, y) in enumerate(zip(*results)):
        assert torch.equal(x, y), i


def test_four_bit_cache_past_32_bits():
    """The last sequence of a cache whose codes take more than 4 GiB each: stored, then read."""
    import torch
    import paper_2603_04411_amd as L
    B, Tk, H, D = 64, 140001, 8, 128
    cache = [torch.zeros(B, H, Tk, w, dtype=torch.uint8, device="cuda") for w in (D // 2, D // 32) * 2]
    assert cache[0].numel() > 1 << 32
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn(B, 1, H, D, device="cuda", generator=gen).bfloat16() for _ in range(3))
    for c in cache[::2]:
        c[-1].copy_(torch.randint(0, 256, (H, Tk, D // 2), device="cuda", generator=gen, dtype=torch.uint8))
    for c in cache[1::2]:
        c[-1].copy_(torch.randint(124, 129, (H, Tk, D // 32), device="cuda", generator=gen, dtype=torch.uint8))
    lens = torch.ones(B, dtype=torch.int32, device="cuda")
    lens[-1] = Tk
    desc = L.make_attn_desc(B, 1, Tk, H, H, D, "bf16", k=L.attn_layout(k), v=L.attn_layout(v))
    out, ws = torch.empty_like(q), torch.empty(L.attn_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    w = torch.zeros(B, H, Tk, device="cuda")
    L.kv4_store(desc, k, v, None, lens, *cache, ws)
    L.kv4_attn(desc, q, *cache, None, lens, out, None, w, 1.0, ws)
    assert L.lmhead_check(ws) == 0
    c, e = A.quantise4(np64(k[-1, 0]))
    assert np.array_equal(cache[0][-1, :, -1].cpu().numpy(), c) and np.array_equal(cache[1][-1, :, -1].cpu().numpy(), e)
    h = H - 1
    K, V = (A.values4(cache[i][-1, h].cpu().numpy(), cache[i + 1][-1, h].cpu().numpy())[None, :, None] for i in (0, 2))
    want, bound = bounds(np64(q[-1:, :, h:]), K, V, [1], [Tk], float(np.float32(D ** -0.5)), 0, 0, "bf16")
    holds(np64(out[-1:, :, h:]), want["out"], bound["out"], "out")
    holds(np64(w[-1:, h:]), want["weight"], bound["weight"], "weight")
    # a sequence of one token answers with its value
    one = A.values4(*A.quantise4(np64(v[:-1, 0])))
    holds(np64(out[:-1, 0]), one, 2.0 ** -8 * np.abs(one) + 1e-30, "out of one token")


@pytest.mark.parametrize("name", ["q", "k", "v"])
def test_gradients_are_difference_quotients(name):
    """<gradient, d> against (f(x + h d) - f(x - h d)) / 2h with f = <out, g>.

    Every output of the two calls keeps its derived bound, so the quotient of the calls is that of 64 bits but for d = (d+ - d-) / 2h, where d+ and d- are
    what the two sums are off by.  The sum of the bounds of 21000 outputs over 2h would hide everything (it is 246, the slopes are 36), so d+ and d- are
    taken as they are, by subtraction in 64 bits, and the triangle inequality leaves: |<gradient, d> - quotient| <= (|d+| + |d-|) / 2h + what a quotient
    of that h is off by in 64 bits + sum of the gradient's bounds times |d|.  A slope in a direction of independent normal numbers is the gradient's norm
    in the mean of squares: the test says something where the bound is a small part of that."""
    import torch
    p = Problem(2, 50, 90, 4, 2, 64, dtype="f32", window=40, sinks=3, len_q=[50, 33], len_k=[90, 60], seed=9)
    at = "qkv".index(name)
    want, _ = p.exact()
    handed = torch.from_numpy(want["out"]).float().cuda()
    p.fwd(weight=False)
    p.bwd(handed)
    rng = np.random.default_rng(3)
    n = (p.lq, p.lk, p.lk)[at]
    d = rng.standard_normal(p.x[at].shape)
    for b in range(2):
        d[b, n[b]:] = 0
    h, g = 2.0 ** -8, p.x[3].copy()
    for b in range(2):
        g[b, p.lq[b]:] = 0
    x0, points, f_gpu, f_64, off = p.x[at].copy(), [], [], [], 0.0
    exact, limit = p.exact(out=np64(handed))
    for sign in (1, -1):
        x = (x0 + sign * h * d).astype(np.float32).astype(np.float64)
        (p.q, p.k, p.v)[at].copy_(torch.from_numpy(x))
        p.x[at] = x
        p.fwd(weight=False)
        r, e = p.exact()
        f_gpu.append(sum((np64(p.out)[b, :m] * g[b, :m]).sum() for b, m in enumerate(p.lq)))
        f_64.append((r["out"] * g).sum())
        holds(np64(p.out), r["out"], e["out"], "out")
        off += abs(f_gpu[-1] - f_64[-1]) / (2 * h)
        points.append(x)
    direction = (points[0] - points[1]) / (2 * h)
    grad, name = np.nan_to_num(np64((p.dq, p.dk, p.dv)[at])), "d" + name
    got, slope = (f_gpu[0] - f_gpu[1]) / (2 * h), sum((grad[b, :m] * direction[b, :m]).sum() for b, m in enumerate(n))
    off += abs((f_64[0] - f_64[1]) / (2 * h) - (exact[name] * direction).sum()) + (limit[name] * np.abs(direction)).sum()
    assert abs(got - slope) <= off and off < 0.2 * np.linalg.norm(grad), (got, slope, off)


def test_tensors_that_do_not_fit_are_refused():
    import torch
    p = Problem(2, 3, 9, 4, 2, 64)
    L, d, ws = p.L, p.desc, p.ws

    def call(**change):
        a = dict(q=p.q, k=p.k, v=p.v, len_q=None, len_k=None, out=p.out, lse=p.lse, weight=None, decay=1.0, ws=ws)
        L.attn_fwd(d, *{**a, **change}.values())
    call()
    for change in (dict(q=p.q.cpu()), dict(q=p.q.float()), dict(k=p.k[:, :8]), dict(k=p.k.transpose(1, 2).contiguous().transpose(1, 2)),
                   dict(v=p.v[:1]), dict(out=p.out.float()), dict(lse=p.lse[:1]), dict(lse=p.lse.double()), dict(weight=p.weight[:, :1]),
                   dict(len_q=torch.ones(2, dtype=torch.int64, device="cuda")), dict(len_k=torch.ones(1, dtype=torch.int32, device="cuda")),
                   dict(ws=ws.cpu()), dict(q=None)):
        with pytest.raises((ValueError, TypeError, AttributeError)):
            call(**change)
    for change, code in ((dict(ws=ws[:256]), -5), (dict(ws=ws[16:]), -4), (dict(out=p.q), -2), (dict(weight=p.weight, decay=-1.0), -2)):
        with pytest.raises(L.LmheadError) as e:
            call(**change)
        assert e.value.code == code
    c = Cache4(2, 1, 40, 4, 2, 64)
    with pytest.raises(ValueError):
        L.kv4_store(c.desc, c.k, c.v, None, None, c.cache[0][:, :1], *c.cache[1:], c.ws)
    with pytest.raises(ValueError):
        L.kv4_attn(c.desc, c.q, c.cache[0].to(torch.int16), *c.cache[1:], None, None, c.out, None, None, 1.0, c.ws)
    ev = L.make_evict_desc(2, 9, 2, 4)
    i32 = dict(dtype=torch.int32, device="cuda")
    for planes in ([p.k[:, :8]], [p.k[:, :, :1]], [p.k[:1]]):
        with pytest.raises(ValueError):
            L.cache_evict(ev, L.make_cache_planes(planes), p.weight, None, torch.empty(2, **i32), torch.empty(2, 2, 4, **i32), ws)
    for planes in ([p.k.cpu()], [p.k[0]], [p.k[..., ::2]]):
        with pytest.raises(ValueError):
            L.make_cache_planes(planes)
