"""Attention over a window and a few first tokens, its backward and the accumulated weights, against the fp64 oracle with derived bounds
(``tests/attention_cases.py``): head widths, groups of heads, lengths on both sides of tiles and blocks, empty rows and sequences, layouts, garbage in
every place that no query sees."""
import numpy as np
import pytest

from tests.attention_cases import bounds, holds

pytestmark = pytest.mark.gpu


def place(x, first, tdt, garbage):
    """x [B, T, H, D] on the device inside a larger buffer of garbage, with the layout that is asked for."""
    import torch
    B, T, H, D = x.shape
    t = torch.from_numpy(np.ascontiguousarray(x)).to(tdt).cuda()
    if first == "dense":
        return t.contiguous()
    if first == "head":                      # [B, H, T, D]
        return t.transpose(1, 2).contiguous().transpose(1, 2)
    if first == "wide":                      # rows and heads apart, sequences in the middle
        big = torch.full((T + 1, B, H + 1, D + 8), garbage, dtype=tdt, device="cuda")
        view = big[:T, :, :H, :D].permute(1, 0, 2, 3)
        view.copy_(t)
        return view
    raise ValueError(first)


class Problem:
    def __init__(self, B, Tq, Tk, Hq, Hkv, D, dtype="bf16", window=0, sinks=0, len_q=None, len_k=None, first="dense", seed=0, scale=None,
                 spread=1.0):
        import torch
        import paper_2603_04411_amd as L
        self.L, self.dtype = L, dtype
        self.tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
        rng = np.random.default_rng(seed + 1000 * Tq + Tk)
        self.window, self.sinks = window, sinks
        self.lq = np.array([Tq] * B if len_q is None else len_q)
        self.lk = np.array([Tk] * B if len_k is None else len_k)
        raw = [rng.standard_normal((B, T, H, D)) * s for T, H, s in ((Tq, Hq, spread), (Tk, Hkv, 1.0), (Tk, Hkv, 1.0), (Tq, Hq, 1.0))]
        self.x = []                          # exactly representable
        for a, n in zip(raw, (self.lq, self.lk, self.lk, self.lq)):
            a = torch.from_numpy(a).to(self.tdt).double().numpy()
            self.x.append(a)
        dirty = [a.copy() for a in self.x]
        for a, n in zip(dirty, (self.lq, self.lk, self.lk, self.lq)):
            for b in range(B):
                a[b, max(0, int(n[b])):] = np.nan      # what lies behind a sequence's end is never used
        self.q, self.k, self.v, self.g = (place(a, first, self.tdt, float("nan")) for a in dirty)
        self.out = place(np.full((B, Tq, Hq, D), 7.0), first, self.tdt, 5.0)
        self.scale = float(np.float32(D ** -0.5 if scale is None else scale))
        self.desc = L.make_attn_desc(B, Tq, Tk, Hq, Hkv, D, dtype, window=window, sinks=sinks, scale=self.scale, q=L.attn_layout(self.q),
                                     k=L.attn_layout(self.k), v=L.attn_layout(self.v), o=L.attn_layout(self.out))
        assert L.attn_validate_desc(self.desc) == 0
        dev = dict(dtype=torch.int32, device="cuda")
        self.len_q = None if len_q is None else torch.tensor(list(len_q), **dev)
        self.len_k = None if len_k is None else torch.tensor(list(len_k), **dev)
        self.lse = torch.full((B, Hq, Tq), 7.0, device="cuda")
        self.weight = torch.rand(B, Hkv, Tk, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))
        self.ws = torch.full((L.attn_workspace_bytes(self.desc),), 255, dtype=torch.uint8, device="cuda")

    def fwd(self, weight=True, decay=0.5):
        self.L.attn_fwd(self.desc, self.q, self.k, self.v, self.len_q, self.len_k, self.out, self.lse, self.weight if weight else None, decay, self.ws)

    def bwd(self, out):
        import torch
        self.dq, self.dk, self.dv = (place(np.full(t.shape, 3.0), "dense", self.tdt, 5.0).as_strided(t.shape, t.stride())
                                     if t.is_contiguous() else _same(t) for t in (self.q, self.k, self.v))
        ws = torch.full((self.L.attn_bwd_workspace_bytes(self.desc),), 255, dtype=torch.uint8, device="cuda")
        self.L.attn_bwd(self.desc, self.q, self.k, self.v, self.len_q, self.len_k, out, self.lse, self.g, self.dq, self.dk, self.dv, ws)
        assert self.L.lmhead_check(ws) == 0

    def exact(self, out=None):
        lq, lk = np.clip(self.lq, 0, self.x[0].shape[1]), np.clip(self.lk, 0, self.x[1].shape[1])
        return bounds(*self.x[:3], lq, lk, self.scale, self.window, self.sinks, self.dtype, out=out, g=None if out is None else self.x[3])


def _same(t):
    """A tensor of t's strides in a buffer of its own, filled with 3."""
    import torch
    n = sum((a - 1) * s for a, s in zip(t.shape, t.stride())) + 1
    return torch.full((n,), 3.0, dtype=t.dtype, device="cuda").as_strided(t.shape, t.stride())


def np64(t):
    return t.double().cpu().numpy()


def check_fwd(p, decay=0.5):
    before = np64(p.weight)
    p.fwd(decay=decay)
    assert p.L.lmhead_check(p.ws) == 0
    want, bound = p.exact()
    holds(np64(p.out), want["out"], bound["out"], "out")
    holds(np64(p.lse), want["lse"], bound["lse"], "lse")
    for b in range(len(p.lk)):
        n = int(p.lk[b])
        old = decay * before[b, :, :n]
        holds(np64(p.weight)[b, :, :n], old + want["weight"][b, :, :n], bound["weight"][b, :, :n] + 2.0 ** -22 * (old + want["weight"][b, :, :n]), "weight")
        assert np.array_equal(np64(p.weight)[b, :, n:], before[b, :, n:])


def check_bwd(p):
    """With the exact output, rounded to the storage type, and lse as the forward left it."""
    import torch
    p.fwd(weight=False)
    want, _ = p.exact()
    out = torch.from_numpy(want["out"]).to(p.tdt)
    handed = _same(p.out)
    handed.copy_(out.cuda())
    p.bwd(handed)
    want, bound = p.exact(out=out.double().numpy())
    for n in ("dq", "dk", "dv"):
        holds(np64(getattr(p, n)), want[n], bound[n], n)


CASES = [
    # B, Tq, Tk, Hq, Hkv, D, dtype, window, sinks, len_q, len_k, first
    dict(B=1, Tq=1, Tk=1, Hq=1, Hkv=1, D=8),
    dict(B=1, Tq=1, Tk=1, Hq=1, Hkv=1, D=8, dtype="f32"),
    dict(B=2, Tq=5, Tk=5, Hq=2, Hkv=1, D=64),
    dict(B=2, Tq=5, Tk=5, Hq=2, Hkv=1, D=64, dtype="f32"),
    dict(B=1, Tq=33, Tk=33, Hq=4, Hkv=4, D=32),
    dict(B=1, Tq=32, Tk=64, Hq=4, Hkv=4, D=40, dtype="f32"),
    dict(B=2, Tq=65, Tk=65, Hq=6, Hkv=2, D=72),
    dict(B=2, Tq=129, Tk=129, Hq=3, Hkv=3, D=128),
    dict(B=2, Tq=129, Tk=129, Hq=3, Hkv=3, D=128, dtype="f32"),
    dict(B=1, Tq=127, Tk=256, Hq=7, Hkv=1, D=96),
    dict(B=1, Tq=127, Tk=256, Hq=7, Hkv=1, D=96, dtype="f32"),
    dict(B=3, Tq=100, Tk=200, Hq=4, Hkv=2, D=128, len_q=[100, 1, 37], len_k=[200, 1, 64]),
    dict(B=3, Tq=100, Tk=200, Hq=4, Hkv=2, D=80, len_q=[100, 1, 37], len_k=[200, 1, 64], dtype="f32"),
    # windows and first tokens
    dict(B=1, Tq=70, Tk=70, Hq=2, Hkv=2, D=64, window=1),
    dict(B=1, Tq=300, Tk=300, Hq=2, Hkv=2, D=64, window=1, sinks=1),
    dict(B=1, Tq=300, Tk=300, Hq=2, Hkv=1, D=128, window=64, sinks=4),
    dict(B=1, Tq=300, Tk=300, Hq=2, Hkv=1, D=128, window=64, sinks=4, dtype="f32"),
    dict(B=1, Tq=260, Tk=260, Hq=4, Hkv=1, D=64, window=33, sinks=100),
    dict(B=1, Tq=200, Tk=200, Hq=1, Hkv=1, D=64, window=1000, sinks=300),
    dict(B=1, Tq=200, Tk=200, Hq=1, Hkv=1, D=64, window=50, sinks=199),
    dict(B=2, Tq=400, Tk=500, Hq=2, Hkv=2, D=64, window=100, sinks=65, len_q=[400, 111], len_k=[500, 333]),
    dict(B=1, Tq=1, Tk=700, Hq=8, Hkv=2, D=128, window=129, sinks=3),
    dict(B=1, Tq=3, Tk=700, Hq=8, Hkv=2, D=128, window=129, sinks=130, dtype="f32"),
    # rows and sequences that see nothing
    dict(B=4, Tq=40, Tk=40, Hq=2, Hkv=2, D=64, len_q=[40, 0, 17, 40], len_k=[7, 40, 0, 40]),
    dict(B=4, Tq=40, Tk=40, Hq=2, Hkv=2, D=64, len_q=[40, 0, 17, 40], len_k=[7, 40, 0, 40], dtype="f32", window=5, sinks=1),
    dict(B=2, Tq=200, Tk=90, Hq=2, Hkv=1, D=128, len_q=[200, 150], len_k=[90, 1]),
    # single tokens over caches, one and several parts
    dict(B=3, Tq=1, Tk=100, Hq=8, Hkv=1, D=128, len_q=[1, 1, 1], len_k=[100, 1, 33]),
    dict(B=2, Tq=1, Tk=1500, Hq=32, Hkv=4, D=128, len_k=[1500, 777]),
    dict(B=2, Tq=1, Tk=1500, Hq=4, Hkv=4, D=64, len_k=[1500, 777], dtype="f32"),
    dict(B=1, Tq=4, Tk=3001, Hq=16, Hkv=2, D=128),
    dict(B=1, Tq=5, Tk=3001, Hq=14, Hkv=2, D=128, window=2000, sinks=1),
    dict(B=2, Tq=16, Tk=2000, Hq=16, Hkv=4, D=96, len_q=[16, 9], len_k=[1999, 64]),
    dict(B=4, Tq=4, Tk=900, Hq=8, Hkv=2, D=128, len_q=[4, 1, 0, 3], len_k=[900, 800, 700, 2]),
    dict(B=3, Tq=8, Tk=1200, Hq=4, Hkv=4, D=64, len_q=[8, 5, 1], len_k=[1200, 1100, 400], window=130, sinks=3),
    dict(B=3, Tq=8, Tk=1200, Hq=8, Hkv=2, D=64, len_q=[8, 5, 1], len_k=[1200, 1100, 400], window=130, sinks=70, dtype="f32"),
    # layouts
    dict(B=2, Tq=90, Tk=130, Hq=4, Hkv=2, D=64, first="head", len_q=[90, 31], len_k=[130, 99]),
    dict(B=2, Tq=90, Tk=130, Hq=4, Hkv=2, D=56, first="wide", len_q=[90, 31], len_k=[130, 99]),
    dict(B=2, Tq=90, Tk=130, Hq=4, Hkv=2, D=56, first="wide", len_q=[90, 31], len_k=[130, 99], dtype="f32", window=40, sinks=2),
    dict(B=2, Tq=1, Tk=600, Hq=4, Hkv=2, D=128, first="wide", len_k=[600, 500]),
    # logits far from 0
    dict(B=1, Tq=130, Tk=130, Hq=2, Hkv=2, D=64, spread=8.0),
    dict(B=1, Tq=130, Tk=130, Hq=2, Hkv=2, D=64, spread=30.0, dtype="f32", window=70, sinks=1),
    dict(B=1, Tq=2, Tk=500, Hq=2, Hkv=2, D=64, spread=30.0, scale=1.5),
]


def _name(c):
    return "-".join(f"{k}{v}" for k, v in c.items()).replace(" ", "")


@pytest.mark.parametrize("case", CASES, ids=_name)
def test_forward_and_weights(case):
    check_fwd(Problem(**case))


@pytest.mark.parametrize("case", CASES, ids=_name)
def test_backward(case):
    check_bwd(Problem(**case))


def test_without_lse_and_weight_and_with_decay_0():
    import torch
    p = Problem(2, 50, 90, 4, 2, 64, len_q=[50, 20], len_k=[90, 60], window=30, sinks=2)
    p.fwd()
    out, lse = p.out.clone(), p.lse
    p.out.fill_(9.0)
    p.lse = None
    p.weight.fill_(float("nan"))
    p.fwd(decay=0.0)
    assert torch.equal(out, p.out)
    want, bound = p.exact()
    for b, n in enumerate((90, 60)):
        holds(np64(p.weight)[b, :, :n], want["weight"][b, :, :n], bound["weight"][b, :, :n] + 2.0 ** -22 * want["weight"][b, :, :n], "weight")
        assert torch.isnan(p.weight[b, :, n:]).all()
    p.out.fill_(9.0)
    p.fwd(weight=False)
    assert torch.equal(out, p.out) and lse is not None


def test_lengths_out_of_range_are_reported_and_taken_as_the_nearest():
    import torch
    p = Problem(3, 40, 60, 2, 1, 64, len_q=[40, 30, 20], len_k=[60, 50, 41])
    q = Problem(3, 40, 60, 2, 1, 64, len_q=[40, 30, 20], len_k=[60, 50, 41])
    p.fwd()
    q.len_q[0], q.len_k[0] = 41, 1000
    q.fwd()
    assert q.L.lmhead_check(q.ws) == -6 and q.L.lmhead_check(p.ws) == 0
    assert torch.equal(p.out, q.out) and torch.equal(p.lse, q.lse)
    q.len_q[1], q.len_k[2] = -5, -(2 ** 31)
    q.fwd()
    assert q.L.lmhead_check(q.ws) == -6
    assert (q.out[1:] == 0).all() and torch.isinf(q.lse[1:]).all()


def test_bits_are_the_same_from_run_to_run():
    import torch
    for c in (CASES[12], CASES[20], CASES[27], CASES[29], CASES[33]):
        p = Problem(**c)
        p.fwd(decay=0.0)
        first = [p.out.clone(), p.lse.clone(), p.weight.clone()]
        p.bwd(p.out)
        first += [p.dq, p.dk, p.dv]
        p.fwd(decay=0.0)
        p.bwd(p.out)
        assert all(torch.equal(a, b) for a, b in zip(first, [p.out, p.lse, p.weight, p.dq, p.dk, p.dv]))


LONG = [      # queries that the weights' pass cuts: with a window and blocks of first tokens, without, in fp32, padded
    dict(B=1, Tq=900, Tk=1300, Hq=4, Hkv=2, D=128, window=100, sinks=140),
    dict(B=2, Tq=700, Tk=700, Hq=7, Hkv=1, D=64, len_q=[700, 333], len_k=[700, 333]),
    dict(B=2, Tq=600, Tk=1000, Hq=2, Hkv=2, D=72, window=64, sinks=3, len_q=[600, 1], len_k=[1000, 900]),
    dict(B=1, Tq=500, Tk=900, Hq=2, Hkv=1, D=128, dtype="f32", window=300, sinks=1),
    dict(B=3, Tq=400, Tk=500, Hq=2, Hkv=1, D=40, window=1, sinks=129, len_q=[400, 0, 7], len_k=[300, 500, 0]),
]


@pytest.mark.parametrize("case", LONG, ids=_name)
def test_weights_of_long_prompts(case):
    check_fwd(Problem(seed=21, **case), decay=0.75)


PACKED = [      # fewer queries than a tile of the weights' pass, whose rows are packed
    dict(B=2, Tq=31, Tk=300, Hq=8, Hkv=2, D=128, window=70, sinks=130, len_q=[31, 5], len_k=[300, 2]),
    dict(B=3, Tq=3, Tk=260, Hq=27, Hkv=3, D=64, len_q=[3, 0, 1], len_k=[260, 129, 128]),
    dict(B=1, Tq=1, Tk=1000, Hq=40, Hkv=1, D=128, window=64, sinks=1, dtype="f32"),
    dict(B=2, Tq=9, Tk=5, Hq=4, Hkv=1, D=96, len_q=[9, 9], len_k=[5, 0], first="wide"),
]


@pytest.mark.parametrize("case", PACKED, ids=_name)
def test_weights_of_packed_rows(case):
    check_fwd(Problem(seed=22, **case), decay=0.5)
