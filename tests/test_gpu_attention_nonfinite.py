"""Infinities and NaN in queries, keys, values and gradients: how far they reach.  What they may not reach has the bits of the same call without them."""
import numpy as np
import pytest

from oracle import attention_oracle as A
from tests.attention_cases import holds
from tests.test_gpu_attention import Problem, np64
from tests.test_gpu_kv_cache import Cache4

pytestmark = pytest.mark.gpu

BAD = pytest.mark.parametrize("bad", [float("nan"), float("inf")], ids=["nan", "inf"])


def _weights(p, run, seen, hk, at):
    """Weights of a call with a query that is not finite: those of the keys that it does not see stay, and with a NaN the others are NaN."""
    import torch
    b, i, h, bad = at
    w0 = p.weight.clone()
    run()
    clean = p.weight.clone()
    p.weight.copy_(w0)
    p.q[b, i, h, 0] = bad
    run()
    want = torch.zeros(clean.shape, dtype=torch.bool)
    want[b, hk, :len(seen)] = torch.from_numpy(seen)
    got, clean = p.weight.cpu(), clean.cpu()
    assert torch.equal(got[~want], clean[~want])
    if bad != bad:
        assert torch.isnan(got[want]).all()


@BAD
@pytest.mark.parametrize("case", [dict(B=2, Tq=4, Tk=300, Hq=4, Hkv=2, D=64), dict(B=2, Tq=4, Tk=300, Hq=4, Hkv=2, D=64, window=50, sinks=3),
                                  dict(B=2, Tq=8, Tk=3000, Hq=2, Hkv=2, D=128, window=1000, sinks=3, dtype="f32"), dict(B=2, Tq=20, Tk=300, Hq=4, Hkv=2, D=64, window=50),
                                  dict(B=1, Tq=100, Tk=300, Hq=4, Hkv=2, D=64, window=50, sinks=40)],
                         ids=["few", "few-window", "few-f32", "packed", "long"])
def test_a_query_gives_weight_only_to_keys_it_sees(case, bad):
    p = Problem(seed=51, **case)
    i, h = p.lq[0] // 2, 1
    seen = A.visible(p.lq[0], p.lk[0], p.window, p.sinks)[i]
    assert 0 < seen.sum() < len(seen)
    _weights(p, lambda: p.fwd(decay=0.5), seen, h // (case["Hq"] // case["Hkv"]), (0, i, h, bad))


@BAD
def test_a_query_over_four_bits_gives_weight_only_to_keys_it_sees(bad):
    p = Cache4(2, 4, 900, 4, 2, 64, window=50, sinks=3, seed=52)
    seen = A.visible(4, 900, 50, 3)[1]
    _weights(p, lambda: p.attend(0.5), seen, 1, (1, 1, 2, bad))


def _copy(ts):
    return [t.clone() for t in ts]


def _seen(p, b, i):
    return A.visible(p.lq[b], p.lk[b], p.window, p.sinks)[i]


CASES = [dict(B=2, Tq=500, Tk=600, Hq=4, Hkv=2, D=64, window=100, sinks=3), dict(B=2, Tq=500, Tk=600, Hq=4, Hkv=2, D=128, window=100, sinks=3, dtype="f32"),
         dict(B=1, Tq=300, Tk=300, Hq=2, Hkv=2, D=64), dict(B=1, Tq=40, Tk=300, Hq=2, Hkv=2, D=64, window=33, sinks=40)]


@BAD
@pytest.mark.parametrize("where", ["q", "g"])
@pytest.mark.parametrize("case", CASES, ids=range(len(CASES)))
def test_a_query_or_its_gradient_reaches_keys_62_positions_from_those_it_sees(case, where, bad):
    """dk and dv of keys further away, of other key heads and of other sequences stay, and dq of other queries."""
    import torch
    p = Problem(seed=53, **case)
    p.fwd(weight=False)
    p.bwd(p.out)
    clean = _copy((p.dq, p.dk, p.dv))
    i, h = 2 * p.lq[0] // 3, 1
    (p.q if where == "q" else p.g)[0, i, h, 5] = bad
    p.fwd(weight=False)
    p.bwd(p.out)
    near = np.zeros(p.lk[0], dtype=bool)
    for j in np.flatnonzero(_seen(p, 0, i)):
        near[max(0, j - 62):j + 63] = True
    assert near.any()
    dq, dk, dv = (x.clone() for x in (p.dq, p.dk, p.dv))
    hk, rows = h // (case["Hq"] // case["Hkv"]), torch.from_numpy(np.flatnonzero(near)).cuda()
    for got, want in ((dk, clean[1]), (dv, clean[2])):
        got[0, rows, hk] = want[0, rows, hk]
        assert torch.equal(got, want)
    dq[0, i, h] = clean[0][0, i, h]
    assert torch.equal(dq, clean[0])


@BAD
@pytest.mark.parametrize("where", ["k", "v"])
@pytest.mark.parametrize("case", CASES, ids=range(len(CASES)))
def test_a_key_or_value_reaches_queries_127_positions_from_those_that_see_it(case, where, bad):
    """out, lse and dq of queries further away, of heads that read another key head and of other sequences stay.  lse of nearer ones that do not see it
    keeps its derived bound: the maximum that a wavefront's exponentials are taken against moves for all of its rows when it moves for one."""
    import torch
    p = Problem(seed=54, **case)
    p.fwd(weight=False)
    p.bwd(p.out)
    clean = _copy((p.out, p.dq, p.lse))
    j = p.lk[0] - p.lq[0] + p.lq[0] // 4
    (p.k if where == "k" else p.v)[0, j, 1, 5] = bad
    p.fwd(weight=False)
    p.bwd(p.out)
    sees = A.visible(p.lq[0], p.lk[0], p.window, p.sinks)[:, j]
    near = np.zeros(p.lq[0], dtype=bool)
    for i in np.flatnonzero(sees):
        near[max(0, i - 127):i + 128] = True
    heads = slice(case["Hq"] // case["Hkv"], 2 * case["Hq"] // case["Hkv"])
    out, dq, lse = _copy((p.out, p.dq, p.lse))
    rows = torch.from_numpy(np.flatnonzero(near)).cuda()
    for got, want in ((out, clean[0]), (dq, clean[1])):
        got[0, rows, heads] = want[0, rows, heads]
        assert torch.equal(got, want)
    far = np.ones(clean[2].shape, dtype=bool)
    far[0, heads] = ~near
    far = torch.from_numpy(far).cuda()
    assert torch.equal(lse[far], clean[2][far])
    want, bound = p.exact()      # of the inputs without the bad one
    for x in (lse, clean[2]):
        holds(np64(x)[0, heads][:, ~sees], want["lse"][0, heads][:, ~sees], bound["lse"][0, heads][:, ~sees], "lse")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Tq,Hq", [(1, 2), (12, 2), (200, 2)], ids=["few", "rows", "prompt"])
def test_logits_of_two_to_the_30(dtype, Tq, Hq):
    """Logits of -2^30 to 2^30 in steps of 2^29: the keys with a query's largest one share its weight equally, whatever the fused product leaves of
    numbers of that size (they leave the same of equal logits).  Values are whole numbers: their mean over up to Tk keys is off by its roundings."""
    import torch
    import paper_2603_04411_amd as L
    Tk, D, tdt = 300, 64, torch.bfloat16 if dtype == "bf16" else torch.float32
    rng = np.random.default_rng(55)
    c = rng.integers(-2, 3, Tk).astype(np.float64)
    c[0] = -2.0      # the first queries see no large one
    sign = rng.choice([-1.0, 1.0], (1, Tq, Hq))
    q, k = np.zeros((1, Tq, Hq, D)), np.zeros((1, Tk, 1, D))
    q[..., 3], k[0, :, 0, 3] = sign * 2.0 ** 15, c * 2.0 ** 14
    v = rng.integers(-8, 9, (1, Tk, 1, D)).astype(np.float64)
    dq, dk, dv = (torch.from_numpy(x).to(tdt).cuda() for x in (q, k, v))
    d = L.make_attn_desc(1, Tq, Tk, Hq, 1, D, dtype, scale=1.0)
    out, lse = torch.empty_like(dq), torch.empty(1, Hq, Tq, device="cuda")
    weight = torch.zeros(1, 1, Tk, device="cuda") if Tq * Hq <= 8 else None      # of more rows P comes from lse, which has steps of 64 here
    ws = torch.empty(L.attn_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    L.attn_fwd(d, dq, dk, dv, None, None, out, lse, weight, 0.0, ws)
    u, total = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}[dtype], np.zeros(Tk)
    for i in range(Tq):
        for h in range(Hq):
            seen = Tk - Tq + i + 1
            z = sign[0, i, h] * c[:seen]
            top = np.flatnonzero(z == z.max())
            total[top] += 1.0 / len(top)
            want = v[0, top, 0].mean(0)
            bound = 1.1 * (u * (np.abs(v[0, top, 0]).mean(0) + np.abs(want)) + 2 * (seen + 8) * 2.0 ** -24 * 8)
            holds(np64(out)[0, i, h], want, bound + 1e-30, "out")
            holds(np64(lse)[0, h, i:i + 1], np.array([z.max() * 2.0 ** 29]), np.array([2.0 ** 6 + 8.0]), "lse")
    if weight is not None:
        holds(np64(weight)[0, 0], total, 1.1 * (Tk + 16) * 2.0 ** -24 * total + 1e-30, "weight")
