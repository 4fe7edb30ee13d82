"""Where bf16 storage does not mean that a factor is rounded to bf16: dS in dk, where at most 512 queries of a head see a block of 128 keys (whatever the
slots for queries), and P in out, of up to 32 rows over a plain cache, are two bf16 numbers.

With two numbers what rounding leaves of x is u^2 |x| (the high part is off by u |x| at most, the difference from it is exact in fp32, and the low part
is off by u of that), where ``attention_cases.bounds`` has u |x|: the bounds here are those less what the coarser rounding was allowed."""
import numpy as np
import pytest

from oracle import attention_oracle as A
from tests.attention_cases import U, holds
from tests.test_gpu_attention import Problem, _same, np64

pytestmark = pytest.mark.gpu


def fine_bound(p, bound, out):
    """Bound of dk with dS in sixteen bits."""
    q, k, v, g = p.x
    less, u = np.zeros(k.shape), U["bf16"]
    for b, (lq, lk) in enumerate(zip(p.lq, p.lk)):
        see = A.visible(lq, lk, p.window, p.sinks)
        for h, hk in A.heads(q.shape[2], k.shape[2]):
            P, _, _ = A.probabilities(q[b, :lq, h], k[b, :lk, hk], p.scale, see)
            go, o = g[b, :lq, h], P @ v[b, :lk, hk]
            dS = P * (go @ v[b, :lk, hk].T - (go * o).sum(1)[:, None])
            less[b, :lk, hk] += p.scale * ((u - u * u) * np.abs(dS)).T @ np.abs(q[b, :lq, h])
    return bound - 1.1 * less


def few_see(p):
    """[B, Tk]: keys of blocks that at most 512 queries of a head see."""
    few = np.zeros((len(p.lk), p.x[1].shape[1]), dtype=bool)
    for b, (lq, lk) in enumerate(zip(p.lq, p.lk)):
        see = A.visible(lq, lk, p.window, p.sinks)
        for s in range(0, lk, 128):
            few[b, s:s + 128] = see[:, s:s + 128].any(1).sum() <= 512
    return few


@pytest.mark.parametrize("case,share", [
    (dict(B=1, Tq=900, Tk=900, Hq=4, Hkv=2, D=64, window=100), 1.0),
    (dict(B=1, Tq=900, Tk=900, Hq=4, Hkv=2, D=128, window=100, sinks=3), 0.85),                          # but for the first block
    (dict(B=3, Tq=1100, Tk=1100, Hq=2, Hkv=1, D=128, len_q=[60, 1100, 300], len_k=[60, 1100, 300]), 0.29),
    (dict(B=2, Tq=600, Tk=600, Hq=2, Hkv=2, D=72, len_q=[512, 513], len_k=[512, 513]), 0.8),             # both sides of the line
    (dict(B=1, Tq=512, Tk=700, Hq=2, Hkv=1, D=64), 1.0),
], ids=["window", "sinks", "padding", "line", "short"])
def test_few_queries_keep_sixteen_bits_of_ds(case, share):
    import torch
    p = Problem(seed=31, **case)
    p.fwd(weight=False)
    want, _ = p.exact()
    out = torch.from_numpy(want["out"]).to(p.tdt)
    handed = _same(p.out)
    handed.copy_(out.cuda())
    p.bwd(handed)
    want, bound = p.exact(out=out.double().numpy())
    few = few_see(p)
    assert few.mean() >= share
    got = np64(p.dk)
    holds(got, want["dk"], bound["dk"], "dk")
    fine = fine_bound(p, bound["dk"], out)
    holds(np.where(few[:, :, None, None], got, 0), np.where(few[:, :, None, None], want["dk"], 0), fine, "dk of few queries")


@pytest.mark.parametrize("case", [
    dict(B=2, Tq=1, Tk=1500, Hq=8, Hkv=2, D=128, len_k=[1500, 777]),
    dict(B=1, Tq=1, Tk=700, Hq=8, Hkv=2, D=64, window=129, sinks=3),
    dict(B=1, Tq=4, Tk=3001, Hq=16, Hkv=2, D=96),
    dict(B=2, Tq=32, Tk=500, Hq=2, Hkv=2, D=128, len_q=[32, 9], len_k=[499, 64]),
], ids=["decode", "window", "draft", "rows"])
def test_few_rows_keep_sixteen_bits_of_p(case):
    p = Problem(seed=32, **case)
    u, (q, k, v, _) = U["bf16"], p.x
    less = np.zeros(q.shape)
    for b, (lq, lk) in enumerate(zip(p.lq, p.lk)):
        see = A.visible(lq, lk, p.window, p.sinks)
        for h, hk in A.heads(q.shape[2], k.shape[2]):
            P, _, _ = A.probabilities(q[b, :lq, h], k[b, :lk, hk], p.scale, see)
            less[b, :lq, h] = (u - u * u) * (P @ np.abs(v[b, :lk, hk]))
    want, bound = p.exact()
    p.fwd(weight=False)
    plain = np64(p.out).copy()
    p.fwd()
    for got in (plain, np64(p.out)):
        holds(got, want["out"], bound["out"] - 1.1 * less, "out")
