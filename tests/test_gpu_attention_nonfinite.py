"""Infinities and NaN in queries, keys, values and gradients: how far they reach.  What they may not reach has the bits of the same call without them."""
import numpy as np
import pytest

from oracle import attention_oracle as A
from tests.test_gpu_attention import Problem
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
