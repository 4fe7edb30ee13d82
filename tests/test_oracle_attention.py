"""Pins of the attention oracle: brute force over single pairs, torch's autograd and softmax, central differences, the 4-bit grid by search, eviction by
a plain sort."""
import itertools

import numpy as np
import pytest

from oracle import attention_oracle as A


def problem(B=2, Tq=5, Tk=7, Hq=4, Hkv=2, D=8, seed=0):
    rng = np.random.default_rng(seed)
    q, k, v = (rng.standard_normal((B, T, H, D)) for T, H in ((Tq, Hq), (Tk, Hkv), (Tk, Hkv)))
    return q, k, v, np.array([Tq, 3][:B]), np.array([Tk, 2][:B])


@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (3, 0), (2, 1), (3, 2), (100, 5)])
def test_forward_pair_by_pair(window, sinks):
    q, k, v, lq, lk = problem()
    out, lse, weight = A.attn_fwd(q, k, v, lq, lk, 0.3, window, sinks)
    want_w = np.zeros_like(weight)
    for b, i, h in itertools.product(range(2), range(5), range(4)):
        p = lk[b] - lq[b] + i
        seen = [j for j in range(7) if i < lq[b] and 0 <= j <= p and j < lk[b] and (window == 0 or j > p - window or j < sinks)]
        if not seen:
            assert (out[b, i, h] == 0).all() and lse[b, h, i] == -np.inf
            continue
        z = [0.3 * float(np.dot(q[b, i, h], k[b, j, h // 2])) for j in seen]
        total = sum(np.exp(x) for x in z)
        P = [np.exp(x) / total for x in z]
        assert np.isclose(lse[b, h, i], np.log(total))
        assert np.allclose(out[b, i, h], sum(x * v[b, j, h // 2] for x, j in zip(P, seen)))
        for x, j in zip(P, seen):
            want_w[b, h // 2, j] += x
    assert np.allclose(weight, want_w)
    assert np.isclose(weight.sum(), np.isfinite(lse).sum())      # every query that sees something gives one


def test_full_attention_is_torch_softmax():
    import torch
    q, k, v, *_ = problem(B=1, Tq=6, Tk=6)
    out, lse, _ = A.attn_fwd(q, k, v, [6], [6], 8 ** -0.5)
    tq, tk, tv = (torch.from_numpy(x).transpose(1, 2) for x in (q, np.repeat(k, 2, 2), np.repeat(v, 2, 2)))
    want = torch.nn.functional.scaled_dot_product_attention(tq, tk, tv, is_causal=True)
    assert np.allclose(out, want.transpose(1, 2).numpy())


def test_backward_is_autograd_and_a_difference_quotient():
    q, k, v, lq, lk = problem(seed=3)
    rng = np.random.default_rng(1)
    g = rng.standard_normal(q.shape)
    args = (lq, lk, 0.4, 3, 1)

    def loss(q, k, v):
        return float((A.attn_fwd(q, k, v, *args)[0] * g).sum())
    out = A.attn_fwd(q, k, v, *args)[0]
    grads = A.attn_bwd(q, k, v, lq, lk, out, g, 0.4, 3, 1)
    for n, x in enumerate((q, k, v)):
        for _ in range(12):
            at = tuple(rng.integers(0, s) for s in x.shape)
            parts = []
            for e in (1e-5, -1e-5):
                y = [q.copy(), k.copy(), v.copy()]
                y[n][at] += e
                parts.append(loss(*y))
            assert abs((parts[0] - parts[1]) / 2e-5 - grads[n][at]) <= 1e-8 + 1e-6 * abs(grads[n][at])
    # queries behind the end, and keys that nobody sees, have none
    assert (grads[0][1, 3:] == 0).all() and (grads[1][1, 2:] == 0).all()


def test_four_bits_by_search():
    rng = np.random.default_rng(4)
    x = rng.standard_normal((40, 64)) * 2.0 ** rng.integers(-20, 20, (40, 1))
    codes, scales = A.quantise4(x)
    back = A.values4(codes, scales)
    for r in range(40):
        for block in range(2):
            y = x[r, 32 * block:32 * block + 32]
            size = 2.0 ** (int(scales[r, block]) - 127)
            assert np.abs(y).max() <= 6 * size and np.abs(y).max() > 3 * size
            for j in range(32):
                off = np.abs(np.concatenate([A.GRID, -A.GRID]) * size - y[j])
                assert abs(back[r, 32 * block + j] - y[j]) == off.min()
    even = np.zeros((1, 32))
    even[0, :8] = [6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    assert A.values4(*A.quantise4(even))[0, :8].tolist() == [6.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0]
    odd = np.full((3, 32), 1.0)
    odd[0, 3], odd[1, 3], odd[2] = np.inf, np.nan, 0.0
    c, s = A.quantise4(odd)
    assert s.tolist() == [[255], [255], [1]] and (c == 0).all() and np.isnan(A.values4(c, s)[:2]).all() and (A.values4(c, s)[2] == 0).all()
    big = np.full((1, 32), 3.3e38)
    assert A.quantise4(big)[1][0, 0] == 252 and np.isfinite(A.values4(*A.quantise4(big)).astype(np.float32)).all()


def test_eviction_by_hand():
    w = np.array([9.0, 1.0, 5.0, 5.0, np.nan, 7.0, 5.0, 0.0], dtype=np.float32)
    assert A.evict(w, 8, 8, 0, 0) == list(range(8)) and A.evict(w, 3, 8, 0, 0) == [0, 1, 2]
    assert A.evict(w, 8, 3, 0, 0) == [0, 2, 5]              # of the three fives the first
    assert A.evict(w, 8, 4, 2, 1) == [0, 1, 5, 7]
    assert A.evict(w, 8, 7, 0, 0) == [0, 1, 2, 3, 5, 6, 7]  # NaN goes before 0
    assert A.evict(w, 8, 2, 1, 1) == [0, 7]
