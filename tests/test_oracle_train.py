"""The oracle of preference loss, embedding and gradient clipping against closed forms, brute force and differences."""
import math

import numpy as np
import pytest

from oracle import train_oracle as O


def _problem(seed, P=3, G=4, T=6):
    r = np.random.default_rng(seed)
    R = P * G
    return dict(logp=-r.random(R * T), ref=-r.random(R * T), reward=r.integers(0, 4, R) / 4.0, lens=r.integers(0, T + 1, R), P=P, G=G, T=T)


@pytest.mark.parametrize("loss", ["logistic", "hinge", "squared"])
@pytest.mark.parametrize("extremes", [False, True])
@pytest.mark.parametrize("mean", [False, True])
def test_preference_gradient_is_the_difference_quotient(loss, extremes, mean):
    q = _problem(7)
    kw = dict(loss=loss, extremes=extremes, mean=mean, per_pair=extremes, beta=0.7, margin=0.2, margin_scale=0.3,
              smoothing=0.1 if loss == "logistic" else 0.0, nll_coef=0.4)

    def f(lp):
        return O.preference_loss(lp, q["ref"], q["reward"], q["lens"], q["P"], q["G"], q["T"], **kw)[0]
    _, g, _, _ = O.preference_loss(q["logp"], q["ref"], q["reward"], q["lens"], q["P"], q["G"], q["T"], **kw)
    for i in range(0, q["logp"].size, 5):
        e = np.zeros_like(q["logp"])
        e[i] = 1e-6
        assert abs((f(q["logp"] + e) - f(q["logp"] - e)) / 2e-6 - g[i]) <= 1e-8 + 1e-6 * abs(g[i])


def test_preference_closed_forms():
    # one pair, one token each: u = (-1 - -2) - (-3 - -1) = 3
    args = ([-1.0, -3.0], [-2.0, -1.0], [1.0, 0.0], [1, 1], 1, 2, 1)
    l, g, ratio, stats = O.preference_loss(*args, beta=0.5)
    assert abs(l + math.log(1 / (1 + math.exp(-1.5)))) < 1e-15 and np.allclose(ratio, [1.0, -2.0])
    assert np.allclose(g, [-0.5 / (1 + math.exp(1.5)), 0.5 / (1 + math.exp(1.5))])
    assert np.allclose(stats, [1.0, 0.5, -1.0, 1.0])
    assert O.preference_loss(*args, loss="hinge", beta=0.5)[0] == 0.0
    assert abs(O.preference_loss(*args, loss="squared", beta=0.5)[0] - 4.0) < 1e-15
    # equal rewards, and NaN: no pairs
    for rw in ([1.0, 1.0], [float("nan"), 1.0]):
        l, g, _, stats = O.preference_loss([-1.0, -3.0], None, rw, [1, 1], 1, 2, 1)
        assert l == 0.0 and not g.any() and not stats.any()
    # the gradients of a pair cancel where nothing is averaged
    q = _problem(3)
    _, g, _, _ = O.preference_loss(q["logp"], None, q["reward"], np.full(12, 6), 3, 4, 6)
    assert abs(g.reshape(3, 24).sum(1)).max() < 1e-15


def test_preference_terms_without_a_factor_are_left_out():
    for side, h in ((0, -math.inf), (1, math.inf)):
        logp = [-1.0, -1.0]
        logp[side] = -math.inf
        for smoothing in (0.0, 0.25, 1.0):
            l, g, _, _ = O.preference_loss(logp, None, [1.0, 0.0], [1, 1], 1, 2, 1, beta=0.5, smoothing=smoothing)
            # -(1 - smoothing) log sigma(h) - smoothing log sigma(-h), and its slope beta (smoothing - sigma(-h))
            left = (1 - smoothing if h < 0 else smoothing)
            assert l == (math.inf if left else 0.0)
            assert g.tolist() == [0.5 * (smoothing - (h < 0)), -0.5 * (smoothing - (h < 0))]


def test_extreme_pairs_take_the_first_of_equals():
    assert O.prompt_pairs([0.5, 1.0, 0.0, 1.0, 0.0, 0.5], 1, 6, True) == [(1, 2, 1)]
    assert O.prompt_pairs([2.0, 1.0, 1.0, 2.0], 2, 2, True) == [(0, 1, 1), (3, 2, 1)]
    assert O.prompt_pairs([0.0, 1.0, 1.0], 1, 3) == [(1, 0, 2), (2, 0, 2)]


def test_embedding_gradient_is_the_transpose():
    r = np.random.default_rng(1)
    R, T, V, d = 3, 5, 7, 4
    tok, lens = r.integers(-1, V + 1, R * T), np.array([5, 0, 3])
    W, g = r.standard_normal((V, d)), r.standard_normal((R * T, d))
    X = O.embed_fwd(W, tok, lens, R, T, 1.7)
    dW, size = O.embed_bwd(g, tok, lens, R, T, V, 1.7)
    assert abs((X * g).sum() - (W * dW).sum()) < 1e-12
    onehot = np.zeros((R * T, V))
    for i in range(R * T):
        if i % T < lens[i // T] and 0 <= tok[i] < V:
            onehot[i, tok[i]] = 1.7
    assert np.allclose(onehot @ W, X) and np.allclose(onehot.T @ g, dW) and (size >= np.abs(dW) - 1e-15).all()


def test_clip_brings_the_norm_to_the_limit():
    t = [np.array([3.0]), np.zeros(0), np.array([[0.0, 4.0]])]
    n, c, out = O.grad_clip(t, 1.0, 0.0)
    assert n == 5.0 and c == 0.2 and abs(O.grad_norm(out) - 1.0) < 1e-15
    assert O.grad_clip(t, 6.0, 0.0)[1] == 1.0
