"""CPU oracle of the operators around the head in a training step (TEST INFRASTRUCTURE ONLY): preference loss, embedding lookup and its
gradient, gradient norm and clipping.  Plain fp64 NumPy, one formula per step, sharing no code with the HIP path.

The formulas are those stated in ``include/lmhead.h``; the paper does not contain them (parity unpinned).  They are pinned by closed
forms, brute force and finite differences in ``tests/test_oracle_train.py``.
"""
from __future__ import annotations

import math

import numpy as np


def prompt_pairs(reward, P, G, extremes=False):
    """[(preferred, other, pairs of the prompt)] in response indices; a NaN reward is in no pair."""
    rw = np.asarray(reward, dtype=np.float64)
    out = []
    for p in range(P):
        at = [i for i in range(p * G, (p + 1) * G) if rw[i] == rw[i]]
        if extremes:
            mine = []
            if at:
                best, worst = at[0], at[0]
                for i in at[1:]:
                    if rw[i] > rw[best]:
                        best = i
                    if rw[i] < rw[worst]:
                        worst = i
                if rw[best] > rw[worst]:
                    mine = [(best, worst)]
        else:
            mine = [(i, j) for i in at for j in at if rw[i] > rw[j]]
        out += [(i, j, len(mine)) for i, j in mine]
    return out


def preference_loss(logp, logp_ref, reward, lens, P, G, T, loss="logistic", extremes=False, mean=False, per_pair=False, beta=0.1,
                    margin=0.0, margin_scale=0.0, smoothing=0.0, nll_coef=0.0):
    """(loss, g_logp[N], ratio[R], stats[4])."""
    R = P * G
    lp = np.asarray(logp, dtype=np.float64).reshape(R, T)
    lr = None if logp_ref is None else np.asarray(logp_ref, dtype=np.float64).reshape(R, T)
    rw = np.asarray(reward, dtype=np.float64)
    lens = np.clip(np.asarray(lens, dtype=np.int64), 0, T)
    ratio, like = np.zeros(R), np.zeros(R)
    for r in range(R):
        n = int(lens[r])
        if n:
            s = math.fsum(lp[r, :n].tolist()) - (0.0 if lr is None else math.fsum(lr[r, :n].tolist()))
            ratio[r] = s / n if mean else s
            like[r] = math.fsum(lp[r, :n].tolist()) / n
    pairs = prompt_pairs(rw, P, G, extremes)
    M = len(pairs)
    total, c, nll = 0.0, np.zeros(R), np.zeros(R)
    stats = np.zeros(4)
    for a, b, m in pairs:
        w = 1.0 / M if per_pair else 1.0 / (P * m)
        u = ratio[a] - ratio[b]
        h = beta * u - margin - (margin_scale * (rw[a] - rw[b]) if margin_scale else 0.0)
        if loss == "logistic":
            # a term whose factor is 0 is left out, also where it is infinite
            each = ((1 - smoothing) * np.logaddexp(0.0, -h) if smoothing != 1 else 0.0) + (smoothing * np.logaddexp(0.0, h) if smoothing else 0.0)
            slope = beta * (smoothing - 0.5 * (1.0 - math.tanh(0.5 * h)))
        elif loss == "hinge":
            each, slope = max(0.0, 1.0 - h), -beta if h < 1.0 else 0.0
        elif loss == "squared":
            e = h / beta - 1.0 / (2.0 * beta)
            each, slope = e * e, 2.0 * e
        else:
            raise ValueError(loss)
        total += w * (each - (nll_coef * like[a] if nll_coef else 0.0))
        c[a] += w * slope
        c[b] -= w * slope
        nll[a] += w * nll_coef
        stats += np.array([float(u > 0), beta * ratio[a], beta * ratio[b], 0.0]) / M
    stats[3] = M
    g = np.zeros((R, T))
    for r in range(R):
        n = int(lens[r])
        if n:
            g[r, :n] = c[r] / (n if mean else 1) - nll[r] / n
    return total, g.reshape(R * T), ratio, stats


def valid_slots(tok, lens, R, T, V):
    """Slots that count: t < len (clamped) and an id in [0, V)."""
    tok = np.asarray(tok, dtype=np.int64)
    n = np.full(R, T) if lens is None else np.clip(np.asarray(lens, dtype=np.int64), 0, T)
    ok = (np.arange(T)[None, :] < n[:, None]).reshape(R * T)
    return ok & (tok >= 0) & (tok < V)


def embed_fwd(W, tok, lens, R, T, scale=1.0):
    W = np.asarray(W, dtype=np.float64)
    ok = valid_slots(tok, lens, R, T, W.shape[0])
    X = np.zeros((R * T, W.shape[1]))
    X[ok] = scale * W[np.asarray(tok, dtype=np.int64)[ok]]
    return X


def embed_bwd(gX, tok, lens, R, T, V, scale=1.0, base=None):
    """dW, and the sum of absolute values behind each element (the yardstick of a sum's rounding)."""
    gX = np.asarray(gX, dtype=np.float64)
    dW = np.zeros((V, gX.shape[1])) if base is None else np.array(base, dtype=np.float64)
    size = np.abs(dW)
    tok = np.asarray(tok, dtype=np.int64)
    for i in np.nonzero(valid_slots(tok, lens, R, T, V))[0]:
        dW[tok[i]] += scale * gX[i]
        size[tok[i]] += abs(scale) * np.abs(gX[i])
    return dW, size


def grad_norm(tensors):
    return math.sqrt(math.fsum(float(np.square(np.asarray(t, dtype=np.float64)).sum()) for t in tensors))


def grad_clip(tensors, max_norm, eps):
    """(norm, c, clipped tensors)."""
    n = grad_norm(tensors)
    c = min(1.0, max_norm / (n + eps))
    return n, c, [c * np.asarray(t, dtype=np.float64) for t in tensors]
