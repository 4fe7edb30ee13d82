"""fp64 NumPy oracle of the operators that read a KV cache and make it smaller (``include/dynakv.h``): one formula per step, test
infrastructure only.  Tensors are [sequence, slot, head, channel]."""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def visible(lq, lk, window, sinks):
    """[lq, lk]: whether query i sees key j."""
    p = np.arange(lk - lq, lk)[:, None]
    j = np.arange(lk)[None, :]
    see = j <= p
    if window:
        see &= (j > p - window) | (j < sinks)
    return see


def probabilities(q, k, scale, see):
    """(P, lse, logits) of one head: q [lq, D], k [lk, D].  A query that sees nothing has P = 0 and lse = -inf."""
    z = scale * (q @ k.T)
    zm = np.where(see, z, -np.inf)
    top = zm.max(1, initial=-np.inf)
    base = np.where(np.isfinite(top), top, 0.0)
    e = np.where(see, np.exp(np.where(see, z, 0.0) - base[:, None]), 0.0)
    total = e.sum(1)
    with np.errstate(divide="ignore", invalid="ignore"):
        P = np.where(total[:, None] > 0, e / total[:, None], 0.0)
        lse = np.where(total > 0, base + np.log(total), -np.inf)
    return P, lse, z


def heads(Hq, Hkv):
    return [(h, h // (Hq // Hkv)) for h in range(Hq)]


def attn_fwd(q, k, v, len_q, len_k, scale, window=0, sinks=0):
    """(out [B, Tq, Hq, D], lse [B, Hq, Tq], weight [B, Hkv, Tk])."""
    B, Tq, Hq, D = q.shape
    Tk, Hkv = k.shape[1:3]
    out, lse, weight = np.zeros(q.shape), np.full((B, Hq, Tq), -np.inf), np.zeros((B, Hkv, Tk))
    for b in range(B):
        lq, lk = int(len_q[b]), int(len_k[b])
        see = visible(lq, lk, window, sinks)
        for h, hk in heads(Hq, Hkv):
            P, l, _ = probabilities(q[b, :lq, h], k[b, :lk, hk], scale, see)
            out[b, :lq, h] = P @ v[b, :lk, hk]
            lse[b, h, :lq] = l
            weight[b, hk, :lk] += P.sum(0)
    return out, lse, weight


def attn_bwd(q, k, v, len_q, len_k, out, g, scale, window=0, sinks=0):
    """(dq, dk, dv) given g = dL/dout; delta is taken from `out` as it is handed in."""
    B, Tq, Hq, D = q.shape
    Hkv = k.shape[2]
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for b in range(B):
        lq, lk = int(len_q[b]), int(len_k[b])
        see = visible(lq, lk, window, sinks)
        for h, hk in heads(Hq, Hkv):
            P, _, _ = probabilities(q[b, :lq, h], k[b, :lk, hk], scale, see)
            go = g[b, :lq, h]
            dP = go @ v[b, :lk, hk].T
            dS = P * (dP - (go * out[b, :lq, h]).sum(1)[:, None])
            dq[b, :lq, h] = scale * dS @ k[b, :lk, hk]
            dk[b, :lk, hk] += scale * dS.T @ q[b, :lq, h]
            dv[b, :lk, hk] += P.T @ go
    return dq, dk, dv


def quantise4(x):
    """(codes [.., D / 2], scale bytes [.., D / 32]) of rows x [.., D]."""
    y = np.asarray(x, dtype=np.float64).reshape(*x.shape[:-1], -1, 32)
    fine = np.isfinite(y).all(-1)
    y = np.where(fine[..., None], y, 0.0)
    top = np.abs(y).max(-1)
    e = np.full(top.shape, -126)
    for c in range(-126, 125):                       # the smallest e with top <= 6 2^e, at most 125
        e = np.where(top > 6.0 * 2.0 ** c, c + 1, e)
    r = np.abs(y) / 2.0 ** e.astype(np.float64)[..., None]
    off = np.abs(r[..., None] - GRID)
    best = off.min(-1, keepdims=True)
    index = np.where((off == best), np.arange(8) % 2 * 8 + np.arange(8), 99).argmin(-1)   # of two as near ones the even index
    code = np.where(fine[..., None], index + 8 * np.signbit(y), 0).astype(np.uint8).reshape(*x.shape[:-1], -1)
    return code[..., 0::2] | code[..., 1::2] << 4, np.where(fine, e + 127, 255).astype(np.uint8)


def values4(codes, scales):
    c = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)
    v = np.where(c & 8, -1.0, 1.0) * GRID[c & 7]
    size = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(size, 32, -1)


def evict(weight, length, keep, sinks, recent):
    """The slots that one key head keeps of `length`, ascending."""
    if length <= keep:
        return list(range(length))
    inner = range(sinks, length - recent)
    order = sorted(inner, key=lambda i: (-weight[i] if weight[i] == weight[i] else np.inf, i))
    nan = [i for i in order if weight[i] != weight[i]]
    order = [i for i in order if weight[i] == weight[i]] + nan
    return sorted(list(range(sinks)) + order[:keep - sinks - recent] + list(range(length - recent, length)))
