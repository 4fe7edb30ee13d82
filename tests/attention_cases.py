"""Inputs of the attention tests, the bounds that their results have to keep, and the bounds' derivation.

With u the half step of the storage type (bf16 2^-8, fp32 2^-24) and w = 2^-24:
 logits    an fp32 sum of D products, each rounded, then a product with the scale: |dz| <= (D + 4) w |scale| sum |q||k|, at most Z in a row
 P         exp2 of the logit less the maximum (an argument of up to A = 2 max|z| log2(e), rounded: A w), a unit of exp2, and its sum over lk
           keys: relative r = 2 Z + (lk + 2 A + 16) w
 out       P rounded to the storage type, products, sums and the output's rounding: u (sum P|v| + |out|) + (r + (lk + 4) w) sum P|v|
 lse       Z + (lk + A + 16) w + 4 w |lse|
 weight    (r + (rows + 4) w) weight + 4 w |result|
 backward  P from the given lse: r' = r + error of lse (the bound above);  dP and delta: e = (D + 4) w (sum |g||v| and sum |g||out|);
           dS: (u + r') |dS| + P e;  dq: scale (sum err(dS) |k| + (lk + 4) w sum |dS||k|) + u |dq|;  dk, dv alike over rows.
           bf16: delta is <g, out> less F = sum dS, which takes the rounding of out away but leaves what F is off by,
           f = sum (r' |dS| + P e) + (lk + 4) w sum |dS|, and u |F| <= u^2 sum |g||out| where F meets rounded P: both times sum P|k| in dq;
           f alone, times P |q|, in dk.  fp32: the rounding of out, w sum |g||out|, is within e
Second orders: every bound times 1.1, and 2^-126 times what a product's second factor can be for subnormal P (they may be flushed).
"""
from __future__ import annotations

import numpy as np

from oracle import attention_oracle as A

W = 2.0 ** -24
TINY = 2.0 ** -100
U = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def bounds(q, k, v, len_q, len_k, scale, window, sinks, dtype, out=None, g=None):
    """Exact results and their bounds; with g the gradients' too (out: the rounded output that the backward was handed)."""
    B, Tq, Hq, D = q.shape
    Tk, Hkv = k.shape[1:3]
    G, u = Hq // Hkv, U[dtype]
    r = dict(out=np.zeros(q.shape), lse=np.full((B, Hq, Tq), -np.inf), weight=np.zeros((B, Hkv, Tk)))
    e = dict(out=np.zeros(q.shape), lse=np.zeros((B, Hq, Tq)), weight=np.zeros((B, Hkv, Tk)))
    if g is not None:
        for n, x in (("dq", q), ("dk", k), ("dv", v)):
            r[n], e[n] = np.zeros(x.shape), np.zeros(x.shape)
    for b in range(B):
        lq, lk = int(len_q[b]), int(len_k[b])
        if lq == 0 or lk == 0:
            continue
        see = A.visible(lq, lk, window, sinks)
        for h, hk in A.heads(Hq, Hkv):
            Q, K, V = q[b, :lq, h], k[b, :lk, hk], v[b, :lk, hk]
            P, lse, z = A.probabilities(Q, K, scale, see)
            Z = np.where(see, (D + 4) * W * scale * (np.abs(Q) @ np.abs(K).T), 0.0).max(1)
            arg = 2 * np.where(see, np.abs(z), 0.0).max(1) * 1.4427
            rel = 2 * Z + (lk + 2 * arg + 16) * W
            o, s = P @ V, P @ np.abs(V)
            r["out"][b, :lq, h], r["lse"][b, h, :lq] = o, lse
            e["out"][b, :lq, h] = u * (s + np.abs(o)) + (rel + (lk + 4) * W)[:, None] * s
            seen = np.isfinite(lse)
            e_lse = np.where(seen, Z + (lk + arg + 16) * W + 4 * W * np.abs(np.where(seen, lse, 0.0)), 0.0)
            e["lse"][b, h, :lq] = e_lse
            r["weight"][b, hk, :lk] += P.sum(0)
            e["weight"][b, hk, :lk] += P.T @ (rel + (lq * G + 4) * W)
            if g is None:
                continue
            go = g[b, :lq, h]
            oo = out[b, :lq, h]
            dP, delta = go @ V.T, (go * o).sum(1)
            dS = P * (dP - delta[:, None])
            rel2 = (rel + e_lse)[:, None]
            err = (D + 4) * W * (np.abs(go) @ np.abs(V).T + (np.abs(go) * np.abs(oo)).sum(1)[:, None])
            go_oo = (np.abs(go) * np.abs(oo)).sum(1)
            e_S = (u + rel2) * np.abs(dS) + (1 + rel2) * P * err
            f = np.zeros(lq)
            if dtype == "bf16":
                f = (rel2 * np.abs(dS) + (1 + rel2) * P * err).sum(1) + (lk + 4) * W * (np.abs(dS) + P * u * go_oo[:, None]).sum(1)
                e_S = e_S + P * f[:, None]
            r["dq"][b, :lq, h] = scale * dS @ K
            if dtype == "bf16":
                e["dq"][b, :lq, h] += scale * (u * u * go_oo)[:, None] * (P @ np.abs(K))
            e["dq"][b, :lq, h] += scale * (e_S + (lk + 4) * W * np.abs(dS)) @ np.abs(K) + u * np.abs(r["dq"][b, :lq, h])
            r["dk"][b, :lk, hk] += scale * dS.T @ Q
            e["dk"][b, :lk, hk] += scale * (e_S + (lq * G + 4) * W * np.abs(dS)).T @ np.abs(Q)
            r["dv"][b, :lk, hk] += P.T @ go
            e["dv"][b, :lk, hk] += ((u + rel2 + (lq * G + 4) * W) * P).T @ np.abs(go)
    if g is not None:
        for n in ("dk", "dv"):
            e[n] += u * np.abs(r[n])
    return r, {n: 1.1 * x + TINY for n, x in e.items()}


def holds(got, want, bound, name):
    got = np.asarray(got, dtype=np.float64)
    nan = np.isnan(got) | np.isnan(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{name}: NaN in {int(np.isnan(got).sum())} places, {int(np.isnan(want).sum())} expected"
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]) and not np.isinf(got[~inf]).any(), f"{name}: infinities differ"
    off = np.abs(np.where(inf | nan, 0.0, got) - np.where(inf | nan, 0.0, want))
    over = off - bound
    at = np.unravel_index(np.argmax(np.where(nan, -1.0, over)), over.shape) if over.size else ()
    assert not over.size or over[at] <= 0, f"{name}{tuple(int(i) for i in at)}: {got[at]} vs {want[at]}, {off[at]:.3g} off, bound {bound[at]:.3g}"
