"""The operators that read a KV cache and make it smaller, as they are measured.

* ``fwd``: attention with a sliding window and a few first tokens that stay visible, over prompts, chunks of prompts and single tokens; with
  ``weight`` the attention weight that each cached token gets is accumulated besides (``attn_fwd``);
* ``train``: the same forward with its backward (``attn_fwd``, ``attn_bwd``);
* ``evict``: the tokens of a cache that got the least weight leave it, per key head, and the others close up (``cache_evict``);
* ``kv4``: a step over a cache held in 4 bits: the new tokens' keys and values are quantised into it, and the new queries attend to it
  (``kv4_store``, ``kv4_attn``).

Where ``own`` is false the operators are computed in their plain form, in elementary torch operations; the references of ``exact`` are
written apart from it, in 64 bits.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False


# ---- the cases -----------------------------------------------------------------------------------------------


def _attn(name, kind, B, Tq, Tk, Hq, Hkv, D, dtype="bf16", window=0, sinks=0, lo=1.0, weight=False, decay=1.0, first="slot"):
    """B sequences of up to Tk keys (lengths lie in [lo * Tk, Tk]) whose last ones, up to Tq, are the queries; first: "slot" where a
    sequence's tokens lie one behind the other with all their heads, "head" where each head's tokens do."""
    c = dict(kind=kind, B=B, Tq=Tq, Tk=Tk, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, window=window, sinks=sinks, lo=lo, weight=weight, decay=decay,
             first=first)
    return dict(c, name=name) if name else c


def _evict(name, B, T, Hkv, D, keep, sinks, recent, dtype="bf16", lo=1.0, first="slot"):
    c = dict(kind="evict", B=B, T=T, Hkv=Hkv, D=D, keep=keep, sinks=sinks, recent=recent, dtype=dtype, lo=lo, first=first)
    return dict(c, name=name) if name else c


def listed():
    return [
        # The 2x4x32 fp32 workload with d = 256 as four heads: unit runs and debugging.
        _attn("fwd-f32-8x32", "fwd", 8, 32, 32, 4, 4, 64, "f32", lo=0.25),
        # Prompts of one sequence length with ragged ends, all keys visible.
        _attn("fwd-8x2048", "fwd", 8, 2048, 2048, 32, 8, 128, lo=0.25),
        # Long responses (the 8x16x8192 workload's) under a window of 1024 and four first tokens.
        _attn("fwd-window-4x8192", "fwd", 4, 8192, 8192, 40, 8, 128, window=1024, sinks=4, lo=0.125),
        # One sequence's decoding step behind a window: latency is all there is.
        _attn("decode-window-1x4096", "fwd", 1, 1, 4096, 32, 8, 128, window=1020, sinks=4, first="head"),
        # A decoding step of 64 sequences over their caches, with the weights that a later eviction goes by.
        _attn("decode-weights-64x8192", "fwd", 64, 1, 8192, 32, 8, 128, lo=0.25, weight=True, decay=0.99, first="head"),
        # The 2x4x32 workload's training pair.
        _attn("train-f32-8x32", "train", 8, 32, 32, 4, 4, 64, "f32", lo=0.25),
        # A micro-batch of the 16x16x4096 workload (28 heads of 128 make d = 3584) under a window.
        _attn("train-8x4096", "train", 8, 4096, 4096, 28, 4, 128, window=1024, sinks=4, lo=0.25),
        # A full cache of two sequences gives up its lightest eighth.
        _evict("evict-2x1024", 2, 1024, 8, 128, 896, 4, 128, first="head"),
        # 32 caches of up to 8192 tokens shrink to half of that.
        _evict("evict-32x8192", 32, 8192, 8, 128, 4096, 4, 512, lo=0.5),
        # One sequence's decoding step over a 4-bit cache.
        _attn("kv4-1x4096", "kv4", 1, 1, 4096, 32, 8, 128),
        # Eight drafted tokens are checked at once over one long context.
        _attn("kv4-draft-1x131072", "kv4", 1, 8, 131072, 32, 8, 128),
        # A decoding step of 64 sequences, odd lengths.
        _attn("kv4-64x16001", "kv4", 64, 1, 16001, 32, 8, 128, lo=0.25),
    ]


def _log_int(rng: random.Random, lo: float, hi: float) -> int:
    return max(int(lo), min(int(hi), int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


_HEADS = [(4, 4, 64), (8, 2, 64), (32, 8, 128), (28, 4, 128), (40, 8, 128), (16, 16, 128), (12, 12, 64), (6, 3, 32), (8, 1, 96), (20, 4, 80)]


def draw(rng: random.Random):
    top = {kind: work(c) for kind, c in (("train", listed()[6]), ("kv4", listed()[11]), ("evict", listed()[8]))}
    while True:
        c = _draw(rng)
        w = work(c)
        if w["flops"] <= top["train"]["flops"] and w["bytes"] <= max(t["bytes"] for t in top.values()):
            return c


def _draw(rng):
    kind = rng.choice(["fwd", "fwd", "decode", "decode", "train", "train", "evict", "kv4", "kv4"])
    Hq, Hkv, D = rng.choice(_HEADS)
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    lo, first = rng.choice([1 / 64, 0.25, 0.5, 1.0]), rng.choice(["slot", "head"])
    B = _log_int(rng, 1, 64)
    if kind == "evict":
        T = _log_int(rng, 16, 16384)
        keep = rng.randint(max(2, T // 8), T)
        recent = rng.randint(0, keep // 2)
        return _evict(None, B, T, Hkv, D, keep, min(rng.choice([0, 1, 4]), keep - recent), recent, dtype, lo, first)
    window = rng.choice([0, 0, 1, 100, 128, 1000, 1024, 4096])
    sinks = rng.choice([0, 1, 4, 64]) if window else 0
    if kind == "train":
        T = _log_int(rng, 1, 4096)
        return _attn(None, kind, min(B, 16), T, T, Hq, Hkv, D, dtype, window, sinks, lo, first=first)
    weight, decay = rng.random() < 0.4, rng.choice([1.0, 0.99, 0.0])
    if kind == "fwd":
        Tk = _log_int(rng, 1, 8192)
        Tq = Tk if rng.random() < 0.6 else _log_int(rng, 1, Tk)
        return _attn(None, kind, min(B, 16), Tq, Tk, Hq, Hkv, D, dtype, window, sinks, lo, weight, decay, first)
    Tk = _log_int(rng, 16, 131072)
    Tq = min(Tk, rng.choice([1, 1, 1, 2, 5, 8]))
    if kind == "kv4":
        Hq, Hkv, D = rng.choice([h for h in _HEADS if h[2] % 32 == 0])
        return _attn(None, kind, B, Tq, Tk, Hq, Hkv, D, dtype, window, sinks, lo, weight, decay)
    return _attn(None, "fwd", B, Tq, Tk, Hq, Hkv, D, dtype, window, sinks, lo, weight, decay, first)


# ---- inputs --------------------------------------------------------------------------------------------------


_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape, std=1.0, dtype=torch.float32):
    """N(0, std^2) drawn in float32 and rounded to the storage type, a sequence at a time."""
    out = torch.empty(*shape, dtype=dtype, device="cuda")
    for part in out:
        part.copy_(torch.randn(part.shape, generator=g, device="cuda").mul_(std))
    return out


def _rows(g, case, T, H, std=1.0):
    """[B, T, H, D] in the order in memory that the case asks for."""
    B, D, t = case["B"], case["D"], _TYPES[case["dtype"]]
    if case["first"] == "head":
        return _normal(g, B, H, T, D, std=std, dtype=t).transpose(1, 2)
    return _normal(g, B, T, H, D, std=std, dtype=t)


def _channels(g, x):
    """Keys of language models have a few channels that are much larger than the others: one in sixteen here, by four."""
    big = 1.0 + 3.0 * (torch.rand(x.shape[2:], generator=g, device="cuda") < 1 / 16)
    for part in x:
        part.mul_(big.to(x.dtype))
    return x


def _lengths(case, rng):
    """(queries, keys) of each sequence."""
    T = case.get("Tk", case.get("T"))
    lk = [rng.randint(max(1, int(case["lo"] * T)), T) for _ in range(case["B"])]
    if "Tq" not in case:
        return lk, lk
    lq = [max(1, min(case["Tq"], n if case["Tq"] == T else round(case["Tq"] * n / T))) for n in lk]
    return lq, lk


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g, rng = _gen(seed), random.Random(seed)
    s = dict(case=case)
    lq, lk = s["lengths"] = _lengths(case, rng)
    f32 = dict(dtype=torch.float32, device="cuda")
    B, Hkv, D = case["B"], case["Hkv"], case["D"]
    if case["kind"] == "evict":
        T = case["T"]
        s["lens"] = _int32(lk)
        s["k"], s["v"] = _channels(g, _rows(g, case, T, Hkv)), _rows(g, case, T, Hkv)
        # accumulated weights: most tokens got little, a few a lot; half of the sequences hold them in steps of 1/64, with ties
        s["weight"] = torch.rand(B, Hkv, T, generator=g, **f32).pow_(8).mul_(30.0)
        s["weight"][::2] = (s["weight"][::2] * 64).round_() / 64
        if own:
            import paper_2603_04411_amd as L
            s["desc"] = L.make_evict_desc(B, T, Hkv, case["keep"], sinks=case["sinks"], recent=case["recent"])
            s["planes"] = L.make_cache_planes([s["k"], s["v"]])
            s["lens_out"] = torch.empty(B, dtype=torch.int32, device="cuda")
            s["kept"] = torch.empty(B, Hkv, case["keep"], dtype=torch.int32, device="cuda")
            s["ws"] = torch.empty(L.evict_workspace_bytes(s["desc"]), dtype=torch.uint8, device="cuda")
        return s
    Tq, Tk, Hq = case["Tq"], case["Tk"], case["Hq"]
    s["len_q"], s["len_k"] = _int32(lq), _int32(lk)
    # logits of a standard deviation around 1.5
    s["q"] = _rows(g, case, Tq, Hq, std=1.2)
    s["weight"] = torch.rand(B, Hkv, Tk, generator=g, **f32) if case["weight"] else None
    if case["kind"] == "kv4":
        s["k"], s["v"] = _channels(g, _rows(g, case, Tq, Hkv)), _rows(g, case, Tq, Hkv)        # of the new tokens
        cache = []
        for x in ("k", "v"):
            codes = torch.randint(0, 256, (B, Hkv, Tk, D // 2), generator=g, dtype=torch.uint8, device="cuda")
            scales = torch.randint(124, 128, (B, Hkv, Tk, D // 32), generator=g, dtype=torch.uint8, device="cuda")
            cache += [codes, scales]
        s["cache"] = cache
    else:
        s["k"], s["v"] = _channels(g, _rows(g, case, Tk, Hkv)), _rows(g, case, Tk, Hkv)
    if case["kind"] == "train":
        s["g_out"] = _rows(g, case, Tq, Hq, std=1.0 / math.sqrt(B * Tq))
    if own:
        import paper_2603_04411_amd as L
        s["out"] = torch.empty_like(s["q"])
        s["desc"] = L.make_attn_desc(B, Tq, Tk, Hq, Hkv, D, case["dtype"], window=case["window"], sinks=case["sinks"],
                                     q=L.attn_layout(s["q"]), k=L.attn_layout(s["k"]), v=L.attn_layout(s["v"]), o=L.attn_layout(s["out"]))
        s["lse"] = torch.empty(B, Hq, Tq, **f32)
        s["ws"] = torch.empty(L.attn_workspace_bytes(s["desc"]), dtype=torch.uint8, device="cuda")
        if case["kind"] == "train":
            s["dq"], s["dk"], s["dv"] = (torch.empty_like(s[x]) for x in "qkv")
            s["ws_bwd"] = torch.empty(L.attn_bwd_workspace_bytes(s["desc"]), dtype=torch.uint8, device="cuda")
    return s


# ---- one pass ------------------------------------------------------------------------------------------------


def run(s):
    return {"fwd": _run_fwd, "train": _run_train, "evict": _run_evict, "kv4": _run_kv4}[s["case"]["kind"]](s, s["case"])


def _run_fwd(s, case):
    if own:
        import paper_2603_04411_amd as L
        L.attn_fwd(s["desc"], s["q"], s["k"], s["v"], s["len_q"], s["len_k"], s["out"], s["lse"], s["weight"], case["decay"], s["ws"])
        return _with_weight(dict(out=s["out"], lse=s["lse"]), s)
    out, lse, _ = _plain(s, case, lambda b: (s["k"][b], s["v"][b]))
    return _with_weight(dict(out=out, lse=lse), s)


def _with_weight(r, s):
    if s["weight"] is not None:
        r["weight"] = s["weight"]
    return r


def _run_train(s, case):
    if own:
        import paper_2603_04411_amd as L
        L.attn_fwd(s["desc"], s["q"], s["k"], s["v"], s["len_q"], s["len_k"], s["out"], s["lse"], None, 0.0, s["ws"])
        L.attn_bwd(s["desc"], s["q"], s["k"], s["v"], s["len_q"], s["len_k"], s["out"], s["lse"], s["g_out"], s["dq"], s["dk"], s["dv"],
                   s["ws_bwd"])
        return dict(out=s["out"], lse=s["lse"], dq=s["dq"], dk=s["dk"], dv=s["dv"])
    out, lse, grads = _plain(s, case, lambda b: (s["k"][b], s["v"][b]))
    return dict(out=out, lse=lse, **grads)


def _run_kv4(s, case):
    if own:
        import paper_2603_04411_amd as L
        L.kv4_store(s["desc"], s["k"], s["v"], s["len_q"], s["len_k"], *s["cache"], s["ws"])
        L.kv4_attn(s["desc"], s["q"], *s["cache"], s["len_q"], s["len_k"], s["out"], s["lse"], s["weight"], case["decay"], s["ws"])
        return _with_weight(dict(out=s["out"], lse=s["lse"]), s)
    lq, lk = s["lengths"]
    for x, codes, scales in (("k", *s["cache"][:2]), ("v", *s["cache"][2:])):
        c, e = _quantise(s[x].transpose(1, 2).float())                 # [B, Hkv, Tq, .]
        for b in range(case["B"]):
            codes[b, :, lk[b] - lq[b]:lk[b]], scales[b, :, lk[b] - lq[b]:lk[b]] = c[b, :, :lq[b]], e[b, :, :lq[b]]
    out, lse, _ = _plain(s, case, lambda b: tuple(_values(s["cache"][i][b, :, :lk[b]], s["cache"][i + 1][b, :, :lk[b]]).transpose(0, 1)
                                                  for i in (0, 2)))
    return _with_weight(dict(out=out, lse=lse), s)


_STEPS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _quantise(x):
    """Codes (two to a byte, the first in the lower half) and scale bytes of the blocks of 32 along the last axis of float32 x."""
    x = x.reshape(*x.shape[:-1], -1, 32)
    top = x.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top)                                    # top = m 2^e, m in [0.5, 1)
    e = torch.where(m > 0.75, e - 2, e - 3)                    # the smallest e with top <= 6 2^e
    e = torch.where(top > 0, e, torch.full_like(e, -126)).clamp(min=-126)
    y = torch.ldexp(x, -e).abs()
    # half steps: up where the value above has the even code
    code = torch.zeros_like(y, dtype=torch.int32)
    for i in range(1, 8):
        half = 0.5 * (_STEPS[i - 1] + _STEPS[i])
        code += (y >= half) if i % 2 == 0 else (y > half)
    code = code | (torch.signbit(x).int() << 3)
    bad = ~torch.isfinite(top)
    scale = torch.where(bad, torch.full_like(e, 255), e + 127)[..., 0]
    code = code.masked_fill(bad, 0).flatten(-2)
    return (code[..., 0::2] | (code[..., 1::2] << 4)).to(torch.uint8), scale.to(torch.uint8)


def _values(codes, scales):
    steps = torch.tensor(_STEPS + [-v for v in _STEPS], device="cuda")
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    size = torch.ldexp(torch.ones((), device="cuda"), scales.int() - 127).masked_fill(scales == 255, float("nan"))
    return steps[c.int()] * size.repeat_interleave(32, -1)


def _plain(s, case, cached):
    """Output, lse and, where there is a gradient of the output, the gradients: sequence by sequence, in blocks of queries over the keys that
    a block can see."""
    B, Tq, Tk, Hq, Hkv, D = (case[x] for x in ("B", "Tq", "Tk", "Hq", "Hkv", "D"))
    G, t, scale, window, sinks = Hq // Hkv, _TYPES[case["dtype"]], 1.0 / math.sqrt(D), case["window"], case["sinks"]
    lengths_q, lengths_k = s["lengths"]
    out = torch.zeros(B, Tq, Hq, D, dtype=t, device="cuda")
    lse = torch.full((B, Hq, Tq), -math.inf, device="cuda")
    grads = {}
    if case["kind"] == "train":
        grads = dict(dq=torch.zeros_like(s["q"]), dk=torch.zeros_like(s["k"]), dv=torch.zeros_like(s["v"]))
    for b in range(B):
        lq, lk = lengths_q[b], lengths_k[b]
        k, v = (x[:lk].float().transpose(0, 1) for x in cached(b))               # [Hkv, lk, D]
        if s["weight"] is not None:
            if case["decay"] == 0.0:
                s["weight"][b, :, :lk] = 0.0
            else:
                s["weight"][b, :, :lk] *= case["decay"]
        if grads:
            dk, dv = torch.zeros_like(k), torch.zeros_like(v)
        for i0 in range(0, lq, 512):
            n = min(512, lq - i0)
            p0 = lk - lq + i0                                                     # key position of the block's first query
            a = max(0, p0 - window + 1) if window else 0
            at = torch.arange(a, p0 + n, device="cuda")
            if a:
                at = torch.cat([torch.arange(min(sinks, a), device="cuda"), at])
            p = torch.arange(p0, p0 + n, device="cuda")
            see = at[None, :] <= p[:, None]
            if window:
                see &= (at[None, :] > p[:, None] - window) | (at[None, :] < sinks)
            see = see.repeat(G, 1)                                                # rows of one key head: [G * n, keys]
            heads = lambda x: x[b, i0:i0 + n].float().reshape(n, Hkv, G, D).permute(1, 2, 0, 3).reshape(Hkv, G * n, D)
            back = lambda x: x.reshape(Hkv, G, n, D).permute(2, 0, 1, 3).reshape(n, Hq, D)
            q, kb, vb = heads(s["q"]), k[:, at], v[:, at]
            z = torch.matmul(q, kb.transpose(1, 2)).mul_(scale).masked_fill_(~see, -math.inf)
            m = z.amax(-1, keepdim=True)
            w = z.sub_(m).exp_()
            total = w.sum(-1, keepdim=True)
            w = w.div_(total)
            o = torch.matmul(w, vb)
            out[b, i0:i0 + n] = back(o).to(t)
            lse[b, :, i0:i0 + n] = (m + total.log())[..., 0].reshape(Hq, n)
            if s["weight"] is not None:
                s["weight"][b].index_add_(1, at, w.sum(1))
            if grads:
                g = heads(s["g_out"])
                dv.index_add_(1, at, torch.matmul(w.transpose(1, 2), g))
                dz = torch.matmul(g, vb.transpose(1, 2))
                dz = dz.sub_((g * o).sum(-1, keepdim=True)).mul_(w).mul_(scale)
                grads["dq"][b, i0:i0 + n] = back(torch.matmul(dz, kb)).to(t)
                dk.index_add_(1, at, torch.matmul(dz.transpose(1, 2), q))
        if grads:
            grads["dk"][b, :lk], grads["dv"][b, :lk] = dk.transpose(0, 1).to(t), dv.transpose(0, 1).to(t)
    return out, lse, grads


def _run_evict(s, case):
    if own:
        import paper_2603_04411_amd as L
        L.cache_evict(s["desc"], s["planes"], s["weight"], s["lens"], s["lens_out"], s["kept"], s["ws"])
        return dict(k=s["k"], v=s["v"], weight=s["weight"], lens=s["lens_out"], kept=s["kept"])
    B, T, Hkv, keep = case["B"], case["T"], case["Hkv"], case["keep"]
    at = torch.arange(T, device="cuda")
    lens = s["lens"].long()[:, None, None]
    rank = s["weight"].masked_fill((at < case["sinks"]) | (at >= lens - case["recent"]), math.inf).masked_fill(at >= lens, -math.inf)
    order = rank.sort(dim=-1, descending=True, stable=True).indices[..., :keep]
    full = (lens > keep).expand(B, Hkv, 1)
    kept = torch.where(full, order.sort(-1).values, torch.where(at[:keep] < lens, at[:keep], -1))
    from_ = torch.where(full, kept, at[:keep])
    for x in (s["k"], s["v"]):
        rows = x.transpose(1, 2)
        rows[:, :, :keep] = rows.gather(2, from_[..., None].expand(B, Hkv, keep, case["D"]))
    left = s["weight"].gather(2, from_)
    s["weight"].masked_fill_(full & (at >= keep) & (at < lens), 0.0)
    s["weight"][..., :keep] = left
    return dict(k=s["k"], v=s["v"], weight=s["weight"], lens=s["lens"].clamp(max=keep), kept=kept.int())


# ---- what a pass cannot do without ---------------------------------------------------------------------------


def _shares(case):
    """(queries, keys) of sequences spread evenly over the range of lengths."""
    T = case.get("Tk", case.get("T"))
    lo = max(1, int(case["lo"] * T))
    n = np.linspace(lo, T, 33)
    return n if "Tq" not in case or case["Tq"] == T else np.maximum(1.0, case["Tq"] * n / T), n


def work(case):
    esz = {"bf16": 2, "f32": 4}[case["dtype"]]
    B, Hkv, D = case["B"], case["Hkv"], case["D"]
    lq, lk = _shares(case)
    if case["kind"] == "evict":
        goes = float(np.mean(lk > case["keep"]))
        n, keep = float(lk.mean()), case["keep"]
        # the weights and their successors, the kept tokens' numbers; rows behind the first one that goes are moved, nearly all
        return dict(bytes=B * Hkv * (4.0 * n + 4.0 * keep + goes * (4.0 * n + 4.0 * keep * D * esz)), flops=B * Hkv * n)
    Hq, w, sinks = case["Hq"], case["window"], case["sinks"]

    def pairs(lq, lk):
        p = np.arange(lk - lq, lk) if lq < 4096 else np.linspace(lk - lq, lk - 1, 4096)
        seen = np.minimum(p + 1, w + np.minimum(sinks, np.maximum(p + 1 - w, 0))) if w else p + 1
        return float(np.maximum(seen, 1).mean() * lq)

    see = float(np.mean([pairs(int(a), int(n)) for a, n in zip(lq, lk)]))
    keys = float(np.mean(np.minimum(lk, (w + lq - 1 + sinks) if w else lk)))
    rows = float(lq.mean())
    flops = 4.0 * B * Hq * D * see
    row = D * esz
    if case["kind"] == "kv4":
        read = keys * Hkv * 2 * (D // 2 + D // 32) + rows * Hkv * 2 * (row + D // 2 + D // 32)
    else:
        read = keys * Hkv * 2 * row
    some = B * (read + rows * Hq * (2 * row + 4))
    if case["weight"]:
        some += B * Hkv * float(lk.mean()) * (4 if case["decay"] == 0.0 else 8)
    if case["kind"] == "train":
        # q, k, v, out and its gradient in, three gradients out
        return dict(bytes=some + B * rows * Hq * 2 * row + B * (2 * rows * Hq + 4 * keys * Hkv) * row, flops=3.5 * flops)
    return dict(bytes=some, flops=flops)


# ---- the definitions, in 64 bits -----------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "evict":
        return _exact_evict(s, case)
    return _exact_attn(s, case)


_E2M1 = np.array([(-1) ** (c >> 3) * ((c & 1) * 0.5 if c & 7 < 2 else (1 + (c & 1) / 2) * 2.0 ** (((c >> 1) & 3) - 1)) for c in range(16)])
_GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def _exact_values(codes, scales):
    table = torch.from_numpy(_E2M1).cuda()
    low, high = table[(codes % 16).long()], table[(codes // 16).long()]
    both = torch.stack([low, high], dim=-1).reshape(*codes.shape[:-1], -1)
    return both * torch.exp2(scales.double() - 127).repeat_interleave(32, dim=-1)


def _exact_new(x):
    """What the rows x stand for once they are held in 4 bits: for each value the nearest of the grid, of two the one with the even code."""
    a = x.double().cpu().numpy().reshape(-1, 32)
    top = np.abs(a).max(1)
    with np.errstate(divide="ignore"):
        e = np.where(top > 0, np.ceil(np.log2(np.maximum(top, 1e-300) / 6.0)), -126.0)
    e += top > 6 * 2.0 ** e                                    # where the logarithm was rounded
    e -= (top > 0) & (top <= 6 * 2.0 ** (e - 1))
    size = 2.0 ** np.maximum(e, -126.0)[:, None]
    y = np.abs(a) / size
    off = np.abs(y[..., None] - _GRID)
    near = off.min(-1, keepdims=True)
    at = np.where((off == near) & (np.arange(8) % 2 == 0), np.arange(8), -1).max(-1)
    at = np.where(at < 0, off.argmin(-1), at)
    return torch.from_numpy((np.sign(a) * _GRID[at] * size).reshape(x.shape)).cuda()


def _exact_attn(s, case):
    B, Tq, Hq, Hkv, D = (case[x] for x in ("B", "Tq", "Hq", "Hkv", "D"))
    G = Hq // Hkv
    f64 = dict(dtype=torch.float64, device="cuda")
    out, lse = torch.zeros(B, Tq, Hq, D, **f64), torch.full((B, Hq, Tq), -math.inf, **f64)
    train = case["kind"] == "train"
    if train:
        dq, dk, dv = (torch.zeros(s[x].shape, **f64) for x in "qkv")
    weight = s["weight"].double() if s["weight"] is not None else None
    for b, (lq, lk) in enumerate(zip(*s["lengths"])):
        gap = torch.arange(lk - lq, lk, device="cuda")[:, None] - torch.arange(lk, device="cuda")[None, :]    # how far a key lies back
        hidden = gap < 0
        if case["window"]:
            hidden = hidden | ((gap >= case["window"]) & (torch.arange(lk, device="cuda")[None, :] >= case["sinks"]))
        for h in range(Hkv):
            if case["kind"] == "kv4":
                k, v = (torch.cat([_exact_values(s["cache"][i][b, h, :lk - lq], s["cache"][i + 1][b, h, :lk - lq]), _exact_new(s[x][b, :lq, h])])
                        for i, x in ((0, "k"), (2, "v")))
            else:
                k, v = s["k"][b, :lk, h].double().requires_grad_(train), s["v"][b, :lk, h].double().requires_grad_(train)
            for j in range(h * G, (h + 1) * G):
                q = s["q"][b, :lq, j].double().requires_grad_(train)
                z = (q @ k.T / math.sqrt(D)).masked_fill(hidden, -math.inf)
                total = torch.logsumexp(z, 1)
                w = torch.exp(z - total[:, None])
                o = w @ v
                if train:
                    o.backward(s["g_out"][b, :lq, j].double())
                    dq[b, :lq, j] = q.grad
                out[b, :lq, j], lse[b, j, :lq] = o.detach(), total.detach()
                if weight is not None:
                    if j == h * G:
                        weight[b, h, :lk] *= case["decay"]
                    weight[b, h, :lk] += w.sum(0)
            if train:
                dk[b, :lk, h], dv[b, :lk, h] = k.grad, v.grad
    r = dict(out=out, lse=lse)
    if train:
        r.update(dq=dq, dk=dk, dv=dv)
    if weight is not None:
        r["weight"] = weight
    return r


def _exact_evict(s, case):
    """Head by head, on the host."""
    B, T, Hkv, keep, sinks, recent = (case[x] for x in ("B", "T", "Hkv", "keep", "sinks", "recent"))
    weight = s["weight"].cpu().numpy().astype(np.float64)
    k, v = s["k"].double(), s["v"].double()
    kept = np.full((B, Hkv, keep), -1, dtype=np.int64)
    lens = np.array(s["lengths"][1])
    for b, n in enumerate(lens):
        if n <= keep:
            kept[b, :, :n] = np.arange(n)
            continue
        for h in range(Hkv):
            inner = np.arange(sinks, n - recent)
            best = inner[np.lexsort((inner, -weight[b, h, inner]))][:keep - sinks - recent]
            kept[b, h] = np.sort(np.concatenate([np.arange(sinks), best, np.arange(n - recent, n)]))
            left = weight[b, h, kept[b, h]].copy()
            weight[b, h, keep:n] = 0.0
            weight[b, h, :keep] = left
            at = torch.from_numpy(kept[b, h]).cuda()
            for x in (k, v):
                x[b, :keep, h] = x[b, at, h].clone()
    return dict(k=k, v=v, weight=weight, lens=np.minimum(lens, keep), kept=kept)
