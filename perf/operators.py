"""The operators of a training step around the LM head, as they are measured.

* ``preference``: a preference loss over the pairs of each prompt's responses, from token log-probabilities, with its
  gradient (``preference_loss``);
* ``embed_fwd`` / ``embed_bwd``: rows of a weight matrix looked up by token id and scaled, and the gradient of that matrix,
  alone or added to what the head's backward left in a tied one (``embed_fwd``, ``embed_bwd``);
* ``grad_norm`` / ``grad_clip``: the norm over all gradients of a step, and their clipping into the buffers that the
  optimiser or a reduction reads (``grad_norm``, ``grad_clip``).

Where ``own`` is false the operators are computed in their plain form, in elementary torch operations; the references of ``exact`` are
written apart from it, in 64 bits.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

VOCAB = 151936


# ---- the cases -----------------------------------------------------------------------------------------------


def _pref(name, P, G, T, lo=0.25, dist="uniform", loss="logistic", pairs="all", mean=False, ref=True, weights="prompt", beta=0.1,
          margin=0.0, margin_scale=0.0, smoothing=0.0, nll=0.0):
    """Response lengths lie in [lo * T, T]; `dist` is their distribution."""
    c = dict(kind="preference", P=P, G=G, T=T, lo=lo, dist=dist, loss=loss, pairs=pairs, mean=mean, ref=ref, weights=weights, beta=beta,
             margin=margin, margin_scale=margin_scale, smoothing=smoothing, nll=nll)
    return dict(c, name=name) if name else c


def _embed(name, kind, R, T, d, V, dtype="bf16", rows="bf16", lo=0.25, dist="uniform", add=False, scale=1.0):
    """dtype: type of the matrix; rows: type of the rows that are written (forward) or of their gradient (backward)."""
    c = dict(kind=kind, R=R, T=T, d=d, V=V, dtype=dtype, rows=rows, lo=lo, dist=dist, add=add, scale=scale)
    return dict(c, name=name) if name else c


def _grads(name, kind, shapes, dtype="f32", out="f32", max_norm=1.0):
    """shapes: "head" V x d and layers' matrices, "kv" the gate's three, "many" `count` ragged ones; see _sizes."""
    c = dict(kind=kind, shapes=shapes, dtype=dtype, out=out, max_norm=max_norm)
    return dict(c, name=name) if name else c


def listed():
    return [
        # Two preferences of 32 tokens: unit runs and debugging, where launches and latency are all there is.
        _pref("pref-2x4x32", 2, 4, 32),
        # Chosen and rejected responses of 64 prompts with long-tailed odd lengths; no reference model, length-normalised, a margin.
        _pref("pref-64x2x1021", 64, 2, 1021, lo=1 / 32, dist="loguniform", mean=True, ref=False, beta=2.0, margin=0.5),
        # All ordered pairs of the 8x16x8192 workload, smoothed, with a likelihood term on what was preferred.
        _pref("pref-8x16x8192", 8, 16, 8192, lo=0.125, weights="pair", smoothing=0.1, nll=0.2),
        # The 2x4x32 workload's prompt rows, fp32.
        _embed("embed-f32-2x4x32", "embed_fwd", 8, 32, 256, 4096, "f32", "f32", scale=16.0),
        # The 32x8x2048 workload: every row of a step's batch.
        _embed("embed-32x8x2048-d4096", "embed_fwd", 256, 2048, 4096, VOCAB),
        # Gradient of the small fp32 workload's matrix.
        _embed("embed-grad-f32-2x4x32", "embed_bwd", 8, 32, 256, 4096, "f32", "f32", scale=16.0),
        # A small policy step (8x8x256) with a tied matrix: added to the head's dW.
        _embed("embed-grad-8x8x256-d2048", "embed_bwd", 64, 256, 2048, VOCAB, add=True, scale=math.sqrt(2048)),
        # A matrix of its own (every row of dW is written), long-tailed lengths, fp32 gradients of the rows.
        _embed("embed-grad-64x500-d3584", "embed_bwd", 64, 500, 3584, 152064, rows="f32", lo=1 / 128, dist="loguniform"),
        # The 32x8x2048 workload's step with a tied matrix.
        _embed("embed-grad-32x8x2048-d4096", "embed_bwd", 256, 2048, 4096, VOCAB, add=True),
        # The gate's three gradients (dU, dW, db at d = 1024): a norm for the log.
        _grads("norm-kv-gate", "grad_norm", "kv-1024"),
        # A small model's 290 tensors, ragged and odd, clipped into one bucket for a reduction.
        _grads("clip-290-tensors", "grad_clip", "many-290-120000000", out="bf16"),
        # The head's dW of the benchmarked workload beside a few layers in bf16, clipped for the optimiser.
        _grads("clip-head-d4096", "grad_clip", "head-151936-4096", dtype="mixed"),
    ]


def _log_int(rng: random.Random, lo: float, hi: float) -> int:
    return max(int(lo), min(int(hi), int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random):
    kind = rng.choice(["preference", "preference", "embed_fwd", "embed_bwd", "embed_bwd", "embed_bwd", "grad_norm", "grad_clip"])
    if kind == "preference":
        G = rng.choice([2, 2, 2, 3, 4, 7, 8, 16])
        T = _log_int(rng, 1, 8192)
        P = max(1, min(_log_int(rng, 1, 512), (1 << 20) // (G * T)))
        loss = rng.choice(["logistic", "logistic", "hinge", "squared"])
        mean = rng.random() < 0.4
        return _pref(None, P, G, T, lo=rng.choice([0.0, 1 / 64, 0.25, 1.0]), dist=rng.choice(["uniform", "loguniform"]), loss=loss,
                     pairs=rng.choice(["all", "all", "extremes"]), mean=mean, ref=rng.random() < 0.7,
                     weights=rng.choice(["prompt", "pair"]), beta=rng.choice([0.5, 2.0]) if mean else rng.choice([0.05, 0.1]),
                     margin=rng.choice([0.0, 0.3]), margin_scale=rng.choice([0.0, 0.0, 0.5]),
                     smoothing=rng.choice([0.0, 0.0, 0.1]) if loss == "logistic" else 0.0, nll=rng.choice([0.0, 0.0, 0.1]))
    if kind.startswith("embed"):
        d = rng.choice([8, 64, 256, 320, 1000, 1024, 2048, 2560, 3584, 4096, 5120])
        V = _log_int(rng, 100, 152064)
        n = _log_int(rng, 1, min(524288, (1 << 31) // d))
        R = min(n, rng.choice([1, 2, 3, 8, 16, 64, 100, 256]))
        return _embed(None, kind, R, n // R, d, V, dtype=rng.choice(["bf16", "bf16", "f32"]), rows=rng.choice(["bf16", "f32"]),
                      lo=rng.choice([0.0, 1 / 64, 0.25, 1.0]), dist=rng.choice(["uniform", "loguniform"]),
                      add=kind == "embed_bwd" and rng.random() < 0.5, scale=rng.choice([1.0, 16.0, 45.25]))
    dtype = rng.choice(["f32", "f32", "bf16", "mixed"])
    shapes = rng.choice(["kv-%d" % (64 * _log_int(rng, 1, 64)), "head-%d-%d" % (_log_int(rng, 100, VOCAB), 64 * _log_int(rng, 1, 40)),
                         "many-%d-%d" % (_log_int(rng, 2, 400), _log_int(rng, 1000, 200000000))])
    return _grads(None, kind, shapes, dtype=dtype, out=rng.choice(["f32", "bf16"]), max_norm=rng.choice([1.0, 0.1, 1e4]))


# ---- inputs --------------------------------------------------------------------------------------------------


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _normal(g, rows, cols, std, dtype):
    """N(0, std^2) drawn in float32 and rounded to the storage type, in blocks of rows."""
    out = torch.empty(rows, cols, dtype=dtype, device="cuda")
    step = max(1, (1 << 28) // cols)
    for r in range(0, rows, step):
        m = min(step, rows - r)
        out[r:r + m] = torch.randn(m, cols, generator=g, device="cuda").mul_(std)
    return out


def _lengths(case, rng, R):
    """Lengths in [lo * T, T]; where lo is 0 some responses are empty."""
    T = case["T"]
    lo = max(0 if case["lo"] == 0 else 1, int(case["lo"] * T))
    if case["dist"] == "uniform":
        return [rng.randint(lo, T) for _ in range(R)]
    return [_log_int(rng, lo + 1, T + 1) - 1 if lo == 0 else _log_int(rng, lo, T) for _ in range(R)]


def _mean_length(case):
    T, lo = case["T"], max(1.0, case["lo"] * case["T"])
    if case["dist"] == "uniform" or lo >= T:
        return 0.5 * (T + min(lo, T))
    return (T - lo) / math.log(T / lo)


def _zipf(V):
    """Zipf(1.1) over the vocabulary, hot ids first: the weights of the token ids."""
    return torch.arange(1, V + 1, dtype=torch.float64, device="cuda").pow_(-1.1)


def _sizes(case):
    """Element counts of the gradients, from the case alone."""
    what, *n = case["shapes"].split("-")
    n = [int(v) for v in n]
    if what == "kv":
        return [n[0] * n[0], n[0] * n[0], n[0]]
    if what == "head":
        d = n[1]
        return [n[0] * d] + [d * d, d * d, 4 * d * d, 4 * d * d, d, d]
    rng = random.Random(case["shapes"])
    raw = [math.exp(rng.uniform(0.0, 9.0)) for _ in range(n[0])]
    return [max(1, int(n[1] * v / sum(raw))) for v in raw]


def _grad_types(case, count):
    """Type of each gradient: "mixed" is fp32 for the first (as the head's backward leaves it) and bf16 for every second after it."""
    if case["dtype"] == "mixed":
        return [torch.bfloat16 if i % 2 else torch.float32 for i in range(count)]
    return [_TYPES[case["dtype"]]] * count


def prepare(case, seed):
    g, rng = _gen(seed), random.Random(seed)
    kind = case["kind"]
    s = dict(case=case)
    f32 = dict(dtype=torch.float32, device="cuda")
    if kind == "preference":
        P, G, T = case["P"], case["G"], case["T"]
        R, N = P * G, P * G * T
        s["lens"] = torch.tensor(_lengths(case, rng, R), dtype=torch.int32, device="cuda")
        # token log-probabilities of a language model: many near 0, a tail to -15; the reference differs a little at each token
        s["logp"] = -torch.rand(N, generator=g, device="cuda").pow_(3).mul_(12.0)
        s["logp_ref"] = (s["logp"] + 0.1 * torch.randn(N, generator=g, device="cuda")).clamp_(max=0.0) if case["ref"] else None
        # rewards on a grid of tenths: ties, which make no pair, occur
        s["reward"] = torch.tensor([rng.randint(0, 10) / 10.0 for _ in range(R)], **f32)
        if own:
            import paper_2603_04411_amd as L
            s["params"] = L.make_preference(loss=case["loss"], pairs=case["pairs"], mean=case["mean"], weights=case["weights"],
                                            beta=case["beta"], margin=case["margin"], margin_scale=case["margin_scale"],
                                            smoothing=case["smoothing"], nll_coef=case["nll"])
            s["loss"], s["g_logp"], s["ratio"] = torch.empty(1, **f32), torch.empty(N, **f32), torch.empty(R, **f32)
            s["stats"] = torch.empty(4, **f32)
            s["ws"] = torch.empty(L.preference_workspace_bytes(P, G, T), dtype=torch.uint8, device="cuda")
        return s
    if kind.startswith("embed"):
        R, T, d, V = case["R"], case["T"], case["d"], case["V"]
        N = R * T
        s["lens"] = torch.tensor(_lengths(case, rng, R), dtype=torch.int32, device="cuda")
        cdf = _zipf(V).cumsum_(0)
        u = torch.rand(N, generator=g, device="cuda", dtype=torch.float64) * cdf[-1]
        s["tok"] = torch.searchsorted(cdf, u, right=True).clamp_(max=V - 1).to(torch.int32)
        if kind == "embed_fwd":
            s["W"] = _normal(g, V, d, 0.02, _TYPES[case["dtype"]])
        else:
            s["gX"] = _normal(g, N, d, 1.0 / math.sqrt(N), _TYPES[case["rows"]])
            if case["add"]:
                s["dW"] = _normal(g, V, d, 1.0 / math.sqrt(N), torch.float32)   # what the head's backward left
        if own:
            import paper_2603_04411_amd as L
            s["desc"] = L.make_embed_desc(R, T, d, V, case["dtype"], rows=case["rows"], flags=L.FLAG_ACCUM_DW if case["add"] else 0)
            s["ws"] = torch.empty(L.embed_workspace_bytes(s["desc"]), dtype=torch.uint8, device="cuda")
            if kind == "embed_fwd":
                s["X"] = torch.empty(N, d, dtype=_TYPES[case["rows"]], device="cuda")
            elif not case["add"]:
                s["dW"] = torch.empty(V, d, **f32)
        return s
    sizes = _sizes(case)
    # layers' gradients differ in scale; a step's norm lies around ten
    total = sum(sizes)
    s["grads"] = [_normal(g, 1, n, 10.0 / math.sqrt(total) * math.exp(rng.uniform(-1.5, 0.5)), t).view(-1)
                  for n, t in zip(sizes, _grad_types(case, len(sizes)))]
    # clipped gradients go into one bucket, each at a multiple of 64 elements
    s["starts"] = np.concatenate([[0], np.cumsum([-(-n // 64) * 64 for n in sizes])]).tolist()
    if own:
        import paper_2603_04411_amd as L
        s["list"] = L.make_grad_list(s["grads"])
        s["norm"] = torch.empty(2, **f32)
        s["ws"] = torch.empty(L.grad_workspace_bytes(), dtype=torch.uint8, device="cuda")
        if kind == "grad_clip":
            s["bucket"] = torch.zeros(s["starts"][-1], dtype=_TYPES[case["out"]], device="cuda")
            s["outs"] = L.make_grad_list([s["bucket"][b:b + n] for b, n in zip(s["starts"], sizes)])
    return s


# ---- one pass ------------------------------------------------------------------------------------------------


def run(s):
    return {"preference": _run_preference, "embed_fwd": _run_embed_fwd, "embed_bwd": _run_embed_bwd, "grad_norm": _run_grad_norm,
            "grad_clip": _run_grad_clip}[s["case"]["kind"]](s, s["case"])


def _run_preference(s, case):
    P, G, T = case["P"], case["G"], case["T"]
    if own:
        import paper_2603_04411_amd as L
        L.preference_loss(s["params"], s["logp"], s["logp_ref"], s["reward"], s["lens"], P, G, T, s["loss"], s["g_logp"], s["ratio"],
                          s["stats"], s["ws"])
        return dict(loss=s["loss"], g_logp=s["g_logp"], ratio=s["ratio"], stats=s["stats"])
    # sums over responses and what is made of them in 64 bits: the difference of two long sums decides the loss
    R, beta = P * G, case["beta"]
    n = s["lens"].clamp(0, T).double()
    valid = torch.arange(T, device="cuda")[None, :] < s["lens"][:, None]
    logp = s["logp"].view(R, T).double().masked_fill(~valid, 0.0)
    delta = logp - s["logp_ref"].view(R, T).double().masked_fill(~valid, 0.0) if case["ref"] else logp
    per = torch.where(n > 0, 1.0 / n.clamp(min=1), 0.0)
    ratio = delta.sum(1) * (per if case["mean"] else 1.0)
    mean_logp = logp.sum(1) * per
    q, rw = ratio.view(P, G), s["reward"].double().view(P, G)
    pair = rw[:, :, None] > rw[:, None, :]                       # [prompt, preferred, other]
    if case["pairs"] == "extremes":
        at = torch.arange(G, device="cuda")
        best = (at[None, :] == rw.argmax(1, keepdim=True))
        worst = (at[None, :] == rw.argmin(1, keepdim=True))
        pair = pair & best[:, :, None] & worst[:, None, :]
    count = pair.sum((1, 2)).double()
    w = (1.0 / (P * count.clamp(min=1)) if case["weights"] == "prompt" else (1.0 / count.sum().clamp(min=1)).expand(P))
    w = pair.double() * w[:, None, None]
    u = q[:, :, None] - q[:, None, :]
    gap = rw[:, :, None] - rw[:, None, :]
    h = beta * u - case["margin"] - case["margin_scale"] * gap
    if case["loss"] == "logistic":
        soft = torch.log1p(torch.exp(-h.abs()))                  # -log sigma(h) = max(-h, 0) + log(1 + e^-|h|)
        e = case["smoothing"]
        each = (1 - e) * ((-h).clamp(min=0) + soft) + e * (h.clamp(min=0) + soft)
        du = beta * (e - 1.0 / (1.0 + torch.exp(h)))
    elif case["loss"] == "hinge":
        each, du = (1.0 - h).clamp(min=0), -beta * (h < 1).double()
    else:
        r = h / beta - 1.0 / (2.0 * beta)
        each, du = r * r, 2.0 * r
    each = each - case["nll"] * mean_logp.view(P, G)[:, :, None]
    du = du * w
    c = (du.sum(2) - du.sum(1)).reshape(R)
    g = c * per if case["mean"] else c
    g = g - case["nll"] * w.sum(2).reshape(R) * per
    m = count.sum()
    share = pair.double() / m.clamp(min=1)
    stats = torch.stack([(share * (u > 0)).sum(), (share * (beta * q)[:, :, None]).sum(), (share * (beta * q)[:, None, :]).sum(), m])
    return dict(loss=(w * each).sum().float().reshape(1), g_logp=torch.where(valid, g[:, None], 0.0).float().reshape(-1),
                ratio=ratio.float(), stats=stats.float())


def _run_embed_fwd(s, case):
    if own:
        import paper_2603_04411_amd as L
        L.embed_fwd(s["desc"], s["W"], s["tok"], s["lens"], case["scale"], s["X"], s["ws"])
        return s["X"]
    valid = (torch.arange(case["T"], device="cuda")[None, :] < s["lens"][:, None]).reshape(-1)
    x = s["W"][torch.where(valid, s["tok"], 0).long()].float().mul_(case["scale"])
    return x.masked_fill_(~valid[:, None], 0.0).to(_TYPES[case["rows"]])


def _run_embed_bwd(s, case):
    if own:
        import paper_2603_04411_amd as L
        L.embed_bwd(s["desc"], s["gX"], s["tok"], s["lens"], case["scale"], s["dW"], s["ws"])
        return s["dW"]
    valid = (torch.arange(case["T"], device="cuda")[None, :] < s["lens"][:, None]).reshape(-1)
    at = valid.nonzero()[:, 0]
    rows = s["gX"][at].float().mul_(case["scale"])
    dW = s["dW"] if case["add"] else torch.zeros(case["V"], case["d"], dtype=torch.float32, device="cuda")
    return dW.index_add_(0, s["tok"][at].long(), rows)


def _plain_norm(s):
    return torch.stack([t.float().square().sum(dtype=torch.float64) for t in s["grads"]]).sum().sqrt()


def _run_grad_norm(s, case):
    if own:
        import paper_2603_04411_amd as L
        L.grad_norm(s["list"], s["norm"], s["ws"])
        return s["norm"][:1]
    return _plain_norm(s).float().reshape(1)


EPS = 1e-6


def _run_grad_clip(s, case):
    if own:
        import paper_2603_04411_amd as L
        L.grad_clip(s["list"], s["outs"], case["max_norm"], EPS, s["norm"], s["ws"])
        return dict(norm=s["norm"], bucket=s["bucket"])
    norm = _plain_norm(s)
    c = (case["max_norm"] / (norm + EPS)).clamp(max=1.0)
    bucket = torch.cat([torch.nn.functional.pad((t.float() * c.float()).to(_TYPES[case["out"]]), (0, -t.numel() % 64)) for t in s["grads"]])
    return dict(norm=torch.stack([norm, c]).float(), bucket=bucket)


# ---- what a pass cannot do without ---------------------------------------------------------------------------


def _different(V, n):
    """Expected number of different ids among n draws."""
    p = np.arange(1, V + 1, dtype=np.float64) ** -1.1
    p /= p.sum()
    return float(-np.expm1(n * np.log1p(-np.minimum(p, 1 - 1e-12))).sum())


def work(case):
    kind = case["kind"]
    if kind == "preference":
        N = case["P"] * case["G"] * case["T"]
        nv = case["P"] * case["G"] * _mean_length(case)
        return dict(bytes=4.0 * nv * (2 if case["ref"] else 1) + 4.0 * N, flops=4.0 * nv)
    if kind.startswith("embed"):
        N, d, V = case["R"] * case["T"], case["d"], case["V"]
        nv = max(1.0, case["R"] * _mean_length(case))
        rows = {"bf16": 2, "f32": 4}[case["rows"]]
        if kind == "embed_fwd":
            return dict(bytes=4.0 * nv + _different(V, nv) * d * {"bf16": 2, "f32": 4}[case["dtype"]] + 1.0 * N * d * rows, flops=nv * d)
        table = 8.0 * _different(V, nv) * d if case["add"] else 4.0 * V * d
        return dict(bytes=4.0 * nv + nv * d * rows + table, flops=nv * d)
    sizes = _sizes(case)
    n = float(sum(sizes))
    read = float(sum(m * t.itemsize for m, t in zip(sizes, _grad_types(case, len(sizes)))))
    if kind == "grad_norm":
        return dict(bytes=read, flops=2 * n)
    return dict(bytes=read + n * _TYPES[case["out"]].itemsize, flops=3 * n)


# ---- the definitions, in 64 bits -----------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    return {"preference": _exact_preference, "embed_fwd": _exact_embed_fwd, "embed_bwd": _exact_embed_bwd, "grad_norm": _exact_grad_norm,
            "grad_clip": _exact_grad_clip}[case["kind"]](s, case)


def _exact_preference(s, case):
    """Pair by pair, on the host."""
    P, G, T, beta, eps = case["P"], case["G"], case["T"], case["beta"], case["smoothing"]
    R = P * G
    logp = s["logp"].cpu().numpy().astype(np.float64).reshape(R, T)
    base = s["logp_ref"].cpu().numpy().astype(np.float64).reshape(R, T) if case["ref"] else np.zeros((R, T))
    lens, rw = s["lens"].cpu().numpy(), s["reward"].cpu().numpy().astype(np.float64)
    ratio, like = np.zeros(R), np.zeros(R)
    for r in range(R):
        n = int(lens[r])
        if n:
            ratio[r] = math.fsum((logp[r, :n] - base[r, :n]).tolist()) / (n if case["mean"] else 1)
            like[r] = math.fsum(logp[r, :n].tolist()) / n
    pairs = []
    for p in range(P):
        at = range(p * G, (p + 1) * G)
        if case["pairs"] == "extremes":
            a, b = max(at, key=lambda i: (rw[i], -i)), min(at, key=lambda i: (rw[i], i))
            mine = [(a, b)] if rw[a] > rw[b] else []
        else:
            mine = [(a, b) for a in at for b in at if rw[a] > rw[b]]
        pairs += [(a, b, 1.0 / (P * len(mine))) for a, b in mine]
    M = len(pairs)
    loss, c, nll, hits, sa, sb = 0.0, np.zeros(R), np.zeros(R), 0, 0.0, 0.0
    for a, b, w in pairs:
        w = w if case["weights"] == "prompt" else 1.0 / M
        u = ratio[a] - ratio[b]
        h = beta * u - case["margin"] - case["margin_scale"] * (rw[a] - rw[b])
        if case["loss"] == "logistic":
            loss += w * ((1 - eps) * np.logaddexp(0.0, -h) + eps * np.logaddexp(0.0, h))
            slope = beta * (eps - 0.5 * (1.0 - math.tanh(0.5 * h)))
        elif case["loss"] == "hinge":
            loss += w * max(0.0, 1.0 - h)
            slope = -beta if h < 1 else 0.0
        else:
            r = h / beta - 0.5 / beta
            loss += w * r * r
            slope = 2.0 * r
        loss -= w * case["nll"] * like[a]
        c[a] += w * slope
        c[b] -= w * slope
        nll[a] += w * case["nll"]
        hits, sa, sb = hits + (u > 0), sa + beta * ratio[a], sb + beta * ratio[b]
    g = np.zeros((R, T))
    for r in range(R):
        n = int(lens[r])
        if n:
            g[r, :n] = c[r] / (n if case["mean"] else 1) - nll[r] / n
    m = max(M, 1)
    return dict(loss=np.array([loss]), g_logp=g.reshape(-1), ratio=ratio, stats=np.array([hits / m, sa / m, sb / m, float(M)]))


def _exact_embed_fwd(s, case):
    T, d = case["T"], case["d"]
    X = torch.zeros(case["R"] * T, d, dtype=torch.float64, device="cuda")
    for r, n in enumerate(s["lens"].tolist()):
        X[r * T:r * T + n] = s["W"][s["tok"][r * T:r * T + n].long()].double() * case["scale"]
    return X


def _exact_embed_bwd(s, case):
    """Rows in the order of their ids, and differences of their running sums: each id's rows end where the next id's begin."""
    T, d, V = case["T"], case["d"], case["V"]
    at = torch.cat([torch.arange(r * T, r * T + n, device="cuda") for r, n in enumerate(s["lens"].tolist())])
    dW = s["dW"].double() if case["add"] else torch.zeros(V, d, dtype=torch.float64, device="cuda")
    if not at.numel():
        return dW
    ids, order = s["tok"][at].long().sort(stable=True)
    at = at[order]
    last = torch.cat([torch.nonzero(ids[1:] != ids[:-1])[:, 0], torch.tensor([ids.numel() - 1], device="cuda")])
    step = max(8, (1 << 27) // at.numel())
    for c in range(0, d, step):
        run_ = s["gX"][:, c:c + step][at].double().cumsum(0)[last]
        run_[1:] -= run_[:-1].clone()
        dW[ids[last], c:c + step] += run_ * case["scale"]
    return dW


def _exact_norm(s):
    return math.sqrt(math.fsum(float(torch.linalg.vector_norm(t.double())) ** 2 for t in s["grads"]))


def _exact_grad_norm(s, case):
    return torch.tensor([_exact_norm(s)], dtype=torch.float64)


def _exact_grad_clip(s, case):
    n = _exact_norm(s)
    c = min(1.0, case["max_norm"] / (n + EPS))
    bucket = torch.zeros(s["starts"][-1], dtype=torch.float64, device="cuda")
    for t, b in zip(s["grads"], s["starts"]):
        bucket[b:b + t.numel()] = t.double() * c
    return dict(norm=torch.tensor([n, c], dtype=torch.float64), bucket=bucket)
