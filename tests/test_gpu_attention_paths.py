"""Attention on the paths that only larger calls take, against the fp64 oracle with its derived bounds: the backward of more than 512 queries, more blocks
of keys than workgroups that share them, outputs that are written past the caches (above 32 MB), plain caches that are read past them (above 256 MB)."""
import numpy as np
import pytest

from tests.attention_cases import bounds, holds
from tests.test_gpu_attention import Problem, _name, check_bwd, check_fwd, np64

pytestmark = pytest.mark.gpu

LONG = [
    dict(B=1, Tq=1030, Tk=1030, Hq=4, Hkv=2, D=128, window=600, sinks=5),
    dict(B=2, Tq=1100, Tk=1100, Hq=2, Hkv=1, D=64, len_q=[1100, 513], len_k=[1100, 700]),
    dict(B=1, Tq=640, Tk=900, Hq=3, Hkv=1, D=96, first="wide"),
    dict(B=2, Tq=800, Tk=800, Hq=3, Hkv=1, D=40, window=1, sinks=129, len_q=[800, 530], len_k=[800, 530]),
    dict(B=1, Tq=700, Tk=900, Hq=2, Hkv=1, D=128, dtype="f32", window=300, sinks=1),
]


@pytest.mark.parametrize("case", LONG, ids=_name)
def test_more_than_512_queries(case):
    p = Problem(seed=41, **case)
    check_fwd(p)
    check_bwd(p)


def _lengths(B, T, seed):
    """Ragged, one of them full, one empty and one of a single token."""
    n = np.random.default_rng(seed).integers(2, T + 1, B)
    n[[0, B // 3, B - 1]] = T, 0, 1
    return n.tolist()


MANY = [      # blocks of keys: 960 for 512 resident workgroups, 384 for 256 in fp32
    dict(B=40, Tq=300, Tk=300, Hq=16, Hkv=8, D=64, len_q=_lengths(40, 300, 1), len_k=_lengths(40, 300, 1), window=150, sinks=2),
    dict(B=40, Tq=160, Tk=300, Hq=8, Hkv=8, D=128),
    dict(B=16, Tq=150, Tk=300, Hq=8, Hkv=8, D=64, dtype="f32", len_q=_lengths(16, 150, 2), len_k=_lengths(16, 300, 3)),
    dict(B=16, Tq=130, Tk=300, Hq=16, Hkv=8, D=72, dtype="f32", window=70, sinks=140),
]


@pytest.mark.parametrize("case", MANY, ids=lambda c: f"{c['B']}x{c['Tq']}x{c['Tk']}-{c.get('dtype', 'bf16')}-{c['D']}")
def test_more_blocks_of_keys_than_workgroups(case):
    """A share covers several blocks of keys, and goes on from one key head to the next."""
    check_bwd(Problem(seed=42, **case))


@pytest.mark.parametrize("case", [dict(B=2, Tq=50, Tk=80, Hq=4, Hkv=2, D=64, len_q=[0, 0], len_k=[0, 0]),
                                  dict(B=2, Tq=200, Tk=300, Hq=4, Hkv=2, D=128, len_q=[0, 200], len_k=[0, 0], window=3, sinks=2),
                                  dict(B=1, Tq=700, Tk=700, Hq=2, Hkv=1, D=64, len_q=[0], len_k=[700], dtype="f32")], ids=range(3))
def test_batches_without_a_single_pair(case):
    p = Problem(seed=45, **case)
    check_fwd(p)
    check_bwd(p)


LARGE = [
    dict(B=8, Tq=260, Tk=260, Hq=64, Hkv=8, D=128, window=200, sinks=3, len_q=_lengths(8, 260, 4), len_k=_lengths(8, 260, 4)),
    dict(B=9, Tq=260, Tk=300, Hq=64, Hkv=8, D=120, first="wide"),
    dict(B=4, Tq=260, Tk=260, Hq=64, Hkv=8, D=128, dtype="f32", first="head", len_q=_lengths(4, 260, 5), len_k=_lengths(4, 260, 5)),
]


@pytest.mark.parametrize("case", LARGE, ids=lambda c: f"{c['B']}x{c['Tq']}x{c['Tk']}-{c.get('dtype', 'bf16')}-{c['D']}")
def test_outputs_past_the_caches(case):
    p = Problem(seed=43, **case)
    assert p.x[0].size * p.q.element_size() > 32 << 20
    check_fwd(p)
    check_bwd(p)


@pytest.mark.parametrize("dtype,Tq,Hq,window,sinks", [("bf16", 1, 32, 0, 0), ("bf16", 1, 96, 0, 0), ("bf16", 4, 64, 3900, 5), ("f32", 1, 32, 0, 0), ("f32", 3, 40, 0, 0),
                                                      ("f32", 4, 64, 3900, 5)])
@pytest.mark.parametrize("D", [64, 120])
def test_plain_caches_past_the_last_level_cache(dtype, Tq, Hq, window, sinks, D):
    """Few rows over caches that count as more than 256 MB: all sequences read one, so that it is quickly made.  (Rows: four with weights from logits, up to
    sixteen, up to 32.)"""
    import torch
    import paper_2603_04411_amd as L
    Hkv, Tk, esz = 8, 4200, 2 if dtype == "bf16" else 4
    B = (256 << 20) // (2 * Hkv * 3904 * D * esz) + 2
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    rng = np.random.default_rng(44 + Tq + Hq)
    q = torch.from_numpy(rng.standard_normal((B, Tq, Hq, D))).to(tdt)
    k, v = (torch.from_numpy(rng.standard_normal((1, Tk, Hkv, D))).to(tdt) for _ in range(2))
    lk = rng.integers(1, Tk + 1, B)
    lk[:3] = Tk, 1, Tk - 1
    lq = np.minimum(rng.integers(0, Tq + 1, B), lk)
    lq[:3] = Tq, 1, Tq
    dq, dk, dv = (x.cuda() for x in (q, k, v))
    dk, dv = (x.expand(B, Tk, Hkv, D) for x in (dk, dv))
    layout = (0, Hkv * D, D)
    desc = L.make_attn_desc(B, Tq, Tk, Hq, Hkv, D, dtype, window=window, sinks=sinks, k=layout, v=layout)
    len_q, len_k = (torch.from_numpy(x.astype(np.int32)).cuda() for x in (lq, lk))
    out, lse = torch.full_like(dq, 7.0), torch.full((B, Hq, Tq), 7.0, device="cuda")
    weight = torch.full((B, Hkv, Tk), 7.0, device="cuda")
    ws = torch.full((L.attn_workspace_bytes(desc),), 255, dtype=torch.uint8, device="cuda")
    L.attn_fwd(desc, dq, dk, dv, len_q, len_k, out, lse, weight, 0.0, ws)
    assert L.lmhead_check(ws) == 0
    plain = torch.full_like(dq, 7.0)
    L.attn_fwd(desc, dq, dk, dv, len_q, len_k, plain, None, None, 0.0, ws)
    at = [0, 1, 2, B // 2, B - 1]
    host = [x.double().numpy() for x in (q, k, v)]
    want, bound = bounds(host[0][at], *(np.broadcast_to(x, (len(at), Tk, Hkv, D)) for x in host[1:]), lq[at], lk[at], float(np.float32(D ** -0.5)), window, sinks,
                         dtype)
    holds(np64(out[at]), want["out"], bound["out"], "out")
    holds(np64(plain[at]), want["out"], bound["out"], "out without weights")
    holds(np64(lse[at]), want["lse"], bound["lse"], "lse")
    got = np64(weight)
    for i, b in enumerate(at):
        n = lk[b]
        holds(got[b, :, :n], want["weight"][i, :, :n], bound["weight"][i, :, :n] + 2.0 ** -22 * want["weight"][i, :, :n], "weight")
    for b in range(B):
        assert (got[b, :, lk[b]:] == 7.0).all() and (np64(out[b, lq[b]:]) == 0).all()
        assert np.allclose(got[b, :, :lk[b]].sum(1), lq[b] * Hq // Hkv, rtol=1e-4)
