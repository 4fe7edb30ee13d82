"""preference_loss against its oracle: every loss, pairing and weighting, lengths from none to several blocks, groups of one to
hundreds, rewards that tie or are no numbers, values in masked places that must not matter."""
import numpy as np
import pytest

from oracle import train_oracle as O
from tests.harness import np64, to_device

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24


def run(q, logp, ref, reward, lens, P, G, T, outs=True, ws=None):
    import torch
    import paper_2603_04411_amd as L
    R, N = P * G, P * G * T
    loss, g = torch.full((1,), 7.0, device="cuda"), torch.full((N,), 7.0, device="cuda")
    ratio, stats = torch.full((R,), 7.0, device="cuda"), torch.full((4,), 7.0, device="cuda")
    if ws is None:
        ws = torch.full((L.preference_workspace_bytes(P, G, T),), 0xFF, dtype=torch.uint8, device="cuda")
    L.preference_loss(q, logp, ref, reward, lens, P, G, T, loss, g if outs else None, ratio if outs else None, stats if outs else None, ws)
    torch.cuda.synchronize()
    return loss, g, ratio, stats


def inputs(P, G, T, seed, lens=None, reward=None):
    r = np.random.default_rng(seed)
    R = P * G
    lens = r.integers(0, T + 1, R) if lens is None else np.asarray(lens)
    reward = r.integers(0, 5, R) / 4 if reward is None else reward
    logp = (-12 * r.random(R * T) ** 3).astype(np.float32)
    ref = (logp + 0.2 * r.standard_normal(R * T)).astype(np.float32)
    # what padding holds must not matter
    pad = (np.arange(T)[None, :] >= np.clip(lens, 0, T)[:, None]).reshape(-1)
    logp[pad] = np.resize(np.array([np.nan, np.inf, -np.inf, 1e38], dtype=np.float32), int(pad.sum()))
    ref[pad] = np.nan
    return logp, ref, np.asarray(reward, dtype=np.float32), lens.astype(np.int32)


def check(P, G, T, seed, lens=None, reward=None, use_ref=True, **kw):
    import paper_2603_04411_amd as L
    logp, ref, rw, lens = inputs(P, G, T, seed, lens, reward)
    ref = ref if use_ref else None
    q = L.make_preference(loss=kw.get("loss", "logistic"), pairs="extremes" if kw.get("extremes") else "all", mean=kw.get("mean", False),
                          weights="pair" if kw.get("per_pair") else "prompt",
                          **{k: kw[k] for k in ("beta", "margin", "margin_scale", "smoothing", "nll_coef") if k in kw})
    got = run(q, to_device(logp), None if ref is None else to_device(ref), to_device(rw), to_device(lens), P, G, T)
    # the parameters are given in fp32
    okw = {k: float(np.float32(v)) if k in ("beta", "margin", "margin_scale", "smoothing", "nll_coef") else v for k, v in kw.items()}
    okw.setdefault("beta", float(np.float32(0.1)))
    want = O.preference_loss(logp, ref, rw, lens, P, G, T, **okw)
    # fp64 throughout and one rounding to fp32: half a step, and what fp64 sums of values up to 12 T leave after cancellation
    tiny = 1e-13 * max(1.0, 12.0 * T * okw["beta"]) * (1 if kw.get("loss") != "squared" else 12.0 * T)
    for name, a, b in zip(("loss", "g_logp", "ratio", "stats"), got, want):
        a, b = np64(a).reshape(-1), np.asarray(b, dtype=np.float64).reshape(-1)
        assert np.all(np.abs(a - b) <= 1.01 * EPS * np.abs(b) + tiny + 1e-12 * (name == "ratio")), (name, float(np.abs(a - b).max()))
    return got, q


@pytest.mark.parametrize("loss", ["logistic", "hinge", "squared"])
@pytest.mark.parametrize("extremes", [False, True])
@pytest.mark.parametrize("mean,per_pair", [(False, False), (True, False), (False, True), (True, True)])
def test_every_form(loss, extremes, mean, per_pair):
    for seed, use_ref in ((1, True), (2, False)):
        check(5, 4, 37, seed, use_ref=use_ref, loss=loss, extremes=extremes, mean=mean, per_pair=per_pair, beta=2.0 if mean else 0.3,
              margin=0.25, margin_scale=0.5 * seed, smoothing=0.1 if loss == "logistic" else 0.0, nll_coef=0.3)


@pytest.mark.parametrize("P,G,T", [(1, 1, 1), (1, 2, 1), (2, 2, 2), (1, 2, 2047), (1, 2, 2048), (1, 2, 2049), (3, 3, 4097), (300, 2, 5),
                                   (2, 4, 1024), (2, 4, 1025), (32, 2, 128), (33, 2, 124), (32, 2, 129), (512, 2, 3), (513, 2, 3), (80, 2, 1025), (81, 2, 1030), (320, 2, 30),
                                   (641, 1, 20), (160, 4, 1024), (3000, 2, 1), (9000, 3, 2), (2, 8, 512), (2, 8, 513), (1, 16, 40), (1, 17, 40), (4, 6, 341), (4, 6, 342), (5, 5, 20), (81, 2, 1024), (163, 1, 7),
                                   (1, 63, 3), (1, 64, 3), (1, 65, 3), (2, 255, 2), (1, 257, 2), (2, 300, 1), (1, 700, 2), (17, 16, 130)])
def test_sizes(P, G, T):
    check(P, G, T, 11, mean=G > 2, per_pair=T % 2 == 0, nll_coef=0.1)
    check(P, G, T, 12, extremes=True, loss="squared", margin=0.1, use_ref=False)
    check(P, G, T, 13, per_pair=T % 2 == 1, lens=[T] * (P * G))


@pytest.mark.parametrize("P,G,T", [(2, 2, 32768), (2, 2, 32769), (1, 3, 100000), (1, 2, 2048 * 1024 + 5)])
def test_long_responses(P, G, T):
    check(P, G, T, 21, mean=True, nll_coef=0.1)
    check(P, G, T, 22, lens=[T, 0, 70, T - 1][:P * G], use_ref=False)


def test_as_many_slots_as_a_call_takes():
    """Two responses of 2^30 - 1 slots, of numbers whose sums are exact."""
    import torch
    import paper_2603_04411_amd as L
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    T, lens = (1 << 30) - 1, [(1 << 30) - 1, (1 << 29) + 3]
    logp = torch.full((2 * T,), -0.5, device="cuda")
    logp[T - 1], logp[T], logp[T + lens[1] - 1], logp[T + lens[1]] = -3.5, -1.5, -7.5, float("nan")
    loss, g, ratio, stats = (torch.full((n,), 7.0, device="cuda") for n in (1, 2 * T, 2, 4))
    ws = torch.empty(L.preference_workspace_bytes(1, 2, T), dtype=torch.uint8, device="cuda")
    q = L.make_preference(mean=True, beta=1.0)
    L.preference_loss(q, logp, None, torch.tensor([1.0, 0.0], device="cuda"), torch.tensor(lens, dtype=torch.int32, device="cuda"), 1, 2, T,
                      loss, g, ratio, stats, ws)
    s = [-0.5 - 3 / lens[0], -0.5 - 8 / lens[1]]
    slope = -1 / (1 + np.exp(s[0] - s[1]))
    assert abs(float(loss) - np.log1p(np.exp(s[1] - s[0]))) <= 1.01 * EPS and np.all(np.abs(np64(ratio) - s) <= 1.01 * EPS * 0.5 + 1e-15)
    want = [slope / lens[0], -slope / lens[1]]
    for r in range(2):
        at = g[r * T:(r + 1) * T]
        got = float(at[0])
        assert abs(got - want[r]) <= 1.01 * EPS * abs(want[r]) and bool((at[:lens[r]] == got).all()) and not bool(at[lens[r]:].any())


@pytest.mark.parametrize("T", [(1 << 31) - 2048, (1 << 31) - 2047, (1 << 31) - 1])
def test_one_response_of_as_many_slots_as_a_call_takes(T):
    """The last block of 2048 slots ends where an int does, or one slot of it lies before that."""
    import torch
    import paper_2603_04411_amd as L
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    logp, lens = torch.full((T,), -0.5, device="cuda"), torch.tensor([T], dtype=torch.int32, device="cuda")
    logp[0], logp[T - 1] = -2.0, -4.0
    loss, g, ratio, stats = (torch.full((n,), 7.0, device="cuda") for n in (1, T, 1, 4))
    ws = torch.empty(L.preference_workspace_bytes(1, 1, T), dtype=torch.uint8, device="cuda")
    L.preference_loss(L.make_preference(), logp, None, torch.zeros(1, device="cuda"), lens, 1, 1, T, loss, g, ratio, stats, ws)
    # one response is in no pair: loss, statistics and the gradient of every slot are 0
    assert float(loss) == 0.0 and not stats.any() and float(ratio) == float(np.float32(-0.5 * T - 5.0))
    assert all(not bool(g[lo:lo + (1 << 28)].any()) for lo in range(0, T, 1 << 28))


@pytest.mark.parametrize("weights", ["prompt", "pair"])
def test_one_prompt_of_as_many_responses_as_a_call_takes(weights):
    """2^31 pairs, all of them level: every loss is log 2, and a response's slope counts those above it and those below."""
    import torch
    import paper_2603_04411_amd as L
    R = 65535
    order = torch.randperm(R, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")
    logp, lens = torch.full((R,), -0.5, device="cuda"), torch.ones(R, dtype=torch.int32, device="cuda")
    loss, g, ratio, stats = run(L.make_preference(weights=weights, beta=0.5), logp, None, order.float(), lens, 1, R, 1)
    pairs = R * (R - 1) // 2
    # one rounding to fp32; fp64 sums of equal numbers, a thousand in a row and those in pairs, are off by 1e-13
    assert abs(float(loss) - np.log(2.0)) <= 1.01 * EPS * np.log(2.0)
    assert bool((ratio == -0.5).all()) and stats.tolist() == [0.0, -0.25, -0.25, float(np.float32(pairs))]
    below = np64(order)
    want = (below - (R - 1 - below)) * -0.25 / pairs
    assert np.all(np.abs(np64(g) - want) <= 1.01 * EPS * np.abs(want) + 1e-25)


def test_lengths_of_none_one_and_out_of_range():
    check(2, 3, 9, 3, lens=[0, 0, 0, 0, 1, 9], nll_coef=0.5)
    check(2, 3, 9, 3, lens=[0, 0, 0, 0, 1, 9], mean=True)
    check(2, 3, 9, 4, lens=[-5, 10, 1 << 30, -(1 << 31), 3, 9])          # clamped


def test_rewards_that_tie_and_are_no_numbers():
    nan, inf = float("nan"), float("inf")
    for extremes in (False, True):
        for per_pair in (False, True):
            kw = dict(extremes=extremes, per_pair=per_pair)
            got, _ = check(2, 3, 5, 5, reward=[1, 1, 1, 2, 2, 2], **kw)          # no pair at all
            assert float(got[0]) == 0.0 and not got[1].any() and not got[3].any()
            check(2, 3, 5, 6, reward=[1, 1, 1, 2, 1, 2], **kw)
            check(2, 3, 5, 7, reward=[nan, 1, 0, nan, nan, nan], **kw)
            check(2, 4, 5, 8, reward=[nan, 1, nan, 1, 0, inf, -inf, inf], **kw)


def test_a_token_of_probability_zero():
    import paper_2603_04411_amd as L
    P, G, T = 1, 2, 3
    logp = np.array([-1, -np.inf, -1, -1, -2, -3], dtype=np.float32)
    q = L.make_preference(beta=0.5)
    d = [to_device(a) for a in (logp, np.array([1, 0], dtype=np.float32), np.array([3, 3], dtype=np.int32))]
    loss, g, ratio, stats = run(q, d[0], None, d[1], d[2], P, G, T)
    assert float(loss) == np.inf and ratio.tolist() == [-np.inf, -6.0] and g.tolist() == [-0.5] * 3 + [0.5] * 3
    # a NaN that counts is seen in the loss
    for kind in ("logistic", "hinge", "squared"):
        logp[1] = np.nan
        loss, *_ = run(L.make_preference(loss=kind), to_device(logp), None, d[1], d[2], P, G, T)
        assert np.isnan(float(loss))


def test_far_apart_responses_neither_overflow_nor_vanish():
    import paper_2603_04411_amd as L
    lens, rw = to_device(np.array([8, 8], dtype=np.int32)), to_device(np.array([1, 0], dtype=np.float32))
    for sign in (1.0, -1.0):
        logp = np.concatenate([np.full(8, -100.0 if sign < 0 else -1e-3), np.full(8, -1e-3 if sign < 0 else -100.0)]).astype(np.float32)
        want = O.preference_loss(logp, None, [1, 0], [8, 8], 1, 2, 8, beta=1.0)
        loss, g, _, _ = run(L.make_preference(beta=1.0), to_device(logp), None, rw, lens, 1, 2, 8)
        assert abs(float(loss) - want[0]) <= 1.01 * EPS * abs(want[0]) + 1e-45      # e^-800 is 0 in fp32
        assert np.all(np.abs(np64(g) - want[1]) <= 1.01 * EPS * np.abs(want[1]) + 1e-45)


def test_the_same_bits_each_time_and_with_fewer_outputs():
    import torch
    import paper_2603_04411_amd as L
    P, G, T = 7, 5, 2100
    a = [to_device(x) for x in inputs(P, G, T, 9)]
    q = L.make_preference(weights="pair", nll_coef=0.2)
    first = run(q, a[0], a[1], a[2], a[3], P, G, T)
    for _ in range(3):
        assert all(torch.equal(x, y) for x, y in zip(run(q, a[0], a[1], a[2], a[3], P, G, T), first))
    loss, g, ratio, stats = run(q, a[0], a[1], a[2], a[3], P, G, T, outs=False)
    assert torch.equal(loss, first[0]) and bool((g == 7).all()) and bool((ratio == 7).all()) and bool((stats == 7).all())


def test_the_gradient_is_the_difference_quotient_of_the_loss():
    import paper_2603_04411_amd as L
    P, G, T = 2, 3, 4
    logp, ref, rw, lens = inputs(P, G, T, 21, lens=[4, 2, 3, 1, 4, 4], reward=[0, 1, 2, 1, 0, 3])
    q = L.make_preference(beta=0.5, smoothing=0.1, nll_coef=0.25)
    d = [to_device(x) for x in (logp, ref, rw, lens)]
    g = np64(run(q, d[0], d[1], d[2], d[3], P, G, T)[1])
    for i in range(P * G * T):
        if i % T >= lens[i // T]:
            assert g[i] == 0
            continue
        step, at = 2.0 ** -5, []
        for sign in (1, -1):
            lp = logp.copy()
            lp[i] += np.float32(sign * step)
            at.append((float(run(q, to_device(lp), d[1], d[2], d[3], P, G, T)[0]), float(lp[i])))
        slope = (at[0][0] - at[1][0]) / (at[0][1] - at[1][1])
        # losses below 4 are known to 2^-23 and divided by 2^-4; the third derivative of the logistic loss is at most beta^3 / 8, times step^2 / 6
        assert abs(slope - g[i]) <= 2 * 2.0 ** -23 * 4 / (2 * step) + 0.5 ** 3 / 8 * step ** 2 / 6 + 1e-7


@pytest.mark.parametrize("side", [0, 1])
@pytest.mark.parametrize("smoothing", [0.0, 0.25, 1.0])
def test_a_term_whose_factor_is_zero_is_left_out(smoothing, side):
    """h is -inf or +inf: what is left of the loss is one logarithm, or none."""
    import paper_2603_04411_amd as L
    logp, lens, rw = np.array([-1, -1, -2, -3], dtype=np.float32), np.array([2, 2], dtype=np.int32), np.array([1, 0], dtype=np.float32)
    logp[2 * side] = -np.inf
    want = O.preference_loss(logp, None, rw, lens, 1, 2, 2, beta=0.5, smoothing=smoothing)
    loss, g, _, _ = run(L.make_preference(beta=0.5, smoothing=smoothing), to_device(logp), None, to_device(rw), to_device(lens), 1, 2, 2)
    assert want[0] == (np.inf if 0 < smoothing < 1 or side == smoothing else 0.0) and float(loss) == want[0]
    assert np.array_equal(np64(g), want[1]) and want[1][0] == (0.5 * (smoothing - 1) if side == 0 else 0.5 * smoothing)


def test_a_hinge_of_no_number_has_no_slope():
    """[h < 1] of a NaN is 0; the pairs that are numbers keep their slopes."""
    import paper_2603_04411_amd as L
    logp, lens, rw = np.array([-1, np.nan, -2, -3], dtype=np.float32), np.ones(4, dtype=np.int32), np.array([2, 1, 0, 0], dtype=np.float32)
    want = O.preference_loss(logp, None, rw, lens, 1, 4, 1, loss="hinge", beta=0.5)
    loss, g, _, _ = run(L.make_preference("hinge", beta=0.5), to_device(logp), None, to_device(rw), to_device(lens), 1, 4, 1)
    assert np.isnan(float(loss))
    # of the five pairs three are NaN, one has h = 0.5 * (3 - 1), where the slope has ended, and one 0.5 * (2 - 1)
    assert want[1].tolist() == [-0.1, 0.0, 0.1, 0.0] and np.all(np.abs(np64(g) - want[1]) <= 1.01 * EPS * np.abs(want[1]))


def test_the_likelihood_is_counted_in_64_bits():
    """One response preferred to six at the same log-ratio: the factor 6 * 1.333483, rounded to fp32 on the way, is off by a whole half step,
    and what the loss then rounds to by another."""
    import paper_2603_04411_amd as L
    x, nll = float(np.float32(-1537.689208984375)), float(np.float32(1.333483))
    for T, G in ((1, 7), (1300, 7)):
        logp, lens = np.full(G * T, x, dtype=np.float32), np.ones(G, dtype=np.int32)
        rw = np.array([1] + [0] * (G - 1), dtype=np.float32)
        for weights in ("prompt", "pair"):
            loss, *_ = run(L.make_preference(nll_coef=nll, weights=weights), to_device(logp), None, to_device(rw), to_device(lens), 1, G, T)
            want = np.log(2.0) - nll * x
            # fp64 sums of a few terms are far below the one rounding to fp32
            assert abs(float(loss) - want) <= 1.01 * EPS * want


def check_each(P, G, T, seed, lens=None, **kw):
    """`check` of the logistic loss with a bound of its own for each output."""
    import paper_2603_04411_amd as L
    logp, ref, rw, lens = inputs(P, G, T, seed, lens)
    beta, nll, mean, per_pair = float(np.float32(kw["beta"])), float(np.float32(kw.get("nll_coef", 0.0))), kw.get("mean", False), kw.get("per_pair", False)
    q = L.make_preference(mean=mean, weights="pair" if per_pair else "prompt", beta=beta, nll_coef=nll)
    got = [np64(t) for t in run(q, to_device(logp), to_device(ref), to_device(rw), to_device(lens), P, G, T)]
    want = O.preference_loss(logp, ref, rw, lens, P, G, T, beta=beta, nll_coef=nll, mean=mean, per_pair=per_pair)
    n = np.clip(lens, 0, T)
    valid = np.arange(T)[None, :] < n[:, None]
    sizes = np.where(valid, np.abs(np.where(valid, logp.reshape(P * G, T), 0.0)) + np.abs(np.where(valid, ref.reshape(P * G, T), 0.0)), 0.0)
    per = np.where(n > 0, 1.0 / np.maximum(n, 1), 0.0)
    # a sum over a response: at most 64 additions one after the other on the way of each slot, half a step of what has been added each
    f64 = 2.0 ** -53
    off = 64 * f64 * sizes.sum(1) * (per if mean else 1.0)
    like = np.where(valid, np.abs(np.where(valid, logp.reshape(P * G, T), 0.0)), 0.0).sum(1) * per
    pairs = O.prompt_pairs(rw, P, G)
    weight = np.zeros(P * G)
    for a, b, m in pairs:
        w = 1.0 / len(pairs) if per_pair else 1.0 / (P * m)
        weight[a] += w
        weight[b] += w
    # the loss of a pair moves by beta for its log-ratio, its slope by beta^2 / 4; what is added up over up to 256 pairs one after the other
    # and with exp and log1p is off by as many half steps
    many = 512 * f64
    e_loss = 2 * beta * off.max() + many * (np.log(2.0) + beta * np.abs(want[2]).max() * 2 + nll * like.max())
    e_g = weight * (beta ** 2 / 4 * 2 * off.max() + many * beta) * (per if mean else 1.0) + weight * nll * many * per
    e_stats = np.array([0.0, beta * (off.max() + many * np.abs(want[2]).max()), beta * (off.max() + many * np.abs(want[2]).max()), 0.0])
    bounds = (e_loss, np.repeat(e_g, T), off + 4 * f64 * np.abs(want[2]), e_stats)
    for name, a, b, e in zip(("loss", "g_logp", "ratio", "stats"), got, want, bounds):
        assert np.all(np.abs(a.reshape(-1) - b) <= 1.01 * EPS * np.abs(b) + e + 2.0 ** -149), name
    # none of these bounds would let a wrong gradient through
    assert not pairs or np.abs(want[1]).max() > 1e3 * (e_g.max() + 2.0 ** -149)
    return len(pairs)


@pytest.mark.parametrize("P,G,T", [(2, 2, 32769), (1, 3, 100000), (1, 2, 2048 * 1024 + 5), (1, 4, 700001)])
@pytest.mark.parametrize("mean", [False, True])
def test_long_responses_each_output_by_itself(P, G, T, mean):
    for seed in (31, 32, 33):
        check_each(P, G, T, seed, mean=mean, beta=0.5 if mean else 1e-3, nll_coef=0.0 if seed == 31 else 0.1, per_pair=seed == 33)


# responses a wavefront each, the last workgroup not full, 161 and 162 workgroups; 160 and 161 responses a workgroup each
@pytest.mark.parametrize("P,G,T", [(55, 3, 7), (107, 6, 20), (215, 3, 20), (40, 4, 1025), (23, 7, 1025)])
def test_counts_and_launches_with_pairs_on_both_sides(P, G, T):
    for per_pair in (False, True):
        assert check_each(P, G, T, 41, beta=0.1, nll_coef=0.1, per_pair=per_pair) > P // 2
        check_each(P, G, T, 42, beta=0.5, mean=True, per_pair=per_pair)
