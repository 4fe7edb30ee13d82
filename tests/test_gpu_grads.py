"""grad_norm and grad_clip against their oracle: types, alignments, counts from one to more than a launch's table, empty tensors, values
whose squares overflow or vanish in fp32, what is written where nothing is clipped."""
import numpy as np
import pytest

from oracle import train_oracle as O
from tests.harness import np64

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24
HALF = {"f32": 0.0, "bf16": 2.0 ** -8}


def tensor(n, dtype, seed, scale=1.0, shift=0):
    """n values, `shift` elements behind an aligned address."""
    import torch
    t = torch.zeros(n + shift, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")[shift:]
    t.copy_(scale * torch.randn(n, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda"))
    return t


def workspace():
    import torch
    import paper_2603_04411_amd as L
    return torch.full((L.grad_workspace_bytes(),), 0xFF, dtype=torch.uint8, device="cuda")


def check(tensors, out_types, max_norm, eps=1e-6, shifts=None, in_place=False):
    import torch
    import paper_2603_04411_amd as L
    src = [np64(t) for t in tensors]
    n, c, want = O.grad_clip(src, float(np.float32(max_norm)), float(np.float32(eps)))
    norm = torch.full((2,), 7.0, device="cuda")
    grads = L.make_grad_list(tensors)
    L.grad_norm(grads, norm, workspace())
    # fp64 sums of up to 2^24 squares: far below one rounding to fp32
    assert abs(float(norm[0]) - n) <= 1.01 * EPS * n and float(norm[1]) == 7.0
    norm.fill_(7.0)
    if in_place:
        outs, out_list = tensors, None
    else:
        outs = [tensor(t.numel(), o, 0, 0.0, s) for t, o, s in zip(tensors, out_types, shifts or [0] * len(tensors))]
        for o in outs:
            o.fill_(9.0)
        out_list = L.make_grad_list(outs)
    L.grad_clip(grads, out_list, max_norm, eps, norm, workspace())
    assert abs(float(norm[0]) - n) <= 1.01 * EPS * n and abs(float(norm[1]) - c) <= 1.01 * EPS * c
    for i, (o, w) in enumerate(zip(outs, want)):
        kind = "bf16" if o.dtype == torch.bfloat16 else "f32"
        # c in fp32, the product in fp32, the output's type
        assert np.all(np.abs(np64(o) - w) <= 1.01 * (2 * EPS + HALF[kind]) * np.abs(w) + 1e-40), i
        if c == 1.0 and kind == ("bf16" if tensors[i].dtype == torch.bfloat16 else "f32"):
            assert np.array_equal(np64(o), src[i]), "not clipped, and still changed"
    if not in_place:
        assert all(np.array_equal(np64(t), s) for t, s in zip(tensors, src)), "the gradients were written"


SIZES = [1, 2, 3, 7, 8, 255, 256, 257, 1000, 8191, 8192, 8193, 16384 + 5, 100003]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("max_norm", [1.0, 1e9])
def test_types_and_sizes(kind, out, max_norm):
    ts = [tensor(n, kind, n) for n in SIZES]
    check(ts, [out] * len(ts), max_norm)
    check(ts[:1], [out], max_norm)
    if kind == out:
        check(ts, None, max_norm, in_place=True)


@pytest.mark.parametrize("shift", [1, 2, 3, 4, 5, 8])
def test_addresses_that_are_not_aligned(shift):
    ts = [tensor(n, k, n, shift=s) for n in (1, 9, 8192, 20001) for k in ("f32", "bf16") for s in (0, shift)]
    outs = ["bf16" if i % 3 else "f32" for i in range(len(ts))]
    check(ts, outs, 1.0, shifts=[shift * (i % 2) for i in range(len(ts))])
    check(ts, None, 1.0, in_place=True)


@pytest.mark.parametrize("count", [47, 48, 49, 95, 96, 97, 164, 165, 192, 193, 328, 329, 500])
def test_more_tensors_than_one_launch_takes(count):
    r = np.random.default_rng(count)
    ts = [tensor(int(n), "bf16" if i % 3 else "f32", i) for i, n in enumerate(np.exp(r.uniform(0, 9, count)).astype(int))]
    check(ts, ["f32" if i % 2 else "bf16" for i in range(count)], 0.5)
    check(ts, None, 2.0, in_place=True)


def test_as_many_tensors_as_a_call_takes():
    import torch
    import paper_2603_04411_amd as L
    sizes = [i % 6 for i in range(65536)]
    starts = np.concatenate([[0], np.cumsum(sizes)[:-1]]).tolist()
    buf = tensor(sum(sizes), "f32", 3)
    before = np64(buf)
    grads, norm = L.make_grad_list([buf[b:b + n] for b, n in zip(starts, sizes)]), torch.empty(2, device="cuda")
    L.grad_clip(grads, None, 1.0, 0.0, norm, workspace())
    n, c, want = O.grad_clip([before], 1.0, 0.0)
    assert abs(float(norm[0]) - n) <= 1.01 * EPS * n and abs(float(norm[1]) - c) <= 1.01 * EPS * c
    assert np.all(np.abs(np64(buf) - want[0]) <= 1.01 * 2 * EPS * np.abs(want[0]) + 1e-40)


def test_one_long_tensor_among_small_ones():
    check([tensor(5, "f32", 1), tensor((1 << 24) + 77, "f32", 2), tensor(0, "bf16", 3), tensor(3, "bf16", 4)], ["bf16"] * 4, 1.0)
    check([tensor((1 << 24) + 77, "bf16", 2), tensor(1, "f32", 1)], None, 1.0, in_place=True)


def ragged(total, count, unit, seed):
    """`count` sizes that take `total` pieces of `unit` elements in all; some are empty, some end with a piece, some in it."""
    r = np.random.default_rng(seed)
    pieces = np.zeros(count, dtype=np.int64)
    full = r.permutation(count)[:max(1, count - count // 8)]
    cuts = np.sort(r.choice(np.arange(1, total), len(full) - 1, replace=False)) if len(full) > 1 else np.array([], dtype=np.int64)
    pieces[full] = np.diff(np.concatenate([[0], cuts, [total]]))
    assert pieces.sum() == total
    return [0 if p == 0 else int(p) * unit - (0 if i % 3 == 0 else int(r.integers(0, unit))) for i, p in enumerate(pieces)]


def check_on_the_card(sizes, kinds, max_norm=1.0):
    """Norm and factor against fp64 sums, every element against the product in fp32 with the factor that was written."""
    import torch
    import paper_2603_04411_amd as L
    types = [torch.bfloat16 if k == "bf16" else torch.float32 for k in kinds]
    starts = np.concatenate([[0], np.cumsum([-(-n // 8) * 8 for n in sizes])]).tolist()
    bufs = {t: torch.randn(starts[-1], generator=torch.Generator(device="cuda").manual_seed(len(sizes)), device="cuda").to(t) for t in set(types)}
    ts = [bufs[t][b:b + n] for t, b, n in zip(types, starts, sizes)]
    # tensors weigh differently: a piece that is left out, or counted with another tensor, shows
    for i, t in enumerate(ts):
        t.mul_(2.0 ** (i % 5))
    n = float(torch.stack([t.double().square().sum() for t in ts]).sum().sqrt())
    c = min(1.0, float(np.float32(max_norm)) / n)
    norm = torch.full((2,), 7.0, device="cuda")
    grads = L.make_grad_list(ts)
    L.grad_norm(grads, norm, workspace())
    assert abs(float(norm[0]) - n) <= 1.01 * EPS * n and float(norm[1]) == 7.0
    outs = [torch.full_like(t, 9.0, dtype=torch.float32 if i % 2 else torch.bfloat16) for i, t in enumerate(ts)]
    for out in (outs, None):
        L.grad_clip(grads, None if out is None else L.make_grad_list(out), max_norm, 0.0, norm, workspace())
        assert abs(float(norm[0]) - n) <= 1.01 * EPS * n and abs(float(norm[1]) - c) <= 1.01 * EPS * c
        if out is not None:
            f = norm[1].clone()
            assert all(torch.equal(o, (t.float() * f).to(o.dtype)) for o, t in zip(out, ts))
            want = [(t.float() * f).to(t.dtype) for t in ts]
    assert all(torch.equal(t, w) for t, w in zip(ts, want))


# where the second pass stops adding up the partial sums itself, where a workgroup takes two pieces and then three; the table in the
# arguments and in the workspace
@pytest.mark.parametrize("count", [1, 90, 96, 97, 300])
@pytest.mark.parametrize("pieces", [511, 512, 513, 4095, 4096, 4097, 6145])
def test_where_the_passes_change(count, pieces):
    sizes = ragged(pieces, count, 8192, pieces + count)
    assert sum(-(-n // 8192) for n in sizes) == pieces
    check_on_the_card(sizes, ["bf16" if i % 3 else "f32" for i in range(count)])


# one workgroup takes up to 48 pieces of 2048 elements
@pytest.mark.parametrize("count", [1, 7, 48])
@pytest.mark.parametrize("pieces", [48, 49])
def test_where_one_workgroup_ends(count, pieces):
    sizes = ragged(pieces, count, 2048, pieces + count)
    assert sum(-(-n // 2048) for n in sizes) == pieces
    check_on_the_card(sizes, ["f32" if i % 3 else "bf16" for i in range(count)])


# sixteen pieces a workgroup, and more where the partial sums would be more than 16384
@pytest.mark.parametrize("pieces", [(1 << 15) - 1, 1 << 15, 1 << 18, (1 << 18) + 1])
def test_where_workgroups_take_sixteen_pieces_and_more(pieces):
    import torch
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    check_on_the_card(ragged(pieces, 60, 8192, pieces), ["bf16"] * 60)


def test_empty_tensors():
    import torch
    import paper_2603_04411_amd as L
    for ts in ([tensor(0, "f32", 1)], [tensor(0, "bf16", 1)] * 200):
        norm = torch.full((2,), 7.0, device="cuda")
        L.grad_clip(L.make_grad_list(ts), None, 1.0, 1e-6, norm, workspace())
        assert norm.tolist() == [0.0, 1.0]
        L.grad_norm(L.make_grad_list(ts), norm, workspace())
        assert float(norm[0]) == 0.0
    check([tensor(0, "f32", 1), tensor(9, "f32", 2), tensor(0, "bf16", 1)], ["f32"] * 3, 1.0)


def test_squares_that_do_not_fit_fp32():
    for scale in (1e30, 1e-30):
        check([tensor(1000, "f32", 1, scale), tensor(777, "bf16", 2, scale)], ["f32", "f32"], scale, eps=0.0)
        check([tensor(1000, "f32", 1, scale), tensor(777, "bf16", 2, scale)], None, scale, eps=0.0, in_place=True)


def test_zeros_and_values_that_are_no_numbers():
    import torch
    import paper_2603_04411_amd as L
    norm = torch.empty(2, device="cuda")

    def clip(t, max_norm=1.0, eps=1e-6):
        t = t.clone()
        L.grad_clip(L.make_grad_list([t]), None, max_norm, eps, norm, workspace())
        return t, norm.tolist()
    t, n = clip(torch.zeros(100, device="cuda"))
    assert n == [0.0, 1.0] and not bool(t.any())
    t, n = clip(torch.tensor([1.0, float("inf"), 0.0], device="cuda"))
    assert n == [float("inf"), 0.0] and t[0] == 0 and bool(t[1].isnan()) and t[2] == 0
    t, n = clip(torch.tensor([1.0, float("nan"), 0.0], device="cuda"))
    assert all(v != v for v in n) and bool(t.isnan().all())
    t, n = clip(torch.tensor([3.0, 4.0], device="cuda"), max_norm=0.0)
    assert n == [5.0, 0.0] and not bool(t.any())
    t, n = clip(torch.tensor([3.0, 4.0], device="cuda"), max_norm=float("inf"))
    assert n == [5.0, 1.0] and t.tolist() == [3.0, 4.0]


def test_what_lies_around_the_tensors_is_left_alone():
    import torch
    import paper_2603_04411_amd as L
    for n, at in ((13, 3), (8192, 8), (8193, 1), (20000, 5)):
        for dtype in (torch.float32, torch.bfloat16):
            buf = torch.full((n + 64,), 9.0, dtype=dtype, device="cuda")
            out = buf.clone()
            L.grad_clip(L.make_grad_list([buf[at:at + n]]), L.make_grad_list([out[at:at + n]]), 1.0, 0.0, torch.empty(2, device="cuda"), workspace())
            assert bool((out[:at] == 9).all()) and bool((out[at + n:] == 9).all()) and bool((buf == 9).all()) and bool((out[at:at + n] < 9).all())


def test_more_elements_than_one_row_of_workgroups():
    """2^35 elements and some: the scaling pass has more workgroups than a launch takes along one axis."""
    import torch
    import paper_2603_04411_amd as L
    n = (1 << 35) + 3 * 8192 + 5
    if torch.cuda.mem_get_info()[0] < 2 * n + (4 << 30):
        pytest.skip("64 GiB of device memory are not free")
    t = torch.empty(n, dtype=torch.bfloat16, device="cuda").zero_()
    at = [0, 8191, 8192, (1 << 34) + 1, (1 << 35) - 1, 1 << 35, (1 << 35) + 8192, n - 2, n - 1]
    for i in at:
        t[i] = 2.0
    norm = torch.empty(2, device="cuda")
    L.grad_clip(L.make_grad_list([t]), None, 3.0, 0.0, norm, workspace())
    assert norm.tolist() == [6.0, 0.5]
    for i in at:
        near = t[max(i - 2, 0):i + 3].tolist()
        assert near[min(i, 2)] == 1.0 and all(v in (0.0, 1.0) for v in near), i
    assert int(sum(int((t[lo:lo + (1 << 32)] != 0).sum()) for lo in range(0, n, 1 << 32))) == len(at)


def test_a_list_keeps_the_memory_that_it_was_made_with():
    import torch
    import paper_2603_04411_amd as L
    t = torch.full((1000,), 2.0, device="cuda")
    grads, norm = L.make_grad_list([t]), torch.empty(2, device="cuda")
    old = t.detach()
    t.data = torch.full((1000,), 5.0, device="cuda")
    assert grads.tensors[0].data_ptr() == old.data_ptr() and grads.array[0].data == old.data_ptr()
    L.grad_clip(grads, None, 1.0, 0.0, norm, workspace())
    assert bool((t == 5.0).all()) and bool((old < 2.0).all())


def test_a_list_refuses_memory_that_was_freed():
    import torch
    import paper_2603_04411_amd as L
    norm, ws = torch.empty(2, device="cuda"), workspace()
    for change in (lambda t: t.resize_(1 << 20), lambda t: t.untyped_storage().resize_(0)):
        keep, moved = tensor(1000, "f32", 1), tensor(2000, "bf16", 2)
        good, bad = L.make_grad_list([keep, keep.clone()]), L.make_grad_list([keep, moved])
        L.grad_clip(bad, None, 1.0, 0.0, norm, ws)
        change(moved)
        before = keep.clone()
        for call in (lambda: L.grad_norm(bad, norm, ws), lambda: L.grad_clip(bad, None, 0.5, 0.0, norm, ws),
                     lambda: L.grad_clip(good, bad, 0.5, 0.0, norm, ws)):
            with pytest.raises(ValueError, match="gradient 1"):
                call()
        assert torch.equal(keep, before)
        L.grad_clip(good, None, 0.5, 0.0, norm, ws)


def test_the_same_bits_each_time():
    import torch
    import paper_2603_04411_amd as L
    ts = [tensor(int(n), "f32", i) for i, n in enumerate((100003, 5, 8193, 77777))]
    grads, norm = L.make_grad_list(ts), torch.empty(2, device="cuda")
    outs = [torch.empty_like(t) for t in ts]
    first = None
    for _ in range(4):
        L.grad_clip(grads, L.make_grad_list(outs), 1.0, 1e-6, norm, workspace())
        got = [norm.clone()] + [o.clone() for o in outs]
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(got, first))


def test_the_binding_refuses_lists_that_do_not_fit():
    import torch
    import paper_2603_04411_amd as L
    a, norm, ws = tensor(64, "f32", 1), torch.empty(2, device="cuda"), workspace()
    for bad in (a.view(8, 8).t(), a.double(), a[::2]):
        with pytest.raises(ValueError):
            L.make_grad_list([bad])
    with pytest.raises(ValueError):
        L.grad_clip(L.make_grad_list([a]), L.make_grad_list([a, a]), 1.0, 0.0, norm, ws)
    with pytest.raises(ValueError):
        L.grad_clip(L.make_grad_list([a]), None, 1.0, 0.0, norm[:1], ws)
    with pytest.raises(L.LmheadError):
        L.grad_clip(L.make_grad_list([a[:40], a[39:]]), None, 1.0, 0.0, norm, ws)
    with pytest.raises(L.LmheadError):
        L.grad_norm(L.make_grad_list([]), norm, ws)
