"""embed_fwd and embed_bwd against their oracle: types, strides, lengths, ids that are rare, frequent, repeated around the edges of the
pieces they are summed in, out of range; what is added to, what is left alone."""
import numpy as np
import pytest

from oracle import train_oracle as O
from tests.harness import np64, to_device

pytestmark = pytest.mark.gpu

EPS = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def types(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


def strided(n, d, ld, dtype, seed):
    """[n x d] with row stride ld, NaN between the rows; and the whole buffer."""
    import torch
    buf = torch.full((n * ld,), float("nan"), dtype=types(dtype), device="cuda")
    x = buf.as_strided((n, d), (ld, 1))
    x.copy_(torch.randn(n, d, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda"))
    return x, buf


def ids(V, N, seed, hot=True):
    r = np.random.default_rng(seed)
    return (np.minimum(r.zipf(1.2, N), V) - 1 if hot else r.integers(0, V, N)).astype(np.int32)


def forward(R, T, d, V, dtype, rows, tok, lens, scale, ldW=None, ldX=None, code=0):
    import torch
    import paper_2603_04411_amd as L
    desc = L.make_embed_desc(R, T, d, V, dtype, rows=rows, ldW=ldW, ldX=ldX)
    W, _ = strided(V, d, ldW or d, dtype, V + d)
    X, buf = strided(R * T, d, ldX or d, rows, 5)
    X.fill_(3.0)
    ws = torch.full((L.embed_workspace_bytes(desc),), 0xFF, dtype=torch.uint8, device="cuda")
    L.embed_fwd(desc, W, to_device(tok), None if lens is None else to_device(np.asarray(lens, dtype=np.int32)), scale, X, ws)
    assert L.lmhead_check(ws) == code
    want = O.embed_fwd(np64(W), tok, lens, R, T, float(np.float32(scale)))
    # the product in fp32, then the rows' type
    got = np64(X)
    assert np.all(np.abs(got - want) <= (EPS["f32"] + (EPS["bf16"] if rows == "bf16" else 0)) * 1.01 * np.abs(want))
    if ldX and ldX > d:
        gap = buf.view(R * T, ldX)[:, d:]
        assert bool(torch.isnan(gap).all()), "what lies between the rows was written"


@pytest.mark.parametrize("dtype,rows", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("R,T,d", [(1, 1, 8), (3, 5, 64), (2, 33, 1000), (1, 7, 520), (5, 1, 4096), (2, 3, 5128)])
def test_forward(dtype, rows, R, T, d):
    V = 97
    tok, lens = ids(V, R * T, R + d), np.random.default_rng(d).integers(0, T + 1, R)
    forward(R, T, d, V, dtype, rows, tok, lens, 1.0)
    forward(R, T, d, V, dtype, rows, tok, None, 45.25, ldW=d + 8, ldX=d + 16)
    # rows that begin 16 bytes apart from any larger power of two
    forward(R, T, d, V, dtype, rows, tok, lens, 3.0, ldW=d + (4 if dtype == "f32" else 8), ldX=d + (4 if rows == "f32" else 8))


def test_forward_of_many_rows():
    forward(7, 9001, 64, 5000, "bf16", "bf16", ids(5000, 63007, 1), [9001, 0, 1, 9000, 17, 4096, 8192], 8.0)
    forward(1, 70000, 8, 3, "f32", "bf16", ids(3, 70000, 2, hot=False), None, 0.5)


def test_forward_reports_what_is_out_of_range():
    tok = np.array([0, 5, -1, 4, 99, 3], dtype=np.int32)
    forward(2, 3, 16, 5, "bf16", "bf16", tok, [3, 3], 1.0, code=-6)
    forward(2, 3, 16, 5, "bf16", "bf16", np.array([0, 4, -1, 4, 99, 3], dtype=np.int32), [2, 1], 1.0)      # only on padding: no fault
    forward(2, 3, 16, 5, "f32", "f32", np.array([0, 1, 2, 4, 4, 3], dtype=np.int32), [4, -1], 1.0, code=-6)
    forward(2, 3, 16, 5, "f32", "f32", np.array([0, 1, 2, 4, 4, 3], dtype=np.int32), [3, 0], 1.0)


def test_rows_of_infinities_come_through():
    import torch
    import paper_2603_04411_amd as L
    W = torch.full((3, 8), float("inf"), device="cuda")
    W[1] = float("nan")
    W[2] = -0.0
    desc = L.make_embed_desc(1, 4, 8, 3, "f32")
    X, ws = torch.ones(4, 8, device="cuda"), torch.empty(L.embed_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    L.embed_fwd(desc, W, torch.tensor([0, 1, 2, 1], dtype=torch.int32, device="cuda"), torch.tensor([3], dtype=torch.int32, device="cuda"), 2.0, X, ws)
    assert bool((X[0] == float("inf")).all()) and bool(X[1].isnan().all()) and bool((X[2] == 0).all()) and bool((X[3] == 0).all())


def backward(R, T, d, V, rows, tok, lens, scale=1.5, ldX=None, add=False, code=0, g=None, ws=None):
    import torch
    import paper_2603_04411_amd as L
    desc = L.make_embed_desc(R, T, d, V, "bf16", rows=rows, ldX=ldX, flags=L.FLAG_ACCUM_DW if add else 0)
    if g is None:
        g, _ = strided(R * T, d, ldX or d, rows, N_SEED + R + T)
    dW = torch.randn(V, d, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    base = dW.clone()
    if ws is None:
        ws = torch.full((L.embed_workspace_bytes(desc),), 0xFF, dtype=torch.uint8, device="cuda")
    dt, dl = to_device(tok), None if lens is None else to_device(np.asarray(lens, dtype=np.int32))
    L.embed_bwd(desc, g, dt, dl, scale, dW, ws)
    assert L.lmhead_check(ws) == code
    ok = O.valid_slots(tok, lens, R, T, V)
    want, size = O.embed_bwd(np64(g), tok, lens, R, T, V, float(np.float32(scale)), np64(base) if add else None)
    count = np.bincount(np.asarray(tok)[ok], minlength=V)[:, None]
    # `count` - 1 additions, the scale, the addition to what was there: each off by half a step of at most the sum of magnitudes
    err = np.abs(np64(dW) - want)
    assert np.all(err <= 1.01 * (count + 1) * 2.0 ** -24 * size + 1e-40), float((err / np.maximum(size, 1e-30)).max())
    absent = torch.from_numpy(count[:, 0] == 0).cuda()
    assert torch.equal(dW[absent], base[absent] if add else torch.zeros_like(base[absent]))
    again = base.clone()
    L.embed_bwd(desc, g, dt, dl, scale, again, ws)
    assert torch.equal(again, dW), "not the same bits twice"
    return dW


N_SEED = 100


def backward_checked_by_torch(N, d, V, tok):
    """A batch for which the oracle's loop would take long: fp64 on the GPU by scattered additions of whole numbers, which are exact."""
    import torch
    import paper_2603_04411_amd as L
    g = torch.randint(-8, 9, (N, d), generator=torch.Generator(device="cuda").manual_seed(N), device="cuda").float()
    desc = L.make_embed_desc(1, N, d, V, "f32")
    dW, ws = torch.full((V, d), 7.0, device="cuda"), torch.full((L.embed_workspace_bytes(desc),), 0xFF, dtype=torch.uint8, device="cuda")
    dt = to_device(tok)
    L.embed_bwd(desc, g, dt, None, 1.0, dW, ws)
    assert L.lmhead_check(ws) == 0
    # sums stay below 2^24: exact in fp32 in any order
    want = torch.zeros(V, d, dtype=torch.float64, device="cuda").index_add_(0, dt.long(), g.double())
    assert torch.equal(dW.double(), want)


@pytest.mark.parametrize("rows", ["bf16", "f32"])
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("R,T,d,V", [(1, 1, 8, 1), (1, 1, 64, 300), (3, 5, 64, 7), (2, 33, 1000, 50), (4, 16, 520, 1), (1, 64, 256, 64),
                                     (1, 65, 512, 2), (2, 200, 136, 511), (2, 200, 136, 512), (2, 200, 136, 513), (3, 700, 72, 40)])
def test_backward(rows, add, R, T, d, V):
    backward(R, T, d, V, rows, ids(V, R * T, T), np.random.default_rng(V).integers(0, T + 1, R), add=add, ldX=d + 8 if add else None)
    backward(R, T, d, V, rows, ids(V, R * T, T + 1, hot=False), None, add=not add)


@pytest.mark.parametrize("piece", [1, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 192, 193, 255, 256, 257, 1000])
def test_ids_that_end_around_the_edges_of_the_pieces(piece):
    # id 0 moves the others off the edges, each id then has `piece` slots, the last one takes the rest
    for lead in (0, 1, 31, 63):
        tok = np.concatenate([np.zeros(lead, dtype=np.int32), 1 + np.arange(1800 - lead, dtype=np.int32) // piece])
        V = int(tok.max()) + 2
        perm = np.random.default_rng(piece).permutation(tok.size)
        backward(1, tok.size, 16, V, "f32" if lead else "bf16", tok[perm].astype(np.int32), None, add=lead == 1)


# rows of 16, 2104, 4104 and 5128 elements: pieces of 8, 16 and 32 slots; and, of many short rows, 64
EDGES = [1, 7, 8, 9, 15, 16, 17, 23, 24, 25, 31, 32, 33, 47, 48, 49, 63, 64, 65, 95, 96, 97, 127, 128, 129, 191, 192, 193, 1000]


@pytest.mark.parametrize("d,N,piece", [(16, 5003, p) for p in EDGES] + [
    (d, N, p) for d, N in ((2104, 5003), (4104, 7001), (5128, 13001)) for p in (1, 8, 9, 16, 17, 24, 25, 32, 33, 49, 65, 97, 1000)])
def test_sorted_ids_that_end_around_the_edges_of_the_pieces(d, N, piece):
    lead = piece % 5
    tok = np.concatenate([np.zeros(lead, dtype=np.int32), 1 + np.arange(N - lead, dtype=np.int32) // piece])
    perm = np.random.default_rng(piece).permutation(tok.size)
    backward(1, N, d, int(tok.max()) + 2, "f32" if piece % 2 else "bf16", tok[perm].astype(np.int32), None, add=piece % 3 == 0)


@pytest.mark.parametrize("piece", [1, 63, 64, 65, 127, 128, 129, 191, 192, 193, 511, 512, 513, 575, 576, 577, 640, 703, 1100, 4133, 70000, 600000])
def test_pieces_of_64(piece):
    N = 530003
    tok = (np.random.default_rng(piece).permutation(N) // piece).astype(np.int32)
    backward_checked_by_torch(N, 8, int(tok.max()) + 1, tok)


# more than one sorting tile, ids of one, two and three digits, one id everywhere
@pytest.mark.parametrize("R,T,V,hot", [(1, 4096, 400, True), (1, 4097, 400, True), (3, 4000, 200000, False), (2, 9000, 300000, True),
                                       (1, 12000, 1, False), (5, 3001, 2, False)])
def test_backward_of_many_rows(R, T, V, hot):
    lens = np.random.default_rng(R).integers(T // 2, T + 1, R)
    backward(R, T, 8, V, "bf16", ids(V, R * T, 9, hot), lens, add=True)
    backward(R, T, 24, V, "f32", ids(V, R * T, 9, hot), None)


# the most slots of each form and one more, the most ids whose tiles are sorted by themselves, zeros that ride along
@pytest.mark.parametrize("n,d,V,add", [(2047, 520, 900, False), (2048, 520, 900, True), (2049, 520, 900, True), (1254, 4096, 300, True),
                                       (1255, 4104, 300, False), (16384, 8, 3000, True), (16385, 8, 3000, True), (65536, 8, 700, False),
                                       (65537, 8, 700, True), (5000, 8, (1 << 22) - 2, True), (5000, 8, (1 << 22) - 1, False),
                                       (5000, 8, 1 << 22, True), (3000, 8, (8 << 20) + 1, False), (300, 8, (1 << 22) + 5, False)])
def test_the_edges_between_the_forms(n, d, V, add):
    import torch
    import paper_2603_04411_amd as L
    g = torch.randint(-8, 9, (n, d), generator=torch.Generator(device="cuda").manual_seed(n), device="cuda").to(torch.bfloat16)
    tok = (torch.rand(n, generator=torch.Generator(device="cuda").manual_seed(V), device="cuda", dtype=torch.float64) ** 6 * V).to(torch.int32)
    tok[0], tok[-1] = V - 1, 0
    desc = L.make_embed_desc(1, n, d, V, "bf16", flags=L.FLAG_ACCUM_DW if add else 0)
    dW = torch.full((V, d), 3.0, device="cuda")
    ws = torch.full((L.embed_workspace_bytes(desc),), 0xFF, dtype=torch.uint8, device="cuda")
    L.embed_bwd(desc, g, tok, None, 2.0, dW, ws)
    assert L.lmhead_check(ws) == 0
    # whole numbers below 2^24: exact in any order
    want = torch.full((V, d), 3.0 if add else 0.0, device="cuda").index_add_(0, tok.long(), 2 * g.float())
    assert torch.equal(dW, want)


def test_forward_in_256_bytes():
    import torch
    import paper_2603_04411_amd as L
    for n in (100, 5000):
        desc = L.make_embed_desc(1, n, 64, 30, "bf16")
        W, X = torch.randn(30, 64, device="cuda").bfloat16(), torch.empty(n, 64, dtype=torch.bfloat16, device="cuda")
        tok = torch.arange(n, device="cuda", dtype=torch.int32) % 30
        ws = torch.full((1024,), 0xFF, dtype=torch.uint8, device="cuda")
        L.embed_fwd(desc, W, tok, None, 1.0, X, ws[:256])
        assert L.lmhead_check(ws) == 0 and torch.equal(X, W[tok.long()]) and bool((ws[256:] == 0xFF).all())


def test_backward_of_nothing():
    for add in (False, True):
        backward(3, 50, 64, 20, "bf16", ids(20, 150, 1), [0, 0, 0], add=add)
        backward(1, 6000, 64, 20, "bf16", ids(20, 6000, 1), [0], add=add)


def test_backward_reports_what_is_out_of_range():
    tok = np.array([0, 5, -1, 4, 99, 3, -(1 << 31), (1 << 31) - 1], dtype=np.int32)
    for add in (False, True):
        backward(2, 4, 16, 5, "bf16", tok, [4, 4], add=add, code=-6)
        backward(2, 4, 16, 5, "bf16", tok, [1, 1], add=add, code=-6)      # the second response's only id is 99
        backward(2, 4, 16, 5, "bf16", tok, [1, 0], add=add)
        backward(2, 4, 16, 5, "bf16", np.abs(tok) % 5, [5, -3], add=add, code=-6)


BAD_IDS = [-1, 500, 501, (1 << 22) - 1, 1 << 22, (1 << 31) - 1, -(1 << 31)]       # of 500


def batch_with_faults(R, T, fault):
    """(ids, lengths, the code that the call leaves): faults at the first, the last and some other slot that counts, on padding alone, or in
    a length."""
    tok, lens, N = ids(500, R * T, R * T), np.full(R, T, dtype=np.int64), R * T
    if fault == "ids":
        tok[np.random.default_rng(N).permutation(N)[:len(BAD_IDS)]] = BAD_IDS
        tok[0], tok[-1] = BAD_IDS[0], BAD_IDS[1]
    elif fault == "first id":
        tok[0] = -1
    elif fault == "last id":
        tok[-1] = 500
    elif fault == "ids on padding":
        lens[:] = T - len(BAD_IDS)
        tok.reshape(R, T)[:, -len(BAD_IDS):] = BAD_IDS
    elif fault == "negative length":
        lens[-1] = -3
    elif fault == "long length":
        lens[0] = T + 1
    return tok, lens, 0 if fault in ("none", "ids on padding") else -6


FAULTS = ["ids", "first id", "last id", "ids on padding", "negative length", "long length"]


# without a sort, tiles sorted by themselves, by digits, by digits with a scan
@pytest.mark.parametrize("R,T", [(3, 300), (3, 1001), (3, 6700), (5, 14001)])
@pytest.mark.parametrize("add", [False, True])
def test_every_sort_reports_what_is_out_of_range(R, T, add):
    import torch
    import paper_2603_04411_amd as L
    d, V = 16, 500
    ws = torch.full((L.embed_workspace_bytes(L.make_embed_desc(R, T, d, V, "bf16")),), 0xFF, dtype=torch.uint8, device="cuda")
    for fault in FAULTS + ["none"]:      # each call starts with what the one before has left
        tok, lens, code = batch_with_faults(R, T, fault)
        backward(R, T, d, V, "bf16", tok, lens, add=add, code=code, ws=ws)


# the line where another workgroup reports what all have met
@pytest.mark.parametrize("R,T", [(4, 1024), (17, 241), (3, 20000)])
@pytest.mark.parametrize("d", [16, 2056])
def test_every_lookup_reports_what_is_out_of_range(R, T, d):
    import torch
    import paper_2603_04411_amd as L
    V = 500
    W = torch.randn(V, d, generator=torch.Generator(device="cuda").manual_seed(d), device="cuda").to(torch.bfloat16)
    desc, ws = L.make_embed_desc(R, T, d, V, "bf16"), torch.full((256,), 0xFF, dtype=torch.uint8, device="cuda")
    for fault in FAULTS + ["none"]:
        tok, lens, code = batch_with_faults(R, T, fault)
        X = torch.full((R * T, d), 3.0, dtype=torch.bfloat16, device="cuda")
        L.embed_fwd(desc, W, to_device(tok), to_device(lens.astype(np.int32)), 1.0, X, ws)
        assert L.lmhead_check(ws) == code, fault
        ok = torch.from_numpy(O.valid_slots(tok, lens, R, T, V)).cuda()
        rows = W[torch.from_numpy(np.where(ok.cpu(), tok, 0).astype(np.int64)).cuda()]
        assert torch.equal(X, torch.where(ok[:, None], rows, torch.zeros_like(rows))), fault


def test_padded_gradients_do_not_matter():
    import torch
    R, T, d, V = 3, 40, 64, 9
    lens = [40, 0, 11]
    g = torch.randn(R * T, d, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    pad = torch.tensor([i % T >= lens[i // T] for i in range(R * T)], device="cuda")
    clean = backward(R, T, d, V, "f32", ids(V, R * T, 4), lens, g=g.masked_fill(pad[:, None], 0.0))
    g[pad] = float("nan")
    import paper_2603_04411_amd as L
    desc = L.make_embed_desc(R, T, d, V, "f32")
    dW, ws = torch.empty(V, d, device="cuda"), torch.empty(L.embed_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    L.embed_bwd(desc, g, to_device(ids(V, R * T, 4)), torch.tensor(lens, dtype=torch.int32, device="cuda"), 1.5, dW, ws)
    assert torch.equal(dW, clean)


def test_a_workspace_of_a_larger_batch_serves():
    import torch
    import paper_2603_04411_amd as L
    big = L.make_embed_desc(9, 5000, 64, 700, "bf16")
    ws = torch.full((L.embed_workspace_bytes(big),), 0xFF, dtype=torch.uint8, device="cuda")
    for R, T, d, V in ((9, 5000, 64, 700), (1, 3, 64, 700), (2, 4100, 64, 700), (1, 300, 8, 5)):
        backward(R, T, d, V, "bf16", ids(V, R * T, T), None, add=T % 2 == 1, ws=ws)


def test_offsets_beyond_32_bits():
    import torch
    import paper_2603_04411_amd as L
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    # the last rows of a matrix and of a batch that are larger than 4 GiB (8.6 and 17.2 GB)
    V, d, N = 1 << 18, 8192, (1 << 18) + 3
    W = torch.zeros(V, d, device="cuda")
    W[-1] = torch.arange(d, device="cuda")
    desc = L.make_embed_desc(1, N, d, V, "f32", rows="f32")
    tok = torch.zeros(N, dtype=torch.int32, device="cuda")
    tok[-2:] = V - 1
    X = torch.full((N, d), 5.0, device="cuda")
    ws = torch.empty(L.embed_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    L.embed_fwd(desc, W, tok, None, 2.0, X, ws)
    assert L.lmhead_check(ws) == 0
    assert torch.equal(X[-1], 2 * W[-1]) and torch.equal(X[-2], 2 * W[-1]) and not bool(X[:-2].any())
    X[:-2] = 0
    X[1] = 1.0
    L.embed_bwd(desc, X, tok, None, 1.0, W, ws)
    assert L.lmhead_check(ws) == 0
    assert torch.equal(W[-1], 2 * X[-1]) and bool((W[0] == 1).all()) and not bool(W[1:-1].any())


def test_more_threads_than_one_row_of_workgroups():
    import torch
    import paper_2603_04411_amd as L
    if torch.cuda.mem_get_info()[0] < 160 << 30:
        pytest.skip("needs 160 GB")
    # rows that are filled up to 2048 columns: 2^33 threads' worth of them
    d, V, N = 1032, 50, (1 << 25) + 1000
    W = torch.randn(V, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    tok = torch.randint(0, V, (N,), dtype=torch.int32, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    X = torch.full((N, d), 5.0, device="cuda")
    ws = torch.empty(256, dtype=torch.uint8, device="cuda")
    L.embed_fwd(L.make_embed_desc(1, N, d, V, "f32"), W, tok, None, 1.0, X, ws)
    assert L.lmhead_check(ws) == 0
    for lo in range(0, N, 1 << 21):
        assert torch.equal(X[lo:lo + (1 << 21)], W[tok[lo:lo + (1 << 21)].long()]), lo
    del X
    # few slots and 2^30 ids of eight columns
    V, ids_ = (1 << 30) + 5, [0, (1 << 30) + 4, 1 << 29, 0]
    g = torch.randn(4, 8, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    dW = torch.full((V, 8), 7.0, device="cuda")
    desc = L.make_embed_desc(1, 4, 8, V, "f32")
    ws = torch.empty(L.embed_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    L.embed_bwd(desc, g, torch.tensor(ids_, dtype=torch.int32, device="cuda"), None, 1.0, dW, ws)
    assert L.lmhead_check(ws) == 0
    for v, row in ((0, g[0] + g[3]), ((1 << 30) + 4, g[1]), (1 << 29, g[2])):
        assert torch.equal(dW[v], row)
        dW[v] = 0.0
    assert all(not bool(dW[lo:lo + (1 << 26)].any()) for lo in range(0, V, 1 << 26))
