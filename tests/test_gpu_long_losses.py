"""The losses over one response of as many slots as a call takes, whose last block of 2048 slots ends where a 32-bit index does."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24
MOST = (1 << 31) - 1
PIECE = 1 << 28


def setup(T):
    import torch
    import paper_2603_04411_amd as L
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    lens = torch.tensor([T], dtype=torch.int32, device="cuda")
    ws = torch.empty(L.loss_workspace_bytes(1, 1, T), dtype=torch.uint8, device="cuda")
    return L, lens, ws, torch.full((1,), 7.0, device="cuda"), torch.full((T,), 7.0, device="cuda")


def filled(T, value, last):
    import torch
    x = torch.full((T,), value, device="cuda")
    x[-1] = last
    return x


def gradients(g, T):
    """The value that every slot but the last one has, and the last one's."""
    first = float(g[0])
    assert all(bool((g[lo:min(lo + PIECE, T - 1)] == first).all()) for lo in range(0, T - 1, PIECE))
    return first, float(g[T - 1])


@pytest.mark.parametrize("T", [MOST - 2046, MOST])
def test_cross_entropy(T):
    L, lens, ws, loss, g = setup(T)
    # the last slot is half of the loss.  Sums of a block and of 4096 of them are exact; some ten additions and a division after that
    L.ce_loss(filled(T, -0.5, -2.0 ** 30), lens, 1, T, loss, g, ws)
    want = (0.5 * (T - 1) + 2.0 ** 30) / T
    assert abs(float(loss) - want) <= 16 * EPS * want
    first, last = gradients(g, T)
    assert first == last and abs(first + 1 / T) <= 2 * EPS / T


@pytest.mark.parametrize("agg", [0, 1])
def test_clipped_surrogate(agg):
    import torch
    T = MOST
    L, lens, ws, loss, g = setup(T)
    stats = torch.full((4,), 7.0, device="cuda")
    # ratios of 1, and of e^21 in the last slot, which an advantage below 0 does not clip
    L.grpo_loss(filled(T, -0.5, -0.5), filled(T, -0.5, -21.5), None, torch.tensor([-1.0], device="cuda"), lens, 1, 1, T, 0.2, 0.2, 0.0, agg,
                loss, g, stats, ws)
    rho = math.exp(21.0)
    want = (T - 1 + rho) / T
    # 4096 blocks one after the other in each thread, some 20 additions around them
    assert abs(float(loss) - want) <= 4120 * EPS * want
    first, last = gradients(g, T)
    assert abs(first - 1 / T) <= 4 * EPS / T and abs(last - rho / T) <= 8 * EPS * rho / T
    assert float(stats[0]) == 0.0 and float(stats[3]) == float(np.float32(T))


def test_trajectory_balance():
    import torch
    T = MOST
    L, lens, ws, loss, g = setup(T)
    gz, resid = torch.full((1,), 7.0, device="cuda"), torch.full((1,), 7.0, device="cuda")
    L.flowrl_tb_loss(filled(T, -0.5, -2.0 ** 30), filled(T, -0.25, -2.0 ** 29), torch.tensor([2.0], device="cuda"), torch.tensor([3.0], device="cuda"),
                     lens, 1, 1, T, 0.5, loss, g, gz, resid, ws)
    a, c = (0.5 * (T - 1) + 2.0 ** 30) / T, (0.25 * (T - 1) + 2.0 ** 29) / T
    delta = 3.0 - a - 1.0 + c
    # sums of whole blocks are exact; a handful of roundings of numbers up to 3 after that
    assert abs(float(resid) - delta) <= 16 * EPS * 3 and abs(float(loss) - delta ** 2) <= 64 * EPS * 3
    assert abs(float(gz) - 2 * delta) <= 64 * EPS * 3
    first, last = gradients(g, T)
    assert first == last and abs(first - 2 * delta / T) <= 64 * EPS * 3 / T
