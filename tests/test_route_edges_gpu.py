"""btx_route where its keys reach the ends of fp32, against the 64-bit statement in oracle/experts_oracle.py."""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as o
from paper_2403_07816_b200 import binding as B
from test_route_scored_gpu import compare

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("T", [3, 8200], ids=["few", "many"])
@pytest.mark.parametrize("score", [0, 1], ids=["softmax", "sigmoid"])
@pytest.mark.parametrize("sign", [-1.0, 1.0], ids=["low", "high"])
@pytest.mark.parametrize("E,G", [(64, 4), (60, 5)], ids=["groups of whole lanes", "other groups"])
def test_sums_of_two_keys_past_the_largest_float(E, G, sign, score, T):
    # The two best keys of every group are finite, their sum is not a finite fp32 number; biases as low as the type goes
    # mask experts in practice.  The groups' order is that of the exact sums.
    size = E // G
    b = torch.empty(E)
    for g, v in enumerate([3.0e38, 2.0e38, 2.5e38, 3.2e38, 2.9e38][:G]):
        b[g * size:(g + 1) * size] = sign * v * (1 - 1e-3 * torch.arange(size))       # (no two alike: fp32 orders a group's experts)
    lowest = torch.full((E,), torch.finfo(torch.float32).min)
    lowest[2 * size:2 * size + 1] = 0.0                     # one expert that is not masked
    lowest[3 * size:4 * size] = -2.0e38
    z = torch.randn(T, E, generator=torch.Generator().manual_seed(E)).to(DEV)
    for bias in (b, lowest):
        for tg in (1, 2):
            rows = [0, 1, 2] if T == 3 else [0, 1, 777, T - 1]
            desc = B.make_route_desc(T, E, 3, torch.float32, score, G, tg, B.GROUP_SUM2, True, 1.0)
            idx, gates = torch.empty(T, 3, dtype=torch.int32, device=DEV), torch.empty(T, 3, device=DEV)
            B.btx_route(desc, z, bias.to(DEV), idx, gates)
            want = o.route(z[rows].double().cpu().numpy(), 3, score, bias.double().numpy(), G, tg, o.GROUP_SUM2)
            assert np.array_equal(idx.cpu().numpy()[rows], want[0])


def test_keys_at_both_ends_of_the_type():
    # sums that are finite, infinite by a bias, or of one candidate, side by side
    z = torch.randn(9, 32, generator=torch.Generator().manual_seed(1)).to(DEV)
    b = torch.zeros(32)
    big = torch.finfo(torch.float32).max
    b[0:4], b[4:8], b[8:12], b[12:16] = big, -big, float("-inf"), 0.0
    b[16], b[17:20] = float("inf"), -big
    b[20:23], b[23] = float("-inf"), 1.0
    z[3, 24:28] = float("-inf")
    for tg in (1, 3, 7):
        compare(z, 3, 1, b.to(DEV), n_group=8, topk_group=tg, group_score=1)
