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


@pytest.mark.parametrize("T", [2, 8200], ids=["few", "many"])
@pytest.mark.parametrize("bar", [float("-inf"), float("nan")], ids=["-inf", "nan"])
def test_a_bias_that_bars_an_expert_leaves_its_score(bar, T):
    # values worked out by hand: the barred expert stays in the sum of the softmax, a logit of -inf does not
    z = torch.tensor([[1.0, 2.0, 3.0, 4.0]]).repeat(T, 1).to(DEV)
    b = torch.tensor([0.0, 0.0, 0.0, bar], device=DEV)
    e = np.exp([1.0, 2.0, 3.0, 4.0])
    sig = 1 / (1 + np.exp([-1.0, -2.0, -3.0, -4.0]))
    off = z.clone()
    off[:, 3] = float("-inf")
    for score, scores in ((0, e / e.sum()), (1, sig)):
        for renorm in (False, True):
            _, got = compare(z, 2, score, b, renorm=renorm, scale=1.5)
            w = 1.5 * scores[[2, 1]] / (scores[[2, 1]].sum() if renorm else 1)
            for t in (0, T - 1):
                assert got["topk_idx"][t].tolist() == [2, 1]
                np.testing.assert_allclose(got["scores"][t].cpu().numpy(), scores, rtol=2.0 ** -17)
                np.testing.assert_allclose(got["gates"][t].cpu().numpy(), w, rtol=2.0 ** -17)
    _, got = compare(off, 2, 0, None, renorm=False)
    np.testing.assert_allclose(got["scores"][0].cpu().numpy(), np.r_[e[:3] / e[:3].sum(), 0.0], rtol=2.0 ** -17)
    np.testing.assert_allclose(got["gates"][0].cpu().numpy(), (e / e[:3].sum())[[2, 1]], rtol=2.0 ** -17)
