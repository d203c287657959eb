"""The gradient of score routing held to a bar of its own in every entry, against the 64-bit statement in
oracle/experts_oracle.py, and what that bar can see (a mistake planted in the statement, on the CPU).

Bar.  A score or weight is a quotient of exponentials: with |z - max| <= 20 each is within (20 + 2) 2^-24 of its value, a
sum of at most 512 adds 21 roundings, quotient and scale 2 more, so it is within (22 + 22 + 23) 2^-24 < 2^-17 = REL.  An
entry is a sum of products of dgates with one or two of them (and, for sigmoid, 1 - s, within 6 2^-24), added up in
at most 12 more roundings: each product is within 2 REL of its own size.  So the entry is within 2 REL of the sum of
the sizes of its products, for the chosen expert of slot j and, without renormalisation, for every expert e of a softmax

  softmax, renormalised   scale p_j (|dw_j| + sum_i p_i |dw_i|)
  sigmoid, renormalised   scale p_j (|dw_j| + sum_i p_i |dw_i|) (1 - s_j)
  softmax                 scale s_e (sum_j |dw_j| s_j) + scale s_j |dw_j|
  sigmoid                 scale |dw_j| s_j (1 - s_j)

over all slots that name the expert, plus half a step of the output type, relative to the entry."""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as o
from paper_2403_07816_b200 import binding as B

REL = 2.0 ** -17
CASES = [(0, True), (0, False), (1, True), (1, False)]


def bars(z, idx, dw, score, renorm, scale):
    """The sizes of the products behind every entry [T, E], times 2 REL."""
    out = np.zeros(z.shape)
    for t in range(len(z)):
        slots = [j for j in range(idx.shape[1]) if 0 <= idx[t, j] < z.shape[1]]
        if not slots:
            continue
        sel, w = idx[t, slots], scale * np.abs(dw[t, slots].astype(np.float64))
        s = o.scores_of_row(z[t], score)
        if renorm:
            p = o.chosen_weights(z[t][sel], score)
            v = p * (w + (p * w).sum())
        else:
            v = s[sel] * w
        if score == o.SIGMOID:
            v = v * o._sigmoid(-z[t][sel])
        np.add.at(out[t], sel, v)
        if score == o.SOFTMAX and not renorm:
            out[t] += s * (s[sel] * w).sum()
    return 2 * REL * out


def outside(got, want, bar, eps):
    """Entries that are further off than their bar (the last step rounds the computed value, not the exact one)."""
    return np.abs(got - want) > bar + eps / 2 * (np.abs(want) + bar) + 1e-40


@pytest.mark.parametrize("eps", [2.0 ** -23, 2.0 ** -7], ids=["f32", "bf16"])
@pytest.mark.parametrize("score,renorm", CASES)
def test_the_bar_sees_a_planted_mistake(score, renorm, eps):
    r = np.random.default_rng(3)
    T, E, k = 60, 256, 8
    z, dw = r.normal(size=(T, E)) * 1.28, r.normal(size=(T, k))
    idx = o.route(z, k, score, renorm=renorm)[0]
    want = o.route_backward(z, idx, dw, score, renorm, 1.75)
    bar = bars(z, idx, dw, score, renorm, 1.75)
    there = want != 0
    assert not outside(want, want, bar, eps).any()
    assert (outside(0 * want, want, bar, eps) == there).mean() > 0.999          # entries left out
    if eps < 2.0 ** -20:
        assert outside(1.01 * want, want, bar, eps)[there].mean() > 0.99        # all off by a hundredth
        # weights of another scale rule: every entry off by a ten-thousandth
        assert outside(1.0001 * want, want, bar, eps)[there].mean() > 0.7
    else:
        assert outside(1.01 * want, want, bar, eps)[there].mean() > 0.95        # (half a step of bf16 is 0.4 %)
    swapped = o.route_backward(z, idx, dw[:, ::-1], score, renorm, 1.75)
    assert outside(swapped, want, bar, eps)[there].mean() > 0.99


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("score,renorm", CASES)
@pytest.mark.parametrize("shape", [(1, 256, 8), (1, 1, 1), (300, 8, 2), (777, 165, 6), (130, 64, 2), (12, 32, 32), (40, 512, 32), (9, 511, 16),
                                   (8201, 40, 8), (8201, 64, 3), (8201, 128, 16), (8201, 250, 8), (8201, 256, 8),
                                   (20000, 512, 8)], ids=lambda s: "x".join(map(str, s)))
def test_gradient_within_its_bar(shape, score, renorm, dtype):
    # a warp walks over many rows of the large batches: masked experts, rows without a choice, the same expert twice
    T, E, k = shape
    dev = "cuda:0"
    z = (torch.randn(T, E, generator=torch.Generator().manual_seed(E + k)) * 1.28).to(dtype).to(dev)
    if E > 2 * k:
        z[17:5000:19, ::3] = float("-inf")
        z[23:5000:29, ::5] = float("nan")
    desc = B.make_route_desc(T, E, k, dtype, score, renorm=renorm, scale=1.75)
    idx, gates = torch.empty(T, k, dtype=torch.int32, device=dev), torch.empty(T, k, device=dev)
    B.btx_route(desc, z, None, idx, gates)
    idx[3::13] = -1
    idx[5::7, 0] = E
    if k > 1:
        idx[6::5, 1] = idx[6::5, 0]
    dw = torch.randn(T, k, generator=torch.Generator().manual_seed(9)).to(dev)
    dz = torch.full((T, E), 7.0, dtype=dtype, device=dev)
    B.btx_route_backward(desc, z, idx, dw, dz)
    rows = np.arange(T) if T <= 130 else np.r_[0:50, T // 2:T // 2 + 40, T - 40:T]
    z64, i, w = z[rows].double().cpu().numpy(), idx.cpu().numpy()[rows], dw.cpu().numpy()[rows]
    want = o.route_backward(z64, i, w, score, renorm, 1.75)
    bad = outside(dz.double().cpu().numpy()[rows], want, bars(z64, i, w, score, renorm, 1.75), torch.finfo(dtype).eps)
    assert not bad.any(), np.argwhere(bad)[:5]
