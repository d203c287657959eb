"""The activations between the FP8 layer's two products, one by one: fp8(silu(h1) h3) against 64 bits.

h1 and h3 are sums of a few terms, whole multiples of 2^-8 below 2^7, so they are exact in fp32; W2 is the identity and the gate 1,
so y is the activation as it was cast.  silu(h1) h3 is within 9 * 2^-24: the exponential counts for two
units of its last place (2^-22), the reciprocal for one (2^-23), and there is half a unit each in 1 + e and in two products.  An
element may go either way only where a border of its cast is nearer than that."""
import numpy as np
import pytest
import torch

from oracle import fp8_oracle as o
from paper_2403_07816_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TOL = 9 * 2.0 ** -24
T, d, F = 8192, 256, 256


def _values(rng, shape, low, high):
    """Random e4m3 values of either sign with exponents low .. high."""
    return (8 + rng.integers(0, 8, shape)) * np.exp2(rng.integers(low, high + 1, shape) - 3.0) * rng.choice([-1.0, 1.0], shape)


def _cast(a, blocks):
    """Values of a [T, F] at the scale of the largest magnitudes `blocks` [T, F / 128]."""
    s = np.exp2(np.ceil(np.log2(blocks / 448))).repeat(128, 1)
    return np.sign(a) * o.E4M3[o._nearest(np.minimum(np.abs(a) / s, 448.0))] * s


@pytest.mark.parametrize("low", [False, True], ids=["around-0", "far-below-0"])
@pytest.mark.parametrize("rows", [128, T])                     # tiles of one CTA, and of pairs
def test_activations_are_the_casts_of_their_values(rows, low):
    rng = np.random.default_rng(5)
    w1, w3 = _values(rng, (F, d), -2, 1 if not low else -1), _values(rng, (F, d), -2, 1)
    w1[:, 0], w3[:, 0] = -1.0, 0.0
    x = np.zeros((T, d))
    at = 1 + np.stack([rng.choice(d - 1, 2, replace=False) for _ in range(T)])
    np.put_along_axis(x, at, _values(rng, (T, 2), 0, 2 if not low else 1), 1)
    if low:                                                      # h1 around -16 .. -60, where silu is h1 e^h1
        x[:, 0] = np.abs(_values(rng, T, 4, 5))
    h1, h3 = x @ w1.T, x @ w3.T
    a = h1 / (1 + np.exp(-h1)) * h3
    top = np.abs(a).reshape(T, F // 128, 128).max(2)
    near = np.exp2(np.ceil(np.log2(top / 448)))
    assert (np.exp2(np.ceil(np.log2(top * (1 + TOL) / 448))) == near).all() and (np.exp2(np.ceil(np.log2(top * (1 - TOL) / 448))) == near).all()
    lo, hi = _cast(a * (1 - TOL), top), _cast(a * (1 + TOL), top)
    assert (lo != hi).mean() < 1e-3                           # the tolerance leaves next to nothing open

    f32 = lambda v: torch.tensor(v, dtype=torch.float32, device=DEV)
    w13, w2 = B.Fp8.empty(1, 2 * F, d, DEV), B.Fp8.empty(1, d, F, DEV)
    B.btx_fp8_quantize(f32(w1), w13, row_first=0, row_step=2)
    B.btx_fp8_quantize(f32(w3), w13, row_first=1, row_step=2)
    B.btx_fp8_quantize(torch.eye(F, device=DEV), w2)
    y = torch.empty(T, d, device=DEV)
    desc = B.make_fp8_moe_desc(rows, d, F, 1, 1, torch.float32)
    ws = torch.empty(B.btx_fp8_moe_workspace_size(desc), dtype=torch.uint8, device=DEV)
    idx, gates, xs = torch.zeros(rows, 1, dtype=torch.int32, device=DEV), torch.ones(rows, 1, device=DEV), f32(x)
    for t in range(0, T, rows):
        B.btx_fp8_moe_forward(desc, xs[t:t + rows], idx, gates, w13, w2, y[t:t + rows], ws)
    got = y.double().cpu().numpy()
    off = (got != lo) & (got != hi)
    assert not off.any(), (int(off.sum()), h1[off][:5], a[off][:5], got[off][:5])
