"""The norm and its gradients where h, the weights or dy are far from 1: no product on the way leaves fp32 where the result does not.

Tolerances are those of the norm's other tests, 2^-19 of y (u = 2^-24: 26 u of 1 / rms, two roundings), 2^-16.9 of the sizes of dx's
terms and 2^-15.4 of dw's, and the last rounding, which below the type's smallest normal number is half of its smallest step."""
import numpy as np
import pytest
import torch

from oracle import fp8_oracle as o
from paper_2403_07816_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
both = pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])


def randn(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(DEV)


def np64(t):
    return t.double().cpu().numpy()


def half(dtype):
    return torch.finfo(dtype).eps / 2


def half_step(dtype):
    return torch.finfo(dtype).smallest_normal * half(dtype)


def rows_of(T, d, exps, dtype):
    """Rows of rms about 2^e, e of exps in turn."""
    e = torch.tensor([exps[t % len(exps)] for t in range(T)], device=DEV, dtype=F32)
    return (randn(T, d, seed=1) * torch.exp2(e)[:, None]).to(dtype)


@both
@pytest.mark.parametrize("spread", [False, True], ids=["alike", "one-apart"])
@pytest.mark.parametrize("e", [-125, -110, -60, 60, 110, 117])
def test_weights_far_from_one(e, spread, dtype):
    T, d = 33, 264                                                     # |h| / rms is below 2^5, so y is below 2^125
    x = rows_of(T, d, [-55, -29, -20, -1, 0, 20, 29, 31, 55], dtype)
    w = randn(d, seed=2).abs() + 0.5
    w = w * 2.0 ** e if not spread else torch.where(torch.arange(d, device=DEV) % 131 == 7, w * 2.0 ** e, w)
    w = w.to(dtype)
    y, q = torch.empty_like(x), B.Fp8.empty(1, T, d, DEV)
    B.btx_rms_norm(B.make_norm_desc(T, d, dtype, 0.0), x, w, y=y, q=q)
    want = o.rms_norm(np64(x), np64(w), 0.0)
    assert (np.abs(np64(y) - want) <= (half(dtype) + 2.0 ** -19) * np.abs(want) + half_step(dtype)).all()
    v = torch.empty(T, d, device=DEV)
    B.btx_fp8_dequantize(q, v)
    top = np.pad(np.abs(want), ((0, 0), (0, -d % 128))).reshape(T, -1, 128).max(2).repeat(128, 1)[:, :d]
    # half a step of e4m3, at least 2^-10 of a scale that is at most 2^-7.8 of the block's largest or 2^-127
    assert (np.abs(np64(v) - want) <= (2.0 ** -4 + 2.0 ** -18) * np.abs(want) + 2.0 ** -17.8 * top + 2.0 ** -136).all()


@both
def test_rows_without_a_number_under_large_weights(dtype):
    x = randn(6, 40, seed=3).to(dtype)
    x[1, 3], x[2], x[3, 5] = float("nan"), 0.0, float("inf")
    x[4] = 1e30                                                        # its sum of squares is infinite: y is 0
    w = torch.full((40,), 2.0 ** 100, device=DEV, dtype=dtype)
    y = torch.empty_like(x)
    B.btx_rms_norm(B.make_norm_desc(6, 40, dtype, 0.0), x, w, y=y)
    assert bool(y[1].isnan().all()) and bool(y[2].isnan().all()) and bool(y[3, 5].isnan()) and bool((y[4] == 0).all())
    assert bool((y[3, :5] == 0).all()) and bool(y[[0, 5]].isfinite().all())


@both
@pytest.mark.parametrize("d", [40, 264, 2051])                          # rows of one warp and of several, on and off 16-byte boundaries
@pytest.mark.parametrize("e,grad", [(110, 1.0), (-110, 1.0), (0, 2.0 ** -100), (0, 1.0), (60, 2.0 ** 40), (117, 0.0)])
def test_gradient_far_from_one(e, grad, d, dtype):
    T, exps = 27, [-35, -29, -20, -1, 0, 20, 29, 31, 35]
    x = rows_of(T, d, exps, dtype)
    w = ((randn(d, seed=2).abs() + 0.5) * 2.0 ** e).to(dtype)
    dy = (randn(T, d, seed=3) + x.float() / x.float().square().mean(1, keepdim=True).sqrt()).mul(grad).to(dtype)     # a part of it along h
    desc = B.make_norm_desc(T, d, dtype, 0.0)
    ws = torch.empty(B.btx_rms_norm_backward_workspace_size(desc), dtype=torch.uint8, device=DEV)
    dx, dw = torch.empty_like(x), torch.empty(d, device=DEV)
    B.btx_rms_norm_backward(desc, x, w, dy, dx, dw, ws)
    h, g = np64(x), np64(dy) * np64(w)
    want_x, want_w = o.rms_norm_backward(h, np64(w), np64(dy), 0.0)
    s = 1 / np.sqrt((h * h).mean(1, keepdims=True))
    size = s * np.abs(g) + np.abs(h) * s ** 3 * np.abs(g * h).mean(1, keepdims=True)
    # g, m and what they are multiplied with are off by half a step of fp32's subnormal numbers at most, times s; dx beyond the type is infinite
    tol = 2.0 ** -16.9 * size + (half(dtype) + 2.0 ** -24) * np.abs(want_x) + half_step(dtype) + 2.0 ** -144 * s
    fits = np.abs(want_x) + tol < torch.finfo(dtype).max
    assert fits.mean() > 0.5
    err = np.abs(np64(dx) - want_x)
    assert (err[fits] <= tol[fits]).all()
    assert (np.abs(np64(dw) - want_w) <= 2.0 ** -15.4 * np.abs(np64(dy) * h * s).sum(0) + 2.0 ** -140).all()


@both
def test_gradient_of_a_row_whose_sum_of_squares_is_infinite(dtype):
    # its y is 0 whatever h is, so it hands on dh alone, and dw has nothing of it
    x = randn(5, 264, seed=1).to(dtype)
    dy, dh = randn(5, 264, seed=2).to(dtype), randn(5, 264, seed=3).to(dtype)
    desc = B.make_norm_desc(5, 264, dtype, 1e-5)
    ws = torch.empty(B.btx_rms_norm_backward_workspace_size(desc), dtype=torch.uint8, device=DEV)
    outs = []
    for large in (False, True):
        if large:
            x[2] = (x[2].float() * 1e30).to(dtype)
            dy[2] = (dy[2].float() * 1e12).to(dtype)
        dx, dw = torch.empty_like(x), torch.empty(264, device=DEV)
        rows = [0, 1, 3, 4]
        B.btx_rms_norm_backward(desc, x, None, dy, dx, dw, ws, dh=dh)
        outs.append(dx[rows].clone())
    want = o.rms_norm_backward(np64(x)[rows], 1.0, np64(dy)[rows], 1e-5)[1]
    s = 1 / np.sqrt((np64(x)[rows] ** 2).mean(1, keepdims=True) + 1e-5)
    assert torch.equal(dx[2], dh[2]) and torch.equal(*outs)
    assert (np.abs(np64(dw) - want) <= 2.0 ** -15.4 * np.abs(np64(dy)[rows] * np64(x)[rows] * s).sum(0)).all()
