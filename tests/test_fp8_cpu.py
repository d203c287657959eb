"""Host-side checks of the FP8 calls and of the norm: refusals before any CUDA call, and the 64-bit statements themselves."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import fp8_oracle as o
from paper_2403_07816_b200 import binding as B
from paper_2403_07816_b200 import build as builder


@pytest.fixture(scope="module")
def L():
    builder.build()
    return B.lib()


A = C.c_void_p(4096)
OFF = C.c_void_p(4104)                                  # 8-byte aligned
ODD = C.c_void_p(4097)
BIG = (1 << 31) - 32


def test_cast_refusals(L):
    sz = C.c_size_t(0)
    assert L.btx_fp8_sizes(2, 130, 513, C.byref(sz), None) == 0 and sz.value == 2 * 130 * 544
    assert L.btx_fp8_sizes(2, 130, 513, None, C.byref(sz)) == 0 and sz.value == 2 * 2 * 2 * 512
    for batch, rows, K, status in ((-1, 8, 64, 1), (1, -1, 64, 1), (1, 8, 0, 1), (1, BIG, 64, 2), (1, 8, BIG, 2), (1, 1 << 30, 1 << 30, 2),
                                   (1 << 30, 1 << 20, 1 << 19, 2)):
        assert L.btx_fp8_sizes(batch, rows, K, C.byref(sz), None) == status
    # dtype, src, row stride, batch stride, batch, rows, K, block rows, out rows, first, step, codes, scales, codes_t, scales_t
    ok = [0, A, 64, 512, 1, 8, 64, 1, 8, 0, 1, A, A, None, None]

    def q(**kw):
        names = "dtype src rs bs batch rows K block out_rows first step codes scales codes_t scales_t".split()
        args = list(ok)
        for k, v in kw.items():
            args[names.index(k)] = v
        return L.btx_fp8_quantize(*args, None)
    for bad in (dict(dtype=2), dict(src=None), dict(src=C.c_void_p(4098)), dict(dtype=1, src=ODD), dict(rs=-1), dict(bs=-1), dict(rows=-1),
                dict(K=0), dict(block=64), dict(block=0), dict(first=1), dict(first=-1), dict(step=0), dict(step=2), dict(codes=OFF),
                dict(scales=OFF), dict(scales=None), dict(codes=None), dict(codes=None, scales=None), dict(codes_t=A), dict(scales_t=A),
                dict(codes_t=OFF, scales_t=A)):
        assert q(**bad) == 1, bad
    assert q(out_rows=BIG) == 2 and q(K=BIG) == 2
    assert q(rows=0, src=None) == 0 and q(batch=0, src=None) == 0
    d = lambda *a: L.btx_fp8_dequantize(*a, None)
    assert d(0, A, A, 1, 8, 64, None) == 1 and d(3, A, A, 1, 8, 64, A) == 1 and d(0, A, A, 1, 8, 64, OFF) == 1
    assert d(0, None, None, 1, 0, 64, None) == 0 and d(0, A, A, 1, 8, BIG, A) == 2


def test_norm_refusals(L):
    mk = lambda T=4, d=64, dtype=torch.float32, eps=1e-5: C.byref(B.make_norm_desc(T, d, dtype, eps))
    sz = C.c_size_t(0)

    def f(desc=None, x=A, xs=64, r=None, rs=0, w=A, h=None, hs=0, y=A, ys=64, codes=None, scales=None):
        return L.btx_rms_norm(desc or mk(), x, xs, r, rs, w, h, hs, y, ys, codes, scales, None)

    def g(desc=None, h=A, hs=64, w=A, dy=A, dys=64, dh=None, dhs=0, dx=A, dxs=64, dw=A, acc=0, ws=A, n=1 << 40):
        return L.btx_rms_norm_backward(desc or mk(), h, hs, w, dy, dys, dh, dhs, dx, dxs, dw, acc, ws, n, None)
    for desc, status in ((mk(T=-1), 1), (mk(d=0), 1), (mk(dtype=3), 1), (mk(eps=-1.0), 1), (mk(eps=float("nan")), 1), (mk(eps=float("inf")), 1),
                         (mk(d=16385), 2), (mk(d=32769, dtype=torch.bfloat16), 2), (mk(T=BIG), 2)):
        assert f(desc=desc) == status and g(desc=desc) == status
        assert L.btx_rms_norm_backward_workspace_size(desc, C.byref(sz)) == status
    for bad in (dict(x=None), dict(y=None), dict(xs=63), dict(ys=63), dict(r=A, rs=63), dict(h=A, hs=63), dict(x=C.c_void_p(4098)),
                dict(w=C.c_void_p(4098)), dict(codes=A), dict(scales=A), dict(codes=OFF, scales=A), dict(y=None, codes=A), dict(xs=-64)):
        assert f(**bad) == 1, bad
    for bad in (dict(h=None), dict(dy=None), dict(dx=None), dict(hs=63), dict(dys=63), dict(dh=A, dhs=63), dict(dxs=63), dict(ws=None),
                dict(ws=OFF), dict(dw=C.c_void_p(4098)), dict(w=ODD)):
        assert g(**bad) == 1, bad
    assert L.btx_rms_norm_backward_workspace_size(mk(), C.byref(sz)) == 0 and g(n=sz.value - 1) == 3
    assert f(desc=mk(T=0), x=None, y=None) == 0
    assert g(desc=mk(T=0), h=None, dy=None, dx=None, dw=None) == 0 and g(desc=mk(T=0), h=None, dy=None, dx=None, acc=1) == 0
    assert L.btx_rms_norm_backward_workspace_size(mk(), None) == 1


def test_product_and_layer_refusals(L):
    sz = C.c_size_t(0)
    mm = lambda *a: L.btx_fp8_matmul(*a, None)
    assert mm(0, 1, 8, 8, 48, A, A, A, A, A, 0, A, 64) == 3
    for bad in ((2, 1, 8, 8, 64), (0, -1, 8, 8, 64), (0, 1, -1, 8, 64), (0, 1, 8, 0, 64), (0, 1, 8, 8, 0)):
        assert mm(*bad, A, A, A, A, A, 0, A, 256) == 1 and L.btx_fp8_matmul_workspace_size(*bad, C.byref(sz)) == 1
    for i in range(5):
        for wrong in (None, OFF):
            ptr = [A] * 5
            ptr[i] = wrong
            assert mm(0, 1, 8, 8, 64, *ptr, 0, A, 256) == 1
    assert mm(0, 1, 8, 8, 64, A, A, A, A, A, 0, None, 256) == 1 and mm(0, 1, 8, 8, 64, A, A, A, A, A, 0, OFF, 256) == 1
    assert mm(1, 1, 8, 8, 64, A, A, A, A, A, 1, A, 256) == 2                    # adding to bf16
    assert mm(0, 1, 1 << 30, 1 << 30, 64, A, A, A, A, A, 0, A, 256) == 2
    for M, N, K in ((BIG, 1, 32), (1, BIG, 32), (1, 1, BIG)):
        assert mm(0, 1, M, N, K, A, A, A, A, A, 0, A, 256) == 2
    assert mm(0, 1, 0, 8, 64, None, None, None, None, None, 0, None, 0) == 0
    mk = lambda T=4, d=64, f=96, E=4, k=2, dt=torch.float32: C.byref(B.make_fp8_moe_desc(T, d, f, E, k, dt))
    run = lambda desc, *ptr, n=1 << 40: L.btx_fp8_moe_forward(desc, *ptr, n, None)
    good = [A, None, A, A, A, A, A, A, A, A]
    for bad, status in ((mk(k=5), 1), (mk(d=24), 2), (mk(f=40), 2), (mk(E=513), 2), (mk(T=-1), 1), (mk(dt=9), 1), (mk(d=BIG + 16), 2),
                        (mk(d=16, f=1 << 30), 2), (mk(T=1 << 28), 2), (mk(d=1 << 20, f=1 << 20, E=1, k=1), 2)):
        assert L.btx_fp8_moe_workspace_size(bad, C.byref(sz)) == status and run(bad, *good) == status
    assert run(mk(), *good, n=16) == 3
    for i in range(10):
        for wrong in (None, C.c_void_p(4098)):
            ptr = list(good)
            ptr[i] = wrong
            if not (i == 1 and wrong is None):
                assert run(mk(), *ptr) == 1, i
    assert run(mk(T=0), *[None] * 10, n=0) == 0


# ---- the statements ----
@pytest.mark.parametrize("std", [1e-42, 1e-30, 0.02, 1.0, 3e37])
def test_cast_is_the_nearest_value_of_the_blocks_grid(std):
    x = (np.random.default_rng(1).normal(size=(130, 300)) * std).astype(np.float32).astype(np.float64)
    for rows in (1, 128):
        codes, scales = o.quantize(x, rows)
        v = o.values(codes, scales)
        assert np.array_equal(o.round_rows(v, rows), v)                       # its own values are left alone
        s = np.exp2(scales.astype(float) - 127).repeat(128, 1)[:, :300]
        for r in range(0, 130, rows):
            for b in range(3):
                at = np.s_[r:r + rows, b * 128:(b + 1) * 128]
                amax, sc = np.abs(x[at]).max(), s[at].max()
                assert s[at].min() == sc and amax <= 448 * sc and (sc == 2.0 ** -127 or amax > 224 * sc)
        p, q = np.abs(x) / s, np.abs(v) / s
        assert np.isin(q, o.E4M3).all() and ((v == 0) | (np.sign(v) == np.sign(x))).all()
        spacing = np.exp2(np.floor(np.log2(np.maximum(p, 2.0 ** -6))) - 3)
        assert (np.abs(p - q) <= spacing / 2).all()


def test_codes_are_torchs():
    v = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(v[:127], o.E4M3) and np.isnan(v[127]) and np.array_equal(v[128:255], -o.E4M3)
    p = np.abs(np.random.default_rng(2).normal(size=20000)) * 80
    p = np.concatenate([p[p <= 448], (o.E4M3[1:] + o.E4M3[:-1]) / 2])         # and every tie
    assert np.array_equal(o._nearest(p), torch.tensor(p, dtype=torch.float64).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_a_block_by_hand():
    # the largest of all 3.5 = 448 * 2^-7: scale 2^-7, byte 120; one unit more makes it 2^-6
    x = np.zeros((2, 128))
    x[0, :6] = [3.5, -1.0, 2.0 ** -7 * 17, 2.0 ** -7 * 19, 2.0 ** -17, 2.0 ** -17 * 1.5]      # 17 and 19 lie between 16, 18 and 20
    x[1, 0] = np.nextafter(np.float32(3.5), np.float32(4))
    codes, scales = o.quantize(x)
    assert scales.ravel().tolist() == [120, 121]
    assert (o.values(codes, scales)[0, :6] * 128).tolist() == [448, -128, 16, 20, 0, 2.0 ** -9]
    assert codes[0, 0] == 126 and codes[0, 1] == 128 + 14 * 8
    t = o.stored_scales(np.arange(130 * 5).reshape(130, 5).astype(np.uint8), 9)
    assert t.shape == (2, 2, 512) and t[1, 1, 16] == (129 * 5 + 4) % 256 and t[1, 1, 17] == 9 and t[0, 0, 3 * 16 + 4 + 2] == (35 * 5 + 2) % 256


def test_norm_gradient_matches_differences():
    r = np.random.default_rng(3)
    h, w, dy, dh = r.normal(size=(3, 7)), r.normal(size=7), r.normal(size=(3, 7)), r.normal(size=(3, 7))
    f = lambda hh, ww: (o.rms_norm(hh, ww, 1e-3) * dy).sum() + (hh * dh).sum()
    dx, dw = o.rms_norm_backward(h, w, dy, 1e-3, dh)
    e = 1e-6
    for i in range(3):
        for j in range(7):
            up, down = h.copy(), h.copy()
            up[i, j] += e
            down[i, j] -= e
            assert abs((f(up, w) - f(down, w)) / (2 * e) - dx[i, j]) < 1e-8    # truncation e^2, cancellation eps / e
    for j in range(7):
        up, down = w.copy(), w.copy()
        up[j] += e
        down[j] -= e
        assert abs((f(h, up) - f(h, down)) / (2 * e) - dw[j]) < 1e-8
