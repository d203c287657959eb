"""Host-side checks of the score routing and its 64-bit statement: refusals before any CUDA call, and the statement's
gradient against differences of its own weights."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import experts_oracle as o
from paper_2403_07816_b200 import binding as B
from paper_2403_07816_b200 import build as builder


@pytest.fixture(scope="module")
def L():
    builder.build()
    return B.lib()


A = C.c_void_p(4096)


def route_status(L, desc, stride=None, ptr=A):
    return L.btx_route(C.byref(desc), ptr, desc.E if stride is None else stride, None, None, A, A, None, None, None)


def test_route_refusals(L):
    mk = B.make_route_desc
    f = torch.float32
    for bad in [mk(-1, 8, 2, f), mk(4, 0, 1, f), mk(4, 8, 0, f), mk(4, 8, 9, f), mk(4, 8, 2, 5), mk(4, 8, 2, f, score=2),
                mk(4, 8, 2, f, n_group=3), mk(4, 8, 2, f, n_group=2, topk_group=3), mk(4, 8, 2, f, n_group=0),
                mk(4, 8, 5, f, n_group=2, topk_group=1), mk(4, 8, 2, f, group_score=2), mk(4, 8, 2, f, scale=0.0),
                mk(4, 8, 2, f, scale=float("nan")), mk(4, 8, 2, f, scale=float("inf"))]:
        assert route_status(L, bad) == 1
    for bad in [mk(4, 513, 2, f), mk(4, 512, 33, f), mk(4, 66, 1, f, n_group=33), mk(1 << 26, 512, 32, f)]:
        assert route_status(L, bad) == 2
    ok = mk(4, 8, 2, f)
    assert route_status(L, ok, stride=7) == 1                  # rows would overlap
    assert route_status(L, ok, ptr=C.c_void_p(4098)) == 1
    assert route_status(L, ok, ptr=None) == 1
    assert L.btx_route_backward(C.byref(ok), A, 8, A, None, A, 8, None) == 1
    assert L.btx_route_backward(C.byref(ok), A, 8, A, A, A, 7, None) == 1
    assert L.btx_route_backward(C.byref(mk(0, 8, 2, f)), None, 8, None, None, None, 8, None) == 0


@pytest.mark.parametrize("score", [o.SOFTMAX, o.SIGMOID])
@pytest.mark.parametrize("renorm", [True, False])
def test_statement_gradient_matches_differences(score, renorm):
    r = np.random.default_rng(4)
    z = r.normal(size=(3, 9))
    dw = r.normal(size=(3, 4))
    b = r.normal(size=9) * 0.1
    idx = o.route(z, 4, score, b, renorm=renorm, scale=1.5)[0]

    def weights(zz):
        # the weights of the fixed choice
        out = 0.0
        for t in range(3):
            s = o.scores_of_row(zz[t], score)[idx[t]]
            out += (1.5 * (s / s.sum() if renorm else s) * dw[t]).sum()
        return out
    got = o.route_backward(z, idx, dw, score, renorm, 1.5)
    h = 1e-6
    for t in range(3):
        for e in range(9):
            zp, zm = z.copy(), z.copy()
            zp[t, e] += h
            zm[t, e] -= h
            # central differences: truncation h^2, cancellation eps / h
            assert abs((weights(zp) - weights(zm)) / (2 * h) - got[t, e]) < 1e-8


def test_statement_route_properties():
    r = np.random.default_rng(5)
    z = r.normal(size=(20, 24))
    # top-k of the softmax is top-k of the logits; renormalised weights are the softmax over the chosen
    idx, w, s, counts = o.route(z, 3, o.SOFTMAX)
    assert np.array_equal(idx, np.argsort(-z, axis=1)[:, :3]) and np.allclose(w.sum(1), 1) and counts.sum() == 60
    # all groups staying is no grouping
    for gs in (o.GROUP_MAX, o.GROUP_SUM2):
        assert np.array_equal(o.route(z, 3, o.SIGMOID, n_group=4, topk_group=4, group_score=gs)[0], idx)
    # a bias that favours one expert puts it first and leaves its weight a score
    b = np.zeros(24)
    b[7] = 5.0
    i2, w2, s2, _ = o.route(z, 3, o.SIGMOID, b, renorm=False)
    assert (i2[:, 0] == 7).all() and np.allclose(w2[:, 0], s2[:, 7])


def test_mx4_and_given_refusals(L):
    sz = C.c_size_t(0)
    assert L.btx_mx4_sizes(1, 8, 48, C.byref(sz), None) == 2                     # K not a multiple of 32
    assert L.btx_mx4_sizes(-1, 8, 64, C.byref(sz), None) == 1
    assert L.btx_mx4_sizes(2, 130, 160, None, C.byref(sz)) == 0 and sz.value == 2 * 2 * 2 * 512
    q = lambda *a: L.btx_mx4_quantize(*a, None)
    assert q(0, A, 64, 512, 1, 8, 64, 8, 1, 1, A, A) == 1                         # last row outside
    assert q(0, A, 64, 512, 1, 8, 64, 8, 0, 0, A, A) == 1
    assert q(2, A, 64, 512, 1, 8, 64, 8, 0, 1, A, A) == 1
    assert q(0, C.c_void_p(4098), 64, 512, 1, 8, 64, 8, 0, 1, A, A) == 1
    assert q(0, A, 64, 512, 1, 8, 64, 8, 0, 1, C.c_void_p(4104), A) == 1
    assert q(0, None, 64, 512, 1, 0, 64, 0, 0, 1, None, None) == 0                # no rows: nothing to do
    mm = lambda *a: L.btx_mx4_matmul(*a, None)
    assert mm(0, 1, 8, 8, 48, A, A, A, A, A, A, 256) == 2
    assert mm(0, 1, 8, 0, 64, A, A, A, A, A, A, 256) == 1
    assert mm(0, 1, 8, 8, 64, A, A, A, A, A, A, 64) == 3
    assert mm(0, 1, 8, 8, 64, A, None, A, A, A, A, 256) == 1
    assert mm(0, 1, 1 << 30, 1 << 30, 64, A, A, A, A, A, A, 256) == 2
    assert mm(0, 1, 0, 8, 64, None, None, None, None, None, None, 0) == 0
    for bad, status in [(B.make_mx4_moe_desc(4, 64, 96, 4, 5, torch.float32), 1), (B.make_mx4_moe_desc(4, 48, 96, 4, 2, torch.float32), 2),
                        (B.make_mx4_moe_desc(4, 64, 80, 4, 2, torch.float32), 2), (B.make_mx4_moe_desc(4, 64, 96, 513, 2, torch.float32), 2),
                        (B.make_mx4_moe_desc(-1, 64, 96, 4, 2, torch.float32), 1), (B.make_mx4_moe_desc(4, 64, 96, 4, 2, 9), 1)]:
        assert L.btx_mx4_moe_workspace_size(C.byref(bad), C.byref(sz)) == status
        assert L.btx_mx4_moe_forward(C.byref(bad), A, A, A, A, A, A, A, A, A, 1 << 40, None) == status
    ok = B.make_mx4_moe_desc(4, 64, 96, 4, 2, torch.float32)
    assert L.btx_mx4_moe_forward(C.byref(ok), A, A, A, A, A, A, A, A, A, 16, None) == 3
    assert L.btx_mx4_moe_forward(C.byref(ok), A, None, A, A, A, A, A, A, A, 1 << 40, None) == 1
    # the caller's routing in the training layer
    mk = lambda alpha: B.make_desc(8, 64, 64, 4, 2, torch.float32, B.ROUTE_GIVEN, alpha, save_for_backward=True)
    with pytest.raises(B.BtxError) as ei:
        B.btx_moe_sizes(mk(0.01))                                                # no router, no loss
    assert ei.value.status == 2
    d = mk(0.0)
    assert L.btx_moe_forward(C.byref(d), A, None, None, None, A, A, A, A, None, A, A, 1 << 40, None) == 1
    r = B.RoutingOut(topk_idx=4096)
    assert L.btx_moe_forward(C.byref(d), A, None, None, None, A, A, A, A, C.byref(r), A, A, 1 << 40, None) == 1   # no gates
    assert L.btx_lb_loss(C.byref(d), A, None, A, A, A, None, A, 1 << 40, None) == 2
    assert L.btx_moe_step_host(C.byref(d), *([A] * 15), 1.0, *([A] * 5), 0, A, A, 1 << 40, None, None) == 2


def test_sizes_past_32_bit_arithmetic_are_refused(L):
    sz, big = C.c_size_t(0), (1 << 31) - 32
    assert L.btx_mx4_sizes(1, 1, 1 << 30, C.byref(sz), None) == 0 and sz.value == 1 << 29
    assert L.btx_mx4_sizes(1, 1, big, C.byref(sz), None) == 2
    assert L.btx_mx4_sizes(1, big, 32, C.byref(sz), None) == 2
    assert L.btx_mx4_quantize(0, A, 32, 32, 1, 1, 32, big, 0, 1, A, A, None) == 2
    for M, N, K in ((big, 1, 32), (1, big, 32), (1, 1, big)):
        assert L.btx_mx4_matmul(0, 1, M, N, K, A, A, A, A, A, A, 256, None) == 2
    for d, f in ((big, 32), (32, 1 << 30)):
        assert L.btx_mx4_moe_workspace_size(C.byref(B.make_mx4_moe_desc(1, d, f, 1, 1, torch.float32)), C.byref(sz)) == 2
    r = B.RoutingOut(topk_idx=4098, gates=4096)
    d = B.make_desc(8, 64, 64, 4, 2, torch.float32, B.ROUTE_GIVEN, 0.0)
    assert L.btx_moe_forward(C.byref(d), A, None, None, None, A, A, A, A, C.byref(r), None, A, 1 << 40, None) == 1


def test_statement_mx4_against_the_format():
    """The statement's cast: nearest value of the grid, ties to the even code, saturation, scale of the block."""
    x = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.9] + [0.0] * 24)
    assert o.mx4_round(x)[:8].tolist() == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0]
    r = np.random.default_rng(0).normal(size=(4, 64))
    v = o.mx4_round(r)
    assert np.array_equal(o.mx4_round(v * 1.0), v) or np.abs(v - r).max() < np.abs(r).max() / 3
    c, s = o.mx4_quantize(r)
    assert np.array_equal(o.mx4_values(c, s), v)
    t = o.mx4_tile_scales(s)
    assert t.shape == (1, 1, 512) and t[0, 0, 3 * 16 + 1] == s[3, 1]
