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
