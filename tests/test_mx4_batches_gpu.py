"""btx_mx4_moe_forward and btx_mx4_matmul as batches change: the launches that stand in for the one-kernel form, and what a
row keeps of its bits when the rows around it are others."""
import numpy as np
import pytest
import torch

from paper_2403_07816_b200 import binding as B
from test_mx4_gpu import DEV, moe, moe_reference, np64, random_routing, randn

pytestmark = pytest.mark.gpu


def layer_inputs(T, d, F, E, k, dtype, empty=0.0, std=0.2):
    x = randn(T, d, seed=T, dtype=dtype)
    w = [randn(E, *s, seed=i, std=std) for i, s in enumerate([(F, d), (F, d), (d, F)])]
    return (x, *random_routing(T, E, k, T + E, empty), *w)


@pytest.fixture
def separate():
    B.btx_selftest_separate_launches(True)
    yield
    B.btx_selftest_separate_launches(False)


# batches that take the one kernel by themselves: one row, part of a tile, several tiles of an expert, many experts, the
# largest batch, a contraction of W2 that is shared by a cluster or by parts (F = 1056 and more)
SMALL = [(1, 128, 160, 4, 2, 0.0), (5, 64, 32, 3, 1, 0.0), (33, 96, 224, 4, 2, 0.3), (7, 32, 64, 512, 8, 0.0), (150, 256, 1056, 2, 2, 0.0),
         (40, 160, 96, 40, 6, 0.0), (256, 96, 2080, 9, 4, 0.1), (2, 320, 4128, 8, 1, 0.0), (64, 192, 1184, 3, 2, 1.1)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("layer", SMALL, ids=lambda s: "x".join(map(str, s)))
def test_separate_launches_of_small_batches(layer, dtype, separate):
    T, d, F, E, k, empty = layer
    x, idx, gates, *w = layer_inputs(T, d, F, E, k, dtype, empty)
    y, _ = moe(x, idx, gates, *w)
    rows = np.arange(T) if T <= 40 else np.r_[0:16, T // 2:T // 2 + 8, T - 16:T]
    want, tol = moe_reference(np64(x)[rows], idx.cpu().numpy()[rows], np64(gates)[rows], *map(np64, w))
    err = np.abs(np64(y)[rows] - want)
    assert (err <= tol + torch.finfo(dtype).eps / 2 * np.abs(want) + 1e-30).all(), (err - tol).max()


def test_the_switch_is_the_threads_own():
    import threading
    t = threading.Thread(target=lambda: B.btx_selftest_separate_launches(True))
    t.start()
    t.join()
    args = layer_inputs(6, 64, 96, 3, 2, torch.float32)
    here, _ = moe(*args)
    B.btx_selftest_separate_launches(True)
    try:
        there, _ = moe(*args)
    finally:
        B.btx_selftest_separate_launches(False)
    assert torch.equal(here, there)                        # one stage of F: nothing is split in either form


def test_a_row_among_others():
    # d = 1024: eight column tiles of W2, F = 2048: eight stages; one or two row tiles split them into 4 parts, five into 2,
    # ten into 1.  The parts' sums are fp32 and added in fp32: both orders are within (F/64 + 8) 2^-22 of the sum of
    # |w2| |a| from the exact sum of the same activations (an activation that 64 bits cast the other way changes that
    # size by less than a quarter), and each y is rounded once to fp32.
    d, F, E = 1024, 2048, 10
    w = [randn(E, *s, seed=i, std=0.05) for i, s in enumerate([(F, d), (F, d), (d, F)])]
    x = randn(200, d, seed=5)
    x[1:] = x[1:].roll(1, 0)
    gates = torch.full((200, 1), 0.75, device=DEV)

    def row0(T, experts):
        idx = (torch.arange(T, device=DEV, dtype=torch.int32) % experts)[:, None].contiguous()
        return moe(x[:T].contiguous(), idx, gates[:T].contiguous(), *w)[0][0]
    alone = row0(1, 1)
    assert torch.equal(row0(1, 1), alone)                                   # again
    assert torch.equal(row0(100, 1), alone) and torch.equal(row0(200, 1), alone) and torch.equal(row0(30, 2), alone)
    from oracle import experts_oracle as o
    xq, w1, w3, w2 = o.mx4_round(np64(x)[0]), *(o.mx4_round(np64(u)[0]) for u in w)
    h1, h3 = w1 @ xq, w3 @ xq
    size = 0.75 * np.abs(w2) @ np.abs(o.mx4_round(h1 / (1 + np.exp(-h1)) * h3))
    for T, experts in ((5, 5), (10, 10), (200, 10)):
        err = np.abs(np64(row0(T, experts)) - np64(alone))
        assert (err <= 2 * 1.25 * (F / 64 + 8) * 2.0 ** -22 * size + 2.0 ** -23 * np.abs(np64(alone))).all()


def test_a_row_of_a_product_among_others():
    # the contraction of one row tile is shared by eight CTAs, that of eight row tiles by two
    N, K = 1024, 4096
    x, wt = randn(1000, K, seed=1), randn(1, N, K, seed=2, std=0.02)
    wq = B.Mx4.empty(1, N, K, DEV)
    B.btx_mx4_quantize(wt, wq)
    ws = torch.empty(256, dtype=torch.uint8, device=DEV)

    def rows(M):
        q, y = B.Mx4.empty(1, M, K, DEV), torch.empty(M, N, device=DEV)
        B.btx_mx4_quantize(x[:M], q)
        B.btx_mx4_matmul(q, wq, y, ws)
        return y
    one = rows(1)
    assert torch.equal(rows(1), one) and torch.equal(rows(100)[:1], one)    # the same split
    from oracle import experts_oracle as o
    size = np.abs(o.mx4_round(np64(x[:1]))) @ np.abs(o.mx4_round(np64(wt)[0])).T
    err = np.abs(np64(rows(1000)[:1]) - np64(one))
    assert (err <= 2 * (K / 64 + 4) * 2.0 ** -22 * size + 2.0 ** -23 * np.abs(np64(one))).all()
