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
