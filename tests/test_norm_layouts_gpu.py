"""The norm and its gradient where the tensors of a call differ in start and row stride, bit for bit against the same call on contiguous
tensors; the longest rows without a second tensor; and 1 / rms by itself."""
import numpy as np
import pytest
import torch

from paper_2403_07816_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
EPS = 1e-5


def randn(*shape, seed=0, dtype=F32):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


class Placed:
    """[T, d] with its first element `first` elements behind a 256-byte boundary and rows `d + more` apart, in a buffer of 7.0."""

    def __init__(self, T, d, first, more, dtype, data=None):
        self.buf = torch.full((first + T * (d + more) + 64,), 7.0, dtype=dtype, device=DEV)
        self.t = self.buf.as_strided((T, d), (d + more, 1), first)
        if data is not None:
            self.t.copy_(data)

    def nothing_beside(self):
        buf = self.buf.clone()
        buf.as_strided(self.t.shape, self.t.stride(), self.t.storage_offset()).fill_(7.0)
        return bool((buf == 7.0).all())


# (first, more) of x, residual or dh, h or dy, y or dx; in bf16 every parity of start and stride beside every other
PLACES = [((0, 0), (1, 1), (2, 0), (1, 0)), ((1, 1), (0, 0), (0, 1), (3, 1)), ((1, 0), (0, 1), (1, 1), (0, 0)), ((0, 1), (1, 0), (3, 2), (2, 3)),
          ((2, 4), (3, 4), (0, 2), (1, 6)), ((8, 5), (5, 8), (4, 7), (7, 4))]
SHAPES = [(70, 1), (70, 2), (66, 7), (40, 8), (90, 255), (61, 257), (300, 264), (37, 777), (20, 2051), (9, 4099), (5, 16397)]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("places", PLACES, ids=lambda p: "_".join(f"{a}+{b}" for a, b in p))
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_tensors_of_different_starts_and_strides(shape, places, dtype):
    T, d = shape
    if d * (2 if dtype == BF16 else 4) > 65536:
        T, d = 5, 12301                                                # fp32 rows have at most 16384 elements
    desc = B.make_norm_desc(T, d, dtype, EPS)
    x, r, w = randn(T, d, seed=1, dtype=dtype), randn(T, d, seed=2, dtype=dtype), randn(d, seed=3, dtype=dtype)
    h, y, q = torch.empty_like(x), torch.empty_like(x), B.Fp8.empty(1, T, d, DEV)
    B.btx_rms_norm(desc, x, w, residual=r, h=h, y=y, q=q)
    px, pr = Placed(T, d, *places[0], dtype, x), Placed(T, d, *places[1], dtype, r)
    ph, py, pq = Placed(T, d, *places[2], dtype), Placed(T, d, *places[3], dtype), B.Fp8.empty(1, T, d, DEV)
    wide = torch.empty(d + 4, dtype=dtype, device=DEV)
    wide[1:d + 1] = w
    B.btx_rms_norm(desc, px.t, wide[1:d + 1], residual=pr.t, h=ph.t, y=py.t, q=pq)
    assert torch.equal(ph.t, h) and torch.equal(py.t, y) and torch.equal(pq.codes, q.codes)
    assert all(p.nothing_beside() for p in (px, pr, ph, py))
    alone, palone = torch.empty_like(x), Placed(T, d, *places[3], dtype)
    B.btx_rms_norm(desc, x, w, y=alone)
    B.btx_rms_norm(desc, px.t, w, y=palone.t)
    assert torch.equal(palone.t, alone) and palone.nothing_beside()
    B.btx_rms_norm(desc, px.t, w, residual=pr.t, h=pr.t, y=py.t)        # in place
    assert torch.equal(pr.t, h) and torch.equal(py.t, y) and pr.nothing_beside()

    dy, dh = randn(T, d, seed=4, dtype=dtype), randn(T, d, seed=5, dtype=dtype)
    ws = torch.empty(B.btx_rms_norm_backward_workspace_size(desc), dtype=torch.uint8, device=DEV)
    for add in (dh, None):
        dx, dw = torch.empty_like(x), torch.empty(d, device=DEV)
        B.btx_rms_norm_backward(desc, x, w, dy, dx, dw, ws, dh=add)
        pdy, pdx, pdw = Placed(T, d, *places[2], dtype, dy), Placed(T, d, *places[3], dtype), torch.empty(d, device=DEV)
        pdh = None if add is None else Placed(T, d, *places[1], dtype, dh)
        B.btx_rms_norm_backward(desc, px.t, wide[1:d + 1], pdy.t, pdx.t, pdw, ws, dh=None if add is None else pdh.t)
        assert torch.equal(pdx.t, dx) and torch.equal(pdw, dw) and pdx.nothing_beside()
        for over in (pdy, px) if add is None else (pdy, pdh, px):
            kept = over.t.clone()
            B.btx_rms_norm_backward(desc, px.t, w, pdy.t, over.t, None, ws, dh=None if add is None else pdh.t)
            assert torch.equal(over.t, dx) and over.nothing_beside()
            over.t.copy_(kept)


@pytest.mark.parametrize("dtype,d", [(BF16, 32768), (BF16, 32761), (BF16, 32767), (F32, 16384), (F32, 16383)], ids=str)
def test_longest_rows_without_a_second_tensor(dtype, d):
    # h of a residual of zeros is x: the same bits, with one tensor fewer to read
    x, zero, w, dy = randn(6, d, seed=1, dtype=dtype), torch.zeros(6, d, dtype=dtype, device=DEV), randn(d, seed=2, dtype=dtype), randn(6, d, seed=3, dtype=dtype)
    desc = B.make_norm_desc(6, d, dtype, EPS)
    y, y2, h, q, q2 = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), B.Fp8.empty(1, 6, d, DEV), B.Fp8.empty(1, 6, d, DEV)
    B.btx_rms_norm(desc, x, w, y=y, q=q)
    B.btx_rms_norm(desc, x, w, residual=zero, h=h, y=y2, q=q2)
    assert torch.equal(y, y2) and torch.equal(h, x) and torch.equal(q.codes, q2.codes)
    v = x.double()
    want = v / torch.sqrt((v * v).mean(1, keepdim=True) + EPS) * w.double()
    assert bool(((y.double() - want).abs() <= (2.0 ** -19 + torch.finfo(dtype).eps / 2) * want.abs() + 1e-40).all())
    ws = torch.empty(B.btx_rms_norm_backward_workspace_size(desc), dtype=torch.uint8, device=DEV)
    dx, dx2, dw, dw2 = torch.empty_like(x), torch.empty_like(x), torch.empty(d, device=DEV), torch.empty(d, device=DEV)
    B.btx_rms_norm_backward(desc, x, w, dy, dx, dw, ws)
    B.btx_rms_norm_backward(desc, x, w, dy, dx2, dw2, ws, dh=zero)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)


@pytest.mark.parametrize("d", [64, 256, 4096, 16384])
def test_one_over_rms_is_within_half_a_unit(d):
    """Integers up to 8: their squares' sum is an integer below 2^24 and d a power of two, so the mean is exact in any order.  The
    first element is 1 and there are no weights, so the first of y is 1 / rms as the kernel has it.  A step of Newton's method
    leaves the square of the error that it starts from (under 2^-22) and one rounding."""
    T = 3000
    x = torch.randint(-8, 9, (T, d), generator=torch.Generator().manual_seed(d)).float()
    x[:, 0] = 1.0
    x[:, 1:] *= (torch.rand(T, 1, generator=torch.Generator().manual_seed(1)) > torch.rand(T, d - 1, generator=torch.Generator().manual_seed(2)))
    y = torch.empty(T, d, device=DEV)
    B.btx_rms_norm(B.make_norm_desc(T, d, F32, 0.0), x.to(DEV), None, y=y)
    want = 1 / np.sqrt((x.double().numpy() ** 2).mean(1))
    unit = np.exp2(np.floor(np.log2(want)) - 23)
    assert (np.abs(y[:, 0].double().cpu().numpy() - want) <= (0.5 + 2.0 ** -10) * unit).all()
