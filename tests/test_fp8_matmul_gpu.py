"""Products of FP8 matrices, and a linear layer's gradients by them, against the products of their values in 64 bits.

Every term a b 2^s is exact in fp32 (eight significant bits).  An MMA adds 32 terms to the running sum with at most one unit of
rounding (2^-23 of sum |a b|, which bounds every partial sum) and loses at most as much in aligning its terms, so an output is
within (K/32 + 4) 2^-22 sum |a b| of the exact sum, plus half a step of the output type."""
import pytest
import torch

from paper_2403_07816_b200 import binding as B
from util import Guarded, check_guards

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
both = pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])


def randn(*shape, seed=0, std=1.0, dtype=F32):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype).to(DEV)


def guarded_fp8(batch, rows, K, fill=0xFF):
    """Unwritten scale bytes read as NaN."""
    bufs = {"codes": Guarded((batch, rows, (K + 31) // 32 * 32), torch.uint8, DEV, fill=fill),
            "scales": Guarded((batch, (rows + 127) // 128, (K + 511) // 512, 512), torch.uint8, DEV, fill=fill)}
    return B.Fp8(bufs["codes"].t, bufs["scales"].t, K), bufs


def cast(x, block=1, transposed=False):
    x = x if x.dim() == 3 else x[None]
    batch, rows, K = x.shape
    q, bufs = guarded_fp8(batch, *((K, rows) if transposed else (rows, K)))
    B.btx_fp8_quantize(x, None if transposed else q, block_rows=block, out_t=q if transposed else None)
    return q, bufs


def values64(q):
    v = torch.empty(q.shape, dtype=F32, device=DEV)
    B.btx_fp8_dequantize(q, v)
    return v.double()


def product(qa, qb, dtype, old=None):
    batch, M, K = qa.shape
    N = qb.shape[1]
    y = Guarded((batch, M, N), dtype, DEV)
    if old is not None:
        y.t.copy_(old)
    ws = Guarded(B.btx_fp8_matmul_workspace_size(M, N, K, dtype, batch), torch.uint8, DEV, fill=0x7F)
    B.btx_fp8_matmul(qa, qb, y.t, ws.t, accumulate=old is not None)
    assert B.btx_device_status(ws.t) == B.BTX_OK
    check_guards({"y": y, "workspace": ws}, "btx_fp8_matmul")
    return y.t


def check_product(y, qa, qb, old=None):
    va, vb = values64(qa), values64(qb)
    want = va @ vb.transpose(1, 2)
    size = va.abs() @ vb.abs().transpose(1, 2)
    if old is not None:
        want, size = want + old.double(), size + old.double().abs()
    tol = (qa.shape[2] / 32 + 4) * 2.0 ** -22 * size + torch.finfo(y.dtype).eps / 2 * want.abs()
    err = (y.double() - want).abs()
    assert bool((err <= tol).all()), float((err - tol).max())


SHAPES = [(1, 1, 1, 1), (1, 1, 128, 64), (1, 128, 128, 128), (1, 5, 200, 96), (1, 129, 255, 161), (1, 300, 64, 1056), (2, 130, 136, 288),
          (3, 1, 1000, 513), (1, 1000, 17, 2048), (1, 64, 4096, 4096), (1, 520, 2056, 545), (1, 33, 130, 7), (1, 2100, 2300, 321),
          (3, 1100, 1300, 96), (1, 4100, 1290, 2081), (1, 1500, 3331, 128), (1, 1500, 3334, 128), (1, 16, 512, 11008), (5, 40, 48, 640)]


@both
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_product(shape, dtype):
    batch, M, N, K = shape
    qa, ba = cast(randn(batch, M, K, seed=M + K))
    qb, bb = cast(randn(batch, N, K, seed=N + K + 1, std=0.02), 128 if (M + N) % 2 else 1)
    y = product(qa, qb, dtype)
    check_guards({"a": ba["codes"], "b": bb["codes"], "sa": ba["scales"], "sb": bb["scales"]}, "btx_fp8_matmul")
    check_product(y, qa, qb)
    assert torch.equal(product(qa, qb, dtype), y)                       # repeats
    if dtype == F32:
        old = randn(batch, M, N, seed=9)
        check_product(product(qa, qb, dtype, old), qa, qb, old)


def test_product_is_exact_on_single_terms():
    # one element of A per row: y is a column of B times it, at every position of the contraction and every scale
    K = 1100
    a = torch.zeros(1, K, K, device=DEV)
    a[0].fill_diagonal_(1.5)
    g = torch.Generator().manual_seed(2)
    b = (torch.randn(1, 40, K, generator=g) * torch.exp2(torch.randint(-8, 8, (1, 40, 9), generator=g).float()).repeat_interleave(128, 2)[..., :K]).to(DEV)
    qa, qb = cast(a)[0], cast(b)[0]
    assert torch.equal(product(qa, qb, F32)[0].double(), (1.5 * values64(qb)[0]).t())
    assert torch.equal(product(qb, qa, F32)[0].double(), 1.5 * values64(qb)[0])


@pytest.mark.parametrize("rows", [1, 40, 1100])
def test_accumulation_keeps_the_small_terms(rows):
    # one large term at the head of each row, then many small ones that a sum of few bits would lose
    K = 4096
    a, b = torch.full((1, rows, K), 1.0, device=DEV), torch.full((1, 600, K), 2.0 ** -9, device=DEV)
    a[..., 0] = 256.0
    b[..., 0] = 1.0
    y = product(cast(a)[0], cast(b)[0], F32)
    want = 256.0 + (K - 1) * 2.0 ** -9                                  # whole multiples of 2^-9 below 2^9: exact in fp32
    assert bool(((y - want).abs() <= (K / 32 + 4) * 2.0 ** -22 * want).all()), float((y - want).abs().max())


def test_scales_of_extreme_size_and_nan_blocks():
    a = randn(1, 40, 300, seed=5)
    a[0, 3] *= 2.0 ** 90
    a[0, 4] *= 2.0 ** -90
    b = randn(1, 70, 300, seed=6)
    b[0, 7, 140] = float("nan")
    b[0, 9] *= 2.0 ** -60
    qa, qb = cast(a)[0], cast(b)[0]
    y = product(qa, qb, F32)
    assert bool(y[0, :, 7].isnan().all())
    keep = [i for i in range(70) if i != 7]
    va, vb = values64(qa)[0], values64(qb)[0][keep]
    err = (y[0][:, keep].double() - va @ vb.t()).abs()
    # sums below 2^-126, the smallest normal fp32 number, hold no relative accuracy (and may be flushed to zero)
    assert bool((err <= 14 * 2.0 ** -22 * (va.abs() @ vb.abs().t()) + 2.0 ** -126).all())


@both
@pytest.mark.parametrize("shape", [(1, 16, 16), (40, 130, 257), (777, 520, 1040), (2049, 2060, 1030)], ids=lambda s: "x".join(map(str, s)))
def test_linear_layer_and_its_gradients(shape, dtype):
    """y = x W^T, dx = dy W, dW = dy^T x: each is the product of the casts' values, and dW adds up over micro-batches."""
    M, N, K = shape
    x, w, dy = randn(M, K, seed=1, dtype=dtype), randn(N, K, seed=2, std=0.05, dtype=dtype), randn(M, N, seed=3, std=0.1, dtype=dtype)
    wq, wt = B.Fp8.empty(1, N, K, DEV), B.Fp8.empty(1, K, N, DEV)
    B.btx_fp8_quantize(w, wq, block_rows=128, out_t=wt)
    assert torch.equal(values64(wq).transpose(1, 2), values64(wt))
    check_product(product(cast(x)[0], wq, dtype), cast(x)[0], wq)
    gq, gt, xt = B.Fp8.empty(1, M, N, DEV), B.Fp8.empty(1, N, M, DEV), B.Fp8.empty(1, K, M, DEV)
    B.btx_fp8_quantize(dy, gq, out_t=gt)
    B.btx_fp8_quantize(x, None, out_t=xt)
    check_product(product(gq, wt, dtype), gq, wt)
    dw = product(gt, xt, F32)
    check_product(dw, gt, xt)
    half = product(gt, xt, F32, dw)
    check_product(half, gt, xt, dw)
    # the gradients of the layer itself, within the casts' rounding: half a step, 2^-4 of an element (and half of 2^-9 of a scale,
    # which is below 2^-7.8 of the block's largest) on both sides of every term
    size = dy.double().abs().t() @ x.double().abs()
    top = dy.double().abs().max() * x.double().abs().max() * M
    assert bool(((dw[0].double() - dy.double().t() @ x.double()).abs() <= 0.13 * size + 2.0 ** -16 * top).all())


def test_layer_step_on_a_stream_and_in_a_graph():
    M, N, K = 130, 260, 400
    x, w, dy = randn(M, K, seed=1, dtype=BF16), randn(N, K, seed=2, std=0.05, dtype=BF16), randn(M, N, seed=3, std=0.1, dtype=BF16)
    e = lambda *s: B.Fp8.empty(1, *s, DEV)
    wq, wt, xq, xt, gq, gt = e(N, K), e(K, N), e(M, K), e(K, M), e(M, N), e(N, M)
    ws = torch.empty(max(B.btx_fp8_matmul_workspace_size(*s, BF16) for s in ((M, N, K), (M, K, N), (N, K, M))), dtype=torch.uint8, device=DEV)
    y, dx, dw = torch.empty(M, N, dtype=BF16, device=DEV), torch.empty(M, K, dtype=BF16, device=DEV), torch.empty(N, K, device=DEV)

    def step():
        B.btx_fp8_quantize(w, wq, block_rows=128, out_t=wt)
        B.btx_fp8_quantize(x, xq, out_t=xt)
        B.btx_fp8_matmul(xq, wq, y, ws)
        B.btx_fp8_quantize(dy, gq, out_t=gt)
        B.btx_fp8_matmul(gq, wt, dx, ws)
        B.btx_fp8_matmul(gt, xt, dw, ws)
    step()
    torch.cuda.synchronize()
    ref = [t.clone() for t in (y, dx, dw)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for t in (y, dx, dw):
            t.zero_()
        step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((y, dx, dw), ref))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(2):
        for t in (y, dx, dw):
            t.zero_()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip((y, dx, dw), ref))


def test_offsets_past_32_bits():
    M, K, N = 600_001, 4096, 4096
    tail = randn(200, K, seed=1, dtype=BF16)
    x = tail[torch.arange(M, device=DEV) % 200]
    q, qt, w = B.Fp8.empty(1, M, K, DEV), B.Fp8.empty(1, 200, K, DEV), B.Fp8.empty(1, N, K, DEV)
    B.btx_fp8_quantize(x, q)
    B.btx_fp8_quantize(tail, qt)
    B.btx_fp8_quantize(randn(N, K, seed=2, dtype=BF16), w, block_rows=128)
    ws = torch.empty(max(B.btx_fp8_matmul_workspace_size(m, N, K, BF16) for m in (200, M)), dtype=torch.uint8, device=DEV)
    small = torch.empty(200, N, dtype=BF16, device=DEV)
    B.btx_fp8_matmul(qt, w, small, ws)
    B.btx_fp8_matmul(q, w, x, ws)
    # sums of another split of the contraction: within the error of K products in fp32
    last = (torch.arange(M - 200, M, device=DEV) % 200)
    scale = float(values64(qt)[0].norm(dim=1).max() * values64(w)[0].norm(dim=1).max())
    assert float((x[-200:].float() - small[last].float()).abs().max()) <= 2.0 ** -8 * float(small.abs().max()) + (K / 32 + 4) * 2.0 ** -21 * scale


def test_binding_refuses_wrong_tensors():
    q = B.Fp8.empty(1, 8, 64, DEV)
    ws = torch.empty(256, dtype=torch.uint8, device=DEV)
    for bad in (lambda: B.btx_fp8_matmul(q, B.Fp8.empty(1, 8, 96, DEV), randn(8, 8), ws), lambda: B.btx_fp8_matmul(q, q, randn(8, 9), ws),
                lambda: B.btx_fp8_matmul(q, B.Fp8.empty(2, 8, 64, DEV), randn(8, 8), ws), lambda: B.btx_fp8_matmul(q, B.Fp8(q.codes, q.scales, 65), randn(8, 8), ws)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(B.BtxError) as ei:
        B.btx_fp8_matmul(q, q, randn(8, 8), ws[:16])
    assert ei.value.status == 3
    with pytest.raises(B.BtxError) as ei:
        B.btx_fp8_matmul(q, q, randn(8, 8, dtype=BF16), ws, accumulate=True)
    assert ei.value.status == 2
