"""MXFP4 casts, products and the expert layer against the 64-bit statement in oracle/experts_oracle.py.

Codes, scales and read-back values are equal bit for bit.  Products: every term a b 2^s is exact in fp32; each step of
64 terms adds them to the running sum with at most one unit of rounding (2^-23 of sum |a b|, which bounds every
partial sum) and loses at most as much in aligning its terms, so an output is within (K/64 + 4) 2^-22 sum |a b| of
the exact sum, plus half a step of the output type.  The expert layer's tolerance is formed by `moe_reference`."""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as o
from paper_2403_07816_b200 import binding as B
from util import Guarded, check_guards

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def randn(*shape, seed=0, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype).to(DEV)


def np64(t):
    return t.double().cpu().numpy()


def guarded_mx4(batch, rows, K, fill=0xA5):
    bufs = {"codes": Guarded((batch, rows, K // 2), torch.uint8, DEV, fill=fill),
            "scales": Guarded((batch, (rows + 127) // 128, (K + 127) // 128, 512), torch.uint8, DEV, fill=fill)}
    return B.Mx4(bufs["codes"].t, bufs["scales"].t), bufs


def expected(x, fill):
    """codes and scale tiles of x [batch, rows, K] as stored, over buffers that held `fill`."""
    codes, tiles = [], []
    for m in x:
        c, s = o.mx4_quantize(m)
        codes.append(o.mx4_pack(c))
        nb = s.shape[1]
        pad = np.zeros((s.shape[0], (nb + 3) // 4 * 4), np.uint8)
        pad[:, :nb] = s
        tiles.append(o.mx4_tile_scales(pad, fill))
    return np.stack(codes), np.stack(tiles)


def special_values(dtype):
    """Blocks around every border of the cast: rounding ties, powers of two, saturation, subnormals, zeros, NaN."""
    rows = []
    base = np.array([0.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 7.96875, 0.5, 1.0, 1.5, 2.0, 3.0])
    both = np.concatenate([base, -base])
    for e in (0, -3, 4, -100, -125, -130, 120, 125):
        with np.errstate(over="ignore"):
            rows.append(both * 2.0 ** e)
    rows.append(np.zeros(32))
    rows.append(-np.zeros(32))
    for amax in (3.9999998, 4.0, 7.9999995, 8.0, 1e-38, 1.1754944e-38, 1e-45, 3.3895e38):
        v = np.linspace(-1, 1, 32) * amax
        v[5] = amax
        rows.append(v)
    for bad in (np.nan, np.inf, -np.inf):
        v = np.linspace(-2, 2, 32)
        v[17] = bad
        rows.append(v)
    x = torch.tensor(np.stack(rows)).float()
    x = torch.where(x.abs() > torch.finfo(dtype).max, torch.sign(x) * torch.finfo(dtype).max, x) if dtype != torch.float32 else x
    return x.to(dtype).reshape(1, -1, 32).to(DEV)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1, 32), (1, 33, 64), (2, 129, 96), (1, 130, 1056), (3, 7, 2080), (1, 300, 160)],
                         ids=lambda s: "x".join(map(str, s)))
def test_cast(shape, dtype):
    x = randn(*shape, seed=sum(shape), dtype=dtype)
    q, bufs = guarded_mx4(*shape)
    B.btx_mx4_quantize(x, q)
    check_guards(bufs, "btx_mx4_quantize")
    codes, tiles = expected(np64(x), 0xA5)
    assert np.array_equal(q.codes.cpu().numpy(), codes) and np.array_equal(q.scales.cpu().numpy(), tiles)
    for out in (torch.float32, torch.bfloat16):
        back = Guarded(shape, out, DEV)
        B.btx_mx4_dequantize(q, back.t)
        check_guards({"dst": back}, "btx_mx4_dequantize")
        assert np.array_equal(np64(back.t), o.mx4_round(np64(x)))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_cast_at_its_borders(dtype):
    x = special_values(dtype)
    q, _ = guarded_mx4(*x.shape)
    B.btx_mx4_quantize(x, q)
    codes, tiles = expected(np64(x), 0xA5)
    assert np.array_equal(q.scales.cpu().numpy(), tiles)
    assert np.array_equal(q.codes.cpu().numpy(), codes)
    back = torch.empty_like(x)
    B.btx_mx4_dequantize(q, back)
    assert np.array_equal(np64(back), o.mx4_round(np64(x)), equal_nan=True)


def test_cast_of_strided_rows_into_interleaved_rows():
    w = randn(2, 70, 200, seed=3)
    for src in (w[:, :, 3:99], w[:, ::2, 8:104], w[:1, :, 100:196]):
        batch, rows, K = src.shape
        q, bufs = guarded_mx4(batch, 2 * rows + 1, K, fill=0x11)
        B.btx_mx4_quantize(src, q, row_first=1, row_step=2)
        check_guards(bufs, "btx_mx4_quantize")
        ref, _ = guarded_mx4(batch, rows, K)
        B.btx_mx4_quantize(src.contiguous(), ref)
        assert torch.equal(q.codes[:, 1::2], ref.codes)
        assert bool((q.codes[:, 0::2] == 0x11).all())      # rows that the call does not name
        for r in range(rows):
            a, b = 2 * r + 1, r
            at = lambda t, i: t[:, i // 128, :, (i % 32) * 16 + (i // 32 % 4) * 4:][:, :, :4]
            assert torch.equal(at(q.scales, a), at(ref.scales, b))
            assert bool((at(q.scales, 2 * r) == 0x11).all())


def matmul(a, b, dtype):
    qa, ba = guarded_mx4(*a.shape)
    qb, bb = guarded_mx4(*b.shape, fill=0xFF)              # unwritten scale bytes read as NaN
    B.btx_mx4_quantize(a, qa)
    B.btx_mx4_quantize(b, qb)
    batch, M, K = a.shape
    N = b.shape[1]
    y = Guarded((batch, M, N), dtype, DEV)
    ws = Guarded(B.btx_mx4_matmul_workspace_size(M, N, K, dtype, batch), torch.uint8, DEV, fill=0x7F)
    B.btx_mx4_matmul(qa, qb, y.t, ws.t)
    assert B.btx_device_status(ws.t) == B.BTX_OK
    check_guards({"y": y, "workspace": ws, "a": ba["codes"], "b": bb["codes"]}, "btx_mx4_matmul")
    return y.t, qa, qb


def values64(q):
    v = torch.empty(q.shape, dtype=torch.float32, device=DEV)
    B.btx_mx4_dequantize(q, v)
    return v.double()


def check_product(y, qa, qb):
    va, vb = values64(qa), values64(qb)
    want = va @ vb.transpose(1, 2)
    size = va.abs() @ vb.abs().transpose(1, 2)
    tol = (qa.shape[2] / 64 + 4) * 2.0 ** -22 * size + torch.finfo(y.dtype).eps / 2 * want.abs()
    err = (y.double() - want).abs()
    assert bool((err <= tol).all()), float((err - tol).max())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1, 1, 32), (1, 1, 128, 64), (1, 128, 128, 256), (1, 5, 200, 96), (1, 129, 255, 160),
                                   (1, 300, 64, 1056), (2, 130, 136, 288), (3, 1, 1000, 512), (1, 1000, 17, 2048),
                                   (1, 64, 4096, 4096), (1, 520, 2056, 544),
                                   (1, 2100, 2300, 320), (3, 1100, 1300, 96), (1, 4100, 1290, 2080), (1, 1500, 3331, 128), (1, 1500, 3334, 128)], ids=lambda s: "x".join(map(str, s)))
def test_product(shape, dtype):
    batch, M, N, K = shape
    y, qa, qb = matmul(randn(batch, M, K, seed=M + K), randn(batch, N, K, seed=N + K + 1, std=0.02), dtype)
    check_product(y, qa, qb)


def test_product_is_exact_on_whole_numbers():
    # one element of A per row: y is a row of B times it, at every position of the contraction and every scale
    K = 320
    a = torch.zeros(1, K, K, device=DEV)
    a[0].fill_diagonal_(1.5)
    g = torch.Generator().manual_seed(2)
    b = torch.randint(-6, 7, (1, 40, K), generator=g).float().to(DEV) * torch.exp2(torch.randint(-8, 8, (1, 40, K // 32), generator=g).float()).to(DEV).repeat_interleave(32, 2)
    y, qa, qb = matmul(a, b, torch.float32)
    assert torch.equal(y[0].double(), (1.5 * values64(qb)[0]).t())


def test_scales_of_extreme_size_and_nan_blocks():
    a = randn(1, 40, 128, seed=5)
    a[0, 3] *= 2.0 ** 90
    a[0, 4] *= 2.0 ** -90
    b = randn(1, 70, 128, seed=6)
    b[0, 7, 40] = float("nan")
    b[0, 9] *= 2.0 ** -60
    y, qa, qb = matmul(a, b, torch.float32)
    assert bool(y[0, :, 7].isnan().all())
    keep = [i for i in range(70) if i != 7]
    va, vb = values64(qa)[0], values64(qb)[0][keep]
    err = (y[0][:, keep].double() - va @ vb.t()).abs()
    # row 4 times row 9 is a sum of 128 terms of at most 36 * 2^-150 * 2^-2: it lies below 2^-126, the smallest normal
    # fp32 number, where fp32 holds no relative accuracy (and the sum may be flushed to zero)
    assert bool((err <= 6 * 2.0 ** -22 * (va.abs() @ vb.abs().t()) + 2.0 ** -126).all())


def random_routing(T, E, k, seed, empty=0.0):
    g = torch.Generator().manual_seed(seed)
    idx = torch.rand(T, E, generator=g).topk(k, dim=1)[1].to(torch.int32)
    if empty:
        idx[torch.rand(T, k, generator=g) < empty] = -1
    return idx.to(DEV), torch.rand(T, k, generator=g).to(DEV)


def moe_reference(x, idx, gates, w1, w3, w2):
    """y and its tolerance, in 64 bits.  The cast of the activations may go the other way for an element whose value
    lies within the error of the first product of a border: `spread` is how far its cast can move, over both ends of
    that error in the element and in the block's largest, and counts in full."""
    T, d = x.shape
    y, tol = np.zeros((T, d)), np.zeros((T, d))
    xq = o.mx4_round(x)
    F = w1.shape[1]
    rounded = {}
    for t in range(T):
        for j in range(idx.shape[1]):
            e = idx[t, j]
            if e < 0 or e >= w1.shape[0]:
                continue
            if e not in rounded:
                rounded[e] = o.mx4_round(w1[e]), o.mx4_round(w3[e]), o.mx4_round(w2[e])
                rounded[e] += tuple(np.abs(u) for u in rounded[e])
            u1, u3, u2, v1, v3, v2 = rounded[e]
            step = (d / 64 + 4) * 2.0 ** -22
            h1, h3 = u1 @ xq[t], u3 @ xq[t]
            d1, d3 = step * (v1 @ np.abs(xq[t])), step * (v3 @ np.abs(xq[t]))
            silu = h1 / (1 + np.exp(-h1))
            a = silu * h3
            da = 1.1 * d1 * (np.abs(h3) + d3) + np.abs(silu) * d3 + 2.0 ** -19 * np.abs(a)   # |silu'| <= 1.1
            blocks, eb = a.reshape(-1, 32), da.reshape(-1, 32)
            amax = np.abs(blocks).max(1)
            casts = []
            for big in (np.maximum(amax - eb.max(1), 0), amax + eb.max(1)):
                exp = np.maximum(np.where(big > 0, np.frexp(big)[1] - 3, -127), -127)
                s = np.exp2(exp.astype(float))[:, None]
                for v in (blocks - eb, blocks, blocks + eb):
                    p = np.abs(v) / s
                    q = o.E2M1[np.abs(p[..., None] - o.E2M1).argmin(-1)]
                    casts.append(np.sign(v) * q * s)
            casts = np.stack(casts)
            spread = (casts.max(0) - casts.min(0)).reshape(-1)
            act = o.mx4_round(a)
            size = v2 @ np.abs(act)
            y[t] += gates[t, j] * (u2 @ act)
            tol[t] += np.abs(gates[t, j]) * (v2 @ spread + (F / 64 + 8) * 2.0 ** -22 * size)
    return y, tol


def moe(x, idx, gates, w1, w3, w2, dst=None):
    T, d = x.shape
    E, F, _ = w1.shape
    w13, b13 = guarded_mx4(E, 2 * F, d, fill=0xFF)
    B.btx_mx4_quantize(w1, w13, 0, 2)
    B.btx_mx4_quantize(w3, w13, 1, 2)
    w2q, b2 = guarded_mx4(E, d, F, fill=0xFF)
    B.btx_mx4_quantize(w2, w2q)
    desc = B.make_mx4_moe_desc(T, d, F, E, idx.shape[1], x.dtype)
    y = Guarded((T, d), x.dtype, DEV)
    ws = Guarded(B.btx_mx4_moe_workspace_size(desc), torch.uint8, DEV, fill=0xFF)
    B.btx_mx4_moe_forward(desc, x, idx, gates, w13, w2q, y.t, ws.t)
    assert B.btx_device_status(ws.t) == B.BTX_OK
    check_guards({"y": y, "workspace": ws, "w13": b13["codes"], "w2": b2["codes"]}, "btx_mx4_moe_forward")
    return y.t, (desc, w13, w2q)


# (T, d, F, E, k, empty)
LAYERS = [(1, 128, 160, 4, 2, 0.0), (5, 64, 32, 3, 1, 0.0), (33, 96, 224, 4, 2, 0.3), (150, 256, 288, 2, 2, 0.0),
          (40, 160, 96, 40, 6, 0.0), (7, 32, 64, 512, 8, 0.0), (300, 64, 96, 1, 1, 0.1), (1100, 32, 64, 7, 3, 0.05),
          (3000, 1056, 160, 2, 2, 0.05), (2500, 544, 1184, 5, 3, 0.0),
          (520, 96, 1056, 3, 3, 0.1), (200, 1184, 96, 6, 5, 0.0), (290, 2080, 64, 9, 3, 0.2), (2, 320, 4128, 8, 1, 0.0)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("layer", LAYERS, ids=lambda s: "x".join(map(str, s)))
def test_expert_layer(layer, dtype):
    T, d, F, E, k, empty = layer
    x = randn(T, d, seed=T, dtype=dtype)
    w1, w3, w2 = (randn(E, *s, seed=i, std=0.2) for i, s in enumerate([(F, d), (F, d), (d, F)]))
    idx, gates = random_routing(T, E, k, T + E, empty)
    y, _ = moe(x, idx, gates, w1, w3, w2)
    rows = np.arange(T) if T <= 64 else np.r_[0:20, T // 2:T // 2 + 20, T - 20:T]
    want, tol = moe_reference(np64(x)[rows], idx.cpu().numpy()[rows], np64(gates)[rows], np64(w1), np64(w3), np64(w2))
    err = np.abs(np64(y)[rows] - want)
    assert (err <= tol + torch.finfo(dtype).eps / 2 * np.abs(want) + 1e-30).all(), (err - tol).max()


def test_expert_layer_empty_slots_only_and_out_of_range():
    x = randn(9, 64, seed=1)
    w1, w3, w2 = (randn(3, *s, seed=i, std=0.2) for i, s in enumerate([(96, 64), (96, 64), (64, 96)]))
    idx, gates = random_routing(9, 3, 2, 4)
    y, _ = moe(x, torch.full_like(idx, -1), gates, w1, w3, w2)
    assert bool((y == 0).all())
    odd = idx.clone()
    odd[2, 0], odd[3, 1], odd[4, 0] = 3, 1 << 30, -7
    ref = idx.clone()
    ref[2, 0], ref[3, 1], ref[4, 0] = -1, -1, -1
    assert torch.equal(moe(x, odd, gates, w1, w3, w2)[0], moe(x, ref, gates, w1, w3, w2)[0])
    twice = idx.clone()
    twice[:, 1] = twice[:, 0]                              # the same expert in both slots
    both = moe(x, twice, gates, w1, w3, w2)[0]
    one = moe(x, twice[:, :1].contiguous(), gates.sum(1, keepdim=True), w1, w3, w2)[0]
    assert float((both - one).abs().max()) <= 2.0 ** -21 * float(one.abs().max())


def test_padded_batch_of_few_tokens_leaves_the_workspace():
    # the few tokens' tiles alone would let every part of the contraction have rows of its own, more than there is room for
    T, d, F, E, k = 128, 1024, 2048, 8, 8
    x = randn(T, d, seed=3, dtype=torch.bfloat16)
    w1, w3, w2 = (randn(E, *s, seed=i, std=0.05) for i, s in enumerate([(F, d), (F, d), (d, F)]))
    idx, gates = random_routing(T, E, k, 11)
    for kept in ([0, 127], [64]):
        few = torch.full_like(idx, -1)
        few[kept, :2] = 5
        y, _ = moe(x, few, gates, w1, w3, w2)             # (looks at the guards around the workspace)
        off = torch.ones(T, dtype=torch.bool)
        off[kept] = False
        assert bool((y[off.to(DEV)] == 0).all())
        one = np.where(few.cpu().numpy()[kept] == 5, 0, -1)
        want, tol = moe_reference(np64(x)[kept], one, np64(gates)[kept], np64(w1[5:6]), np64(w3[5:6]), np64(w2[5:6]))
        assert (np.abs(np64(y)[kept] - want) <= tol + 2.0 ** -8 * np.abs(want)).all()


@pytest.mark.parametrize("layer", [(33, 96, 224, 4, 2), (600, 96, 160, 4, 2), (3000, 1056, 160, 2, 2)], ids=lambda s: "x".join(map(str, s)))
def test_rows_that_are_not_numbers_stay_by_themselves(layer):
    # NaN in rows without an expert (and in the gates of empty slots) is not read; in other rows it reaches that row alone
    T, d, F, E, k = layer
    x = randn(T, d, seed=T, dtype=torch.bfloat16)
    w1, w3, w2 = (randn(E, *s, seed=i, std=0.2) for i, s in enumerate([(F, d), (F, d), (d, F)]))
    idx, gates = random_routing(T, E, k, T)
    idx[2::9] = -1
    idx[3, 0] = -1
    clean, _ = moe(x, idx, gates, w1, w3, w2)
    x[2::9] = float("nan")
    gates[2::9] = float("inf")
    gates[3, 0] = float("nan")
    x[5, 40], x[7, 33] = float("inf"), float("nan")
    y, _ = moe(x, idx, gates, w1, w3, w2)
    bad = torch.zeros(T, dtype=torch.bool, device=DEV)
    bad[[5, 7]] = True
    assert bool(torch.isnan(y[bad]).all()) and torch.equal(y[~bad], clean[~bad]) and bool((y[2::9] == 0).all())


def test_layer_is_the_same_whatever_shares_its_batch():
    # a row's result does not depend on the rows around it (tiles of 128, one or several dispatch blocks)
    T, d, F, E, k = 3000, 96, 160, 5, 2
    x = randn(T, d, seed=2, dtype=torch.bfloat16)
    w1, w3, w2 = (randn(E, *s, seed=i, std=0.2) for i, s in enumerate([(F, d), (F, d), (d, F)]))
    idx, gates = random_routing(T, E, k, 8)
    big, _ = moe(x, idx, gates, w1, w3, w2)
    for a, b in ((0, 1), (17, 60), (1000, 2500), (2999, 3000)):
        part, _ = moe(x[a:b].contiguous(), idx[a:b].contiguous(), gates[a:b].contiguous(), w1, w3, w2)
        assert torch.equal(part, big[a:b])
    again, _ = moe(x, idx, gates, w1, w3, w2)
    assert torch.equal(again, big)


def test_large_tiles_give_the_rows_of_small_ones():
    # enough rows per expert for products by CTA pairs; the parts are too small for them
    T, d, F, E, k = 4000, 1280, 320, 3, 2
    x = randn(T, d, seed=2, dtype=torch.bfloat16)
    w1, w3, w2 = (randn(E, *s, seed=i, std=0.2) for i, s in enumerate([(F, d), (F, d), (d, F)]))
    idx, gates = random_routing(T, E, k, 8, 0.1)
    big, _ = moe(x, idx, gates, w1, w3, w2)
    for a, b in ((0, 1), (100, 300), (3990, 4000)):
        part, _ = moe(x[a:b].contiguous(), idx[a:b].contiguous(), gates[a:b].contiguous(), w1, w3, w2)
        assert torch.equal(part, big[a:b])


def test_route_then_layer_on_a_stream_and_in_a_graph():
    T, d, F, E, k = 48, 128, 192, 64, 4
    x = randn(T, d, seed=2, dtype=torch.bfloat16)
    w1, w3, w2 = (randn(E, *s, seed=i, std=0.2) for i, s in enumerate([(F, d), (F, d), (d, F)]))
    wr, bias = randn(E, d, seed=7, std=0.1), randn(E, seed=8, std=0.1)
    logits = x.float() @ wr.t()
    rd = B.make_route_desc(T, E, k, torch.float32, B.SCORE_SIGMOID, 8, 4, B.GROUP_SUM2, True, 2.5)
    idx, gates = torch.empty(T, k, dtype=torch.int32, device=DEV), torch.empty(T, k, device=DEV)
    B.btx_route(rd, logits, bias, idx, gates)
    ref, (desc, w13, w2q) = moe(x, idx, gates, w1, w3, w2)
    want, tol = moe_reference(np64(x), idx.cpu().numpy(), np64(gates), np64(w1), np64(w3), np64(w2))
    assert (np.abs(np64(ref) - want) <= tol + 2.0 ** -8 * np.abs(want)).all()
    y = torch.empty_like(x)
    ws = torch.empty(B.btx_mx4_moe_workspace_size(desc), dtype=torch.uint8, device=DEV)
    zin, xin = logits.clone(), x.clone()

    def step():
        B.btx_route(rd, zin, bias, idx, gates)
        B.btx_mx4_moe_forward(desc, xin, idx, gates, w13, w2q, y, ws)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    assert torch.equal(y, ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for shift in (0, 5, 0):
        zin.copy_(logits.roll(shift, 0))
        xin.copy_(x.roll(shift, 0))
        y.fill_(7)
        graph.replay()
        assert torch.equal(y, ref.roll(shift, 0))


def test_layers_on_two_streams_at_once():
    # small batches run as cooperative kernels that want the whole device: neither may keep the other from finishing
    T, d, F, E, k = 24, 512, 1024, 6, 2
    w1, w3, w2 = (randn(E, *s, seed=i, std=0.1) for i, s in enumerate([(F, d), (F, d), (d, F)]))
    runs = []
    for i in range(2):
        x = randn(T, d, seed=20 + i, dtype=torch.bfloat16)
        idx, gates = random_routing(T, E, k, 30 + i)
        ref, (desc, w13, w2q) = moe(x, idx, gates, w1, w3, w2)
        ws = torch.empty(B.btx_mx4_moe_workspace_size(desc), dtype=torch.uint8, device=DEV)
        runs.append((x, idx, gates, ref, desc, w13, w2q, torch.empty_like(x), ws, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for x, idx, gates, ref, desc, w13, w2q, y, ws, stream in runs:
            with torch.cuda.stream(stream):
                B.btx_mx4_moe_forward(desc, x, idx, gates, w13, w2q, y, ws)
    torch.cuda.synchronize()
    for x, idx, gates, ref, desc, w13, w2q, y, ws, stream in runs:
        assert torch.equal(y, ref) and B.btx_device_status(ws) == B.BTX_OK


def test_offsets_past_32_bits():
    # 2.4 G elements in x, in y and in the layer's rows: the last rows are those of a small call
    M, K, N = 600_001, 4096, 4096
    x = torch.empty(M, K, dtype=torch.bfloat16, device=DEV)
    tail = randn(200, K, seed=1, dtype=torch.bfloat16)
    x[:-200] = tail[0]
    x[-200:] = tail
    q, qt, w = B.Mx4.empty(1, M, K, DEV), B.Mx4.empty(1, 200, K, DEV), B.Mx4.empty(1, N, K, DEV)
    B.btx_mx4_quantize(x, q)
    B.btx_mx4_quantize(tail, qt)
    B.btx_mx4_quantize(randn(N, K, seed=2, dtype=torch.bfloat16), w)
    assert torch.equal(q.codes[0, -200:], qt.codes[0])
    B.btx_mx4_dequantize(q, x)
    back = torch.empty_like(tail)
    B.btx_mx4_dequantize(qt, back)
    assert torch.equal(x[-200:], back)
    ws, small = torch.empty(256, dtype=torch.uint8, device=DEV), torch.empty(200, N, dtype=torch.bfloat16, device=DEV)
    B.btx_mx4_matmul(qt, w, small, ws)
    B.btx_mx4_matmul(q, w, x, ws)
    # sums of another split of the contraction: within the error of K products in fp32
    scale = float(back.float().norm(dim=1).max())
    assert float((x[-200:].float() - small.float()).abs().max()) <= 2.0 ** -8 * float(small.abs().max()) + 2.0 ** -20 * scale ** 2
    del x, q
    T, d, F, E, k = 300_001, 4096, 64, 3, 2
    xs = tail[torch.arange(T, device=DEV) % 200].contiguous()
    w13, w2 = B.Mx4.empty(E, 2 * F, d, DEV), B.Mx4.empty(E, d, F, DEV)
    B.btx_mx4_quantize(randn(E, 2 * F, d, seed=3, std=0.02), w13)
    B.btx_mx4_quantize(randn(E, d, F, seed=4, std=0.2), w2)
    idx, gates = random_routing(200, E, k, 5)
    big = [t[torch.arange(T, device=DEV) % 200].contiguous() for t in (idx, gates)]
    ys = []
    for n, xi, ii, gi in ((T, xs, *big), (200, tail, idx, gates)):
        desc = B.make_mx4_moe_desc(n, d, F, E, k, torch.bfloat16)
        ws = torch.empty(B.btx_mx4_moe_workspace_size(desc), dtype=torch.uint8, device=DEV)
        ys.append(torch.empty_like(xi))
        B.btx_mx4_moe_forward(desc, xi, ii, gi, w13, w2, ys[-1], ws)
    assert torch.equal(ys[0][:200], ys[1]) and torch.equal(ys[0][T // 200 * 200 - 200:T // 200 * 200], ys[1])
    assert torch.equal(ys[0][-1], ys[1][(T - 1) % 200])


def test_binding_refuses_wrong_tensors():
    q = B.Mx4.empty(1, 8, 64, DEV)
    x = randn(8, 64)
    for bad in (lambda: B.btx_mx4_quantize(randn(8, 96), q), lambda: B.btx_mx4_quantize(x, B.Mx4(q.codes, q.scales[..., :256])),
                lambda: B.btx_mx4_dequantize(q, randn(8, 32)),
                lambda: B.btx_mx4_matmul(q, B.Mx4.empty(1, 8, 96, DEV), randn(8, 8), torch.empty(256, dtype=torch.uint8, device=DEV)),
                lambda: B.btx_mx4_matmul(q, q, randn(8, 9), torch.empty(256, dtype=torch.uint8, device=DEV))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(RuntimeError):
        B.btx_mx4_quantize(randn(64, 8).t(), q)
    with pytest.raises(B.BtxError) as ei:
        B.btx_mx4_quantize(x, q, row_first=1)              # the last row would fall outside
    assert ei.value.status == 1
    with pytest.raises(B.BtxError) as ei:
        B.btx_mx4_matmul(q, q, randn(8, 8), torch.empty(16, dtype=torch.uint8, device=DEV))
    assert ei.value.status == 3
    with pytest.raises(TypeError):
        B.btx_mx4_quantize(x.half(), q)
