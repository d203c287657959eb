"""The expert layer on FP8 experts, and the norm, the score routing and the layer together, against 64-bit statements.

The layer's tolerance is formed by `moe_reference`."""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as eo
from oracle import fp8_oracle as o
from paper_2403_07816_b200 import binding as B
from util import Guarded, check_guards

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def randn(*shape, seed=0, std=1.0, dtype=F32):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype).to(DEV)


def np64(t):
    return t.double().cpu().numpy()


def guarded_fp8(batch, rows, K, fill=0xFF):
    """Unwritten scale bytes read as NaN."""
    bufs = {"codes": Guarded((batch, rows, (K + 31) // 32 * 32), torch.uint8, DEV, fill=fill),
            "scales": Guarded((batch, (rows + 127) // 128, (K + 511) // 512, 512), torch.uint8, DEV, fill=fill)}
    return B.Fp8(bufs["codes"].t, bufs["scales"].t, K), bufs


def random_routing(T, E, k, seed, empty=0.0):
    g = torch.Generator().manual_seed(seed)
    idx = torch.rand(T, E, generator=g).topk(k, dim=1)[1].to(torch.int32)
    if empty:
        idx[torch.rand(T, k, generator=g) < empty] = -1
    return idx.to(DEV), torch.rand(T, k, generator=g).to(DEV)


def moe_reference(xq, idx, gates, w1, w3, w2, weights=None):
    """y and its tolerance from the FP8 values xq of x, in 64 bits.  A product is within (K/32 + 4) 2^-22 of the sizes of its terms.
    The cast of the activations may go the other way for an element whose value lies within the error of the first product of
    a border: `spread` is how far its cast can move, over both ends of that error in the element and in the block's largest,
    and counts in full."""
    T, d = xq.shape
    F = w1.shape[1]
    nb = -(-F // 128)
    y, tol = np.zeros((T, d)), np.zeros((T, d))
    rounded = {} if weights is None else weights
    pad = lambda v: np.pad(v, (0, nb * 128 - F)).reshape(nb, 128)
    for t in range(T):
        for j in range(idx.shape[1]):
            e = idx[t, j]
            if e < 0 or e >= w1.shape[0]:
                continue
            if e not in rounded:
                rounded[e] = tuple(o.round_rows(w, 128) for w in (w1[e], w3[e], w2[e]))
            u1, u3, u2 = rounded[e]
            step = (d / 32 + 4) * 2.0 ** -22
            h1, h3 = u1 @ xq[t], u3 @ xq[t]
            d1, d3 = step * (np.abs(u1) @ np.abs(xq[t])), step * (np.abs(u3) @ np.abs(xq[t]))
            silu = h1 / (1 + np.exp(-h1))
            a = silu * h3
            da = 1.1 * d1 * (np.abs(h3) + d3) + np.abs(silu) * d3 + 2.0 ** -19 * np.abs(a)   # |silu'| <= 1.1
            blocks, eb = pad(a), pad(da)
            amax, off = np.abs(blocks).max(1), eb.max(1)
            casts = []
            for big in (np.maximum(amax - off, 0), amax + off):
                exp = np.where(big > 0, np.maximum(np.ceil(np.log2(np.maximum(big, 1e-300) / 448)), -127), -127)
                s = np.exp2(exp)[:, None]
                for v in (blocks - eb, blocks, blocks + eb):
                    casts.append(np.sign(v) * o.E4M3[o._nearest(np.minimum(np.abs(v) / s, 448))] * s)
            casts = np.stack(casts)
            spread = (casts.max(0) - casts.min(0)).reshape(-1)[:F]
            act = o.round_rows(a[None])[0]
            y[t] += gates[t, j] * (u2 @ act)
            tol[t] += np.abs(gates[t, j]) * (np.abs(u2) @ spread + (F / 32 + 8) * 2.0 ** -22 * (np.abs(u2) @ np.abs(act)))
    return y, tol


def experts(w1, w3, w2):
    E, F, d = w1.shape
    (w13, b13), (w2q, b2) = guarded_fp8(E, 2 * F, d), guarded_fp8(E, d, F)
    B.btx_fp8_quantize(w1, w13, block_rows=128, row_first=0, row_step=2)
    B.btx_fp8_quantize(w3, w13, block_rows=128, row_first=1, row_step=2)
    B.btx_fp8_quantize(w2, w2q, block_rows=128)
    return w13, w2q, {"w13": b13["codes"], "w2": b2["codes"]}


def moe(x, idx, gates, w1, w3, w2, dtype=None):
    T, d = x.shape[-2:]
    E, F, _ = w1.shape
    dtype = dtype or x.dtype
    w13, w2q, bufs = experts(w1, w3, w2)
    desc = B.make_fp8_moe_desc(T, d, F, E, idx.shape[1], dtype)
    bufs["y"] = Guarded((T, d), dtype, DEV)
    bufs["workspace"] = Guarded(B.btx_fp8_moe_workspace_size(desc), torch.uint8, DEV, fill=0xFF)
    B.btx_fp8_moe_forward(desc, x, idx, gates, w13, w2q, bufs["y"].t, bufs["workspace"].t)
    assert B.btx_device_status(bufs["workspace"].t) == B.BTX_OK
    check_guards(bufs, "btx_fp8_moe_forward")
    return bufs["y"].t, (desc, w13, w2q)


def weights_of(E, F, d, std=0.2):
    return tuple(randn(E, *s, seed=i, std=std) for i, s in enumerate([(F, d), (F, d), (d, F)]))


# (T, d, F, E, k, empty): one tile and many, few and many rows for each expert, units that end inside a tile or a block
LAYERS = [(1, 128, 160, 4, 2, 0.0), (5, 64, 16, 3, 1, 0.0), (33, 96, 224, 4, 2, 0.3), (150, 256, 288, 2, 2, 0.0),
          (40, 160, 112, 40, 6, 0.0), (7, 32, 64, 512, 8, 0.0), (300, 64, 96, 1, 1, 0.1), (1100, 48, 64, 7, 3, 0.05),
          (3000, 1056, 176, 2, 2, 0.05), (2500, 544, 1184, 5, 3, 0.0), (520, 112, 1056, 3, 3, 0.1), (200, 1184, 96, 6, 5, 0.0),
          (290, 2064, 64, 9, 3, 0.2), (2, 320, 4112, 8, 1, 0.0), (3000, 1040, 400, 1, 1, 0.0), (2, 16, 16, 1, 1, 0.0)]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("layer", LAYERS, ids=lambda s: "x".join(map(str, s)))
def test_expert_layer(layer, dtype):
    T, d, F, E, k, empty = layer
    x, w = randn(T, d, seed=T, dtype=dtype), weights_of(E, F, d)
    idx, gates = random_routing(T, E, k, T + E, empty)
    y, (desc, w13, w2q) = moe(x, idx, gates, *w)
    rows = np.arange(T) if T <= 64 else np.r_[0:20, T // 2:T // 2 + 20, T - 20:T]
    want, tol = moe_reference(o.round_rows(np64(x)[rows]), idx.cpu().numpy()[rows], np64(gates)[rows], *map(np64, w))
    err = np.abs(np64(y)[rows] - want)
    assert (err <= tol + torch.finfo(dtype).eps / 2 * np.abs(want) + 1e-30).all(), (err - tol).max()
    q = B.Fp8.empty(1, T, d, DEV)                              # the same from the FP8 form of x
    B.btx_fp8_quantize(x, q)
    y2 = torch.empty_like(y)
    ws = torch.empty(B.btx_fp8_moe_workspace_size(desc), dtype=torch.uint8, device=DEV)
    B.btx_fp8_moe_forward(desc, q, idx, gates, w13, w2q, y2, ws)
    assert torch.equal(y2, y)


def test_expert_layer_empty_slots_only_and_out_of_range():
    x, w = randn(9, 64, seed=1), weights_of(3, 96, 64)
    idx, gates = random_routing(9, 3, 2, 4)
    y, _ = moe(x, torch.full_like(idx, -1), gates, *w)
    assert bool((y == 0).all())
    odd, ref = idx.clone(), idx.clone()
    odd[2, 0], odd[3, 1], odd[4, 0] = 3, 1 << 30, -7
    ref[2, 0], ref[3, 1], ref[4, 0] = -1, -1, -1
    assert torch.equal(moe(x, odd, gates, *w)[0], moe(x, ref, gates, *w)[0])
    twice = idx.clone()
    twice[:, 1] = twice[:, 0]                              # the same expert in both slots
    two = moe(x, twice, gates, *w)[0]
    one = moe(x, twice[:, :1].contiguous(), gates.sum(1, keepdim=True), *w)[0]
    assert float((two - one).abs().max()) <= 2.0 ** -21 * float(one.abs().max())


@pytest.mark.parametrize("layer", [(33, 96, 224, 4, 2), (600, 96, 160, 4, 2), (3000, 1056, 160, 2, 2)], ids=lambda s: "x".join(map(str, s)))
def test_rows_that_are_not_numbers_stay_by_themselves(layer):
    # NaN in rows without an expert (and in the gates of empty slots) is not read; in other rows it reaches that row alone
    T, d, F, E, k = layer
    x, w = randn(T, d, seed=T, dtype=BF16), weights_of(E, F, d)
    idx, gates = random_routing(T, E, k, T)
    idx[2::9] = -1
    idx[3, 0] = -1
    clean, _ = moe(x, idx, gates, *w)
    x[2::9] = float("nan")
    gates[2::9] = float("inf")
    gates[3, 0] = float("nan")
    x[5, 40], x[7, 33] = float("inf"), float("nan")
    y, _ = moe(x, idx, gates, *w)
    bad = torch.zeros(T, dtype=torch.bool, device=DEV)
    bad[[5, 7]] = True
    assert bool(torch.isnan(y[bad]).all()) and torch.equal(y[~bad], clean[~bad]) and bool((y[2::9] == 0).all())


def test_layer_is_the_same_whatever_shares_its_batch():
    # a row's result does not depend on the rows around it (tiles of 128, one or several dispatch blocks; tiles of 256)
    for T, d, F, E, k in ((3000, 96, 160, 5, 2), (4000, 1280, 320, 3, 2)):
        x, w = randn(T, d, seed=2, dtype=BF16), weights_of(E, F, d)
        idx, gates = random_routing(T, E, k, 8, 0.1)
        big, _ = moe(x, idx, gates, *w)
        for a, b in ((0, 1), (17, 60), (1000, 2500), (T - 1, T)):
            part, _ = moe(x[a:b].contiguous(), idx[a:b].contiguous(), gates[a:b].contiguous(), *w)
            assert float((part.float() - big[a:b].float()).abs().max()) <= 2.0 ** -7 * float(big.float().abs().max())
        again, _ = moe(x, idx, gates, *w)
        assert torch.equal(again, big)


def test_norm_route_and_layer_on_a_stream_and_in_a_graph():
    """A serving step of the sublayer: residual and norm, router logits, choice of experts, experts on the norm's FP8 output."""
    T, d, F, E, k = 48, 128, 192, 64, 4
    x, r, wn = randn(T, d, seed=2, dtype=BF16), randn(T, d, seed=3, std=3.0, dtype=BF16), (1 + randn(d, seed=4, std=0.2)).to(BF16)
    wr, bias, w = randn(E, d, seed=7, std=0.1), randn(E, seed=8, std=0.1), weights_of(E, F, d)
    w13, w2q, _ = experts(*w)
    wrq = B.Fp8.empty(1, E, d, DEV)
    B.btx_fp8_quantize(wr, wrq)
    nd, rd = B.make_norm_desc(T, d, BF16), B.make_route_desc(T, E, k, F32, B.SCORE_SIGMOID, 8, 4, B.GROUP_SUM2, True, 2.5)
    md = B.make_fp8_moe_desc(T, d, F, E, k, BF16)
    h, q, z = torch.empty_like(x), B.Fp8.empty(1, T, d, DEV), torch.empty(T, E, device=DEV)
    idx, gates, y = torch.empty(T, k, dtype=torch.int32, device=DEV), torch.empty(T, k, device=DEV), torch.empty_like(x)
    ws = torch.empty(max(256, B.btx_fp8_moe_workspace_size(md)), dtype=torch.uint8, device=DEV)
    xin, rin = x.clone(), r.clone()

    def step():
        B.btx_rms_norm(nd, xin, wn, residual=rin, h=h, q=q)
        B.btx_fp8_matmul(q, wrq, z, ws)
        B.btx_route(rd, z, bias, idx, gates)
        B.btx_fp8_moe_forward(md, q, idx, gates, w13, w2q, y, ws)
    step()
    torch.cuda.synchronize()
    ref = y.clone()
    v = torch.empty(T, d, device=DEV)
    B.btx_fp8_dequantize(q, v)
    # each step from what the one before left: the cast's rounding borders are the norm's test
    n64 = o.rms_norm(np64(h), np64(wn), 1e-5)
    assert (np.abs(np64(v) - n64) <= 2.0 ** -4 * np.abs(n64) + 2.0 ** -17 * np.abs(n64).max()).all()
    want_z = np64(v) @ o.round_rows(np64(wr)).T
    assert np.abs(np64(z) - want_z).max() <= 8 * 2.0 ** -22 * (np.abs(np64(v)) @ np.abs(np64(wr)).T).max() * 1.07
    assert np.array_equal(idx.cpu().numpy(), eo.route(np64(z), k, eo.SIGMOID, np64(bias), 8, 4, eo.GROUP_SUM2, True, 2.5)[0])
    want, tol = moe_reference(np64(v), idx.cpu().numpy(), np64(gates), *map(np64, w))
    assert (np.abs(np64(y) - want) <= tol + 2.0 ** -8 * np.abs(want)).all()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        y.fill_(7)
        step()
    side.synchronize()
    assert torch.equal(y, ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for shift in (0, 5, 0):
        xin.copy_(x.roll(shift, 0))
        rin.copy_(r.roll(shift, 0))
        y.fill_(7)
        graph.replay()
        assert torch.equal(y, ref.roll(shift, 0))


def test_weights_written_right_before_the_layer_and_the_product():
    # kernels start before the one in front has ended, and the layer's weights are read early: not before they are written
    T, d, F, E, k = 40, 512, 2048, 4, 2
    x = randn(T, d, seed=1, dtype=BF16)
    idx, gates = random_routing(T, E, k, 2)
    sets = [tuple(randn(E, *s, seed=10 * i + j, std=0.1) for j, s in enumerate([(F, d), (F, d), (d, F)])) for i in range(2)]
    refs = [moe(x, idx, gates, *w)[0].clone() for w in sets]
    w13, w2q, _ = experts(*sets[0])
    desc = B.make_fp8_moe_desc(T, d, F, E, k, BF16)
    ws, y = torch.empty(B.btx_fp8_moe_workspace_size(desc), dtype=torch.uint8, device=DEV), torch.empty_like(x)
    big = [randn(4096, d, seed=30 + i) for i in range(2)]
    xq, wq, z = B.Fp8.empty(1, T, d, DEV), B.Fp8.empty(1, 4096, d, DEV), torch.empty(T, 4096, device=DEV)
    B.btx_fp8_quantize(x, xq)
    products = []
    for w in big:
        B.btx_fp8_quantize(w, wq)
        torch.cuda.synchronize()
        B.btx_fp8_matmul(xq, wq, z, ws)
        products.append(z.clone())
    outs = []
    torch.cuda.synchronize()
    for i in range(30):
        w1, w3, w2 = sets[i % 2]
        B.btx_fp8_quantize(w2, w2q, block_rows=128)
        B.btx_fp8_quantize(w1, w13, block_rows=128, row_first=0, row_step=2)
        B.btx_fp8_quantize(w3, w13, block_rows=128, row_first=1, row_step=2)
        B.btx_fp8_moe_forward(desc, x, idx, gates, w13, w2q, y, ws)
        B.btx_fp8_quantize(big[i % 2], wq)
        B.btx_fp8_matmul(xq, wq, z, ws)
        outs.append((y.clone(), z.clone()))
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(outs):
        assert torch.equal(a, refs[i % 2]) and torch.equal(b, products[i % 2]), i


def test_two_captured_layers_with_a_workspace_each():
    T, d, F, E, k = 24, 256, 512, 6, 2
    w = weights_of(E, F, d, 0.1)
    w13, w2q, _ = experts(*w)
    desc = B.make_fp8_moe_desc(T, d, F, E, k, BF16)
    runs = []
    for i in range(2):
        x = randn(T, d, seed=40 + i, dtype=BF16)
        idx, gates = random_routing(T, E, k, 50 + i)
        ref = moe(x, idx, gates, *w)[0]
        ws, y = torch.empty(B.btx_fp8_moe_workspace_size(desc), dtype=torch.uint8, device=DEV), torch.empty_like(x)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.btx_fp8_moe_forward(desc, x, idx, gates, w13, w2q, y, ws)
        runs.append((graph, y, ref, torch.cuda.Stream(), x, idx, gates, ws))
    for _ in range(10):
        for graph, y, _, stream, *_ in runs:
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for _, y, ref, *_ in runs:
        assert torch.equal(y, ref)


def test_layers_on_two_streams_at_once():
    T, d, F, E, k = 24, 512, 1024, 6, 2
    w = weights_of(E, F, d, 0.1)
    runs = []
    for i in range(2):
        x = randn(T, d, seed=20 + i, dtype=BF16)
        idx, gates = random_routing(T, E, k, 30 + i)
        ref, (desc, w13, w2q) = moe(x, idx, gates, *w)
        ws = torch.empty(B.btx_fp8_moe_workspace_size(desc), dtype=torch.uint8, device=DEV)
        runs.append((x, idx, gates, ref, desc, w13, w2q, torch.empty_like(x), ws, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for x, idx, gates, ref, desc, w13, w2q, y, ws, stream in runs:
            with torch.cuda.stream(stream):
                B.btx_fp8_moe_forward(desc, x, idx, gates, w13, w2q, y, ws)
    torch.cuda.synchronize()
    for x, idx, gates, ref, desc, w13, w2q, y, ws, stream in runs:
        assert torch.equal(y, ref) and B.btx_device_status(ws) == B.BTX_OK


def test_offsets_past_32_bits():
    T, d, F, E, k = 300_001, 4096, 64, 3, 2                 # 2.4 G elements in the rows, 1.2 G in x and y
    tail = randn(200, d, seed=1, dtype=BF16)
    pick = torch.arange(T, device=DEV) % 200
    w13, w2 = B.Fp8.empty(E, 2 * F, d, DEV), B.Fp8.empty(E, d, F, DEV)
    B.btx_fp8_quantize(randn(E, 2 * F, d, seed=3, std=0.02), w13)
    B.btx_fp8_quantize(randn(E, d, F, seed=4, std=0.2), w2)
    idx, gates = random_routing(200, E, k, 5)
    ys = []
    for n, xi, ii, gi in ((T, tail[pick].contiguous(), idx[pick].contiguous(), gates[pick].contiguous()), (200, tail, idx, gates)):
        desc = B.make_fp8_moe_desc(n, d, F, E, k, BF16)
        ws = torch.empty(B.btx_fp8_moe_workspace_size(desc), dtype=torch.uint8, device=DEV)
        ys.append(torch.empty_like(xi))
        B.btx_fp8_moe_forward(desc, xi, ii, gi, w13, w2, ys[-1], ws)
    # sums of other splits and tiles; an activation at a border of its cast may have moved by a step
    most = 2.0 ** -7 * float(ys[1].float().abs().max())
    for at in (0, T // 2 // 200 * 200, (T // 200 - 1) * 200):
        assert float((ys[0][at:at + 200].float() - ys[1].float()).abs().max()) <= most
    assert float((ys[0][-1].float() - ys[1][(T - 1) % 200].float()).abs().max()) <= most


def test_binding_refuses_wrong_tensors():
    x, (idx, gates) = randn(9, 64, seed=1), random_routing(9, 3, 2, 4)
    y, (desc, w13, w2q) = moe(x, idx, gates, *weights_of(3, 96, 64))
    ws = torch.empty(B.btx_fp8_moe_workspace_size(desc), dtype=torch.uint8, device=DEV)
    run = lambda x=x, idx=idx, gates=gates, w13=w13, w2=w2q, y=y, ws=ws: B.btx_fp8_moe_forward(desc, x, idx, gates, w13, w2, y, ws)
    for bad in (dict(x=x[:4]), dict(x=x.bfloat16()), dict(x=B.Fp8.empty(1, 9, 80, DEV)), dict(idx=idx.long()), dict(gates=gates[:, :1]),
                dict(w13=w2q), dict(w2=w13), dict(y=y.bfloat16())):
        with pytest.raises(ValueError):
            run(**bad)
    with pytest.raises(B.BtxError) as ei:
        run(ws=ws[:512])
    assert ei.value.status == 3
