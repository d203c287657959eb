"""btx_route and btx_route_backward against the 64-bit statement in oracle/experts_oracle.py: every score, group rule
and type at even and ragged sizes, rows whose order 32 bits do not settle, masked rows, strides, streams, graphs.

Tolerances.  Indices and counts are equal.  A gate is a quotient of exponentials: with |z - max| <= 20 each exponential
is within (20 + 2) 2^-24 of its value, the sum of at most 512 of them adds 21 roundings, quotient and scale 2 more:
(22 + 22 + 23) 2^-24 < 2^-17 relative.  A gradient is a sum of two products of such factors with dgates, so it is
within 2 * 2^-17 of scale * max|dgates| * max score, plus half a step of the output type."""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as o
from paper_2403_07816_b200 import binding as B
from util import Guarded, check_guards

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
REL = 2.0 ** -17

# (T, E, k, n_group, topk_group)
SHAPES = [(1, 256, 8, 8, 4), (1, 1, 1, 1, 1), (17, 33, 5, 1, 1), (130, 64, 2, 1, 1), (64, 160, 6, 8, 3), (50, 165, 6, 3, 2),
          (9, 512, 32, 1, 1), (40, 512, 16, 32, 7), (33, 128, 32, 4, 4), (300, 8, 2, 4, 2), (21, 6, 3, 3, 3), (12, 32, 32, 1, 1),
          (5, 62, 1, 31, 1)]


def run(z, k, score, bias=None, n_group=1, topk_group=1, group_score=0, renorm=True, scale=1.0, valid=None, scores=True):
    T, E = z.shape
    desc = B.make_route_desc(T, E, k, z.dtype, score, n_group, topk_group, group_score, renorm, scale)
    bufs = {"topk_idx": Guarded((T, k), torch.int32, z.device), "gates": Guarded((T, k), torch.float32, z.device),
            "counts": Guarded((E,), torch.int32, z.device)}
    if scores:
        bufs["scores"] = Guarded((T, E), torch.float32, z.device)
    B.btx_route(desc, z, bias, bufs["topk_idx"].t, bufs["gates"].t, bufs["scores"].t if scores else None, bufs["counts"].t,
                valid)
    check_guards(bufs, "btx_route")
    return desc, {n: g.t for n, g in bufs.items()}


def compare(z, k, score, bias=None, valid=None, **kw):
    desc, got = run(z, k, score, bias, valid=valid, **kw)
    kw.pop("scores", None)
    want = o.route(z.double().cpu().numpy(), k, score, None if bias is None else bias.double().cpu().numpy(),
                   valid=None if valid is None else valid.cpu().numpy() != 0, **kw)
    assert np.array_equal(got["topk_idx"].cpu().numpy(), want[0])
    assert np.array_equal(got["counts"].cpu().numpy(), want[3])
    np.testing.assert_allclose(got["gates"].double().cpu().numpy(), want[1], rtol=REL, atol=1e-36)
    if "scores" in got:
        np.testing.assert_allclose(got["scores"].double().cpu().numpy(), want[2], rtol=REL, atol=1e-36)
    return desc, got


def logits_of(T, E, dtype, seed, std=1.28):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(T, E, generator=g) * std).to(dtype).to(DEV), (torch.randn(E, generator=g) * 0.1).to(DEV)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("score", [0, 1], ids=["softmax", "sigmoid"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_choice_and_weights(shape, score, dtype):
    T, E, k, G, tg = shape
    z, b = logits_of(T, E, dtype, T * 7 + E)
    for bias in (None, b):
        for gs in ((0, 1) if G > 1 else (0,)):
            compare(z, k, score, bias, n_group=G, topk_group=tg, group_score=gs, renorm=bool(gs) or bias is None,
                    scale=2.5 if gs else 1.0)


@pytest.mark.parametrize("score", [0, 1], ids=["softmax", "sigmoid"])
@pytest.mark.parametrize("G,tg,gs", [(1, 1, 0), (16, 5, 0), (16, 5, 1)])
def test_order_that_fp32_cannot_settle(score, G, tg, gs):
    # scores plus bias fall within a few fp32 steps of one another: most rows are decided in 64 bits
    g = torch.Generator().manual_seed(3)
    z = (torch.randn(600, 128, generator=g) * 2e-6).to(DEV)
    b = (torch.randn(128, generator=g) * 1e-6).to(DEV)
    compare(z, 8, score, b, n_group=G, topk_group=tg, group_score=gs)
    # a bias that undoes the score to the last bit of fp32
    z = torch.randn(1, 128, generator=g)
    s = torch.sigmoid(z.double()) if score else torch.softmax(z.double(), 1)
    compare(z.repeat(5, 1).to(DEV), 8, score, (0.5 - s[0]).float().to(DEV), n_group=G, topk_group=tg, group_score=gs)


@pytest.mark.parametrize("bias", [False, True])
def test_equal_logits_go_to_the_lower_index(bias):
    z = torch.zeros(7, 96, device=DEV)
    z[3] = -0.0
    z[4, 50:] = 1.0
    b = torch.zeros(96, device=DEV) if bias else None
    for score in (0, 1):
        for gs in (0, 1):
            _, got = compare(z, 6, score, b, n_group=8, topk_group=2, group_score=gs)
            assert got["topk_idx"][0].tolist() == list(range(6))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("score", [0, 1], ids=["softmax", "sigmoid"])
def test_masked_experts_and_rows(score, dtype):
    z, b = logits_of(40, 48, dtype, 5)
    z[0] = float("-inf")                                  # nothing left
    z[1, 3:] = float("-inf")                              # fewer experts than slots
    z[2] = float("nan")
    z[3, ::2] = float("nan")
    z[4, 7] = float("inf")
    z[5, [1, 9, 30]] = float("inf")
    z[6] = torch.finfo(dtype).min                         # the type's lowest value is a number, not a mask
    z[7, 6:] = float("-inf")                              # whole groups without a candidate
    z[8, :42] = float("-inf")
    z[9, 1:6] = float("-inf")                             # one candidate in a group
    valid = torch.ones(40, dtype=torch.uint8, device=DEV)
    valid[20:25] = 0
    valid[39] = 0
    z[21] = float("nan")
    for bias in (None, b):
        for gs in (0, 1):
            for renorm in (True, False):
                compare(z, 5, score, bias, valid, n_group=8, topk_group=2, group_score=gs, renorm=renorm, scale=1.5)
                compare(z, 5, score, bias, valid, renorm=renorm)
    off = b.clone()
    off[4], off[9], off[11] = float("-inf"), float("nan"), float("inf")
    compare(z[10:], 5, score, off, valid[10:].contiguous())


def test_weights_of_scores_that_underflow():
    z = torch.full((3, 64), -400.0, device=DEV)
    z += torch.arange(64, device=DEV) * 0.25
    z[1] -= 3.0e4
    for score in (0, 1):
        _, got = compare(z, 4, score, torch.linspace(1, 2, 64, device=DEV), scores=False)
        assert bool((got["gates"].sum(1) - 1).abs().max() < 1e-5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("score", [0, 1], ids=["softmax", "sigmoid"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_gradient(shape, score, renorm, dtype):
    T, E, k, G, tg = shape
    z, b = logits_of(T, E, dtype, T + 3 * E)
    desc, got = run(z, k, score, b, n_group=G, topk_group=tg, renorm=renorm, scale=1.75)
    idx = got["topk_idx"].clone()
    if T > 8:
        idx[2] = -1                                       # a padding row
        idx[3, 0] = -1
        idx[4, k - 1] = E + 5                             # out of range: adds nothing
    dw = torch.randn(T, k, generator=torch.Generator().manual_seed(9)).to(DEV)
    out = Guarded((T, E), dtype, DEV)
    B.btx_route_backward(desc, z, idx, dw, out.t)
    check_guards({"dlogits": out}, "btx_route_backward")
    z64 = z.double().cpu().numpy()
    want = o.route_backward(z64, idx.cpu().numpy(), dw.cpu().numpy(), score, renorm, 1.75)
    smax = 1.0 if renorm or score else max(o.scores_of_row(r, score).max() for r in z64)
    atol = 2 * REL * 1.75 * float(dw.abs().max()) * smax
    err = np.abs(out.t.double().cpu().numpy() - want)
    assert (err <= atol + torch.finfo(dtype).eps / 2 * np.abs(want)).all(), err.max()


def test_strided_rows_in_and_out():
    wide = torch.randn(100, 300, generator=torch.Generator().manual_seed(1)).to(DEV)
    for first, E in ((0, 64), (3, 96), (100, 165)):
        z = wide[:, first:first + E]
        desc, got = compare(z, 4, 1, n_group=3 if E % 3 == 0 else 1, topk_group=2 if E % 3 == 0 else 1)
        dw = torch.ones(100, 4, device=DEV) * torch.arange(4, device=DEV)
        back = torch.full((100, 400), 7.0, device=DEV)
        B.btx_route_backward(desc, z, got["topk_idx"], dw, back[:, 5:5 + E])
        flat = torch.empty(100, E, device=DEV)
        B.btx_route_backward(desc, z.contiguous(), got["topk_idx"], dw, flat)
        assert torch.equal(back[:, 5:5 + E], flat)
        assert bool((back[:, :5] == 7).all()) and bool((back[:, 5 + E:] == 7).all())


def test_no_rows():
    z = torch.empty(0, 16, device=DEV)
    _, got = run(z, 2, 1)
    assert got["counts"].tolist() == [0] * 16


def test_other_stream_capture_and_repeat():
    z, b = logits_of(500, 256, torch.float32, 11)
    kw = dict(n_group=8, topk_group=4, group_score=1, scale=2.5)
    desc, ref = compare(z, 8, 1, b, **kw)
    dw = torch.randn(500, 8, device=DEV)
    dref = torch.empty(500, 256, device=DEV)
    B.btx_route_backward(desc, z, ref["topk_idx"], dw, dref)
    zin = z.clone()
    idx, gates = torch.empty_like(ref["topk_idx"]), torch.empty_like(ref["gates"])
    counts, dz = torch.empty_like(ref["counts"]), torch.empty_like(dref)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        B.btx_route(desc, zin, b, idx, gates, counts=counts)
        B.btx_route_backward(desc, zin, idx, dw, dz)
    side.synchronize()
    assert torch.equal(idx, ref["topk_idx"]) and torch.equal(gates, ref["gates"]) and torch.equal(counts, ref["counts"])
    assert torch.equal(dz, dref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.btx_route(desc, zin, b, idx, gates, counts=counts)
        B.btx_route_backward(desc, zin, idx, dw, dz)
    for seed in (1, 2):
        fresh = torch.randn(500, 256, generator=torch.Generator().manual_seed(seed)).to(DEV)
        zin.copy_(fresh)
        graph.replay()
        _, want = compare(fresh, 8, 1, b, **kw)
        assert torch.equal(idx, want["topk_idx"]) and torch.equal(counts, want["counts"]) and torch.equal(gates, want["gates"])


def test_large_batch_matches_in_every_row():
    z, b = logits_of(20001, 256, torch.float32, 13)
    desc, got = run(z, 8, 1, b, n_group=8, topk_group=4, group_score=1, scores=False)
    s = torch.sigmoid(z.double())
    c = s + b.double()
    g = c.view(-1, 8, 32).topk(2, dim=2)[0].sum(2)
    keep = torch.zeros_like(g).scatter_(1, g.topk(4, dim=1)[1], 1.0).repeat_interleave(32, 1)
    want = c.masked_fill(keep == 0, float("-inf")).topk(8, dim=1)[1]
    assert torch.equal(got["topk_idx"].long(), want)
    assert torch.equal(got["counts"].long(), torch.bincount(want.flatten(), minlength=256))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("score", [0, 1], ids=["softmax", "sigmoid"])
@pytest.mark.parametrize("shape", [(33, 5, 1, 1), (30, 6, 5, 3), (64, 8, 8, 4), (120, 12, 10, 3), (128, 16, 4, 2), (165, 6, 3, 2),
                                   (256, 8, 8, 4), (256, 16, 16, 9), (256, 20, 2, 1), (512, 8, 8, 4)], ids=lambda s: "x".join(map(str, s)))
def test_large_batches_share_a_warp_between_rows(shape, score, dtype):
    # several rows per warp: ordinary rows beside rows that are masked, tied, or not settled by fp32
    E, k, G, tg = shape
    T = 8200
    z, b = logits_of(T, E, dtype, E + k)
    z[5:5000:7] *= 1e-6                                    # scores plus bias within a few fp32 steps where b is
    z[11:5000:13] = 0
    z[17:5000:19] = float("-inf")
    z[23:5000:29, ::3] = float("nan")
    z[31, :] = float("inf")
    valid = torch.ones(T, dtype=torch.uint8, device=DEV)
    valid[3::11] = 0
    rows = np.r_[0:60, 2000:2030, T - 30:T]
    for bias in (None, b, b * 1e-6):
        for gs in (0, 1):
            kw = dict(n_group=G, topk_group=tg, group_score=gs, renorm=bool(gs), scale=1.5)
            _, got = run(z, k, score, bias, valid=valid, scores=False, **kw)
            want = o.route(z[rows].double().cpu().numpy(), k, score, None if bias is None else bias.double().cpu().numpy(),
                           valid=valid.cpu().numpy()[rows] != 0, **kw)
            assert np.array_equal(got["topk_idx"].cpu().numpy()[rows], want[0])
            np.testing.assert_allclose(got["gates"].double().cpu().numpy()[rows], want[1], rtol=REL, atol=1e-36)
            # a batch below the limit runs a warp per row: the same choice
            _, part = run(z[:4000].contiguous(), k, score, bias, valid=valid[:4000].contiguous(), scores=False, **kw)
            assert torch.equal(part["topk_idx"], got["topk_idx"][:4000]) and torch.equal(part["gates"], got["gates"][:4000])
            flat = got["topk_idx"].flatten()
            assert torch.equal(got["counts"].long(), torch.bincount(flat[flat >= 0], minlength=E))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("score,renorm", [(0, True), (0, False), (1, True), (1, False)])
@pytest.mark.parametrize("shape", [(40, 8), (63, 3), (64, 8), (65, 2), (100, 16), (128, 9), (165, 7), (256, 8), (256, 16), (200, 20)],
                         ids=lambda s: "x".join(map(str, s)))
def test_gradient_of_large_batches(shape, score, renorm, dtype):
    # several rows per warp: masked rows, rows without a choice, the same expert twice
    E, k = shape
    T = 8201
    z, _ = logits_of(T, E, dtype, 2 * E + k)
    z[17:5000:19, ::3] = float("-inf")
    z[23:5000:29, ::5] = float("nan")
    _, got = run(z, k, score, None, scores=False, renorm=renorm)
    idx = got["topk_idx"].clone()
    idx[3::13] = -1
    idx[5::7, 0] = E
    idx[6::5, 1] = idx[6::5, 0]
    dw = torch.randn(T, k, generator=torch.Generator().manual_seed(9)).to(DEV)
    mk = lambda n: B.make_route_desc(n, E, k, dtype, score, renorm=renorm, scale=1.75)
    out = Guarded((T, E), dtype, DEV)
    B.btx_route_backward(mk(T), z, idx, dw, out.t)
    check_guards({"dlogits": out}, "btx_route_backward")
    rows = np.r_[0:60, 2000:2040, T - 30:T]
    z64 = z[rows].double().cpu().numpy()
    want = o.route_backward(z64, idx.cpu().numpy()[rows], dw.cpu().numpy()[rows], score, renorm, 1.75)
    atol = 2 * REL * 1.75 * float(dw.abs().max()) * 2          # the same expert in two slots adds two weights
    err = np.abs(out.t.double().cpu().numpy()[rows] - want)
    assert (err <= atol + torch.finfo(dtype).eps / 2 * np.abs(want)).all(), err.max()
    # a batch below the limit runs a warp per row: the same gradient
    part = torch.empty(4000, E, dtype=dtype, device=DEV)
    B.btx_route_backward(mk(4000), z[:4000].contiguous(), idx[:4000].contiguous(), dw[:4000].contiguous(), part)
    assert torch.equal(part, out.t[:4000])


def test_offsets_past_32_bits():
    T, E, k = 4_300_001, 512, 4
    z = torch.empty(T, E, dtype=torch.bfloat16, device=DEV)
    part, b = logits_of(1000, E, torch.bfloat16, 3)
    z[:-1000] = part[0]
    z[-1000:] = part
    _, big = run(z, k, 1, b, scores=False)
    _, small = run(part, k, 1, b, scores=False)
    assert torch.equal(big["topk_idx"][-1000:], small["topk_idx"]) and torch.equal(big["gates"][-1000:], small["gates"])
    assert int(big["counts"].sum()) == T * k
    dw = torch.ones(T, k, device=DEV) * torch.arange(k, device=DEV)
    desc = B.make_route_desc(T, E, k, torch.bfloat16, 1)
    dz = torch.empty_like(z)
    B.btx_route_backward(desc, z, big["topk_idx"], dw, dz)
    dp = torch.empty_like(part)
    B.btx_route_backward(B.make_route_desc(1000, E, k, torch.bfloat16, 1), part, small["topk_idx"], dw[:1000].contiguous(), dp)
    assert torch.equal(dz[-1000:], dp)


def test_binding_refuses_wrong_tensors():
    z = torch.randn(4, 16, device=DEV)
    desc = B.make_route_desc(4, 16, 2, torch.float32)
    idx, g = torch.empty(4, 2, dtype=torch.int32, device=DEV), torch.empty(4, 2, device=DEV)
    for bad in (lambda: B.btx_route(desc, z, None, idx.long(), g), lambda: B.btx_route(desc, z, None, idx[:3], g),
                lambda: B.btx_route(desc, z.half(), None, idx, g), lambda: B.btx_route(desc, z, z[0, :8], idx, g),
                lambda: B.btx_route_backward(desc, z, idx, g.double(), z)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(RuntimeError):
        B.btx_route(B.make_route_desc(16, 4, 2, torch.float32), z.t(), None, torch.empty(16, 2, dtype=torch.int32, device=DEV),
                    torch.empty(16, 2, device=DEV))
