"""BTX_ROUTE_GIVEN: the layer and its gradients under the caller's routing, against a 64-bit statement written here, and
the whole training step score routing -> layer -> d gates -> d logits.  Bars are those of the other parity tests:
max|err| / max|ref| of 1e-5 (FP32) and 1e-2 (BF16) per tensor."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import experts_oracle as eo
from paper_2403_07816_b200 import binding as B
from paper_2403_07816_b200 import synth
from util import TOL, Guarded, check_guards, gpu_backward, gpu_forward, np64, rel_err

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def statement(inp, idx, gates):
    """y and the gradients of <y, dy> in 64 bits."""
    x, w1, w3, w2, dy = (np64(inp[n]) for n in ("x", "w1", "w3", "w2", "dy"))
    E = w1.shape[0]
    out = dict(y=np.zeros_like(x), dx=np.zeros_like(x), dgates=np.zeros(idx.shape), dw1=np.zeros_like(w1), dw3=np.zeros_like(w3),
               dw2=np.zeros_like(w2))
    for e in range(E):
        t, j = np.nonzero(idx == e)
        if len(t) == 0:
            continue
        g = gates[t, j][:, None]
        h1, h3 = x[t] @ w1[e].T, x[t] @ w3[e].T
        s = 1 / (1 + np.exp(-h1))
        a = h1 * s * h3
        f = a @ w2[e].T
        np.add.at(out["y"], t, g * f)
        out["dgates"][t, j] = (f * dy[t]).sum(1)
        da = g * (dy[t] @ w2[e])
        dh1, dh3 = da * h3 * s * (1 + h1 * (1 - s)), da * h1 * s
        np.add.at(out["dx"], t, dh1 @ w1[e] + dh3 @ w3[e])
        out["dw1"][e], out["dw3"][e], out["dw2"][e] = dh1.T @ x[t], dh3.T @ x[t], (g * dy[t]).T @ a
    return out


def run(inp, idx, gates, save=True, frozen=False, cf=0.0, accumulate=False):
    x = inp["x"]
    T, d = x.shape
    E, F, _ = inp["w1"].shape
    k = idx.shape[1]
    desc = B.make_desc(T, d, F, E, k, x.dtype, B.ROUTE_GIVEN, 0.0, save_for_backward=save, skip_wgrad=frozen, capacity_factor=cf)
    wsb, svb = B.btx_moe_sizes(desc)
    bufs = {"workspace": Guarded(wsb, torch.uint8, DEV, fill=0x7F), "saved": Guarded(max(svb, 16), torch.uint8, DEV, fill=0x7F),
            "y": Guarded(x.shape, x.dtype, DEV), "dx": Guarded(x.shape, x.dtype, DEV), "dgates": Guarded((T, k), torch.float32, DEV)}
    r = B.Routing.given(desc, idx, gates)
    ws, saved = bufs["workspace"].t, bufs["saved"].t
    B.btx_moe_forward(desc, x, None, None, inp["w1"], inp["w3"], inp["w2"], bufs["y"].t, r, saved if save else None, ws)
    assert B.btx_device_status(ws) == B.BTX_OK
    check_guards(bufs, "forward")
    out = dict(y=bufs["y"].t, routing=r)
    if save:
        dw = {}
        for n, s in (("dw1", (E, F, d)), ("dw3", (E, F, d)), ("dw2", (E, d, F))):
            if not frozen:
                bufs[n] = Guarded(s, torch.float32, DEV, fill=0.25 if accumulate else None)
            dw[n] = None if frozen else bufs[n].t
        ws.fill_(0x7F)
        B.btx_moe_backward(desc, x, None, None, inp["w1"], inp["w3"], inp["w2"], inp["dy"], 1.0, saved, bufs["dx"].t, None, None,
                           dw["dw1"], dw["dw3"], dw["dw2"], int(accumulate), ws, dlogits=bufs["dgates"].t)
        assert B.btx_device_status(ws) == B.BTX_OK
        check_guards(bufs, "backward")
        out.update(dx=bufs["dx"].t, dgates=bufs["dgates"].t, **dw)
    return out


def routing(T, E, k, seed, kind):
    g = torch.Generator().manual_seed(seed)
    idx = torch.rand(T, E, generator=g).topk(k, 1)[1].to(torch.int32)
    if kind == "empty":
        idx[torch.rand(T, k, generator=g) < 0.4] = -1
        idx[T // 2] = E + 3
    if kind == "twice":
        idx[:, -1] = idx[:, 0]
    if kind == "one":
        idx[:] = 1
    if kind == "none":
        idx[:] = -1
    return idx.to(DEV), (torch.rand(T, k, generator=g) + 0.1).to(DEV)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("kind", ["all", "empty", "twice", "one", "none"])
@pytest.mark.parametrize("shape", [(1, 64, 96, 3, 2), (50, 128, 136, 4, 2), (200, 64, 80, 8, 3), (700, 96, 72, 5, 2),
                                   (120, 64, 96, 64, 8)], ids=lambda s: "x".join(map(str, s)))
def test_layer_and_gradients(shape, kind, dtype):
    T, d, F, E, k = shape
    inp = synth.moe_inputs(T, d, F, E, T + E, dtype, DEV)
    idx, gates = routing(T, E, k, T, kind)
    accumulate, frozen = kind == "empty", kind == "twice" and T == 50
    got = run(inp, idx, gates, accumulate=accumulate, frozen=frozen)
    want = statement(inp, idx.cpu().numpy(), np64(gates))
    for n in ("y", "dx", "dgates", "dw1", "dw3", "dw2"):
        if got[n] is None:
            continue
        ref = want[n] + 0.25 if accumulate and n.startswith("dw") else want[n]
        assert rel_err(np64(got[n]), ref) <= TOL[dtype], n
    kept = (idx >= 0) & (idx < E)
    r = got["routing"]
    flat = idx.flatten().cpu().numpy()
    order = [i for e in range(E) for i in np.nonzero(flat == e)[0]]
    assert r.counts.cpu().tolist() == [int((flat == e).sum()) for e in range(E)]
    perm, inv = r.perm.cpu().numpy(), r.inv_perm.cpu().numpy()
    assert perm[:len(order)].tolist() == order and (perm[len(order):] == -1).all()
    assert (inv[order] == np.arange(len(order))).all() and (inv[~kept.flatten().cpu().numpy()] == -1).all()
    assert torch.equal(run(inp, idx, gates, save=False)["y"], got["y"])      # nothing kept for backward: same kernels


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_agrees_with_the_layers_own_router(dtype):
    for T in (40, 900):
        inp = synth.moe_inputs(T, 128, 96, 4, 3, dtype, DEV)
        fwd = gpu_forward(inp, 2)
        ref = gpu_backward(inp, fwd, lb_scale=0.0)
        got = run(inp, fwd["routing"].topk_idx.contiguous(), fwd["routing"].gates.contiguous())
        assert torch.equal(got["y"], fwd["y"]) and torch.equal(got["routing"].perm, fwd["routing"].perm)
        for n in ("dw1", "dw3", "dw2"):
            assert torch.equal(got[n], ref[n])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T", [60, 900])
def test_rows_without_an_expert_are_not_read(T, dtype):
    # padding tokens may hold anything: it reaches no output and no gradient
    inp = synth.moe_inputs(T, 64, 96, 4, 7, dtype, DEV)
    idx, gates = routing(T, 4, 2, T, "all")
    idx[1::5] = -1
    idx[2, 1] = 9
    clean = run(inp, idx, gates)
    clean = {n: clean[n].clone() for n in ("y", "dx", "dgates", "dw1", "dw3", "dw2")}
    inp["x"][1::5] = float("nan")
    inp["dy"][1::5] = float("inf")
    gates[1::5] = float("nan")
    gates[2, 1] = float("inf")
    got = run(inp, idx, gates)
    for n, ref in clean.items():
        assert torch.equal(got[n], ref), n
    assert bool((got["y"][1::5] == 0).all()) and bool((got["dx"][1::5] == 0).all()) and bool((got["dgates"][1::5] == 0).all())


def test_capacity_limit_applies_to_a_given_routing():
    inp = synth.moe_inputs(64, 64, 96, 4, 3, torch.float32, DEV)
    idx, gates = routing(64, 4, 1, 1, "one")
    got = run(inp, idx, gates, cf=1.0)                   # 16 rows per expert
    assert got["routing"].counts.tolist() == [0, 16, 0, 0]
    cut = idx.cpu().numpy().copy()
    cut[16:] = -1
    want = statement(inp, cut, np64(gates))
    for n in ("y", "dx", "dgates", "dw1", "dw3", "dw2"):
        assert rel_err(np64(got[n]), want[n]) <= 1e-5, n


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("score,renorm", [(0, True), (0, False), (1, True), (1, False)])
def test_training_step_through_score_routing(score, renorm, dtype):
    T, d, F, E, k = 90, 64, 96, 16, 3
    inp = synth.moe_inputs(T, d, F, E, 11, dtype, DEV)
    z = synth.normal((T, E), 1.28, 5, 50, torch.float32, DEV)
    bias = synth.normal((E,), 0.1, 5, 51, torch.float32, DEV)
    desc = B.make_route_desc(T, E, k, torch.float32, score, 4, 2, B.GROUP_SUM2, renorm, 1.5)
    idx, gates = torch.empty(T, k, dtype=torch.int32, device=DEV), torch.empty(T, k, device=DEV)
    counts = torch.empty(E, dtype=torch.int32, device=DEV)
    valid = torch.ones(T, dtype=torch.uint8, device=DEV)
    valid[80:] = 0
    B.btx_route(desc, z, bias, idx, gates, counts=counts, row_valid=valid)
    got = run(inp, idx, gates)
    assert torch.equal(got["routing"].counts, counts)
    dz = torch.empty_like(z)
    B.btx_route_backward(desc, z, idx, got["dgates"], dz)
    i64 = idx.cpu().numpy()
    want = statement(inp, i64, eo.route(np64(z), k, score, np64(bias), 4, 2, 1, renorm, 1.5, valid.cpu().numpy())[1])
    assert rel_err(np64(got["y"]), want["y"]) <= TOL[dtype]
    assert bool((got["y"][80:] == 0).all()) and bool((got["dx"][80:] == 0).all()) and bool((dz[80:] == 0).all())
    ref = eo.route_backward(np64(z), i64, want["dgates"], score, renorm, 1.5)
    assert rel_err(np64(dz), ref) <= TOL[dtype]


def test_given_step_in_a_graph():
    T, d, F, E, k = 300, 64, 96, 8, 2
    inp = synth.moe_inputs(T, d, F, E, 4, torch.bfloat16, DEV)
    idx, gates = routing(T, E, k, 2, "empty")
    ref = run(inp, idx, gates)
    idx2, gates2 = routing(T, E, k, 9, "all")
    ref2 = run(inp, idx2, gates2)
    desc = B.make_desc(T, d, F, E, k, torch.bfloat16, B.ROUTE_GIVEN, 0.0, save_for_backward=True)
    ws, saved = B.alloc_buffers(desc, DEV)
    r = B.Routing.given(desc, idx.clone(), gates.clone())
    y, dx, dg = torch.empty_like(inp["x"]), torch.empty_like(inp["x"]), torch.empty(T, k, device=DEV)
    dw = [torch.empty(s, device=DEV) for s in ((E, F, d), (E, F, d), (E, d, F))]

    def step():
        B.btx_moe_forward(desc, inp["x"], None, None, inp["w1"], inp["w3"], inp["w2"], y, r, saved, ws)
        B.btx_moe_backward(desc, inp["x"], None, None, inp["w1"], inp["w3"], inp["w2"], inp["dy"], 1.0, saved, dx, None, None,
                           dw[0], dw[1], dw[2], 0, ws, dlogits=dg)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for (i, g), want in (((idx2, gates2), ref2), ((idx, gates), ref)):
        r.topk_idx.copy_(i)
        r.gates.copy_(g)
        graph.replay()
        assert torch.equal(y, want["y"]) and torch.equal(dx, want["dx"]) and torch.equal(dg, want["dgates"])
        assert torch.equal(dw[0], want["dw1"]) and torch.equal(dw[2], want["dw2"])


def test_refusals():
    inp = synth.moe_inputs(8, 64, 96, 4, 3, torch.float32, DEV)
    desc = B.make_desc(8, 64, 96, 4, 2, torch.float32, B.ROUTE_GIVEN, 0.0)
    ws, _ = B.alloc_buffers(desc, DEV)
    y = torch.empty(8, 64, device=DEV)
    with pytest.raises(B.BtxError) as ei:
        B.btx_moe_forward(desc, inp["x"], None, None, inp["w1"], inp["w3"], inp["w2"], y, None, None, ws)
    assert ei.value.status == 1
    with pytest.raises(ValueError):
        B.Routing.given(desc, torch.zeros(8, 3, dtype=torch.int32, device=DEV), torch.zeros(8, 2, device=DEV))
