"""What is measured of the expert-routing and 4-bit (MXFP4) expert operators, and their plain forms.

Five operators, each as a user's program calls it:

  route           scores (softmax or sigmoid) of the router logits, a balance bias that only takes part in the choice,
                  expert groups, top-k, renormalised weights, tokens per expert
  route_backward  the gradient with respect to the logits, from the gradient with respect to the weights
  cast            a tensor to MXFP4 (e2m1 elements, one power-of-two scale per 32 of them) and the values read back
  product         y = x W^T with W held in MXFP4 and x cast to MXFP4 within the call
  moe             the SwiGLU expert layer with MXFP4 experts under a given routing

`run` computes them in elementary torch operations (`own = False`) or through the library (`own = True`).
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
BLOCK = 32                     # elements that share a scale


# ------------------------------------------------------------------------------------------------
# Cases
# ------------------------------------------------------------------------------------------------
def _route(T, E, k, score, dtype, bias=True, n_group=1, topk_group=1, group_score="max", renorm=True, scale=1.0,
           padded=0.0, op="route"):
    return dict(op=op, T=T, E=E, k=k, score=score, dtype=dtype, bias=bias, n_group=n_group, topk_group=topk_group,
                group_score=group_score, renorm=renorm, scale=scale, padded=padded)


def listed():
    return [
        # one decoding step of one sequence through a router of many small experts: pure latency
        dict(_route(1, 256, 8, "sigmoid", "f32", True, 8, 4, "sum2", True, 2.5), name="route_one_token"),
        # a training batch of four sequences of 4096, few experts, logits as a bf16 layer leaves them
        dict(_route(16384, 64, 2, "softmax", "bf16", False), name="route_softmax_train"),
        # the same batch with grouped sigmoid routing balanced by a bias, an eighth of it padding
        dict(_route(16384, 256, 8, "sigmoid", "f32", True, 8, 4, "sum2", True, 2.5, 0.125), name="route_grouped_train"),
        # training: plain softmax weights, whose gradient reaches every logit
        dict(_route(16384, 256, 8, "softmax", "f32", True, 1, 1, "max", False, 1.0, 0.0, "route_backward"),
             name="route_backward_softmax"),
        # a ragged batch with an odd number of experts, gradients in bf16
        dict(_route(777, 165, 6, "sigmoid", "bf16", True, 3, 2, "max", True, 1.0, 0.0, "route_backward"),
             name="route_backward_ragged"),
        # the activations of one decoding step
        dict(op="cast", batch=1, rows=32, K=4096, dtype="bf16", name="cast_decode_activations"),
        # the up matrices of four experts, once at load time
        dict(op="cast", batch=4, rows=11008, K=4096, dtype="bf16", name="cast_expert_weights"),
        # one token through a down projection
        dict(op="product", M=1, N=4096, K=11008, dtype="bf16", name="product_one_token"),
        # odd sizes everywhere, fp32 in and out
        dict(op="product", M=333, N=1001, K=2080, dtype="f32", name="product_ragged"),
        # two sequences of 4096 through an up projection
        dict(op="product", M=8192, N=11008, K=4096, dtype="bf16", name="product_prefill"),
        # a decoding batch: every expert's weights are read for a handful of tokens each
        dict(op="moe", T=32, d=4096, F=11008, E=4, k=2, dtype="bf16", name="moe_decode"),
        # one sequence of 4096 through the layer
        dict(op="moe", T=4096, d=4096, F=11008, E=4, k=2, dtype="bf16", name="moe_prefill"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["route", "route", "route_backward", "cast", "product", "product", "moe", "moe"])
    if op in ("route", "route_backward"):
        n_group = rng.choice([1, 1, 2, 3, 4, 8])
        per = _log_int(rng, 2, 512 // n_group)
        E = n_group * per
        topk_group = rng.randint(1, n_group)
        k = rng.randint(1, min(16, topk_group * per))
        T = min(_log_int(rng, 1, 32768), (16384 * 256) // E)
        return _route(max(1, T), E, k, rng.choice(["softmax", "sigmoid"]), rng.choice(["f32", "bf16"]),
                      rng.random() < 0.7, n_group, topk_group, rng.choice(["max", "sum2"]), rng.random() < 0.6,
                      rng.choice([1.0, 2.5]), rng.choice([0.0, 0.0, 0.3]), op)
    if op == "cast":
        batch, K = rng.randint(1, 4), BLOCK * _log_int(rng, 2, 344)
        rows = min(_log_int(rng, 1, 11008), (4 * 11008 * 4096) // (batch * K))
        return dict(op=op, batch=batch, rows=max(1, rows), K=K, dtype=rng.choice(["f32", "bf16"]))
    if op == "product":
        M, N, K = _log_int(rng, 1, 8192), _log_int(rng, 16, 11008), BLOCK * _log_int(rng, 2, 344)
        M = max(1, min(M, (8192 * 11008 * 4096) // (N * K)))
        return dict(op=op, M=M, N=N, K=K, dtype=rng.choice(["f32", "bf16"]))
    E = _log_int(rng, 1, 64)
    k = rng.randint(1, min(8, E))
    d, F = BLOCK * _log_int(rng, 4, 128), BLOCK * _log_int(rng, 4, 344)
    F = max(BLOCK, min(F, (4 * 11008 * 4096) // (E * d) // BLOCK * BLOCK))
    T = min(_log_int(rng, 1, 4096), (4096 * 2 * 4096 * 11008) // (k * d * F))
    return dict(op=op, T=max(1, T), d=d, F=F, E=E, k=k, dtype=rng.choice(["f32", "bf16"]))


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    op = case["op"]
    if op == "route":
        T, E, k = case["T"], case["E"], case["k"]
        return {"bytes": T * E * size + (4 * E if case["bias"] else 0) + 8 * T * k + 4 * E + T * (case["padded"] > 0),
                "flops": 4 * T * E}
    if op == "route_backward":
        T, E, k = case["T"], case["E"], case["k"]
        dense = case["score"] == "softmax" and not case["renorm"]      # else only the chosen logits are needed
        return {"bytes": (T * E if dense else T * k) * size + 8 * T * k + T * E * size, "flops": 4 * T * E}
    if op == "cast":
        n = case["batch"] * case["rows"] * case["K"]
        return {"bytes": 2 * n * size + n * 17 // 32, "flops": 2 * n}
    if op == "product":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": M * K * size + N * K * 17 // 32 + M * N * size, "flops": 2 * M * N * K}
    T, d, F, E, k = (case[n] for n in ("T", "d", "F", "E", "k"))
    used = E * (1.0 - (1.0 - k / E) ** T)                               # experts that hold a token
    return {"bytes": int(2 * T * d * size + 8 * T * k + used * 3 * d * F * 17 / 32), "flops": 6 * T * k * d * F}


# ------------------------------------------------------------------------------------------------
# Inputs
# ------------------------------------------------------------------------------------------------
def _gen(seed, tensor):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + tensor)
    return g


def _normal(shape, std, seed, tensor, dtype):
    return torch.randn(shape, generator=_gen(seed, tensor), device=DEV, dtype=torch.float32).mul_(std).to(dtype)


def _inputs(case, seed):
    """The data of a case: activations ~ N(0, 1), weights ~ N(0, 0.02^2), and router logits as such activations of
    width 4096 and such weights give them, N(0, 1.28^2)."""
    dt, op = _dtype(case), case["op"]
    if op in ("route", "route_backward"):
        T, E, k = case["T"], case["E"], case["k"]
        out = {"logits": _normal((T, E), 1.28, seed, 1, dt),
               "bias": _normal((E,), 0.1, seed, 2, torch.float32) if case["bias"] else None, "valid": None}
        if case["padded"] > 0:
            v = torch.ones(T, dtype=torch.uint8, device=DEV)
            v[T - int(T * case["padded"]):] = 0
            out["valid"] = v
        if op == "route_backward":
            out["dgates"] = _normal((T, k), 1.0, seed, 3, torch.float32)
        return out
    if op == "cast":
        return {"x": _normal((case["batch"], case["rows"], case["K"]), 0.02, seed, 1, dt)}
    if op == "product":
        return {"x": _normal((case["M"], case["K"]), 1.0, seed, 1, dt),
                "w": _normal((1, case["N"], case["K"]), 0.02, seed, 2, dt)}
    T, d, F, E, k = (case[n] for n in ("T", "d", "F", "E", "k"))
    z = _normal((T, E), 1.28, seed, 5, torch.float32)
    top, idx = torch.sort(z, dim=1, descending=True, stable=True)
    return {"x": _normal((T, d), 1.0, seed, 1, dt), "w1": _normal((E, F, d), 0.02, seed, 2, dt),
            "w3": _normal((E, F, d), 0.02, seed, 3, dt), "w2": _normal((E, d, F), 0.02, seed, 4, dt),
            "topk_idx": idx[:, :k].to(torch.int32).contiguous(), "gates": torch.softmax(top[:, :k], 1).contiguous()}


def _route_desc(B, case):
    return B.make_route_desc(case["T"], case["E"], case["k"], _dtype(case),
                             score=B.SCORE_SOFTMAX if case["score"] == "softmax" else B.SCORE_SIGMOID,
                             n_group=case["n_group"], topk_group=case["topk_group"],
                             group_score=B.GROUP_MAX if case["group_score"] == "max" else B.GROUP_SUM2,
                             renorm=case["renorm"], scale=case["scale"])


def prepare(case, seed):
    s, op, dt = _inputs(case, seed), case["op"], _dtype(case)
    s["case"] = case
    if op == "route_backward":                             # the forward's choice is in hand
        s["topk_idx"] = _plain_route(s)[0]
    if not own:
        # the plain forms keep 4-bit weights as the values they stand for (exact in bf16)
        for name in ("w", "w1", "w2", "w3"):
            if name in s:
                s[name] = _by_slices(_mx4_values, s[name], torch.bfloat16)
        return s
    from paper_2403_07816_b200 import binding as B
    s["B"] = B
    if op in ("route", "route_backward"):
        T, E, k = case["T"], case["E"], case["k"]
        s["desc"] = _route_desc(B, case)
        if op == "route":
            s["topk_idx"] = torch.empty((T, k), dtype=torch.int32, device=DEV)
            s["gates"] = torch.empty((T, k), dtype=torch.float32, device=DEV)
            s["counts"] = torch.empty(E, dtype=torch.int32, device=DEV)
        else:
            s["dlogits"] = torch.empty((T, E), dtype=dt, device=DEV)
    elif op == "cast":
        s["q"] = B.Mx4.empty(case["batch"], case["rows"], case["K"], DEV)
        s["values"] = torch.empty_like(s["x"])
    elif op == "product":
        M, N, K = case["M"], case["N"], case["K"]
        s["wq"] = B.Mx4.empty(1, N, K, DEV)
        B.btx_mx4_quantize(s.pop("w"), s["wq"])
        s["xq"] = B.Mx4.empty(1, M, K, DEV)
        s["y"] = torch.empty((M, N), dtype=dt, device=DEV)
        s["ws"] = torch.empty(B.btx_mx4_matmul_workspace_size(M, N, K, dt), dtype=torch.uint8, device=DEV)
    else:
        T, d, F, E, k = (case[n] for n in ("T", "d", "F", "E", "k"))
        s["w13"] = B.Mx4.empty(E, 2 * F, d, DEV)           # rows of W1 and W3 in turn
        B.btx_mx4_quantize(s.pop("w1"), s["w13"], row_first=0, row_step=2)
        B.btx_mx4_quantize(s.pop("w3"), s["w13"], row_first=1, row_step=2)
        s["w2q"] = B.Mx4.empty(E, d, F, DEV)
        B.btx_mx4_quantize(s.pop("w2"), s["w2q"])
        s["desc"] = B.make_mx4_moe_desc(T, d, F, E, k, dt)
        s["y"] = torch.empty((T, d), dtype=dt, device=DEV)
        s["ws"] = torch.empty(B.btx_mx4_moe_workspace_size(s["desc"]), dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------
# Plain forms
# ------------------------------------------------------------------------------------------------
def _by_slices(fn, x, dtype):
    """fn over the leading index of x: bounds the memory of the plain cast of large weights."""
    out = torch.empty(x.shape, dtype=dtype, device=x.device)
    for i in range(x.shape[0]):
        out[i] = fn(x[i])
    return out


def _mx4_values(x):
    """The values that x's MXFP4 form stands for, in fp32: per 32 elements the scale 2^(floor(log2 max|x|) - 2), not
    below 2^-127, and x / scale to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (ties to the even code, 6 at most)."""
    v = x.float().unflatten(-1, (-1, BLOCK))
    amax = v.abs().amax(-1, keepdim=True)
    exp = torch.where(amax > 0, torch.frexp(amax)[1] - 3, -127).clamp_(min=-127)
    p = torch.ldexp(v, -exp)
    a = p.abs()
    q = torch.zeros_like(a)
    for above, value in ((a > 0.25, 0.5), (a >= 0.75, 1.0), (a > 1.25, 1.5), (a >= 1.75, 2.0), (a > 2.5, 3.0),
                         (a >= 3.5, 4.0), (a > 5.0, 6.0)):
        q = torch.where(above, value, q)
    return torch.ldexp(torch.where(p < 0, -q, q), exp).flatten(-2)


def _plain_route(s):
    """Scores and keys in 64 bits: which expert is chosen is decided between values that lie close together."""
    c = s["case"]
    z = s["logits"].double()
    E, k, G = c["E"], c["k"], c["n_group"]
    score = torch.sigmoid(z) if c["score"] == "sigmoid" else torch.softmax(z, 1)
    key = z if s["bias"] is None else score + s["bias"].double()
    if G > 1:
        by_group = (score if s["bias"] is None and c["group_score"] == "sum2" else key).view(-1, G, E // G)
        best = by_group.sort(dim=2, descending=True)[0]
        g = best[:, :, 0] if c["group_score"] == "max" or E == G else best[:, :, 0] + best[:, :, 1]
        kept = g.sort(dim=1, descending=True, stable=True)[1][:, :c["topk_group"]]
        mask = torch.zeros_like(g).scatter_(1, kept, 1.0).repeat_interleave(E // G, dim=1)
        key = torch.where(mask > 0, key, -math.inf)
    idx = key.sort(dim=1, descending=True, stable=True)[1][:, :k]
    w = score.gather(1, idx)
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True)
    w = (w * c["scale"]).float()
    idx = idx.to(torch.int32)
    if s["valid"] is not None:
        off = s["valid"][:, None] == 0
        idx, w = idx.masked_fill(off, -1), w.masked_fill(off, 0.0)
    experts = torch.arange(E, device=z.device, dtype=torch.int32)
    counts = torch.zeros(E, dtype=torch.int32, device=z.device)
    for j in range(k):
        counts += (idx[:, j, None] == experts).sum(0).to(torch.int32)
    return idx, w, counts


def _plain_route_backward(s):
    c = s["case"]
    z = s["logits"].float()
    chosen = (s["topk_idx"] >= 0).float()
    idx = s["topk_idx"].clamp(min=0).long()
    dw = s["dgates"] * chosen * c["scale"]
    e = torch.exp(z - z.amax(1, keepdim=True))
    score = 1.0 / (1.0 + torch.exp(-z)) if c["score"] == "sigmoid" else e / e.sum(1, keepdim=True)
    sel = score.gather(1, idx) * chosen
    ds = dw
    if c["renorm"]:
        total = sel.sum(1, keepdim=True).clamp(min=torch.finfo(torch.float32).tiny)
        ds = chosen * (dw - (dw * sel).sum(1, keepdim=True) / total) / total
    dscore = torch.zeros_like(z).scatter_add_(1, idx, ds)
    if c["score"] == "sigmoid":
        dz = dscore * score * (1.0 - score)
    elif c["renorm"]:                                      # the inner product with the scores is zero
        dz = dscore * score
    else:
        dz = score * (dscore - (dscore * score).sum(1, keepdim=True))
    return dz.to(s["logits"].dtype)


def _plain_moe(s):
    c = s["case"]
    F = c["F"]
    x = _mx4_values(s["x"])
    rows = torch.zeros((c["T"], c["k"], c["d"]), dtype=torch.float32, device=x.device)
    for e in range(c["E"]):
        t, slot = (s["topk_idx"] == e).nonzero(as_tuple=True)
        if t.numel() == 0:
            continue
        xe = x[t]
        h1, h3 = xe @ s["w1"][e].float().t(), xe @ s["w3"][e].float().t()
        act = _mx4_values(h1 / (1.0 + torch.exp(-h1)) * h3)
        rows[t, slot] = (act @ s["w2"][e].float().t()) * s["gates"][t, slot][:, None]
    return rows.sum(1).to(s["x"].dtype)


def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        if op == "route":
            return _plain_route(s)
        if op == "route_backward":
            return _plain_route_backward(s)
        if op == "cast":
            return _by_slices(_mx4_values, s["x"], s["x"].dtype)
        if op == "product":
            return (_mx4_values(s["x"]) @ s["w"][0].float().t()).to(s["x"].dtype)
        return _plain_moe(s)
    B = s["B"]
    if op == "route":
        B.btx_route(s["desc"], s["logits"], s["bias"], s["topk_idx"], s["gates"], counts=s["counts"], row_valid=s["valid"])
        return s["topk_idx"], s["gates"], s["counts"]
    if op == "route_backward":
        B.btx_route_backward(s["desc"], s["logits"], s["topk_idx"], s["dgates"], s["dlogits"])
        return s["dlogits"]
    if op == "cast":
        B.btx_mx4_quantize(s["x"], s["q"])
        B.btx_mx4_dequantize(s["q"], s["values"])
        return s["values"]
    if op == "product":
        B.btx_mx4_quantize(s["x"], s["xq"])
        B.btx_mx4_matmul(s["xq"], s["wq"], s["y"], s["ws"])
        return s["y"]
    B.btx_mx4_moe_forward(s["desc"], s["x"], s["topk_idx"], s["gates"], s["w13"], s["w2q"], s["y"], s["ws"])
    return s["y"]


# ------------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ------------------------------------------------------------------------------------------------
def _exact_mx4(x):
    """MXFP4 values in fp64: rounding to the spacing of e2m1 at each value's size (half to even)."""
    v = x.double().unflatten(-1, (-1, BLOCK))
    amax = v.abs().amax(-1, keepdim=True)
    scale = torch.exp2(torch.floor(torch.log2(amax.clamp(min=2.0 ** -149))).sub_(2).clamp_(min=-127))
    p = v / scale
    step = torch.exp2(torch.floor(torch.log2(p.abs().clamp(min=1.0))) - 1)
    return (torch.round(p / step) * step).clamp_(-6.0, 6.0).mul_(scale).flatten(-2)


def _exact_route(case, s):
    z = s["logits"].double().cpu().numpy()
    b = None if s["bias"] is None else s["bias"].double().cpu().numpy()
    valid = np.ones(len(z), bool) if s["valid"] is None else s["valid"].cpu().numpy() > 0
    T, E = z.shape
    k, G = case["k"], case["n_group"]
    if case["score"] == "sigmoid":
        score = np.reciprocal(1.0 + np.exp(-z))
    else:
        score = np.exp(z - z.max(1, keepdims=True))
        score /= score.sum(1, keepdims=True)
    key = z if b is None else score + b
    if G > 1:
        size = E // G
        per = (score if b is None and case["group_score"] == "sum2" else key).reshape(T, G, size)
        take = 1 if case["group_score"] == "max" else min(2, size)
        group = np.partition(per, size - take, axis=2)[:, :, size - take:].sum(2)
        rank = np.argsort(np.argsort(-group, axis=1, kind="stable"), axis=1)
        key = np.where(np.repeat(rank < case["topk_group"], size, axis=1), key, -np.inf)
    idx = np.argsort(-key, axis=1, kind="stable")[:, :k]
    w = np.take_along_axis(score, idx, 1)
    if case["renorm"]:
        w = w / w.sum(1, keepdims=True)
    w = np.where(valid[:, None], w * case["scale"], 0.0)
    idx = np.where(valid[:, None], idx, -1).astype(np.int32)
    counts = np.bincount(idx[valid].ravel(), minlength=E).astype(np.int32)
    return torch.from_numpy(idx), torch.from_numpy(w), torch.from_numpy(counts)


def _exact_route_backward(case, s):
    """From the derivative of the log of a weight: d w_j / d z = w_j d(log w_j) / d z."""
    z = s["logits"].double().cpu().numpy()
    idx = _exact_route(case, s)[0].numpy().astype(np.int64)
    dw = np.where(idx >= 0, s["dgates"].double().cpu().numpy(), 0.0)
    idx = np.maximum(idx, 0)                               # a padding row has no choice and no gradient
    zs = np.take_along_axis(z, idx, 1)
    out = np.zeros_like(z)
    if case["score"] == "sigmoid":
        score = np.reciprocal(1.0 + np.exp(-zs))
        w = score / score.sum(1, keepdims=True) if case["renorm"] else score
        dlog = case["scale"] * dw * w                      # gradient of log(score_j)
        if case["renorm"]:
            dlog = dlog - w * dlog.sum(1, keepdims=True)
        np.put_along_axis(out, idx, dlog * (1.0 - score), 1)
    else:
        over = zs if case["renorm"] else z
        top = over.max(1, keepdims=True)
        w = np.exp(zs - top) / np.exp(over - top).sum(1, keepdims=True)
        dlog = case["scale"] * dw * w
        total = dlog.sum(1, keepdims=True)
        if case["renorm"]:
            np.put_along_axis(out, idx, dlog - w * total, 1)
        else:
            np.put_along_axis(out, idx, dlog, 1)
            out -= np.exp(z - top) / np.exp(z - top).sum(1, keepdims=True) * total
    return torch.from_numpy(out)


def exact(case, seed):
    s, op = _inputs(case, seed), case["op"]
    if op == "route":
        return _exact_route(case, s)
    if op == "route_backward":
        return _exact_route_backward(case, s)
    if op == "cast":
        return _by_slices(_exact_mx4, s["x"], torch.float64)
    if op == "product":
        return _exact_mx4(s["x"]) @ _exact_mx4(s["w"][0]).t()
    x = _exact_mx4(s["x"])
    y = torch.zeros_like(x)
    for e in range(case["E"]):
        gate = (s["gates"].double() * (s["topk_idx"] == e)).sum(1)
        t = (s["topk_idx"] == e).any(1).nonzero().flatten()
        if t.numel() == 0:
            continue
        h1 = x[t] @ _exact_mx4(s["w1"][e]).t()
        h3 = x[t] @ _exact_mx4(s["w3"][e]).t()
        act = _exact_mx4(h1 * torch.sigmoid(h1) * h3)
        y[t] += gate[t, None] * (act @ _exact_mx4(s["w2"][e]).t())
    return y
