"""What is measured of the 8-bit (FP8) path of the feed-forward sublayer and of the norm in front of it, and their plain forms.

Five operators, each as a user's program calls it:

  norm            h = x + residual, y = h / sqrt(mean h^2 + eps) * w, and y in FP8 for the products behind it
  norm_backward   gradients with respect to the norm's input and its weight, the residual stream's own gradient added
  cast            a tensor to FP8 (e4m3 elements, one power-of-two scale per 128 of a row, or per 128 x 128 block), as it
                  stands and transposed, and the values read back
  product         a linear layer with both operands in FP8: y = x W^T, or both gradients from dy; activations and
                  gradients are cast within the call
  moe             the SwiGLU expert layer with FP8 experts under a given routing

`run` computes them in elementary torch operations (`own = False`) or through the library (`own = True`).  Values of FP8
tensors are returned in bf16, which holds them exactly.
"""
import math

import torch

own = False

DEV = "cuda"
BLOCK = 128                    # elements that share a scale
EPS = 1e-5


# ------------------------------------------------------------------------------------------------
# Cases
# ------------------------------------------------------------------------------------------------
def listed():
    return [
        # one decoding step of one sequence: residual, norm, and the FP8 input of the products behind it; pure latency
        dict(op="norm", T=1, d=4096, dtype="bf16", residual=True, fp8=True, name="norm_one_token"),
        # a training batch of four sequences of 4096
        dict(op="norm", T=16384, d=4096, dtype="bf16", residual=True, fp8=True, name="norm_train"),
        # the same batch on its way back, the gradient of the residual stream added
        dict(op="norm_backward", T=16384, d=4096, dtype="bf16", residual=True, name="norm_backward_train"),
        # a ragged batch of odd width in fp32, the first norm of a network (nothing joins its gradient)
        dict(op="norm_backward", T=777, d=1365, dtype="f32", residual=False, name="norm_backward_ragged"),
        # activations of a training batch, along the tokens too for the weight gradient
        dict(op="cast", batch=1, rows=16384, K=4096, dtype="bf16", block=1, both=True, name="cast_train_activations"),
        # the up matrices of two experts, in blocks of 128 x 128, once after an update: forward and input gradient
        dict(op="cast", batch=2, rows=11008, K=4096, dtype="f32", block=128, both=True, name="cast_expert_weights"),
        # one token through a down projection
        dict(op="product", M=1, N=4096, K=11008, dtype="bf16", direction="forward", name="product_one_token"),
        # odd sizes everywhere, fp32 in and out
        dict(op="product", M=333, N=1001, K=2083, dtype="f32", direction="forward", name="product_ragged"),
        # two sequences of 4096 through an up projection
        dict(op="product", M=8192, N=11008, K=4096, dtype="bf16", direction="forward", name="product_prefill"),
        # a micro-batch of odd length on its way back through it: input gradient and weight gradient
        dict(op="product", M=4001, N=11008, K=4096, dtype="bf16", direction="backward", name="product_backward"),
        # a decoding batch: every expert's weights are read for a handful of tokens each
        dict(op="moe", T=32, d=4096, F=11008, E=4, k=2, dtype="bf16", name="moe_decode"),
        # one sequence of 4096 through the layer
        dict(op="moe", T=4096, d=4096, F=11008, E=4, k=2, dtype="bf16", name="moe_prefill"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_backward", "cast", "product", "product", "product", "moe", "moe"])
    dtype = rng.choice(["f32", "bf16"])
    if op in ("norm", "norm_backward"):
        d = _log_int(rng, 32, 16384)
        T = max(1, min(_log_int(rng, 1, 16384), 16384 * 4096 * 2 // (d * (4 if dtype == "f32" else 2))))
        case = dict(op=op, T=T, d=d, dtype=dtype, residual=rng.random() < 0.7)
        return case if op == "norm_backward" else dict(case, fp8=rng.random() < 0.6)
    if op == "cast":
        batch, K = rng.randint(1, 4), _log_int(rng, 17, 11008)
        rows = max(1, min(_log_int(rng, 1, 16384), 16384 * 4096 // (batch * K)))
        return dict(op=op, batch=batch, rows=rows, K=K, dtype=dtype, block=rng.choice([1, 128]), both=rng.random() < 0.5)
    if op == "product":
        direction = rng.choice(["forward", "forward", "backward"])
        M, N, K = _log_int(rng, 1, 8192), _log_int(rng, 16, 11008), _log_int(rng, 16, 11008)
        most = 8192 * 11008 * 4096 // (1 if direction == "forward" else 2)
        return dict(op=op, M=max(1, min(M, most // (N * K))), N=N, K=K, dtype=dtype, direction=direction)
    E = _log_int(rng, 1, 64)
    k = rng.randint(1, min(8, E))
    d, F = 16 * _log_int(rng, 4, 256), 16 * _log_int(rng, 4, 688)
    F = max(16, min(F, (4 * 11008 * 4096) // (E * d) // 16 * 16))
    T = min(_log_int(rng, 1, 4096), (4096 * 2 * 4096 * 11008) // (k * d * F))
    return dict(op=op, T=max(1, T), d=d, F=F, E=E, k=k, dtype="bf16")


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _fp8_bytes(rows, K):
    return rows * K + rows * ((K + BLOCK - 1) // BLOCK)


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    op = case["op"]
    if op == "norm":
        n, res = case["T"] * case["d"], case["residual"]
        return {"bytes": n * size * (4 if res else 2) + case["d"] * size + ((2 * n + _fp8_bytes(case["T"], case["d"])) if case["fp8"] else 0),
                "flops": 4 * n}
    if op == "norm_backward":
        n = case["T"] * case["d"]
        return {"bytes": n * size * (4 if case["residual"] else 3) + case["d"] * (size + 4), "flops": 10 * n}
    if op == "cast":
        batch, rows, K = case["batch"], case["rows"], case["K"]
        n = batch * rows * K
        out = 2 * n + batch * _fp8_bytes(rows, K)
        out_t = (2 * n + batch * _fp8_bytes(K, rows)) if case["both"] else 0
        return {"bytes": n * size + out + out_t, "flops": 2 * n}
    if op == "product":
        M, N, K = case["M"], case["N"], case["K"]
        if case["direction"] == "forward":
            return {"bytes": M * K * size + _fp8_bytes(N, K) + M * N * size, "flops": 2 * M * N * K}
        return {"bytes": M * N * size + 2 * M * K * size + _fp8_bytes(K, N) + 4 * N * K, "flops": 4 * M * N * K}
    T, d, F, E, k = (case[n] for n in ("T", "d", "F", "E", "k"))
    used = E * (1.0 - (1.0 - k / E) ** T)                               # experts that hold a token
    return {"bytes": int(2 * T * d * size + 8 * T * k + used * 3 * d * F * 129 / 128), "flops": 6 * T * k * d * F}


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
    """The data of a case: activations ~ N(0, 1) (the residual stream wider, as it grows with depth), weights ~
    N(0, 0.02^2), norm weights around 1, gradients ~ N(0, 0.01^2), router logits ~ N(0, 1.28^2)."""
    dt, op = _dtype(case), case["op"]
    if op in ("norm", "norm_backward"):
        T, d = case["T"], case["d"]
        out = {"w": (1.0 + _normal((d,), 0.1, seed, 3, torch.float32)).to(dt)}
        if op == "norm":
            out["x"] = _normal((T, d), 1.0, seed, 1, dt)
            out["residual"] = _normal((T, d), 4.0, seed, 2, dt) if case["residual"] else None
        else:
            out["h"] = _normal((T, d), 4.0, seed, 1, dt)
            out["dy"] = _normal((T, d), 0.01, seed, 2, dt)
            out["dh"] = _normal((T, d), 0.01, seed, 4, dt) if case["residual"] else None
        return out
    if op == "cast":
        return {"x": _normal((case["batch"], case["rows"], case["K"]), 0.02 if case["block"] > 1 else 1.0, seed, 1, dt)}
    if op == "product":
        M, N, K = case["M"], case["N"], case["K"]
        out = {"x": _normal((M, K), 1.0, seed, 1, dt), "w": _normal((N, K), 0.02, seed, 2, dt)}
        if case["direction"] == "backward":
            out["dy"] = _normal((M, N), 0.01, seed, 3, dt)
        return out
    T, d, F, E, k = (case[n] for n in ("T", "d", "F", "E", "k"))
    top, idx = torch.sort(_normal((T, E), 1.28, seed, 5, torch.float32), dim=1, descending=True, stable=True)
    return {"x": _normal((T, d), 1.0, seed, 1, dt), "w1": _normal((E, F, d), 0.02, seed, 2, dt),
            "w3": _normal((E, F, d), 0.02, seed, 3, dt), "w2": _normal((E, d, F), 0.02, seed, 4, dt),
            "topk_idx": idx[:, :k].to(torch.int32).contiguous(), "gates": torch.softmax(top[:, :k], 1).contiguous()}


def prepare(case, seed):
    s, op, dt = _inputs(case, seed), case["op"], _dtype(case)
    s["case"] = case
    if not own:
        # the plain forms keep 8-bit weights as the values they stand for (exact in bf16)
        if op in ("product", "moe"):
            for name in ("w", "w1", "w2", "w3"):
                if name in s:
                    s[name] = _block_values(s[name]).to(torch.bfloat16)
        return s
    from paper_2403_07816_b200 import binding as B
    s["B"] = B
    workspace = lambda n: torch.empty(n, dtype=torch.uint8, device=DEV)
    if op == "norm":
        T, d = case["T"], case["d"]
        s["desc"] = B.make_norm_desc(T, d, dt, EPS)
        s["h"] = torch.empty_like(s["x"]) if case["residual"] else None
        s["y"] = torch.empty_like(s["x"])
        if case["fp8"]:
            s["q"] = B.Fp8.empty(1, T, d, DEV)
            s["values"] = torch.empty((T, d), dtype=torch.bfloat16, device=DEV)
    elif op == "norm_backward":
        s["desc"] = B.make_norm_desc(case["T"], case["d"], dt, EPS)
        s["dx"] = torch.empty_like(s["h"])
        s["dw"] = torch.empty(case["d"], dtype=torch.float32, device=DEV)
        s["ws"] = workspace(B.btx_rms_norm_backward_workspace_size(s["desc"]))
    elif op == "cast":
        batch, rows, K = s["x"].shape
        s["q"], s["values"] = B.Fp8.empty(batch, rows, K, DEV), torch.empty((batch, rows, K), dtype=torch.bfloat16, device=DEV)
        if case["both"]:
            s["qt"], s["values_t"] = B.Fp8.empty(batch, K, rows, DEV), torch.empty((batch, K, rows), dtype=torch.bfloat16, device=DEV)
    elif op == "product":
        M, N, K = case["M"], case["N"], case["K"]
        if case["direction"] == "forward":
            s["wq"], s["xq"] = B.Fp8.empty(1, N, K, DEV), B.Fp8.empty(1, M, K, DEV)
            B.btx_fp8_quantize(s.pop("w"), s["wq"], block_rows=BLOCK)
            s["y"] = torch.empty((M, N), dtype=dt, device=DEV)
            s["ws"] = workspace(B.btx_fp8_matmul_workspace_size(M, N, K, dt))
        else:
            s["wt"] = B.Fp8.empty(1, K, N, DEV)
            B.btx_fp8_quantize(s.pop("w"), None, block_rows=BLOCK, out_t=s["wt"])
            s["gq"], s["gt"], s["xt"] = B.Fp8.empty(1, M, N, DEV), B.Fp8.empty(1, N, M, DEV), B.Fp8.empty(1, K, M, DEV)
            s["dx"] = torch.empty((M, K), dtype=dt, device=DEV)
            s["dw"] = torch.empty((N, K), dtype=torch.float32, device=DEV)
            s["ws"] = workspace(max(B.btx_fp8_matmul_workspace_size(M, K, N, dt),
                                    B.btx_fp8_matmul_workspace_size(N, K, M, torch.float32)))
    else:
        T, d, F, E, k = (case[n] for n in ("T", "d", "F", "E", "k"))
        s["w13"], s["w2q"] = B.Fp8.empty(E, 2 * F, d, DEV), B.Fp8.empty(E, d, F, DEV)    # rows of W1 and W3 in turn
        B.btx_fp8_quantize(s.pop("w1"), s["w13"], block_rows=BLOCK, row_first=0, row_step=2)
        B.btx_fp8_quantize(s.pop("w3"), s["w13"], block_rows=BLOCK, row_first=1, row_step=2)
        B.btx_fp8_quantize(s.pop("w2"), s["w2q"], block_rows=BLOCK)
        s["desc"] = B.make_fp8_moe_desc(T, d, F, E, k, dt)
        s["y"] = torch.empty((T, d), dtype=dt, device=DEV)
        s["ws"] = workspace(B.btx_fp8_moe_workspace_size(s["desc"]))
    return s


# ------------------------------------------------------------------------------------------------
# Plain forms
# ------------------------------------------------------------------------------------------------
def _round_fp8(x, amax):
    """The FP8 values of x in fp32 where `amax`, of a shape that broadcasts, is the largest magnitude of an element's
    block: scale 2^e, the smallest (not below 2^-127) with amax / 2^e <= 448, and x / 2^e to the nearest e4m3 value
    (four significant bits, spacing 2^-9 at least; ties to even)."""
    m, e = torch.frexp(amax)
    exp = torch.where(amax > 0, e - 9 + (m > 0.875).int(), -127).clamp_(min=-127)
    p = torch.ldexp(x, -exp)
    step = torch.frexp(p)[1].clamp_(min=-5) - 4
    return torch.ldexp(torch.ldexp(torch.round(torch.ldexp(p, -step)), step), exp)


def _padded(x, rows, cols):
    """x with zeros behind its last row and column, to whole blocks."""
    return torch.nn.functional.pad(x.float(), (0, -x.shape[-1] % cols, 0, -x.shape[-2] % rows))


def _row_values(x):
    """FP8 values of [.., rows, K], a scale per 128 elements of a row."""
    v = _padded(x, 1, BLOCK).unflatten(-1, (-1, BLOCK))
    return _round_fp8(v, v.abs().amax(-1, keepdim=True)).flatten(-2)[..., :x.shape[-1]]


def _block_values(x):
    """FP8 values of [.., rows, K], a scale per 128 x 128 block."""
    v = _padded(x, BLOCK, BLOCK).unflatten(-1, (-1, BLOCK)).unflatten(-3, (-1, BLOCK))
    v = _round_fp8(v, v.abs().amax((-3, -1), keepdim=True)).flatten(-4, -3).flatten(-2)
    return v[..., :x.shape[-2], :x.shape[-1]]


def _plain_norm(s):
    x = s["x"]
    h = x if s["residual"] is None else (x.float() + s["residual"].float()).to(x.dtype)
    v = h.float()
    y = v / torch.sqrt((v * v).mean(1, keepdim=True) + EPS) * s["w"].float()
    out = [y.to(x.dtype)]
    if s["residual"] is not None:
        out.append(h)
    if s["case"]["fp8"]:
        out.append(_row_values(y).to(torch.bfloat16))
    return out


def _plain_norm_backward(s):
    h, dy = s["h"].float(), s["dy"].float()
    scale = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
    unit = h * scale
    g = dy * s["w"].float()
    dx = scale * (g - unit * (g * unit).mean(1, keepdim=True))
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    return dx.to(s["h"].dtype), (dy * unit).sum(0)


def _plain_cast(s):
    c, x = s["case"], s["x"]
    if c["block"] > 1:
        v = _block_values(x).to(torch.bfloat16)
        return (v, v.transpose(1, 2).contiguous()) if c["both"] else (v,)
    v = _row_values(x).to(torch.bfloat16)
    return (v, _row_values(x.transpose(1, 2)).to(torch.bfloat16)) if c["both"] else (v,)


def _plain_product(s):
    dt, w = s["x"].dtype, s["w"].float()
    if s["case"]["direction"] == "forward":
        return (_row_values(s["x"]) @ w.t()).to(dt)
    dx = (_row_values(s["dy"]) @ w).to(dt)
    return dx, _row_values(s["dy"].t()) @ _row_values(s["x"].t()).t()


def _plain_moe(s):
    c = s["case"]
    x = _row_values(s["x"])
    rows = torch.zeros((c["T"], c["k"], c["d"]), dtype=torch.float32, device=x.device)
    for e in range(c["E"]):
        t, slot = (s["topk_idx"] == e).nonzero(as_tuple=True)
        if t.numel() == 0:
            continue
        xe = x[t]
        h1, h3 = xe @ s["w1"][e].float().t(), xe @ s["w3"][e].float().t()
        act = _row_values(h1 / (1.0 + torch.exp(-h1)) * h3)
        rows[t, slot] = (act @ s["w2"][e].float().t()) * s["gates"][t, slot][:, None]
    return rows.sum(1).to(s["x"].dtype)


PLAIN = {"norm": _plain_norm, "norm_backward": _plain_norm_backward, "cast": _plain_cast, "product": _plain_product,
         "moe": _plain_moe}


# ------------------------------------------------------------------------------------------------
# The library's calls
# ------------------------------------------------------------------------------------------------
def _own_norm(s, B):
    B.btx_rms_norm(s["desc"], s["x"], s["w"], residual=s["residual"], h=s["h"], y=s["y"], q=s.get("q"))
    out = [s["y"]]
    if s["h"] is not None:
        out.append(s["h"])
    if "q" in s:
        B.btx_fp8_dequantize(s["q"], s["values"])
        out.append(s["values"])
    return out


def _own_norm_backward(s, B):
    B.btx_rms_norm_backward(s["desc"], s["h"], s["w"], s["dy"], s["dx"], s["dw"], s["ws"], dh=s["dh"])
    return s["dx"], s["dw"]


def _own_cast(s, B):
    B.btx_fp8_quantize(s["x"], s["q"], block_rows=s["case"]["block"], out_t=s.get("qt"))
    B.btx_fp8_dequantize(s["q"], s["values"])
    if "qt" not in s:
        return (s["values"],)
    B.btx_fp8_dequantize(s["qt"], s["values_t"])
    return s["values"], s["values_t"]


def _own_product(s, B):
    if s["case"]["direction"] == "forward":
        B.btx_fp8_quantize(s["x"], s["xq"])
        B.btx_fp8_matmul(s["xq"], s["wq"], s["y"], s["ws"])
        return s["y"]
    B.btx_fp8_quantize(s["dy"], s["gq"], out_t=s["gt"])
    B.btx_fp8_quantize(s["x"], None, out_t=s["xt"])
    B.btx_fp8_matmul(s["gq"], s["wt"], s["dx"], s["ws"])
    B.btx_fp8_matmul(s["gt"], s["xt"], s["dw"], s["ws"])
    return s["dx"], s["dw"]


def _own_moe(s, B):
    B.btx_fp8_moe_forward(s["desc"], s["x"], s["topk_idx"], s["gates"], s["w13"], s["w2q"], s["y"], s["ws"])
    return s["y"]


OWN = {"norm": _own_norm, "norm_backward": _own_norm_backward, "cast": _own_cast, "product": _own_product, "moe": _own_moe}


def run(state):
    op = state["case"]["op"]
    return OWN[op](state, state["B"]) if own else PLAIN[op](state)


# ------------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ------------------------------------------------------------------------------------------------
def _exact_fp8(x, rows):
    """FP8 values in fp64 of [batch, R, K], a scale per `rows` x 128 elements: the rounding that the spacing of e4m3 at
    each value's size gives (half to even)."""
    b, R, K = x.shape
    nr, nk = -(-R // rows), -(-K // BLOCK)
    v = torch.zeros((b, nr * rows, nk * BLOCK), dtype=torch.float64, device=x.device)
    v[:, :R, :K] = x.double()
    v = v.view(b, nr, rows, nk, BLOCK)
    amax = v.abs().amax((2, 4), keepdim=True).clamp_(min=2.0 ** -149)
    scale = torch.exp2(torch.ceil(torch.log2(amax / 448.0)).clamp_(min=-127.0))
    p = v / scale
    step = torch.exp2(torch.floor(torch.log2(p.abs().clamp(min=2.0 ** -6))) - 3.0)
    return (torch.round(p / step) * step * scale).view(b, nr * rows, nk * BLOCK)[:, :R, :K]


def _exact_rows(x):
    return _exact_fp8(x[None], 1)[0]


def _exact_weight(w):
    return _exact_fp8(w[None], BLOCK)[0]


def _exact_norm(case, s):
    # the sum is rounded to the tensor's type, which is what later layers see
    h = s["x"].double()
    if s["residual"] is not None:
        h = (h + s["residual"].double()).to(s["x"].dtype).double()
    y = h * torch.rsqrt(h.square().sum(1, keepdim=True) / case["d"] + EPS) * s["w"].double()
    out = [y]
    if s["residual"] is not None:
        out.append(h)
    if case["fp8"]:
        out.append(_exact_rows(y))
    return out


def _exact_norm_backward(case, s):
    """From y_i = h_i w_i n^-1/2, n = mean h^2 + eps: dh_j = w_j dy_j n^-1/2 - h_j / d n^-3/2 sum_i dy_i w_i h_i."""
    h, dy, w = s["h"].double(), s["dy"].double(), s["w"].double()
    n = h.square().sum(1, keepdim=True) / case["d"] + EPS
    dot = torch.matmul(dy * h, w[:, None])
    dx = w * dy * n.pow(-0.5) - h * (dot / case["d"]) * n.pow(-1.5)
    if s["dh"] is not None:
        dx += s["dh"].double()
    return dx, torch.matmul(n.pow(-0.5).t(), dy * h)[0]


def exact(case, seed):
    s, op = _inputs(case, seed), case["op"]
    if op == "norm":
        return _exact_norm(case, s)
    if op == "norm_backward":
        return _exact_norm_backward(case, s)
    if op == "cast":
        v = _exact_fp8(s["x"], case["block"])
        if not case["both"]:
            return (v,)
        return v, _exact_fp8(s["x"].transpose(1, 2).contiguous(), case["block"])
    if op == "product":
        w = _exact_weight(s["w"])
        if case["direction"] == "forward":
            return torch.matmul(_exact_rows(s["x"]), w.t())
        dy = s["dy"]
        return torch.matmul(_exact_rows(dy), w), torch.matmul(_exact_rows(dy.t().contiguous()), _exact_rows(s["x"].t().contiguous()).t())
    x = _exact_rows(s["x"])
    y = torch.zeros_like(x)
    for e in range(case["E"]):
        gate = (s["gates"].double() * (s["topk_idx"] == e)).sum(1)
        t = (s["topk_idx"] == e).any(1).nonzero().flatten()
        if t.numel() == 0:
            continue
        h1, h3 = x[t] @ _exact_weight(s["w1"][e]).t(), x[t] @ _exact_weight(s["w3"][e]).t()
        act = _exact_rows(h1 * torch.sigmoid(h1) * h3)
        y[t] += gate[t, None] * (act @ _exact_weight(s["w2"][e]).t())
    return y
