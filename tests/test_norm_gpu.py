"""The root-mean-square norm and its gradients against the 64-bit statement in oracle/fp8_oracle.py.

u = 2^-24, half a step of fp32.  A sum over a row adds at most 32 terms in a thread and joins threads in at most 10 steps: it is
within 45 u of the sum of magnitudes.  1 / sqrt(.) halves that error and adds three roundings: s is within 26 u.  y = h s w has
two more: 28 u < 2^-19.  In dx = dh + s (g - h s m), m = s mean(g h) is within (45 + 26 + 3) u of its terms' sizes, h s within
27 u, and products, differences and the outer s add 26 + 4: 131 u < 2^-16.9 of the sizes of the terms.  A column of dw adds
products within 29 u, at most T / 148 + 1 rows in a block and the shares of at most 32 blocks for each of 148
multiprocessors, a sixteenth in a row: with T <= 3000 within (29 + 22 + 296 + 16) u < 2^-15.4.  The last rounding is half a step
of the output's type."""
import numpy as np
import pytest
import torch

from oracle import fp8_oracle as o
from paper_2403_07816_b200 import binding as B
from util import Guarded, check_guards

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-5
F32, BF16 = torch.float32, torch.bfloat16
SHAPES = [(1, 1), (1, 7), (3, 8), (5, 127), (9, 128), (4, 130), (300, 64), (2, 520), (37, 1000), (700, 1365), (9, 4096), (130, 4104),
          (3, 8200), (3, 16384)]
both = pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])


def randn(*shape, seed=0, std=1.0, dtype=F32):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype).to(DEV)


def np64(t):
    return t.double().cpu().numpy()


def half(dtype):
    return torch.finfo(dtype).eps / 2


def check_fp8(q, y, tol):
    """The FP8 form of values known to lie within tol of y: the scale is that of a largest magnitude within tol, and every element
    lies between the casts of both ends at that scale."""
    T, d = y.shape
    nb = -(-d // 128)
    scales = q.scales.cpu().numpy()[0]
    r, b = np.arange(T)[:, None], np.arange(nb)[None]
    byte = scales[r // 128, b // 4, (r % 32) * 16 + (r % 128 // 32) * 4 + b % 4]
    pad = lambda a: np.pad(a, ((0, 0), (0, -d % 128))).reshape(T, nb, 128)
    amax, off = np.abs(pad(y)).max(2), pad(tol).max(2)
    expo = lambda m: np.where(m > 0, np.maximum(np.ceil(np.log2(np.maximum(m, 1e-300) / 448)), -127), -127) + 127
    assert (byte >= expo(amax - off)).all() and (byte <= expo(amax + off)).all()
    codes = q.codes.cpu().numpy()[0]
    assert (codes[:, d:] == 0).all()
    got = o.values(codes[:, :d], byte)
    s = np.exp2(byte.astype(float) - 127).repeat(128, 1)[:, :d]
    cast = lambda v: np.sign(v) * o.E4M3[o._nearest(np.minimum(np.abs(v) / s, 448))] * s
    assert (got >= cast(y - tol)).all() and (got <= cast(y + tol)).all()


def norm(x, w, residual, dtype, fp8=True):
    T, d = x.shape
    desc = B.make_norm_desc(T, d, dtype, EPS)
    bufs = {"h": Guarded((T, d), dtype, DEV), "y": Guarded((T, d), dtype, DEV)}
    q = None
    if fp8:
        bufs["codes"] = Guarded((1, T, (d + 31) // 32 * 32), torch.uint8, DEV, fill=0xEE)
        bufs["scales"] = Guarded((1, (T + 127) // 128, (d + 511) // 512, 512), torch.uint8, DEV, fill=0xEE)
        q = B.Fp8(bufs["codes"].t, bufs["scales"].t, d)
    B.btx_rms_norm(desc, x, w, residual=residual, h=bufs["h"].t, y=bufs["y"].t, q=q)
    check_guards(bufs, "btx_rms_norm")
    return bufs["h"].t, bufs["y"].t, q


def check_forward(x, w, residual, h, y, q):
    T, d = x.shape
    want_h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    assert torch.equal(h, want_h)
    want = o.rms_norm(np64(want_h), np64(w) if w is not None else 1.0, EPS)
    tol = 2.0 ** -19 * np.abs(want)
    assert (np.abs(np64(y) - want) <= tol + half(x.dtype) * np.abs(want) + 1e-45).all()
    if q is not None:
        check_fp8(q, want, tol + 1e-45)


@both
@pytest.mark.parametrize("residual", [True, False], ids=["residual", "alone"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_norm(shape, residual, dtype):
    T, d = shape
    x, w = randn(T, d, seed=d, dtype=dtype), (1 + randn(d, seed=2, std=0.3)).to(dtype)
    r = randn(T, d, seed=3, std=4.0, dtype=dtype) if residual else None
    h, y, q = norm(x, w, r, dtype)
    check_forward(x, w, r, h, y, q)


def test_longest_rows():
    for dtype, d in ((BF16, 32768), (BF16, 32761), (F32, 16383)):
        x, r = randn(5, d, seed=1, dtype=dtype), randn(5, d, seed=2, dtype=dtype)
        check_forward(x, None, r, *norm(x, None, r, dtype))
        check_backward(5, d, dtype, True, True)


@both
def test_strided_rows_and_outputs_in_place(dtype):
    T, d = 50, 264
    for first, wide in ((0, 300), (3, 301), (8, 512)):                # rows on and off 16-byte boundaries
        big_x, big_r, big_y = randn(T, wide, seed=1, dtype=dtype), randn(T, wide, seed=2, dtype=dtype), randn(T, wide, seed=4, dtype=dtype)
        w = randn(wide, seed=3, dtype=dtype)[first:first + d].clone()
        x, r, y = big_x[:, first:first + d], big_r[:, first:first + d], big_y[:, first:first + d]
        if x.shape[1] < d:
            continue
        h0, y0, q0 = norm(x.contiguous(), w, r.contiguous(), dtype)
        check_forward(x, w, r, h0, y0, q0)
        kept = [t.clone() for t in (big_x, big_r, big_y)]
        desc = B.make_norm_desc(T, d, dtype, EPS)
        q = B.Fp8.empty(1, T, d, DEV)
        B.btx_rms_norm(desc, x, w, residual=r, h=r, y=y, q=q)         # the residual stream in place
        assert torch.equal(r, h0) and torch.equal(y, y0) and torch.equal(q.codes, q0.codes) and torch.equal(big_x, kept[0])
        for big, was in ((big_r, kept[1]), (big_y, kept[2])):         # nothing beside the rows
            out = torch.ones(wide, dtype=torch.bool)
            out[first:first + d] = False
            assert torch.equal(big[:, out.to(DEV)], was[:, out.to(DEV)])
        B.btx_rms_norm(desc, x, w, residual=kept[1][:, first:first + d], h=x)
        assert torch.equal(x, h0)
        B.btx_rms_norm(desc, x, w, y=x)                               # y over x: the norm of h
        assert torch.equal(x, y0)


@both
def test_outputs_left_out_and_no_weight(dtype):
    T, d = 33, 777
    x = randn(T, d, seed=5, dtype=dtype)
    h, y, q = norm(x, None, None, dtype)
    check_forward(x, None, None, h, y, q)
    desc = B.make_norm_desc(T, d, dtype, EPS)
    only = B.Fp8.empty(1, T, d, DEV)
    B.btx_rms_norm(desc, x, None, q=only)
    assert torch.equal(only.codes, q.codes)
    y2 = torch.empty_like(x)
    B.btx_rms_norm(desc, x, None, y=y2)
    assert torch.equal(y2, y)
    B.btx_rms_norm(B.make_norm_desc(0, d, dtype, EPS), x[:0], None, y=y2[:0])


@both
def test_rows_that_are_not_numbers_stay_by_themselves(dtype):
    T, d = 20, 300
    x = randn(T, d, seed=6, dtype=dtype)
    h0, y0, q0 = norm(x, None, None, dtype)
    x[3, 5], x[7, 299], x[9] = float("nan"), float("inf"), 0.0
    x[11] = 1e25                                                      # its sum of squares is infinite
    h, y, q = norm(x, None, None, dtype)
    other = [t for t in range(T) if t not in (3, 7, 9, 11)]
    assert torch.equal(y[other], y0[other]) and torch.equal(q.codes[0, other], q0.codes[0, other])
    v = torch.empty(T, d, device=DEV)
    B.btx_fp8_dequantize(q, v)
    assert bool(y[3].isnan().all()) and bool(v[3].isnan().all())
    finite = torch.isfinite(x[7])
    assert bool((y[7][finite] == 0).all()) and bool(y[7, 299].isnan()) and bool(v[7, 256:].isnan().all()) and bool((v[7, :256] == 0).all())
    assert bool((y[9] == 0).all()) and bool((v[9] == 0).all()) and bool((y[11] == 0).all()) and bool((v[11] == 0).all())
    # eps = 0: 1 / sqrt(0) is infinite and 0 times it is not a number; no other row is touched
    zero = torch.zeros(2, 8, dtype=dtype, device=DEV)
    zero[1] = 1
    out = torch.empty_like(zero)
    B.btx_rms_norm(B.make_norm_desc(2, 8, dtype, 0.0), zero, None, y=out)
    assert bool(out[0].isnan().all()) and bool((out[1] == 1).all())


def check_backward(T, d, dtype, with_dh, with_w):
    h, dy = randn(T, d, seed=d, std=3.0, dtype=dtype), randn(T, d, seed=2, std=0.1, dtype=dtype)
    w = (1 + randn(d, seed=3, std=0.3)).to(dtype) if with_w else None
    dh = randn(T, d, seed=4, std=0.1, dtype=dtype) if with_dh else None
    desc = B.make_norm_desc(T, d, dtype, EPS)
    bufs = {"dx": Guarded((T, d), dtype, DEV), "dw": Guarded((d,), F32, DEV),
            "ws": Guarded(B.btx_rms_norm_backward_workspace_size(desc), torch.uint8, DEV, fill=0x7F)}
    B.btx_rms_norm_backward(desc, h, w, dy, bufs["dx"].t, bufs["dw"].t, bufs["ws"].t, dh=dh)
    check_guards(bufs, "btx_rms_norm_backward")
    assert B.btx_device_status(bufs["ws"].t) == B.BTX_OK
    h64, dy64, w64 = np64(h), np64(dy), np64(w) if with_w else np.ones(d)
    dx, dw = o.rms_norm_backward(h64, w64, dy64, EPS, np64(dh) if with_dh else None)
    s = 1 / np.sqrt((h64 * h64).mean(1, keepdims=True) + EPS)
    size = s * np.abs(dy64 * w64) + np.abs(h64) * s ** 3 * np.abs(dy64 * w64 * h64).mean(1, keepdims=True)
    err = np.abs(np64(bufs["dx"].t) - dx)
    assert (err <= 2.0 ** -16.9 * size + (half(dtype) + 2.0 ** -24) * np.abs(dx)).all()
    assert (np.abs(np64(bufs["dw"].t) - dw) <= 2.0 ** -15.4 * np.abs(dy64 * h64 * s).sum(0)).all()
    return h, w, dy, dh, bufs["dx"].t, bufs["dw"].t


@both
@pytest.mark.parametrize("with_dh,with_w", [(True, True), (False, True), (True, False)], ids=["all", "no-dh", "no-w"])
@pytest.mark.parametrize("shape", SHAPES + [(3000, 40)], ids=lambda s: "x".join(map(str, s)))
def test_norm_backward(shape, with_dh, with_w, dtype):
    check_backward(*shape, dtype, with_dh, with_w)


@both
def test_backward_accumulates_in_place_and_repeats(dtype):
    T, d = 2000, 520
    h, w, dy, dh, dx, dw = check_backward(T, d, dtype, True, True)
    desc = B.make_norm_desc(T, d, dtype, EPS)
    ws = torch.empty(B.btx_rms_norm_backward_workspace_size(desc), dtype=torch.uint8, device=DEV)
    twice, again = dw.clone(), torch.empty_like(dx)
    B.btx_rms_norm_backward(desc, h, w, dy, again, twice, ws, dh=dh, accumulate=True)
    assert torch.equal(again, dx)                                      # the same bits
    assert bool(((twice - 2 * dw).abs() <= 2.0 ** -14 * (dy.float() * h.float()).abs().sum(0)).all())
    B.btx_rms_norm_backward(desc, h, w, dy, again, None, ws, dh=dh)
    assert torch.equal(again, dx)
    for over in ("dy", "dh", "h"):
        t = {"dy": dy.clone(), "dh": dh.clone(), "h": h.clone()}
        B.btx_rms_norm_backward(desc, t["h"], w, t["dy"], t[over], again_dw := torch.empty_like(dw), ws, dh=t["dh"])
        assert torch.equal(t[over], dx) and torch.equal(again_dw, dw)
    # rows apart, off 16-byte boundaries
    wide = [torch.zeros(T, d + 5, dtype=dtype, device=DEV) for _ in range(4)]
    views = [b[:, 3:3 + d] for b in wide]
    for v, t in zip(views, (h, dy, dh, dx)):
        v.copy_(t)
    views[3].zero_()
    B.btx_rms_norm_backward(desc, views[0], w, views[1], views[3], again_dw, ws, dh=views[2])
    assert torch.equal(views[3], dx) and torch.equal(again_dw, dw) and bool((wide[3][:, :3] == 0).all()) and bool((wide[3][:, 3 + d:] == 0).all())
    empty = B.make_norm_desc(0, d, dtype, EPS)
    B.btx_rms_norm_backward(empty, h[:0], w, dy[:0], dx[:0], twice, ws, accumulate=True)
    assert bool((twice != 0).any())
    B.btx_rms_norm_backward(empty, h[:0], w, dy[:0], dx[:0], twice, ws)
    assert bool((twice == 0).all())


def test_backward_of_a_large_row_keeps_its_scale():
    # s is small where h is large: s^3 alone would leave fp32
    for size in (1e15, 1e-12):
        h, dy = randn(4, 200, seed=1) * size, randn(4, 200, seed=2)
        desc = B.make_norm_desc(4, 200, F32, 0.0)
        ws = torch.empty(B.btx_rms_norm_backward_workspace_size(desc), dtype=torch.uint8, device=DEV)
        dx, dw = torch.empty_like(h), torch.empty(200, device=DEV)
        B.btx_rms_norm_backward(desc, h, None, dy, dx, dw, ws)
        want = o.rms_norm_backward(np64(h), 1.0, np64(dy), 0.0)
        assert np.abs(np64(dx) - want[0]).max() <= 2.0 ** -15 * np.abs(want[0]).max()
        assert np.abs(np64(dw) - want[1]).max() <= 2.0 ** -15 * np.abs(want[1]).max()


def test_gradient_against_differences():
    T, d = 3, 48
    h, w, dy = randn(T, d, seed=1), 1 + randn(d, seed=2, std=0.3), randn(T, d, seed=3)
    desc = B.make_norm_desc(T, d, F32, 1e-3)
    ws = torch.empty(B.btx_rms_norm_backward_workspace_size(desc), dtype=torch.uint8, device=DEV)
    dx, dw, y = torch.empty_like(h), torch.empty(d, device=DEV), torch.empty(2, d, device=DEV)
    B.btx_rms_norm_backward(desc, h, w, dy, dx, dw, ws)
    two, e = B.make_norm_desc(2, d, F32, 1e-3), 2.0 ** -7
    for t in range(T):
        for j in range(0, d, 5):
            pair = h[t].repeat(2, 1)
            pair[0, j] += e
            pair[1, j] -= e
            B.btx_rms_norm(two, pair, w, y=y)
            diff = float(((y[0].double() - y[1].double()) * dy[t].double()).sum()) / (float(pair[0, j]) - float(pair[1, j]))
            # third differences e^2 / 6 times a few, and roundings of y (2^-23 each) over 2 e
            assert abs(diff - float(dx[t, j])) < 5 * e * e + 48 * 2.0 ** -21 / (2 * e)


def test_on_a_stream_and_in_a_graph():
    T, d = 64, 512
    x, r, w = randn(T, d, seed=1, dtype=BF16), randn(T, d, seed=2, dtype=BF16), randn(d, seed=3, dtype=BF16)
    h0, y0, q0 = norm(x, w, r, BF16)
    desc = B.make_norm_desc(T, d, BF16, EPS)
    ws = torch.empty(B.btx_rms_norm_backward_workspace_size(desc), dtype=torch.uint8, device=DEV)
    y, h, q, dx, dw = torch.empty_like(x), torch.empty_like(x), B.Fp8.empty(1, T, d, DEV), torch.empty_like(x), torch.empty(d, device=DEV)

    def step():
        B.btx_rms_norm(desc, x, w, residual=r, h=h, y=y, q=q)
        B.btx_rms_norm_backward(desc, h, w, y, dx, dw, ws, dh=r)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    assert torch.equal(y, y0) and torch.equal(h, h0) and torch.equal(q.codes, q0.codes)
    first = [dx.clone(), dw.clone()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t in (y, h, dx, dw):
        t.zero_()
    graph.replay()
    graph.replay()
    assert torch.equal(y, y0) and torch.equal(dx, first[0]) and torch.equal(dw, first[1])


def test_offsets_past_32_bits():
    T, d = 540_001, 4096                                                # 2.2 G elements
    x = torch.empty(T, d, dtype=BF16, device=DEV)
    tail = randn(100, d, seed=1, dtype=BF16)
    x[:-100] = tail[0]
    x[-100:] = tail
    h0, y0, q0 = norm(tail, None, None, BF16)
    q = B.Fp8.empty(1, T, d, DEV)
    y = torch.empty_like(x)
    desc = B.make_norm_desc(T, d, BF16, EPS)
    B.btx_rms_norm(desc, x, None, y=y, q=q)
    assert torch.equal(y[-100:], y0) and torch.equal(q.codes[0, -100:], q0.codes[0]) and torch.equal(y[-101], y0[0])
    del q
    ws = torch.empty(B.btx_rms_norm_backward_workspace_size(desc), dtype=torch.uint8, device=DEV)
    B.btx_rms_norm_backward(desc, x, None, x, y, None, ws)
    small = torch.empty_like(tail)
    B.btx_rms_norm_backward(B.make_norm_desc(100, d, BF16, EPS), tail, None, tail, small, None, ws)
    assert torch.equal(y[-100:], small)


def test_binding_refuses_wrong_tensors():
    x, q = randn(8, 64), B.Fp8.empty(1, 8, 64, DEV)
    d = B.make_norm_desc(8, 64, F32)
    ws = torch.empty(B.btx_rms_norm_backward_workspace_size(d), dtype=torch.uint8, device=DEV)
    for bad in (lambda: B.btx_rms_norm(d, x.bfloat16(), None, y=x), lambda: B.btx_rms_norm(d, x[:4], None, y=x),
                lambda: B.btx_rms_norm(d, x, randn(32), y=x), lambda: B.btx_rms_norm(d, x, None, q=B.Fp8.empty(1, 8, 80, DEV)),
                lambda: B.btx_rms_norm_backward(d, x, None, x, randn(8, 60), None, ws),
                lambda: B.btx_rms_norm_backward(d, x, None, x, x, randn(64).bfloat16(), ws)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(RuntimeError):
        B.btx_rms_norm(d, randn(64, 8).t(), None, y=x)
    with pytest.raises(B.BtxError) as ei:
        B.btx_rms_norm(d, x, None)                                      # no output
    assert ei.value.status == 1
    with pytest.raises(B.BtxError) as ei:
        B.btx_rms_norm_backward(d, x, None, x, x, None, ws[:256])
    assert ei.value.status == 3


# rows that take three vectors a thread, on and off 16-byte boundaries, one and several rows of a block; four for the longer ones
@both
@pytest.mark.parametrize("shape", [(600, 4104), (601, 4107), (310, 5120), (299, 2051), (450, 9001), (20, 5606), (7, 12291)], ids=lambda s: "x".join(map(str, s)))
def test_rows_a_little_longer_than_a_power_of_two(shape, dtype):
    T, d = shape
    x, w, r = randn(T, d, seed=d, dtype=dtype), (1 + randn(d, seed=2, std=0.3)).to(dtype), randn(T, d, seed=3, dtype=dtype)
    h, y, q = norm(x, w, r, dtype)
    check_forward(x, w, r, h, y, q)
    check_backward(T, d, dtype, True, True)
    for a, b in ((0, 1), (3, 7)):                                          # whatever rows there are beside them, the same bits
        h1, y1, _ = norm(x[a:b].contiguous(), w, r[a:b].contiguous(), dtype)
        assert torch.equal(h1, h[a:b]) and torch.equal(y1, y[a:b])
    alone, y2 = norm(h, w, None, dtype)[1], torch.empty_like(h)
    assert torch.equal(alone, y)
    B.btx_rms_norm(B.make_norm_desc(T, d, dtype, EPS), h, w, y=y2)
    assert torch.equal(y2, y)


@both
def test_rows_far_from_one_under_large_and_small_weights(dtype):
    # every row's rms is 2^e; h w alone leaves fp32 for some of them, h s w for none
    T, d = 9, 264
    x = randn(T, d, seed=1, dtype=dtype)
    x = (x.float() * torch.exp2(torch.tensor([-55.0, -50, -40, -20, 0, 20, 40, 50, 55], device=DEV))[:, None]).to(dtype)
    x[4] = 1.5 * 2.0 ** 126                                                # the sum of squares is infinite
    for e in (-80.0, 0.0, 80.0):
        w = (randn(d, seed=2).abs() + 0.5).mul(2.0 ** e).to(dtype)
        y = torch.empty_like(x)
        B.btx_rms_norm(B.make_norm_desc(T, d, dtype, 0.0), x, w, y=y)
        h64 = np64(x)
        want = h64 / np.sqrt((h64 * h64).mean(1, keepdims=True)) * np64(w)
        want[4] = 0.0
        assert (np.abs(np64(y) - want) <= (half(dtype) + 2.0 ** -19) * np.abs(want) + 2.0 ** -140).all()
