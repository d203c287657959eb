"""FP8 casts and the values read back against the 64-bit statement in oracle/fp8_oracle.py: codes, scales and values are equal bit
for bit, as they stand and transposed."""
import numpy as np
import pytest
import torch

from oracle import fp8_oracle as o
from paper_2403_07816_b200 import binding as B
from util import Guarded, check_guards

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
both = pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
SHAPES = [(1, 1, 1), (1, 1, 16), (1, 3, 127), (2, 33, 128), (1, 129, 130), (2, 128, 512), (3, 7, 1041), (1, 300, 260), (1, 257, 1336),
          (2, 16, 8), (1, 40, 2056)]


def randn(*shape, seed=0, std=1.0, dtype=F32):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype).to(DEV)


def np64(t):
    return t.double().cpu().numpy()


def guarded_fp8(batch, rows, K, fill=0xA5):
    bufs = {"codes": Guarded((batch, rows, (K + 31) // 32 * 32), torch.uint8, DEV, fill=fill),
            "scales": Guarded((batch, (rows + 127) // 128, (K + 511) // 512, 512), torch.uint8, DEV, fill=fill)}
    return B.Fp8(bufs["codes"].t, bufs["scales"].t, K), bufs


def check(q, x, rows, fill=0xA5):
    """q holds the cast of x [batch, R, K], a scale per `rows` x 128."""
    for i, m in enumerate(x):
        codes, scales = o.quantize(m, rows)
        assert np.array_equal(q.scales[i].cpu().numpy(), o.stored_scales(scales, fill))
        assert np.array_equal(q.codes[i].cpu().numpy(), o.stored_codes(codes))


def check_square_t(q, x, fill=0xA5):
    """q holds the transpose of the square-block cast of x."""
    for i, m in enumerate(x):
        codes, scales = o.quantize(m, 128)
        by_block = scales[::128].T.repeat(128, 0)[:m.shape[1]]
        assert np.array_equal(q.scales[i].cpu().numpy(), o.stored_scales(by_block, fill))
        assert np.array_equal(q.codes[i].cpu().numpy(), o.stored_codes(codes.T.copy()))


def special_values(dtype):
    """Blocks around the borders of the cast: scales at 448, ties, subnormal results, the ends of the type, zeros, NaN."""
    rows = []
    ties = (o.E4M3[1:] + o.E4M3[:-1]) / 2
    grid = np.concatenate([ties[-63:], -ties[-62:], [448.0, 0.0, -0.0]])
    low = np.concatenate([ties[:63], -ties[:62], [448.0, 2.0 ** -9, 2.0 ** -11]])
    for e in (0, 1, -7, -100, -125, -134, 119):
        rows += [grid * 2.0 ** e, low * 2.0 ** e]
    for amax in (3.5, 3.5000002, 3.515625, 1.75, 448.0, 448.0001, 450.0, 1.1754944e-38, 1e-45, 3.3895e38, 2.0 ** -118 * 1.75):
        v = np.linspace(-1, 1, 128) * amax
        v[5] = amax
        rows.append(v)
    rows += [np.zeros(128), -np.zeros(128)]
    for bad in (np.nan, np.inf, -np.inf):
        v = np.linspace(-2, 2, 128)
        v[17] = bad
        rows.append(v)
    x = torch.tensor(np.stack(rows)).float()
    x = torch.where(x.isfinite() & (x.abs() > torch.finfo(dtype).max), torch.sign(x) * torch.finfo(dtype).max, x)
    return x.to(dtype).reshape(1, -1, 128).to(DEV)


@both
@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_cast(shape, rows, dtype):
    batch, R, K = shape
    x = randn(*shape, seed=sum(shape), dtype=dtype) * torch.exp2(torch.randint(-6, 7, (batch, R, 1), generator=torch.Generator().manual_seed(1)).float()).to(DEV).to(dtype)
    xt = np64(x).transpose(0, 2, 1)
    for with_out, with_t in ((True, False), (True, True), (False, True)):
        (q, b), (t, bt) = guarded_fp8(batch, R, K), guarded_fp8(batch, K, R)
        B.btx_fp8_quantize(x, q if with_out else None, block_rows=rows, out_t=t if with_t else None)
        check_guards({**b, **{"t_" + n: g for n, g in bt.items()}}, "btx_fp8_quantize")
        if with_out:
            check(q, np64(x), rows)
            for out in (F32, BF16):
                back = Guarded(shape, out, DEV)
                B.btx_fp8_dequantize(q, back.t)
                check_guards({"dst": back}, "btx_fp8_dequantize")
                assert np.array_equal(np64(back.t), np.stack([o.round_rows(m, rows) for m in np64(x)]))
        else:
            assert bool((q.codes == 0xA5).all())
        if with_t:
            check(t, xt, 1) if rows == 1 else check_square_t(t, np64(x))
        else:
            assert bool((t.codes == 0xA5).all())


@both
def test_cast_at_its_borders(dtype):
    x = special_values(dtype)
    q, _ = guarded_fp8(*x.shape)
    B.btx_fp8_quantize(x, q)
    check(q, np64(x), 1)
    back = torch.empty(x.shape, dtype=F32, device=DEV)
    B.btx_fp8_dequantize(q, back)
    # elements above 1.9375 * 2^127 go to 2^128, for which fp32 has no number but infinity
    with np.errstate(over="ignore"):
        want = o.round_rows(np64(x)[0]).astype(np.float32)
    assert np.array_equal(back[0].cpu().numpy(), want, equal_nan=True)
    xt = x.transpose(1, 2).contiguous()                              # the same blocks along the columns
    t, _ = guarded_fp8(*x.shape)
    B.btx_fp8_quantize(xt, None, out_t=t)
    assert torch.equal(t.codes, q.codes) and torch.equal(t.scales, q.scales)
    one, _ = guarded_fp8(1, 128, 256)                                # a square block with one NaN, beside one without
    y = randn(1, 128, 256, seed=1, dtype=dtype)
    y[0, 77, 3] = float("nan")
    B.btx_fp8_quantize(y, one, block_rows=128)
    check(one, np64(y), 128)


@both
def test_cast_of_strided_rows_into_interleaved_rows(dtype):
    w = randn(2, 270, 600, seed=3, dtype=dtype)
    for src in (w[:, :, 3:301], w[:, ::2, 8:408], w[:1, :, 100:101], w[:, :, 16:272]):
        batch, rows, K = src.shape
        for block in (1, 128):
            q, bufs = guarded_fp8(batch, 2 * rows + 1, K, fill=0x11)
            t, bt = guarded_fp8(batch, K, rows)
            B.btx_fp8_quantize(src, q, block_rows=block, row_first=1, row_step=2, out_t=t)
            check_guards({**bufs, **{"t_" + n: g for n, g in bt.items()}}, "btx_fp8_quantize")
            ref, ref_t = B.Fp8.empty(batch, rows, K, DEV), B.Fp8.empty(batch, K, rows, DEV)
            B.btx_fp8_quantize(src.contiguous(), ref, block_rows=block, out_t=ref_t)
            assert torch.equal(q.codes[:, 1::2], ref.codes) and bool((q.codes[:, 0::2] == 0x11).all())
            assert torch.equal(t.codes, ref_t.codes)
            nb = (K + 127) // 128
            at = lambda s, i: s[:, i // 128, :, (i % 32) * 16 + (i // 32 % 4) * 4:][:, :, :4].reshape(batch, -1)[:, :nb]
            for r in range(rows):
                assert torch.equal(at(q.scales, 2 * r + 1), at(ref.scales, r)) and bool((at(q.scales, 2 * r) == 0x11).all())
    x = randn(40, 64, seed=1, dtype=dtype)
    rep, flat = B.Fp8.empty(1, 40, 64, DEV), B.Fp8.empty(1, 40, 64, DEV)
    B.btx_fp8_quantize(x[:1].expand(40, 64), rep)                    # one row, 40 times
    B.btx_fp8_quantize(x[:1].repeat(40, 1), flat)
    assert torch.equal(rep.codes, flat.codes)


def test_offsets_past_32_bits():
    rows, K = 539_914, 4097                                          # 2.2 G elements, rows off 16-byte boundaries
    x = torch.empty(rows, K, dtype=BF16, device=DEV)
    tail = randn(138, K, seed=1, dtype=BF16)                         # (from a multiple of 128 on)
    x[:-138] = tail[0]
    x[-138:] = tail
    assert (rows - 138) % 128 == 0
    q, t = B.Fp8.empty(1, rows, K, DEV), B.Fp8.empty(1, K, rows, DEV)
    sq, st = B.Fp8.empty(1, 138, K, DEV), B.Fp8.empty(1, K, 138, DEV)
    for block in (1, 128):
        B.btx_fp8_quantize(x, q, block_rows=block, out_t=t)
        B.btx_fp8_quantize(tail, sq, block_rows=block, out_t=st)
        assert torch.equal(q.codes[0, -138:], sq.codes[0]) and torch.equal(t.codes[0, :, rows - 138:rows], st.codes[0, :, :138])
    B.btx_fp8_quantize(x, q)
    B.btx_fp8_dequantize(q, x)
    back = torch.empty(138, K, dtype=BF16, device=DEV)
    B.btx_fp8_quantize(tail, sq)
    B.btx_fp8_dequantize(sq, back)
    assert torch.equal(x[-138:], back)


def test_binding_refuses_wrong_tensors():
    q, x = B.Fp8.empty(1, 8, 64, DEV), randn(8, 64)
    for bad in (lambda: B.btx_fp8_quantize(randn(8, 96), q), lambda: B.btx_fp8_quantize(x, B.Fp8(q.codes, q.scales[..., :256], 64)),
                lambda: B.btx_fp8_quantize(x, B.Fp8(q.codes, q.scales, 80)), lambda: B.btx_fp8_quantize(x, q, out_t=q),
                lambda: B.btx_fp8_dequantize(q, randn(8, 32))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(RuntimeError):
        B.btx_fp8_quantize(randn(64, 8).t(), q)
    with pytest.raises(TypeError):
        B.btx_fp8_quantize(x.half(), q)
    for bad in (lambda: B.btx_fp8_quantize(x, None), lambda: B.btx_fp8_quantize(x, q, row_first=1), lambda: B.btx_fp8_quantize(x, q, block_rows=64)):
        with pytest.raises(B.BtxError) as ei:
            bad()
        assert ei.value.status == 1
