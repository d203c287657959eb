"""The MXFP4 cast of oracle/experts_oracle.py against the format itself, element by element."""
import numpy as np
import pytest

from oracle import experts_oracle as o


@pytest.mark.parametrize("std", [1e-30, 0.02, 1.0, 3e7])
def test_cast_is_the_nearest_value_of_the_blocks_grid(std):
    x = np.random.default_rng(1).normal(size=(40, 256)) * std
    codes, scales = o.mx4_quantize(x)
    v = o.mx4_values(codes, scales)
    assert np.array_equal(o.mx4_round(v), v)                              # its own values are left alone
    block = np.exp2(scales.astype(float) - 127).repeat(o.BLOCK, 1)
    amax = np.abs(x).reshape(40, -1, o.BLOCK).max(-1).repeat(o.BLOCK, 1)
    assert (4 * block <= amax).all() and (amax < 8 * block).all()         # 2^(floor(log2 max) - 2)
    p, q = np.abs(x) / block, np.abs(v) / block
    assert np.isin(q, o.E2M1).all() and ((v == 0) | (np.sign(v) == np.sign(x))).all()
    # half the spacing of e2m1 where the element lies: 0.5 below 2, 1 below 4, 2 below 6; above 6 it is 6
    half = np.where(p < 2, 0.25, np.where(p < 4, 0.5, 1.0))
    assert (np.abs(p - q) <= np.where(p > 6, p - 6, half)).all() and (q[p > 6] == 6).all()
    # and no other value is nearer
    assert (np.abs(p - q) == np.abs(p[..., None] - o.E2M1).min(-1)).all()


def test_a_block_by_hand():
    # largest 0.4375 = 1.75 * 2^-2: scale 2^-4, byte 123; elements over it, with the ties 0.25, 0.75, 1.25, 2.5 and 5
    s = 2.0 ** -4
    over = [7.0, 5.0, 4.9, 3.5, 2.5, 2.4, 1.75, 1.25, 1.2, 0.75, 0.7, 0.25, 0.2, 0.0, -6.0, -0.3]
    want = [6.0, 4.0, 4.0, 4.0, 2.0, 2.0, 2.0, 1.0, 1.0, 1.0, 0.5, 0.0, 0.0, 0.0, -6.0, -0.5]
    code = [7, 6, 6, 6, 4, 4, 4, 2, 2, 2, 1, 0, 0, 0, 15, 9]
    x = np.array(over + [0.0] * 16) * s
    codes, scales = o.mx4_quantize(x)
    assert scales.tolist() == [123] and codes[:16].tolist() == code
    assert o.mx4_values(codes, scales)[:16].tolist() == (np.array(want) * s).tolist()
    assert o.mx4_pack(codes)[:3].tolist() == [0x67, 0x66, 0x44]
