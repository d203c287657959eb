"""An Fp8 is checked when it is made: what was checked cannot be changed under the calls that rely on it.  And the numbers that go
over to the library: of any integer type, none cut to 32 bits."""
import copy

import numpy as np
import pytest
import torch

from paper_2403_07816_b200 import binding as B
from paper_2403_07816_b200 import build as builder


@pytest.fixture
def fp8(monkeypatch):
    builder.build()
    monkeypatch.setattr(B, "_device", lambda t: t.get_device())          # (-1: the host's tensors pass the checks, no call is made)
    return lambda: B.Fp8.empty(2, 130, 200, "cpu")


@pytest.mark.parametrize("name", ["codes", "scales", "K", "shape", "device", "sizes"])
def test_attributes_are_read_only(fp8, name):
    q = fp8()
    was = getattr(q, name)
    with pytest.raises(AttributeError):
        setattr(q, name, was)
    with pytest.raises(AttributeError):
        delattr(q, name)
    with pytest.raises(AttributeError):
        q.another = 1
    assert getattr(q, name) is was


@pytest.mark.parametrize("name", ["codes", "scales"])
def test_tensors_resized_since_are_refused(fp8, name):
    q = fp8()
    shape = (2, 130, 200)
    assert B._fp8(q, "q", shape, -1) == (q.codes.data_ptr(), q.scales.data_ptr())
    getattr(q, name).resize_(1, 1, 32)
    with pytest.raises(ValueError, match="resized"):
        B._fp8(q, "q", shape, -1)
    q = fp8()
    getattr(q, name).data = torch.empty(64, dtype=torch.uint8)
    with pytest.raises(ValueError, match="resized"):
        B._fp8(q, "q", shape, -1)


def test_copies_are_checked_again(fp8):
    q = fp8()
    same, own = copy.copy(q), copy.deepcopy(q)
    assert same.codes is q.codes and own.codes is not q.codes and torch.equal(own.codes, q.codes) and own.shape == q.shape
    q.scales.resize_(512)
    with pytest.raises(ValueError):
        copy.copy(q)


def test_integers_of_other_types_go_over(fp8, monkeypatch):
    got = []
    monkeypatch.setattr(B, "_launch", lambda name, dev, *args: got.append((name, args)))
    one, dim = np.int64(1), torch.tensor(200)
    q = B.Fp8(fp8().codes, fp8().scales, dim)
    assert type(q.K) is int and q.shape == (2, 130, 200)
    B.btx_fp8_quantize(torch.zeros(2, 65, 200), q, block_rows=np.int32(128), row_first=one, row_step=np.int64(2))
    B.btx_fp8_dequantize(q, torch.zeros(2, 130, 200))
    for name, args in got:
        for value, kind in zip(args, getattr(B.lib(), name).argtypes):
            kind.from_param(value)
    assert got[0][1][7:11] == (128, 130, 1, 2)
    with pytest.raises(TypeError):
        B.btx_fp8_quantize(torch.zeros(2, 65, 200), q, row_step=2.0)


def test_sizes_past_32_bits_are_refused(fp8, monkeypatch):
    monkeypatch.setattr(B, "_launch", lambda *args: pytest.fail("the library would see other sizes"))
    q, x = fp8(), torch.zeros(2, 130, 200)
    for bad in (dict(row_first=1 << 32), dict(row_step=(1 << 32) + 1), dict(block_rows=(1 << 32) + 1), dict(row_first=-(1 << 32))):
        with pytest.raises(ValueError, match="32 bits"):
            B.btx_fp8_quantize(x, q, **bad)
    with pytest.raises(ValueError, match="32 bits"):
        B.btx_fp8_quantize(x[:, :1].expand(2, (1 << 32) + 130, 200), q)
    rows = (1 << 32) + 5
    with pytest.raises(ValueError, match="32 bits"):
        B.Fp8(torch.empty(1, rows, 32, dtype=torch.uint8, device="meta"), torch.empty(1, (rows + 127) // 128, 1, 512, dtype=torch.uint8, device="meta"), 7)
