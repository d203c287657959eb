"""Host-side limits of the MXFP4 calls, refused before any CUDA call: sizes whose bytes do not fit the arithmetic that
follows, or whose matrices are longer than a tensor map can describe (a product would be refused after the cast)."""
import ctypes as C

import pytest
import torch

from paper_2403_07816_b200 import binding as B
from paper_2403_07816_b200 import build as builder

A = C.c_void_p(4096)


@pytest.fixture(scope="module")
def L():
    builder.build()
    return B.lib()


def test_sizes_that_wrap_around_are_refused(L):
    codes, scales = C.c_size_t(0), C.c_size_t(0)
    top = (1 << 31) - 1
    for batch, rows, K in ((top, 1 << 30, 1 << 30), (top, 1 << 30, 1 << 8), (top, 1, 1 << 30), (1 << 30, 1 << 20, 1 << 18)):
        assert L.btx_mx4_sizes(batch, rows, K, C.byref(codes), C.byref(scales)) == 2
        assert L.btx_mx4_quantize(0, A, K, 0, batch, rows, K, rows, 0, 1, A, A, None) == 2
        assert L.btx_mx4_dequantize(0, A, A, batch, rows, K, A, None) == 2
    # the largest that can be held: one byte more of a row's codes would pass the limit of a matrix
    assert L.btx_mx4_sizes(1, (1 << 15) - 1, 1 << 26, C.byref(codes), C.byref(scales)) == 0
    assert codes.value == ((1 << 15) - 1) << 25 and scales.value == (1 << 8) * (1 << 19) * 512
    assert L.btx_mx4_sizes(1, 1 << 15, 1 << 26, None, None) == 2


def test_the_rows_that_are_written_count_not_only_those_that_are_cast(L):
    # a few rows into a matrix of too many
    assert L.btx_mx4_quantize(0, A, 1 << 26, 0, 1, 2, 1 << 26, 1 << 15, 0, 1, A, A, None) == 2
    assert L.btx_mx4_quantize(0, A, 1 << 20, 0, (1 << 31) - 1, 2, 1 << 20, 1 << 20, 0, 1, A, A, None) == 2


def test_products_that_no_tensor_map_describes_are_refused(L):
    sz = C.c_size_t(0)
    for M, N, K in ((1, 1 << 20, 1 << 21), (1 << 20, 1, 1 << 21), (8, 1 << 30, 1 << 11)):
        assert L.btx_mx4_matmul_workspace_size(0, 1, M, N, K, C.byref(sz)) == 2
        assert L.btx_mx4_matmul(0, 1, M, N, K, A, A, A, A, A, A, 256, None) == 2
    for d, f in ((1 << 20, 1 << 20), (1 << 12, 1 << 28), (1 << 29, 1 << 11)):
        desc = B.make_mx4_moe_desc(1, d, f, 1, 1, torch.float32)
        assert L.btx_mx4_moe_workspace_size(C.byref(desc), C.byref(sz)) == 2
        assert L.btx_mx4_moe_forward(C.byref(desc), A, A, A, A, A, A, A, A, A, 1 << 62, None) == 2
