"""Matrices in 8-bit floating point from tensors of the caller's (no GPU: what they are is checked on any device)."""
import pytest
import torch

from paper_2412_20796_amd import ops


@pytest.mark.parametrize("rows,br", [(0, 1), (1, 1), (2, 1), (9, 1), (9, 128), (300, 128)])
def test_no_columns(rows, br):
    """Codes and scales of no columns, whose strides say nothing; a matrix's own are taken back."""
    empty = lambda n, t: torch.zeros(n, 0, dtype=torch.uint8).view(t)
    m = ops.Fp8Matrix(empty(rows, torch.float8_e4m3fn), empty(-(-rows // br), torch.float8_e8m0fnu), br)
    assert m.shape == (rows, 0) and (m._c.ld, m._c.ld_scale) == (0, 0)
    own = ops.Fp8Matrix.empty(rows, 0, br, "cpu")
    assert ops.Fp8Matrix(own.codes, own.scale, br).shape == (rows, 0)


@pytest.mark.parametrize("rows,cols,br", [(1, 1, 1), (5, 16, 1), (5, 200, 128), (300, 1000, 128), (3, 128, 1)])
def test_its_own_codes_and_scales(rows, cols, br):
    own = ops.Fp8Matrix.empty(rows, cols, br, "cpu")
    m = ops.Fp8Matrix(own.codes, own.scale, br)
    assert m.shape == (rows, cols) and (m._c.codes, m._c.scale) == (own._c.codes, own._c.scale)
    assert rows == 1 or m._c.ld == own._c.ld
