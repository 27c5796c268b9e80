"""Matrices in 8-bit floating point from tensors of the caller's (no GPU: what they are is checked on any device)."""
import pytest
import torch

from paper_2412_20796_amd import binding as bd
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


def test_both_forms_into_one_matrix_are_refused(monkeypatch):
    """A square x has two forms of one shape, each of which would be written over the other's codes."""
    monkeypatch.setattr(ops, "_start", lambda name, t: (*t.shape, t.dtype, 0, t.shape[1], t.get_device()))
    monkeypatch.setattr(ops, "_call", lambda *a: None)  # (no GPU)
    x = torch.zeros(64, 64)
    m = ops.Fp8Matrix.empty(64, 64, 1, "cpu")
    again = ops.Fp8Matrix(m.codes, m.scale)
    for t in (m, again):
        with pytest.raises(bd.ChgnetError) as e:
            ops.fp8_quantize_both(x, 1, m, t)
        assert e.value.code == bd.CHGNET_EINVAL and "same codes" in str(e.value)
    other = ops.Fp8Matrix.empty(64, 64, 1, "cpu")
    assert ops.fp8_quantize_both(x, 1, m, other) == (m, other)
    none = ops.Fp8Matrix.empty(0, 0, 1, "cpu")
    assert ops.fp8_quantize_both(torch.zeros(0, 0), 1, none, none) == (none, none)
