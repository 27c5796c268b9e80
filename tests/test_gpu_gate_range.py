"""The gate's forward and backward pass at values of 1e18 and more: both take a row's variance up to fp32's largest number
and count the row as all at its mean beyond it, at the same line, whatever the width."""
import pytest
import torch

import ops_reference as ref
from paper_2412_20796_amd import ops

pytestmark = pytest.mark.gpu


def _rows(rows, d, size, half):
    """z [rows, 2d] whose `half` has the deviation `size` in every row (to fp32's rounding of its values)."""
    g = torch.Generator().manual_seed(31 * d + half)
    z = torch.randn(rows, 2 * d, generator=g, dtype=torch.float64)
    x = z[:, half * d:(half + 1) * d]
    x -= x.mean(1, keepdim=True)
    x *= size / x.square().mean(1, keepdim=True).sqrt()
    ln = torch.randn(4, d, generator=g) * 0.3 + torch.tensor([[1.0], [0.0], [1.0], [0.0]])
    return z.float(), ln, torch.randn(rows, d, generator=g)


def _passes(z, ln, dphi):
    phi, kept = ops.gate_forward(z.cuda(), ln.cuda())
    return (phi, kept, *ops.gate_backward(kept, ln.cuda(), dphi.cuda()))


@pytest.mark.parametrize("half", [0, 1])
@pytest.mark.parametrize("d", [2, 3, 17, 64, 70, 130, 333, 1000, 1024])
@pytest.mark.parametrize("size", [5e17, 1e18, 3e18, 1e19, 1.8e19])
def test_variance_within_the_range(size, d, half):
    """Up to 1.8e19 a row's variance is at most 3.24e38, in fp32's range: both passes are those of the definition. (The
    checkpoint's deviation is off by 1/510 of the range at most, half a percent where three values make a row: 3.28e38.)"""
    z, ln, dphi = _rows(37, d, size, half)
    phi, kept, dz, dln = _passes(z, ln, dphi)
    r, b = ref.gate(z, ln)
    ref.assert_within(phi, r, b, what="phi")
    q, step, _ = ref.checkpoint(z)
    assert torch.equal(kept.codes.cpu().double(), q) and torch.equal(kept.step.cpu().double(), step)
    rz, rl, bz, bl = ref.gate_grad(q, step, ln, dphi)
    ref.assert_within(dz, rz, bz, what="dz")
    ref.assert_within(dln, rl, bl, what="dln")


@pytest.mark.parametrize("half", [0, 1])
@pytest.mark.parametrize("d", [2, 3, 17, 64, 70, 130, 333, 1000, 1024])
@pytest.mark.parametrize("size", [1.9e19, 5e19, 1e25])
def test_variance_past_the_range(size, d, half):
    """From 1.9e19 on it is at least 3.6e38, past fp32's range: the half counts as all at its mean in both passes."""
    z, ln, dphi = _rows(37, d, size, half)
    phi, kept, dz, dln = _passes(z, ln, dphi)
    s = slice(half * d, (half + 1) * d)
    mid = z.clone()
    mid[:, s] = 0
    r, b = ref.gate(mid, ln)
    ref.assert_within(phi, r, b, what="phi")
    assert not bool(dz[:, s].any()) and not bool(dln[2 * half].any())


@pytest.mark.parametrize("d", [2, 64, 70, 333, 1024])
@pytest.mark.parametrize("value", [1e30, -1e36, 1e37, 3e38])
def test_sum_past_the_range(value, d):
    """A half of large equal values, whose sum passes fp32's range: its mean does not, so that phi is a number. d values of
    which the mean is exact (d a power of two) are all at their mean, 0; else the mean's rounding is 1e-7 of the value."""
    z, ln, _ = _rows(9, d, 1.0, 1)
    z[:, :d] = value
    phi = ops.gate_forward(z.cuda(), ln.cuda(), save=False)
    mid = z.clone()
    mid[:, :d] = 0
    if d & (d - 1) == 0:
        r, b = ref.gate(mid, ln)
        ref.assert_within(phi, r, b)
    else:
        assert bool(torch.isfinite(phi).all())


def test_scales_up_to_the_range():
    """A LayerNorm scale next to fp32's largest number, at a value next to its row's mean: their product is in range, and
    phi a number."""
    z, ln, _ = _rows(37, 64, 1.0, 0)
    ln[0, 5] = 3e38
    z[:, 5] = z[:, [k for k in range(64) if k != 5]].mean(1)
    assert bool(torch.isfinite(ops.gate_forward(z.cuda(), ln.cuda(), save=False)).all())
