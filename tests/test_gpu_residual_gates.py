"""The gate's gradient in the residual connection for gates that are nearly open or shut, where s (1 - s) is small: it is as
good there, for its size, as elsewhere."""
import pytest
import torch

import block_reference as ref
from ops_reference import assert_within
from paper_2412_20796_amd import ops

pytestmark = pytest.mark.gpu
U = ref.U


def _relative(g):
    """Relative error of dy t s (1 - s), counted in last places: with e = exp(-|g|) off by (2 |g| + 2) U (the constant, the
    argument, the exponential), 1 / (1 + e) by (|g| + 4) U (at most half of e's, the sum, the reciprocal), of s and 1 - s one is that and the
    other its product with e, and there are five more products and sums."""
    return (4 * g.abs() + 20) * U


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [8, 72, 333, 1000, 2048, 16384])
@pytest.mark.parametrize("cols", [1, None])
def test_gates_from_shut_to_open(cols, d, dtype):
    g = torch.Generator().manual_seed(d)
    values = torch.tensor([-80.0, -40.0, -20.0, -17.0, -15.0, -12.0, -3.0, -1.0, 0.0, 1.0, 3.0, 8.0, 12.0, 15.0, 17.0, 18.0, 20.0,
                           40.0, 80.0])
    n = cols or d
    gate = values[(torch.arange(19)[:, None] + torch.arange(n)) % 19].to(dtype)
    x, f, dy = (torch.randn(19, d, generator=g).to(dtype) for _ in range(3))
    y, _ = ops.residual_forward(x.cuda(), f.cuda(), gate=gate.cuda())
    got = ops.residual_backward(y, f.cuda(), dy.cuda(), gate=gate.cuda()).dgate
    v = gate.double()
    # (1 - s as a sigmoid of its own: nothing cancels)
    slope, term = torch.sigmoid(v) * torch.sigmoid(-v), dy.double() * f.double()
    want, size = (term * slope, term.abs() * slope) if cols is None else (
        (term * slope).sum(1, keepdim=True), (term * slope).abs().sum(1, keepdim=True))
    bound = (_relative(v) + (0 if cols is None else ref.D * U)) * size + 1e-37
    assert_within(got, want, bound, dtype, "d=%d" % d)


def test_gates_at_the_ends():
    """Gates of infinity pass all or nothing, and no gradient; a gate of NaN is its own value's and row's only."""
    x = torch.ones(4, 64, device="cuda")
    gate = torch.zeros(4, 64, device="cuda")
    gate[0], gate[1], gate[2, 5] = float("inf"), float("-inf"), float("nan")
    y, _ = ops.residual_forward(x, x, gate=gate)
    grad = ops.residual_backward(y, x, x, gate=gate)
    assert torch.equal(y[0], 2 * x[0]) and torch.equal(y[1], x[1]) and torch.equal(y[3], 1.5 * x[3])
    assert not grad.dgate[:2].any() and torch.equal(grad.df[0], x[0]) and not grad.df[1].any()
    nan = torch.isnan(torch.stack([y, grad.dgate, grad.df]))
    assert bool(nan[:, 2, 5].all()) and int(nan.sum()) == 3
    assert torch.equal(grad.dgate[3], 0.25 * x[3]) and torch.equal(grad.dx, x)


@pytest.mark.parametrize("cols", [1, 40])
def test_against_differences(cols):
    """Central differences in 64 bits of the definition, for gates from -18 to 18. f and dy are whole numbers, and each gate's
    difference is taken where its slope is: relative to it."""
    g = torch.Generator().manual_seed(3)
    f, dy = (torch.randint(1, 9, (37, 40), generator=g).double() for _ in range(2))
    gate = torch.arange(-18, 19).double()[:, None].repeat(1, cols)
    x = torch.zeros(37, 40, device="cuda")
    y, _ = ops.residual_forward(x, f.float().cuda(), gate=gate.float().cuda())
    got = ops.residual_backward(y, f.float().cuda(), dy.float().cuda(), gate=gate.float().cuda()).dgate.cpu().double()
    # of sigmoid(v) for v < 0, of sigmoid(v) - 1 = -sigmoid(-v) else, which differ by a constant: nothing cancels but the step
    part = lambda v: torch.where(gate < 0, torch.sigmoid(v), -torch.sigmoid(-v))
    h = 1e-4
    num = ((part(gate + h) - part(gate - h)) / (2 * h) * (f * dy if cols > 1 else (f * dy).sum(1, keepdim=True)))
    # the step's: h^2 / 6 of the third derivative, which is at most 1 times the slope; 2^-50 / h for roundings of the two values
    # (at most twice the slope) and 2^-48 / h for those of gate + h
    assert bool(((got - num).abs() <= ((4 * 18 + 20 + ref.D) * U + h * h / 6 + 2.0 ** -47 / h) * num.abs()).all())
