"""Dropout's p counts in steps of 2^-16, rounded from the number that the caller gives and not from that number in fp32, which
may lie on the other side of a half step."""
import math

import pytest
import torch

import block_reference as ref
from paper_2412_20796_amd import binding as bd
from paper_2412_20796_amd import ops

# steps above and below a half by less than fp32 resolves there (a tie goes up), and a number met by chance
NEAR = [0.2692794774414212] + [(k + 0.5) / 65536 + e for k in (17647, 40000, 65534) for e in (-1e-9, 0.0, 1e-9)]
P = NEAR + [0.0, 2.0 ** -18, 2.0 ** -17, 0.1, 0.5, 0.9, 1.0 - 2.0 ** -18, 1.0]
STEPS = {p: math.floor(p * 65536 + 0.5) for p in P}


def _cfg_rate(p):
    """As residual_forward and residual_backward pass it on (no GPU is needed for that)."""
    f = torch.zeros(4, 8)
    return ops._residual(f, None, None, None, None, "rms", 1.0, 1.0, p, 1, 2, None, 1e-5, 4, 8, torch.float32, -1)[0].p


@pytest.mark.parametrize("p", P)
def test_rate_of_the_residual_connection(p):
    assert _cfg_rate(p) * 65536 == STEPS[p]


def test_some_of_these_rates_are_others_in_fp32():
    """Else the tests here would not see a rounding to fp32 before the one to steps."""
    assert sum(math.floor(float(torch.tensor(p, dtype=torch.float32)) * 65536 + 0.5) != STEPS[p] for p in NEAR) >= 3


@pytest.mark.parametrize("p", [-1e-9, 1.0 + 1e-9, 2.0, float("nan"), float("inf"), -1.0])
def test_rates_out_of_range(p):
    with pytest.raises(bd.ChgnetError) as e:
        _cfg_rate(p)
    assert e.value.code == bd.CHGNET_EINVAL and "p must be" in str(e.value)


@pytest.mark.gpu
@pytest.mark.parametrize("p", P)
def test_mask_and_factor(p):
    """The mask of the definition's step, whose half is a number in fp32 too, and its factor. 65,536 values and more: one in
    as many tells two steps apart; and the residual connection's."""
    rows, d, seed, call = 4000, 72, 5, 6
    x = torch.ones(rows, d)
    q = STEPS[p] / 65536
    want = ref.dropout(x, q, seed, call)
    assert torch.equal(ops.dropout(x.cuda(), p, seed, call).cpu(), want)
    zero = torch.zeros(rows, d, device="cuda")
    y, _ = ops.residual_forward(zero, x.cuda(), p=p, seed=seed, call=call)
    assert torch.equal(y.cpu(), want)
    grad = ops.residual_backward(y, x.cuda(), x.cuda(), p=p, seed=seed, call=call)
    assert torch.equal(grad.df.cpu(), want)


@pytest.mark.gpu
@pytest.mark.parametrize("p", [-1e-9, 1.0 + 1e-9, float("nan"), None, "0.1"])
def test_refusals(p):
    x = torch.zeros(4, 8, device="cuda")
    for call in (lambda: ops.dropout(x, p, 1), lambda: ops.residual_forward(x, x, p=p)):
        with pytest.raises(bd.ChgnetError) as e:
            call()
        assert e.value.code == bd.CHGNET_EINVAL
