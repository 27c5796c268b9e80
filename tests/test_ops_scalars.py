"""Factors and rates that a call of the operators gets: their values at the call count, whatever object holds them."""
import numpy as np
import pytest
import torch

from paper_2412_20796_amd import binding as bd
from paper_2412_20796_amd import ops

FACTORS = ("alpha", "beta", "eps", "p")


def _cfg(**kw):
    """The struct that residual_forward and residual_backward pass on (its checks do not need a GPU)."""
    how = dict(dict(alpha=1.0, beta=1.0, p=0.25, seed=1, call=2, step=None, eps=1e-5), **kw)
    f = torch.zeros(4, 8)
    return ops._residual(f, None, None, None, None, "rms", rows=4, d=8, dtype=torch.float32, gpu=-1, **how)[0]


@pytest.mark.parametrize("make", [lambda v: torch.tensor(v), lambda v: torch.tensor(v, dtype=torch.float64),
                                  lambda v: torch.tensor([v])])
@pytest.mark.parametrize("name", FACTORS)
def test_a_tensor_that_changes(name, make):
    """A factor in a tensor that is updated in place between two calls."""
    t = make(0.5)
    assert getattr(_cfg(**{name: t}), name) == 0.5
    t.fill_(0.75)
    assert getattr(_cfg(**{name: t}), name) == 0.75
    t.fill_(0.5)
    assert getattr(_cfg(**{name: t}), name) == 0.5


@pytest.mark.parametrize("name", FACTORS)
def test_an_object_that_changes(name):
    class Factor:
        value = 0.5

        def __float__(self):
            return self.value

    f = Factor()
    assert getattr(_cfg(**{name: f}), name) == 0.5
    f.value = 0.25
    assert getattr(_cfg(**{name: f}), name) == 0.25


@pytest.mark.parametrize("value", [1, True, np.float32(1), np.float64(1), np.int64(1)])
def test_other_numbers(value):
    for name in FACTORS:
        assert getattr(_cfg(**{name: value}), name) == 1.0


@pytest.mark.parametrize("name", FACTORS)
def test_what_is_no_number_and_what_autograd_follows(name):
    for bad in (None, "a", torch.zeros(2), [1.0]):
        with pytest.raises(bd.ChgnetError) as e:
            _cfg(**{name: bad})
        assert e.value.code == bd.CHGNET_EINVAL and name in str(e.value)
    t = torch.tensor(0.5, requires_grad=True)
    with pytest.raises(bd.ChgnetError) as e:
        _cfg(**{name: t})
    assert "gradient" in str(e.value)
    with torch.no_grad():
        assert getattr(_cfg(**{name: t}), name) == 0.5


@pytest.mark.gpu
def test_a_learned_factor_between_two_steps():
    g = torch.Generator().manual_seed(1)
    x, f, dy = (torch.randn(9, 72, generator=g).cuda() for _ in range(3))
    alpha, beta = torch.tensor(1.0), torch.tensor(0.5)
    for a, b in ((1.0, 0.5), (2.0, -0.25), (1.0, 0.5)):
        alpha.fill_(a)
        beta.fill_(b)
        y, _ = ops.residual_forward(x, f, alpha=alpha, beta=beta)
        grad = ops.residual_backward(y, f, dy, alpha=alpha, beta=beta)
        # (powers of two: the products are exact)
        assert torch.equal(y, a * x + b * f) and torch.equal(grad.dx, a * dy) and torch.equal(grad.df, b * dy)
