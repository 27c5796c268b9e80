"""The plain forms of block_reference.py: the generator against published answers, gradients against autograd."""
import numpy as np
import pytest
import torch

import block_reference as ref


@pytest.mark.parametrize("counter,key,want", [
    ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
    ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
    ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0),
     (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1)),
])
def test_published_answers_of_the_generator(counter, key, want):
    """The known answers that the generator's authors publish with it."""
    assert tuple(int(v) for v in ref.philox(*counter, *key)) == want


def test_share_of_kept_values():
    for p in (0.1, 0.5, 0.9):
        m, f = ref.kept(500, 333, p, 12345, 7)
        n = m.numel()
        assert abs(float(m.double().mean()) - (1 - p)) < 5 * (p * (1 - p) / n) ** 0.5 + 2.0 ** -17
        assert abs(f * (1 - p) - 1) < 2e-4


@pytest.mark.parametrize("pre_kind", ["rms", "layer"])
@pytest.mark.parametrize("post_kind", ["rms", "layer", "none", None])
@pytest.mark.parametrize("cols", [0, 1, 20])
def test_gradients_are_those_of_autograd(cols, post_kind, pre_kind):
    g = torch.Generator().manual_seed(cols)
    t = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64).requires_grad_(True)
    x, f, pre = t(5, 20), t(5, 20), t(2, 20)
    gate, post = (t(5, cols) if cols else None), (t(2, 20) if post_kind else None)
    dy, dh = torch.randn(5, 20, generator=g, dtype=torch.float64), torch.randn(5, 20, generator=g, dtype=torch.float64)
    mask, factor = ref.kept(5, 20, 0.3, 9, 1)
    kind = post_kind or "none"
    y, _ = ref.residual(x, f, post, kind, gate, 1.5, 0.7, mask, factor, 1e-5)
    h, _ = ref.norm(y, pre, pre_kind, 1e-5)
    leaves = [v for v in (x, f, gate, post, pre) if v is not None]
    want = torch.autograd.grad((y * dy).sum() + (h * dh).sum(), leaves)
    with torch.no_grad():
        got, bound = ref.residual_grad(y, f, dy, dh, post, kind, gate, pre, pre_kind, 1.5, 0.7, mask, factor, 1e-5)
    got = [got[n] for n in ("dx", "df", "dgate", "dpost", "dpre") if got[n] is not None]
    for a, b in zip(got, want):
        assert torch.allclose(a, b, rtol=1e-9, atol=1e-11)
