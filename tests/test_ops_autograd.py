"""The operators and autograd: inputs that it follows are refused, Functions of the caller's give their gradients."""
import pytest
import torch

from paper_2412_20796_amd import binding as bd
from paper_2412_20796_amd import ops

gpu = pytest.mark.gpu


def test_inputs_that_autograd_follows_are_refused():
    """Their gradient would be lost without a word; with gradients off, as in a Function of the caller's, they are taken (and
    refused here only for lying in host memory)."""
    z, ln, up = torch.zeros(4, 128), torch.zeros(4, 64), torch.zeros(4, 64)
    table, tok, kept = torch.zeros(9, 64), torch.zeros(4, dtype=torch.int32), ops.GateCheckpoint.empty(4, 64, "cpu")
    f = lambda t: t.clone().requires_grad_(True)
    for call in (lambda: ops.gate_forward(f(z), ln), lambda: ops.gate_forward(z, f(ln), save=False),
                 lambda: ops.gate_backward(kept, f(ln), up), lambda: ops.gate_backward(kept, ln, f(up)),
                 lambda: ops.embed_forward(f(table), tok), lambda: ops.embed_backward(tok, f(up), 9)):
        with pytest.raises(bd.ChgnetError) as e:
            call()
        assert e.value.code == bd.CHGNET_EINVAL and "gradient" in str(e.value)
        with torch.no_grad(), pytest.raises(bd.ChgnetError) as e:
            call()
        assert "gradient" not in str(e.value) and "GPU" in str(e.value)


@gpu
def test_a_function_of_the_callers():
    """The gate and the lookup in torch.autograd.Functions, as documented: their gradients arrive."""

    class Gate(torch.autograd.Function):
        @staticmethod
        def forward(ctx, z, ln):
            phi, ctx.kept = ops.gate_forward(z, ln)
            ctx.ln = ln
            return phi

        @staticmethod
        def backward(ctx, dphi):
            return ops.gate_backward(ctx.kept, ctx.ln, dphi.contiguous())

    class Embed(torch.autograd.Function):
        @staticmethod
        def forward(ctx, table, tok):
            ctx.tok, ctx.vocab = tok, table.shape[0]
            return ops.embed_forward(table, tok, scale=2.0)

        @staticmethod
        def backward(ctx, dout):
            return ops.embed_backward(ctx.tok, dout.contiguous(), ctx.vocab, scale=2.0), None

    g = torch.Generator().manual_seed(8)
    table, ln = torch.randn(20, 128, generator=g).cuda().requires_grad_(True), torch.randn(4, 64, generator=g).cuda().requires_grad_(True)
    tok, up = torch.randint(0, 20, (300,), generator=g, dtype=torch.int32).cuda(), torch.randn(300, 64, generator=g).cuda()
    (Gate.apply(Embed.apply(table, tok), ln) * up).sum().backward()
    with torch.no_grad():
        _, kept = ops.gate_forward(ops.embed_forward(table, tok, scale=2.0), ln)
        dz, dln = ops.gate_backward(kept, ln, up)
        assert torch.equal(ln.grad, dln) and torch.equal(table.grad, ops.embed_backward(tok, dz, 20, scale=2.0))
