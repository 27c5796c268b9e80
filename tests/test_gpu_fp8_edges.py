"""8-bit matrices and their products at the edges of what they take."""
import pytest
import torch

import fp8_reference as ref
from ops_reference import assert_within
from paper_2412_20796_amd import ops

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows", [1, 16, 17, 300, 3000, 16400, 20000])
@pytest.mark.parametrize("N", [1, 100, 128, 129, 200, 256, 257, 1000])
def test_linear_without_columns(N, rows, dtype):
    """A weight [N, 0] has no codes and no scales, and may have no memory: every result is an empty sum."""
    w = ops.Fp8Matrix.empty(N, 0, 128)
    out = torch.full((rows, N), 7.0, dtype=dtype, device="cuda")
    ops.fp8_linear(torch.empty(rows, 0, dtype=dtype, device="cuda"), w, out=out)
    assert not out.any()


@pytest.mark.parametrize("M,N", [(1, 40), (16, 8200), (17, 40), (300, 515), (4100, 4100), (17000, 200)])
def test_products_without_columns(M, N):
    a, b = ops.Fp8Matrix.empty(M, 0), ops.Fp8Matrix.empty(N, 0, 128)
    for dtype in (torch.float32, torch.bfloat16):
        out = torch.full((M, N), 7.0, dtype=dtype, device="cuda")
        assert bool((ops.fp8_matmul(a, b, out=out, accumulate=True) == 7).all())
        assert not ops.fp8_matmul(a, b, out=out).any()


def _held(m):
    """A matrix's values in 64 bits, of its codes and scales (which are checked elsewhere)."""
    rows = m.scale.float().double().repeat_interleave(m.block_rows, 0)[:m.rows]
    return (m.codes.float().double() * rows.repeat_interleave(128, 1)[:, :m.cols]).cpu()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("N", [100, 128, 200, 256])
@pytest.mark.parametrize("rows,K", [(16384, 2048), (16399, 1400)])
def test_many_rows_of_many_steps(rows, K, N, dtype):
    """Rows that are quantised on their way, where a step's codes of the weight arrive behind the rows of the next: each call
    of several has the same bits, and those of the definition."""
    g = torch.Generator().manual_seed(rows + N)
    x = torch.randn(rows, K, generator=g).to(dtype).cuda()
    w = ops.fp8_quantize(torch.randn(N, K, generator=g).cuda() / K ** 0.5, 128)
    out = ops.fp8_linear(x, w)
    for _ in range(3):
        assert torch.equal(ops.fp8_linear(x, w), out)
    r, b = ref.product(_held(ops.fp8_quantize(x)), _held(w), dtype)
    assert_within(out, r, b, dtype)
