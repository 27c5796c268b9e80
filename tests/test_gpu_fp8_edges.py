"""8-bit matrices and their products at the edges of what they take."""
import pytest
import torch

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
