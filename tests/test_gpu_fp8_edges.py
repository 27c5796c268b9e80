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


@pytest.mark.parametrize("br", [1, 128])
@pytest.mark.parametrize("M", [1, 3])
def test_more_columns_than_one_launch_has(M, br):
    """2^28 columns and some for few rows: 2^32 threads and more in blocks of 32 columns."""
    N, K, part = (1 << 28) + 37, 16, 1 << 20
    g = torch.Generator().manual_seed(M)
    few = ops.fp8_quantize(torch.randn(part, K, generator=g).cuda(), br)
    codes = torch.empty(N, K, dtype=torch.uint8, device="cuda")
    scale = torch.zeros(-(-N // br), 4, dtype=torch.uint8, device="cuda")
    for n in range(0, N, part):
        m = min(part, N - n)
        codes[n:n + m] = few.codes.view(torch.uint8)[:m]
        scale[n // br:-(-(n + m) // br), :1] = few.scale.view(torch.uint8)[:-(-m // br)]
    w = ops.Fp8Matrix(codes.view(torch.float8_e4m3fn), scale.view(torch.float8_e8m0fnu)[:, :1], br)
    x = torch.randn(M, K, generator=g).to(torch.bfloat16).cuda()
    want = ops.fp8_linear(x, few)
    r, b = ref.product(_held(ops.fp8_quantize(x)), _held(few), torch.bfloat16)
    assert_within(want, r, b, torch.bfloat16)
    for out in (ops.fp8_linear(x, w), ops.fp8_matmul(ops.fp8_quantize(x), w)):
        assert out.shape == (M, N)
        for n in range(0, N, part):
            m = min(part, N - n)
            assert torch.equal(out[:, n:n + m], want[:, :m]), n


def _whole(rows, cols, most, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-most, most + 1, (rows, cols), generator=g).float().cuda()


# values up to `most`, whose sums (of standard deviation most (most + 1) / 3 sqrt K) mostly are numbers of the type; all are of
# fp32 (up to 9,000 8^2), so that a result is the sum rounded once
WHOLE = [(torch.bfloat16, 1), (torch.float16, 3), (torch.float32, 8)]


@pytest.mark.parametrize("dtype,most", WHOLE)
@pytest.mark.parametrize("M,N,K", [(1, 300, 3000), (16, 8200, 3000), (17, 40, 3000), (130, 257, 3000), (300, 515, 9000),
                                   (2050, 2050, 1000), (4100, 4100, 1000)])
def test_sums_of_whole_numbers_are_exact(M, N, K, dtype, most):
    """In all product kernels and types: products of whole numbers up to 2^6 are far from being cut off."""
    a, b = _whole(M, K, most, 1), _whole(N, K, min(most, 1 if K > 3000 else most), 2)
    want = a.double() @ b.double().T
    got = ops.fp8_matmul(ops.fp8_quantize(a), ops.fp8_quantize(b, 128), dtype)
    assert torch.equal(got, want.to(dtype))


@pytest.mark.parametrize("dtype,most", WHOLE)
@pytest.mark.parametrize("rows,N,K", [(1, 300, 3000), (16, 8200, 3000), (40, 300, 3000), (16400, 100, 3000), (16400, 200, 3000),
                                      (16400, 200, 500)])
def test_linear_layers_of_whole_numbers_are_exact(rows, N, K, dtype, most):
    x, w = _whole(rows, K, most, 3), _whole(N, K, most, 4)
    want = x.double() @ w.double().T
    assert torch.equal(ops.fp8_linear(x.to(dtype), ops.fp8_quantize(w, 128)), want.to(dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,N,K", [(3, 4096, 4096), (1000, 1000, 4096), (2048, 2048, 4096), (4096, 4096, 4096)])
def test_sums_behind_16_bit_results(M, N, K, dtype):
    """How far sums are off before they are rounded to 16 bits, for normal values: what is left after adding the product to the
    rounded result's negative, which is off by half a step of what is left only (half a step squared, of the result).

    Of eight products of 8 significant bits, those below 2^-6 of the largest one's power of two lose bits, less than 2^-13 of
    it. Of normal values these are 2.4 %, and the root mean square of their largest losses is 3.9e-5 of a product's (modelled in
    64 bits); signs are random, so that a sum's relative to its size is the same. fp32's own sums are off by less than 1e-6."""
    g = torch.Generator().manual_seed(M)
    a, b = (ops.fp8_quantize(torch.randn(n, K, generator=g).cuda(), br) for n, br in ((M, 1), (N, 128)))
    exact = _held(a).cuda() @ _held(b).cuda().T
    out = (-exact).to(dtype)
    half = torch.finfo(dtype).eps / 2
    left = exact + out.double()
    ops.fp8_matmul(a, b, out=out, accumulate=True)
    off = float((out.double() - left).norm() / exact.norm())
    assert off <= 4e-5 + half * half, off
