"""chgnet_fp8_quantize, chgnet_fp8_matmul and chgnet_fp8_linear against their definitions (fp8_reference.py): codes and scales
bit for bit, products within the bound derived there; sizes around tiles, blocks and 16 bytes, strides, matrices of the
caller's, scales to the ends of their range, values that are not finite, parts of K, streams and graphs."""
import itertools

import pytest
import torch

import fp8_reference as ref
from ops_reference import assert_within
from paper_2412_20796_amd import binding as bd
from paper_2412_20796_amd import ops

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _x(rows, cols, dtype=torch.float32, seed=0):
    g = torch.Generator().manual_seed(rows + 7919 * cols + seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(torch.randn(rows, 1, generator=g)) * torch.exp(
        0.5 * torch.randn(1, cols, generator=g))
    if rows > 4:
        x[2, :130] = 0  # blocks of zeros
    return x.to(dtype)


def _check_matrix(m, x, block_rows, what=""):
    q, byte = ref.quantize(x, block_rows)
    assert torch.equal(m.scale.cpu().view(torch.uint8).long(), byte), what
    fine = (byte != 255).repeat_interleave(block_rows, 0)[:x.shape[0]].repeat_interleave(128, 1)[:, :x.shape[1]]
    got = m.codes.cpu().float().double()
    assert torch.equal(torch.where(fine, got, 0.0), torch.where(fine, q, 0.0)), what
    if m._data is not None and m.cols % 16 and m.rows:
        raw = m._data[:m.rows * m._c.ld].view(m.rows, -1)[:, m.cols:-(-m.cols // 16) * 16]
        assert not raw.any(), what
    return ref.values(q, byte, block_rows)


def _random(rows, cols, block_rows=1, seed=0, spread=6):
    """An Fp8Matrix and its values, from codes and scales of their own."""
    g = torch.Generator().manual_seed(rows * 31 + cols * 17 + seed)
    ld, lds = -(-cols // 16) * 16, -(-cols // 512) * 4
    codes = torch.zeros(rows, ld)
    codes[:, :cols] = torch.randn(rows, cols, generator=g) * 30
    codes = codes.to(torch.float8_e4m3fn)
    byte = torch.zeros(-(-rows // block_rows), lds, dtype=torch.uint8)
    nb = -(-cols // 128)
    byte[:, :nb] = torch.randint(127 - spread, 127 + spread, (byte.shape[0], nb), generator=g).to(torch.uint8)
    m = ops.Fp8Matrix(codes.cuda()[:, :cols], byte.cuda().view(torch.float8_e8m0fnu)[:, :nb], block_rows)
    return m, ref.values(codes[:, :cols].double(), byte[:, :nb].long(), block_rows)


SIZES = [(1, 1), (1, 128), (3, 127), (2, 16), (5, 200), (128, 128), (129, 130), (256, 512), (37, 1000), (513, 96), (300, 257)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_quantize(rows, cols, dtype):
    x = _x(rows, cols, dtype)
    for br in (1, 128):
        what = "%s %s %d" % ((rows, cols), dtype, br)
        _check_matrix(ops.fp8_quantize(x.cuda(), br), x, br, what)
        _check_matrix(ops.fp8_quantize(x.cuda(), br, transposed=True), x.T, br, what + " T")
        q, t = ops.fp8_quantize_both(x.cuda(), br)
        _check_matrix(q, x, br, what + " both")
        _check_matrix(t, x.T, br, what + " both T")
        if br == 128:
            assert torch.equal(q.codes.cpu().float().T, t.codes.cpu().float())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (8, 1), (16, 8)])
def test_quantize_strided_rows(pad, shift, dtype):
    x = _x(70, 200, dtype)
    buf = torch.full((shift + 70 * (200 + pad),), float("nan"), dtype=dtype, device="cuda")
    v = buf[shift:].reshape(70, 200 + pad)[:, :200]
    v.copy_(x)
    for q, y in zip(ops.fp8_quantize_both(v), (x, x.T)):
        _check_matrix(q, y, 1)
    _check_matrix(ops.fp8_quantize(v), x, 1)


def test_quantize_at_the_borders_of_the_scale():
    """Largest magnitudes of 448 2^k and next to it, of fp32's largest, of subnormal numbers, of zero; ties."""
    up = lambda v: float(torch.nextafter(torch.tensor(v), torch.tensor(float("inf"))))
    down = lambda v: float(torch.nextafter(torch.tensor(v), torch.tensor(0.0)))
    most = torch.finfo(torch.float32).max
    bigs = [448.0, up(448.0), down(448.0), 1.75, up(1.75), 1.0, 2.0 ** -130, 2.0 ** -149, 448 * 2.0 ** -126, up(448 * 2.0 ** -126),
            most, 1.75 * 2.0 ** 127, up(1.75 * 2.0 ** 127), 1e-20, 3e30, 0.0]
    x = torch.rand(len(bigs), 128, generator=torch.Generator().manual_seed(1)) * 2 - 1
    x = x * torch.tensor(bigs)[:, None]
    x[:, 5] = -torch.tensor(bigs)
    x[0, 6:22] = torch.arange(16) / 2 + 0.25  # between two codes
    x[0, 22:40] = (torch.arange(18) - 9 + 0.5) * 2.0 ** -9  # subnormal codes' ties
    _check_matrix(ops.fp8_quantize(x.cuda()), x, 1)
    q, t = ops.fp8_quantize_both(x.cuda())
    _check_matrix(q, x, 1)
    _check_matrix(t, x.T, 1)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_values_that_are_not_finite(value):
    """NaN in their blocks' scales, and so in the results of their row and column, and in no others."""
    a, b = _x(40, 300), _x(50, 300, seed=1)
    a[7, 200] = value
    for q in (ops.fp8_quantize(a.cuda()), ops.fp8_quantize_both(a.cuda())[0]):
        _check_matrix(q, a, 1)
        out = ops.fp8_matmul(q, ops.fp8_quantize(b.cuda()), torch.float32).cpu()
        assert bool(torch.isnan(out[7]).all()) and not bool(torch.isnan(out[torch.arange(40) != 7]).any())
        out = ops.fp8_matmul(ops.fp8_quantize(b.cuda()), q, torch.float32).cpu()
        assert bool(torch.isnan(out[:, 7]).all()) and not bool(torch.isnan(out[:, torch.arange(40) != 7]).any())
    for rows in (40, 3):
        out = ops.fp8_linear(a[5:5 + rows].cuda(), ops.fp8_quantize(b.cuda())).cpu()
        assert bool(torch.isnan(out[2]).all()) and not bool(torch.isnan(out[torch.arange(out.shape[0]) != 2]).any())


@pytest.mark.parametrize("N,K", [(100, 200), (200, 200), (200, 700)])
def test_values_that_are_not_finite_in_many_rows(N, K):
    x, w = _x(16400, K), ops.fp8_quantize(_x(N, K, seed=1).cuda(), 128)
    x[33, K - 1], x[16399, 0] = float("nan"), float("-inf")
    out = ops.fp8_linear(x.cuda(), w).cpu()
    rows = torch.zeros(16400, dtype=torch.bool)
    rows[[33, 16399]] = True
    assert bool(torch.isnan(out[rows]).all()) and bool(torch.isfinite(out[~rows]).all())


def _check_product(a, va, b, vb, dtype=torch.float32, what="", **kw):
    out = ops.fp8_matmul(a, b, dtype, **kw)
    r, bound = ref.product(va, vb, dtype)
    assert_within(out, r, bound, dtype, what)
    return out


@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 33, 64, 65, 100, 128, 129, 255, 256, 257, 300])
@pytest.mark.parametrize("N,K", [(1, 1), (16, 16), (17, 100), (64, 128), (100, 129), (128, 640), (129, 500), (256, 127),
                                 (260, 1040), (515, 256)])
def test_products(M, N, K):
    for bra, brb in ((1, 128), (1, 1)):
        a, va = _random(M, K, bra, 1)
        b, vb = _random(N, K, brb, 2)
        _check_product(a, va, b, vb, what="%s %s" % ((M, N, K), (bra, brb)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(5, 300, 384), (130, 70, 256), (300, 515, 200), (1, 4096, 4096), (64, 1000, 2048),
                                   (2000, 1030, 300), (1030, 2100, 131)])
def test_types(M, N, K, dtype):
    a, va = _random(M, K, 1, 3, spread=2)
    b, vb = _random(N, K, 128, 4, spread=2)
    va, vb = va / 1024, vb / 1024  # (in fp16's range)
    a._scale.view(torch.uint8).sub_(10)
    b._scale.view(torch.uint8).sub_(10)
    _check_product(a, va, b, vb, dtype, "%s %s" % ((M, N, K), dtype))


def test_both_blocks_of_128_rows():
    a, va = _random(200, 300, 128, 3)
    b, vb = _random(150, 300, 128, 4)
    _check_product(a, va, b, vb)


@pytest.mark.parametrize("M,N,K", [(256, 512, 20000), (40, 50, 70001), (1, 1, 100000), (300, 200, 9000), (128, 128, 4096),
                                   (1000, 500, 24600), (1000, 1030, 49200)])
def test_long_sums(M, N, K):
    """Products whose K is divided."""
    a, va = _random(M, K, 1, 5)
    b, vb = _random(N, K, 1, 6)
    first = _check_product(a, va, b, vb)
    assert torch.equal(first, ops.fp8_matmul(a, b, torch.float32))
    base = torch.randn(M, N, generator=torch.Generator().manual_seed(1)).cuda()
    got = ops.fp8_matmul(a, b, out=base.clone(), accumulate=True)
    assert torch.equal(got, base + first)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(5, 40, 256), (100, 201, 300), (300, 515, 9000), (2000, 2050, 200)])
def test_accumulate(M, N, K, dtype):
    a, va = _random(M, K, 1, 5, spread=1)
    b, vb = _random(N, K, 128, 6, spread=1)
    a._scale.view(torch.uint8).sub_(8)
    va = va / 256
    base = torch.randn(M, N, generator=torch.Generator().manual_seed(1)).to(dtype)
    got = ops.fp8_matmul(a, b, out=base.cuda(), accumulate=True)
    r, bound = ref.product(va, vb, dtype)
    # one more rounding of the sum in fp32, and the one to the type
    assert_within(got, r + base.double(), bound + ref.U * (r.abs() + base.double().abs()), dtype)


@pytest.mark.parametrize("M,N,K", [(0, 5, 64), (5, 0, 64), (5, 7, 0)])
def test_empty(M, N, K):
    a, b = (ops.fp8_quantize(torch.ones(r, K, device="cuda")) for r in (M, N))
    out = ops.fp8_matmul(a, b, torch.float32)
    assert out.shape == (M, N) and not out.any()
    if K == 0:
        kept = torch.full((M, N), 3.0, device="cuda")
        assert bool((ops.fp8_matmul(a, b, out=kept, accumulate=True) == 3).all())
    y = ops.fp8_linear(torch.ones(M, K, device="cuda"), b)
    assert y.shape == (M, N) and not y.any()


def test_scales_to_the_ends_of_their_range():
    """2^-127 to 2^127 in one factor, their inverses in the other; for results in fp32 as far as the values are fp32 numbers
    (bf16's least normal one is the same)."""
    K = 512
    a, va = _random(64, K, 1, 7)
    b, vb = _random(64, K, 1, 8)
    for dtype, e in [(torch.bfloat16, e) for e in (0, 1, 100, 200, 254)] + [(torch.float32, e) for e in (20, 100, 200, 234)]:
        a._scale.view(torch.uint8).fill_(e)
        b._scale.view(torch.uint8).fill_(254 - e)
        _check_product(a, a.codes.cpu().double(), b, b.codes.cpu().double(), dtype, "2^%d" % (e - 127))
    # results next to the ends of fp32's range
    for ea, eb in ((127 + 60, 127 + 50), (127 - 60, 127 - 50)):
        a._scale.view(torch.uint8).fill_(ea)
        b._scale.view(torch.uint8).fill_(eb)
        f = 2.0 ** (ea + eb - 254)
        _check_product(a, a.codes.cpu().double() * f, b, b.codes.cpu().double())


def test_sums_of_whole_numbers_are_exact():
    g = torch.Generator().manual_seed(3)
    a, b = (torch.randint(-8, 9, (n, 3000), generator=g).float() for n in (130, 257))
    out = ops.fp8_matmul(ops.fp8_quantize(a.cuda()), ops.fp8_quantize(b.cuda()), torch.float32)
    assert torch.equal(out.cpu().double(), a.double() @ b.double().T)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,pad,shift", [(64, 4, 0), (64, 3, 0), (64, 4, 1), (333, 7, 2)])
def test_strided_results(N, pad, shift, dtype):
    a, va = _random(150, 256, 1, 9, spread=1)
    b, vb = _random(N, 256, 128, 10, spread=1)
    va, a = va / 64, (a._scale.view(torch.uint8).sub_(6), a)[1]
    buf = torch.full((shift + 150 * (N + pad),), 7.0, dtype=dtype, device="cuda")
    v = buf[shift:].reshape(150, N + pad)[:, :N]
    ops.fp8_matmul(a, b, out=v)
    r, bound = ref.product(va, vb, dtype)
    assert_within(v, r, bound, dtype)
    v.fill_(7.0)
    assert bool((buf == 7).all())


def test_strided_factors():
    """Codes and scales inside wider buffers, which hold NaN elsewhere."""
    M, N, K = 70, 90, 272
    made = []
    for rows, br, seed in ((M, 1, 1), (N, 128, 2)):
        m, v = _random(rows, K, br, seed)
        codes = torch.full((rows, K + 64), 0x7F, dtype=torch.uint8, device="cuda")
        scale = torch.full((-(-rows // br), 16), 255, dtype=torch.uint8, device="cuda")
        codes[:, 16:16 + K] = m.codes.view(torch.uint8)
        scale[:, 4:7] = m.scale.view(torch.uint8)
        made.append((ops.Fp8Matrix(codes.view(torch.float8_e4m3fn)[:, 16:16 + K], scale.view(torch.float8_e8m0fnu)[:, 4:7], br), v))
    _check_product(*made[0], *made[1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [1, 2, 3, 8, 16, 17, 31, 32, 33, 64, 65, 200, 1500])
@pytest.mark.parametrize("N,K,br", [(64, 128, 128), (129, 500, 1), (256, 512, 128), (1000, 1100, 128)])
def test_linear(rows, N, K, br, dtype):
    x, w = _x(rows, K, dtype), _x(N, K, torch.float32, 5) / 8
    m = ops.fp8_quantize(w.cuda(), br)
    out = ops.fp8_linear(x.cuda(), m)
    r, b = ref.product(ref.values(*ref.quantize(x)), ref.values(*ref.quantize(w, br), br), dtype)
    assert_within(out, r, b, dtype, str((rows, N, K, br)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,K,N,br", [(16400, 128, 256, 128), (16385, 100, 1, 1), (16500, 520, 128, 128), (17001, 300, 130, 1),
                                         (16384, 384, 200, 1), (16390, 640, 250, 128), (40001, 512, 256, 128),
                                         (20000, 16, 129, 1)])
def test_linear_of_many_rows(rows, K, N, br, dtype):
    x, w = _x(rows, K, dtype), _x(N, K, torch.float32, 5) / 8
    x[2] = 0
    m = ops.fp8_quantize(w.cuda(), br)
    out = ops.fp8_linear(x.cuda(), m)
    some = torch.cat([torch.arange(0, 70), torch.arange(rows - 70, rows), torch.arange(5000, 5070)])
    r, b = ref.product(ref.values(*ref.quantize(x[some])), ref.values(*ref.quantize(w, br), br), dtype)
    assert_within(out.cpu()[some], r, b, dtype)
    # and all of them at the codes that the quantiser gives, which are checked elsewhere
    q = ops.fp8_quantize(x.cuda())
    held = q.codes.float().double() * q.scale.float().double().repeat_interleave(128, 1)[:, :K]
    r, b = ref.product(held.cpu(), ref.values(*ref.quantize(w, br), br), dtype)
    assert_within(out, r, b, dtype)


@pytest.mark.parametrize("pad,shift", [(8, 0), (5, 0), (8, 3)])
@pytest.mark.parametrize("rows", [1, 5, 40, 300, 16400])
def test_linear_strided(rows, pad, shift):
    K, N = 328, 200
    x, w = _x(rows, K, torch.bfloat16), _x(N, K, torch.float32, 5)
    buf = torch.full((shift + rows * (K + pad),), float("nan"), dtype=torch.bfloat16, device="cuda")
    v = buf[shift:].reshape(rows, K + pad)[:, :K]
    v.copy_(x)
    ob = torch.full((shift + rows * (N + pad),), 7.0, dtype=torch.bfloat16, device="cuda")
    o = ob[shift:].reshape(rows, N + pad)[:, :N]
    ops.fp8_linear(v, ops.fp8_quantize(w.cuda(), 128), out=o)
    some = slice(max(0, rows - 300), rows)
    r, b = ref.product(ref.values(*ref.quantize(x[some])), ref.values(*ref.quantize(w, 128), 128), torch.bfloat16)
    assert_within(o[some], r, b, torch.bfloat16)
    o.fill_(7.0)
    assert bool((ob == 7).all())


def test_linear_of_a_row_does_not_depend_on_the_others():
    """Of as many rows; the order of a sum may be another for other numbers of rows."""
    w = ops.fp8_quantize(_x(250, 1024).cuda(), 128)
    for rows in (4, 100, 700, 20000):
        x = _x(rows, 1024, torch.bfloat16).cuda()
        y = x.clone()
        y[1:] = float("nan")
        assert torch.equal(ops.fp8_linear(x, w)[0], ops.fp8_linear(y, w)[0])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,K,N", [(1, 64, 96), (130, 200, 72), (1111, 130, 257), (3000, 256, 128)])
def test_training_step(M, K, N, dtype):
    """The three products of a linear layer at the quantised values."""
    x, w, up = _x(M, K, dtype), _x(N, K, dtype, 1), _x(M, N, dtype, 2)
    (xq, xt), (wq, wt), (uq, ut) = (ops.fp8_quantize_both(t.cuda(), br) for t, br in ((x, 1), (w, 128), (up, 1)))
    held = lambda t, br=1: ref.values(*ref.quantize(t, br), br)
    for got, a, b, t in ((ops.fp8_matmul(xq, wq, dtype), held(x), held(w, 128), dtype),
                         (ops.fp8_matmul(uq, wt, dtype), held(up), held(w, 128).T, dtype),
                         (ops.fp8_matmul(ut, xt, torch.float32), held(up.T), held(x.T), torch.float32)):
        r, bound = ref.product(a, b, t)
        assert_within(got, r, bound, t)


def test_gradients_against_differences():
    """A product is linear in each factor: differences at values that need no rounding."""
    g = torch.Generator().manual_seed(2)
    x, w, up = (torch.randint(-8, 9, s, generator=g).double() for s in ((6, 40), (9, 40), (6, 9)))
    (xq, xt), (wq, wt), (uq, ut) = (ops.fp8_quantize_both(t.float().cuda(), br) for t, br in ((x, 1), (w, 128), (up, 1)))
    dx, dw = ops.fp8_matmul(uq, wt, torch.float32).cpu().double(), ops.fp8_matmul(ut, xt, torch.float32).cpu().double()
    f = lambda a, b: float(((a @ b.T) * up).sum())
    for i, k in itertools.product(range(6), range(0, 40, 7)):
        e = torch.zeros_like(x)
        e[i, k] = 1
        assert float(dx[i, k]) == (f(x + e, w) - f(x - e, w)) / 2
    for n, k in itertools.product(range(9), range(0, 40, 7)):
        e = torch.zeros_like(w)
        e[n, k] = 1
        assert float(dw[n, k]) == (f(x, w + e) - f(x, w - e)) / 2


def test_given_outputs_and_another_stream():
    x, w = _x(500, 600, torch.bfloat16), _x(200, 600)
    xc, wc = x.cuda(), w.cuda()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        q, t = ops.Fp8Matrix.empty(500, 600), ops.Fp8Matrix.empty(600, 500)
        assert ops.fp8_quantize_both(xc, out=q, out_t=t) == (q, t)
        m = ops.fp8_quantize(wc, 128, out=ops.Fp8Matrix.empty(200, 600, 128))
        out = torch.empty(500, 200, device="cuda")
        assert ops.fp8_matmul(q, m, out=out) is out
    s.synchronize()
    _check_matrix(q, x, 1)
    _check_matrix(t, x.T, 1)
    r, b = ref.product(ref.values(*ref.quantize(x)), ref.values(*ref.quantize(w, 128), 128))
    assert_within(out, r, b)


def test_replayed_graph():
    """A step of a layer, replayed with other inputs, with eager work between the replays."""
    M, K, N = 700, 512, 256
    x, w, up = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((M, K), (N, K), (M, N)))
    ws = bd.Workspace()

    def step():
        (xq, xt), (wq, wt), (uq, ut) = (ops.fp8_quantize_both(t, br) for t, br in ((x, 1), (w, 128), (up, 1)))
        return (ops.fp8_matmul(xq, wq, ws=ws), ops.fp8_matmul(uq, wt, ws=ws), ops.fp8_matmul(ut, xt, torch.float32, ws=ws),
                ops.fp8_linear(x[:3], wq, ws=ws), ops.fp8_linear(x, wq, ws=ws))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for k in range(4):
        for t, seed in ((x, 0), (w, 1), (up, 2)):
            t.copy_(_x(*t.shape, torch.bfloat16, seed + 10 * k))
        graph.replay()
        torch.cuda.synchronize()
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k


def test_scales_behind_the_last_block_stay():
    """A matrix of the caller's, whose rows of scales are in a wider buffer: four row blocks a word, and the rest."""
    rows, cols = 512 * 40 + 300, 128 * 40
    x = _x(300, 128).repeat(rows // 300 + 1, 40)[:rows].to(torch.bfloat16)
    codes = torch.zeros(cols, -(-rows // 16) * 16, device="cuda").to(torch.float8_e4m3fn)
    buf = torch.full((cols, 172), 9, dtype=torch.uint8, device="cuda")
    nb = -(-rows // 128)
    t = ops.Fp8Matrix(codes[:, :rows], buf.view(torch.float8_e8m0fnu)[:, 4:4 + nb])
    ops.fp8_quantize(x.cuda(), transposed=True, out=t)
    assert nb % 4 and bool((buf[:, :4] == 9).all()) and bool((buf[:, 4 + nb:] == 9).all())
    some = torch.arange(0, cols, 777)
    q, byte = ref.quantize(x.T[some])
    assert torch.equal(buf[:, 4:4 + nb].cpu()[some].long(), byte)
    assert torch.equal(codes[:, :rows].cpu()[some].float().double(), q)


def test_sizes_past_32_bits():
    """Codes, values and results at offsets of more than 2^32 bytes and 2^31 values."""
    M, K = 1 << 19, 8320
    x = torch.empty(M, K, dtype=torch.bfloat16, device="cuda")
    part = _x(512, K, torch.bfloat16).cuda()
    for i in range(0, M, 512):
        x[i:i + 512] = part
    q, t = ops.fp8_quantize_both(x)
    w = _x(40, K, seed=3)
    m = ops.fp8_quantize(w.cuda())
    last = slice(M - 200, M)
    held = ref.values(*ref.quantize(part.cpu()[-200:]))
    for out in (ops.fp8_matmul(q, m), ops.fp8_linear(x, m)):
        r, b = ref.product(held, ref.values(*ref.quantize(w)), torch.bfloat16)
        assert_within(out[last], r, b, torch.bfloat16)
    tq, tb = ref.quantize(part.cpu()[-128:, -30:].T)
    assert torch.equal(t.codes[-30:, -128:].cpu().float().double(), tq)
    assert torch.equal(t.scale[-30:, -1:].cpu().view(torch.uint8).long(), tb)
    few = ops.fp8_matmul(m, q, torch.float32)
    r, b = ref.product(ref.values(*ref.quantize(w)), held)
    assert_within(few[:, last], r, b)


def test_two_at_once():
    w = ops.fp8_quantize(_x(256, 4096).cuda(), 128)
    xs = [_x(n, 4096, torch.bfloat16, n).cuda() for n in (2, 40, 300)]
    want = [ops.fp8_linear(x, w) for x in xs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in xs], []
    for x, s in zip(xs, streams):
        with torch.cuda.stream(s):
            got.append(ops.fp8_linear(x, w))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_refusals():
    x = torch.zeros(8, 64, device="cuda")
    q, w = ops.fp8_quantize(x), ops.fp8_quantize(torch.zeros(9, 65, device="cuda"))
    z = lambda *s, **k: torch.zeros(*s, device="cuda", **k)
    codes, scale = z(8, 64).to(torch.float8_e4m3fn), z(8, 4, dtype=torch.uint8).view(torch.float8_e8m0fnu)[:, :1]
    for call in (lambda: ops.fp8_quantize(x.double()), lambda: ops.fp8_quantize(x, 64), lambda: ops.fp8_quantize(x[0]),
                 lambda: ops.fp8_quantize(x.T), lambda: ops.fp8_quantize(x, out=w), lambda: ops.fp8_quantize_both(x, 1, q, q),
                 lambda: ops.fp8_matmul(q, w), lambda: ops.fp8_matmul(q, q, torch.float64),
                 lambda: ops.fp8_matmul(q, q, accumulate=True), lambda: ops.fp8_matmul(q, q, out=z(8, 9)),
                 lambda: ops.fp8_matmul(q, q, out=z(8, 8).double()), lambda: ops.fp8_linear(x, w),
                 lambda: ops.fp8_linear(x, q, out=z(8, 8).half()), lambda: ops.Fp8Matrix(x, scale),
                 lambda: ops.Fp8Matrix(codes, scale, 2), lambda: ops.Fp8Matrix(codes, scale, 128),
                 lambda: ops.Fp8Matrix(codes, scale.view(torch.uint8)), lambda: ops.Fp8Matrix(codes, scale.cpu()),
                 lambda: ops.Fp8Matrix(codes, scale.contiguous()), lambda: ops.Fp8Matrix(codes[:, :63], scale.contiguous()),
                 lambda: ops.Fp8Matrix(codes[:, 1:], scale), lambda: ops.Fp8Matrix(codes.T, z(64, 4, dtype=torch.uint8).view(
                     torch.float8_e8m0fnu)[:, :1])):
        with pytest.raises(bd.ChgnetError) as e:
            call()
        assert e.value.code == bd.CHGNET_EINVAL
