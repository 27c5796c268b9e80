"""chgnet_gate_forward and chgnet_gate_backward against their definition in 64 bits (ops_reference.py): the checkpoint bit
for bit, phi, dz and the LayerNorm gradients within the bounds derived there; widths and rows around the kernels' lanes and
passes, strides, types, rows of one value, of NaN and infinities, many rows; streams and captured graphs."""
import math

import pytest
import torch

import ops_reference as ref
from paper_2412_20796_amd import binding as bd
from paper_2412_20796_amd import ops

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _inputs(rows, d, dtype, seed=0):
    g = torch.Generator().manual_seed(1000 * rows + 10 * d + seed)
    z = torch.randn(rows, 2 * d, generator=g) * torch.exp(torch.randn(rows, 1, generator=g)) + torch.randn(
        1, 2 * d, generator=g)
    ln = torch.randn(4, d, generator=g) * 0.3 + torch.tensor([[1.0], [0.0], [1.0], [0.0]])
    dphi = torch.randn(rows, d, generator=g) * torch.rand(rows, 1, generator=g)
    if rows > 2:
        dphi[1] = 0  # a row whose mask leaves nothing
    return z.to(dtype), ln, dphi.to(dtype)


def _check(z, ln, dphi, phi, kept, dz, dln, what=""):
    dtype = z.dtype
    q, step, _ = ref.checkpoint(z)
    assert torch.equal(kept.codes.cpu().double(), q), what
    assert torch.equal(kept.step.cpu().double(), step), what
    r, b = ref.gate(z, ln)
    ref.assert_within(phi, r, b, dtype, what + " phi")
    rz, rl, bz, bl = ref.gate_grad(q, step, ln, dphi)
    ref.assert_within(dz, rz, bz, dtype, what + " dz")
    ref.assert_within(dln, rl, bl, what=what + " dln")


def _run(z, ln, dphi, **kw):
    zc, lc, pc = z.cuda(), ln.cuda(), dphi.cuda()
    phi, kept = ops.gate_forward(zc, lc)
    dz, dln = ops.gate_backward(kept, lc, pc, **kw)
    return phi, kept, dz, dln


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [1, 2, 3, 4, 5, 15, 16, 17, 60, 63, 64, 65, 68, 100, 127, 128, 129, 132, 200, 256, 257, 260,
                               500, 512, 513, 600, 1000, 1023, 1024])
def test_widths(d, dtype):
    rows = 67
    z, ln, dphi = _inputs(rows, d, dtype)
    _check(z, ln, dphi, *_run(z, ln, dphi), what="d=%d %s" % (d, dtype))


@pytest.mark.parametrize("d", [64, 128, 250])
@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 15, 16, 17, 31, 32, 33, 63, 64, 65, 255, 257, 5000])
def test_rows(rows, d):
    z, ln, dphi = _inputs(rows, d, torch.float32)
    _check(z, ln, dphi, *_run(z, ln, dphi), what="rows=%d d=%d" % (rows, d))


@pytest.mark.parametrize("rows,d", [(70001, 64), (40003, 128), (20011, 333)])
def test_more_rows_than_one_pass(rows, d):
    z, ln, dphi = _inputs(rows, d, torch.float32)
    _check(z, ln, dphi, *_run(z, ln, dphi), what="rows=%d" % rows)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,pad,shift", [(64, 4, 0), (64, 3, 0), (64, 0, 1), (128, 8, 4), (128, 1, 2), (50, 6, 2), (96, 32, 0)])
def test_strides_and_alignment(d, pad, shift, dtype):
    """Rows inside wider buffers, at offsets that do and do not allow vector loads; what lies between the rows stays."""
    rows = 37
    z, ln, dphi = _inputs(rows, d, dtype)

    def view(cols, fill=None):
        buf = torch.full((shift + rows * (cols + pad),), 7.0, dtype=dtype, device="cuda")
        v = buf[shift:].reshape(rows, cols + pad)[:, :cols]
        if fill is not None:
            v.copy_(fill)
        return buf, v

    _, zv = view(2 * d, z)
    _, pv = view(d, dphi)
    bphi, phi = view(d)
    bdz, dz = view(2 * d)
    lbuf = torch.zeros(4 * d + 1, device="cuda")  # as in the flat parameter vector: at any float
    lv = lbuf[1:].reshape(4, d)
    lv.copy_(ln)
    codes = torch.empty(rows * 2 * d + 1, dtype=torch.uint8, device="cuda")[1:].reshape(rows, 2 * d)
    kept = ops.GateCheckpoint(codes if pad == 3 else ops.GateCheckpoint.empty(rows, d).codes,
                              torch.empty(rows, 2, device="cuda"))
    ops.gate_forward(zv, lv, phi=phi, kept=kept)
    dz, dln = ops.gate_backward(kept, lv, pv, dz=dz)
    _check(z, ln, dphi, phi, kept, dz, dln, "pad=%d shift=%d" % (pad, shift))
    for buf, cols in ((bphi, d), (bdz, 2 * d)):
        assert bool((buf[:shift] == 7).all())
        assert bool((buf[shift:].reshape(rows, cols + pad)[:, cols:] == 7).all())


@pytest.mark.parametrize("d", [64, 128, 90])
def test_rows_after_the_last_stay(d):
    z, ln, dphi = _inputs(21, d, torch.float32)
    phi, dz = torch.full((24, d), 5.0, device="cuda"), torch.full((24, 2 * d), 5.0, device="cuda")
    codes, step = torch.full((24, 2 * d), 9, dtype=torch.uint8, device="cuda"), torch.full((24, 2), 5.0, device="cuda")
    kept = ops.GateCheckpoint(codes[:21], step[:21])
    ops.gate_forward(z.cuda(), ln.cuda(), phi=phi[:21], kept=kept)
    _, dln = ops.gate_backward(kept, ln.cuda(), dphi.cuda(), dz=dz[:21])
    _check(z, ln, dphi, phi[:21], kept, dz[:21], dln)
    for t, v in ((phi, 5), (dz, 5), (codes, 9), (step, 5)):
        assert bool((t[21:] == v).all())


def test_inference_has_the_same_bits_and_none_of_the_checkpoint():
    for rows, d, dtype in ((1, 64, torch.float32), (77, 128, torch.bfloat16), (77, 51, torch.float32)):
        z, ln, _ = _inputs(rows, d, dtype)
        a = ops.gate_forward(z.cuda(), ln.cuda(), save=False)
        b, _ = ops.gate_forward(z.cuda(), ln.cuda())
        assert torch.equal(a, b)


def test_gradients_against_differences():
    """dz of the definition at the checkpoint's values, by central differences in 64 bits of the phi-weighted sum."""
    rows, d = 3, 12
    z, ln, dphi = _inputs(rows, d, torch.float32, seed=5)
    _, kept, dz, dln = _run(z, ln, dphi)
    x = kept.codes.cpu().double() * kept.step.cpu().double().repeat_interleave(d, 1)
    f = lambda x, p: (ref.gate(x, p)[0] * dphi.double()).sum()
    h = 1e-6
    for i in range(rows):
        for k in range(0, 2 * d, 5):
            e = torch.zeros_like(x)
            e[i, k] = h
            num = float(f(x + e, ln.double()) - f(x - e, ln.double())) / (2 * h)
            # differences of values near 1 in 64 bits: 1e-16 / h, and h^2 times a third derivative of a few tens
            assert abs(float(dz[i, k]) - num) <= 2e-6 + 1e-5 * abs(num)
    for a in range(4):
        e = torch.zeros(4, d, dtype=torch.float64)
        e[a, 3] = h
        num = float(f(x, ln.double() + e) - f(x, ln.double() - e)) / (2 * h)
        assert abs(float(dln[a, 3]) - num) <= 2e-6 + 1e-5 * abs(num)


def test_rows_of_one_value():
    """No range: the least step, codes of 0, xhat 0, and a gradient of r = 1 / sqrt(eps) times the centred one."""
    for d in (64, 100, 333):
        z, ln, dphi = _inputs(9, d, torch.float32)
        z[2] = 3.25
        z[4, :d] = 0.0
        z[5, d:] = -1e30
        out = _run(z, ln, dphi)
        _check(z, ln, dphi, *out, what="d=%d" % d)
        assert float(out[1].step[2, 0]) == 2.0 ** -100 and int(out[1].codes[2].sum()) == 0


def test_far_from_zero():
    """Halves a thousand deviations from zero: the codes count from the least value, so the step stays the range's."""
    z, ln, dphi = _inputs(40, 128, torch.float32)
    z = z + 1000 * z.std(1, keepdim=True)
    _check(z, ln, dphi, *_run(z, ln, dphi))


def test_large_and_small_values():
    z, ln, dphi = _inputs(40, 64, torch.float32)
    for scale in (1e-38, 1e-20, 1e10):
        x = z * scale
        phi, kept, dz, dln = _run(x, ln, dphi)
        q, step, _ = ref.checkpoint(x)
        assert torch.equal(kept.codes.cpu().double(), q) and torch.equal(kept.step.cpu().double(), step)
        rz, _, bz, _ = ref.gate_grad(q, step, ln, dphi)
        # r U of the row's size: the bound's r is that of the values
        ref.assert_within(dz, rz, bz, what="scale %g" % scale)


@pytest.mark.parametrize("d", [64, 70, 600])
@pytest.mark.parametrize("size", [1e21, 1e30])
def test_variance_past_the_range(size, d):
    """A core whose variance is infinite in fp32 counts as all at its mean, and no gradient passes it."""
    rows = 37
    z, ln, dphi = _inputs(rows, d, torch.float32)
    z[:, :d] *= size
    mid = z.clone()
    mid[:, :d] = 0
    phi, kept, dz, dln = _run(z, ln, dphi)
    q, step, _ = ref.checkpoint(z)
    assert torch.equal(kept.codes.cpu().double(), q) and torch.equal(kept.step.cpu().double(), step)
    r, b = ref.gate(mid, ln)
    ref.assert_within(phi, r, b)
    q[:, :d] = 0
    rz, rl, bz, bl = ref.gate_grad(q, step, ln, dphi)
    assert (dz[:, :d] == 0).all() and (dln[0] == 0).all()
    ref.assert_within(dz[:, d:], rz[:, d:], bz[:, d:])
    ref.assert_within(dln, rl, bl)


@pytest.mark.parametrize("d", [64, 128, 70])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_values_that_are_not_finite(value, d):
    """They stay in their row: phi and dz of the others are as without them, the LayerNorm gradients are NaN."""
    z, ln, dphi = _inputs(33, d, torch.float32)
    clean = _run(z, ln, dphi)
    z[7, 3] = value
    z[20, d + d // 2] = value
    phi, kept, dz, dln = _run(z, ln, dphi)
    rows = torch.ones(33, dtype=torch.bool)
    rows[[7, 20]] = False
    assert torch.equal(phi.cpu()[rows], clean[0].cpu()[rows]) and torch.equal(dz.cpu()[rows], clean[2].cpu()[rows])
    assert not bool(torch.isfinite(phi.cpu()[~rows]).any()) and bool(torch.isnan(dz.cpu()[7, :d]).all())
    assert bool(torch.isnan(dz.cpu()[20, d:]).all()) and bool(torch.isnan(dln).any())
    assert not bool(torch.isfinite(kept.step.cpu()[7, 0])) and not bool(torch.isfinite(kept.step.cpu()[20, 1]))


@pytest.mark.parametrize("rows", [0, 5, 3000])
def test_accumulate(rows):
    d = 64
    z, ln, dphi = _inputs(rows, d, torch.float32)
    lc = ln.cuda()
    _, kept = ops.gate_forward(z.cuda(), lc)
    once = ops.gate_backward(kept, lc, dphi.cuda())[1]
    if rows == 0:
        assert not bool(once.any())
    base = torch.randn(4, d, device="cuda")
    got = ops.gate_backward(kept, lc, dphi.cuda(), dln=base.clone(), accumulate=True)[1]
    assert torch.equal(got, base + once)


def test_bitwise_reproducible():
    z, ln, dphi = _inputs(30001, 128, torch.float32)
    a, b = _run(z, ln, dphi), _run(z, ln, dphi)
    assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2]) and torch.equal(a[3], b[3])


def test_offsets_past_32_bits():
    """9,000,001 rows of 256 values: the last rows lie past 2^31 values (and their codes past 2^31 bytes)."""
    rows, d = 9_000_001, 128
    z, ln, dphi = _inputs(4099, d, torch.float32)
    zc, lc, pc = z.cuda(), ln.cuda(), dphi.cuda()
    phi, kept, dz, _ = _run(z, ln, dphi)
    k = math.ceil(rows / 4099)
    big = zc.repeat(k, 1)[:rows]
    bphi, bkept = ops.gate_forward(big, lc)
    del big
    bdz, _ = ops.gate_backward(bkept, lc, pc.repeat(k, 1)[:rows])
    for lo in (0, 4099 * 1000, 4099 * (k - 2)):
        for x, y in ((bphi, phi), (bkept.codes, kept.codes), (bkept.step, kept.step), (bdz, dz)):
            assert torch.equal(x[lo:lo + 4099], y), lo


def test_other_stream():
    z, ln, dphi = _inputs(2000, 64, torch.float32)
    s = torch.cuda.Stream()
    zc, lc, pc = z.cuda(), ln.cuda(), dphi.cuda()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        phi, kept = ops.gate_forward(zc, lc)
        dz, dln = ops.gate_backward(kept, lc, pc)
    torch.cuda.current_stream().wait_stream(s)
    _check(z, ln, dphi, phi, kept, dz, dln)


def test_captured_and_replayed():
    """Two graphs with workspaces of their own, replayed in turn with new inputs and eager calls between them."""
    shapes = [(1300, 64), (700, 128)]
    made = []
    s = torch.cuda.Stream()
    for rows, d in shapes:
        x = dict(z=torch.empty(rows, 2 * d, device="cuda"), ln=torch.empty(4, d, device="cuda"),
                 dphi=torch.empty(rows, d, device="cuda"), ws=bd.Workspace())
        fill = lambda x, seed: [x[k].copy_(t) for k, t in zip(("z", "ln", "dphi"), _inputs(*shapes[len(made)], torch.float32, seed))]
        fill(x, 0)
        with torch.cuda.stream(s):
            x["phi"], kept = ops.gate_forward(x["z"], x["ln"])
            ops.gate_backward(kept, x["ln"], x["dphi"], ws=x["ws"])
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            x["phi"], x["kept"] = ops.gate_forward(x["z"], x["ln"])
            x["dz"], x["dln"] = ops.gate_backward(x["kept"], x["ln"], x["dphi"], ws=x["ws"])
        x["graph"] = g
        made.append(x)
    for turn in range(3):
        for k, x in enumerate(made):
            z, ln, dphi = _inputs(*shapes[k], torch.float32, seed=turn + 1)
            for name, t in (("z", z), ("ln", ln), ("dphi", dphi)):
                x[name].copy_(t)
            x["graph"].replay()
        torch.cuda.synchronize()
        for k, x in enumerate(made):
            z, ln, dphi = _inputs(*shapes[k], torch.float32, seed=turn + 1)
            eager = _run(z, ln, dphi)
            assert torch.equal(x["phi"], eager[0]) and torch.equal(x["dz"], eager[2]) and torch.equal(x["dln"], eager[3])
            assert torch.equal(x["kept"].codes, eager[1].codes)


def test_what_the_binding_refuses():
    dev = dict(device="cuda")
    z, ln, up = torch.zeros(6, 16, **dev), torch.zeros(4, 8, **dev), torch.zeros(6, 8, **dev)
    _, kept = ops.gate_forward(z, ln)
    for call in (lambda: ops.gate_forward(z[:, :15], ln), lambda: ops.gate_forward(z.double(), ln),
                 lambda: ops.gate_forward(z[0], ln), lambda: ops.gate_forward(z.t().contiguous().t(), ln),
                 lambda: ops.gate_forward(z[:1].expand(6, 16), ln), lambda: ops.gate_forward(z, ln[:, :7]),
                 lambda: ops.gate_forward(z, ln.double()), lambda: ops.gate_forward(z, ln.cpu()),
                 lambda: ops.gate_forward(z, ln, phi=torch.zeros(5, 8, **dev)),
                 lambda: ops.gate_forward(z, ln, save=False, kept=kept),
                 lambda: ops.gate_forward(z[:5], ln, kept=kept),
                 lambda: ops.gate_forward(z, ln, kept=ops.GateCheckpoint(kept.codes[:, :15], kept.step)),
                 lambda: ops.gate_forward(torch.zeros(2, 2050, **dev), torch.zeros(4, 1025, **dev)),
                 lambda: ops.gate_backward(kept, ln, up[:5]), lambda: ops.gate_backward(kept, ln, up.double()),
                 lambda: ops.gate_backward(kept, ln, up[:1].expand(6, 8)),
                 lambda: ops.gate_backward(kept, ln, up, dz=torch.zeros(6, 16, **dev, dtype=torch.float16)),
                 lambda: ops.gate_backward(kept, ln, up, accumulate=True),
                 lambda: ops.gate_backward(kept, ln, up, dln=torch.zeros(8, 4, **dev)),
                 lambda: ops.gate_backward(kept, ln, up, ws=bd.Workspace("cpu")),
                 lambda: ops.gate_backward(ops.GateCheckpoint(kept.codes.int(), kept.step), ln, up)):
        with pytest.raises(bd.ChgnetError) as e:
            call()
        assert e.value.code == bd.CHGNET_EINVAL


def test_checkpoint_of_given_tensors_and_of_one_allocation_agree():
    rows, d = 50, 64
    z, ln, dphi = (t.cuda() for t in _inputs(rows, d, torch.float32))
    two = ops.GateCheckpoint(torch.empty(rows, 2 * d, dtype=torch.uint8, device="cuda"), torch.empty(rows, 2, device="cuda"))
    _, one = ops.gate_forward(z, ln)
    ops.gate_forward(z, ln, kept=two)
    assert torch.equal(one.codes, two.codes) and torch.equal(one.step, two.step)
    assert one.nbytes == two.nbytes == rows * (2 * d + 8)
    a, b = ops.gate_backward(one, ln, dphi), ops.gate_backward(two, ln, dphi)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
