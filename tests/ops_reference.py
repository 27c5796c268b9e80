"""Plain 64-bit forms of the operators in include/chgnet_ops.h, and how far fp32
arithmetic may be off them. Test infrastructure; shares no code with the library.

U = 2^-24 is half a last place of fp32. Counts of roundings below are generous
(they take worst cases and do not use that errors have signs).
"""
import numpy as np
import torch

U = 2.0 ** -24
LN_EPS = 1e-5
LEAST_STEP = 2.0 ** -100


def half_step(dtype):
    """Largest relative error of one rounding to dtype, and half its least subnormal."""
    if dtype == torch.float32:
        return 0.0, 0.0
    return torch.finfo(dtype).eps / 2, {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}[dtype]


def checkpoint(z):
    """Codes [rows, 2d] and step [rows, 2] of z [rows, 2d] (any float values of at most 24 bits, CPU): each operation
    is formed in 64 bits and rounded once to 32 (no double rounding: 53 >= 2 * 24 + 2)."""
    x = z.double().reshape(z.shape[0], 2, -1)
    f32 = lambda t: t.float().double()
    lo, hi = x.amin(2, keepdim=True), x.amax(2, keepdim=True)
    third = float(np.float32(1) / np.float32(255))
    step = f32(f32(hi - lo) * third)
    step = torch.where(step < LEAST_STEP, torch.full_like(step, LEAST_STEP), step)
    q = torch.round(f32(x - lo) * f32(1 / step))
    return q.reshape(z.shape), step.reshape(-1, 2), lo


def _ln(x):
    m = x.mean(-1, keepdim=True)
    r = 1 / torch.sqrt(((x - m) ** 2).mean(-1, keepdim=True) + LN_EPS)
    return (x - m) * r, r


def gate(z, ln):
    """phi of z [rows, 2d] in 64 bits, and a bound of fp32's error.

    xhat: a mean of d values is off by at most 24 roundings (16 in a lane, 6 over lanes, the division) of the largest |x|;
    the deviation by half of as many, and 3 for the reciprocal root. So |error of xhat| <= r 26 U max|x| + 16 U |xhat|.
    y = g xhat + b adds 2 roundings. A sigmoid has a relative error of at most (2 |y| + 8) U (argument, exponential,
    sum and reciprocal at 1 ulp); |d SiLU| <= 1.1, |d sigmoid| <= 1/4."""
    x, g = z.double().reshape(z.shape[0], 2, -1), ln.double()
    xh, r = _ln(x)
    yc, yg = g[0] * xh[:, 0] + g[1], g[2] * xh[:, 1] + g[3]
    sc, sg = torch.sigmoid(yc), torch.sigmoid(yg)
    phi = yc * sc * sg
    ex = r * 26 * U * x.abs().amax(2, keepdim=True) + 16 * U * xh.abs()
    ec = g[0].abs() * ex[:, 0] + 2 * U * ((g[0] * xh[:, 0]).abs() + g[1].abs())
    eg = g[2].abs() * ex[:, 1] + 2 * U * ((g[2] * xh[:, 1]).abs() + g[3].abs())
    bound = 1.1 * ec + 0.25 * (yc * sc).abs() * eg + phi.abs() * (2 * yc.abs() + 2 * yg.abs() + 20) * U
    return phi, 1.01 * bound + 1e-37


def gate_grad(q, step, ln, dphi):
    """(dz, dln) in 64 bits at the values of the checkpoint, by autograd of the definition, and bounds of fp32's errors.

    The codes' sums are exact, so xhat is off by at most ex = 18 U |xhat| + 2 U max|xhat| (scale, deviation and its
    reciprocal root, the mean's rounding), and y by ey = |g| ex + 2 U (|g xhat| + |b|). The derivatives' own factors carry
    w = (2 |y_c| + 2 |y_g| + 30) U; the derivative of SiLU changes by at most 1/2, SiLU by 1.1, the sigmoid by 1/4 and its
    derivative by 0.1 times an error of y. dz = r (dy - mean dy - xhat mean(dy xhat)): the errors of dy, of the two means (24
    roundings each) and of xhat in both of its places, and 24 U of the whole for r, products and differences."""
    g = ln.double().clone().requires_grad_(True)
    x = (q.double().reshape(q.shape[0], 2, -1) * step.double()[:, :, None]).requires_grad_(True)
    xh, r = _ln(x)
    yc, yg = g[0] * xh[:, 0] + g[1], g[2] * xh[:, 1] + g[3]
    phi = yc * torch.sigmoid(yc) * torch.sigmoid(yg)
    dz, dln = torch.autograd.grad(phi, [x, g], dphi.double())
    xh, r, yc, yg, g, up = xh.detach(), r.detach(), yc.detach(), yg.detach(), g.detach(), dphi.double().abs()
    ex = 18 * U * xh.abs() + 2 * U * xh.abs().amax(2, keepdim=True)
    ga = torch.stack([g[0], g[2]]).abs()
    ey = ga * ex + 2 * U * (ga * xh.abs() + torch.stack([g[1], g[3]]).abs())
    w = (2 * yc.abs() + 2 * yg.abs() + 30) * U
    sc, sg = torch.sigmoid(yc), torch.sigmoid(yg)
    silu, dsilu = (yc * sc).abs(), (sc * (1 + yc * (1 - sc))).abs()
    # |1 + y (1 - s)| cancels near y = -1.28: its roundings are of 1 + |y|
    gy = torch.stack([up * sg * dsilu, up * silu * sg * (1 - sg)], 1)
    egy = torch.stack([up * (0.5 * ey[:, 0] * sg + dsilu * 0.25 * ey[:, 1] + sg * sc * (1 + yc.abs()) * w),
                       up * (1.1 * ey[:, 0] * 0.25 + silu * 0.1 * ey[:, 1] + silu * w)], 1)
    dy, edy = ga * gy, ga * egy
    mean = lambda t: t.mean(2, keepdim=True)
    s2 = mean(dy * xh.abs())
    whole = dy + mean(dy) + xh.abs() * s2
    bz = r * (edy + mean(edy) + xh.abs() * mean(edy * xh.abs()) + xh.abs() * mean(dy * ex) + ex * s2
              + 24 * U * (mean(dy) + xh.abs() * s2) + 24 * U * whole)
    # sums over rows: each term's error, and at most 64 roundings in a lane, a block and the join
    depth = 64 + q.shape[0] / 4096
    bg, bb = egy * xh.abs() + gy * ex + depth * U * gy * xh.abs(), egy + depth * U * gy
    bl = torch.stack([bg.sum(0), bb.sum(0)], 1).reshape(4, -1)
    return dz.reshape(q.shape), dln, 1.01 * bz.reshape(q.shape) + 1e-37, 1.01 * bl + 1e-37


def table_rows(tok, first, vocab):
    r = tok.long() - first
    return torch.where((r < 0) | (r >= vocab), torch.full_like(r, vocab), r)


def embed(table, tok, scale, first):
    """The lookup as it has to be, bit for bit: one fp32 product, one rounding to the table's type."""
    r = table_rows(tok, first, table.shape[0])
    W = torch.cat([table.float() * scale, torch.zeros(1, table.shape[1])]).to(table.dtype)
    return W[r]


def embed_grad(tok, dout, vocab, scale, first):
    """The sums in 64 bits, and a bound: at most 300 + m / 4096 roundings of a sum of m rows (256 of a chunk, its parts
    and their join), one of the product and one of the addition to what was there."""
    r = table_rows(tok, first, vocab)
    x = dout.double()
    s = torch.zeros(vocab + 1, x.shape[1], dtype=torch.float64).index_add_(0, r, x)[:vocab]
    a = torch.zeros(vocab + 1, x.shape[1], dtype=torch.float64).index_add_(0, r, x.abs())[:vocab]
    m = torch.bincount(r, minlength=vocab + 1)[:vocab, None].double()
    return scale * s, abs(scale) * a * U * (torch.minimum(m, 300 + m / 4096) + 2)


def assert_within(got, ref, bound, dtype=torch.float32, what=""):
    """|got - ref| <= bound, plus one rounding to dtype."""
    got, ref = got.detach().cpu().double(), ref.detach().double()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    rel, least = half_step(dtype)
    err, most = (got - ref).abs(), bound + rel * (ref.abs() + bound) + least
    bad = ~(err <= most)
    if bad.any():
        k = int((err / most).nan_to_num(nan=float("inf")).argmax())
        raise AssertionError("%s: %d of %d off; worst at %d: got %.9g, ref %.9g, bound %.3g" % (
            what, int(bad.sum()), bad.numel(), k, got.reshape(-1)[k], ref.reshape(-1)[k], most.reshape(-1)[k]))
