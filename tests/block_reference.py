"""Plain 64-bit forms of the norms, the residual connection and dropout in include/chgnet_ops.h, and how far fp32 arithmetic
may be off them. Test infrastructure; shares no code with the library.

U = 2^-24 is half a last place of fp32. A sum over a row has at most D = 44 roundings one after another (16 in a thread, 6
over lanes, 15 over wavefronts, its factors), a sum over rows at most 64 + rows / 512. Counts are generous: they take worst
cases and do not use that errors have signs.
"""
import numpy as np
import torch

U = 2.0 ** -24
D = 44


def philox(c0, c1, c2, c3, k0, k1):
    """Philox4x32-10 of Salmon et al. on uint64 arrays holding 32 bits."""
    m = np.uint64(0xFFFFFFFF)
    c = [np.asarray(v, dtype=np.uint64) for v in (c0, c1, c2, c3)]
    k0, k1 = int(k0), int(k1)
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), q & m, (p >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), p & m]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c


def kept(rows, d, p, seed, n):
    """(mask [rows, d], factor of the kept values)."""
    n &= 2 ** 64 - 1
    g = np.arange((d + 7) // 8)[None].repeat(rows, 0)
    r = np.arange(rows)[:, None].repeat(g.shape[1], 1)
    w = philox(g, r, np.full_like(g, n & 0xFFFFFFFF), np.full_like(g, n >> 32), seed & 0xFFFFFFFF, seed >> 32)
    bits = np.stack([np.stack([x & np.uint64(0xFFFF), x >> np.uint64(16)], -1) for x in w], -2).reshape(rows, -1)[:, :d]
    cut = int(np.floor(float(np.float32(p)) * 65536 + 0.5))
    return torch.from_numpy(bits.astype(np.int64) >= cut), (65536 / (65536 - cut) if cut < 65536 else 0.0)


def dropout(x, p, seed, n):
    """The result bit for bit: one fp32 product with the factor rounded to fp32, one rounding to the type."""
    m, f = kept(*x.shape, p, seed, n)
    return torch.where(m, x.float() * float(np.float32(f)), torch.zeros(())).to(x.dtype)


def normed(x, kind, eps):
    """(n(x), r, bound of the error of n) in 64 bits."""
    if kind == "none":
        return x, None, torch.zeros_like(x)
    c = x - x.mean(1, keepdim=True) if kind == "layer" else x
    r = 1 / torch.sqrt((c * c).mean(1, keepdim=True) + eps)
    e = 30 * U * (c * r).abs()
    if kind == "layer":
        e = e + r * D * U * x.abs().mean(1, keepdim=True)
    return c * r, r, e


def _affine(n, e, w):
    y = n * w[0] + (w[1] if w.shape[0] == 2 else 0)
    return y, w[0].abs() * e + 3 * U * ((n * w[0]).abs() + (w[1].abs() if w.shape[0] == 2 else 0))


def norm(x, w, kind, eps):
    n, _, e = normed(x.double(), kind, eps)
    h, b = _affine(n, e, w.double())
    return h, b + 1e-37


def _norm_back(up, e_up, w, n, r, ex, kind):
    """Gradient of x through w n(x) from `up`, and its bound."""
    g, eg = up * w[0], e_up * w[0].abs() + 2 * U * (up * w[0]).abs()
    if kind == "none":
        return g, eg
    mean = lambda t: t.mean(1, keepdim=True)
    m = mean(g) if kind == "layer" else torch.zeros_like(r)
    s = mean((g * n).abs())
    dx = r * (g - m - n * mean(g * n))
    whole = g.abs() + (mean(g.abs()) if kind == "layer" else 0) + n.abs() * s
    err = eg + (mean(eg) if kind == "layer" else 0) + n.abs() * mean(eg * n.abs() + g.abs() * ex) + ex * s
    return dx, r * (err + 100 * U * whole)


def norm_grad(x, w, dh, kind, eps):
    """(dx, dw, their bounds) in 64 bits."""
    x, w, up = x.double(), w.double(), dh.double()
    n, r, ex = normed(x, kind, eps)
    dx, ed = _norm_back(up, torch.zeros_like(up), w, n, r, ex, kind)
    depth = (64 + x.shape[0] / 512) * U
    dw, ew = [(up * n).sum(0), up.sum(0)], [(up.abs() * ex + depth * (up * n).abs()).sum(0), depth * up.abs().sum(0)]
    k = w.shape[0]
    return dx, torch.stack(dw[:k]), ed + 1e-37, torch.stack(ew[:k]) + 1e-37


def residual(x, f, post, post_kind, gate, alpha, beta, mask, factor, eps):
    """(y, bound before its rounding) in 64 bits."""
    t, et = f.double(), torch.zeros(())
    if post is not None:
        n, _, ex = normed(t, post_kind, eps)
        t, et = _affine(n, ex, post.double())
    s, rel = 1.0, 0.0
    if gate is not None:
        g = gate.double()
        s, rel = torch.sigmoid(g), (2 * g.abs() + 8) * U
    zero = torch.zeros((), dtype=torch.float64)
    v = torch.where(mask, beta * factor * s * t, zero)
    ev = torch.where(mask, abs(beta) * factor * s * et + v.abs() * (rel + 8 * U), zero)
    y = alpha * x.double() + v
    return y, ev + 3 * U * ((alpha * x.double()).abs() + v.abs()) + 1e-37


def residual_grad(y, f, dy, dh, post, post_kind, gate, pre, pre_kind, alpha, beta, mask, factor, eps):
    """({name: gradient}, {name: bound}) in 64 bits from the stored y; None where there is none."""
    rows, d = y.shape
    depth = (64 + rows / 512) * U
    zero = torch.zeros((), dtype=torch.float64)
    up, eu = (torch.zeros(rows, d, dtype=torch.float64) if dy is None else dy.double()), torch.zeros(rows, d, dtype=torch.float64)
    out, bound = dict.fromkeys(("dx", "df", "dgate", "dpost", "dpre")), {}
    if pre is not None:
        dx, out["dpre"], ex, bound["dpre"] = norm_grad(y, pre, dh, pre_kind, eps)
        up, eu = up + dx, ex + 3 * U * (up.abs() + dx.abs())
    out["dx"], bound["dx"] = alpha * up, abs(alpha) * (eu + 2 * U * up.abs()) + 1e-37
    w = torch.ones(1, d, dtype=torch.float64) if post is None else post.double()
    n, r, ex = normed(f.double(), post_kind, eps)
    t, et = _affine(n, ex, w) if post is not None else (n, torch.zeros_like(n))
    du = torch.where(mask, beta * factor * up, zero)
    eu = torch.where(mask, abs(beta) * factor * eu + 3 * U * du.abs(), zero)
    s, es = 1.0, 0.0
    if gate is not None:
        g = gate.double()
        s = torch.sigmoid(g)
        rel = (2 * g.abs() + 8) * U
        es, ds = s * rel, s * (1 - s)
        tt = torch.where(mask, t, zero)
        dg = du * tt * ds
        eg = eu * tt.abs() * ds + du.abs() * et * ds + (du * tt).abs() * s * (rel + 4 * U) + 6 * U * dg.abs()
        if gate.shape[1] == 1 and d > 1:
            eg = eg.sum(1, keepdim=True) + D * U * dg.abs().sum(1, keepdim=True)
            dg = dg.sum(1, keepdim=True)
        out["dgate"], bound["dgate"] = dg, eg + 1e-37
    dt = du * s
    et = eu * s + du.abs() * es + 2 * U * dt.abs()
    if post is not None:
        nn = torch.where(mask, n, zero)
        dw = [(dt * nn).sum(0), dt.sum(0)]
        ew = [(et * nn.abs() + dt.abs() * ex + depth * (dt * nn).abs()).sum(0), (et + depth * dt.abs()).sum(0)]
        out["dpost"] = torch.stack(dw[:post.shape[0]])
        bound["dpost"] = torch.stack(ew[:post.shape[0]]) + 1e-37
    out["df"], b = _norm_back(dt, et, w, n, r, ex, post_kind)
    bound["df"] = b + 1e-37
    return out, bound
