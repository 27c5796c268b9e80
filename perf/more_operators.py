"""What surrounds a block of a residual network: its norms, gate, residual scale and dropout, and its linear layers in 8 bits.

Residual connection (x the stream, f the block's output, g its gate's pre-activations, all of d columns or g of one):
    t = w_p n(f) + b_p,  y = alpha x + beta Drop(sigmoid(g) t),  h = w n(y) + b
with n the RMS norm or the LayerNorm, each part but x and f optional; h is the next block's input and takes y as it is stored.
Training returns the gradients of all of them for given dy and dh. A norm alone is h.

Dropout: out = x / (1 - p) where a counter-based generator (Philox4x32-10 of the seed, the call's number, the row and
the group of eight columns; 16 bits a value) says so, else 0; p counts in steps of 2^-16. The same call is its gradient.

Linear layers: both factors as e4m3 codes with a power of two for each block of 128 along the contraction (weights: 128 x 128),
the least one with the block's largest magnitude within 448 (at least 2^-126). Inference quantises x and has the weight quantised;
training quantises x, the upstream gradient and the weight, each also along its rows, and forms the output and both gradients.

Sizes are those of the crystals of this repository's workloads (edges and angles of one 8-atom cell up to 128 crystals of width
128; four features of a width to two halves of a gate), and generic ones: one token, wide rows, odd sizes, 16-bit types.
"""
import math

import torch

own = False

EPS = 1e-5
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
# work of the largest listed cases: values of a residual connection, operations and values of a linear layer
MOST_VALUES = 16384 * 8192
MOST_PRODUCT = 16384 * 4096 * 16384


def listed():
    res = dict(pre="rms", post="rms", gate="none", alpha=1.0, beta=1.0, p=0.0)
    return [
        # the LayerNorm before a block, forward and backward: a layer's 397,934 angles of 128 crystals at width 128
        dict(name="norm_train_wide128", kind="norm_train", rows=397934, d=128, dtype="fp32", pre="layer"),
        # one new token between two blocks, where only latency counts
        dict(name="residual_infer_token", kind="residual_infer", rows=1, d=4096, dtype="bf16", **res),
        # training step of 40 crystals: a layer's 85,274 edges, gated feature by feature, with dropout
        dict(name="residual_train_tri40", kind="residual_train", rows=85274, d=64, dtype="fp32",
             **{**res, "pre": "layer", "post": "layer", "gate": "all", "p": 0.1}),
        # rows of odd width in 16 bits, one gate a row, a learned scale in place of the norm after, a scaled branch
        dict(name="residual_train_odd", kind="residual_train", rows=20011, d=333, dtype="bf16",
             **{**res, "post": "none", "gate": "row", "beta": 0.22}),
        # 16,384 tokens of a wide network with everything, the largest
        dict(name="residual_train_8k", kind="residual_train", rows=16384, d=8192, dtype="bf16",
             **{**res, "gate": "all", "p": 0.1, "alpha": 1.25}),
        # dropout of the 920 edges of one 8-atom cell, where only latency counts
        dict(name="dropout_cell8", kind="dropout", rows=920, d=64, dtype="fp32", p=0.1),
        # dropout of 16,384 tokens of a wide network
        dict(name="dropout_8k", kind="dropout", rows=16384, d=8192, dtype="bf16", p=0.1),
        # a linear layer at one new token
        dict(name="linear_infer_token", kind="linear_infer", rows=1, k=4096, n=4096, dtype="bf16"),
        # inference of 128 crystals at width 128: a layer's 397,934 angles, four features to the halves of a gate
        dict(name="linear_infer_wide128", kind="linear_infer", rows=397934, k=512, n=256, dtype="bf16"),
        # the same layer in a training step
        dict(name="linear_train_wide128", kind="linear_train", rows=397934, k=512, n=256, dtype="bf16"),
        # odd sizes in fp32
        dict(name="linear_train_odd", kind="linear_train", rows=1111, k=777, n=1003, dtype="fp32"),
        # training step of a wide layer, 16,384 tokens, the largest
        dict(name="linear_train_4k", kind="linear_train", rows=16384, k=4096, n=16384, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["norm_infer", "norm_train", "residual_infer", "residual_train", "residual_train", "dropout",
                       "linear_infer", "linear_infer", "linear_train", "linear_train"])
    dtype = rng.choice(["fp32", "bf16", "bf16", "fp16"])
    if kind.startswith("linear"):
        k, n = (rng.choice([128, 256, 512, 1024, 4096, 8192, _log(rng, 16, 16384)]) for _ in "kn")
        return dict(kind=kind, rows=_log(rng, 1, min(397934, MOST_PRODUCT // (k * n), 2 * MOST_VALUES // max(k, n))), k=k, n=n,
                    dtype=dtype)
    d = rng.choice([64, 128, 256, 1024, 4096, 8192, _log(rng, 16, 16384)])
    c = dict(kind=kind, rows=_log(rng, 1, min(397934, MOST_VALUES // d)), d=d, dtype=dtype)
    if kind == "dropout":
        return dict(c, p=rng.choice([0.1, 0.5, rng.random()]))
    c["pre"] = rng.choice(["rms", "layer"])
    if kind.startswith("norm"):
        return c
    return dict(c, pre=rng.choice([c["pre"], c["pre"], "no"]), post=rng.choice(["rms", "layer", "none", "no"]),
                gate=rng.choice(["none", "row", "all"]), alpha=rng.choice([1.0, 1.0, 1.25]), beta=rng.choice([1.0, 0.22]),
                p=rng.choice([0.0, 0.1]) if kind.endswith("train") else 0.0)


def prepare(case, seed):
    c = case
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    t = TYPES[c["dtype"]]
    randn = lambda *s: torch.randn(*s, device=dev, generator=g)
    s = {"case": dict(c), "seed": int(seed) * 0x9E3779B97F4A7C15 % 2 ** 63, "call": 7 + int(seed) % 1000}
    if c["kind"].startswith("linear"):
        M, K, N = c["rows"], c["k"], c["n"]
        # features with a few loud columns and rows of their own scale
        s["x"] = (randn(M, K) * torch.exp(0.5 * randn(1, K)) * torch.exp(0.3 * randn(M, 1))).to(t)
        w = (randn(N, K) / K ** 0.5).to(t)
        if c["kind"] == "linear_train":
            s["w"], s["dy"] = w, (1e-3 * randn(M, N) * torch.exp(randn(M, 1))).to(t)
            return s
        # the weight as the program keeps it: codes whose rows end on 16 bytes (zeros behind the last column), the exponents'
        # rows on 4
        codes, e = _quantized(w.float(), 128)
        held = torch.zeros(N, -(-K // 16) * 16, device=dev)
        held[:, :K] = codes
        exps = torch.zeros(e.shape[0], -(-e.shape[1] // 4) * 4, dtype=torch.uint8, device=dev)
        exps[:, :e.shape[1]] = (e + 127).to(torch.uint8)
        s["codes"], s["scale"] = held.to(torch.float8_e4m3fn)[:, :K], exps.view(torch.float8_e8m0fnu)[:, :e.shape[1]]
        return s
    R, d = c["rows"], c["d"]
    s["x"] = (randn(R, d) * torch.exp(0.5 * randn(1, d))).to(t)
    if c["kind"] == "dropout":
        s["up"] = (1e-2 * randn(R, d)).to(t)
        return s
    norm = lambda kind: None if kind == "no" else torch.stack(
        [1 + 0.1 * randn(d), 0.1 * randn(d)] if kind == "layer" else [1 + 0.1 * randn(d)])
    s["pre"] = norm(c["pre"])
    if c["kind"].endswith("train") and c["pre"] != "no":
        s["dh"] = (1e-2 * randn(R, d)).to(t)
    if c["kind"].startswith("residual"):
        s["f"], s["post"] = (3 * randn(R, d) + 0.5 * randn(1, d)).to(t), norm(c["post"])
        s["g"] = None if c["gate"] == "none" else randn(R, d if c["gate"] == "all" else 1).to(t)
        if c["kind"].endswith("train"):
            s["dy"] = (1e-2 * randn(R, d)).to(t)
    return s


# --- plain forms -----------------------------------------------------------------------------------------------------------

def _kept(rows, d, p, seed, call, dev):
    """Whether dropout keeps a value [rows, d], and the factor of those it keeps."""
    cut = math.floor(p * 65536 + 0.5)
    M = 0xFFFFFFFF
    n = -(-d // 8)
    c0 = torch.arange(n, device=dev).repeat(rows, 1)
    c1 = torch.arange(rows, device=dev)[:, None].repeat(1, n)
    c2, c3 = torch.full_like(c0, call & M), torch.full_like(c0, call >> 32 & M)
    k0, k1 = seed & M, seed >> 32 & M
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # 64 bits, of which the upper ones may be the sign
        c0, c1, c2, c3 = (b >> 32 & M) ^ c1 ^ k0, b & M, (a >> 32 & M) ^ c3 ^ k1, a & M
        k0, k1 = (k0 + 0x9E3779B9) & M, (k1 + 0xBB67AE85) & M
    words = torch.stack([c0, c1, c2, c3], 2)
    bits = torch.stack([words & 0xFFFF, words >> 16], 3).reshape(rows, 8 * n)[:, :d]
    return bits >= cut, (65536.0 / (65536 - cut) if cut < 65536 else 0.0)


def _norm(x, w, kind):
    """w n(x) + b, n(x), and 1 / deviation (None without a norm)."""
    if kind == "no":
        return x, x, None
    n, r = x, None
    if kind != "none":
        if kind == "layer":
            x = x - x.mean(1, keepdim=True)
        r = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
        n = x * r
    return n * w[0] + (w[1] if w.shape[0] == 2 else 0), n, r


def _norm_grad(up, w, n, r, kind):
    """Gradients of x and of w."""
    if kind == "no":
        return up, None
    dw = torch.stack([(up * n).sum(0), up.sum(0)][:w.shape[0]])
    dn = up * w[0]
    if kind == "none":
        return dn, dw
    dx = dn - n * (dn * n).mean(1, keepdim=True)
    return r * (dx - dn.mean(1, keepdim=True) if kind == "layer" else dx), dw


def _power(e):
    """2^e for whole -126 <= e <= 127, from its bits: torch.ldexp forms it with pow, which may be off in its last place."""
    return (e + 127 << 23).to(torch.int32).view(torch.float32)


def _quantized(x, block_rows):
    """Codes of x [rows, columns] (fp32 holding e4m3 values) and the exponents of its blocks."""
    R, C = x.shape
    nb, nr = -(-C // 128), -(-R // block_rows)
    big = torch.nn.functional.pad(x.abs(), (0, 128 * nb - C, 0, block_rows * nr - R))
    big = big.reshape(nr, block_rows, nb, 128).amax((1, 3))
    m, e = torch.frexp(big)
    e = torch.where(big > 0, e - 9 + (m > 0.875).int(), -126).clamp(min=-126)
    inv = _power(-e).repeat_interleave(block_rows, 0)[:R].repeat_interleave(128, 1)[:, :C]
    return (x * inv).to(torch.float8_e4m3fn).float(), e


def _held(x, block_rows=1):
    """x at the values that its codes stand for."""
    q, e = _quantized(x, block_rows)
    return q * _power(e).repeat_interleave(block_rows, 0)[:x.shape[0]].repeat_interleave(128, 1)[:, :x.shape[1]]


def run(state):
    s, c = state, state["case"]
    kind = c["kind"]
    if own:
        from paper_2412_20796_amd import ops

        if kind == "dropout":
            how = dict(p=c["p"], seed=s["seed"], call=s["call"])
            return {"out": ops.dropout(s["x"], **how), "grad": ops.dropout(s["up"], **how)}
        if kind.startswith("norm"):
            h = ops.norm_forward(s["x"], s["pre"], c["pre"], eps=EPS)
            if kind == "norm_infer":
                return h
            dx, dw = ops.norm_backward(s["x"], s["pre"], s["dh"], c["pre"], eps=EPS)
            return {"h": h, "dx": dx, "dpre": dw}
        if kind.startswith("residual"):
            how = dict(post=s["post"], post_kind=c["post"] if c["post"] != "no" else "none", gate=s["g"], pre=s["pre"],
                       pre_kind=c["pre"] if c["pre"] != "no" else "rms", alpha=c["alpha"], beta=c["beta"], p=c["p"],
                       seed=s["seed"], call=s["call"], eps=EPS)
            y, h = ops.residual_forward(s["x"], s["f"], **how)
            if kind == "residual_infer":
                return {"y": y, "h": h}
            grad = ops.residual_backward(y, s["f"], s["dy"], s.get("dh"), **how)
            return {"y": y, "h": h, "dx": grad.dx, "df": grad.df, "dgate": grad.dgate, "dpost": grad.dpost, "dpre": grad.dpre}
        if kind == "linear_infer":
            return ops.fp8_linear(s["x"], ops.Fp8Matrix(s["codes"], s["scale"], block_rows=128))
        x, xt = ops.fp8_quantize_both(s["x"])
        w, wt = ops.fp8_quantize_both(s["w"], block_rows=128)
        up, upt = ops.fp8_quantize_both(s["dy"])
        t = s["x"].dtype
        return {"y": ops.fp8_matmul(x, w, dtype=t), "dx": ops.fp8_matmul(up, wt, dtype=t),
                "dw": ops.fp8_matmul(upt, xt, dtype=torch.float32)}
    t = TYPES[c["dtype"]]
    x = s["x"].float()
    if kind == "dropout":
        keep, f = _kept(*x.shape, c["p"], s["seed"], s["call"], x.device)
        return {k: torch.where(keep, s[n].float() * f, 0.0).to(t) for k, n in (("out", "x"), ("grad", "up"))}
    if kind.startswith("linear"):
        if kind == "linear_infer":
            w = s["codes"].float() * s["scale"].float().repeat_interleave(128, 0)[:c["n"]].repeat_interleave(128, 1)[:, :c["k"]]
            return (_held(x) @ w.T).to(t)
        w, up = s["w"].float(), s["dy"].float()
        wq = _held(w, 128)
        return {"y": (_held(x) @ wq.T).to(t), "dx": (_held(up) @ wq).to(t),
                "dw": _held(up.T.contiguous()) @ _held(x.T.contiguous()).T}
    if kind.startswith("norm"):
        h, n, r = _norm(x, s["pre"], c["pre"])
        if kind == "norm_infer":
            return h.to(t)
        dx, dw = _norm_grad(s["dh"].float(), s["pre"], n, r, c["pre"])
        return {"h": h.to(t), "dx": dx.to(t), "dpre": dw}
    v, fn, fr = _norm(s["f"].float(), s["post"], c["post"])
    gate = 1.0 if s["g"] is None else 1 / (1 + torch.exp(-s["g"].float()))
    keep, scale = _kept(*x.shape, c["p"], s["seed"], s["call"], x.device) if c["p"] > 0 else (True, 1.0)
    mask = c["beta"] * scale * keep
    y = (c["alpha"] * x + mask * (gate * v)).to(t)
    h, yn, yr = _norm(y.float(), s["pre"], c["pre"])
    out = {"y": y, "h": None if c["pre"] == "no" else h.to(t)}
    if kind == "residual_infer":
        return out
    dy, dpre = s["dy"].float(), None
    if c["pre"] != "no":
        dx, dpre = _norm_grad(s["dh"].float(), s["pre"], yn, yr, c["pre"])
        dy = dy + dx
    du = mask * dy
    df, dpost = _norm_grad(du * gate, s["post"], fn, fr, c["post"])
    dg = None if s["g"] is None else du * v * gate * (1 - gate)
    if c["gate"] == "row":
        dg = dg.sum(1, keepdim=True)
    return {**out, "dx": (c["alpha"] * dy).to(t), "df": df.to(t), "dgate": None if dg is None else dg.to(t), "dpost": dpost,
            "dpre": dpre}


def work(case):
    """Inputs and outputs once each; what a forward pass gives out is also the backward pass's input."""
    c = case
    es = 4 if c["dtype"] == "fp32" else 2
    if c["kind"].startswith("linear"):
        M, K, N = c["rows"], c["k"], c["n"]
        if c["kind"] == "linear_infer":
            return {"bytes": M * K * es + N * K + M * N * es, "flops": 2 * M * N * K}
        return {"bytes": 2 * (M * K + M * N) * es + N * K * (es + 4), "flops": 6 * M * N * K}
    v = c["rows"] * c["d"]
    if c["kind"] == "dropout":
        return {"bytes": 4 * v * es, "flops": 2 * 12 * v}
    fwd, bwd, ops = 2, 3, 8
    if c["kind"].startswith("residual"):
        g = {"none": 0, "row": 1 / c["d"], "all": 1}[c["gate"]]
        h = c["pre"] != "no"
        # x, f, g -> y, h; y (for the norm), f (for a norm, a scale or a gate), g, dy, dh -> dx, df, dg
        fwd, bwd = 3 + h + g, 3 + 2 * h + (c["post"] != "no" or g > 0) + 2 * g
        ops = 20 + (12 if c["p"] > 0 else 0)
    if c["kind"].endswith("infer"):
        bwd = 0
    return {"bytes": int((fwd + bwd) * v * es), "flops": ops * v * (1 if bwd == 0 else 3)}


# --- the same in 64 bits ---------------------------------------------------------------------------------------------------

def _exact_kept(rows, d, p, seed, call):
    """The generator in halves of 16 bits, whose products need no more than 32."""
    half = lambda v: (v & 0xFFFF, v >> 16)
    low, dev = (1 << 32) - 1, "cuda"

    def times(m, v):  # (upper, lower) 32 bits of m v
        (ml, mh), (vl, vh) = half(m), half(v)
        ll, mid = vl * ml, vl * mh + (vh * ml & low)
        carry = (ll >> 16) + (mid & 0xFFFF)
        top = vh * mh + (mid >> 16)
        return top + (carry >> 16) & low, (carry & 0xFFFF) << 16 | ll & 0xFFFF

    row, group = torch.meshgrid(torch.arange(rows, device=dev), torch.arange((d + 7) // 8, device=dev), indexing="ij")
    v = [group, row, torch.zeros_like(row) + call % 2 ** 32, torch.zeros_like(row) + call // 2 ** 32]
    for i in range(10):
        keys = [(word + i * step) % 2 ** 32 for word, step in ((seed % 2 ** 32, 2654435769), (seed // 2 ** 32, 3144134277))]
        h0, l0 = times(3528531795, v[0])
        h1, l1 = times(3449720151, v[2])
        v = [h1 ^ v[1] ^ keys[0], l1, h0 ^ v[3] ^ keys[1], l0]
    keep = torch.empty(rows, v[0].shape[1], 8, dtype=torch.bool, device=dev)
    cut = int(p * 65536 + 0.5)
    for i in range(4):
        lo, hi = half(v[i])
        keep[:, :, 2 * i], keep[:, :, 2 * i + 1] = lo >= cut, hi >= cut
    return keep.flatten(1)[:, :d], 0.0 if cut == 65536 else 1.0 / (1.0 - cut / 65536.0)


def _power_of_2(e):
    return ((e.long() + 1023) * 2 ** 52).view(torch.float64)


def _exact_held(x, block_rows=1):
    """x (64 bits) rounded to three bits after the leading one, in units of its block's power of two."""
    out = torch.empty_like(x)
    R, C = x.shape
    for c0 in range(0, C, 128):
        b = x[:, c0:c0 + 128]
        big = b.abs().amax(1)
        if block_rows > 1:
            big = torch.cat([big[r:r + block_rows].amax().expand(min(block_rows, R - r)) for r in range(0, R, block_rows)])
        # (a logarithm may be off a whole number where it is one, and so may a product with 1 / 448)
        m, e = torch.frexp(big / torch.full_like(big, 448))
        unit = _power_of_2((e - (m == 0.5).int()).clamp(min=-126))[:, None]
        v = b / unit
        lead = _power_of_2((torch.frexp(v)[1] - 1).clamp(min=-6) - 3)
        out[:, c0:c0 + 128] = torch.round(v / lead) * lead * unit
    return out


def exact(case, seed):
    c, s = case, prepare(case, seed)
    kind = c["kind"]
    x = s["x"].double()
    if kind == "dropout":
        keep, f = _exact_kept(*x.shape, c["p"], s["seed"], s["call"])
        return {"out": (x * f).masked_fill(~keep, 0), "grad": (s["up"].double() * f).masked_fill(~keep, 0)}
    if kind == "linear_infer":
        N, K = c["n"], c["k"]
        w = s["codes"].double() * torch.kron(s["scale"].double(), torch.ones(128, 128, dtype=torch.float64, device=x.device))[:N, :K]
        return _exact_held(x) @ w.T
    if kind == "linear_train":
        w, up = _exact_held(s["w"].double(), 128), s["dy"].double()
        return {"y": _exact_held(x) @ w.T, "dx": _exact_held(up) @ w,
                "dw": _exact_held(up.T.contiguous()) @ _exact_held(x.T.contiguous()).T}

    def normed(v, w, how):
        if how == "no":
            return v
        if how == "layer":
            var, mean = torch.var_mean(v, dim=1, unbiased=False, keepdim=True)
            v = (v - mean) / torch.sqrt(var + EPS)
        elif how == "rms":
            v = v / torch.sqrt(v.square().mean(dim=1, keepdim=True) + EPS)
        return torch.addcmul(w[1], v, w[0]) if w.shape[0] == 2 else v * w[0]

    leaf = lambda v: None if v is None else v.double().requires_grad_(True)
    pre = leaf(s["pre"])
    with torch.enable_grad():
        if kind.startswith("norm"):
            x.requires_grad_(True)
            h = normed(x, pre, c["pre"])
            if kind == "norm_infer":
                return h.detach()
            dx, dpre = torch.autograd.grad(h, [x, pre], s["dh"].double())
            return {"h": h.detach(), "dx": dx, "dpre": dpre}
        f, g, post = leaf(s["f"]), leaf(s["g"]), leaf(s["post"])
        x.requires_grad_(True)
        branch = normed(f, post, c["post"])
        if g is not None:
            branch = branch * torch.sigmoid(g)
        if c["p"] > 0:
            keep, scale = _exact_kept(*x.shape, c["p"], s["seed"], s["call"])
            branch = (branch * scale).masked_fill(~keep, 0)
        y = c["alpha"] * x + c["beta"] * branch
        held = y.detach().to(TYPES[c["dtype"]]).double().requires_grad_(True)  # the norm takes what is stored
        h = normed(held, pre, c["pre"])
        out = {"y": y.detach(), "h": None if c["pre"] == "no" else h.detach()}
        if kind == "residual_infer":
            return out
        up, dpre = s["dy"].double(), None
        if pre is not None:
            d, dpre = torch.autograd.grad(h, [held, pre], s["dh"].double())
            up = up + d
        names = [n for n, v in (("dx", x), ("df", f), ("dgate", g), ("dpost", post)) if v is not None]
        grads = dict(zip(names, torch.autograd.grad(y, [v for v in (x, f, g, post) if v is not None], up)))
    return {**out, **{n: grads.get(n) for n in ("dx", "df", "dgate", "dpost")}, "dpre": dpre}
