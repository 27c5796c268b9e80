"""chgnet_norm_* and chgnet_residual_* against their definitions in 64 bits (block_reference.py): widths around the layouts,
rows around blocks and turns, each combination of norms, gate and dropout, types, strides, rows of one value and of values
that are not finite, streams, graphs, autograd and differences."""
import itertools

import pytest
import torch

import block_reference as ref
from ops_reference import assert_within
from paper_2412_20796_amd import binding as bd
from paper_2412_20796_amd import ops

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
WIDTHS = [1, 2, 3, 7, 8, 9, 16, 31, 32, 63, 64, 65, 72, 128, 129, 200, 256, 264, 333, 512, 520, 1000, 1024, 1025, 1032, 2048,
          2056, 4096, 4104, 5001, 8192, 8200, 9001, 16383, 16384]


def _inputs(rows, d, dtype, seed=0, cols=0, post=0, pre=0):
    g = torch.Generator().manual_seed(1000 * rows + 10 * d + seed)
    n = lambda *s: torch.randn(*s, generator=g)
    x = (n(rows, d) * torch.exp(0.5 * n(rows, 1))).to(dtype)
    f = (2 * n(rows, d) + n(1, d)).to(dtype)
    dy, dh = (n(rows, d) * torch.rand(rows, 1, generator=g)).to(dtype), n(rows, d).to(dtype)
    if rows > 2:
        dy[1], dh[1] = 0, 0
    w = lambda k: None if not k else n(k, d) * 0.3 + torch.tensor([[1.0], [0.0]])[:k]
    return x, f, dy, dh, (2 * n(rows, cols)).to(dtype) if cols else None, w(post), w(pre)


def _cuda(t):
    return None if t is None else t.cuda()


def _check(x, f, dy, dh, gate, post, pre, post_kind="rms", pre_kind="rms", alpha=1.0, beta=1.0, p=0.0, seed=3, call=4,
           eps=1e-5, what="", out=(), grads=()):
    """Both passes against the reference; returns (y, h, gradients)."""
    rows, d = x.shape
    dtype = x.dtype
    if post is None:
        post_kind = "none"
    how = dict(post=_cuda(post), post_kind=post_kind, gate=_cuda(gate), pre=_cuda(pre), pre_kind=pre_kind, alpha=alpha,
               beta=beta, p=p, seed=seed, call=call, eps=eps)
    fc = _cuda(f)
    y, h = ops.residual_forward(_cuda(x), fc, **how, **dict(out))
    got = ops.residual_backward(y, fc, _cuda(dy), _cuda(dh) if pre is not None else None, **how, **dict(grads))
    mask, factor = ref.kept(rows, d, p, seed, call) if p else (torch.ones(rows, d, dtype=torch.bool), 1.0)
    # the factors as the call has them: fp32 numbers
    alpha, beta, eps = (float(torch.tensor(v, dtype=torch.float32)) for v in (alpha, beta, eps))
    ry, by = ref.residual(x, f, post, post_kind, gate, alpha, beta, mask, factor, eps)
    assert_within(y, ry, by, dtype, what + " y")
    if pre is not None:
        rh, bh = ref.norm(y.cpu(), pre, pre_kind, eps)
        assert_within(h, rh, bh, dtype, what + " h")
    else:
        assert h is None
    want, bound = ref.residual_grad(y.cpu(), f, dy, dh if pre is not None else None, post, post_kind, gate, pre, pre_kind, alpha,
                                    beta, mask, factor, eps)
    for name, r in want.items():
        t = getattr(got, name)
        assert (t is None) == (r is None), name
        if r is not None:
            assert_within(t, r, bound[name], dtype if name in ("dx", "df", "dgate") else torch.float32, what + " " + name)
    return y, h, got


def _check_norm(x, w, dh, kind, what="", **kw):
    h = ops.norm_forward(_cuda(x), _cuda(w), kind)
    dx, dw = ops.norm_backward(_cuda(x), _cuda(w), _cuda(dh), kind, **kw)
    eps = float(torch.tensor(1e-5, dtype=torch.float32))
    r, b = ref.norm(x, w, kind, eps)
    assert_within(h, r, b, x.dtype, what + " h")
    rx, rw, bx, bw = ref.norm_grad(x, w, dh, kind, eps)
    assert_within(dx, rx, bx, x.dtype, what + " dx")
    assert_within(dw, rw, bw, what=what + " dw")
    return h, dx, dw


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", WIDTHS)
def test_norm_widths(d, dtype):
    rows = 21 if d > 1100 else 67
    for kind, k in (("rms", 1), ("layer", 2)):
        x, _, _, dh, _, _, w = _inputs(rows, d, dtype, pre=k)
        _check_norm(x, w, dh, kind, "d=%d %s %s" % (d, kind, dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", WIDTHS)
def test_residual_widths(d, dtype):
    rows = 13 if d > 1100 else 37
    _check(*_inputs(rows, d, dtype, cols=d, post=2, pre=2), post_kind="layer", pre_kind="layer", p=0.2, alpha=1.25, beta=0.5,
           what="layer d=%d %s" % (d, dtype))
    _check(*_inputs(rows, d, dtype, cols=1, post=1, pre=1), what="rms d=%d %s" % (d, dtype))


@pytest.mark.parametrize("d", [64, 128, 250, 1024, 2048])
@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 15, 16, 17, 31, 33, 63, 64, 65, 129, 255, 257, 1025, 5000])
def test_rows(rows, d):
    _check(*_inputs(rows, d, torch.float32, cols=d, post=2, pre=2), post_kind="layer", p=0.1, what="rows=%d d=%d" % (rows, d))


@pytest.mark.parametrize("rows,d,dtype", [(70001, 64, torch.float32), (40003, 128, torch.bfloat16), (20011, 333, torch.bfloat16)])
def test_more_rows_than_one_pass(rows, d, dtype):
    x, f, dy, dh, gate, post, pre = _inputs(rows, d, dtype, cols=1, post=2, pre=2)
    _check(x, f, dy, dh, gate, post, pre, pre_kind="layer", p=0.1)
    _check_norm(x, pre, dh, "layer")


@pytest.mark.parametrize("cols,post_kind,pre_kind,p", itertools.product([0, 1, 96], ["rms", "layer", "none", None],
                                                                        ["rms", "layer", None], [0.0, 0.4]))
@pytest.mark.parametrize("k", [1, 2])
def test_forms(k, cols, post_kind, pre_kind, p):
    i = _inputs(29, 96, torch.float32, cols=cols, post=k if post_kind else 0, pre=k if pre_kind else 0)
    _check(*i, post_kind=post_kind, pre_kind=pre_kind or "rms", p=p, alpha=0.75, beta=-1.5)


def test_gradient_of_h_alone():
    x, f, _, dh, gate, post, pre = _inputs(40, 128, torch.float32, cols=128, post=1, pre=1)
    _check(x, f, None, dh, gate, post, pre)


@pytest.mark.parametrize("alpha,beta", [(0.0, 1.0), (1.0, 0.0), (-2.0, 0.22)])
def test_factors(alpha, beta):
    _check(*_inputs(40, 72, torch.float32, cols=1, post=2, pre=2), alpha=alpha, beta=beta)


def test_all_or_none_dropped():
    for p in (1.0, 2.0 ** -18):
        _check(*_inputs(40, 72, torch.float32, cols=72, post=2, pre=2), p=p)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,pad,shift", [(64, 8, 0), (64, 3, 0), (64, 8, 1), (128, 8, 4), (50, 6, 2), (1000, 24, 0), (2048, 1, 0)])
def test_strides_and_alignment(d, pad, shift, dtype):
    """Rows inside wider buffers, at offsets that do and do not allow vector loads; what lies between the rows stays."""
    rows = 37
    x, f, dy, dh, gate, post, pre = _inputs(rows, d, dtype, cols=d, post=2, pre=2)
    bufs = []

    def view(fill=None, cols=d):
        buf = torch.full((shift + rows * (cols + pad),), 7.0, dtype=dtype, device="cuda")
        v = buf[shift:].reshape(rows, cols + pad)[:, :cols]
        if fill is not None:
            v.copy_(fill)
        bufs.append((buf, v))
        return v

    odd = lambda t: torch.cat([torch.zeros(1), t.reshape(-1)]).cuda()[1:].reshape(t.shape)  # at any float
    how = dict(post=odd(post), post_kind="layer", gate=view(gate), pre=odd(pre), pre_kind="layer", p=0.1, seed=3, call=4)
    y, h = ops.residual_forward(view(x), view(f), **how, y=view(), h=view())
    got = ops.residual_backward(y, view(f), view(dy), view(dh), **how, dx=view(), df=view(), dgate=view())
    y2, h2, got2 = _check(x, f, dy, dh, gate, post, pre, post_kind="layer", pre_kind="layer", p=0.1)
    hn = ops.norm_forward(y, odd(pre), "layer", h=view())
    dxn, _ = ops.norm_backward(y, odd(pre), view(dh), "layer", dx=view())
    want, bound = ref.residual_grad(y.cpu(), f, dy, dh, post, "layer", gate, pre, "layer", 1.0, 1.0,
                                    *ref.kept(rows, d, 0.1, 3, 4), float(torch.tensor(1e-5)))
    for name in want:
        assert_within(getattr(got, name), want[name], bound[name], torch.float32 if name[1] == "p" else dtype, name)
    r, b = ref.norm(y.cpu(), pre, "layer", float(torch.tensor(1e-5)))
    assert_within(h, r, b, dtype) or assert_within(hn, r, b, dtype)
    rx, _, bx, _ = ref.norm_grad(y.cpu(), pre, dh, "layer", float(torch.tensor(1e-5)))
    assert_within(dxn, rx, bx, dtype)
    for buf, v in bufs:
        v.fill_(7.0)
        assert bool((buf == 7).all())


def test_h_is_the_norm_of_the_stored_y():
    for dtype in TYPES:
        x, f, _, _, _, post, pre = _inputs(50, 256, dtype, post=1, pre=1)
        y, h = ops.residual_forward(x.cuda(), f.cuda(), post.cuda(), pre=pre.cuda())
        assert torch.equal(h, ops.norm_forward(y, pre.cuda()))


def test_rows_do_not_depend_on_their_number():
    x, f, _, _, gate, post, pre = _inputs(300, 512, torch.bfloat16, cols=512, post=1, pre=1)
    a = ops.residual_forward(x.cuda(), f.cuda(), post.cuda(), gate=gate.cuda(), pre=pre.cuda())
    for n in (1, 7):
        b = ops.residual_forward(x[:n].cuda(), f[:n].cuda(), post.cuda(), gate=gate[:n].cuda(), pre=pre.cuda())
        assert torch.equal(a[0][:n], b[0]) and torch.equal(a[1][:n], b[1])


def test_rows_of_one_value_and_large_and_small_ones():
    for d in (64, 100, 2048):
        for kind in ("rms", "layer"):
            x, f, dy, dh, gate, post, pre = _inputs(9, d, torch.float32, cols=1, post=2, pre=2)
            f[2], x[3], f[3] = 3.25, 0.0, 0.0
            f[4] *= 1e-18
            f[5] *= 1e15
            dy[6], dh[6] = 0, 0
            _check(x, f, dy, dh, gate, post, pre, post_kind=kind, pre_kind=kind, what="d=%d %s" % (d, kind))


@pytest.mark.parametrize("d", [64, 70, 2048])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_up_to_the_ranges_end(kind, d):
    """Mean squares next to fp32's largest number are in range; past it n(x) is 0, and no gradient passes."""
    x, _, _, dh, _, _, w = _inputs(11, d, torch.float32, pre=2)
    x = x / x.double().square().mean(1, keepdim=True).sqrt().float()
    _check_norm(x * 1.2e19, w, dh, kind)
    far = x * 1e21
    h, dx = ops.norm_forward(far.cuda(), w.cuda(), kind), ops.norm_backward(far.cuda(), w.cuda(), dh.cuda(), kind)[0]
    assert torch.equal(h.cpu(), w[1].expand(11, d)) and not dx.any()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("d", [64, 70, 2048])
def test_values_that_are_not_finite(d, value):
    """They stay in their row, and have no part in anything where dropout takes them out (no norm after the block)."""
    i = _inputs(33, d, torch.float32, cols=d, pre=1)
    x, f, dy, dh, gate, _, pre = i
    mask, _ = ref.kept(33, d, 0.3, 3, 4)
    clean = _check(*i, p=0.3)
    f2, g2 = torch.where(mask, f, torch.tensor(value)), torch.where(mask, gate, torch.tensor(value))
    how = dict(gate=g2.cuda(), pre=pre.cuda(), p=0.3, seed=3, call=4)
    y, h = ops.residual_forward(x.cuda(), f2.cuda(), **how)
    got = ops.residual_backward(y, f2.cuda(), dy.cuda(), dh.cuda(), **how)
    for a, b in zip((y, h, *got), (clean[0], clean[1], *clean[2])):
        assert (a is None and b is None) or torch.equal(a, b)
    x[7, 3] = value
    y, h = ops.residual_forward(x.cuda(), f.cuda(), **{**how, "gate": gate.cuda()})
    got = ops.residual_backward(y, f.cuda(), dy.cuda(), dh.cuda(), **{**how, "gate": gate.cuda()})
    rows = torch.arange(33) != 7
    for a, b in ((y, clean[0]), (h, clean[1]), (got.dx, clean[2].dx), (got.df, clean[2].df), (got.dgate, clean[2].dgate)):
        assert torch.equal(a.cpu()[rows], b.cpu()[rows])
    # (df and dgate of an infinity alone may be where dropout takes it out)
    assert not any(bool(torch.isfinite(a.cpu()[7]).all()) for a in (y, h, got.dx))


@pytest.mark.parametrize("rows", [0, 5, 3000])
def test_accumulate(rows):
    x, f, dy, dh, gate, post, pre = (_cuda(t) for t in _inputs(rows, 64, torch.float32, cols=1, post=2, pre=2))
    how = dict(post=post, post_kind="layer", gate=gate, pre=pre)
    y, h = ops.residual_forward(x, f, **how)
    once = ops.residual_backward(y, f, dy, dh, **how)
    if rows == 0:
        assert not once.dpost.any() and not once.dpre.any()
    a, b = torch.full_like(post, 3.0), torch.full_like(pre, -2.0)
    twice = ops.residual_backward(y, f, dy, dh, **how, dpost=a, dpre=b, accumulate=True)
    assert twice.dpost is a and torch.equal(a, once.dpost + 3.0) and torch.equal(b, once.dpre - 2.0)
    dw = torch.ones_like(pre)
    one = ops.norm_backward(y, pre, dh, "layer")[1]
    assert torch.equal(ops.norm_backward(y, pre, dh, "layer", dw=dw, accumulate=True)[1], one + 1.0)


def test_the_same_bits_each_time():
    for rows, d, dtype in ((5000, 64, torch.float32), (3001, 333, torch.bfloat16), (700, 8192, torch.bfloat16)):
        i = [_cuda(t) for t in _inputs(rows, d, dtype, cols=d, post=1, pre=1)]
        x, f, dy, dh, gate, post, pre = i
        how = dict(post=post, gate=gate, pre=pre, p=0.1, seed=1)
        y, _ = ops.residual_forward(x, f, **how)
        first = ops.residual_backward(y, f, dy, dh, **how)
        for _ in range(3):
            assert all(torch.equal(a, b) for a, b in zip(first, ops.residual_backward(y, f, dy, dh, **how)))


def test_streams_and_a_graph_with_a_shared_workspace():
    i = [_cuda(t) for t in _inputs(2000, 128, torch.bfloat16, cols=128, post=1, pre=1)]
    x, f, dy, dh, gate, post, pre = i
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    how = dict(post=post, gate=gate, pre=pre, p=0.1, seed=5, call=11, step=step)
    ws = bd.Workspace()

    def both():
        y, h = ops.residual_forward(x, f, **how)
        return (y, h, *ops.residual_backward(y, f, dy, dh, **how, ws=ws))

    want = []
    for k in range(3):
        step.fill_(k)
        want.append([t.clone() for t in both()])
    assert not torch.equal(want[0][0], want[1][0])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step.fill_(0)
        got = both()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want[0]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = both()
        step.add_(1)
    step.zero_()
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want[k])), k


def test_gradients_against_differences():
    """The gradients by central differences in 64 bits of the definition (with dropout's mask)."""
    rows, d = 3, 10
    x, f, dy, dh, gate, post, pre = _inputs(rows, d, torch.float32, cols=1, post=2, pre=2, seed=1)
    _, _, got = _check(x, f, dy, dh, gate, post, pre, post_kind="layer", pre_kind="layer", p=0.3, alpha=1.25, beta=0.5)
    mask, factor = ref.kept(rows, d, 0.3, 3, 4)
    v = {"dx": x.double(), "df": f.double(), "dgate": gate.double(), "dpost": post.double(), "dpre": pre.double()}

    def total(v):
        y, _ = ref.residual(v["dx"], v["df"], v["dpost"], "layer", v["dgate"], 1.25, 0.5, mask, factor, 1e-5)
        h, _ = ref.norm(y, v["dpre"], "layer", 1e-5)
        return float((y * dy.double()).sum() + (h * dh.double()).sum())

    step = 1e-6
    for name, t in v.items():
        for k in range(0, t.numel(), 3):
            e = torch.zeros(t.numel(), dtype=torch.float64)
            e[k] = step
            e = e.reshape(t.shape)
            num = (total({**v, name: t + e}) - total({**v, name: t - e})) / (2 * step)
            have = float(getattr(got, name).reshape(-1)[k])
            # y is stored in fp32 (2^-24 of values of a few); differences: 1e-15 / step, and step^2 times a third derivative
            assert abs(have - num) <= 2e-5 + 2e-5 * abs(num), (name, k, have, num)


def test_a_function_of_the_callers():
    """In a torch.autograd.Function, as documented."""

    class Connect(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, f, gate, post, pre):
            ctx.how = dict(post=post, gate=gate, pre=pre, p=0.1, seed=2)
            y, h = ops.residual_forward(x, f, **ctx.how)
            ctx.y, ctx.f = y, f
            return y, h

        @staticmethod
        def backward(ctx, dy, dh):
            g = ops.residual_backward(ctx.y, ctx.f, dy.contiguous(), dh.contiguous(), **ctx.how)
            return g.dx, g.df, g.dgate, g.dpost, g.dpre

    x, f, dy, dh, gate, post, pre = (_cuda(t) for t in _inputs(64, 128, torch.float32, cols=1, post=1, pre=1))
    leaves = [t.clone().requires_grad_(True) for t in (x, f, gate, post, pre)]
    y, h = Connect.apply(*leaves)
    ((y * dy).sum() + (h * dh).sum()).backward()
    with torch.no_grad():
        want = ops.residual_backward(y, f, dy, dh, post=post, gate=gate, pre=pre, p=0.1, seed=2)
    assert all(torch.equal(t.grad, g) for t, g in zip(leaves, want))


def test_sizes_past_32_bits():
    rows, d = 270000, 8200
    x, f, dy, dh, gate, post, pre = _inputs(512, d, torch.bfloat16, cols=1, post=1, pre=1)
    big = lambda t: t.cuda().repeat(rows // 512 + 1, 1)[:rows]
    how = dict(post=post.cuda(), pre=pre.cuda())
    xb, fb, gb = big(x), big(f), big(gate)
    y, h = ops.residual_forward(xb, fb, gate=gb, **how)
    some = slice(rows - 100, rows)
    small = ops.residual_forward(xb[some].contiguous(), fb[some].contiguous(), gate=gb[some].contiguous(), **how)
    assert torch.equal(y[some], small[0]) and torch.equal(h[some], small[1])
    dyb, dhb = big(dy), big(dh)
    got = ops.residual_backward(y, fb, dyb, dhb, gate=gb, **how)
    part = ops.residual_backward(small[0], fb[some].contiguous(), dyb[some].contiguous(), dhb[some].contiguous(),
                                 gate=gb[some].contiguous(), **how)
    assert all(torch.equal(getattr(got, n)[some], getattr(part, n)) for n in ("dx", "df", "dgate"))


def test_refusals():
    x, f, dy, dh, gate, post, pre = (_cuda(t) for t in _inputs(8, 64, torch.float32, cols=64, post=2, pre=2))
    z = lambda *s, **k: torch.zeros(*s, device="cuda", **k)
    fwd, bwd = ops.residual_forward, ops.residual_backward
    for call in (lambda: fwd(x, f[:7]), lambda: fwd(x, f.half()), lambda: fwd(x, f, post[:, :63]), lambda: fwd(x, f, z(3, 64)),
                 lambda: fwd(x, f, post, "bad"), lambda: fwd(x, f, None, "rms"), lambda: fwd(x, f, pre=pre, pre_kind="none"),
                 lambda: fwd(x, f, gate=z(8, 2)), lambda: fwd(x, f, gate=z(7, 1)), lambda: fwd(x, f, h=z(8, 64)),
                 lambda: fwd(x, f, p=2.0), lambda: fwd(x, f, eps=0.0), lambda: fwd(x, f, eps=2.0), lambda: fwd(x, f, seed=-1),
                 lambda: fwd(x, f, p=0.1, step=z(1)), lambda: fwd(x, f, y=z(8, 63)), lambda: fwd(x, f, x.double()),
                 lambda: bwd(x, f, None), lambda: bwd(x, f, dy, dh), lambda: bwd(x, f, dy, None, pre=pre),
                 lambda: bwd(x, f, dy, dgate=z(8, 64)), lambda: bwd(x, f, dy, dpost=z(2, 64)),
                 lambda: bwd(x, f, dy, post=post, accumulate=True), lambda: bwd(x, f, dy, post=post, dpost=z(1, 64)),
                 lambda: bwd(x, f, dy[:, ::2]), lambda: ops.norm_forward(x, pre, "none"), lambda: ops.norm_forward(x, pre[0]),
                 lambda: ops.norm_forward(z(2, 16385), z(1, 16385)), lambda: ops.norm_backward(x, pre, dh.half()),
                 lambda: ops.norm_backward(x, pre, dh, accumulate=True), lambda: ops.norm_forward(x, pre.cpu())):
        with pytest.raises(bd.ChgnetError) as e:
            call()
        assert e.value.code == bd.CHGNET_EINVAL
