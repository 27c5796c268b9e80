"""Training with the gates' pre-activations kept in 8 bits (chgnet_hparams.act_bits = 8) against the fp64 oracle whose
backward pass reads the same checkpoint: every output has the bits of the fp32 path, and every gradient is the one at the
kept values; both interaction blocks, both widths, sparse cells, and the operators of chgnet_ops.h run together as a
training step of the caller's own."""
import numpy as np
import pytest
import torch

import ops_reference as ref
from gpu_helpers import ATOL, RTOL
from oracle import graph as og
from oracle import model as om
from paper_2412_20796_amd import binding as bd
from paper_2412_20796_amd import ops, synth

gpu = pytest.mark.gpu
W = (2.0, 1.5, 0.1, 0.1)


def _dev(x):
    return torch.as_tensor(np.ascontiguousarray(x)).to("cuda")


def _held(z, d, nudge):
    """What the checkpoint of z [rows, 2d] stands for. nudge: values whose code rounding of the forward pass may turn (within
    nudge of the row's largest |z|, where fp32's z may differ from 64 bits') take the other code."""
    out = []
    for x in (z[:, :d], z[:, d:]):
        lo, hi = x.min(1, keepdims=True), x.max(1, keepdims=True)
        step = np.maximum((hi - lo) / 255.0, 2.0 ** -100)
        t = (x - lo) / step
        q = np.rint(t)
        if nudge:
            edge = np.abs(np.abs(t - np.floor(t)) - 0.5) * step < nudge * np.abs(x).max(1, keepdims=True)
            q = np.where(edge, 2 * np.floor(t) + 1 - q, q)
        out.append(lo + q * step)
    return np.concatenate(out, 1)


def _phi(z, P, pre, d):
    yc = om.layernorm(z[:, :d], P[pre + "g_c"], P[pre + "b_c"])[0]
    return om.silu(yc) * om.sigmoid(om.layernorm(z[:, d:], P[pre + "g_g"], P[pre + "b_g"])[0])


def _keep8(cache, d, nudge=0.0):
    """The forward pass's cache with the checkpoint's values in place of the pre-activations, and phi at them."""
    layers = []
    for t, L in enumerate(cache["layers"]):
        L, P, pre = dict(L), cache["P"], "L%d_" % t
        L["zv"], L["ze"] = _held(L["zv"], d, nudge), _held(L["ze"], d, nudge)
        L["phiv"], L["phie"] = _phi(L["zv"], P, pre + "av_", d), _phi(L["ze"], P, pre + "be_", d)
        if L["za"] is not None:
            L["za"] = _held(L["za"], d, nudge)
        layers.append(L)
    return dict(cache, layers=layers)


def _oracle(ohp, b, graph, params, targets, delta):
    """Loss, gradient at the checkpoint, what turned codes can make of it (per value), and the gradient in full."""
    E, F, S, cache = om.forward(ohp, b, graph, params.astype(np.float64))
    loss, dE, dF, dS = om.loss_and_grads(E, F, S, cache["g"]["n_per"], *targets[:3], w=W[:3], delta=delta)
    dM = None
    if ohp.magmom:
        lm, dM = om.magmom_loss(cache["magmom"], targets[3], W[3], delta)
        loss += lm
    back = lambda c: om.backward(ohp, c, dE, dF, dS, dM)
    g8 = back(_keep8(cache, ohp.d))
    # fp32's z is within 3e-6 of the row's largest (products of 31 to 512 terms, a few layers deep)
    return loss, g8, np.abs(back(_keep8(cache, ohp.d, 3e-6)) - g8), back(cache)


def _check(b, d, T, name, magmom=False, sequential=False, delta=None, seed=(5, 0)):
    params = synth.make_params(d, T, seed=(seed[0], 1, seed[1]), magmom=magmom)
    targets = synth.make_targets(b, seed=(seed[0], 2, seed[1]), magmom=magmom)
    ohp = om.HParams(d=d, n_layers=T, magmom=magmom, sequential=sequential)
    rl, g8, turned, g_full = _oracle(ohp, b, og.build_graph(b.atom_ptr, b.pos, b.lattice), params, targets, delta)
    db, p, tg = bd.DeviceBatch.from_host(b), _dev(params), [_dev(x) for x in targets]
    got = {}
    for bits in (0, 8):
        hp = bd.hparams(d=d, n_layers=T, magmom=magmom, sequential=sequential, act_bits=bits)
        ws, g = bd.Workspace(), bd.DeviceGraph(b.n_atoms, 64, 16, 64)
        loss, grad = bd.step(hp, db, g, p, tg, ws, loss_w=W, huber_delta=delta or 0.0)
        outs = bd.forward(hp, db, g, p, ws)
        got[bits] = (loss, *outs, grad)
    for x, y in zip(got[0][:-1], got[8][:-1]):
        assert torch.equal(x, y), name
    assert abs(float(got[8][0]) - rl) <= ATOL + RTOL * abs(rl)
    gg = got[8][-1].cpu().numpy().astype(np.float64)
    for tname, (off, shape) in om.layout(ohp)[0].items():
        s = slice(off, off + int(np.prod(shape)))
        # the parity bound of the fp32 path, and twice the tensor's largest change by codes that may turn
        tol = ATOL + RTOL * np.abs(g8[s]) + 2 * turned[s].max(initial=0.0)
        err = np.abs(gg[s] - g8[s])
        assert (err <= tol).all(), (name, tname, err.max(), tol[np.argmax(err - tol)])
    return gg, g8, g_full


@gpu
@pytest.mark.parametrize("name", ["cubic8", "triclinic40"])
def test_gradient_is_that_of_the_checkpoint(name):
    gg, g8, full = _check(synth.make_batch(name), 64, 4, name)
    # and not the fp32 path's: the checkpoint's rounding shows, and the result follows it
    assert np.linalg.norm(gg - g8) < 0.1 * np.linalg.norm(full - g8)
    assert np.linalg.norm(full - g8) < 0.02 * np.linalg.norm(full)


@gpu
def test_variants():
    b = synth.random_crystals(seed=11, n_struct=3, n_lo=4, n_hi=12)
    _check(b, 64, 1, "T1")
    _check(b, 64, 3, "eq10 magmom huber", sequential=True, magmom=True, delta=0.1, seed=(6, 1))
    _check(b, 128, 3, "d128", seed=(6, 2))
    _check(b, 128, 2, "d128 eq10", sequential=True, magmom=True, seed=(6, 3))
    for seed in range(3):
        br = synth.random_crystals(seed=320 + seed, n_struct=1 + seed, n_lo=2, n_hi=14, rho=(0.06, 0.12))
        _check(br, 64, 3, "random%d" % seed, seed=(6, 4 + seed))


@gpu
def test_sparse_cells():
    """No bonds (B = A = 0) and an atom without edges (E = 0)."""
    b = synth.make_custom_batch([np.eye(3) * 8.5], [np.array([[0.0, 0.0, 0.0], [0.5, 0.5, 0.5]])], [np.array([3, 17])])
    _check(b, 64, 2, "no bonds")
    _check(b, 128, 2, "no bonds eq10", sequential=True)
    b1 = synth.make_custom_batch([np.eye(3) * 13.0], [np.zeros((1, 3))], [np.array([26])])
    _check(b1, 64, 2, "no edges")


def _grad(bits, b, d, T, dE, dF, dS, params):
    hp = bd.hparams(d=d, n_layers=T, act_bits=bits)
    ws, g, db, p = bd.Workspace(), bd.DeviceGraph(b.n_atoms, 64, 16, 64), bd.DeviceBatch.from_host(b), _dev(params)
    bd.build_graph(hp, db, g, ws)
    outs = bd.forward(hp, db, g, p, ws)
    return (*outs, bd.backward(hp, db, g, p, dE, dF, dS, ws))


def _copies(b, k):
    return synth.Batch(np.concatenate([[0]] + [b.atom_ptr[1:] + i * b.n_atoms for i in range(k)]).astype(np.int32),
                       np.tile(b.pos, (k, 1)), np.tile(b.lattice, (k, 1, 1)), np.tile(b.Z, k))


@gpu
@pytest.mark.parametrize("d,k", [(64, 4), (128, 2)])
def test_large_batch_is_the_sum_of_its_copies(d, k):
    """A batch of k copies of 40 crystals (341,096 edges at d = 64, whose gates take the tall tiles) has k times the
    gradient, and its outputs have the bits of the fp32 path."""
    b = synth.make_batch("triclinic40")
    params = synth.make_params(d, 3, seed=(7, 1, d))
    rng = np.random.default_rng(3)
    up = [rng.standard_normal(s).astype(np.float32) for s in ((b.n_struct,), (b.n_atoms, 3), (b.n_struct, 3, 3))]
    one = _grad(8, b, d, 3, *map(_dev, up), params)
    bk, upk = _copies(b, k), [_dev(np.concatenate([x] * k)) for x in up]
    many, plain = _grad(8, bk, d, 3, *upk, params), _grad(0, bk, d, 3, *upk, params)
    for x, y in zip(many[:3], plain[:3]):
        assert torch.equal(x, y)
    a, c, f = (t[-1].cpu().double().numpy() for t in (one, many, plain))
    # a row's products round by its parity in the batch, so a few codes turn: 1e-4 of the values by one step of 255, against
    # the rounding of all of them by up to half a step (`f`)
    assert np.linalg.norm(c - k * a) < 0.1 * np.linalg.norm(c - f)
    assert np.linalg.norm(c - f) < 0.02 * np.linalg.norm(f)


@gpu
def test_bitwise_reproducible_and_captured():
    """The same bits from two runs, and from a captured forward and backward pass replayed with eager steps between."""
    b = synth.make_batch("triclinic40")
    d, T = 64, 4
    hp, params = bd.hparams(d=d, n_layers=T, act_bits=8), synth.make_params(d, T, seed=(8, 1, 0))
    db, p = bd.DeviceBatch.from_host(b), _dev(params)
    rng = np.random.default_rng(4)
    up = [_dev(rng.standard_normal(s).astype(np.float32)) for s in ((b.n_struct,), (b.n_atoms, 3), (b.n_struct, 3, 3))]
    ws, g = bd.Workspace(), bd.DeviceGraph(b.n_atoms, 64, 16, 64)
    bd.build_graph(hp, db, g, ws)

    def passes(ws):
        return (*bd.forward(hp, db, g, p, ws), bd.backward(hp, db, g, p, *up, ws))

    want = [t.clone() for t in passes(ws)]
    for x, y in zip(want, passes(ws)):
        assert torch.equal(x, y)
    s, ws2 = torch.cuda.Stream(), bd.Workspace()
    with torch.cuda.stream(s):
        passes(ws2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        out = passes(ws2)
    for _ in range(3):
        for t in out:
            t.zero_()
        graph.replay()
        eager = passes(ws)
        torch.cuda.synchronize()
        for x, y, z in zip(want, out, eager):
            assert torch.equal(x, y) and torch.equal(x, z)


@gpu
def test_inference_and_md_have_the_bits_of_the_fp32_path():
    b = synth.make_batch("cubic8")
    params = synth.make_params(64, 4, seed=(11, 1, 0))
    got = []
    for bits in (0, 8):
        hp, db, p, ws = bd.hparams(act_bits=bits), bd.DeviceBatch.from_host(b), _dev(params), bd.Workspace()
        g = bd.DeviceGraph(b.n_atoms, 64, 16, 64)
        bd.build_graph(hp, db, g, ws)
        outs = list(bd.forward(hp, db, g, p, ws, save_for_backward=False))
        vel, im = torch.zeros(b.n_atoms, 3, device="cuda"), _dev((1.0 / (2.1 * b.Z)).astype(np.float32))
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            outs += bd.md(hp, db, g, p, vel, im, 0.5, 6, ws, skin=1.0)
        torch.cuda.synchronize()
        got.append(outs + [db.pos, vel])
    for x, y in zip(*got):
        assert torch.equal(x, y)


def test_workspace_is_smaller():
    """2 d + 8 bytes a gate row in place of 8 d: at least 6 d - 8 a row of every layer, less the arrays' alignment."""
    N, S = 1000, 20
    for d, T, E, B, A in ((64, 4, 85274, 9970, 86458), (128, 5, 430300, 49826, 397934), (64, 1, 0, 0, 0)):
        full, small = (bd.workspace_size(bd.hparams(d=d, n_layers=T, act_bits=q), N, E, B, A, S) for q in (0, 8))
        saved = T * (E + 2 * A) * (6 * d - 8)
        assert abs((full - small) - saved) <= T * 5 * 256


def test_what_is_refused():
    for kw in (dict(act_bits=4), dict(act_bits=32), dict(act_bits=-8), dict(act_bits=8, conservative=True)):
        with pytest.raises(bd.ChgnetError) as e:
            bd.param_count(bd.hparams(**kw))
        assert e.value.code == bd.CHGNET_EINVAL and "act_bits" in str(e.value)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_operators_together(dtype):
    """A training step of the caller's own: atoms embedded, one gated MLP, a second element table on the result's side; the
    gradients of both tables, the weight and the LayerNorm against autograd in 64 bits at the same checkpoint."""
    n, d, V, scale = 3000, 64, 94, 2.0
    g = torch.Generator().manual_seed(9)
    table = torch.randn(V, d, generator=g).to(dtype)
    Wt = (torch.randn(d, 2 * d, generator=g) / 8).to(dtype)
    ln = 0.3 * torch.randn(4, d, generator=g) + torch.tensor([[1.0], [0.0], [1.0], [0.0]])
    Z = torch.randint(1, V + 1, (n,), generator=g, dtype=torch.int32)
    up = torch.randn(n, d, generator=g).to(dtype)
    tc, Wc, lc, Zc = table.cuda(), Wt.cuda(), ln.cuda(), Z.cuda()
    x = ops.embed_forward(tc, Zc, scale=scale, first=1)
    z = x @ Wc
    phi, kept = ops.gate_forward(z, lc)
    dz, dln = ops.gate_backward(kept, lc, up.cuda())
    dx = dz @ Wc.t().contiguous()
    dtable = ops.embed_backward(Zc, dx, V, scale=scale, first=1)
    # each step against its own definition at what the step before it gave
    assert torch.equal(x.cpu(), ref.embed(table, Z, scale, 1))
    r, b = ref.gate(z.cpu(), ln)
    ref.assert_within(phi, r, b, dtype)
    q, step, lo = ref.checkpoint(z.cpu())
    assert torch.equal(kept.codes.cpu().double(), q)
    rz, rl, bz, bl = ref.gate_grad(q, step, ln, up)
    ref.assert_within(dz, rz, bz, dtype)
    ref.assert_within(dln, rl, bl)
    rt, bt = ref.embed_grad(Z, dx.cpu(), V, scale, 1)
    ref.assert_within(dtable, rt, bt)
    # and the whole against autograd through x W at the checkpoint's z: a product in `dtype` rounds z and dx (and the
    # results dz, dx) by eps each, the sums over the rows of an element do not add to that relative to their terms
    T64 = table.double().requires_grad_(True)
    zz = (T64[Z.long() - 1] * scale) @ Wt.double()
    at = (q.reshape(n, 2, d) * step[:, :, None] + lo).reshape(n, 2 * d)
    zz = at + (zz - zz.detach())
    yc, yg = (ref._ln(h)[0] for h in (zz[:, :d], zz[:, d:]))
    yc, yg = ln[0].double() * yc + ln[1].double(), ln[2].double() * yg + ln[3].double()
    (yc * torch.sigmoid(yc) * torch.sigmoid(yg) * up.double()).sum().backward()
    terms = torch.zeros(V, dtype=torch.float64).index_add_(0, Z.long() - 1, (dz.cpu().double().abs() @ Wt.double().abs().t()).amax(1))
    eps = torch.finfo(dtype).eps
    assert bool(((dtable.cpu().double() - T64.grad).abs() <= 4 * eps * scale * terms[:, None] + 1e-5).all())


@gpu
@pytest.mark.parametrize("k,kw", [(8, {}), (16, {}), (16, dict(act_bits=8)), (8, dict(conservative=True))])
def test_element_table_of_a_large_batch(k, kw):
    """8 and 16 copies of 40 crystals (8,632 and 17,264 atoms: the embedding operator's gradient with and without the
    ordering of the atoms) give k times the element table's gradient of one."""
    b = synth.make_batch("triclinic40")
    d, T = 64, 1
    params = synth.make_params(d, T, seed=(10, 1, 0))
    targets = synth.make_targets(b, seed=(10, 2, 0))
    hp, p = bd.hparams(d=d, n_layers=T, **kw), _dev(params)
    g = []
    for n in (1, k):
        bb, tg = _copies(b, n), [_dev(np.concatenate([x] * n)) for x in targets]
        loss, grad = bd.step(hp, bd.DeviceBatch.from_host(bb), bd.DeviceGraph(bb.n_atoms, 64, 16, 64), p, tg, bd.Workspace())
        g.append(grad[:94 * d].cpu().double().numpy())
    # the loss's means over k times as many values make the sums of k copies one copy's; sums of up to 16 x 20 rows round
    # by 2^-24 of their terms each, and the rows themselves by a few 1e-7 from batch to batch (codes that turn: 1e-4)
    scale = np.abs(g[0]).max()
    assert np.abs(g[1] - g[0]).max() <= (1e-3 if kw.get("act_bits") else 2e-5) * scale
