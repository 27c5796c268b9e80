"""A residual block out of the operators, as a model has it: norm, 8-bit linear layer, gate, linear layer, the residual
connection with its norms, gate and dropout; forward and backward, and replayed as a graph. Each operator is checked against its
definition in 64 bits at the inputs that it was given, and the whole against its formula in 64 bits without 8-bit rounding."""
import pytest
import torch

import block_reference as ref
import fp8_reference as fp8
import ops_reference as gate_ref
from ops_reference import assert_within
from paper_2412_20796_amd import binding as bd
from paper_2412_20796_amd import ops

pytestmark = pytest.mark.gpu
EPS = float(torch.tensor(1e-5))


def _model(rows, d, dtype):
    g = torch.Generator().manual_seed(rows + d)
    n = lambda *s: torch.randn(*s, generator=g)
    gates = lambda k: 0.1 * n(k, d) + torch.tensor([1.0, 0.0, 1.0, 0.0])[:k, None]
    return {k: v.cuda() for k, v in dict(
        x=n(rows, d).to(dtype), pre0=gates(2), w1=(n(2 * d, d) / d ** 0.5).to(dtype), ln=gates(4),
        w2=(n(d, d) / d ** 0.5).to(dtype), post=gates(1), pre1=gates(2), g=n(rows, 1).to(dtype),
        dy=n(rows, d).to(dtype), dh=n(rows, d).to(dtype)).items()}


def _step(m, ws, step=None):
    """Forward and backward of y, h; {name: tensor} of everything on the way."""
    how = dict(post=m["post"], post_kind="rms", gate=m["g"], pre=m["pre1"], pre_kind="layer", beta=0.5, p=0.1, seed=11, call=3,
               step=step)
    t = m["x"].dtype
    r = {}
    r["h0"] = ops.norm_forward(m["x"], m["pre0"], "layer")
    (hq, ht), (w1, w1t), (w2, w2t) = (ops.fp8_quantize_both(v, br)
                                      for v, br in ((r["h0"], 1), (m["w1"], 128), (m["w2"], 128)))
    r["z"] = ops.fp8_matmul(hq, w1, t, ws=ws)
    r["phi"], kept = ops.gate_forward(r["z"], m["ln"])
    pq, pt = ops.fp8_quantize_both(r["phi"])
    r["f"] = ops.fp8_matmul(pq, w2, t, ws=ws)
    r["y"], r["h"] = ops.residual_forward(m["x"], r["f"], **how)
    grad = ops.residual_backward(r["y"], r["f"], m["dy"], m["dh"], **how, ws=ws)
    r.update(df=grad.df, dg=grad.dgate, dpost=grad.dpost, dpre1=grad.dpre)
    fq, ft = ops.fp8_quantize_both(grad.df)
    r["dw2"] = ops.fp8_matmul(ft, pt, torch.float32, ws=ws)
    r["dphi"] = ops.fp8_matmul(fq, w2t, t, ws=ws)
    r["dz"], r["dln"] = ops.gate_backward(kept, m["ln"], r["dphi"], ws=ws)
    zq, zt = ops.fp8_quantize_both(r["dz"])
    r["dw1"] = ops.fp8_matmul(zt, ht, torch.float32, ws=ws)
    r["dh0"] = ops.fp8_matmul(zq, w1t, t, ws=ws)
    dx, r["dpre0"] = ops.norm_backward(m["x"], m["pre0"], r["dh0"], "layer", ws=ws)
    r["dx"] = dx + grad.dx
    return r


def _exact(m):
    """The same formulas in 64 bits by autograd, without rounding to 8 bits."""
    v = {k: t.double().cpu() for k, t in m.items()}
    for k in ("x", "pre0", "w1", "ln", "w2", "post", "pre1", "g"):
        v[k].requires_grad_(True)
    h0, _ = ref.norm(v["x"], v["pre0"], "layer", EPS)
    z = h0 @ v["w1"].T
    d = v["x"].shape[1]
    core, gate = (torch.nn.functional.layer_norm(z[:, k * d:(k + 1) * d], (d,), v["ln"][2 * k], v["ln"][2 * k + 1], EPS)
                  for k in (0, 1))
    f = (torch.nn.functional.silu(core) * torch.sigmoid(gate)) @ v["w2"].T
    mask, factor = ref.kept(*v["x"].shape, 0.1, 11, 3)
    y, _ = ref.residual(v["x"], f, v["post"], "rms", v["g"], 1.0, 0.5, mask, factor, EPS)
    h, _ = ref.norm(y, v["pre1"], "layer", EPS)
    names = dict(dx="x", dpre0="pre0", dw1="w1", dln="ln", dw2="w2", dpost="post", dpre1="pre1", dg="g")
    grads = torch.autograd.grad((y * v["dy"]).sum() + (h * v["dh"]).sum(), [v[k] for k in names.values()])
    return dict(zip(names, grads), y=y.detach(), h=h.detach())


@pytest.mark.parametrize("rows,d,dtype", [(1, 64, torch.float32), (300, 128, torch.bfloat16), (1111, 200, torch.float32)])
def test_step(rows, d, dtype):
    m = _model(rows, d, dtype)
    r = _step(m, bd.Workspace())
    c = {k: t.cpu() for k, t in {**m, **r}.items()}
    h, b = ref.norm(c["x"], c["pre0"], "layer", EPS)
    assert_within(r["h0"], h, b, dtype, "h0")
    held = lambda t, br=1: fp8.values(*fp8.quantize(t, br), br)
    for name, a, w, t in (("z", held(c["h0"]), held(c["w1"], 128), dtype), ("f", held(c["phi"]), held(c["w2"], 128), dtype),
                          ("dphi", held(c["df"]), held(c["w2"], 128).T, dtype), ("dh0", held(c["dz"]), held(c["w1"], 128).T, dtype),
                          ("dw2", held(c["df"].T), held(c["phi"].T), torch.float32),
                          ("dw1", held(c["dz"].T), held(c["h0"].T), torch.float32)):
        want, bound = fp8.product(a, w, t)
        assert_within(r[name], want, bound, t, name)
    phi, b = gate_ref.gate(c["z"], c["ln"])
    assert_within(r["phi"], phi, b, dtype, "phi")
    mask, factor = ref.kept(rows, d, 0.1, 11, 3)
    y, b = ref.residual(c["x"], c["f"], c["post"], "rms", c["g"], 1.0, 0.5, mask, factor, EPS)
    assert_within(r["y"], y, b, dtype, "y")
    want, bound = ref.residual_grad(c["y"], c["f"], c["dy"], c["dh"], c["post"], "rms", c["g"], c["pre1"], "layer", 1.0, 0.5,
                                    mask, factor, EPS)
    for name, key in (("df", "df"), ("dg", "dgate"), ("dpost", "dpost"), ("dpre1", "dpre")):
        assert_within(r[name], want[key], bound[key], dtype if name in ("df", "dg") else torch.float32, name)
    # the whole: each of at most 8 roundings to 8 bits on a path is off by at most 2^-4 of its value, of random sign, so
    # that a sum's error is at most 2^-4 of its terms' root mean square each: 8 of them 2^-4 8^(1/2) < 0.18
    whole = _exact(m)
    for name, want in whole.items():
        got = r[name].cpu().double()
        assert float((got - want).norm()) <= 0.18 * float(want.norm()) + 1e-6, (name, float((got - want).norm() / want.norm()))


def test_replayed_step():
    m = _model(640, 128, torch.bfloat16)
    step, ws = torch.zeros(1, dtype=torch.int64, device="cuda"), bd.Workspace()
    want = []
    for k in range(3):
        step.fill_(k)
        want.append({n: t.clone() for n, t in _step(m, ws, step).items()})
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _step(m, ws, step)
        step.add_(1)
    step.zero_()
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], want[k][n]) for n in got), k
        assert float(want[k]["y"].float().sum()) == float(want[k]["y"].float().sum())
    assert not torch.equal(want[0]["y"], want[1]["y"])
