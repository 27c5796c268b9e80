"""What the norms, the residual connection and dropout refuse, and their workspace sizes (no GPU: every call here ends in its
checks)."""
import ctypes

import pytest
import torch

from paper_2412_20796_amd import binding as bd
from paper_2412_20796_amd import ops

P = 1 << 20  # an address that is aligned and never read: the calls below are refused before any launch
CFG = dict(post_kind=1, post_rows=1, pre_kind=2, pre_rows=2, gate_cols=64, alpha=1.0, beta=1.0, eps=1e-5, p=0.1, seed=1, call=2,
           step=None)
NORM_F = dict(rows=8, d=64, dtype=0, x=P, ldx=64, kind=1, w=P, w_rows=1, eps=1e-5, h=P, ldh=64, stream=None)
NORM_B = dict(rows=8, d=64, dtype=0, x=P, ldx=64, kind=1, w=P, w_rows=1, eps=1e-5, dh=P, lddh=64, dx=P, lddx=64, dw=P,
              accumulate=0, ws=P, ws_bytes=1 << 20, stream=None)
RES_F = dict(rows=8, d=64, dtype=0, cfg=CFG, x=P, ldx=64, f=P, ldf=64, g=P, ldg=64, post=P, pre=P, y=P, ldy=64, h=P, ldh=64,
             stream=None)
RES_B = dict(rows=8, d=64, dtype=0, cfg=CFG, y=P, ldy=64, f=P, ldf=64, g=P, ldg=64, post=P, pre=P, dy=P, lddy=64, dh=P,
             lddh=64, dx=P, lddx=64, df=P, lddf=64, dg=P, lddg=64, dpost=P, dpre=P, accumulate=0, ws=P, ws_bytes=1 << 20,
             stream=None)
DROP = dict(rows=8, d=64, dtype=0, x=P, ldx=64, p=0.1, seed=1, call=2, step=None, out=P, ldout=64, stream=None)


def _call(fn, base, **kw):
    a = dict(base)
    cfg = dict(a.get("cfg") or {})
    for k, v in kw.items():
        assert k in a or k in cfg, k
        (a if k in a else cfg)[k] = v
    if a.get("cfg") is not None:
        a["cfg"] = ctypes.addressof(held := ops._Residual(**cfg))
    return getattr(ops.lib(), fn)(*a.values())


SHAPES = [dict(rows=-1), dict(rows=1 << 32), dict(d=0), dict(dtype=3), dict(d=-4)]
WIDE = [dict(d=16385)]
BAD = ([("chgnet_norm_forward", NORM_F, k) for k in SHAPES + WIDE + [
            dict(kind=0), dict(kind=3), dict(w=None), dict(w_rows=0), dict(w_rows=3), dict(w=P + 2), dict(eps=0.0),
            dict(eps=float("nan")), dict(eps=1.5), dict(x=None), dict(h=None), dict(ldx=63), dict(ldh=0), dict(x=P + 2),
            dict(dtype=1, h=P + 1)]]
       + [("chgnet_norm_backward", NORM_B, k) for k in SHAPES + WIDE + [
            dict(kind=0), dict(w=None), dict(w_rows=3), dict(eps=-1.0), dict(x=None), dict(dh=None), dict(dx=None),
            dict(dw=None), dict(rows=0, dw=None), dict(dw=P + 2), dict(ldx=63), dict(lddh=63), dict(lddx=63), dict(ws=P + 8)]]
       + [("chgnet_residual_forward", RES_F, k) for k in SHAPES + WIDE + [
            dict(cfg=None), dict(post_kind=3), dict(post=None), dict(post_rows=0), dict(pre_kind=0), dict(pre_rows=3),
            dict(pre=None), dict(h=None), dict(gate_cols=2), dict(gate_cols=0), dict(ldg=63), dict(eps=0.0), dict(p=-0.1),
            dict(p=1.01), dict(p=float("nan")), dict(step=P + 4), dict(x=None), dict(f=None), dict(y=None), dict(ldx=63),
            dict(ldf=63), dict(ldy=63), dict(ldh=63), dict(g=P + 2), dict(post=P + 1), dict(pre=P + 2)]]
       + [("chgnet_residual_backward", RES_B, k) for k in SHAPES + WIDE + [
            dict(cfg=None), dict(post=None), dict(dpost=None), dict(dpre=None), dict(dh=None), dict(dg=None), dict(g=None),
            dict(f=None), dict(y=None), dict(dx=None), dict(df=None), dict(lddx=63), dict(lddf=63), dict(lddg=63),
            dict(lddy=63), dict(lddh=63), dict(ldy=63), dict(eps=2.0), dict(p=7.0), dict(dpost=P + 2), dict(ws=P + 4),
            dict(pre=None, dpre=None, dh=None, dy=None)]]
       + [("chgnet_dropout", DROP, k) for k in SHAPES + [
            dict(d=(1 << 30) + 1, ldx=1 << 31, ldout=1 << 31), dict(p=-1e-6), dict(p=1.5), dict(p=float("nan")), dict(x=None),
            dict(out=None), dict(ldx=63), dict(ldout=63), dict(step=P + 4), dict(x=P + 2), dict(dtype=2, out=P + 1)]])


@pytest.mark.parametrize("fn,base,kw", BAD)
def test_bad_arguments(fn, base, kw):
    assert _call(fn, base, **kw) == bd.CHGNET_EINVAL
    assert fn[len("chgnet_"):].encode() in bd.lib().chgnet_last_error_string()


@pytest.mark.parametrize("fn,base,kw", [
    ("chgnet_norm_backward", NORM_B, dict(ws=None)), ("chgnet_norm_backward", NORM_B, dict(ws_bytes=8 * 64 * 4 - 1)),
    ("chgnet_residual_backward", RES_B, dict(ws=None)), ("chgnet_residual_backward", RES_B, dict(ws_bytes=8 * 3 * 64 * 4 - 1)),
])
def test_small_workspace(fn, base, kw):
    assert _call(fn, base, **kw) == bd.CHGNET_EWORKSPACE


def test_no_rows_need_no_arrays():
    assert _call("chgnet_norm_forward", NORM_F, rows=0, x=None, h=None) == bd.CHGNET_OK
    assert _call("chgnet_norm_backward", NORM_B, rows=0, x=None, dh=None, dx=None, ws=None, ws_bytes=0,
                 accumulate=1) == bd.CHGNET_OK
    assert _call("chgnet_residual_forward", RES_F, rows=0, x=None, f=None, g=None, y=None, h=None) == bd.CHGNET_OK
    assert _call("chgnet_residual_backward", RES_B, rows=0, y=None, f=None, g=None, dy=None, dh=None, dx=None, df=None,
                 dg=None, ws=None, ws_bytes=0, accumulate=1) == bd.CHGNET_OK
    assert _call("chgnet_dropout", DROP, rows=0, x=None, out=None) == bd.CHGNET_OK


def test_workspace_sizes():
    n = ctypes.c_size_t()
    f = ops.lib().chgnet_residual_backward_workspace
    last = 0
    for rows in (0, 1, 7, 1000, 10 ** 6, (1 << 32) - 1):
        assert f(rows, 16384, 4, ctypes.byref(n)) == bd.CHGNET_OK and n.value >= last
        last = n.value
    assert 0 < last <= 512 * 4 * 16384 * 4
    assert f(100, 64, 0, ctypes.byref(n)) == bd.CHGNET_OK and n.value == 0
    for bad in ((-1, 64, 1), (8, 0, 1), (8, 16385, 1), (8, 64, 5), (8, 64, -1)):
        assert f(*bad, ctypes.byref(n)) == bd.CHGNET_EINVAL
    assert f(8, 64, 1, None) == bd.CHGNET_EINVAL


def test_host_tensors_and_inputs_that_autograd_follows_are_refused():
    x, w = torch.zeros(4, 64), torch.ones(1, 64)
    f = lambda t: t.clone().requires_grad_(True)
    for call in (lambda g: ops.norm_forward(g(x), w), lambda g: ops.norm_forward(x, g(w)),
                 lambda g: ops.norm_backward(x, w, g(x)), lambda g: ops.residual_forward(x, g(x)),
                 lambda g: ops.residual_forward(x, x, g(w)), lambda g: ops.residual_forward(x, x, gate=g(x)),
                 lambda g: ops.residual_backward(x, x, g(x)), lambda g: ops.residual_backward(x, x, x, g(x), pre=w),
                 lambda g: ops.dropout(g(x), 0.1, 1)):
        for g, word in ((f, "gradient"), (lambda t: t, "GPU")):
            with pytest.raises(bd.ChgnetError) as e:
                call(g)
            assert e.value.code == bd.CHGNET_EINVAL and word in str(e.value)
