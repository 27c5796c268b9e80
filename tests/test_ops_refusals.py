"""What the operators of include/chgnet_ops.h refuse, and their workspace sizes (no GPU: every call here ends in its
checks), and that the header, the library and the binding name the same entry points."""
import ctypes
import os
import re

import pytest
import torch

from paper_2412_20796_amd import binding as bd
from paper_2412_20796_amd import ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20  # an address that is aligned and never read: the calls below are refused before any launch


def _call(fn, base, **kw):
    a = dict(base)
    assert set(kw) <= set(a), kw
    a.update(kw)
    return getattr(ops.lib(), fn)(*a.values())


GATE_F = dict(rows=8, d=64, dtype=0, z=P, ldz=128, ln=P, phi=P, ldphi=64, codes=P, step=P, stream=None)
GATE_B = dict(rows=8, d=64, dtype=0, codes=P, step=P, ln=P, dphi=P, lddphi=64, dz=P, lddz=128, dln=P, accumulate=0, ws=P,
              ws_bytes=1 << 20, stream=None)
EMB_F = dict(n=8, d=64, vocab=94, dtype=0, tok=P, first=1, table=P, ldtable=64, scale=1.0, out=P, ldout=64, stream=None)
EMB_B = dict(n=20000, d=64, vocab=94, dtype=0, tok=P, first=1, dout=P, lddout=64, scale=1.0, dtable=P, lddtable=64,
             accumulate=0, ws=P, ws_bytes=1 << 26, stream=None)
BAD = [
    ("chgnet_gate_forward", GATE_F, dict(rows=-1)),
    ("chgnet_gate_forward", GATE_F, dict(d=0)),
    ("chgnet_gate_forward", GATE_F, dict(d=1025, ldz=2050, ldphi=1025)),
    ("chgnet_gate_forward", GATE_F, dict(dtype=3)),
    ("chgnet_gate_forward", GATE_F, dict(ldz=127)),
    ("chgnet_gate_forward", GATE_F, dict(ldphi=63)),
    ("chgnet_gate_forward", GATE_F, dict(z=None)),
    ("chgnet_gate_forward", GATE_F, dict(ln=None)),
    ("chgnet_gate_forward", GATE_F, dict(phi=None)),
    ("chgnet_gate_forward", GATE_F, dict(codes=None)),
    ("chgnet_gate_forward", GATE_F, dict(step=None)),
    ("chgnet_gate_forward", GATE_F, dict(step=P + 4)),
    ("chgnet_gate_forward", GATE_F, dict(z=P + 2)),
    ("chgnet_gate_forward", GATE_F, dict(dtype=1, phi=P + 1)),
    ("chgnet_gate_backward", GATE_B, dict(rows=-5)),
    ("chgnet_gate_backward", GATE_B, dict(d=-64)),
    ("chgnet_gate_backward", GATE_B, dict(dtype=-1)),
    ("chgnet_gate_backward", GATE_B, dict(lddz=64)),
    ("chgnet_gate_backward", GATE_B, dict(lddphi=0)),
    ("chgnet_gate_backward", GATE_B, dict(codes=None)),
    ("chgnet_gate_backward", GATE_B, dict(step=None)),
    ("chgnet_gate_backward", GATE_B, dict(dphi=None)),
    ("chgnet_gate_backward", GATE_B, dict(dz=None)),
    ("chgnet_gate_backward", GATE_B, dict(dln=None)),
    ("chgnet_gate_backward", GATE_B, dict(rows=0, dln=None)),
    ("chgnet_gate_backward", GATE_B, dict(step=P + 4)),
    ("chgnet_gate_backward", GATE_B, dict(ws=P + 8)),
    ("chgnet_embed_forward", EMB_F, dict(n=-1)),
    ("chgnet_embed_forward", EMB_F, dict(d=0)),
    ("chgnet_embed_forward", EMB_F, dict(d=65537, ldtable=65537, ldout=65537)),
    ("chgnet_embed_forward", EMB_F, dict(vocab=0)),
    ("chgnet_embed_forward", EMB_F, dict(vocab=1 << 31)),
    ("chgnet_embed_forward", EMB_F, dict(first=-1)),
    ("chgnet_embed_forward", EMB_F, dict(dtype=9)),
    ("chgnet_embed_forward", EMB_F, dict(ldtable=63)),
    ("chgnet_embed_forward", EMB_F, dict(ldout=63)),
    ("chgnet_embed_forward", EMB_F, dict(tok=None)),
    ("chgnet_embed_forward", EMB_F, dict(table=None)),
    ("chgnet_embed_forward", EMB_F, dict(out=None)),
    ("chgnet_embed_forward", EMB_F, dict(tok=P + 2)),
    ("chgnet_embed_backward", EMB_B, dict(n=-1)),
    ("chgnet_embed_backward", EMB_B, dict(n=(1 << 30) + 1)),
    ("chgnet_embed_backward", EMB_B, dict(d=0)),
    ("chgnet_embed_backward", EMB_B, dict(vocab=-3)),
    ("chgnet_embed_backward", EMB_B, dict(lddout=63)),
    ("chgnet_embed_backward", EMB_B, dict(lddtable=63)),
    ("chgnet_embed_backward", EMB_B, dict(tok=None)),
    ("chgnet_embed_backward", EMB_B, dict(dout=None)),
    ("chgnet_embed_backward", EMB_B, dict(dtable=None)),
    ("chgnet_embed_backward", EMB_B, dict(n=0, dtable=None)),
    ("chgnet_embed_backward", EMB_B, dict(dtable=P + 2)),
    ("chgnet_embed_backward", EMB_B, dict(ws=P + 4)),
]


@pytest.mark.parametrize("fn,base,kw", BAD)
def test_bad_arguments(fn, base, kw):
    assert _call(fn, base, **kw) == bd.CHGNET_EINVAL
    assert fn[len("chgnet_"):].encode() in bd.lib().chgnet_last_error_string()


@pytest.mark.parametrize("fn,base,kw", [
    ("chgnet_gate_backward", GATE_B, dict(ws=None)),
    ("chgnet_gate_backward", GATE_B, dict(ws_bytes=4 * 4 * 64 - 1)),
    ("chgnet_embed_backward", EMB_B, dict(ws=None)),
    ("chgnet_embed_backward", EMB_B, dict(ws_bytes=1 << 16)),
])
def test_small_workspace(fn, base, kw):
    assert _call(fn, base, **kw) == bd.CHGNET_EWORKSPACE


def test_no_rows_need_no_arrays():
    assert _call("chgnet_gate_forward", GATE_F, rows=0, z=None, ln=None, phi=None, codes=None, step=None) == bd.CHGNET_OK
    assert _call("chgnet_gate_backward", GATE_B, rows=0, codes=None, step=None, ln=None, dphi=None, dz=None, ws=None,
                 ws_bytes=0, accumulate=1) == bd.CHGNET_OK
    assert _call("chgnet_embed_forward", EMB_F, n=0, tok=None, table=None, out=None) == bd.CHGNET_OK
    assert _call("chgnet_embed_backward", EMB_B, n=0, tok=None, dout=None, ws=None, ws_bytes=0,
                 accumulate=1) == bd.CHGNET_OK


def test_workspace_sizes():
    n = ctypes.c_size_t()
    f = ops.lib().chgnet_gate_backward_workspace
    last = 0
    for rows in (0, 1, 8, 9, 1000, 4096, 10 ** 9):
        assert f(rows, 128, ctypes.byref(n)) == bd.CHGNET_OK and n.value >= last
        last = n.value
    assert 0 < last <= 512 * 4 * 128 * 4
    assert f(-1, 128, ctypes.byref(n)) == f(8, 0, ctypes.byref(n)) == f(8, 64, None) == bd.CHGNET_EINVAL
    g = ops.lib().chgnet_embed_backward_workspace
    for tokens in (0, 1, 5000, 10 ** 6, 1 << 30):
        assert g(tokens, 128, 94, ctypes.byref(n)) == bd.CHGNET_OK
    assert n.value >= 16 << 30
    for bad in ((-1, 128, 94), ((1 << 30) + 1, 128, 94), (8, 0, 94), (8, 128, 0)):
        assert g(*bad, ctypes.byref(n)) == bd.CHGNET_EINVAL
    assert g(8, 128, 94, None) == bd.CHGNET_EINVAL


def test_header_library_and_binding_agree():
    src = open(os.path.join(ROOT, "include", "chgnet_ops.h")).read()
    names = set(re.findall(r"^int\s+(chgnet_\w+)\s*\(", src, re.M))
    assert names == set(ops.EXPORTED)
    lib = ctypes.CDLL(bd._LIB_PATH)
    assert all(hasattr(lib, n) for n in names)


def test_host_tensors_are_refused():
    z, ln, tok = torch.zeros(4, 128), torch.zeros(4, 64), torch.zeros(4, dtype=torch.int32)
    kept = ops.GateCheckpoint.empty(4, 64, "cpu")
    for call in (lambda: ops.gate_forward(z, ln), lambda: ops.gate_backward(kept, ln, torch.zeros(4, 64)),
                 lambda: ops.embed_forward(ln, tok), lambda: ops.embed_backward(tok, ln, 94)):
        with pytest.raises(bd.ChgnetError) as e:
            call()
        assert e.value.code == bd.CHGNET_EINVAL and "GPU" in str(e.value)
