"""What the 8-bit matrices and their products refuse, and their workspace sizes (no GPU: every call here ends in its checks)."""
import ctypes

import pytest
import torch

from paper_2412_20796_amd import binding as bd
from paper_2412_20796_amd import ops

P = 1 << 20  # an address that is aligned and never read: the calls below are refused before any launch
A = dict(rows=8, cols=200, codes=P, ld=208, scale=P, ld_scale=4, block_rows=1)
B = dict(A, rows=9, block_rows=128)
T = dict(rows=200, cols=8, codes=P, ld=16, scale=P, ld_scale=4, block_rows=1)
QUANT = dict(rows=8, cols=200, dtype=0, x=P, ldx=200, q=A, t=T, stream=None)
MUL = dict(a=A, b=B, dtype=0, out=P, ldout=9, accumulate=0, ws=None, ws_bytes=0, stream=None)
LIN = dict(rows=100, dtype=1, x=P, ldx=200, w=B, out=P, ldout=9, ws=P, ws_bytes=1 << 20, stream=None)


def _call(fn, base, **kw):
    a = {k: dict(v) if isinstance(v, dict) else v for k, v in base.items()}
    for k, v in kw.items():
        if "_" in k and k.split("_", 1)[0] in "abqtw" and isinstance(a[k[0]], dict):
            assert k[2:] in a[k[0]], k
            a[k[0]][k[2:]] = v
        else:
            assert k in a, k
            a[k] = v
    held = []
    for k, v in a.items():
        if isinstance(v, dict):
            held.append(ops._Fp8(**v))
            a[k] = ctypes.addressof(held[-1])
    return getattr(ops.lib(), fn)(*a.values())


BAD = ([("chgnet_fp8_quantize", QUANT, k) for k in (
            dict(rows=-1), dict(cols=-1), dict(rows=(1 << 23) + 1), dict(cols=(1 << 23) + 1), dict(dtype=3), dict(ldx=199),
            dict(q=None, t=None), dict(x=None), dict(x=P + 2), dict(q_rows=7), dict(q_cols=199), dict(t_rows=199),
            dict(t_cols=9), dict(q_codes=None), dict(q_scale=None), dict(t_codes=None), dict(q_codes=P + 8), dict(q_scale=P + 2),
            dict(q_ld=200), dict(q_ld=192), dict(q_ld_scale=2), dict(q_ld_scale=6), dict(t_ld=0), dict(q_block_rows=2),
            dict(t_block_rows=128))]
       + [("chgnet_fp8_matmul", MUL, k) for k in (
            dict(a=None), dict(b=None), dict(dtype=7), dict(ldout=8), dict(out=None), dict(out=P + 2), dict(a_cols=199),
            dict(b_cols=201), dict(a_rows=-1), dict(b_rows=1 << 31), dict(a_codes=None), dict(b_scale=None),
            dict(a_codes=P + 4), dict(b_scale=P + 1), dict(a_ld=200), dict(b_ld=100), dict(a_ld_scale=0), dict(b_ld_scale=3),
            dict(a_block_rows=0), dict(b_block_rows=64), dict(a_cols=(1 << 23) + 1, b_cols=(1 << 23) + 1), dict(ws=P + 8))]
       + [("chgnet_fp8_linear", LIN, k) for k in (
            dict(rows=-1), dict(rows=(1 << 23) + 1), dict(dtype=-1), dict(w=None), dict(ldx=199), dict(ldout=8), dict(x=None),
            dict(out=None), dict(x=P + 1), dict(out=P + 1), dict(w_codes=None), dict(w_ld=200), dict(w_block_rows=3),
            dict(ws=P + 8))])


@pytest.mark.parametrize("fn,base,kw", BAD)
def test_bad_arguments(fn, base, kw):
    assert _call(fn, base, **kw) == bd.CHGNET_EINVAL
    assert fn[len("chgnet_"):].encode() in bd.lib().chgnet_last_error_string()


def test_small_workspace():
    assert _call("chgnet_fp8_linear", LIN, rows=300, ws_bytes=100) == bd.CHGNET_EWORKSPACE
    assert _call("chgnet_fp8_linear", LIN, rows=300, ws=None) == bd.CHGNET_EWORKSPACE
    long = dict(a_rows=100, a_cols=1 << 20, a_ld=1 << 20, a_ld_scale=1 << 13, b_cols=1 << 20, b_ld=1 << 20, b_ld_scale=1 << 13)
    assert _call("chgnet_fp8_matmul", MUL, **long) == bd.CHGNET_EWORKSPACE


def test_no_rows_need_no_arrays():
    assert _call("chgnet_fp8_quantize", QUANT, rows=0, x=None, q_rows=0, t_cols=0, q_codes=None, q_scale=None) == bd.CHGNET_OK
    assert _call("chgnet_fp8_matmul", MUL, a_rows=0, a_codes=None, a_scale=None, out=None) == bd.CHGNET_OK
    assert _call("chgnet_fp8_matmul", MUL, b_rows=0, b_codes=None, b_scale=None, out=None) == bd.CHGNET_OK
    assert _call("chgnet_fp8_linear", LIN, rows=0, x=None, out=None, ws=None, ws_bytes=0) == bd.CHGNET_OK


def test_workspace_sizes():
    n = ctypes.c_size_t()
    for name in ("chgnet_fp8_matmul_workspace", "chgnet_fp8_linear_workspace"):
        f = getattr(ops.lib(), name)
        for m, k, cols in ((0, 5, 5), (5, 0, 5), (5, 5, 0), (1, 1, 1), (100, 300, 1 << 23), (1 << 20, 1 << 20, 128)):
            assert f(m, k, cols, ctypes.byref(n)) == bd.CHGNET_OK, (m, k, cols)
        for bad in ((-1, 5, 5), (5, -1, 5), (5, 5, -1), (5, 5, (1 << 23) + 1), (1 << 31, 5, 5), (5, 1 << 31, 5)):
            assert f(*bad, ctypes.byref(n)) == bd.CHGNET_EINVAL
        assert f(5, 5, 5, None) == bd.CHGNET_EINVAL


def test_host_tensors_and_inputs_that_autograd_follows_are_refused():
    x = torch.zeros(4, 64)
    m = ops.Fp8Matrix(torch.zeros(8, 64).to(torch.float8_e4m3fn), torch.zeros(8, 4, dtype=torch.uint8).view(
        torch.float8_e8m0fnu)[:, :1])
    follow = lambda t: t.clone().requires_grad_(True)
    for call in (lambda g: ops.fp8_quantize(g(x)), lambda g: ops.fp8_quantize_both(g(x)), lambda g: ops.fp8_linear(g(x), m)):
        for g, word in ((follow, "gradient"), (lambda t: t, "GPU")):
            with pytest.raises(bd.ChgnetError) as e:
                call(g)
            assert e.value.code == bd.CHGNET_EINVAL and word in str(e.value)
    with pytest.raises(bd.ChgnetError) as e:
        ops.fp8_matmul(m, m)
    assert e.value.code == bd.CHGNET_EINVAL and "GPU" in str(e.value)
