"""Thin ctypes binding of the operators in include/chgnet_ops.h: the gate of the
gated MLP with an 8-bit checkpoint of its input, and the scaled embedding lookup
with its gradient.

Argument marshalling and checks only, as in ``binding``: torch tensors supply
device memory and the stream (the current one of the tensors' device), and a
missing library raises. Every tensor of a call is on one GPU; rows may have a
stride, columns are contiguous. Inputs are not differentiated by autograd: a
``torch.autograd.Function`` of the caller's calls the two passes.
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass

import torch

from . import binding as bd

EXPORTED = ("chgnet_gate_forward", "chgnet_gate_backward_workspace", "chgnet_gate_backward", "chgnet_embed_forward",
            "chgnet_embed_backward_workspace", "chgnet_embed_backward")
DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_lib = None


def lib():
    global _lib
    if _lib is None:
        L = bd.lib()
        vp, i64, i32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t
        L.chgnet_gate_forward.argtypes = [i64, i32, i32, vp, i64, vp, vp, i64, vp, vp, vp]
        L.chgnet_gate_backward_workspace.argtypes = [i64, i32, ctypes.POINTER(sz)]
        L.chgnet_gate_backward.argtypes = [i64, i32, i32, vp, vp, vp, vp, i64, vp, i64, vp, ctypes.c_int, vp, sz, vp]
        L.chgnet_embed_forward.argtypes = [i64, i32, i64, i32, vp, i32, vp, i64, ctypes.c_float, vp, i64, vp]
        L.chgnet_embed_backward_workspace.argtypes = [i64, i32, i64, ctypes.POINTER(sz)]
        L.chgnet_embed_backward.argtypes = [i64, i32, i64, i32, vp, i32, vp, i64, ctypes.c_float, vp, i64,
                                            ctypes.c_int, vp, sz, vp]
        for name in EXPORTED:
            getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def _bad(msg):
    raise bd.ChgnetError(bd.CHGNET_EINVAL, msg)


def _matrix(name, t, rows, cols, dtypes, device):
    """Row stride of a [rows, cols] tensor of one of `dtypes` on `device`."""
    if t.dim() != 2 or t.dtype not in dtypes or t.device != device or tuple(t.shape) != (rows, cols):
        _bad("%s must be [%d, %d] of %s on %s, not %s %s on %s"
             % (name, rows, cols, " or ".join(map(str, dtypes)), device, list(t.shape), t.dtype, t.device))
    if cols > 1 and t.stride(1) != 1:
        _bad("%s must have contiguous columns" % name)
    ld = t.stride(0) if rows > 1 else max(cols, t.stride(0))
    if ld < cols:
        _bad("%s has overlapping rows" % name)
    return ld


def _packed(name, t, shape, dtype, device):
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype or t.device != device or not t.is_contiguous():
        _bad("%s must be contiguous %s of %s on %s, not %s %s on %s"
             % (name, list(shape), dtype, device, list(t.shape), t.dtype, t.device))


def _gpu(name, t):
    if not t.is_cuda:
        _bad("%s must be on a GPU" % name)
    return t.device


class _On:
    """The tensors' device as the current one for a call, and its current stream."""

    def __init__(self, device):
        self.index = device.index

    def __enter__(self):
        self.before = torch.cuda.current_device()
        if self.before != self.index:
            torch.cuda.set_device(self.index)
        return torch.cuda.current_stream(self.index).cuda_stream

    def __exit__(self, *exc):
        if self.before != self.index:
            torch.cuda.set_device(self.before)


def _workspace(ws, nbytes, device):
    """(pointer, size, owner) of the caller's Workspace grown to nbytes, or of memory for this call."""
    if ws is not None:
        if torch.device(ws.device).type != "cuda" or ws.ensure(nbytes).device != device:
            _bad("the workspace must be on %s" % device)
        return ws.buf.data_ptr(), ws.nbytes, ws
    buf = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=device)
    return buf.data_ptr(), buf.numel(), buf


@dataclass
class GateCheckpoint:
    """8-bit checkpoint of a gate's input: codes [rows, 2d] uint8 and step [rows, 2] fp32 (core, gate)."""
    codes: torch.Tensor
    step: torch.Tensor

    @classmethod
    def empty(cls, rows, d, device="cuda"):
        return cls(torch.empty(rows, 2 * d, dtype=torch.uint8, device=device),
                   torch.empty(rows, 2, dtype=torch.float32, device=device))

    @property
    def nbytes(self):
        return self.codes.numel() + 4 * self.step.numel()


def gate_forward(z, ln, save=True, phi=None, kept=None):
    """phi [rows, d] of z [rows, 2d] (core | gate) and ln [4, d] fp32 (g_c, b_c, g_g, b_g); z in fp32, bf16 or fp16.
    With `save` returns (phi, GateCheckpoint) for gate_backward, else phi. phi and kept: tensors to write into."""
    if z.dim() != 2 or z.shape[1] % 2 or z.shape[1] == 0 or z.dtype not in DTYPES:
        _bad("z must be [rows, 2d] in fp32, bf16 or fp16, not %s %s" % (list(z.shape), z.dtype))
    dev = _gpu("z", z)
    rows, d = z.shape[0], z.shape[1] // 2
    ldz = _matrix("z", z, rows, 2 * d, (z.dtype,), dev)
    _packed("ln", ln, (4, d), torch.float32, dev)
    if phi is None:
        phi = torch.empty(rows, d, dtype=z.dtype, device=dev)
    ldp = _matrix("phi", phi, rows, d, (z.dtype,), dev)
    if not save:
        if kept is not None:
            _bad("a checkpoint is given but not to be kept")
    elif kept is None:
        kept = GateCheckpoint.empty(rows, d, dev)
    else:
        _packed("kept.codes", kept.codes, (rows, 2 * d), torch.uint8, dev)
        _packed("kept.step", kept.step, (rows, 2), torch.float32, dev)
    with _On(dev) as stream:
        bd._check(lib().chgnet_gate_forward(rows, d, DTYPES[z.dtype], z.data_ptr(), ldz, ln.data_ptr(), phi.data_ptr(),
                                            ldp, kept.codes.data_ptr() or None if save else None,
                                            kept.step.data_ptr() or None if save else None, stream))
    return (phi, kept) if save else phi


def gate_backward(kept, ln, dphi, dz=None, dln=None, accumulate=False, ws=None):
    """(dz [rows, 2d], dln [4, d]) from the checkpoint of gate_forward and dphi [rows, d]; dln is fp32 and added to what
    it holds with `accumulate`. ws: a Workspace of the caller's (one for each call that may run at the same time)."""
    if dphi.dim() != 2 or dphi.dtype not in DTYPES:
        _bad("dphi must be [rows, d] in fp32, bf16 or fp16, not %s %s" % (list(dphi.shape), dphi.dtype))
    dev = _gpu("dphi", dphi)
    rows, d = dphi.shape
    ldp = _matrix("dphi", dphi, rows, d, (dphi.dtype,), dev)
    _packed("kept.codes", kept.codes, (rows, 2 * d), torch.uint8, dev)
    _packed("kept.step", kept.step, (rows, 2), torch.float32, dev)
    _packed("ln", ln, (4, d), torch.float32, dev)
    if dz is None:
        dz = torch.empty(rows, 2 * d, dtype=dphi.dtype, device=dev)
    ldz = _matrix("dz", dz, rows, 2 * d, (dphi.dtype,), dev)
    if dln is None:
        if accumulate:
            _bad("accumulate needs a dln to add to")
        dln = torch.empty(4, d, dtype=torch.float32, device=dev)
    _packed("dln", dln, (4, d), torch.float32, dev)
    need = ctypes.c_size_t()
    bd._check(lib().chgnet_gate_backward_workspace(rows, d, ctypes.byref(need)))
    with _On(dev) as stream:
        p, nbytes, _keep = _workspace(ws, need.value, dev)
        bd._check(lib().chgnet_gate_backward(rows, d, DTYPES[dphi.dtype], kept.codes.data_ptr(), kept.step.data_ptr(),
                                             ln.data_ptr(), dphi.data_ptr(), ldp, dz.data_ptr(), ldz, dln.data_ptr(),
                                             int(accumulate), p, nbytes, stream))
    return dz, dln


def embed_forward(table, tok, scale=1.0, first=0, out=None):
    """out [n, d] = scale * table[tok - first] for int32 tokens [n]; zeros for tokens outside the table [vocab, d]."""
    if table.dim() != 2 or table.dtype not in DTYPES:
        _bad("table must be [vocab, d] in fp32, bf16 or fp16, not %s %s" % (list(table.shape), table.dtype))
    dev = _gpu("table", table)
    vocab, d = table.shape
    ldt = _matrix("table", table, vocab, d, (table.dtype,), dev)
    n = tok.numel()
    _packed("tok", tok, (n,), torch.int32, dev)
    if out is None:
        out = torch.empty(n, d, dtype=table.dtype, device=dev)
    ldo = _matrix("out", out, n, d, (table.dtype,), dev)
    with _On(dev) as stream:
        bd._check(lib().chgnet_embed_forward(n, d, vocab, DTYPES[table.dtype], tok.data_ptr(), first, table.data_ptr(),
                                             ldt, scale, out.data_ptr(), ldo, stream))
    return out


def embed_backward(tok, dout, vocab, scale=1.0, first=0, dtable=None, accumulate=False, ws=None):
    """dtable [vocab, d] fp32: row v = scale * the sum of dout [n, d] over the tokens with tok - first = v, added to what
    it holds with `accumulate`. ws: a Workspace of the caller's (one for each call that may run at the same time)."""
    if dout.dim() != 2 or dout.dtype not in DTYPES:
        _bad("dout must be [n, d] in fp32, bf16 or fp16, not %s %s" % (list(dout.shape), dout.dtype))
    dev = _gpu("dout", dout)
    if vocab < 1:
        _bad("vocab must be at least 1")
    n, d = dout.shape
    ldo = _matrix("dout", dout, n, d, (dout.dtype,), dev)
    _packed("tok", tok, (n,), torch.int32, dev)
    if dtable is None:
        if accumulate:
            _bad("accumulate needs a dtable to add to")
        dtable = torch.empty(vocab, d, dtype=torch.float32, device=dev)
    ldw = _matrix("dtable", dtable, vocab, d, (torch.float32,), dev)
    need = ctypes.c_size_t()
    bd._check(lib().chgnet_embed_backward_workspace(n, d, vocab, ctypes.byref(need)))
    with _On(dev) as stream:
        p, nbytes, _keep = _workspace(ws, need.value, dev)
        bd._check(lib().chgnet_embed_backward(n, d, vocab, DTYPES[dout.dtype], tok.data_ptr(), first, dout.data_ptr(),
                                              ldo, scale, dtable.data_ptr(), ldw, int(accumulate), p, nbytes, stream))
    return dtable
