"""Thin ctypes binding of the operators in include/chgnet_ops.h: the gate of the
gated MLP with an 8-bit checkpoint of its input, the scaled embedding lookup with
its gradient, norms and the residual connection around a block with its gate and
dropout.

Argument marshalling and checks only, as in ``binding``: torch tensors supply
device memory and the stream (the current one of the tensors' device), and a
missing library raises. Every tensor of a call is on one GPU; rows may have a
stride, columns are contiguous. Inputs are not differentiated by autograd: a
``torch.autograd.Function`` of the caller's calls the two passes. An input that
autograd follows (it requires a gradient, outside ``torch.no_grad()`` and such a
Function) is refused, since its gradient would be lost.

The calls on few rows take as long as their launches, about 4 us each; the checks
are written so that they add little to that (a dozen attribute reads).
"""
from __future__ import annotations

import ctypes
from collections import namedtuple
from functools import lru_cache

import torch

from . import binding as bd

EXPORTED = ("chgnet_gate_forward", "chgnet_gate_backward_workspace", "chgnet_gate_backward", "chgnet_embed_forward",
            "chgnet_embed_backward_workspace", "chgnet_embed_backward", "chgnet_norm_forward", "chgnet_norm_backward",
            "chgnet_residual_forward", "chgnet_residual_backward_workspace", "chgnet_residual_backward", "chgnet_dropout")
# (torch.cuda.current_stream and current_device, without the objects and checks around them: 1.3 us a call)
_raw_stream, _current_gpu = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
NORMS = {"none": 0, "rms": 1, "layer": 2}
DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_lib = None


class _Residual(ctypes.Structure):
    """chgnet_residual"""

    _fields_ = ([(n, ctypes.c_int32) for n in ("post_kind", "post_rows", "pre_kind", "pre_rows", "gate_cols")]
                + [(n, ctypes.c_float) for n in ("alpha", "beta", "eps", "p")]
                + [("seed", ctypes.c_uint64), ("call", ctypes.c_uint64), ("step", ctypes.c_void_p)])


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
        f32, u64, cint = ctypes.c_float, ctypes.c_uint64, ctypes.c_int
        L.chgnet_norm_forward.argtypes = [i64, i32, i32, vp, i64, i32, vp, i32, f32, vp, i64, vp]
        L.chgnet_norm_backward.argtypes = [i64, i32, i32, vp, i64, i32, vp, i32, f32, vp, i64, vp, i64, vp, cint, vp, sz, vp]
        L.chgnet_residual_forward.argtypes = [i64, i32, i32, vp, vp, i64, vp, i64, vp, i64, vp, vp, vp, i64, vp, i64, vp]
        L.chgnet_residual_backward_workspace.argtypes = [i64, i32, i32, ctypes.POINTER(sz)]
        L.chgnet_residual_backward.argtypes = [i64, i32, i32, vp, vp, i64, vp, i64, vp, i64, vp, vp, vp, i64, vp, i64, vp, i64,
                                               vp, i64, vp, i64, vp, vp, cint, vp, sz, vp]
        L.chgnet_dropout.argtypes = [i64, i32, i32, vp, i64, f32, u64, u64, vp, vp, i64, vp]
        for name in EXPORTED:
            getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def _bad(msg):
    raise bd.ChgnetError(bd.CHGNET_EINVAL, msg)


def _wrong(name, t, shape, what, gpu):
    _bad("%s must be %s of %s on GPU %d, not %s %s on %s" % (name, list(shape), what, gpu, list(t.shape), t.dtype, t.device))


def _rows(name, t, rows, cols, dtype, gpu):
    """Row stride of a [rows, cols] tensor of `dtype` on GPU `gpu`."""
    if t.dtype is not dtype or t.get_device() != gpu or t.shape != (rows, cols):
        _wrong(name, t, (rows, cols), dtype, gpu)
    return _stride(name, t, rows, cols)


def _stride(name, t, rows, cols):
    ld, step = t.stride()
    if step != 1 and cols > 1:
        _bad("%s must have contiguous columns" % name)
    if ld < cols:
        if rows > 1:
            _bad("%s has overlapping rows" % name)
        ld = cols
    return ld


def _packed(name, t, shape, dtype, gpu):
    if t.dtype is not dtype or t.get_device() != gpu or t.shape != shape or not t.is_contiguous():
        _wrong(name, t, shape, "contiguous %s" % dtype, gpu)


def _start(name, t):
    """(rows, columns, type, type code, row stride, GPU) of a call's first tensor."""
    dtype, shape = t.dtype, t.shape
    code = DTYPES.get(dtype)
    if code is None or len(shape) != 2:
        _bad("%s must be a matrix of fp32, bf16 or fp16, not %s %s" % (name, list(shape), dtype))
    gpu = t.get_device()
    if gpu < 0:
        _bad("%s must be on a GPU" % name)
    rows, cols = shape
    return rows, cols, dtype, code, _stride(name, t, rows, cols), gpu


def _followed(name):
    _bad("%s requires a gradient, which this call does not pass on: call it from a torch.autograd.Function or under "
         "torch.no_grad()" % name)


def _first(first):
    if not 0 <= first < 1 << 31:  # (ctypes would keep the low bits)
        _bad("first must be in 0 .. 2^31 - 1")


def _call(fn, gpu, args):
    """The call on the GPU's current stream, with the GPU as the current device."""
    if _current_gpu() == gpu:
        code = fn(*args, _raw_stream(gpu))
    else:
        with torch.cuda.device(gpu):
            code = fn(*args, _raw_stream(gpu))
    if code:
        bd._check(code)


@lru_cache(maxsize=4096)
def _gate_bytes(rows, d):
    need = ctypes.c_size_t()
    bd._check(lib().chgnet_gate_backward_workspace(rows, d, ctypes.byref(need)))
    return need.value


@lru_cache(maxsize=4096)
def _embed_bytes(n, d, vocab):
    need = ctypes.c_size_t()
    bd._check(lib().chgnet_embed_backward_workspace(n, d, vocab, ctypes.byref(need)))
    return need.value


def _workspace(ws, nbytes, gpu, like):
    """(pointer, size, owner) of the caller's Workspace grown to nbytes, or of memory for this call."""
    if ws is None:
        buf = torch.empty(nbytes or 1, dtype=torch.uint8, device=like.device)
    else:
        buf = ws.ensure(nbytes)
        if buf.get_device() != gpu:
            _bad("the workspace must be on GPU %d" % gpu)
    return buf.data_ptr(), buf.numel(), buf


class GateCheckpoint:
    """8-bit checkpoint of a gate's input: codes [rows, 2d] uint8 and step [rows, 2] fp32 (core, gate), two tensors of the
    caller's or views of one allocation (`empty`)."""

    __slots__ = ("_codes", "_step", "_data", "_rows", "_d")

    def __init__(self, codes, step):
        self._codes, self._step, self._data = codes, step, None

    @classmethod
    def empty(cls, rows, d, device="cuda"):
        self = cls(None, None)
        self._data = torch.empty(rows * (2 * d + 8), dtype=torch.uint8, device=device)
        self._rows, self._d = rows, d
        return self

    @property
    def codes(self):
        if self._codes is None:
            self._codes = self._data[8 * self._rows:].view(self._rows, 2 * self._d)
        return self._codes

    @property
    def step(self):
        if self._step is None:
            self._step = self._data[:8 * self._rows].view(torch.float32).view(self._rows, 2)
        return self._step

    @property
    def nbytes(self):
        return self.codes.numel() + 4 * self.step.numel()

    def _pointers(self, rows, d, gpu):
        """(codes, step) addresses of a checkpoint of [rows, 2d] on GPU `gpu`."""
        t = self._data
        if t is not None:
            if self._rows != rows or self._d != d or t.get_device() != gpu:
                _bad("the checkpoint is of [%d, %d] on %s, not of [%d, %d] on GPU %d"
                     % (self._rows, 2 * self._d, t.device, rows, 2 * d, gpu))
            p = t.data_ptr()
            return (p + 8 * rows, p) if rows else (None, None)
        _packed("kept.codes", self._codes, (rows, 2 * d), torch.uint8, gpu)
        _packed("kept.step", self._step, (rows, 2), torch.float32, gpu)
        return self._codes.data_ptr() or None, self._step.data_ptr() or None


def gate_forward(z, ln, save=True, phi=None, kept=None):
    """phi [rows, d] of z [rows, 2d] (core | gate) and ln [4, d] fp32 (g_c, b_c, g_g, b_g); z in fp32, bf16 or fp16.
    With `save` returns (phi, GateCheckpoint) for gate_backward, else phi. phi and kept: tensors to write into."""
    if (z.requires_grad or ln.requires_grad) and torch.is_grad_enabled():
        _followed("z or ln")
    rows, cols, dtype, code, ldz, gpu = _start("z", z)
    d = cols // 2
    if cols != 2 * d:
        _bad("z must have an even number of columns, core | gate")
    _packed("ln", ln, (4, d), torch.float32, gpu)
    if phi is None:
        phi, ldp = torch.empty((rows, d), dtype=dtype, device=z.device), d
    else:
        ldp = _rows("phi", phi, rows, d, dtype, gpu)
    if not save:
        if kept is not None:
            _bad("a checkpoint is given but not to be kept")
        _call(lib().chgnet_gate_forward, gpu, (rows, d, code, z.data_ptr(), ldz, ln.data_ptr(), phi.data_ptr(), ldp,
                                               None, None))
        return phi
    if kept is None:
        kept = GateCheckpoint.empty(rows, d, z.device)
    _call(lib().chgnet_gate_forward, gpu, (rows, d, code, z.data_ptr(), ldz, ln.data_ptr(), phi.data_ptr(), ldp,
                                           *kept._pointers(rows, d, gpu)))
    return phi, kept


def gate_backward(kept, ln, dphi, dz=None, dln=None, accumulate=False, ws=None):
    """(dz [rows, 2d], dln [4, d]) from the checkpoint of gate_forward and dphi [rows, d]; dln is fp32 and added to what
    it holds with `accumulate`. ws: a Workspace of the caller's (one for each call that may run at the same time)."""
    if (dphi.requires_grad or ln.requires_grad) and torch.is_grad_enabled():
        _followed("dphi or ln")
    rows, d, dtype, code, ldp, gpu = _start("dphi", dphi)
    codes, step = kept._pointers(rows, d, gpu)
    _packed("ln", ln, (4, d), torch.float32, gpu)
    if dz is None:
        dz, ldz = torch.empty((rows, 2 * d), dtype=dtype, device=dphi.device), 2 * d
    else:
        ldz = _rows("dz", dz, rows, 2 * d, dtype, gpu)
    if dln is None:
        if accumulate:
            _bad("accumulate needs a dln to add to")
        dln = torch.empty((4, d), dtype=torch.float32, device=dphi.device)
    else:
        _packed("dln", dln, (4, d), torch.float32, gpu)
    p, nbytes, _keep = _workspace(ws, _gate_bytes(rows, d), gpu, dphi)
    _call(lib().chgnet_gate_backward, gpu, (rows, d, code, codes, step, ln.data_ptr(), dphi.data_ptr(), ldp,
                                            dz.data_ptr(), ldz, dln.data_ptr(), bool(accumulate), p, nbytes))
    return dz, dln


def embed_forward(table, tok, scale=1.0, first=0, out=None):
    """out [n, d] = scale * table[tok - first] for int32 tokens [n]; zeros for tokens outside the table [vocab, d]."""
    if table.requires_grad and torch.is_grad_enabled():
        _followed("table")
    vocab, d, dtype, code, ldt, gpu = _start("table", table)
    n = tok.numel()
    _packed("tok", tok, (n,), torch.int32, gpu)
    _first(first)
    if out is None:
        out, ldo = torch.empty((n, d), dtype=dtype, device=table.device), d
    else:
        ldo = _rows("out", out, n, d, dtype, gpu)
    _call(lib().chgnet_embed_forward, gpu, (n, d, vocab, code, tok.data_ptr(), first, table.data_ptr(), ldt, scale,
                                            out.data_ptr(), ldo))
    return out


def embed_backward(tok, dout, vocab, scale=1.0, first=0, dtable=None, accumulate=False, ws=None):
    """dtable [vocab, d] fp32: row v = scale * the sum of dout [n, d] over the tokens with tok - first = v, added to what
    it holds with `accumulate`. ws: a Workspace of the caller's (one for each call that may run at the same time)."""
    if dout.requires_grad and torch.is_grad_enabled():
        _followed("dout")
    n, d, _, code, ldo, gpu = _start("dout", dout)
    if vocab < 1:
        _bad("vocab must be at least 1")
    _packed("tok", tok, (n,), torch.int32, gpu)
    _first(first)
    if dtable is None:
        if accumulate:
            _bad("accumulate needs a dtable to add to")
        dtable, ldw = torch.empty((vocab, d), dtype=torch.float32, device=dout.device), d
    else:
        ldw = _rows("dtable", dtable, vocab, d, torch.float32, gpu)
    need = _embed_bytes(n, d, vocab)
    p, nbytes, _keep = _workspace(ws, need, gpu, dout) if need else (None, 0, None)
    _call(lib().chgnet_embed_backward, gpu, (n, d, vocab, code, tok.data_ptr(), first, dout.data_ptr(), ldo, scale,
                                             dtable.data_ptr(), ldw, bool(accumulate), p, nbytes))
    return dtable


@lru_cache(maxsize=4096)
def _residual_bytes(rows, d, param_rows):
    need = ctypes.c_size_t()
    bd._check(lib().chgnet_residual_backward_workspace(rows, d, param_rows, ctypes.byref(need)))
    return need.value


def _params(name, w, d, gpu):
    """Rows of a norm's fp32 parameters [1, d] (scale) or [2, d] (scale, shift)."""
    if w.dim() != 2 or w.shape[0] not in (1, 2):
        _bad("%s must be [1, %d] (scale) or [2, %d] (scale, shift), not %s" % (name, d, d, list(w.shape)))
    _packed(name, w, (w.shape[0], d), torch.float32, gpu)
    return w.shape[0]


def _norm_kind(kind):
    if kind not in NORMS:
        _bad("unknown norm %r: one of %s" % (kind, ", ".join(NORMS)))
    return NORMS[kind]


def _like(name, out, rows, cols, dtype, gpu, like):
    """(tensor, row stride) of a call's output: the caller's or a new one."""
    if out is None:
        return torch.empty((rows, cols), dtype=dtype, device=like.device), cols
    return out, _rows(name, out, rows, cols, dtype, gpu)


def _param_grad(name, out, w, accumulate, gpu):
    if out is None:
        if accumulate:
            _bad("accumulate needs a %s to add to" % name)
        return torch.empty_like(w)
    _packed(name, out, w.shape, torch.float32, gpu)
    return out


def _draw(seed, call, step, gpu):
    """Address of `step`; seed and call are checked (ctypes would keep the low bits)."""
    if not (0 <= seed < 1 << 64 and 0 <= call < 1 << 64):
        _bad("seed and call must be in 0 .. 2^64 - 1")
    if step is None:
        return None
    _packed("step", step, (1,), torch.int64, gpu)
    return step.data_ptr()


def dropout(x, p, seed, call=0, step=None, out=None):
    """x [rows, d] / (1 - p) where the counter-based generator keeps a value, else 0 (p counts in steps of 2^-16). The mask
    is that of (seed, call + step) whatever the type and strides, and is not stored: the same call on the upstream gradient is
    the backward pass. step: int64 [1] on the GPU, for graphs whose replays draw anew."""
    if x.requires_grad and torch.is_grad_enabled():
        _followed("x")
    rows, d, dtype, code, ldx, gpu = _start("x", x)
    at = _draw(seed, call, step, gpu)
    out, ldo = _like("out", out, rows, d, dtype, gpu, x)
    _call(lib().chgnet_dropout, gpu, (rows, d, code, x.data_ptr(), ldx, p, seed, call, at, out.data_ptr(), ldo))
    return out


def norm_forward(x, w, kind="rms", eps=1e-5, h=None):
    """h [rows, d] = w[0] n(x) + w[1] with n the RMS norm ("rms") or the LayerNorm ("layer") of each row; w fp32 [1, d] (no
    shift) or [2, d]; x in fp32, bf16 or fp16."""
    if (x.requires_grad or w.requires_grad) and torch.is_grad_enabled():
        _followed("x or w")
    rows, d, dtype, code, ldx, gpu = _start("x", x)
    n = _params("w", w, d, gpu)
    h, ldh = _like("h", h, rows, d, dtype, gpu, x)
    _call(lib().chgnet_norm_forward, gpu, (rows, d, code, x.data_ptr(), ldx, _norm_kind(kind), w.data_ptr(), n, eps,
                                           h.data_ptr(), ldh))
    return h


def norm_backward(x, w, dh, kind="rms", eps=1e-5, dx=None, dw=None, accumulate=False, ws=None):
    """(dx [rows, d], dw like w) of norm_forward from dh [rows, d]; dw is fp32 and added to what it holds with `accumulate`.
    ws: a Workspace of the caller's (one for each call that may run at the same time)."""
    if (x.requires_grad or w.requires_grad or dh.requires_grad) and torch.is_grad_enabled():
        _followed("x, w or dh")
    rows, d, dtype, code, ldx, gpu = _start("x", x)
    n = _params("w", w, d, gpu)
    ldu = _rows("dh", dh, rows, d, dtype, gpu)
    dx, ldd = _like("dx", dx, rows, d, dtype, gpu, x)
    dw = _param_grad("dw", dw, w, accumulate, gpu)
    p, nbytes, _keep = _workspace(ws, _residual_bytes(rows, d, n), gpu, x)
    _call(lib().chgnet_norm_backward, gpu, (rows, d, code, x.data_ptr(), ldx, _norm_kind(kind), w.data_ptr(), n, eps,
                                            dh.data_ptr(), ldu, dx.data_ptr(), ldd, dw.data_ptr(), bool(accumulate), p, nbytes))
    return dx, dw


@lru_cache(maxsize=64)
def _residual_cfg(*fields):
    return _Residual(*fields)


def _residual(f, post, post_kind, gate, pre, pre_kind, alpha, beta, p, seed, call, step, eps, rows, d, dtype, gpu):
    """(chgnet_residual, its pointer arguments from f to pre, rows of parameters, the gate's columns)."""
    ldf = _rows("f", f, rows, d, dtype, gpu)
    if post_kind is None:
        post_kind = "none" if post is None else "rms"
    post_n = post_rows = pre_rows = cols = ldg = 0
    post_n, pre_n = _norm_kind(post_kind), _norm_kind(pre_kind)
    if post is not None:
        post_rows = _params("post", post, d, gpu)
    elif post_n:
        _bad("the norm after the block needs its parameters, post")
    if pre is not None:
        pre_rows = _params("pre", pre, d, gpu)
        if not pre_n:
            _bad("pre_kind must be rms or layer")
    if gate is not None:
        cols = d if gate.shape == (rows, d) else 1
        ldg = _rows("gate", gate, rows, cols, dtype, gpu)
    at = _draw(seed, call, step, gpu)
    # (by values, never for a step: a cached struct holds no address)
    make = _residual_cfg if at is None else _Residual
    cfg = make(post_n, post_rows, pre_n, pre_rows, cols, alpha, beta, eps, p, seed, call, at)
    return cfg, (f.data_ptr(), ldf, gate.data_ptr() if cols else None, ldg, post.data_ptr() if post_rows else None,
                 pre.data_ptr() if pre_rows else None), post_rows + pre_rows, cols


def _any_followed(*tensors):
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


def residual_forward(x, f, post=None, post_kind=None, gate=None, pre=None, pre_kind="rms", alpha=1.0, beta=1.0, p=0.0, seed=0,
                     call=0, step=None, eps=1e-5, y=None, h=None):
    """The residual connection around a block: its stream x and its output f [rows, d], the norm after it, its gate, dropout
    and residual scale, and the norm before the next block. Returns (y, h):
        y = alpha x + beta Drop(sigmoid(gate) (post[0] n(f) + post[1])),  h = pre[0] n(y) + pre[1]  (None without pre)
    post, pre: fp32 [1, d] (scale) or [2, d] (scale, shift); kinds "rms", "layer", and after the block also "none" (a learned
    scale). gate: pre-activations [rows, d] or [rows, 1]. p, seed, call, step: as in `dropout`."""
    if _any_followed(x, f, post, gate, pre):
        _followed("x, f, post, gate or pre")
    rows, d, dtype, code, ldx, gpu = _start("x", x)
    cfg, args, _, _ = _residual(f, post, post_kind, gate, pre, pre_kind, alpha, beta, p, seed, call, step, eps, rows, d,
                                dtype, gpu)
    y, ldy = _like("y", y, rows, d, dtype, gpu, x)
    ldh = d
    if pre is not None:
        h, ldh = _like("h", h, rows, d, dtype, gpu, x)
    elif h is not None:
        _bad("h needs the parameters pre of its norm")
    _call(lib().chgnet_residual_forward, gpu, (rows, d, code, ctypes.byref(cfg), x.data_ptr(), ldx, *args, y.data_ptr(), ldy,
                                               None if h is None else h.data_ptr(), ldh))
    return y, h


ResidualGradients = namedtuple("ResidualGradients", "dx df dgate dpost dpre")


def residual_backward(y, f, dy, dh=None, post=None, post_kind=None, gate=None, pre=None, pre_kind="rms", alpha=1.0, beta=1.0,
                      p=0.0, seed=0, call=0, step=None, eps=1e-5, dx=None, df=None, dgate=None, dpost=None, dpre=None,
                      accumulate=False, ws=None):
    """ResidualGradients of residual_forward from the gradients dy of its y (None: zero) and dh of its h; y is what it returned,
    the other arguments are as they were. dpost and dpre are fp32 and added to what they hold with `accumulate`; the gradients
    of what is not there are None. ws: a Workspace of the caller's (one for each call that may run at the same time)."""
    if _any_followed(y, f, dy, dh, post, gate, pre):
        _followed("y, f, dy, dh, post, gate or pre")
    rows, d, dtype, code, ldy, gpu = _start("y", y)
    cfg, args, n, cols = _residual(f, post, post_kind, gate, pre, pre_kind, alpha, beta, p, seed, call, step, eps, rows, d,
                                   dtype, gpu)
    if (dh is None) != (pre is None):
        _bad("dh goes with pre")
    if dy is None and dh is None:
        _bad("neither dy nor dh is given")
    ldu = 0 if dy is None else _rows("dy", dy, rows, d, dtype, gpu)
    ldh = 0 if dh is None else _rows("dh", dh, rows, d, dtype, gpu)
    dx, ldx = _like("dx", dx, rows, d, dtype, gpu, y)
    df, ldf = _like("df", df, rows, d, dtype, gpu, y)
    ldg = 0
    if cols:
        dgate, ldg = _like("dgate", dgate, rows, cols, dtype, gpu, y)
    for name, out, of in (("dgate", dgate, gate), ("dpost", dpost, post), ("dpre", dpre, pre)):
        if of is None and out is not None:
            _bad("%s is given but not %s" % (name, name[1:]))
    if post is not None:
        dpost = _param_grad("dpost", dpost, post, accumulate, gpu)
    if pre is not None:
        dpre = _param_grad("dpre", dpre, pre, accumulate, gpu)
    w, nbytes, _keep = _workspace(ws, _residual_bytes(rows, d, n), gpu, y) if n else (None, 0, None)
    ptr = lambda t: None if t is None else t.data_ptr()
    _call(lib().chgnet_residual_backward, gpu, (
        rows, d, code, ctypes.byref(cfg), y.data_ptr(), ldy, *args, ptr(dy), ldu, ptr(dh), ldh, dx.data_ptr(), ldx,
        df.data_ptr(), ldf, ptr(dgate), ldg, ptr(dpost), ptr(dpre), bool(accumulate), w, nbytes))
    return ResidualGradients(dx, df, dgate, dpost, dpre)
