"""Thin ctypes binding of the operators in include/chgnet_ops.h: the gate of the
gated MLP with an 8-bit checkpoint of its input, the scaled embedding lookup with
its gradient, norms and the residual connection around a block with its gate and
dropout, linear layers in 8-bit floating point.

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
import math
from collections import namedtuple
from functools import lru_cache

import torch

from . import binding as bd

EXPORTED = ("chgnet_gate_forward", "chgnet_gate_backward_workspace", "chgnet_gate_backward", "chgnet_embed_forward",
            "chgnet_embed_backward_workspace", "chgnet_embed_backward", "chgnet_norm_forward", "chgnet_norm_backward",
            "chgnet_residual_forward", "chgnet_residual_backward_workspace", "chgnet_residual_backward", "chgnet_dropout",
            "chgnet_fp8_quantize", "chgnet_fp8_matmul_workspace", "chgnet_fp8_matmul", "chgnet_fp8_linear_workspace",
            "chgnet_fp8_linear")
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


class _Fp8(ctypes.Structure):
    """chgnet_fp8"""

    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("codes", ctypes.c_void_p), ("ld", ctypes.c_int64),
                ("scale", ctypes.c_void_p), ("ld_scale", ctypes.c_int64), ("block_rows", ctypes.c_int32)]


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
        psz = ctypes.POINTER(sz)
        L.chgnet_fp8_quantize.argtypes = [i64, i64, i32, vp, i64, vp, vp, vp]
        L.chgnet_fp8_matmul_workspace.argtypes = L.chgnet_fp8_linear_workspace.argtypes = [i64, i64, i64, psz]
        L.chgnet_fp8_matmul.argtypes = [vp, vp, i32, vp, i64, cint, vp, sz, vp]
        L.chgnet_fp8_linear.argtypes = [i64, i32, vp, i64, vp, vp, i64, vp, sz, vp]
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
    shape = w.shape
    if len(shape) != 2 or shape[0] not in (1, 2):
        _bad("%s must be [1, %d] (scale) or [2, %d] (scale, shift), not %s" % (name, d, d, list(shape)))
    if shape[1] != d or w.dtype is not torch.float32 or w.get_device() != gpu or not w.is_contiguous():
        _wrong(name, w, (shape[0], d), "contiguous torch.float32", gpu)
    return shape[0]


def _norm_kind(kind):
    if kind not in NORMS:
        _bad("unknown norm %r: one of %s" % (kind, ", ".join(NORMS)))
    return NORMS[kind]


def _like(name, out, rows, cols, dtype, gpu, like):
    """(tensor, row stride) of a call's output: the caller's or a new one (of `like`'s type)."""
    if out is None:
        # (0.6 us less than torch.empty)
        return torch.empty_like(like, memory_format=torch.contiguous_format) if cols == like.shape[1] else torch.empty(
            (rows, cols), dtype=dtype, device=like.device), cols
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


def _number(name, v):
    """A factor's value as it is now (of a tensor, too, which may hold another one at the next call)."""
    if type(v) is float:
        return v
    if isinstance(v, torch.Tensor) and v.requires_grad and torch.is_grad_enabled():
        _followed(name)
    try:
        if not isinstance(v, (str, bytes)):
            return float(v)
    except (TypeError, ValueError, RuntimeError):
        pass
    _bad("%s must be a number, not %r" % (name, v))


def _rate(p):
    """p in steps of 2^-16, rounded from the number given: the call takes fp32, whose own rounding may pass a half step."""
    p = _number("p", p)
    if not 0.0 <= p <= 1.0:
        _bad("p must be in 0 .. 1, not %r" % p)
    return math.floor(p * 65536.0 + 0.5) / 65536.0


def dropout(x, p, seed, call=0, step=None, out=None):
    """x [rows, d] / (1 - p) where the counter-based generator keeps a value, else 0 (p counts in steps of 2^-16, to the
    nearest of which it is rounded). The mask is that of (seed, call + step) whatever the type and strides, and is not stored: the
    same call on the upstream gradient is the backward pass. step: int64 [1] on the GPU, for graphs whose replays draw anew."""
    if x.requires_grad and torch.is_grad_enabled():
        _followed("x")
    rows, d, dtype, code, ldx, gpu = _start("x", x)
    p, at = _rate(p), _draw(seed, call, step, gpu)
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
    """Of Python's own numbers only: an object of another type may be its own key and change its value."""
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
    cfg = make(post_n, post_rows, pre_n, pre_rows, cols, _number("alpha", alpha), _number("beta", beta), _number("eps", eps),
               _rate(p), seed, call, at)
    return cfg, (f.data_ptr(), ldf, gate.data_ptr() if cols else None, ldg, post.data_ptr() if post_rows else None,
                 pre.data_ptr() if pre_rows else None), post_rows + pre_rows, cols


def _any_followed(*tensors):
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                return True
    return False


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


class Fp8Matrix:
    """A matrix [rows, cols] in 8-bit floating point: codes (torch.float8_e4m3fn) and a power of two (torch.float8_e8m0fnu) for
    each block of block_rows (1 or 128) x 128 of them; its values are codes.float() times their block's scale.float(). From
    tensors of the caller's, codes [rows, cols] in rows that start on 16 bytes and, up to the next multiple of 16 columns, end
    in zeros; scale [rows / block_rows, cols / 128], rounded up, in rows that start on 4 bytes. Or made by fp8_quantize."""

    __slots__ = ("rows", "cols", "block_rows", "_codes", "_scale", "_data", "_c", "_gpu")

    def __init__(self, codes, scale, block_rows=1):
        if codes.dim() != 2 or codes.dtype is not torch.float8_e4m3fn:
            _bad("codes must be a matrix of torch.float8_e4m3fn, not %s %s" % (list(codes.shape), codes.dtype))
        if block_rows not in (1, 128):
            _bad("block_rows must be 1 or 128")
        rows, cols = codes.shape
        shape = (-(-rows // block_rows), -(-cols // 128))
        gpu = codes.get_device()
        if scale.dtype is not torch.float8_e8m0fnu or scale.shape != shape or scale.get_device() != gpu:
            _bad("scale must be %s of torch.float8_e8m0fnu on %s, not %s %s on %s"
                 % (list(shape), codes.device, list(scale.shape), scale.dtype, scale.device))
        self._codes, self._scale, self._data, self._gpu = codes, scale, None, gpu
        self._make(rows, cols, block_rows, codes.data_ptr(), self._row("codes", codes, 16), scale.data_ptr(),
                   self._row("scale", scale, 4))

    @staticmethod
    def _row(name, t, unit):
        """Row stride of bytes whose rows start on `unit` bytes and can be read up to the next multiple of it."""
        rows, cols = t.shape
        whole = -(-cols // unit) * unit
        ld = t.stride(0) if rows > 1 and cols else whole  # (of rows without bytes it says nothing)
        if (cols > 1 and t.stride(1) != 1) or ld % unit or ld < whole or t.data_ptr() % unit:
            _bad("%s must have contiguous columns, and rows that start on %d bytes and do not overlap" % (name, unit))
        if whole != cols and rows and t.storage_offset() + (rows - 1) * ld + whole > t.untyped_storage().nbytes():
            _bad("%s must have %d bytes in its last row too" % (name, whole))
        return ld

    def _make(self, rows, cols, block_rows, codes, ld, scale, ld_scale):
        self.rows, self.cols, self.block_rows = rows, cols, block_rows
        self._c = _Fp8(rows, cols, codes, ld, scale, ld_scale, block_rows)

    @classmethod
    def empty(cls, rows, cols, block_rows=1, device="cuda"):
        """One allocation for fp8_quantize to write to."""
        self = cls.__new__(cls)
        # whole lines of 128 bytes: rows that start within one cost a third more writes (512 rows of 397,934 codes: 191 -> 151 us)
        unit = 16 if cols <= 128 else 128
        ld, lds = -(-cols // unit) * unit, -(-cols // 512) * 4
        self._data = torch.empty(rows * ld + -(-rows // block_rows) * lds, dtype=torch.uint8, device=device)
        self._gpu = self._data.get_device()
        p = self._data.data_ptr()
        self._make(rows, cols, block_rows, p, ld, p + rows * ld, lds)
        self._codes = self._scale = None
        return self

    @property
    def shape(self):
        return (self.rows, self.cols)

    @property
    def codes(self):
        if self._codes is None:
            n = self.rows * self._c.ld
            self._codes = self._data[:n].view(torch.float8_e4m3fn).view(self.rows, self._c.ld)[:, :self.cols]
        return self._codes

    @property
    def scale(self):
        if self._scale is None:
            n, rows = self.rows * self._c.ld, -(-self.rows // self.block_rows)
            self._scale = self._data[n:].view(torch.float8_e8m0fnu).view(rows, self._c.ld_scale)[:, :-(-self.cols // 128)]
        return self._scale


def _fp8_out(name, m, rows, cols, block_rows, gpu, like):
    if m is None:
        return Fp8Matrix.empty(rows, cols, block_rows, like.device)
    if m.rows != rows or m.cols != cols or m.block_rows != block_rows or m._gpu != gpu:
        _bad("%s must be of [%d, %d] with block_rows %d on GPU %d" % (name, rows, cols, block_rows, gpu))
    return m


def _fp8_quantize(x, block_rows, want, want_t, out, out_t):
    if x.requires_grad and torch.is_grad_enabled():
        _followed("x")
    rows, cols, _, code, ldx, gpu = _start("x", x)
    if block_rows not in (1, 128):
        _bad("block_rows must be 1 or 128")
    q = _fp8_out("out", out, rows, cols, block_rows, gpu, x) if want else None
    t = _fp8_out("out_t", out_t, cols, rows, block_rows, gpu, x) if want_t else None
    if q is not None and t is not None and q._c.codes == t._c.codes and q._c.codes:
        _bad("out and out_t have the same codes")
    _call(lib().chgnet_fp8_quantize, gpu, (rows, cols, code, x.data_ptr(), ldx, ctypes.byref(q._c) if want else None,
                                           ctypes.byref(t._c) if want_t else None))
    return q, t


def fp8_quantize(x, block_rows=1, transposed=False, out=None):
    """x [rows, cols] in fp32, bf16 or fp16 as an Fp8Matrix, with a power of two for each block of block_rows (1, or 128 for
    weights) x 128; with `transposed` its transpose [cols, rows], whose blocks run along the rows of x."""
    q, t = _fp8_quantize(x, block_rows, not transposed, transposed, out, out)
    return t if transposed else q


def fp8_quantize_both(x, block_rows=1, out=None, out_t=None):
    """Both forms in one pass over x: what a training step needs of a linear layer's input, weight and upstream gradient."""
    return _fp8_quantize(x, block_rows, True, True, out, out_t)


@lru_cache(maxsize=4096)
def _fp8_bytes(fn, m, n, k):
    need = ctypes.c_size_t()
    bd._check(getattr(lib(), fn)(m, n, k, ctypes.byref(need)))
    return need.value


def fp8_matmul(a, b, dtype=torch.bfloat16, out=None, accumulate=False, ws=None):
    """out [M, N] = a b^T of Fp8Matrix a [M, K] and b [N, K], summed in fp32, in `dtype` (or out's); added to what it holds with
    `accumulate`. With (q, t) of fp8_quantize_both a linear layer's output is (x.q, w.q), its input's gradient (dy.q, w.t) and
    its weight's (dy.t, x.t). ws: a Workspace of the caller's (one for each call that may run at the same time)."""
    gpu, m, n, k = a._gpu, a.rows, b.rows, a.cols
    if gpu < 0 or b._gpu != gpu:
        _bad("both matrices must be on one GPU")
    if out is None:
        if accumulate:
            _bad("accumulate needs an out to add to")
        if dtype not in DTYPES:
            _bad("dtype must be fp32, bf16 or fp16, not %s" % dtype)
        out, ldo = torch.empty((m, n), dtype=dtype, device=torch.device("cuda", gpu)), n
    else:
        dtype = out.dtype
        if dtype not in DTYPES:
            _bad("out must be fp32, bf16 or fp16, not %s" % dtype)
        ldo = _rows("out", out, m, n, dtype, gpu)
    need = _fp8_bytes("chgnet_fp8_matmul_workspace", m, n, k)
    p, nbytes, _keep = _workspace(ws, need, gpu, out) if need else (None, 0, None)
    _call(lib().chgnet_fp8_matmul, gpu, (ctypes.byref(a._c), ctypes.byref(b._c), DTYPES[dtype], out.data_ptr(), ldo,
                                         bool(accumulate), p, nbytes))
    return out


def fp8_linear(x, w, out=None, ws=None):
    """out [rows, N] = q(x) w^T of x [rows, K] in fp32, bf16 or fp16 and an Fp8Matrix w [N, K], where q(x) is fp8_quantize's
    x; out is of x's type, summed as fp8_matmul does for that (for sums to fp32's last place of 16-bit x: fp8_matmul of
    fp8_quantize(x) in fp32). ws: a Workspace of the caller's (one for each call that may run at the same time)."""
    if x.requires_grad and torch.is_grad_enabled():
        _followed("x")
    rows, k, dtype, code, ldx, gpu = _start("x", x)
    if k != w.cols or w._gpu != gpu:
        _bad("w must be of [N, %d] on GPU %d, not of [%d, %d]" % (k, gpu, w.rows, w.cols))
    out, ldo = _like("out", out, rows, w.rows, dtype, gpu, x)
    need = _fp8_bytes("chgnet_fp8_linear_workspace", rows, w.rows, k)
    p, nbytes, _keep = _workspace(ws, need, gpu, x) if need else (None, 0, None)
    _call(lib().chgnet_fp8_linear, gpu, (rows, code, x.data_ptr(), ldx, ctypes.byref(w._c), out.data_ptr(), ldo, p, nbytes))
    return out
