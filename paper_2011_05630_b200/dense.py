"""Dense operators on torch tensors: fully connected layers and gated feed-forward blocks, forwards and backwards.

    linear            y = act(x w^T + bias + residual)
    linear_backward   its gradients, from dy and the sum z that `linear(..., save=True)` kept
    gated             h = act(x wg^T + bg) * (x wu^T + bu)
    gated_backward    its gradients, from dh and the two sums that `gated(..., save=True)` kept

Matrices are two-dimensional CUDA tensors of one 16-bit type (float16 or bfloat16) on one device; rows may lie any distance apart
(`x[:, :k]` of a wider tensor is fine), the values of a row side by side.  Weights are [out][in], biases float32.  Every call
enqueues on the current stream of the tensors' device and computes inside libdlfusion.so (see include/dlfusion.h for the formulas
and their roundings); PyTorch allocates the outputs and, where a call needs one, its workspace.  Nothing is recorded for autograd: while autograd
records (outside torch.no_grad() and a Function's forward and backward), tensors that require gradients are refused.
"""
from __future__ import annotations

import ctypes as C
import struct
import threading

import torch

from . import binding as B

_DTYPES = {torch.float16: B.DTYPES["f16"], torch.bfloat16: B.DTYPES["bf16"]}
_LINEAR = struct.Struct("@ii3q6P5q")          # the argument structs of include/dlfusion.h
_LINEAR_GRAD = struct.Struct("@ii3q8P7q")
_GATED = struct.Struct("@ii3q8P6q")
_GATED_GRAD = struct.Struct("@ii3q11P9q")
_ops = {}   # name -> (call, its workspace query)
_heard = {}   # thread -> list, while `kernels` listens there (a thread-local variable costs every call 0.4 us)


def _enter(x, act, *tensors):
    """What a call's first matrix and its activation are to the library, once nothing speaks against the call as such."""
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise ValueError("a CUDA tensor is required: there is no CPU path")
    dtype, a = _DTYPES.get(x.dtype), B.DENSE_ACTS.get(act)
    if dtype is None:
        raise ValueError("float16 or bfloat16 is required, got %s" % x.dtype)
    if a is None:
        raise ValueError("act is one of %s, got %r" % (", ".join(B.DENSE_ACTS), act))
    if x.dim() != 2:
        raise ValueError("matrices have two dimensions, got %d" % x.dim())
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                raise ValueError("a tensor requires a gradient, and nothing would be recorded for it: call under torch.no_grad(), or with detached tensors")
    return dtype, a


def _size(t, name, i):
    """Rows (i 0) or columns (1) of what has to be a matrix."""
    try:
        return t.shape[i]
    except IndexError:
        raise ValueError("%s: matrices have two dimensions, got %d" % (name, t.dim())) from None


def _mat(t, name, shape, like):
    """(pointer, row length) of a matrix, or what is wrong with it."""
    if t is None:
        return 0, 0
    if t.dtype is not like.dtype or t.get_device() != like.get_device():
        raise ValueError("%s: %s on %s is required, got %s on %s" % (name, like.dtype, like.device, t.dtype, t.device))
    if t.shape != shape:
        raise ValueError("%s: shape %s is required, got %s" % (name, shape, tuple(t.shape)))
    if t.is_contiguous():
        return t.data_ptr(), shape[1]
    ld, step = t.stride()
    if (step != 1 and shape[1] > 1) or (ld < shape[1] and shape[0] > 1):
        raise ValueError("%s: the values of a row have to lie side by side and rows must not overlap (strides %s)" % (name, t.stride()))
    return t.data_ptr(), ld


def _vec(t, name, n, like):
    if t is None:
        return 0
    if t.dtype is not torch.float32 or t.get_device() != like.get_device() or t.dim() != 1 or t.numel() != n or not t.is_contiguous():
        raise ValueError("%s: %d float32 values side by side on %s are required" % (name, n, like.device))
    return t.data_ptr()


def _call(op, args, like, ask):
    """Enqueues on the current stream of the tensors' device, with a workspace if the call wants one (`ask`: it mostly does)."""
    index = like.get_device()
    if index != torch.cuda.current_device():
        with torch.cuda.device(index):
            return _call(op, args, like, ask)
    fns = _ops.get(op)
    if fns is None:
        fns = _ops[op] = getattr(B.lib(), op), getattr(B.lib(), op + "_workspace_bytes")
    stream = torch._C._cuda_getCurrentRawStream(index)   # (torch.cuda.current_stream(index).cuda_stream, 2 us faster)
    status = B.E_WORKSPACE if ask else fns[0](args, None, 0, stream)
    if status == B.E_WORKSPACE:   # (nothing was enqueued)
        need = C.c_size_t()
        B._check(fns[1](args, C.byref(need)), op)
        ws = like.new_empty(need.value, dtype=torch.uint8) if need.value else None
        status = fns[0](args, ws.data_ptr() if need.value else None, need.value, stream)
    if status != B.OK:
        raise B.DlfError(status, op)
    if _heard and threading.get_ident() in _heard:
        text = C.create_string_buffer(1024)
        B._check(getattr(B.lib(), op + "_kernels")(args, 0, text, len(text)), op)
        _heard[threading.get_ident()].append(text.value.decode())


def kernels(call):
    """Makes the call (a function without arguments) and says what its dense operators launched: a text for each (see dlf_linear_kernels)."""
    me, texts = threading.get_ident(), []
    before = _heard.get(me)
    _heard[me] = texts
    try:
        call()
    finally:
        if before is None:
            del _heard[me]
        else:
            _heard[me] = before
    return texts


def synchronize(device=None):
    """Waits for the current stream; raises if a dense operator's kernel on the device gave up (see dlf_dense_sync)."""
    with torch.cuda.device(device):
        B._check(B.lib().dlf_dense_sync(torch.cuda.current_stream().cuda_stream), "dlf_dense_sync")


def linear(x, w, bias=None, residual=None, act="none", save=False, out=None):
    """y = act(x w^T + bias + residual) for x [m][k], w [n][k], residual [m][n]; with `save` (y, z), z being the sum that the
    activation was applied to.  `out` receives y and may be the residual itself."""
    dtype, a = _enter(x, act, x, w, bias, residual, out)
    m, k = x.shape
    n = _size(w, "w", 0)
    xp, ldx = _mat(x, "x", (m, k), x)
    wp, ldw = _mat(w, "w", (n, k), x)
    rp, ldr = _mat(residual, "residual", (m, n), x)
    y = x.new_empty(m, n) if out is None else out
    yp, ldy = (y.data_ptr(), n) if out is None else _mat(y, "out", (m, n), x)
    z = x.new_empty(m, n) if save else None
    _call("dlf_linear", _LINEAR.pack(dtype, a, m, k, n, xp, wp, _vec(bias, "bias", n, x), rp, yp, z.data_ptr() if save else 0,
                                     ldx, ldw, ldr, ldy, n), x, False)
    return (y, z) if save else y


def linear_backward(dy, x, w, z=None, act="none", bias=True, residual=False, need_dx=True, need_dw=True):
    """(dx, dw, db, dr): the gradients of `linear`'s inputs, None for one that is not asked for.  z: what `linear(..., save=True)`
    kept, needed with an activation.  dr, the residual's gradient, is dy itself where there is no activation."""
    dtype, a = _enter(dy, act, dy, x, w, z)
    m, n = dy.shape
    k = _size(x, "x", 1) if x is not None else _size(w, "w", 1) if w is not None else 1
    if a and z is None:
        raise ValueError("z: the sum that the forward call kept is required with an activation")
    if (need_dw and x is None) or (need_dx and w is None):
        raise ValueError("x is required for dw, w for dx")
    dyp, lddy = _mat(dy, "dy", (m, n), dy)
    xp, ldx = _mat(x, "x", (m, k), dy)
    wp, ldw = _mat(w, "w", (n, k), dy)
    zp, ldz = _mat(z, "z", (m, n), dy) if a else (0, 0)
    dx = (torch.empty_like(x) if x is not None else dy.new_empty(m, k)) if need_dx else None
    dw = (torch.empty_like(w) if w is not None else dy.new_empty(n, k)) if need_dw else None
    db = dy.new_empty(n, dtype=torch.float32) if bias else None
    dr = torch.empty_like(dy) if residual and a else None
    ptr = lambda t: 0 if t is None else t.data_ptr()
    _call("dlf_linear_grad", _LINEAR_GRAD.pack(dtype, a, m, k, n, dyp, xp, wp, zp, ptr(dx), ptr(dw), ptr(db), ptr(dr),
                                               lddy, ldx, ldw, ldz, k, k, n), dy, a != 0)
    return dx, dw, db, dy if residual and not a else dr


def gated(x, wg, wu, bg=None, bu=None, act="silu", save=False, out=None):
    """h = act(x wg^T + bg) * (x wu^T + bu) for x [m][k], wg and wu [n][k]; with `save` (h, g, u), g and u being the two sums."""
    dtype, a = _enter(x, act, x, wg, wu, bg, bu, out)
    m, k = x.shape
    n = _size(wg, "wg", 0)
    xp, ldx = _mat(x, "x", (m, k), x)
    gp, ldwg = _mat(wg, "wg", (n, k), x)
    up, ldwu = _mat(wu, "wu", (n, k), x)
    h = x.new_empty(m, n) if out is None else out
    hp, ldh = (h.data_ptr(), n) if out is None else _mat(h, "out", (m, n), x)
    g = x.new_empty(m, n) if save else None
    u = x.new_empty(m, n) if save else None
    _call("dlf_gated", _GATED.pack(dtype, a, m, k, n, xp, gp, up, _vec(bg, "bg", n, x), _vec(bu, "bu", n, x), hp,
                                   g.data_ptr() if save else 0, u.data_ptr() if save else 0, ldx, ldwg, ldwu, ldh, n, n), x, False)
    return (h, g, u) if save else h


def gated_backward(dh, x, wg, wu, g, u, act="silu", bias=False, need_dx=True, need_dw=True):
    """(dx, dwg, dwu, dbg, dbu): the gradients of `gated`'s inputs, None for one that is not asked for.  g and u: what
    `gated(..., save=True)` kept."""
    dtype, a = _enter(dh, act, dh, x, wg, wu, g, u)
    m, n = dh.shape
    k = _size(x, "x", 1) if x is not None else _size(wg, "wg", 1) if wg is not None else 1
    if (need_dw and x is None) or (need_dx and (wg is None or wu is None)) or g is None or u is None:
        raise ValueError("g and u are required, x for the weights' gradients, wg and wu for dx")
    dhp, lddh = _mat(dh, "dh", (m, n), dh)
    xp, ldx = _mat(x, "x", (m, k), dh)
    wgp, ldwg = _mat(wg, "wg", (n, k), dh)
    wup, ldwu = _mat(wu, "wu", (n, k), dh)
    gp, ldg = _mat(g, "g", (m, n), dh)
    up, ldu = _mat(u, "u", (m, n), dh)
    dx = (torch.empty_like(x) if x is not None else dh.new_empty(m, k)) if need_dx else None
    dwg, dwu = (torch.empty_like(wg) if wg is not None else dh.new_empty(n, k) for _ in range(2)) if need_dw else (None, None)
    dbg, dbu = (dh.new_empty(n, dtype=torch.float32) for _ in range(2)) if bias else (None, None)
    ptr = lambda t: 0 if t is None else t.data_ptr()
    _call("dlf_gated_grad", _GATED_GRAD.pack(dtype, a, m, k, n, dhp, xp, wgp, wup, gp, up, ptr(dx), ptr(dwg), ptr(dwu), ptr(dbg),
                                             ptr(dbu), lddh, ldx, ldwg, ldwu, ldg, ldu, k, k, k), dh, True)
    return dx, dwg, dwu, dbg, dbu
