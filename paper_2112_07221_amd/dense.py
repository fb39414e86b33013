"""ctypes binding of the dense layers (`include/het_dense.h`): layer norm, linear layers and activations kept in 8 bits, forward and
backward, in the kernels of `libhet_cache.so`.

Matrices are 2-D GPU tensors whose rows may lie apart (any row stride, values of a row side by side); outputs are the caller's.
Calls run on the current torch stream of the current device unless `stream` says otherwise, and can be captured into a graph.  What a
call needs beyond its arguments it takes from torch's allocator on that stream, or from `workspace` (a contiguous GPU
tensor of at least `*_workspace()` bytes; calls that may run at the same time need one each).
"""
from __future__ import annotations

import contextlib
import ctypes as C

from . import hetcache
from .hetcache import HET_OK, HetError

F32, BF16, F16 = 0, 1, 2
ACT_NONE, ACT_RELU, ACT_GELU, ACT_SILU = 0, 1, 2, 3
PACK_BLOCK = 32

EXPORTS = ("het_layer_norm", "het_layer_norm_backward", "het_layer_norm_workspace", "het_pack", "het_expand", "het_linear",
           "het_linear_backward", "het_linear_workspace")


class Linear(C.Structure):
    """het_linear_t."""
    _fields_ = [("rows", C.c_int64), ("inp", C.c_int32), ("out", C.c_int32), ("type", C.c_int32), ("y_type", C.c_int32),
                ("act", C.c_int32), ("x_act", C.c_int32)] + \
               [(n, C.c_int64 if n.startswith("ld") else C.c_void_p) for n in (
                   "x", "ldx", "xq", "xe", "x_gamma", "x_beta", "w", "ldw", "bias", "residual", "ld_residual", "y", "ldy", "z", "ldz",
                   "zq", "ze", "dy", "lddy", "dz", "lddz", "dx", "lddx", "dw", "lddw", "dbias", "workspace")] + \
               [("workspace_bytes", C.c_int64)]


_lib = _torch = _types = _current_device = _raw_stream = None


def load() -> C.CDLL:
    """The library, with the dense layers' entry points declared."""
    global _lib, _torch, _types, _current_device, _raw_stream
    if _lib is not None:
        return _lib
    lib = hetcache.load()
    import torch
    p, i64, i32 = C.c_void_p, C.c_int64, C.c_int32
    lib.het_layer_norm.argtypes = [p, i32, i64, p, p, p, i32, i64, p, p, p, p, i64, i32, C.c_float, p]
    lib.het_layer_norm_backward.argtypes = [p, i32, i64, p, i32, i64, p, p, p, p, p, p, i64, p, i64, p, p, i64, i32, p, i64, p]
    lib.het_layer_norm_workspace.argtypes = [i64, i32]
    lib.het_pack.argtypes = [p, i32, i64, p, p, i64, i32, p]
    lib.het_expand.argtypes = [p, p, i64, i32, p, p, i32, p, i32, i64, p]
    lib.het_linear.argtypes = [C.POINTER(Linear), p]
    lib.het_linear_backward.argtypes = [C.POINTER(Linear), p]
    lib.het_linear_workspace.argtypes = [C.POINTER(Linear), i32]
    for name in EXPORTS:
        getattr(lib, name).restype = i64 if name.endswith("_workspace") else C.c_int
    _torch, _types = torch, {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
    _current_device, _raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
    _lib = lib
    return lib


class Packed:
    """A matrix [rows, dim] in the 8-bit form: q int8 [rows, pitch], e uint8 [rows, pitch / 32], pitch the width rounded up to 32."""
    __slots__ = ("q", "e", "dim")

    def __init__(self, q, e, dim):
        self.q, self.e, self.dim = q, e, dim

    @staticmethod
    def empty(rows, dim, device="cuda"):
        import torch
        pitch = -(-dim // PACK_BLOCK) * PACK_BLOCK
        return Packed(torch.empty(rows, pitch, dtype=torch.int8, device=device),
                      torch.empty(rows, pitch // PACK_BLOCK, dtype=torch.uint8, device=device), dim)

    @property
    def rows(self):
        return self.q.shape[0]


# ---- checks: what the library cannot see from pointers ------------------------------------------------
def _device(t, what):
    if not isinstance(t, _torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what} must be a tensor on the GPU")
    if t.get_device() != _current_device():
        raise ValueError(f"{what} is on another device than the current one")
    return t


def _matrix(t, what, rows, dim, dtype=None):
    """(pointer, row distance, type) of a [rows, dim] matrix."""
    _device(t, what)
    kind = _types.get(t.dtype)
    if kind is None or (dtype is not None and t.dtype != dtype):
        raise TypeError(f"{what} must be {dtype or 'float32, bfloat16 or float16'}")
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != dim:
        raise ValueError(f"{what} must be a matrix of {rows} rows of {dim} values")
    ld, along = t.stride()
    if along != 1 and dim > 1:
        raise ValueError(f"the values of a row of {what} must lie side by side")
    return t.data_ptr(), (ld if rows > 1 else max(ld, dim)), kind


def _vector(t, what, n):
    """Pointer of a contiguous fp32 vector of n values; None stays None."""
    if t is None:
        return None
    _device(t, what)
    if t.dtype != _torch.float32 or t.numel() != n or not t.is_contiguous():
        raise TypeError(f"{what} must be a contiguous float32 vector of {n} values")
    return t.data_ptr()


def _packed(p, what, rows, dim):
    """(q, e) pointers; None gives None twice."""
    if p is None:
        return None, None
    pitch = -(-dim // PACK_BLOCK) * PACK_BLOCK
    for t, dtype, width in ((_device(p.q, what), _torch.int8, pitch), (_device(p.e, what), _torch.uint8, pitch // PACK_BLOCK)):
        if p.dim != dim or t.dtype != dtype or t.shape != (rows, width) or not t.is_contiguous():
            raise ValueError(f"{what} must be the 8-bit form of a matrix of {rows} rows of {dim} values")
    return p.q.data_ptr(), p.e.data_ptr()


def _stream(stream):
    return _raw_stream(_current_device()) if stream is None else stream.cuda_stream


def _scratch(need, workspace, stream):
    """(tensor, pointer, bytes) of a call's workspace."""
    if need < 0:
        raise HetError(need, "workspace")
    if workspace is not None:
        _device(workspace, "workspace")
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
        return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()
    if need == 0:
        return None, None, 0
    with contextlib.nullcontext() if stream is None else _torch.cuda.stream(stream):
        t = _torch.empty(need, dtype=_torch.uint8, device="cuda")
    return t, t.data_ptr(), need


def _rc(status, what):
    if status != HET_OK:
        raise HetError(status, what)


def _shape(t, what):
    if isinstance(t, Packed):
        return t.rows, t.dim
    if not isinstance(t, _torch.Tensor) or t.dim() != 2:
        raise TypeError(f"{what} must be a matrix on the GPU")
    return t.shape


# ---- the calls ----------------------------------------------------------------------------------------
def layer_norm(x, gamma, beta, y, mean=None, rstd=None, packed=None, eps=1e-5, stream=None):
    """y = gamma (x - mean) rstd + beta by rows (het_layer_norm).  packed (a Packed or None) keeps the normalised rows in 8 bits."""
    lib = _lib or load()
    rows, dim = _shape(x, "x")
    px, ldx, tx = _matrix(x, "x", rows, dim)
    py, ldy, ty = _matrix(y, "y", rows, dim)
    q, e = _packed(packed, "packed", rows, dim)
    _rc(lib.het_layer_norm(px, tx, ldx, _vector(gamma, "gamma", dim), _vector(beta, "beta", dim), py, ty, ldy, _vector(mean, "mean", rows),
                           _vector(rstd, "rstd", rows), q, e, rows, dim, eps, _stream(stream)), "het_layer_norm")


def layer_norm_workspace(rows, dim):
    """Bytes of workspace layer_norm_backward takes."""
    return (_lib or load()).het_layer_norm_workspace(rows, dim)


def layer_norm_backward(dy, x, gamma, mean, rstd, dx, dgamma=None, dbeta=None, residual=None, workspace=None, stream=None):
    """dx, dgamma and dbeta of layer_norm (het_layer_norm_backward).  x: the input, with mean; or what the forward pass kept (a Packed;
    mean is not looked at).  residual: a gradient added to dx."""
    lib = _lib or load()
    rows, dim = _shape(dy, "dy")
    pdy, lddy, ty = _matrix(dy, "dy", rows, dim)
    pdx, lddx, tx = _matrix(dx, "dx", rows, dim)
    kept = isinstance(x, Packed)
    px, ldx = (None, 0) if kept else _matrix(x, "x", rows, dim, dx.dtype)[:2]
    q, e = _packed(x if kept else None, "x", rows, dim)
    pr, ldr = (None, 0) if residual is None else _matrix(residual, "residual", rows, dim, dx.dtype)[:2]
    if rows and (rstd is None or (not kept and mean is None)):
        raise ValueError("rstd (and mean, with x itself) must be what layer_norm gave")
    keep, ws, have = _scratch(lib.het_layer_norm_workspace(rows, dim), workspace, stream)
    _rc(lib.het_layer_norm_backward(pdy, ty, lddy, px, tx, ldx, None if kept else _vector(mean, "mean", rows), _vector(rstd, "rstd", rows), q, e,
                                    _vector(gamma, "gamma", dim), pr, ldr, pdx, lddx, _vector(dgamma, "dgamma", dim),
                                    _vector(dbeta, "dbeta", dim), rows, dim, ws, have, _stream(stream)), "het_layer_norm_backward")


def pack(x, packed, stream=None):
    """x in 8 bits into `packed` (het_pack)."""
    lib = _lib or load()
    rows, dim = _shape(x, "x")
    px, ldx, tx = _matrix(x, "x", rows, dim)
    q, e = _packed(packed, "packed", rows, dim)
    _rc(lib.het_pack(px, tx, ldx, q, e, rows, dim, _stream(stream)), "het_pack")


def expand(packed, y, act=ACT_NONE, gamma=None, beta=None, stream=None):
    """y = act(gamma v + beta) of the values v that `packed` holds (het_expand)."""
    lib = _lib or load()
    rows, dim = _shape(packed, "packed")
    py, ldy, ty = _matrix(y, "y", rows, dim)
    q, e = _packed(packed, "packed", rows, dim)
    _rc(lib.het_expand(q, e, rows, dim, _vector(gamma, "gamma", dim), _vector(beta, "beta", dim), act, py, ty, ldy, _stream(stream)), "het_expand")


def _run_linear(lib, l, call, what, backward, workspace, stream):
    keep, l.workspace, l.workspace_bytes = _scratch(lib.het_linear_workspace(C.byref(l), backward), workspace, stream)
    _rc(call(C.byref(l), _stream(stream)), what)


def linear(x, w, bias, y, act=ACT_NONE, residual=None, z=None, workspace=None, stream=None):
    """y = act(x w^T + bias) + residual (het_linear).  z keeps x w^T + bias: a tensor of x's type, or a Packed.  y and residual have
    x's type, or are float32."""
    lib = _lib or load()
    rows, inp = _shape(x, "x")
    out = _shape(w, "w")[0]
    l = Linear(rows=rows, inp=inp, out=out, act=act)
    l.x, l.ldx, l.type = _matrix(x, "x", rows, inp)
    l.w, l.ldw, _ = _matrix(w, "w", out, inp, x.dtype)
    l.bias = _vector(bias, "bias", out)
    l.y, l.ldy, l.y_type = _matrix(y, "y", rows, out)
    if residual is not None:
        l.residual, l.ld_residual, _ = _matrix(residual, "residual", rows, out, y.dtype)
    if isinstance(z, Packed):
        l.zq, l.ze = _packed(z, "z", rows, out)
    elif z is not None:
        l.z, l.ldz, _ = _matrix(z, "z", rows, out, x.dtype)
    _run_linear(lib, l, lib.het_linear, "het_linear", 0, workspace, stream)


def linear_backward(dy, x, w, z, act, dz, dx, dw, dbias=None, x_act=ACT_NONE, x_gamma=None, x_beta=None, workspace=None, stream=None):
    """dz = dy act'(z), dbias, dx = dz w and dw = dz^T x (het_linear_backward); each of dx, dw and dbias may be None.  z and x: tensors, or
    what the forward pass kept (a Packed); an x so kept stands for x_act(x_gamma v + x_beta).  dz may be None where it would be dy."""
    lib = _lib or load()
    rows, out = _shape(dy, "dy")
    ref = w if w is not None else dw
    if ref is None:
        raise ValueError("w or dw says how wide the layer's input is")
    inp, dtype = _shape(ref, "w")[1], ref.dtype
    l = Linear(rows=rows, inp=inp, out=out, act=act, x_act=x_act)
    if dtype not in _types:
        raise TypeError("w must be float32, bfloat16 or float16")
    l.type = _types[dtype]
    l.dy, l.lddy, l.y_type = _matrix(dy, "dy", rows, out)
    if dz is not None:
        l.dz, l.lddz, _ = _matrix(dz, "dz", rows, out, dtype)
    if isinstance(z, Packed):
        l.zq, l.ze = _packed(z, "z", rows, out)
    elif z is not None:
        l.z, l.ldz, _ = _matrix(z, "z", rows, out, dtype)
    if dx is not None:
        if w is None:
            raise ValueError("dx needs w")
        l.dx, l.lddx, _ = _matrix(dx, "dx", rows, inp, dtype)
        l.w, l.ldw, _ = _matrix(w, "w", out, inp, dtype)
    if dw is not None:
        l.dw, l.lddw, _ = _matrix(dw, "dw", out, inp, dtype)
        if isinstance(x, Packed):
            l.xq, l.xe = _packed(x, "x", rows, inp)
            l.x_gamma, l.x_beta = _vector(x_gamma, "x_gamma", inp), _vector(x_beta, "x_beta", inp)
        elif x is None:
            raise ValueError("dw needs x")
        else:
            l.x, l.ldx, _ = _matrix(x, "x", rows, inp, dtype)
            if x_act != ACT_NONE or x_gamma is not None or x_beta is not None:
                raise ValueError("x_act, x_gamma and x_beta are for an x kept in 8 bits")
    l.dbias = _vector(dbias, "dbias", out)
    _run_linear(lib, l, lib.het_linear_backward, "het_linear_backward", 1, workspace, stream)


def linear_workspace(rows, inp, out, dtype, backward=False, x_packed=False, dx=True, dw=True, dbias=True):
    """Bytes of workspace linear or linear_backward takes; x_packed: x is kept in 8 bits; dx, dw, dbias: which of them are wanted."""
    lib = _lib or load()
    l = Linear(rows=rows, inp=inp, out=out, type=_types[dtype], xq=1 if x_packed else None, dx=1 if dx else None, dw=1 if dw else None,
               dbias=1 if dbias else None)
    return lib.het_linear_workspace(C.byref(l), 1 if backward else 0)
