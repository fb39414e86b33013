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
import functools
import struct

from . import hetcache
from .hetcache import HET_OK, HetError

F32, BF16, F16 = 0, 1, 2
ACT_NONE, ACT_RELU, ACT_GELU, ACT_SILU = 0, 1, 2, 3
PACK_BLOCK = 32

EXPORTS = ("het_layer_norm", "het_layer_norm_backward", "het_layer_norm_workspace", "het_pack", "het_expand", "het_linear",
           "het_linear_backward", "het_linear_workspace")


# het_linear_t: the header's fields in order; `ld*` and sizes are whole numbers, the others pointers
LINEAR_FIELDS = ("rows", "inp", "out", "type", "y_type", "act", "x_act", "x", "ldx", "xq", "xe", "x_gamma", "x_beta", "w", "ldw", "bias", "residual",
                 "ld_residual", "y", "ldy", "z", "ldz", "zq", "ze", "dy", "lddy", "dz", "lddz", "dx", "lddx", "dw", "lddw", "dbias", "workspace",
                 "workspace_bytes")
_linear_t = struct.Struct("@q6i28q")


def linear_struct(**fields):
    """het_linear_t with these fields (None: NULL), the others 0."""
    return _linear_t.pack(*(fields.get(n) or 0 for n in LINEAR_FIELDS))


_lib = _torch = _types = _tensor = _f32 = _current_device = _raw_stream = None


def load() -> C.CDLL:
    """The library, with the dense layers' entry points declared."""
    global _lib, _torch, _types, _tensor, _f32, _current_device, _raw_stream
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
    lib.het_linear.argtypes = [p, p]
    lib.het_linear_backward.argtypes = [p, p]
    lib.het_linear_workspace.argtypes = [p, i32]
    for name in EXPORTS:
        getattr(lib, name).restype = i64 if name.endswith("_workspace") else C.c_int
    _torch, _types = torch, {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
    _tensor, _f32 = torch.Tensor, torch.float32
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
# A small call is launches and these lines, so they ask torch for each property once (and for a tensor's class only where something is wrong:
# torch.Tensor's isinstance is slow).
def _not_here(t, what):
    if not isinstance(t, _tensor) or not t.is_cuda:
        raise TypeError(f"{what} must be a tensor on the GPU")
    raise ValueError(f"{what} is on another device than the current one")


def _first(t, what):
    """(pointer, row distance, type, rows, dim, current device) of the matrix that says how large a call is."""
    try:
        dev = t.get_device()
        kind = _types.get(t.dtype)
        shape = t.shape
    except AttributeError:
        raise TypeError(f"{what} must be a matrix on the GPU") from None
    if dev < 0 or dev != _current_device():
        _not_here(t, what)
    if kind is None:
        raise TypeError(f"{what} must be float32, bfloat16 or float16")
    if len(shape) != 2:
        raise TypeError(f"{what} must be a matrix")
    rows, dim = shape
    ld, along = t.stride()
    if along != 1 and dim > 1:
        raise ValueError(f"the values of a row of {what} must lie side by side")
    return t.data_ptr(), ld if rows > 1 or ld > dim else dim, kind, rows, dim, dev


def _matrix(t, what, rows, dim, dev, dtype=None):
    """(pointer, row distance, type) of a [rows, dim] matrix."""
    try:
        if t.get_device() != dev:
            _not_here(t, what)
        have = t.dtype
    except AttributeError:
        raise TypeError(f"{what} must be a matrix on the GPU") from None
    kind = _types.get(have)
    if kind is None or (dtype is not None and have is not dtype):
        raise TypeError(f"{what} must be {dtype or 'float32, bfloat16 or float16'}")
    if t.shape != (rows, dim):
        raise ValueError(f"{what} must be a matrix of {rows} rows of {dim} values")
    ld, along = t.stride()
    if along != 1 and dim > 1:
        raise ValueError(f"the values of a row of {what} must lie side by side")
    return t.data_ptr(), ld if rows > 1 or ld > dim else dim, kind


def _vector(t, what, n, dev):
    """Pointer of a contiguous fp32 vector of n values; None stays None."""
    if t is None:
        return None
    try:
        if t.get_device() != dev:
            _not_here(t, what)
        if t.dtype is _f32 and t.numel() == n and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    raise TypeError(f"{what} must be a contiguous float32 vector of {n} values")


def _packed(p, what, rows, dim, dev):
    """(q, e) pointers; None gives None twice."""
    if p is None:
        return None, None
    pitch = -(-dim // PACK_BLOCK) * PACK_BLOCK
    try:
        q, e = p.q, p.e
        if q.get_device() != dev or e.get_device() != dev:
            _not_here(q if q.get_device() != dev else e, what)
        if p.dim == dim and q.dtype is _torch.int8 and e.dtype is _torch.uint8 and q.shape == (rows, pitch) and e.shape == (rows, pitch // PACK_BLOCK) and \
                q.is_contiguous() and e.is_contiguous():
            return q.data_ptr(), e.data_ptr()
    except AttributeError:
        raise TypeError(f"{what} must be a Packed") from None
    raise ValueError(f"{what} must be the 8-bit form of a matrix of {rows} rows of {dim} values")


def _stream(stream, dev):
    if stream is None:
        return _raw_stream(dev)
    if stream.device_index != dev:
        raise ValueError("stream is on another device than the current one")
    return stream.cuda_stream


def _scratch(need, workspace, stream, dev):
    """(tensor, pointer, bytes) of a call's workspace."""
    if workspace is not None:
        if not isinstance(workspace, _tensor) or workspace.get_device() != dev:
            _not_here(workspace, "workspace")
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
        return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()
    if need <= 0:                                          # (below 0: sizes that the call itself refuses)
        return None, None, 0
    with contextlib.nullcontext() if stream is None else _torch.cuda.stream(stream):
        t = _torch.empty(need, dtype=_torch.uint8, device="cuda")
    return t, t.data_ptr(), need


def _rc(status, what):
    if status != HET_OK:
        raise HetError(status, what)


# ---- the calls ----------------------------------------------------------------------------------------
def layer_norm(x, gamma, beta, y, mean=None, rstd=None, packed=None, eps=1e-5, stream=None):
    """y = gamma (x - mean) rstd + beta by rows (het_layer_norm).  packed (a Packed or None) keeps the normalised rows in 8 bits."""
    lib = _lib or load()
    px, ldx, tx, rows, dim, dev = _first(x, "x")
    py, ldy, ty = _matrix(y, "y", rows, dim, dev)
    q, e = _packed(packed, "packed", rows, dim, dev)
    _rc(lib.het_layer_norm(px, tx, ldx, _vector(gamma, "gamma", dim, dev), _vector(beta, "beta", dim, dev), py, ty, ldy,
                           _vector(mean, "mean", rows, dev), _vector(rstd, "rstd", rows, dev), q, e, rows, dim, eps, _stream(stream, dev)),
        "het_layer_norm")


@functools.lru_cache(maxsize=4096)
def layer_norm_workspace(rows, dim):
    """Bytes of workspace layer_norm_backward takes."""
    return (_lib or load()).het_layer_norm_workspace(rows, dim)


def layer_norm_backward(dy, x, gamma, mean, rstd, dx, dgamma=None, dbeta=None, residual=None, workspace=None, stream=None):
    """dx, dgamma and dbeta of layer_norm (het_layer_norm_backward).  x: the input, with mean; or what the forward pass kept (a Packed;
    mean is not looked at).  residual: a gradient added to dx."""
    lib = _lib or load()
    pdy, lddy, ty, rows, dim, dev = _first(dy, "dy")
    pdx, lddx, tx = _matrix(dx, "dx", rows, dim, dev)
    px = q = e = pm = pr = None
    ldx = ldr = 0
    if isinstance(x, Packed):
        q, e = _packed(x, "x", rows, dim, dev)
    else:
        px, ldx, _ = _matrix(x, "x", rows, dim, dev, dx.dtype)
        pm = _vector(mean, "mean", rows, dev)
    if residual is not None:
        pr, ldr, _ = _matrix(residual, "residual", rows, dim, dev, dx.dtype)
    if rows and (rstd is None or (px is not None and pm is None)):
        raise ValueError("rstd (and mean, with x itself) must be what layer_norm gave")
    keep, ws, have = _scratch(layer_norm_workspace(rows, dim), workspace, stream, dev)
    _rc(lib.het_layer_norm_backward(pdy, ty, lddy, px, tx, ldx, pm, _vector(rstd, "rstd", rows, dev), q, e, _vector(gamma, "gamma", dim, dev), pr, ldr, pdx, lddx,
                                    _vector(dgamma, "dgamma", dim, dev), _vector(dbeta, "dbeta", dim, dev), rows, dim, ws, have, _stream(stream, dev)),
        "het_layer_norm_backward")


def pack(x, packed, stream=None):
    """x in 8 bits into `packed` (het_pack)."""
    lib = _lib or load()
    px, ldx, tx, rows, dim, dev = _first(x, "x")
    q, e = _packed(packed, "packed", rows, dim, dev)
    _rc(lib.het_pack(px, tx, ldx, q, e, rows, dim, _stream(stream, dev)), "het_pack")


def expand(packed, y, act=ACT_NONE, gamma=None, beta=None, stream=None):
    """y = act(gamma v + beta) of the values v that `packed` holds (het_expand)."""
    lib = _lib or load()
    py, ldy, ty, rows, dim, dev = _first(y, "y")
    q, e = _packed(packed, "packed", rows, dim, dev)
    _rc(lib.het_expand(q, e, rows, dim, _vector(gamma, "gamma", dim, dev), _vector(beta, "beta", dim, dev), act, py, ty, ldy, _stream(stream, dev)), "het_expand")


@functools.lru_cache(maxsize=4096)
def _linear_workspace(rows, inp, out, kind, backward, x, ldx, w, ldw, dz, lddz, xq, dx, dw, dbias):
    """Of the operands' addresses only what they are modulo 16 matters: callers pass 16 + that."""
    l = linear_struct(rows=rows, inp=inp, out=out, type=kind, x=x, ldx=ldx, w=w, ldw=ldw, dz=dz, lddz=lddz, xq=xq, dx=dx, dw=dw, dbias=dbias)
    return (_lib or load()).het_linear_workspace(l, backward)


def linear_workspace(rows, inp, out, dtype, backward=False, x_packed=False, dx=True, dw=True, dbias=True, views=False):
    """Bytes of workspace linear or linear_backward takes.  x_packed: x is kept in 8 bits; dx, dw, dbias: which of them are wanted; views: x, w
    and dz may lie in wider matrices or begin anywhere (else they are contiguous and begin at multiples of 16 bytes)."""
    load()
    kind = _types[dtype]
    at = (16, 17) if views else (16,)
    return max(_linear_workspace(rows, inp, out, kind, int(backward), x, inp, w, inp, dz, out, int(x_packed), int(dx), int(dw), int(dbias))
               for x in at for w in at for dz in at)


def linear(x, w, bias, y, act=ACT_NONE, residual=None, z=None, workspace=None, stream=None):
    """y = act(x w^T + bias) + residual (het_linear).  z keeps x w^T + bias: a tensor of x's type, or a Packed.  y and residual have
    x's type, or are float32."""
    lib = _lib or load()
    px, ldx, kind, rows, inp, dev = _first(x, "x")
    pw, ldw, w_kind, out, w_inp, _ = _first(w, "w")
    if w_kind != kind:
        raise TypeError(f"w must be {x.dtype}")
    if w_inp != inp:
        raise ValueError(f"w must have rows of {inp} values")
    py, ldy, y_kind = _matrix(y, "y", rows, out, dev)
    pr = pz = zq = ze = None
    ldr = ldz = 0
    if residual is not None:
        pr, ldr, _ = _matrix(residual, "residual", rows, out, dev, y.dtype)
    if isinstance(z, Packed):
        zq, ze = _packed(z, "z", rows, out, dev)
    elif z is not None:
        pz, ldz, _ = _matrix(z, "z", rows, out, dev, x.dtype)
    keep, ws, have = _scratch(_linear_workspace(rows, inp, out, kind, 0, px % 16 + 16, ldx, pw % 16 + 16, ldw, 0, 0, 0, 0, 0, 0), workspace, stream, dev)
    _rc(lib.het_linear(_linear_t.pack(rows, inp, out, kind, y_kind, act, 0, px, ldx, 0, 0, 0, 0, pw, ldw, _vector(bias, "bias", out, dev) or 0, pr or 0, ldr, py, ldy,
                                      pz or 0, ldz, zq or 0, ze or 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, ws or 0, have), _stream(stream, dev)), "het_linear")


def linear_backward(dy, x, w, z, act, dz, dx, dw, dbias=None, x_act=ACT_NONE, x_gamma=None, x_beta=None, workspace=None, stream=None):
    """dz = dy act'(z), dbias, dx = dz w and dw = dz^T x (het_linear_backward); each of dx, dw and dbias may be None.  z and x: tensors, or
    what the forward pass kept (a Packed); an x so kept stands for x_act(x_gamma v + x_beta).  dz may be None where it would be dy."""
    lib = _lib or load()
    pdy, lddy, y_kind, rows, out, dev = _first(dy, "dy")
    ref = w if w is not None else dw
    if ref is None:
        raise ValueError("w or dw says how wide the layer's input is")
    _, _, kind, _, inp, _ = _first(ref, "w")
    dtype = ref.dtype
    px = pxq = pxe = pg = pb = pw = pz = pzq = pze = pdz = pdx = pdw = None
    ldx = ldw = ldz = lddz = lddx = lddw = 0
    if dz is not None:
        pdz, lddz, _ = _matrix(dz, "dz", rows, out, dev, dtype)
    if isinstance(z, Packed):
        pzq, pze = _packed(z, "z", rows, out, dev)
    elif z is not None:
        pz, ldz, _ = _matrix(z, "z", rows, out, dev, dtype)
    if dx is not None:
        if w is None:
            raise ValueError("dx needs w")
        pdx, lddx, _ = _matrix(dx, "dx", rows, inp, dev, dtype)
        pw, ldw, _ = _matrix(w, "w", out, inp, dev, dtype)
    if dw is not None:
        pdw, lddw, _ = _matrix(dw, "dw", out, inp, dev, dtype)
        if isinstance(x, Packed):
            pxq, pxe = _packed(x, "x", rows, inp, dev)
            pg, pb = _vector(x_gamma, "x_gamma", inp, dev), _vector(x_beta, "x_beta", inp, dev)
        elif x is None:
            raise ValueError("dw needs x")
        else:
            px, ldx, _ = _matrix(x, "x", rows, inp, dev, dtype)
            if x_act != ACT_NONE or x_gamma is not None or x_beta is not None:
                raise ValueError("x_act, x_gamma and x_beta are for an x kept in 8 bits")
    pdb = _vector(dbias, "dbias", out, dev)
    need = _linear_workspace(rows, inp, out, kind, 1, (px or 0) % 16 + 16, ldx, (pw or 0) % 16 + 16, ldw, (pdz or pdy) % 16 + 16, lddz if pdz else lddy, 1 if pxq else 0,
                             1 if pdx else 0, 1 if pdw else 0, 1 if pdb else 0)
    keep, ws, have = _scratch(need, workspace, stream, dev)
    _rc(lib.het_linear_backward(_linear_t.pack(rows, inp, out, kind, y_kind, act, x_act, px or 0, ldx, pxq or 0, pxe or 0, pg or 0, pb or 0, pw or 0, ldw, 0, 0, 0, 0, 0,
                                               pz or 0, ldz, pzq or 0, pze or 0, pdy, lddy, pdz or 0, lddz, pdx or 0, lddx, pdw or 0, lddw, pdb or 0, ws or 0, have),
                                _stream(stream, dev)), "het_linear_backward")


class BlockScratch:
    """What a ResidualBlock needs only while one of its passes runs: the layers' inputs and their gradients (rows x (dim + hidden) values) and the calls' workspace.
    Blocks of these sizes that run one after the other on one stream may share one; a captured pass writes to it at every replay.

    keep8: for blocks that keep their activations in 8 bits too (the workspace has room for a layer's input made from them)."""

    def __init__(self, rows, dim, hidden, dtype=None, keep8=True, device="cuda"):
        load()
        import torch
        self.rows, self.dim, self.hidden, self.keep8 = rows, dim, hidden, keep8
        dtype = self.dtype = dtype or torch.bfloat16
        self.h, self.u = torch.empty(rows, dim, dtype=dtype, device=device), torch.empty(rows, hidden, dtype=dtype, device=device)
        need = max([linear_workspace(rows, dim, hidden, dtype), linear_workspace(rows, hidden, dim, dtype), layer_norm_workspace(rows, dim), 16] +
                   [linear_workspace(rows, i, o, dtype, True, packed) for i, o in ((dim, hidden), (hidden, dim)) for packed in ((False, True) if keep8 else (False,))])
        self.workspace = torch.empty(need, dtype=torch.uint8, device=device)


class ResidualBlock:
    """y = x + w2 act(w1 norm(x) + b1) + b2 over rows of `dim` values with `hidden` values inside, in a float32 residual stream: what
    stands between the rows a lookup hands out (x) and the gradient an update takes (dx).  Weights and what is multiplied are of `dtype`.

    keep8: between the passes the normalised rows and the pre-activations are kept in 8 bits (8.25 bits a value, and rstd; the layers' inputs are made
    from them again), else mean, rstd, the normalised rows with their weights, z and act(z) are kept whole, and x by the caller.  At 4096 rows of 1664
    values, 4096 inside, in bf16: 24 MB, or 81 and x's 27.  What is needed within a pass alone, 47 MB and a workspace of 35 (7 for blocks that keep
    whole), is in `scratch`: one BlockScratch for any number of blocks that run one after the other, or the block's own (None).  All is taken at construction, for
    `rows` rows: passes of so many allocate nothing, ones of fewer rows (the last batch of an epoch) take their workspace from torch's allocator.  A block is used
    on one stream at a time."""

    def __init__(self, rows, dim, hidden, dtype=None, act=ACT_GELU, eps=1e-5, keep8=True, generator=None, device="cuda", scratch=None):
        load()
        import torch
        self.rows, self.dim, self.hidden, self.act, self.eps, self.keep8 = rows, dim, hidden, act, eps, keep8
        dtype = self.dtype = dtype or torch.bfloat16

        def new(*shape, dtype=torch.float32):
            return torch.empty(*shape, dtype=dtype, device=device)

        self.gamma, self.beta = new(dim).fill_(1), new(dim).zero_()
        self.w1 = (torch.randn(hidden, dim, generator=generator, device=device) / dim ** 0.5).to(dtype)
        self.w2 = (torch.randn(dim, hidden, generator=generator, device=device) / hidden ** 0.5).to(dtype)
        self.b1, self.b2 = new(hidden).zero_(), new(dim).zero_()
        self.dgamma, self.dbeta, self.dw1, self.dw2 = new(dim), new(dim), new(hidden, dim, dtype=dtype), new(dim, hidden, dtype=dtype)
        self.db1, self.db2 = new(hidden), new(dim)
        # between the passes
        self._x, self._now = None, None
        mean, rstd = None if keep8 else new(rows), new(rows)
        n8 = Packed.empty(rows, dim, device) if keep8 else None
        z = Packed.empty(rows, hidden, device) if keep8 else new(rows, hidden, dtype=dtype)
        # within one
        scratch = scratch or BlockScratch(rows, dim, hidden, dtype, keep8, device)
        if (scratch.rows, scratch.dim, scratch.hidden, scratch.dtype) != (rows, dim, hidden, dtype) or scratch.keep8 < keep8:
            raise ValueError("the scratch is for blocks of other sizes or another type, or for ones that keep their activations whole")
        # (the forward pass' h and u are free when it ends if they are kept in 8 bits)
        h, u = (scratch.h, scratch.u) if keep8 else (new(rows, dim, dtype=dtype), new(rows, hidden, dtype=dtype))
        self._all = (h, u, n8, z, mean, rstd, scratch.h, scratch.u, scratch.workspace)

    def _of(self, rows):
        """h, u, n8, z, mean, rstd, dh, du and the workspace of a pass of so many rows: the buffers' first ones.  (A call of fewer rows may split its sums into more
        parts and so need more workspace; it takes its own.)"""
        if rows == self.rows:
            return self._all
        if rows > self.rows:
            raise ValueError(f"the block has room for {self.rows} rows")
        return tuple(None if v is None else Packed(v.q[:rows], v.e[:rows], v.dim) if isinstance(v, Packed) else v[:rows] for v in self._all[:-1]) + (None,)

    def parameters(self):
        """[(parameter, gradient)]; the gradients are written by backward."""
        return [(self.gamma, self.dgamma), (self.beta, self.dbeta), (self.w1, self.dw1), (self.b1, self.db1), (self.w2, self.dw2), (self.b2, self.db2)]

    def forward(self, x, y):
        """y of x, both float32 [rows, dim] with as many rows as the block has or fewer; x has to stay until backward if activations are kept whole."""
        self._now = None                                   # (a call that is refused half way leaves nothing for backward)
        h, u, n8, z, mean, rstd, _, _, ws = now = self._of(len(x))
        layer_norm(x, self.gamma, self.beta, h, mean, rstd, packed=n8, eps=self.eps)
        linear(h, self.w1, self.b1, u, self.act, z=z, workspace=ws)
        linear(u, self.w2, self.b2, y, residual=x, workspace=ws)
        self._x, self._now = None if self.keep8 else x, now

    def backward(self, dy, dx):
        """dx and the parameters' gradients from dy (float32, as many rows as the forward pass had), once for a forward pass.  dx may be dy itself."""
        keep8 = self.keep8
        if self._now is None:
            raise RuntimeError("backward follows a forward pass")
        (h, u, n8, z, mean, rstd, dh, du, ws), self._now = self._now, None
        # dz2 lies where dh will
        linear_backward(dy, z if keep8 else u, self.w2, None, ACT_NONE, dh, du, self.dw2, self.db2, x_act=self.act if keep8 else ACT_NONE, workspace=ws)
        # dz1 takes du's place: slope and product follow each other
        linear_backward(du, n8 if keep8 else h, self.w1, z, self.act, du, dh, self.dw1, self.db1, x_gamma=self.gamma if keep8 else None,
                        x_beta=self.beta if keep8 else None, workspace=ws)
        layer_norm_backward(dh, n8 if keep8 else self._x, self.gamma, mean, rstd, dx, self.dgamma, self.dbeta, residual=dy, workspace=ws)
        self._x = None
