"""The dense layers on the GPU against plain forms in 64 bits on the CPU.

Tolerances are sums of roundings.  A value rounded to type T is off by at most finfo(T).eps / 2 of it (H below).  A sum of n products in
fp32 in any order is off by at most n 2^-24 of the sum of their magnitudes; for the matrix instructions, whose inner order and rounding
are not specified, twice that is allowed.  Functions (exp, erf, sqrt) are within 4 ulp.
"""
import math

import pytest
import torch

from paper_2112_07221_amd import dense
from paper_2112_07221_amd.hetcache import HetError

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U = 2.0 ** -24
ACTS = {"none": dense.ACT_NONE, "relu": dense.ACT_RELU, "gelu": dense.ACT_GELU, "silu": dense.ACT_SILU}


def H(t):
    return torch.finfo(t).eps / 2


def tiny(t):
    """Half of the smallest subnormal: the rounding of values next to zero."""
    return torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def rows_in(g, rows, dim, t, scale=1.0, at=0.0, extra=0, offset=0):
    """A [rows, dim] matrix on the GPU of type t; `extra`: values between its rows, `offset`: values before the first."""
    v = (at + scale * torch.randn(rows, dim, generator=g)).to(t)
    if not extra and not offset:
        return v.cuda()
    flat = torch.full((offset + rows * (dim + extra),), 7.0, dtype=t, device="cuda")
    m = flat[offset:].view(rows, dim + extra)[:, :dim]
    m.copy_(v)
    return m


class Guarded:
    """An output with values before, between and behind its rows that have to stay as they are."""

    def __init__(self, rows, dim, t, extra=3, offset=1):
        self.flat = torch.full((offset + (rows + 2) * (dim + extra),), -5.0, dtype=t, device="cuda")
        self.m = self.flat[offset:].view(rows + 2, dim + extra)[:rows, :dim]
        self.rows, self.dim, self.offset, self.extra = rows, dim, offset, extra

    def untouched(self):
        f = self.flat.clone()
        f[self.offset:].view(self.rows + 2, self.dim + self.extra)[:self.rows, :self.dim] = -5.0
        return bool((f == -5.0).all())


def D(t):
    return t.detach().cpu().double()


def near(got, want, tol, what=""):
    got = D(got)
    assert got.shape == want.shape
    off = (got - want).abs()
    bad = ~(off <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} are off, the worst {float(off[bad].max())} at {bad.nonzero()[0].tolist()}, allowed {float((tol + 0 * off)[bad][0])}"


# ---- the 8-bit form, in whole numbers ------------------------------------------------------------------
def pitch(dim):
    return -(-dim // 32) * 32


def packed_by_rule(v):
    """(q, e) of fp32 values, from the rule's words, with Python's exact fractions of powers of two (doubles hold all of them)."""
    rows, dim = v.shape
    q = torch.zeros(rows, pitch(dim), dtype=torch.int8)
    e = torch.zeros(rows, pitch(dim) // 32, dtype=torch.uint8)
    for r in range(rows):
        for b in range(pitch(dim) // 32):
            block = [float(x) for x in v[r, 32 * b:32 * b + 32]]
            if any(not math.isfinite(x) for x in block):
                e[r, b] = 255
                continue
            most = max(abs(x) for x in block)
            k = -126
            while round(most / 2.0 ** k) > 127 and k < 122:
                k += 1
            limit = 63 if k == 122 else 127
            e[r, b] = k + 127
            for j, x in enumerate(block):
                q[r, 32 * b + j] = max(-limit, min(limit, round(x / 2.0 ** k)))
    return q, e


def values(p):
    q, e = D(p.q), D(p.e)
    v = q * torch.exp2(e - 127).repeat_interleave(32, 1)
    v[(D(p.e) == 255).repeat_interleave(32, 1)] = math.nan
    return v[:, :p.dim]


def act64(name, v):
    if name == "relu":
        return torch.where(v > 0, v, torch.where(v == v, torch.zeros_like(v), v))
    if name == "gelu":
        return v * torch.special.ndtr(v)
    if name == "silu":
        return v * torch.sigmoid(v)
    return v


def slope64(name, v):
    if name == "relu":
        return (v > 0).double()
    if name == "gelu":
        return torch.special.ndtr(v) + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = torch.sigmoid(v)
        return s + v * s * (1 - s)
    return torch.ones_like(v)


# gelu and silu: what the fp32 form of the function itself is off by, for |v| up to 20.  Both are v times (or sums with v times) a factor within
# [0, 1.13] that is off by at most 16 ulp: 4 of the function, the rest of its argument's and the formula's roundings (exp's argument is off by
# 2 ulp of up to 20 in the exponent where the factor is below e^-20, which is far below the bound).
def act_off(v):
    return 20 * 2 * U * (1 + v.abs())


# ---- layer norm ----------------------------------------------------------------------------------------
NORM_TYPES = [(F32, F32), (F32, BF16), (F32, F16), (BF16, BF16), (F16, F16)]
# widths at which lanes, chunks a lane and wave or workgroup change, and odd ones; rows: one, not a workgroup's, more than one pass of the backward's grid
NORM_SHAPES = [(1, 1), (1, 2), (3, 5), (7, 8), (33, 10), (5, 31), (130, 32), (129, 33), (17, 64), (9, 127), (70, 260), (5, 512), (6, 513), (3, 1001), (4, 1664), (2, 2048),
               (3, 2049), (2, 4097), (1, 8192), (2, 8193), (1, 16385), (2, 32768), (20011, 10), (6001, 64), (1100, 300)]


def norm64(x, gamma, beta, eps):
    x = D(x)
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = 1 / torch.sqrt((d * d).mean(1, keepdim=True) + eps)
    n = d * rstd
    y = n * (1 if gamma is None else D(gamma)) + (0 if beta is None else D(beta))
    # fp32: a row's sum goes through at most 32 values a lane, 6 steps over lanes and 15 over waves: 53 roundings, 56 with the division
    mean_off = 56 * U * x.abs().mean(1, keepdim=True)
    d_off = mean_off + U * d.abs()
    var = (d * d).mean(1, keepdim=True)
    var_off = 58 * U * var + 2 * (d_off * d.abs()).mean(1, keepdim=True) + (d_off * d_off).mean(1, keepdim=True)
    rstd_off = rstd * (0.5 * var_off * rstd * rstd * 1.01 + 6 * U)
    n_off = d_off * rstd + d.abs() * rstd_off + U * n.abs()
    return mean, rstd, n, y, mean_off, rstd_off, n_off


@pytest.mark.parametrize("tx,ty", NORM_TYPES)
@pytest.mark.parametrize("rows,dim", NORM_SHAPES)
def test_layer_norm(rows, dim, tx, ty):
    g = gen(rows * 1000 + dim)
    x = rows_in(g, rows, dim, tx, 2.0, 0.7, extra=dim % 3, offset=dim % 2)
    gamma, beta = (1 + 0.2 * torch.randn(dim, generator=g)).cuda(), torch.randn(dim, generator=g).cuda()
    y = Guarded(rows, dim, ty)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    kept = dense.Packed.empty(rows, dim)
    dense.layer_norm(x, gamma, beta, y.m, mean, rstd, packed=kept)
    m64, r64, n64, y64, m_off, r_off, n_off = norm64(x, gamma, beta, 1e-5)
    near(mean, m64[:, 0], m_off[:, 0], "mean")
    near(rstd, r64[:, 0], r_off[:, 0], "rstd")
    off = n_off * D(gamma).abs() + 2 * U * (n64.abs() * D(gamma).abs() + y64.abs())
    near(y.m, y64, off + H(ty) * (y64.abs() + off) + tiny(ty), "y")
    assert y.untouched()
    check_packed_of_computed(kept, n64, n_off)
    # the same without what nobody asks for, into the same bits
    again = torch.empty(rows, dim, dtype=ty, device="cuda")
    dense.layer_norm(x, gamma, beta, again)
    assert torch.equal(again, y.m)
    plain = torch.empty(rows, dim, dtype=ty, device="cuda")
    dense.layer_norm(x, None, None, plain)
    near(plain, n64, n_off + H(ty) * (n64.abs() + n_off) + tiny(ty), "without weights")


def check_packed_of_computed(p, want, off):
    """The 8-bit form of values that are `want` within `off`: at most the step the rule gives them, half a step off, zero behind the row."""
    rows, dim = want.shape
    e = D(p.e)
    v = torch.nn.functional.pad(want.abs() + off, (0, pitch(dim) - dim)).reshape(rows, -1, 32).amax(2)
    step = torch.exp2(e - 127)
    assert bool(((step <= v / 63.5 * (1 + 1e-9)) | (e == 1)).all()), "a step is too large"
    assert bool((e >= 1).all())
    q = D(p.q)
    assert bool((q.abs() <= 127).all())
    if pitch(dim) > dim:
        assert bool((q[:, dim:] == 0).all())
    wide = step.repeat_interleave(32, 1)[:, :dim]
    near(values(p), want, wide / 2 + off, "8-bit form")


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("tx,ty", NORM_TYPES)
@pytest.mark.parametrize("rows,dim", NORM_SHAPES)
def test_layer_norm_backward(rows, dim, tx, ty, residual, kept):
    g = gen(rows * 1000 + dim + 1)
    x = rows_in(g, rows, dim, tx, 2.0, 0.7, extra=dim % 3)
    dy = rows_in(g, rows, dim, ty, 1.0, 0.2, extra=dim % 2, offset=1)
    gamma = (1 + 0.2 * torch.randn(dim, generator=g)).cuda()
    mean, rstd = D(x).mean(1).float().cuda(), (D(x).var(1, unbiased=False) + 1e-5).rsqrt().float().cuda()
    n64 = (D(x) - D(mean)[:, None]) * D(rstd)[:, None]
    n_off = 3 * U * n64.abs()
    if kept:
        p = dense.Packed.empty(rows, dim)
        dense.pack(n64.float().cuda(), p)
        n64, n_off = values(p), torch.zeros(rows, dim, dtype=torch.float64)
    r = rows_in(g, rows, dim, tx, 1.0) if residual else None
    dx = Guarded(rows, dim, tx)
    dgamma, dbeta = torch.full((dim,), 9.0, device="cuda"), torch.full((dim,), 9.0, device="cuda")

    def call(to, dg, db):
        dense.layer_norm_backward(dy, p if kept else x, gamma, None if kept else mean, rstd, to, dg, db, residual=r)

    call(dx.m, dgamma, dbeta)
    d64 = D(dy)
    g64 = d64 * D(gamma)
    m1, m2 = g64.mean(1, keepdim=True), (g64 * n64).mean(1, keepdim=True)
    R = D(rstd)[:, None]
    want = R * (g64 - m1 - n64 * m2) + (D(r) if residual else 0)
    m1_off = 58 * U * g64.abs().mean(1, keepdim=True)
    m2_off = 60 * U * (g64 * n64).abs().mean(1, keepdim=True) + (g64.abs() * n_off).mean(1, keepdim=True)
    off = R * (m1_off + n64.abs() * m2_off + n_off * m2.abs() + 5 * U * (g64.abs() + m1.abs() + (n64 * m2).abs())) + 2 * U * want.abs()
    near(dx.m, want, off + H(tx) * (want.abs() + off) + tiny(tx), "dx")
    assert dx.untouched()
    near(dgamma, (d64 * n64).sum(0), (rows + 2) * U * (d64 * n64).abs().sum(0) + (d64.abs() * n_off).sum(0), "dgamma")
    near(dbeta, d64.sum(0), rows * U * d64.abs().sum(0), "dbeta")
    again, dg, db = torch.empty(rows, dim, dtype=tx, device="cuda"), torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
    call(again, dg, db)
    assert torch.equal(again, dx.m) and torch.equal(dg, dgamma) and torch.equal(db, dbeta), "the same call gives the same bits"


def test_layer_norm_gradient_against_differences():
    """The formula's gradient against differences of the formula in 64 bits, and the kernels' against the formula (above)."""
    g = gen(5)
    x, gamma, beta, dy = torch.randn(4, 40, generator=g).double(), 1 + torch.rand(40, generator=g).double(), torch.randn(40, generator=g).double(), torch.randn(4, 40, generator=g)
    f = lambda x, gamma: (norm64(x, gamma, beta, 1e-5)[3] * dy.double()).sum()  # noqa: E731
    rstd = norm64(x, gamma, beta, 1e-5)[1][:, 0]
    X = x.float().cuda()
    dx, dg, db = torch.empty_like(X), torch.empty(40, device="cuda"), torch.empty(40, device="cuda")
    dense.layer_norm_backward(dy.cuda(), X, gamma.float().cuda(), x.mean(1).float().cuda(), rstd.float().cuda(), dx, dg, db)
    h = 1e-5                     # third differences of the formula are below 100 here: h^2 100 / 6 = 2e-9, and 1e-16 / h of rounding; fp32 dominates
    for r, c in ((0, 0), (1, 17), (3, 39)):
        up, down = x.clone(), x.clone()
        up[r, c] += h
        down[r, c] -= h
        diff = float(f(up, gamma) - f(down, gamma)) / (2 * h)
        assert abs(float(dx[r, c]) - diff) <= 1e-7 + 200 * U * (1 + abs(diff)) * 4
        up, down = gamma.clone(), gamma.clone()
        up[c] += h
        down[c] -= h
        diff = float(f(x, up) - f(x, down)) / (2 * h)
        assert abs(float(dg[c]) - diff) <= 1e-7 + 200 * U * (1 + abs(diff)) * 4


def test_layer_norm_in_place_and_rows_that_are_not_numbers():
    g = gen(11)
    x = rows_in(g, 50, 100, BF16)
    want = torch.empty_like(x)
    dense.layer_norm(x, None, None, want)
    y = x.clone()
    dense.layer_norm(y, None, None, y)
    assert torch.equal(y, want)
    x[3, 7], x[20, 99], x[31, 0] = math.nan, math.inf, -math.inf
    p, y = dense.Packed.empty(50, 100), torch.empty_like(x)
    dense.layer_norm(x, None, None, y, packed=p)
    bad = torch.zeros(50, dtype=torch.bool)
    bad[[3, 20, 31]] = True
    assert bool(torch.isnan(y[bad.cuda()]).all()) and torch.equal(y[~bad.cuda()], want[~bad.cuda()])
    assert bool((p.e[bad.cuda()] == 255).all()) and bool((p.e[~bad.cuda()] < 255).all())
    # a constant row: no spread, the norm is zero and finite
    x = torch.full((2, 77), 3.0, device="cuda")
    y = torch.empty_like(x)
    dense.layer_norm(x, None, None, y)
    assert bool((y == 0).all())


def test_layer_norm_backward_in_place():
    g = gen(12)
    dy, x, r = rows_in(g, 40, 200, F32), rows_in(g, 40, 200, F32), rows_in(g, 40, 200, F32)
    mean, rstd = x.mean(1), (x.var(1, unbiased=False) + 1e-5).rsqrt()
    want = torch.empty_like(x)
    dense.layer_norm_backward(dy, x, None, mean, rstd, want, residual=r)
    into = r.clone()
    dense.layer_norm_backward(dy, x, None, mean, rstd, into, residual=into)
    assert torch.equal(into, want)
    into = dy.clone()
    dense.layer_norm_backward(into, x, None, mean, rstd, into, residual=r)
    assert torch.equal(into, want)


def test_gradients_without_rows_are_zero():
    e = torch.empty(0, 40, device="cuda")
    dg, db = torch.full((40,), 5.0, device="cuda"), torch.full((40,), 5.0, device="cuda")
    dense.layer_norm_backward(e, e, None, torch.empty(0, device="cuda"), torch.empty(0, device="cuda"), e, dg, db)
    assert bool((dg == 0).all()) and bool((db == 0).all())
    w = torch.ones(24, 40, device="cuda")
    dw, dbias = torch.full((24, 40), 5.0, device="cuda"), torch.full((24,), 5.0, device="cuda")
    dense.linear_backward(torch.empty(0, 24, device="cuda"), e, w, None, dense.ACT_NONE, None, e, dw, dbias)
    assert bool((dw == 0).all()) and bool((dbias == 0).all())
    dense.linear_backward(torch.empty(0, 24, device="cuda"), dense.Packed.empty(0, 40), w, dense.Packed.empty(0, 24), dense.ACT_GELU, torch.empty(0, 24, device="cuda"), e,
                          dw.fill_(5), dbias.fill_(5))
    assert bool((dw == 0).all()) and bool((dbias == 0).all())


# ---- to 8 bits and back --------------------------------------------------------------------------------
@pytest.mark.parametrize("t", [F32, BF16, F16])
@pytest.mark.parametrize("rows,dim", [(1, 1), (3, 7), (5, 8), (2, 31), (4, 32), (3, 33), (2, 64), (5, 100), (3, 257), (40, 96)])
def test_pack_is_the_rule(rows, dim, t):
    g = gen(rows + dim)
    v = torch.randn(rows, dim, generator=g) * torch.exp(2 * torch.randn(rows, 1, generator=g))
    if dim > 40:
        v[0, 32:64] = 0
        v[1, 0] = 127.5                 # halves: ties to even, and the step that 127.5 steps need
        v[1, 1:9] = torch.tensor([0.5, 1.5, 2.5, -0.5, -1.5, 63.5, 64.0, -127.0])
    x = rows_in(g, rows, dim, t, extra=1, offset=1)
    x.copy_(v)
    p = dense.Packed.empty(rows, dim)
    p.q.fill_(99)
    dense.pack(x, p)
    q, e = packed_by_rule(x.cpu().float())
    assert torch.equal(p.e.cpu(), e) and torch.equal(p.q.cpu(), q)
    y = Guarded(rows, dim, t)
    dense.expand(p, y.m)
    near(y.m, values(p), H(t) * values(p).abs() + tiny(t) if t is F16 else torch.zeros(()).double(), "back")
    assert y.untouched()


def test_pack_at_the_ends_of_the_range():
    big, small = torch.finfo(F32).max, 2.0 ** -149
    v = torch.zeros(9, 40)
    v[0, 0], v[0, 1], v[0, 39] = big, -big, 1.0                       # e at its top: 63 steps, not 64 of 2^122
    v[1, 5] = math.inf
    v[2, 6], v[2, 39] = math.nan, 2.0
    v[3, 7], v[3, 8] = small, 2.0 ** -126                             # the smallest step: what is below half of it is zero
    v[4, 0] = 2.0 ** -120
    v[5, 0], v[5, 1] = 127.0, 1.0
    v[6, 0], v[6, 1] = 127.49999, 1.0
    v[7, 0], v[7, 1] = 127.5, 1.0
    v[8, 0], v[8, 1] = -128.0, 3.0
    p = dense.Packed.empty(9, 40)
    dense.pack(v.cuda(), p)
    q, e = packed_by_rule(v)
    assert torch.equal(p.e.cpu(), e) and torch.equal(p.q.cpu(), q)
    y = torch.empty(9, 40, device="cuda")
    dense.expand(p, y)
    back = y.cpu()
    assert bool(torch.isfinite(back[[0, 3, 4, 5, 6, 7, 8]]).all())
    assert bool(torch.isnan(back[1, :32]).all()) and bool((back[1, 32:] == 0).all())
    assert bool(torch.isnan(back[2, :32]).all()) and float(back[2, 39]) == 2.0
    # fp16: its largest numbers round up to 65536 in whole steps, and are handed back as the largest number
    h = torch.full((1, 32), 65504.0, dtype=F16, device="cuda")
    p, y = dense.Packed.empty(1, 32), torch.empty(1, 32, dtype=F16, device="cuda")
    dense.pack(h, p)
    dense.expand(p, y)
    assert bool((y == 65504.0).all())
    dense.expand(p, y, gamma=torch.full((32,), -1.0, device="cuda"))
    assert bool((y == -65504.0).all())


@pytest.mark.parametrize("t", [F32, BF16, F16])
@pytest.mark.parametrize("act", sorted(ACTS))
@pytest.mark.parametrize("rows,dim,affine", [(1, 1, False), (33, 45, True), (7, 256, False), (300, 64, True)])
def test_expand_through_weights_and_activation(rows, dim, affine, act, t):
    g = gen(dim)
    p = dense.Packed.empty(rows, dim)
    dense.pack(rows_in(g, rows, dim, F32, 3.0), p)
    gamma, beta = ((1 + torch.rand(dim, generator=g)).cuda(), torch.randn(dim, generator=g).cuda()) if affine else (None, None)
    y = Guarded(rows, dim, t, extra=2)
    dense.expand(p, y.m, ACTS[act], gamma, beta)
    z = values(p)
    off = torch.zeros_like(z)
    if affine:
        z = z * D(gamma) + D(beta)
        off = 2 * U * (values(p).abs() * D(gamma) + z.abs())
    want = act64(act, z)
    off = 1.13 * off + (act_off(z) if act in ("gelu", "silu") else 0)
    near(y.m, want, off + H(t) * (want.abs() + off) + tiny(t), "expand")
    assert y.untouched()


# ---- linear layers -------------------------------------------------------------------------------------
# (rows, in, out): single tokens and the sizes at which the kernel for few rows gives way; edges of a tile (128, 32), of a step (32, 64) and of a piece; long
# sums over few tiles (split); widths of one
LINEAR_SHAPES = [(1, 1, 1), (1, 64, 16), (1, 1664, 33), (2, 7, 5), (8, 130, 40), (16, 64, 32), (17, 96, 31), (33, 200, 65), (64, 72, 48), (65, 64, 128), (100, 33, 17),
                 (128, 128, 128), (129, 65, 127), (200, 31, 260), (130, 640, 129), (257, 1001, 70), (66, 3000, 130), (384, 192, 256), (300, 8, 300), (520, 320, 264),
                 (700, 2000, 640), (640, 4200, 1030), (300, 8200, 200)]
LINEAR_TYPES = [(F32, F32), (BF16, BF16), (F16, F16), (BF16, F32), (F16, F32)]


def linear64(x, w, bias, steps=2):
    """z, and what fp32 sums of its products may be off by."""
    x, w = D(x), D(w)
    z = x @ w.t() + (0 if bias is None else D(bias))
    return z, (steps * (x.shape[1] + 1) + 2) * U * (x.abs() @ w.abs().t()) + 2 * U * z.abs()


@pytest.mark.parametrize("t,ty", LINEAR_TYPES)
@pytest.mark.parametrize("rows,inp,out", LINEAR_SHAPES)
def test_linear(rows, inp, out, t, ty):
    g = gen(rows + inp + out)
    x = rows_in(g, rows, inp, t, extra=inp % 2, offset=out % 2)
    w = rows_in(g, out, inp, t, 1 / math.sqrt(inp), extra=3 * (rows % 2))
    bias = torch.randn(out, generator=g).cuda()
    r = rows_in(g, rows, out, ty, extra=1)
    z64, z_off = linear64(x, w, bias)
    for n, (act, with_bias, with_res, keep) in enumerate((("none", False, False, None), ("relu", True, False, "q"), ("gelu", True, True, "both"), ("silu", False, True, "z"))):
        b = bias if with_bias else None
        zz, zo = (z64, z_off) if with_bias else linear64(x, w, None)
        y = Guarded(rows, out, ty, extra=n)
        p, z = dense.Packed.empty(rows, out), Guarded(rows, out, t)
        if keep == "both":                                     # first into a tensor, then in 8 bits
            dense.linear(x, w, b, y.m, ACTS[act], r if with_res else None, z=z.m)
            first = y.m.clone()
            near(z.m, zz, zo + H(t) * (zz.abs() + zo) + tiny(t), "z")
            y.m.fill_(3.0)
        dense.linear(x, w, b, y.m, ACTS[act], r if with_res else None, z={None: None, "q": p, "both": p, "z": z.m}[keep])
        if keep == "both":
            assert torch.equal(first, y.m)
        if keep in ("q", "both"):
            check_packed_of_computed(p, zz, zo)
        if keep == "z":
            near(z.m, zz, zo + H(t) * (zz.abs() + zo) + tiny(t), "z")
        want = act64(act, zz) + (D(r) if with_res else 0)
        off = 1.13 * zo + (act_off(zz) if act in ("gelu", "silu") else 0) + U * want.abs()
        near(y.m, want, off + H(ty) * (want.abs() + off) + tiny(ty), f"y with {act}")
        assert y.untouched() and z.untouched()
        into = r.clone() if with_res else torch.empty(rows, out, dtype=ty, device="cuda")
        dense.linear(x, w, b, into, ACTS[act], into if with_res else None)                  # into the residual itself; the same bits
        assert torch.equal(into, y.m)


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("t,ty", LINEAR_TYPES)
@pytest.mark.parametrize("rows,inp,out", LINEAR_SHAPES)
def test_linear_backward(rows, inp, out, t, ty, kept):
    g = gen(rows + inp + out + 7)
    x, z = rows_in(g, rows, inp, t, extra=inp % 2, offset=1), rows_in(g, rows, out, t, 2.0, extra=out % 2)
    w = rows_in(g, out, inp, t, 1 / math.sqrt(inp), extra=rows % 2)
    dy = rows_in(g, rows, out, ty, extra=1)
    if kept:
        xp, zp = dense.Packed.empty(rows, inp), dense.Packed.empty(rows, out)
        dense.pack(x, xp)
        dense.pack(z, zp)
    for n, act in enumerate(sorted(ACTS)):
        x_act, gamma, beta = "none", None, None
        if kept and n % 2:
            x_act, gamma, beta = ("gelu", "relu")[n // 2], (1 + torch.rand(inp, generator=g)).cuda(), torch.randn(inp, generator=g).cuda()
        z64 = values(zp) if kept else D(z)
        want = D(dy) * slope64(act, z64)
        dz, dx, dw, db = Guarded(rows, out, t), Guarded(rows, inp, t), Guarded(out, inp, t), torch.full((out,), 9.0, device="cuda")
        dense.linear_backward(dy, xp if kept else x, w, zp if kept else z, ACTS[act], dz.m, dx.m, dw.m, db, x_act=ACTS[x_act], x_gamma=gamma, x_beta=beta)
        off = D(dy).abs() * (act_off(z64) if act in ("gelu", "silu") else 0) + U * want.abs()
        near(dz.m, want, off + H(t) * (want.abs() + off) + tiny(t), "dz")
        near(db, want.sum(0), rows * U * want.abs().sum(0) + off.sum(0), "dbias")
        h64 = D(dz.m)                                           # the products are of what was handed out
        if kept:
            taken = torch.empty(rows, inp, dtype=t, device="cuda")
            dense.expand(xp, taken, ACTS[x_act], gamma, beta)
        else:
            taken = x
        for got, a, b, what in ((dx, h64, D(w), "dx"), (dw, h64.t(), D(taken), "dw")):
            v, o = a @ b, (2 * a.shape[1] + 2) * U * (a.abs() @ b.abs())
            near(got.m, v, o + H(t) * (v.abs() + o) + tiny(t), what)
        assert dz.untouched() and dx.untouched() and dw.untouched()
        again = torch.empty(out, inp, dtype=t, device="cuda")
        dense.linear_backward(dy, xp if kept else x, w, zp if kept else z, ACTS[act], dz.m, None, again, None, x_act=ACTS[x_act], x_gamma=gamma, x_beta=beta)
        assert torch.equal(again, dw.m), "one output alone: the same bits"
    if t == ty:                                                 # no activation: dz is dy, written into itself or not at all
        a, b = torch.empty(rows, inp, dtype=t, device="cuda"), torch.empty(rows, inp, dtype=t, device="cuda")
        same = dy.clone()                                       # (how an operand lies decides how its sums are divided: the same in both calls)
        dense.linear_backward(same, None, w, None, dense.ACT_NONE, None, a, None)
        dense.linear_backward(same, None, w, None, dense.ACT_NONE, same, b, None, db)
        assert torch.equal(a, b) and torch.equal(same, dy)


@pytest.mark.parametrize("t", [F32, BF16, F16])
@pytest.mark.parametrize("rows,inp,out", [(1, 40, 24), (300, 48, 96), (700, 200, 96), (1500, 33, 20)])
def test_gradients_asked_for_together_or_alone(rows, inp, out, t):
    """A small layer's gradients come out of one launch; each asked for alone has the same bits.  A captured call repeats them."""
    g = gen(rows + inp)
    x, z, dy = rows_in(g, rows, inp, t), rows_in(g, rows, out, t, 2.0), rows_in(g, rows, out, t)
    w = rows_in(g, out, inp, t, 1 / math.sqrt(inp))
    dz = torch.empty_like(dy)

    def grads(dx=None, dw=None, db=None):
        dense.linear_backward(dy, x, w, z, dense.ACT_SILU, dz, dx, dw, db)

    def empty():
        return torch.empty_like(x), torch.empty_like(w), torch.empty(out, device="cuda")

    (dx, dw, db), (a, b, c) = empty(), empty()
    grads(dx, dw, db)
    grads(dx=a)
    grads(dw=b)
    grads(db=c)
    assert torch.equal(dx, a) and torch.equal(dw, b) and torch.equal(db, c)
    near(db, (D(dy) * slope64("silu", D(z))).sum(0), (D(dy).abs() * act_off(D(z))).sum(0) + (rows + 1) * U * (D(dy) * slope64("silu", D(z))).abs().sum(0), "dbias")
    for u in (a, b, c):
        u.fill_(7.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        grads(a, b, c)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        grads(a, b, c)
    for _ in range(3):
        for u in (a, b, c):
            u.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dx, a) and torch.equal(dw, b) and torch.equal(db, c)


@pytest.mark.parametrize("t", [BF16, F16, F32])
@pytest.mark.parametrize("inp", [255, 256, 257, 320, 449, 1000])
def test_tiles_with_copies_far_ahead(inp, t):
    """Sums of 4 to 16 steps over few tiles: the copies that are asked for beyond the end read as zero, whatever the step the sum ends in."""
    g = gen(inp)
    rows, out = 1100, 700
    x, w = rows_in(g, rows, inp, t), rows_in(g, out, inp, t, 1 / math.sqrt(inp))
    x[-1], w[-1] = math.inf, 1.0                                   # (the row behind which the copies go on)
    y = Guarded(rows, out, t)
    dense.linear(x, w, None, y.m)
    a, b = D(x)[:-1], D(w)
    v, o = a @ b.t(), (2 * inp + 2) * U * (a.abs() @ b.abs().t())
    near(y.m[:-1], v, o + H(t) * (v.abs() + o) + tiny(t), "y")
    assert not bool(torch.isfinite(y.m[-1]).any()) and y.untouched()


def test_the_shapes_reach_split_sums():
    """(300, 8200, 200) is added up from splits (bias, residual, kept z and activation come behind them), forward and in dw's long sum over rows."""
    assert dense.linear_workspace(300, 8200, 200, BF16) > 0
    assert dense.linear_workspace(30000, 256, 200, BF16, backward=True, dx=False, dbias=False) > 0


@pytest.mark.parametrize("t", [F32, BF16, F16])
@pytest.mark.parametrize("rows,inp,out", [(4113, 136, 3592), (4113, 3592, 136), (136, 3592, 4112), (30000, 256, 200)])
def test_large_tiles_and_long_sums(rows, inp, out, t):
    """Sizes at which the large tiles are taken, with edges, and sums over many rows; the reference in 64 bits on the GPU (contiguous operands)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(rows + inp + out)
    x, w = torch.randn(rows, inp, generator=g, device="cuda").to(t), (torch.randn(out, inp, generator=g, device="cuda") / math.sqrt(inp)).to(t)
    bias, r, dy = torch.randn(out, generator=g, device="cuda"), torch.randn(rows, out, generator=g, device="cuda"), torch.randn(rows, out, generator=g, device="cuda").to(t)
    y, p = Guarded(rows, out, F32), dense.Packed.empty(rows, out)
    dense.linear(x, w, bias, y.m, dense.ACT_RELU, residual=r, z=p)

    def within(got, want, tol, what):
        off = (got.double() - want).abs()
        assert bool((off <= tol).all()), (what, float((off - tol).max()))

    wt = w.double().t().contiguous()
    z = torch.mm(x.double(), wt) + bias.double()
    z_off = (2 * (inp + 1) + 2) * U * torch.mm(x.double().abs(), wt.abs()) + 2 * U * z.abs()
    want = z.clamp(min=0) + r.double()
    within(y.m, want, z_off + 2 * U * want.abs(), "y")
    assert y.untouched()
    step = torch.exp2(p.e.double() - 127).repeat_interleave(32, 1)
    within((p.q.double() * step)[:, :out], z, (step / 2)[:, :out] + z_off, "z in 8 bits")
    dz, dx, dw, db = torch.empty(rows, out, dtype=t, device="cuda"), Guarded(rows, inp, t), Guarded(out, inp, t), torch.empty(out, device="cuda")
    dense.linear_backward(dy, x, w, p, dense.ACT_RELU, dz, dx.m, dw.m, db)
    assert torch.equal(dz, torch.where(p.q[:, :out] > 0, dy, torch.zeros((), dtype=t, device="cuda")))
    d = dz.double()
    for got, a, b, what in ((dx, d, w.double(), "dx"), (dw, d.t().contiguous(), x.double(), "dw")):
        v = torch.mm(a, b)
        o = (2 * a.shape[1] + 2) * U * torch.mm(a.abs(), b.abs())
        within(got.m, v, o + H(t) * (v.abs() + o) + tiny(t), what)
        assert got.untouched()
    within(db, d.sum(0), rows * U * d.abs().sum(0), "dbias")


def test_linear_gradient_against_differences():
    g = gen(3)
    x, w, b, dy = (torch.randn(s, generator=g).double() for s in ((6, 20), (9, 20), (9,), (6, 9)))
    for act in ("gelu", "silu", "relu"):
        f = lambda x, w, b: (act64(act, x @ w.t() + b) * dy).sum()  # noqa: E731
        z = (x @ w.t() + b).float().cuda()
        dz, dx, dw, db = torch.empty(6, 9, device="cuda"), torch.empty(6, 20, device="cuda"), torch.empty(9, 20, device="cuda"), torch.empty(9, device="cuda")
        dense.linear_backward(dy.float().cuda(), x.float().cuda(), w.float().cuda(), z, ACTS[act], dz, dx, dw, db)
        h = 1e-6                 # second and third derivatives are below 1000 here: h^2 1000; relu's kink is 1e-3 away from every z
        assert float(z.abs().min()) > 1e-4
        for at, grad in ((0, dx), (1, dw), (2, db)):
            for i in (0, 11, 53):
                up, down = [x.clone(), w.clone(), b.clone()], [x.clone(), w.clone(), b.clone()]
                i %= up[at].numel()
                up[at].view(-1)[i] += h
                down[at].view(-1)[i] -= h
                diff = float(f(*up) - f(*down)) / (2 * h)
                assert abs(float(grad.reshape(-1)[i]) - diff) <= 1e-6 + 1e3 * U * (1 + abs(diff)), (act, at, i)


@pytest.mark.parametrize("rows", [5, 60, 300])
@pytest.mark.parametrize("t", [F32, BF16])
def test_values_that_are_not_numbers_stay_in_their_rows(rows, t):
    """A NaN in x reaches its own row alone (edges of a tile hold other rows beside it), one in w its own column."""
    g = gen(rows)
    x, w = rows_in(g, rows, 70, t), rows_in(g, 45, 70, t)
    want = torch.empty(rows, 45, dtype=t, device="cuda")
    dense.linear(x, w, None, want, dense.ACT_RELU)
    x[rows - 1, 69], w[44, 3] = math.nan, math.inf
    got, p = torch.empty_like(want), dense.Packed.empty(rows, 45)
    dense.linear(x, w, None, got, dense.ACT_RELU, z=p)
    assert torch.equal(got[:-1, :-1], want[:-1, :-1])
    assert bool(torch.isnan(got[-1]).all())
    assert bool((p.e[-1] == 255).all()) and bool((p.e[:, 1] == 255).all()) and bool((p.e[:-1, 0] < 255).all())


def test_a_layer_of_no_input_rows_beyond_and_offsets_past_32_bits():
    """Rows that lie further apart than 2^31 values together: 20 rows, 2^27 values from one to the next."""
    far = 1 << 27
    flat = torch.empty(19 * far + 4096, dtype=BF16, device="cuda")
    x = torch.as_strided(flat, (20, 200), (far, 1))
    to = torch.as_strided(flat, (20, 200), (far, 1), 2048)
    g = gen(1)
    v = torch.randn(20, 200, generator=g).to(BF16).cuda()
    x.copy_(v)
    want = torch.empty_like(v)
    dense.layer_norm(v, None, None, want)
    dense.layer_norm(x, None, None, to)
    assert torch.equal(to, want)
    p, q = dense.Packed.empty(20, 200), dense.Packed.empty(20, 200)
    dense.pack(v, p)
    dense.pack(x, q)
    assert torch.equal(p.q, q.q) and torch.equal(p.e, q.e)
    dense.expand(p, want)
    dense.expand(p, to)
    assert torch.equal(to, want)
    w = torch.randn(200, 200, generator=g).to(BF16).cuda()
    dense.linear(v, w, None, want)
    dense.linear(x, w, None, to)                                  # few rows
    assert torch.equal(to, want)
    dw, dw2 = torch.empty(20, 200, dtype=BF16, device="cuda"), torch.empty(20, 200, dtype=BF16, device="cuda")
    dy = torch.randn(300, 20, generator=g).to(BF16).cuda()
    y, y2 = torch.empty(300, 20, dtype=BF16, device="cuda"), torch.empty(300, 20, dtype=BF16, device="cuda")
    many = torch.randn(300, 200, generator=g).to(BF16).cuda()
    dense.linear(many, v, None, y)                                # w far apart
    dense.linear(many, x, None, y2)
    assert torch.equal(y, y2)
    dx, dx2 = torch.empty_like(many), torch.empty_like(many)
    dense.linear_backward(dy, many, v, None, dense.ACT_NONE, None, dx, dw)
    dense.linear_backward(dy, many, x, None, dense.ACT_NONE, None, dx2, dw2)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)


def test_more_threads_than_a_launch_holds():
    """2^30 and some narrow rows: over 2^32 threads at a few for a row.  The rows repeat, and so do the results, bit for bit: a row's are its own."""
    period, times = 65537, 16385
    rows = period * times
    assert rows > 1 << 30
    g = gen(8)

    def repeats(got, want):
        return all(bool((part == want).all()) for part in got.view(times, period, -1).split(1024))

    base = torch.randint(-64, 65, (period, 2), generator=g).to(BF16).cuda()         # (whole numbers: products and sums are exact, whichever kernel)
    x = base.repeat(times, 1)
    want, y = torch.empty_like(base), torch.empty_like(x)
    dense.layer_norm(base, None, None, want)
    dense.layer_norm(x, None, None, y)
    assert repeats(y, want)
    w = torch.tensor([[3.0, -5.0]], dtype=BF16, device="cuda")
    bias = torch.randn(1, generator=g).cuda()
    want, want_z = (torch.empty(period, 1, dtype=BF16, device="cuda") for _ in range(2))
    y, z = (torch.empty(rows, 1, dtype=BF16, device="cuda") for _ in range(2))
    dense.linear(base, w, bias, want, dense.ACT_SILU, None, want_z)
    dense.linear(x, w, bias, y, dense.ACT_SILU, None, z)
    assert repeats(y, want) and repeats(z, want_z)
    dy, want = torch.randn(period, 1, generator=g).to(BF16).cuda(), torch.empty_like(base)
    all_dy = dy.repeat(times, 1)
    dense.linear_backward(dy, base, w, None, dense.ACT_NONE, None, want, None)
    dense.linear_backward(all_dy, x, w, None, dense.ACT_NONE, None, x, None)         # (x is not read: no dw is asked for)
    assert repeats(x, want)
    del x, z, all_dy
    want, got = dense.Packed.empty(period, 1), dense.Packed.empty(rows, 1)
    dense.pack(dy, want)
    dense.pack(dy.repeat(times, 1), got)
    assert repeats(got.q, want.q) and repeats(got.e, want.e)
    back = torch.empty_like(dy)
    dense.expand(want, back)
    dense.expand(got, y)
    assert repeats(y, back)


def test_a_workspace_that_is_too_small_is_refused():
    x, w, y = torch.zeros(1000, 16384, device="cuda"), torch.zeros(300, 16384, device="cuda"), torch.zeros(1000, 300, device="cuda")
    need = dense.linear_workspace(1000, 16384, 300, F32)                # a long sum over few tiles is split
    assert need > 16
    with pytest.raises(HetError):
        dense.linear(x, w, None, y, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
    dense.linear(x, w, None, y, workspace=torch.empty(need, dtype=torch.uint8, device="cuda"))
    v = torch.zeros(1000, device="cuda")
    with pytest.raises(HetError):
        dense.layer_norm_backward(y, y, None, v, v, y, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))


def test_the_binding_refuses_shapes_and_types():
    x, w, y = torch.zeros(70, 40, device="cuda"), torch.zeros(30, 40, device="cuda"), torch.zeros(70, 30, device="cuda")
    v = torch.zeros(40, device="cuda")
    p = dense.Packed.empty(70, 40)
    for call in (lambda: dense.linear(x, w.t(), None, y), lambda: dense.linear(x, w, None, y[:69]), lambda: dense.linear(x.t().contiguous().t(), w, None, y),
                 lambda: dense.layer_norm(x, v, v, y), lambda: dense.pack(x[:69], p), lambda: dense.expand(p, y), lambda: dense.linear(x, w, None, y, z=p),
                 lambda: dense.linear_backward(y, x, w, None, 0, None, x, w, x_act=dense.ACT_RELU), lambda: dense.linear_backward(y, None, w, None, 0, None, x, w),
                 lambda: dense.layer_norm_backward(x, x, v, None, None, x)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: dense.linear(x, w.half(), None, y), lambda: dense.linear(x, w, v[:30].double(), y), lambda: dense.linear(x, w, v, y), lambda: dense.pack(x.double(), p),
                 lambda: dense.layer_norm(x, v[::2], v, x)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: dense.linear(x, w, None, y, act=7), lambda: dense.expand(p, x, act=-1), lambda: dense.linear_backward(y, x, w, None, dense.ACT_GELU, None, x, w),
                 lambda: dense.layer_norm(x, v, v, x, eps=-1.0), lambda: dense.layer_norm(x.bfloat16(), v, v, x), lambda: dense.linear(x[:1].expand(70, 40), w, None, y)):
        with pytest.raises(HetError):
            call()


# ---- streams, graphs, and all of them together -----------------------------------------------------------
class Block:
    """y = x + W2 gelu(W1 norm(x) + b1) + b2 in a float32 residual stream, with activations kept in 8 bits: as a model uses the calls."""

    def __init__(self, rows, dim, hidden, t, seed):
        g = gen(seed)
        self.t, self.rows, self.dim, self.hidden = t, rows, dim, hidden
        self.gamma, self.beta = (1 + 0.1 * torch.randn(dim, generator=g)).cuda(), (0.1 * torch.randn(dim, generator=g)).cuda()
        self.w1, self.w2 = (torch.randn(hidden, dim, generator=g) / math.sqrt(dim)).to(t).cuda(), (torch.randn(dim, hidden, generator=g) / math.sqrt(hidden)).to(t).cuda()
        self.b1, self.b2 = (0.1 * torch.randn(hidden, generator=g)).cuda(), (0.1 * torch.randn(dim, generator=g)).cuda()
        new = lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
        self.h, self.u, self.y = new(rows, dim, dtype=t), new(rows, hidden, dtype=t), new(rows, dim)
        self.rstd, self.n8, self.z8 = new(rows), dense.Packed.empty(rows, dim), dense.Packed.empty(rows, hidden)
        self.dz2, self.du, self.dz1, self.dh, self.dx = new(rows, dim, dtype=t), new(rows, hidden, dtype=t), new(rows, hidden, dtype=t), new(rows, dim, dtype=t), new(rows, dim)
        self.dw1, self.dw2, self.db1, self.db2 = new(hidden, dim, dtype=t), new(dim, hidden, dtype=t), new(hidden), new(dim)
        self.dgamma, self.dbeta = new(dim), new(dim)

    def forward(self, x):
        dense.layer_norm(x, self.gamma, self.beta, self.h, None, self.rstd, packed=self.n8)
        dense.linear(self.h, self.w1, self.b1, self.u, dense.ACT_GELU, z=self.z8)
        dense.linear(self.u, self.w2, self.b2, self.y, residual=x)

    def backward(self, dy):
        dense.linear_backward(dy, self.z8, self.w2, None, dense.ACT_NONE, self.dz2, self.du, self.dw2, self.db2, x_act=dense.ACT_GELU)
        dense.linear_backward(self.du, self.n8, self.w1, self.z8, dense.ACT_GELU, self.dz1, self.dh, self.dw1, self.db1, x_gamma=self.gamma, x_beta=self.beta)
        dense.layer_norm_backward(self.dh, self.n8, self.gamma, None, self.rstd, self.dx, self.dgamma, self.dbeta, residual=dy)

    def outputs(self):
        return [self.y, self.dx, self.dw1, self.dw2, self.db1, self.db2, self.dgamma, self.dbeta, self.n8.q, self.n8.e, self.z8.q, self.z8.e]


def block64(b, x, dy):
    """Forward and backward in 64 bits, with autograd, nothing kept in fewer bits."""
    p = [D(v).requires_grad_() for v in (x, b.w1, b.w2, b.b1, b.b2, b.gamma, b.beta)]
    x, w1, w2, b1, b2, gamma, beta = p
    mean = x.mean(1, keepdim=True)
    n = (x - mean) / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + 1e-5)
    z = (n * gamma + beta) @ w1.t() + b1
    y = x + (z * torch.special.ndtr(z)) @ w2.t() + b2
    return [y.detach()] + list(torch.autograd.grad(y, p, D(dy)))


@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("rows,dim,hidden", [(5, 40, 100), (300, 96, 250), (700, 260, 512)])
def test_a_block_against_its_gradient_in_64_bits(rows, dim, hidden, t):
    """Forward: roundings to t alone.  Backward: what is kept in 8 bits is off by at most 1/127 of its block's largest value, which is below 5 of the
    spread of normal values, and evenly so: sqrt(1/3) 5 / 127 = 2.3e-2 of the spread at most, n twice and z once.  In the 2-norm over all values such errors add
    in squares along the chain of five products: below 6e-2 of the gradient.  y keeps within the roundings of h, u and w's products: four of H(t)."""
    b = Block(rows, dim, hidden, t, 17)
    g = gen(18)
    x, dy = torch.randn(rows, dim, generator=g).cuda(), torch.randn(rows, dim, generator=g).cuda()
    b.forward(x)
    b.backward(dy)
    y, dx, dw1, dw2, db1, db2, dgamma, dbeta = block64(b, x, dy)
    rel = lambda got, want: float((D(got) - want).norm() / want.norm())  # noqa: E731
    assert rel(b.y, y) <= 4 * H(t) + 64 * U
    for got, want, what in ((b.dx, dx, "dx"), (b.dw1, dw1, "dw1"), (b.dw2, dw2, "dw2"), (b.db1, db1, "db1"), (b.dgamma, dgamma, "dgamma"), (b.dbeta, dbeta, "dbeta")):
        assert rel(got, want) <= 6e-2 + 4 * H(t), what
    assert rel(b.db2, db2) <= rows * U                                # nothing lies between dy and it


@pytest.mark.parametrize("t", [F32, BF16, F16])
def test_a_captured_block_replays_with_new_inputs(t):
    b, e = Block(333, 260, 520, t, 3), Block(333, 260, 520, t, 3)
    g = gen(4)
    x, dy = torch.randn(333, 260, generator=g).cuda(), torch.randn(333, 260, generator=g).cuda()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b.forward(x)
        b.backward(dy)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.forward(x)
        b.backward(dy)
    for _ in range(4):
        x.copy_(torch.randn(333, 260, generator=g))
        dy.copy_(torch.randn(333, 260, generator=g))
        for o in b.outputs():
            o.fill_(1)
        graph.replay()
        torch.cuda.synchronize()
        e.forward(x)
        e.backward(dy)
        torch.cuda.synchronize()
        for got, want in zip(b.outputs(), e.outputs()):
            assert torch.equal(got, want)


def test_two_streams_at_once():
    g = gen(8)
    blocks = [Block(700, 256, 512, BF16, 5), Block(650, 256, 512, BF16, 6)]
    data = [(torch.randn(b.rows, 256, generator=g).cuda(), torch.randn(b.rows, 256, generator=g).cuda()) for b in blocks]
    want = []
    for b, (x, dy) in zip(blocks, data):
        b.forward(x)
        b.backward(dy)
        want.append([o.clone() for o in b.outputs()])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for b, (x, dy), s in zip(blocks, data, streams):
            with torch.cuda.stream(s):
                for o in b.outputs():
                    o.fill_(1)
                b.forward(x)
                b.backward(dy)
    torch.cuda.synchronize()
    for b, w in zip(blocks, want):
        for got, x in zip(b.outputs(), w):
            assert torch.equal(got, x)
    # a stream named in the call: the workspace is that stream's too
    s = torch.cuda.Stream()
    b, (x, dy) = blocks[0], data[0]
    s.wait_stream(torch.cuda.current_stream())
    y = torch.zeros(300, 40, device="cuda")
    a, w = torch.ones(300, 4000, device="cuda"), torch.ones(40, 4000, device="cuda")
    torch.cuda.synchronize()
    dense.linear(a, w, None, y, stream=s)
    s.synchronize()
    assert bool((y == 4000).all())


# ---- sums beyond the type's range --------------------------------------------------------------------------
@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("t", [F32, BF16, F16])
def test_slopes_at_infinity(t, act):
    """A kept z that is infinite has the slope's limit, 1 or 0: not the NaN of infinity times nothing.  A NaN stays one.  (rows of whole chunks and odd ones)"""
    for out in (24, 13):
        g = gen(out)
        z, dy = rows_in(g, 9, out, t, 2.0), rows_in(g, 9, out, t)
        z[:, 0], z[:, 5], z[4, 9] = math.inf, -math.inf, math.nan
        x, w = rows_in(g, 9, 10, t), rows_in(g, out, 10, t)
        dz, dx, dw, db = torch.empty_like(dy), torch.empty_like(x), torch.empty_like(w), torch.empty(out, device="cuda")
        dense.linear_backward(dy, x, w, z, ACTS[act], dz, dx, dw, db)
        assert torch.equal(dz[:, 0], dy[:, 0]) and bool((dz[:, 5] == 0).all())
        assert bool(torch.isnan(dz[4, 9]))
        nan = torch.zeros_like(dz, dtype=torch.bool)
        nan[4, 9] = True
        assert bool(torch.isfinite(dz[~nan]).all())
        assert bool(torch.isnan(dx[4]).all()) and bool(torch.isfinite(torch.cat((dx[:4], dx[5:]))).all())
        assert bool(torch.isnan(dw[9]).all()) and bool(torch.isfinite(torch.cat((dw[:9], dw[10:]))).all())
        assert bool(torch.isnan(db[9])) and bool(torch.isfinite(torch.cat((db[:9], db[10:]))).all())


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("ty", [F16, F32])
@pytest.mark.parametrize("rows", [40, 300])
def test_sums_beyond_fp16_kept_in_fp16(rows, ty, act):
    """Two units whose sums are +-72000: kept as infinities, their outputs (0, and 72000 in fp32) and every gradient are what they would be."""
    g = gen(rows)
    x, w = torch.ones(rows, 8), torch.randn(20, 8, generator=g)
    w[3], w[4] = 9000.0, -9000.0
    x, w, dy = x.to(F16).cuda(), w.to(F16).cuda(), rows_in(g, rows, 20, ty, 0.01)
    y, z = torch.empty(rows, 20, dtype=ty, device="cuda"), torch.empty(rows, 20, dtype=F16, device="cuda")
    dense.linear(x, w, None, y, ACTS[act], z=z)
    assert bool((z[:, 3] == math.inf).all()) and bool((z[:, 4] == -math.inf).all())
    assert bool((y[:, 3] == (math.inf if ty is F16 else 72000.0)).all()) and bool((y[:, 4] == 0).all())
    dz, dx, dw, db = torch.empty_like(z), torch.empty_like(x), torch.empty_like(w), torch.empty(20, device="cuda")
    dense.linear_backward(dy, x, w, z, ACTS[act], dz, dx, dw, db)
    want = D(dy) * slope64(act, D(z).clamp(-1e3, 1e3))
    off = D(dy).abs() * act_off(D(z).clamp(-20, 20)) + U * want.abs()
    near(dz, want, off + H(F16) * (want.abs() + off) + tiny(F16), "dz")
    near(db, want.sum(0), rows * U * want.abs().sum(0) + off.sum(0), "dbias")
    h = D(dz)
    for got, a, b, what in ((dx, h, D(w), "dx"), (dw, h.t(), D(x), "dw")):
        v, o = a @ b, (2 * a.shape[1] + 2) * U * (a.abs() @ b.abs())
        near(got, v, o + H(F16) * (v.abs() + o) + tiny(F16), what)


# ---- the functions themselves ------------------------------------------------------------------------------
# gelu's negative part is |v| Phi(-|v|), with Phi(-x) = exp2(E), E = -x^2 / 2 log2(e) + q(x) and q a polynomial in x up to 8.  Relative to it: the fit is off by at most 6.1e-7.
# E: two roundings and the constant's of 0.72 x^2, E's own (E < 0.73 x^2 + 6); Horner's rule for q, by the running bound (the sum of every step's result times the power it
# is still multiplied by), 1, 3.1, 5.3, 8.3, 14.3, 30.1, 76.6, 210, 567 U at x = 0 .. 8; all of that times ln 2; exp2 1 ulp and the products: below U (10 + 3 x^2 + 1.5 2^x).
# Beyond 8, 8 Phi'(v) stands for |v| Phi(v), where Phi' goes on with q(8): x R(x), R(x) = Phi(-x) exp(x^2 / 2), grows by less than 1 / 64 from there on.
def gelu_tail_off(v):
    x = v.abs()
    near8 = x.clamp(max=8.0)
    return U * (10 + 3 * x * x + 1.5 * torch.exp2(near8)) + 6.1e-7 + torch.where(x > 8, 1 / 64, 0.0)


def lower_tail(v):
    """Phi(v) in 64 bits for negative v too (torch.special.ndtr is (1 + erf) / 2, which has lost half of its digits at -6 and all at -8.5)."""
    return torch.special.erfc(-v * 0.5 ** 0.5) / 2


# silu: exp's argument is off by 2 ulp of it, the exponential, the sum, the reciprocal and the product by 1 each: the sigmoid p is off by U (8 + 2.1 |v|) of it where v is
# negative, by 5 U otherwise.  Its slope p (1 + v (1 - p)): that times 1 + |v|, and the roundings of 1 - p and the products.
def sigmoid_off(v):
    return torch.where(v < 0, U * (8 + 2.1 * v.abs()), 5 * U)


@pytest.mark.parametrize("t", [F32, BF16, F16])
@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_activations_over_their_range(act, t):
    """Values and slopes on a grid, against 64 bits: down the negative tail to where the type ends, and small arguments."""
    v = torch.cat((torch.linspace(-14, 14, 28 * 2048 + 1), -torch.logspace(-20, 0, 500), torch.logspace(-20, 0, 500), torch.tensor([0.0, 8.0, -8.0, 30.0, -30.0])))
    least = 2.0 ** -126                     # an exponential below it may be zero; gelu's are multiplied by at most 8
    # values: of zero steps plus a weight, which is exactly the argument
    y = torch.empty(1, v.numel(), dtype=t, device="cuda")
    p = dense.Packed(torch.zeros(1, pitch(v.numel()), dtype=torch.int8, device="cuda"), torch.full((1, pitch(v.numel()) // 32), 127, dtype=torch.uint8, device="cuda"), v.numel())
    dense.expand(p, y, ACTS[act], None, v.cuda())
    v64 = D(v)
    want = (v64 * lower_tail(v64) if act == "gelu" else act64(act, v64))[None]
    off = (v64.abs() * lower_tail(-v64.abs()) * gelu_tail_off(v64) if act == "gelu" else want.abs() * sigmoid_off(v64)) + U * want.abs() + 8 * least
    near(y, want, off + H(t) * (want.abs() + off) + tiny(t), "values")
    # slopes: of arguments in the layer's type, with a gradient of ones
    z = v.to(t).cuda().view(1, -1)
    dz = torch.empty_like(z)
    dense.linear_backward(torch.ones_like(z), None, torch.zeros(z.shape[1], 1, dtype=t, device="cuda"), z, ACTS[act], dz, None, None)
    z64 = D(z)
    want, x = slope64(act, z64), z64.abs()
    if act == "gelu":
        bell = x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
        tail = lower_tail(-x)
        want = lower_tail(z64) + torch.sign(z64) * bell
        off = tail * (gelu_tail_off(z64) + torch.where(x > 8, 1.0, 0.0)) + bell * U * (8 + 2.2 * x * x) + 2 * U * (want.abs() + torch.where(z64 < 0, 0.0, 1.0)) + 8 * least
    else:
        s = torch.sigmoid(z64)
        off = s * (sigmoid_off(z64) + 4 * U) * (1 + x) + U * want.abs() + 100 * least          # (p below it, times 1 + |v|)
    near(dz, want, off + H(t) * (want.abs() + off) + tiny(t), "slopes")



# ---- z kept in both forms ----------------------------------------------------------------------------------
@pytest.mark.parametrize("t", [F32, BF16, F16])
@pytest.mark.parametrize("rows,inp,out", [(9, 200, 65), (33, 200, 65), (2048, 512, 1000), (2048, 512, 1024), (300, 8200, 200)])
def test_z_kept_whole_and_in_8_bits_at_once(rows, inp, out, t):
    """One call of the C entry may write both; the same bits as two calls.  Few rows, a small product, tiles with edges and without, split sums."""
    g = gen(rows + out)
    x, w = rows_in(g, rows, inp, t), rows_in(g, out, inp, t, 1 / math.sqrt(inp))
    bias, r = torch.randn(out, generator=g).cuda(), rows_in(g, rows, out, F32)
    want, want_z, want_p = torch.empty(rows, out, device="cuda"), torch.empty(rows, out, dtype=t, device="cuda"), dense.Packed.empty(rows, out)
    dense.linear(x, w, bias, want, dense.ACT_GELU, r, z=want_z)
    dense.linear(x, w, bias, want, dense.ACT_GELU, r, z=want_p)
    y, z, p = Guarded(rows, out, F32), Guarded(rows, out, t), dense.Packed.empty(rows, out)
    need = dense.linear_workspace(rows, inp, out, t)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    kind = {F32: dense.F32, BF16: dense.BF16, F16: dense.F16}[t]
    l = dense.linear_struct(rows=rows, inp=inp, out=out, type=kind, y_type=dense.F32, act=dense.ACT_GELU, x=x.data_ptr(), ldx=inp, w=w.data_ptr(), ldw=inp, bias=bias.data_ptr(),
                            residual=r.data_ptr(), ld_residual=out, y=y.m.data_ptr(), ldy=y.m.stride(0), z=z.m.data_ptr(), ldz=z.m.stride(0), zq=p.q.data_ptr(), ze=p.e.data_ptr(),
                            workspace=ws.data_ptr(), workspace_bytes=need)
    assert dense.load().het_linear(l, torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(y.m, want) and torch.equal(z.m, want_z) and torch.equal(p.q, want_p.q) and torch.equal(p.e, want_p.e)
    assert y.untouched() and z.untouched()


def test_norm_gradients_without_rows_kept_in_8_bits_are_zero():
    e, dg, db = torch.empty(0, 40, device="cuda"), torch.full((40,), 5.0, device="cuda"), torch.full((40,), 5.0, device="cuda")
    dense.layer_norm_backward(e, dense.Packed.empty(0, 40), None, None, torch.empty(0, device="cuda"), e, dg, db)
    assert bool((dg == 0).all()) and bool((db == 0).all())
