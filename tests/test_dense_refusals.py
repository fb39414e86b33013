"""The dense layers' entry points: exported as declared, and what they refuse (no GPU needed: a refused call reaches none)."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2112_07221_amd import dense
from paper_2112_07221_amd.hetcache import HET_EINVAL, HET_OK, LIB_PATH

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 4096            # stands for a pointer: a refused call does not look behind it


def test_library_exports_every_declared_symbol():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "het_dense.h")).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(het_[a-z_]+)\s*\(", text))) == sorted(dense.EXPORTS)
    lib = C.CDLL(LIB_PATH)
    for n in dense.EXPORTS:
        assert hasattr(lib, n), n


def test_the_struct_is_the_headers():
    """Names and order of het_linear_t's fields, from the header's text."""
    text = open(os.path.join(ROOT, "include", "het_dense.h")).read()
    body = re.sub(r"/\*.*?\*/", "", re.search(r"typedef struct het_linear_t \{(.*?)\} het_linear_t;", text, re.S).group(1), flags=re.S)
    names = [n.strip(" *") for line in body.split(";") if line.strip() for n in re.sub(r"^\s*(const\s+)?\w+", "", line).split(",")]
    assert [{"in": "inp"}.get(n, n) for n in names] == list(dense.LINEAR_FIELDS)


def norm(lib, **kw):
    a = dict(x=P, tx=0, ldx=64, gamma=P, beta=P, y=P, ty=0, ldy=64, mean=None, rstd=None, q=None, e=None, rows=4, dim=64, eps=1e-5)
    a.update(kw)
    return lib.het_layer_norm(*a.values(), None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(y=None), dict(dim=0), dict(dim=-1), dict(dim=32769, ldx=32769, ldy=32769), dict(rows=-1), dict(rows=1 << 31),
                                 dict(eps=-1.0), dict(eps=float("nan")), dict(ldx=63), dict(ldy=63), dict(tx=1, ty=0), dict(tx=1, ty=2), dict(tx=3), dict(ty=-1),
                                 dict(q=P), dict(e=P), dict(q=P + 8, e=P)])
def test_layer_norm_refuses(bad):
    assert norm(dense.load(), **bad) == HET_EINVAL


def back(lib, **kw):
    a = dict(dy=P, ty=0, lddy=64, x=P, tx=0, ldx=64, mean=P, rstd=P, q=None, e=None, gamma=P, residual=None, ldr=0, dx=P, lddx=64, dgamma=P, dbeta=P,
             rows=4, dim=64, ws=P, bytes=1 << 20)
    a.update(kw)
    return lib.het_layer_norm_backward(*a.values(), None)


@pytest.mark.parametrize("bad", [dict(dy=None), dict(dx=None), dict(rstd=None), dict(mean=None), dict(x=None), dict(q=P), dict(e=P), dict(q=P + 1, e=P), dict(lddy=63),
                                 dict(ldx=63), dict(lddx=63), dict(residual=P, ldr=63), dict(ws=None), dict(ws=P + 4), dict(bytes=4 * 64 * 2 - 1), dict(dim=0),
                                 dict(rows=-1), dict(tx=2, ty=1), dict(tx=1, ty=0)])
def test_layer_norm_backward_refuses(bad):
    assert back(dense.load(), **bad) == HET_EINVAL


def test_pack_and_expand_refuse():
    lib = dense.load()
    ok = dict(x=P, t=1, ldx=40, q=P, e=P, rows=3, dim=40)
    for bad in (dict(x=None), dict(q=None), dict(e=None), dict(q=P + 8), dict(t=3), dict(ldx=39), dict(rows=-1), dict(rows=1 << 31), dict(dim=0),
                dict(dim=(1 << 20) + 1, ldx=1 << 21), dict(rows=(1 << 31) - 1, dim=1 << 10, ldx=1 << 10)):
        assert lib.het_pack(*{**ok, **bad}.values(), None) == HET_EINVAL, bad
    ok = dict(q=P, e=P, rows=3, dim=40, gamma=None, beta=None, act=0, y=P, t=1, ldy=40)
    for bad in (dict(y=None), dict(q=None), dict(e=None), dict(q=P + 8), dict(t=-1), dict(ldy=39), dict(rows=-1), dict(dim=0), dict(act=4), dict(act=-1)):
        assert lib.het_expand(*{**ok, **bad}.values(), None) == HET_EINVAL, bad


def linear_args(**kw):
    a = dict(rows=300, inp=256, out=128, type=1, y_type=1, act=2, x=P, ldx=256, w=P, ldw=256, bias=P, y=P, ldy=128, dy=P, lddy=128, dz=P, lddz=128, dx=P, lddx=256,
             dw=P, lddw=256, dbias=P, zq=P, ze=P, workspace=P, workspace_bytes=1 << 30)
    a.update(kw)
    return dense.linear_struct(**a)


COMMON = [dict(rows=-1), dict(rows=(1 << 31) - 1), dict(inp=0), dict(out=0), dict(inp=(1 << 20) + 1, ldx=1 << 21, ldw=1 << 21), dict(type=3), dict(type=0, y_type=1),
          dict(type=1, y_type=2), dict(act=4), dict(act=-1), dict(rows=(1 << 31) - 256, inp=1 << 10, ldx=1 << 10, ldw=1 << 10), dict(ldw=255), dict(ze=None)]


@pytest.mark.parametrize("bad", COMMON + [dict(x=None), dict(w=None), dict(y=None), dict(ldx=255), dict(ldy=127), dict(residual=P, ld_residual=127), dict(z=P, ldz=127),
                                          dict(zq=P + 8), dict(zq=None)])
def test_linear_refuses(bad):
    assert dense.load().het_linear(linear_args(**bad), None) == HET_EINVAL


@pytest.mark.parametrize("bad", COMMON + [dict(dy=None), dict(dz=None), dict(zq=None), dict(zq=None, ze=None), dict(zq=None, ze=None, z=P, ldz=127), dict(w=None),
                                          dict(x=None), dict(lddy=127), dict(lddz=127), dict(lddx=255), dict(lddw=255), dict(ldx=255), dict(xq=P), dict(xe=P),
                                          dict(xq=P + 8, xe=P), dict(x_act=9), dict(dz=None, act=0, y_type=0), dict(workspace=None), dict(workspace=P + 4),
                                          dict(workspace_bytes=0)])
def test_linear_backward_refuses(bad):
    assert dense.load().het_linear_backward(linear_args(**bad), None) == HET_EINVAL


def test_a_null_layer_is_refused():
    lib = dense.load()
    assert lib.het_linear(None, None) == lib.het_linear_backward(None, None) == lib.het_linear_workspace(None, 0) == HET_EINVAL


def test_calls_without_rows_have_nothing_to_do():
    lib = dense.load()
    assert norm(lib, rows=0, x=None, y=None) == HET_OK
    assert lib.het_pack(None, 1, 40, None, None, 0, 40, None) == HET_OK
    assert lib.het_expand(None, None, 0, 40, None, None, 0, None, 1, 40, None) == HET_OK
    assert lib.het_linear(linear_args(rows=0, x=None, y=None, zq=None, ze=None), None) == HET_OK
    assert back(lib, rows=0, dy=None, x=None, dx=None, mean=None, rstd=None, dgamma=None, dbeta=None) == HET_OK


def test_a_workspace_of_the_size_that_is_named_is_needed():
    lib = dense.load()
    for rows, inp, out, dtype in ((300, 4096, 128, torch.bfloat16), (257, 5000, 9, torch.float32), (700, 9000, 40, torch.float16)):
        need = dense.linear_workspace(rows, inp, out, dtype, backward=True)
        assert need > 0
        l = linear_args(rows=rows, inp=inp, out=out, type=dense.load() and dense._types[dtype], y_type=dense._types[dtype], ldx=inp, ldw=inp, lddx=inp, lddw=inp, lddy=out,
                        lddz=out, ldy=out, workspace_bytes=need - 1)
        assert lib.het_linear_backward(l, None) == HET_EINVAL
    assert dense.linear_workspace(1, 5000, 9, torch.float32, backward=True) == 0           # few rows' sums are ended where they are formed
    assert dense.linear_workspace(-1, 8, 8, torch.float32) == HET_EINVAL
    assert dense.layer_norm_workspace(4, 0) == HET_EINVAL


def test_the_binding_refuses_what_is_not_on_the_gpu():
    x, v = torch.zeros(4, 64), torch.zeros(64)
    p = dense.Packed.empty(4, 64, "cpu")
    assert p.rows == 4 and p.q.shape == (4, 64) and p.e.shape == (4, 2)
    assert dense.Packed.empty(2, 33, "cpu").q.shape == (2, 64)
    for call in (lambda: dense.layer_norm(x, v, v, x), lambda: dense.layer_norm_backward(x, x, v, v, v, x), lambda: dense.pack(x, p), lambda: dense.expand(p, x),
                 lambda: dense.linear(x, x, None, x), lambda: dense.linear_backward(x, x, x, None, 0, None, x, x), lambda: dense.pack(None, p), lambda: dense.pack(v, p)):
        with pytest.raises(TypeError):
            call()


def test_layer_norm_backward_of_no_rows_kept_in_8_bits():
    """What is kept of no rows has no address, and x is not given."""
    lib = dense.load()
    assert back(lib, rows=0, dy=None, x=None, ldx=0, dx=None, mean=None, rstd=None, dgamma=None, dbeta=None) == HET_OK
    assert back(lib, rows=1, ldx=0) == HET_EINVAL


def test_a_gradient_of_too_many_values_for_a_launch_is_refused():
    """dw of 2^40 values, with all of the workspace that is named for it."""
    lib = dense.load()
    n = 1 << 20
    big = dict(rows=8, inp=n, out=n, ldx=n, ldw=n, lddx=n, lddw=n, lddy=n, lddz=n, act=0, zq=None, ze=None)
    need = lib.het_linear_workspace(linear_args(**big), 1)
    assert need >= 0
    assert lib.het_linear_backward(linear_args(**big, workspace_bytes=need), None) == HET_EINVAL


def test_a_stream_of_another_device_is_refused():
    class Stream:
        cuda_stream, device_index = 40, 1

    assert dense._stream(Stream, 1) == 40
    with pytest.raises(ValueError):
        dense._stream(Stream, 0)
