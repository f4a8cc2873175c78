"""Calls that the operators on a token's way refuse, before any device work: checked without a GPU."""
import ctypes as C

import pytest

import paper_2609_39350_b200 as hap
from paper_2609_39350_b200.tokens import _lib, _Routing

INVALID, RANGE = 1, 4
A, B = 1 << 20, 1 << 21         # aligned addresses that are never read


def refused(call, good, changes, want=INVALID):
    for change in changes:
        assert call(**{**good, **change}) == want, change


def test_route_refuses():
    L = _lib()
    keep = []

    def spec(**c):
        r = dict(E=64, k=8, scores=0, groups=4, kept_groups=2, group_best=2, renormalise=1, scale=1.0) | c
        keep.append(_Routing(*r.values()))
        return C.addressof(keep[-1])

    def forward(r=None, dtype=0, rows=8, z=A, ld=64, bias=0, e=A, w=A):
        return L.hap_route(spec() if r is None else r, dtype, rows, z, ld, bias, e, w, None)

    def backward(r=None, dtype=0, rows=8, z=A, ld=64, e=A, g=A, dz=B, ldd=64):
        return L.hap_route_backward(spec() if r is None else r, dtype, rows, z, ld, e, g, dz, ldd, None)

    bad = [dict(E=0), dict(E=1025, groups=1, kept_groups=1), dict(k=0), dict(k=33), dict(E=4, k=5), dict(scores=2), dict(groups=0), dict(groups=33, E=66), dict(groups=3),
           dict(kept_groups=0), dict(kept_groups=5), dict(group_best=0)]
    for c in bad:
        assert forward(r=spec(**c)) == INVALID and backward(r=spec(**c)) == INVALID, c
    refused(forward, {}, [dict(r=0), dict(dtype=3), dict(dtype=-1), dict(rows=-1), dict(z=0), dict(ld=63), dict(e=0), dict(w=0), dict(z=A + 1), dict(dtype=2, z=A + 2), dict(e=A + 2),
                          dict(w=A + 1), dict(bias=A + 2)])
    refused(backward, {}, [dict(r=0), dict(dtype=3), dict(rows=-1), dict(z=0), dict(ld=63), dict(ldd=63), dict(e=0), dict(g=0), dict(dz=0), dict(dz=A), dict(dz=B + 1)])
    assert forward(rows=0, z=0, e=0, w=0) == 0 and backward(rows=0, z=0, e=0, g=0, dz=0) == 0
    refused(forward, {}, [dict(rows=1 << 40)], RANGE)


def test_order_refuses():
    L = _lib()
    n = C.c_uint64()

    def space(rows, k, E):
        assert L.hap_expert_order_workspace(rows, k, E, C.byref(n)) == 0
        return n.value

    assert space(0, 1, 1) == 0 and space(256, 8, 64) == 0 and 0 < space(32768, 8, 256) < 1 << 20
    for bad in ((-1, 1, 1), (1, 0, 1), (1, 33, 1), (1, 1, 0), (1, 1, 1025), (1 << 30, 2, 1)):
        assert L.hap_expert_order_workspace(*bad, C.byref(n)) == INVALID, bad
    assert L.hap_expert_order_workspace(1, 1, 1, None) == INVALID

    def call(rows=32768, k=8, first=0, E=256, e=A, off=A, p=A, ws=A, size=None):
        return L.hap_expert_order(rows, k, first, E, e, off, p, ws, space(32768, 8, 256) if size is None else size, None)

    refused(call, {}, [dict(rows=-1), dict(k=0), dict(E=0), dict(E=1025), dict(e=0), dict(off=0), dict(p=0), dict(e=A + 2), dict(off=A + 4), dict(p=A + 1), dict(ws=0), dict(ws=A + 64),
                       dict(size=space(32768, 8, 256) - 1)])


def test_rows_refuse():
    L = _lib()

    def dispatch(dtype=0, rows=8, k=2, H=64, placed=16, x=A, ldx=64, p=A, o=B, ldo=64):
        return L.hap_expert_dispatch(dtype, rows, k, H, placed, x, ldx, p, o, ldo, None)

    def combine(dtype=0, rows=8, k=2, H=64, placed=16, y=A, ldy=64, p=A, w=A, b=A, ldb=64, o=B, ldo=64):
        return L.hap_expert_combine(dtype, rows, k, H, placed, y, ldy, p, w, b, ldb, o, ldo, None)

    def backward(dtype=0, rows=8, k=2, H=64, placed=16, d=A, ldd=64, y=A, ldy=64, p=A, w=A, dy=B, lddy=64, dw=B):
        return L.hap_expert_combine_backward(dtype, rows, k, H, placed, d, ldd, y, ldy, p, w, dy, lddy, dw, None)

    sizes = [dict(dtype=3), dict(rows=-1), dict(rows=1 << 31), dict(k=0), dict(k=33), dict(H=0), dict(H=1 << 28), dict(placed=-1), dict(p=0), dict(p=A + 2)]
    refused(dispatch, {}, sizes + [dict(x=0), dict(o=0), dict(ldx=63), dict(ldo=63), dict(x=A + 1), dict(o=A + 1), dict(dtype=2, x=A + 2)])
    refused(combine, {}, sizes + [dict(y=0), dict(o=0), dict(ldy=63), dict(ldb=63), dict(ldo=63), dict(y=A + 1), dict(b=A + 1), dict(w=A + 2)])
    refused(backward, {}, sizes + [dict(d=0), dict(y=0), dict(ldd=63), dict(ldy=63), dict(lddy=63), dict(dy=A, lddy=72), dict(dw=A + 2), dict(dy=B + 1)])
    assert dispatch(rows=0, x=0, o=0, p=0) == 0 and combine(rows=0, y=0, o=0, p=0) == 0 and backward(dy=0, dw=0) == 0 and dispatch(placed=0, o=0) == 0


def test_embedding_refuses():
    L = _lib()
    n = C.c_uint64()

    def space(*a):
        assert L.hap_embedding_backward_workspace(*a, C.byref(n)) == 0
        return n.value

    for bad in ((-1, 8, 8), (1 << 31, 8, 8), (8, 0, 8), (8, 8, 0), (8, 8, 1 << 28)):
        assert L.hap_embedding_backward_workspace(*bad, C.byref(n)) == INVALID, bad
    assert L.hap_embedding_backward_workspace(1, 1, 1, None) == INVALID

    def forward(dtype=0, n=8, H=64, V=100, first=0, t=A, w=A, ldw=64, o=B, ldo=64):
        return L.hap_embedding(dtype, n, H, V, first, t, w, ldw, 1.0, o, ldo, None)

    def backward(dtype=0, out=0, acc=0, n=8, H=64, V=100, t=A, dy=A, ldy=64, dw=B, ldw=64, ws=A, size=None):
        return L.hap_embedding_backward(dtype, out, acc, n, H, V, 0, t, dy, ldy, 1.0, dw, ldw, ws, space(8, 64, 100) if size is None else size, None)

    sizes = [dict(dtype=3), dict(n=-1), dict(H=0), dict(V=0), dict(V=1 << 28), dict(t=0), dict(t=A + 4)]
    refused(forward, {}, sizes + [dict(w=0), dict(o=0), dict(ldw=63), dict(ldo=63), dict(w=A + 1)])
    refused(backward, {}, sizes + [dict(out=1), dict(dtype=2, out=0), dict(dy=0), dict(dw=0), dict(ldy=63), dict(ldw=63), dict(ws=0), dict(ws=A + 8), dict(size=space(8, 64, 100) - 1),
                                   dict(out=2, dw=B + 2)])
    assert forward(n=0, t=0, w=0, o=0) == 0 and backward(n=0, acc=1) == 0


def test_norm_refuses():
    L = _lib()
    n = C.c_uint64()
    assert L.hap_layer_norm_backward_workspace(100, 64, C.byref(n)) == 0 and n.value > 0
    need = n.value
    for bad in ((-1, 8), (8, 0), (8, 16385)):
        assert L.hap_layer_norm_backward_workspace(*bad, C.byref(n)) == INVALID, bad
    assert L.hap_layer_norm_backward_workspace(1, 1, None) == INVALID

    def forward(dtype=0, pt=0, centred=1, rows=100, H=64, x=A, ldx=64, w=A, b=A, eps=1e-5, y=B, ldy=64, m=A, r=A):
        return L.hap_layer_norm(dtype, pt, centred, rows, H, x, ldx, w, b, eps, y, ldy, m, r, None)

    def backward(dtype=0, pt=0, gt=0, acc=0, centred=1, rows=100, H=64, dy=A, ldy=64, x=A, ldx=64, w=A, m=A, r=A, b=0, ldb=0, dx=B, lddx=64, dw=B, db=B, ws=A, size=need):
        return L.hap_layer_norm_backward(dtype, pt, gt, acc, centred, rows, H, dy, ldy, x, ldx, w, m, r, b, ldb, dx, lddx, dw, db, ws, size, None)

    refused(forward, {}, [dict(dtype=3), dict(pt=1), dict(dtype=2, pt=0), dict(rows=-1), dict(H=0), dict(H=16385), dict(x=0), dict(y=0), dict(ldx=63), dict(ldy=63), dict(eps=-1.0),
                          dict(eps=float("nan")), dict(x=A + 1), dict(w=A + 1), dict(m=A + 2), dict(r=A + 2)])
    refused(backward, {}, [dict(dtype=3), dict(pt=1), dict(gt=1), dict(rows=-1), dict(H=0), dict(H=16385), dict(dy=0), dict(x=0), dict(r=0), dict(m=0), dict(ldy=63), dict(ldx=63), dict(lddx=63),
                           dict(b=A, ldb=63), dict(ws=0), dict(ws=A + 8), dict(size=need - 1), dict(centred=0), dict(dx=A, lddx=72), dict(gt=2, dw=B + 2)])
    assert forward(rows=0, x=0, y=0) == 0 and backward(rows=0, acc=1) == 0 and backward(dx=0, dw=0, db=0, ws=0) == 0


def test_the_binding_refuses():
    for bad in (dict(E=0), dict(k=9), dict(scores=2), dict(groups=3), dict(kept_groups=3), dict(group_best=0)):
        with pytest.raises(hap.HapError):
            hap.hap_routing(**{**dict(E=8, k=2, groups=2), **bad})
    import torch
    with pytest.raises((hap.HapError, RuntimeError, AssertionError)):
        hap.hap_route(hap.hap_routing(8, 2), torch.zeros(3, 8))
