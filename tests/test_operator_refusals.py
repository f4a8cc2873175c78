"""Calls that the training operators refuse, before any device work: checked without a GPU."""
import ctypes as C

import pytest

import paper_2609_39350_b200 as hap
from paper_2609_39350_b200.operators import _AdamWOptions, _AdamWTensor

INVALID, RANGE = 1, 4
A = C.c_void_p(1 << 20)         # an aligned address that is never read
N0 = C.c_void_p(0)


def i32(x):
    return C.c_int32(x)


def i64(x):
    return C.c_int64(x)


def matmul(form=0, dtype=0, out=0, acc=0, E=2, rows=64, N=32, K=64, off=A, a=A, lda=64, b=A, ldb=64, o=A, ldo=64):
    return hap.load_library().hap_expert_matmul(i32(form), i32(dtype), i32(out), i32(acc), i32(E), i64(rows), i32(N), i32(K), off, a, i64(lda), b, i64(ldb), o, i64(ldo), N0)


@pytest.mark.parametrize("change", [dict(form=3), dict(form=-1), dict(dtype=2), dict(dtype=5), dict(out=1), dict(E=0), dict(E=1025), dict(rows=-1), dict(rows=1 << 30),
                                    dict(N=0), dict(K=-8), dict(off=N0), dict(a=N0), dict(b=N0), dict(o=N0), dict(lda=63), dict(ldb=32), dict(ldo=31),
                                    dict(a=C.c_void_p(4097)), dict(out=2, o=C.c_void_p(4098)), dict(off=C.c_void_p(4100))], ids=str)
def test_matmul_refuses(change):
    assert matmul(**change) == INVALID


def test_nothing_to_do_is_no_error():
    assert matmul(rows=0, a=N0, b=N0) == 0
    L = hap.load_library()
    assert L.hap_expert_gated(i32(0), i32(1), i64(0), i32(8), i32(8), A, N0, i64(8), N0, i64(8), N0, i64(0), N0, i64(8), N0) == 0
    o = _AdamWOptions(1e-3, 0.9, 0.999, 1e-8, 0.0, 1)
    assert L.hap_adamw_step(N0, i32(0), i32(0), i32(0), i32(0), i32(32), C.byref(o), N0, N0) == 0
    t = (_AdamWTensor * 1)()                    # a tensor without values needs no addresses
    assert L.hap_adamw_step(t, i32(1), i32(0), i32(0), i32(0), i32(32), C.byref(o), N0, N0) == 0


def test_gated_refuses():
    L = hap.load_library()

    def forward(dtype=0, E=1, rows=8, H=64, F=32, off=A, x=A, ldx=64, w=A, ldw=64, gu=A, ldgu=64, h=A, ldh=32):
        return L.hap_expert_gated(i32(dtype), i32(E), i64(rows), i32(H), i32(F), off, x, i64(ldx), w, i64(ldw), gu, i64(ldgu), h, i64(ldh), N0)

    def backward(ldy=64, ldw=32, gu=A, ldgu=64, dgu=C.c_void_p(1 << 21), lddgu=64, h=N0, ldh=0, F=32):
        return L.hap_expert_gated_backward(i32(0), i32(1), i64(8), i32(64), i32(F), A, A, i64(ldy), A, i64(ldw), gu, i64(ldgu), dgu, i64(lddgu), h, i64(ldh), N0)

    for bad in (dict(dtype=2), dict(E=0), dict(F=0), dict(H=0), dict(off=N0), dict(x=N0), dict(w=N0), dict(h=N0), dict(ldx=63), dict(ldw=63), dict(ldgu=63), dict(ldh=31), dict(F=1 << 28)):
        assert forward(**bad) == INVALID, bad
    for bad in (dict(ldy=63), dict(ldw=31), dict(gu=N0), dict(dgu=N0), dict(ldgu=63), dict(lddgu=63), dict(h=A, ldh=31), dict(dgu=A, lddgu=72)):
        assert backward(**bad) == INVALID, bad


def test_loss_refuses():
    L = hap.load_library()
    n = C.c_uint64()

    def space(rows, H, V):
        assert L.hap_linear_cross_entropy_workspace(i64(rows), i32(H), i64(V), C.byref(n)) == 0
        return n.value

    assert space(0, 64, 1000) == 0 and space(8192, 8192, 128000) < 512 << 20     # far below the 2 GB of the logits
    assert L.hap_linear_cross_entropy_workspace(i64(1), i32(0), i64(1), C.byref(n)) == INVALID
    assert L.hap_linear_cross_entropy_workspace(i64(-1), i32(8), i64(1), C.byref(n)) == INVALID
    assert L.hap_linear_cross_entropy_workspace(i64(1), i32(8), i64(1), N0) == INVALID

    def forward(dtype=0, rows=8, H=64, V=100, x=A, ldx=64, w=A, ldw=64, t=A, loss=A, lse=A, ws=A, size=None):
        return L.hap_linear_cross_entropy(i32(dtype), i64(rows), i32(H), i64(V), x, i64(ldx), w, i64(ldw), t, i64(-100), loss, lse, ws,
                                          C.c_uint64(space(8, 64, 100) if size is None else size), N0)

    def backward(grad=A, lse=A, dx=A, lddx=64, dw=A, lddw=64, ws=A):
        return L.hap_linear_cross_entropy_backward(i32(0), i64(8), i32(64), i64(100), A, i64(64), A, i64(64), A, i64(-100), lse, grad, dx, i64(lddx), dw, i64(lddw), ws,
                                                   C.c_uint64(space(8, 64, 100)), N0)

    for bad in (dict(dtype=2), dict(H=0), dict(V=0), dict(x=N0), dict(w=N0), dict(t=N0), dict(loss=N0), dict(lse=N0), dict(ldx=63), dict(ldw=63), dict(ws=N0),
                dict(ws=C.c_void_p(4097)), dict(size=space(8, 64, 100) - 1)):
        assert forward(**bad) == INVALID, bad
    for bad in (dict(grad=N0), dict(lse=N0), dict(lddx=63), dict(lddw=63), dict(ws=N0)):
        assert backward(**bad) == INVALID, bad


def test_adamw_refuses():
    L = hap.load_library()

    def step(bits=32, pt=0, gt=0, ct=0, scales=False, options=None, **fields):
        t = (_AdamWTensor * 1)()
        t[0].param = t[0].grad = t[0].m = t[0].v = 1 << 20
        t[0].count = 100
        if scales:
            t[0].m_scale = t[0].v_scale = 1 << 20
        for k, v in fields.items():
            setattr(t[0], k, v)
        o = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, step=1) | (options or {})
        return L.hap_adamw_step(t, i32(1), i32(pt), i32(gt), i32(ct), i32(bits), C.byref(_AdamWOptions(*o.values())), N0, N0)

    for bad in (dict(bits=16), dict(pt=3), dict(gt=1), dict(pt=1, gt=0), dict(bits=8), dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(param=(1 << 20) + 1),
                dict(m=(1 << 20) + 2), dict(copy=1 << 20), dict(pt=2, copy=1 << 20, ct=2), dict(bits=8, scales=True, m_scale=(1 << 20) + 2)):
        assert step(**bad) == INVALID, bad
    for bad in (dict(step=0), dict(beta1=1.0), dict(beta2=-0.1), dict(beta2=float("nan")), dict(eps=-1.0), dict(lr=float("inf")), dict(weight_decay=float("nan"))):
        assert step(options=bad) == INVALID, bad
    assert step(count=1 << 43) == RANGE
    assert L.hap_adamw_step(N0, i32(1), i32(0), i32(0), i32(0), i32(32), C.byref(_AdamWOptions(1e-3, 0.9, 0.9, 1e-8, 0, 1)), N0, N0) == INVALID
    assert L.hap_operator_status(N0) == INVALID
