"""The workspace that measuring a profile asks for, against every set of buffers that it lays out: counted here a second time."""
import ctypes as C

import numpy as np
import pytest

import paper_2609_39350_b200 as hap
from gen import problems

UPDATE = 2 * (2 << 24) + 2 * (4 << 24)              # the optimizer's step: bf16 parameters and gradients, two fp32 states


def up(n):
    return -(-n // 256) * 256


def share(n, by):
    return -(-(-(-n // by)) // 8) * 8


def block(rows, H, F, E):
    """Offsets; x, y, dy, dx; g and u with their gradient; h; both weights with their gradients."""
    return up(8 * (E + 1)) + 4 * up(2 * rows * H) + 2 * up(4 * rows * F) + up(2 * rows * F) + 2 * (up(4 * E * F * H) + up(2 * E * F * H))


def head(rows, H, V):
    n = C.c_uint64()
    assert hap.load_library().hap_linear_cross_entropy_workspace(C.c_int64(rows), C.c_int32(H), C.c_int64(V), C.byref(n)) == 0
    return 2 * up(2 * rows * H) + 2 * up(2 * V * H) + up(8 * rows) + 2 * up(4 * rows) + up(4) + up(n.value)


def layouts(pb):
    tokens = {max(1, int(b) * pb.S // int(cp)) for b in pb.mb_list for cp in pb.cp_list}
    for t in tokens:
        for tp in map(int, pb.tp_list):
            yield from (block(t, pb.H, share(F, tp), 1) for F in (pb.F_dense, pb.F_exp) if F > 0)
            yield head(t, pb.H, share(pb.V, tp))
    if pb.E > 0 and pb.k > 0 and pb.F_exp > 0:
        t, e, F = max(tokens), min(pb.E, 8), share(pb.F_exp, 1)
        rows = max(e, t * pb.k * e // pb.E)
        yield block(t, pb.H, F, 1)                  # of the whole width, whatever the degrees are
        yield from (block(n * rows, pb.H, F, e) for n in (1, 2))
    yield UPDATE


def lists(tp, cp, mb):
    return {k: np.array(v, np.int32) for k, v in dict(tp_list=tp, cp_list=cp, mb_list=mb).items()}


CASES = [
    dict(S=8192, H=1024, E=64, k=1, F_dense=0, F_exp=4096, V=32000, **lists([4, 8], [1], [1, 2, 4])),
    dict(S=32768, H=5120, E=128, k=1, F_dense=0, F_exp=8192, V=202048, **lists([8], [1, 2], [1, 2, 4])),
    dict(S=65536, H=5120, E=160, k=6, F_dense=0, F_exp=1536, V=102400, **lists([8], [1], [1])),
    dict(S=4096, H=2048, E=16, k=1, F_dense=8192, F_exp=8192, V=32000, **lists([2], [1], [4])),
    dict(S=4096, H=512, E=4, k=2, F_dense=0, F_exp=1000, V=1000, **lists([2, 3, 7], [1, 5], [1, 3])),
    dict(S=200, H=64, E=0, k=0, F_dense=64, F_exp=0, V=2000000, **lists([1], [1, 2], [1])),         # a head that needs more for 100 rows than for 200
    dict(S=4096, H=1024, E=8, k=2, F_dense=4096, F_exp=4096, V=32000, **lists([1, 2], [1, 2], [1, 2])),
]


@pytest.mark.parametrize("change", CASES, ids=lambda c: f"H{c['H']}-E{c['E']}k{c['k']}-TP{min(c['tp_list'])}")
def test_workspace_holds_every_layout(change):
    pb = problems.tiny().copy(**change)
    assert hap.hap_measure_workspace(pb) == max(layouts(pb))


def test_workspace_of_the_configurations():
    for make in (problems.tiny, problems.small, problems.mixtral, problems.dsv2, problems.stress):
        pb = make()
        if pb.beta == 2.0:
            assert hap.hap_measure_workspace(pb) == max(layouts(pb))


@pytest.mark.gpu
def test_measuring_stays_inside_of_its_workspace():
    import torch
    pb = problems.tiny().copy(**{**CASES[0], **lists([4, 8], [1], [1, 2])})
    for name, n in (("tdf", pb.N), ("tdb", pb.N), ("tff", pb.N), ("tfb", pb.N)):
        setattr(pb, name, np.ones((pb.T, 2, 1, 2, n)))
    pb.tpre, pb.tpost = np.ones((pb.T, 2, 1, 2)), np.ones((pb.T, 2, 1, 2))
    n = hap.hap_measure_workspace(pb)
    space = torch.full((n + (64 << 20),), 0x5A, dtype=torch.uint8, device="cuda")
    _, got = hap.hap_measure_profile(pb, 1, workspace=space[:n])
    assert (space[n:] == 0x5A).all()
    assert (got["tff"][..., 1] > 0).all() and 0 < got["eta"] <= 1 and hap.hap_operator_status() == 0
    with pytest.raises(hap.HapError):
        hap.hap_measure_profile(pb, 1, workspace=space[:n - 1])
