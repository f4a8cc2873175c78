"""Measured entries of embedding, norms and router: the workspace, counted a second time, and plans made from them."""
import ctypes as C

import numpy as np
import pytest

import paper_2609_39350_b200 as hap
from gen import problems
from oracle import Oracle
from paper_2609_39350_b200.tokens import _lib
from test_measure_workspace import lists, share, up


def asked(name, *sizes):
    n = C.c_uint64()
    assert getattr(_lib(), name)(*sizes, C.byref(n)) == 0
    return n.value


def embedding(t, H, V):
    return up(8 * t) + 2 * up(2 * V * H) + 2 * up(2 * t * H) + up(asked("hap_embedding_backward_workspace", t, H, V))


def norm(t, H):
    return 4 * up(2 * t * H) + 4 * up(2 * H) + 2 * up(4 * t) + up(asked("hap_layer_norm_backward_workspace", t, H))


def router(t, H, E, k):
    ld = -(-E // 8) * 8
    return (3 * up(2 * t * H) + 2 * up(2 * E * H) + 2 * up(2 * t * ld) + 2 * up(2 * t * k * H) + 2 * up(4 * t * k) + up(8 * (E + 1)) + up(16) + 2 * up(4 * t * k)
            + up(asked("hap_expert_order_workspace", t, k, E)))


def layouts(pb):
    tokens = {max(1, int(b) * pb.S // int(cp)) for b in pb.mb_list for cp in pb.cp_list}
    for t in tokens:
        yield from (embedding(t, pb.H, share(pb.V, int(tp))) for tp in pb.tp_list)
        if pb.H <= 16384:
            yield norm(t, pb.H)
    if 0 < pb.E <= 1024 and 0 < pb.k <= 32:
        yield router(min(max(tokens), 8192), pb.H, pb.E, pb.k)


CASES = [
    dict(S=8192, H=1024, E=64, k=8, F_dense=0, F_exp=4096, V=32000, **lists([4, 8], [1], [1, 2, 4])),
    dict(S=4096, H=512, E=5, k=2, F_dense=0, F_exp=1000, V=1000, **lists([2, 3, 7], [1, 5], [1, 3])),
    dict(S=200, H=64, E=0, k=0, F_dense=64, F_exp=0, V=2000000, **lists([1], [1, 2], [1])),
    dict(S=10, H=20000, E=2000, k=2, F_dense=64, F_exp=64, V=1000, **lists([1], [1], [1])),
]


@pytest.mark.parametrize("change", CASES, ids=lambda c: f"H{c['H']}-E{c['E']}")
def test_workspace_holds_every_layout(change):
    pb = problems.tiny().copy(**change)
    assert hap.hap_measure_tokens_workspace(pb) == max(layouts(pb))


def test_measuring_refuses():
    pb = problems.tiny()
    for change in (dict(beta=4.0), dict(H=1023), dict(mb_list=np.zeros(0, np.int32)), dict(V=0), dict(k=9)):
        with pytest.raises(hap.HapError):
            hap.hap_measure_tokens_workspace(pb.copy(**change))
    with pytest.raises(hap.HapError):
        hap.hap_measure_tokens(pb, 2)


def shaped(pb, change):
    pb = pb.copy(**change)
    n = tuple(len(x) for x in (pb.tp_list, pb.cp_list, pb.mb_list))
    for name in ("tdf", "tdb", "tff", "tfb"):
        setattr(pb, name, np.ones((pb.T, *n, pb.N)))
    pb.tpre, pb.tpost = np.ones((pb.T, *n)), np.ones((pb.T, *n))
    return pb


@pytest.mark.gpu
@pytest.mark.parametrize("change", [CASES[0], CASES[1], CASES[3]], ids=lambda c: f"H{c['H']}-E{c['E']}")
def test_measuring_stays_inside_of_its_workspace(change):
    import torch
    pb = shaped(problems.tiny(), change)
    n = hap.hap_measure_tokens_workspace(pb)
    space = torch.full((n + (64 << 20),), 0x5A, dtype=torch.uint8, device="cuda")
    new, got = hap.hap_measure_tokens(pb, 1, workspace=space[:n])
    assert (space[n:] == 0x5A).all()
    assert (got["tpre"] > 0).all() and ((got["tnorm"] > 0).all() if pb.H <= 16384 else not got["tnorm"].any())
    assert got["croute"] > 0 if pb.E <= 1024 else got["croute"] == 0
    assert np.array_equal(new.tpre[1], got["tpre"]) and np.array_equal(new.tpre[0], pb.tpre[0]) and new.croute[1] == got["croute"] and new.croute[0] == pb.croute[0]
    # the same sizes are measured once
    tokens = np.array([[[max(1, b * pb.S // cp) for b in pb.mb_list] for cp in pb.cp_list] for _ in pb.tp_list])
    for t in np.unique(tokens):
        assert len({tuple(x) for x in got["tnorm"][tokens == t]}) == 1
    with pytest.raises(hap.HapError):
        hap.hap_measure_tokens(pb, 1, workspace=space[:n - 1])


@pytest.mark.gpu
def test_a_plan_from_measured_entries():
    pb = problems.tiny()
    new, got = hap.hap_measure_tokens(pb, 0)
    tokens, H = 8 * pb.S, pb.H
    # bytes that have to be moved, at twice the device's nominal rate: rows there and back, forwards and backwards
    assert got["croute"] * 3 > 2 * (2 * pb.k * 3 + 4) / 16000
    assert (got["tpre"].max() > 4 * tokens * H / 16000) and (got["tnorm"][0, 0, -1] > 4 * tokens * H / 16000).all()
    assert np.array_equal(new.tdf, pb.tdf) and np.array_equal(pb.tpre, problems.tiny().tpre)
    hp = hap.hap_problem_create(new)
    hap.hap_enumerate(hp)
    plan, _ = hap.hap_search_best(hp)
    hap.hap_problem_destroy(hp)
    _, _, best, _ = Oracle(new).search()
    assert plan["index"] == best["index"] and plan["T_iter"] == best["T_iter"]


@pytest.mark.gpu
def test_measuring_refuses_a_captured_stream():
    import torch
    pb = problems.tiny()
    space = torch.empty(hap.hap_measure_tokens_workspace(pb), dtype=torch.uint8, device="cuda")
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        with pytest.raises(hap.HapError):
            hap.hap_measure_tokens(pb, 0, workspace=space)
