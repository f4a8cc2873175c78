"""Measured profiles: the operators' times as entries of a planning problem, and plans made from them."""
import numpy as np
import pytest
import torch

import paper_2609_39350_b200 as hap
from gen import problems
from oracle import Oracle


def _problem():
    pb = problems.tiny()
    pb.kind[:2] = problems.DENSE                    # both kinds of layer
    return pb


def test_measuring_refuses():
    pb = _problem()
    assert hap.hap_measure_workspace(pb) > 0
    for change in (dict(beta=4.0), dict(H=1023), dict(mb_list=np.zeros(0, np.int32)), dict(V=0), dict(k=9)):
        with pytest.raises(hap.HapError):
            hap.hap_measure_workspace(pb.copy(**change))
    with pytest.raises(hap.HapError):
        hap.hap_measure_profile(pb, 2)


@pytest.mark.gpu
def test_measured_profile_is_a_profile_and_is_planned_with():
    pb = _problem()
    new, got = hap.hap_measure_profile(pb, 1)
    for name in ("tff", "tfb", "tpost"):
        assert np.isfinite(got[name]).all() and (got[name] > 0).all()
    assert 0 < got["eta"] <= 1 and 0 <= got["gamma"] <= 1 and 0 < got["copt"] < 1
    assert got["tff"].shape == (len(pb.tp_list), len(pb.cp_list), len(pb.mb_list), 2) and got["tpost"].shape == got["tff"].shape[:3]
    # the other type and the caller's problem are as they were; what is not measured of a layer is kept
    for name in ("tdf", "tdb", "tff", "tfb", "tpost", "eta", "copt"):
        assert np.array_equal(getattr(new, name)[0], getattr(pb, name)[0])
        assert not np.array_equal(getattr(new, name)[1], getattr(pb, name)[1])
    assert np.allclose(new.tdf[1] - new.tff[1], pb.tdf[1] - pb.tff[1]) and np.allclose(new.tdb[1] - new.tfb[1], pb.tdb[1] - pb.tfb[1])
    assert np.array_equal(new.tff[1][..., 0], got["tff"][..., problems.DENSE]) and np.array_equal(new.tff[1][..., -1], got["tff"][..., problems.MOE])
    # work can be counted: no time is shorter than the work at four times the device's nominal rate
    tokens = np.array([[[b * pb.S / cp for b in pb.mb_list] for cp in pb.cp_list] for _ in pb.tp_list])
    width = np.array([[[pb.F_exp / tp for _ in pb.mb_list] for _ in pb.cp_list] for tp in pb.tp_list])
    assert (got["tff"][..., 1] > 6 * tokens * width * pb.H / 9e6).all()
    hp = hap.hap_problem_create(new)
    hap.hap_enumerate(hp)
    plan, _ = hap.hap_search_best(hp)
    hap.hap_problem_destroy(hp)
    costs, _, best, _ = Oracle(new).search()
    assert plan["index"] == best["index"] and plan["T_iter"] == best["T_iter"] and plan["n"] == best["n"]
    assert hap.hap_operator_status() == 0


@pytest.mark.gpu
def test_measuring_refuses_a_captured_stream():
    pb = _problem()
    space = torch.empty(hap.hap_measure_workspace(pb), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(hap.HapError):
            hap.hap_measure_profile(pb, 0, workspace=space)
    with pytest.raises(hap.HapError):
        hap.hap_measure_profile(pb, 0, workspace=space[:256])
