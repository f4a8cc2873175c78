"""The router's rows one after the other, in every layout of its lanes: rows without an order, and warps that take several rows."""
import math

import pytest
import torch

import paper_2609_39350_b200 as hap
from test_gpu_operators import BF, F32, FP, normal
from test_gpu_tokens import check_route

pytestmark = pytest.mark.gpu
INF = math.inf

# sums of more than two values and groups that do not fit the lanes take a way of their own; (24, 2) has eight rows in a warp
SLOW = [(96, dict(k=6, groups=12, kept=2, best=3)), (1020, dict(k=8, groups=17, kept=3, best=2)), (24, dict(k=12, groups=2, kept=1, best=20)), (1008, dict(k=32, groups=9, kept=4, best=2))]


def named(x):
    return str(x) if isinstance(x, int) else "-".join(f"{k}{v}" for k, v in x.items())


@pytest.mark.parametrize("dtype", [BF, FP, F32])
@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,spec", SLOW, ids=named)
def test_rows_without_an_order_the_slow_way(E, spec, scores, dtype):
    """They have experts 0 .. k - 1 and weights NaN, in front of rows that are in order and between them."""
    rows, k = 41, spec["k"]
    spec = dict(spec, scores=scores, renormalise=True, scale=1.5)
    bad = [0, 1, 5, 6, 17, 40]
    for x in [math.nan, INF] if scores == "softmax" else [math.nan]:
        for several in (True, False):
            z = normal(rows, E, seed=3, dtype=dtype)
            for i, row in enumerate(bad if several else [0]):
                z[row, (i * 7 + E - 1) % E] = x
            experts = check_route(z, **spec)
            assert experts[0].tolist() == list(range(k))
    bias = normal(E, seed=4, dtype=F32, scale=0.1)
    for x in (math.nan, INF):
        bias[E // 2] = x                                    # no row has an order
        routing = hap.hap_routing(E, k, hap.SOFTMAX if scores == "softmax" else hap.SIGMOID, spec["groups"], spec["kept"], spec["best"])
        e, w = hap.hap_route(routing, normal(rows, E, seed=5, dtype=dtype), bias=bias)
        assert w.isnan().all() and (e == torch.arange(k, device="cuda")).all()
