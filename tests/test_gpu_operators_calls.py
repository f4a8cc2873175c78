"""Calls of the operators that their description allows and that are easily forgotten."""
import os
import subprocess
import sys

import pytest
import torch

import paper_2609_39350_b200 as hap
from test_gpu_operators import BF, D, F32, FP, U, close, loss_reference, normal, offsets_of, wide

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("rows", [1, 2, 9, 300])
@pytest.mark.parametrize("pad", [0, 3])
def test_rows_that_belong_to_no_expert(rows, pad):
    """Every output is left as it is."""
    off = torch.full((4,), min(rows, 2), dtype=torch.int64, device="cuda")
    E, N, K = 3, 72, 64
    at = lambda t: wide(t, pad) if pad else t  # noqa: E731
    x, dy, w, w2, gu = at(normal(rows, K)), at(normal(rows, N)), at(normal(E, N, K)), at(normal(E, N, K // 2)), at(normal(rows, K))
    for form, a, cols in ((hap.EXPERT_FORWARD, x, N), (hap.EXPERT_GRAD_INPUT, dy, K)):
        for dtype in (BF, F32):
            out = torch.full((rows, cols), 7.0, dtype=dtype, device="cuda")
            hap.hap_expert_matmul(a, w, off, form, out=out)
            hap.hap_expert_matmul(a, w, off, form, out=out, accumulate=True)
            assert (out == 7).all()
    kept, h = torch.full((rows, N), 7.0, dtype=BF, device="cuda"), torch.full((rows, N // 2), 7.0, dtype=BF, device="cuda")
    hap.hap_expert_gated(x, w, off, gu=kept, h=h)
    assert (kept == 7).all() and (h == 7).all()
    dgu, h = torch.full((rows, K), 7.0, dtype=BF, device="cuda"), torch.full((rows, K // 2), 7.0, dtype=BF, device="cuda")
    hap.hap_expert_gated_backward(dy, w2, off, gu, dgu=dgu, h=h)
    assert (dgu == 7).all() and (h == 7).all() and hap.hap_operator_status() == 0


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("pads", [(0, 0), (8, 3), (3, 8)], ids=str)
@pytest.mark.parametrize("N,K", [(264, 328), (8, 8), (40, 1000)])
def test_weight_gradients_in_16_bits_added_to(N, K, pads, dtype):
    off, o = offsets_of([90, 0, 301, 1])
    E, rows, (pi, po) = 4, o[-1], pads
    a, b = wide(normal(rows, N, dtype=dtype), pi), wide(normal(rows, K, seed=1, dtype=dtype, scale=0.1), pi)
    out = wide(normal(E, N, K, seed=2, dtype=dtype), po)
    before = out.to(D)
    hap.hap_expert_matmul(a, b, off, hap.EXPERT_GRAD_WEIGHT, out=out, accumulate=True)
    for e in range(E):
        g, x = a[o[e]:o[e + 1]].to(D), b[o[e]:o[e + 1]].to(D)
        s = g.abs().T @ x.abs()
        close(out[e], before[e] + g.T @ x, (len(g) + 8) * U * s + U * (before[e].abs() + s), dtype)
    assert torch.equal(out[1].to(D), before[1])


@pytest.mark.parametrize("N,K", [(1, 1), (3, 2), (1, 300), (300, 1), (5, 6)])
def test_products_of_the_smallest_sizes(N, K):
    for loads in ([1], [2], [1, 0, 5]):
        off, o = offsets_of(loads)
        E, rows = len(loads), o[-1]
        x, dy, w = normal(rows, K), normal(rows, N, seed=1), normal(E, N, K, seed=2)
        y, dx, dw = hap.hap_expert_matmul(x, w, off), hap.hap_expert_matmul(dy, w, off, hap.EXPERT_GRAD_INPUT), hap.hap_expert_matmul(dy, x, off, hap.EXPERT_GRAD_WEIGHT)
        for e in range(E):
            a, g, m = x[o[e]:o[e + 1]].to(D), dy[o[e]:o[e + 1]].to(D), w[e].to(D)
            close(y[o[e]:o[e + 1]], a @ m.T, (K + 8) * U * (a.abs() @ m.abs().T), BF)
            close(dx[o[e]:o[e + 1]], g @ m, (N + 8) * U * (g.abs() @ m.abs()), BF)
            close(dw[e], g.T @ a, (len(a) + 8) * U * (g.abs().T @ a.abs()), BF)


@pytest.mark.parametrize("rows", [7, 200])
def test_class_that_is_ignored(rows):
    """ignore_index may be a class: its rows add nothing, and it stays in the others' sums."""
    x, w = normal(rows, 64), normal(300, 64, seed=1, scale=0.25)
    target = (torch.arange(rows, device="cuda") * 43) % 300
    target[::3] = 5
    grad = torch.full((), 1.0, device="cuda")
    loss, lse = hap.hap_linear_cross_entropy(x, w, target, ignore_index=5)
    dx, dw = hap.hap_linear_cross_entropy_backward(x, w, target, lse, grad, ignore_index=5)
    refs = loss_reference(x, w, torch.where(target == 5, -100, target), grad.to(D), BF)
    for got, (ref, off), t in zip((loss, lse, dx, dw), refs, (F32, F32, BF, BF)):
        close(got, ref, off, t)
    assert not loss[::3].any() and not dx[::3].any()


def test_only_ignored_rows():
    x, w = normal(150, 64), normal(300, 64, seed=1)
    target = torch.full((150,), -100, device="cuda")
    loss, lse = hap.hap_linear_cross_entropy(x, w, target)
    dx, dw = hap.hap_linear_cross_entropy_backward(x, w, target, lse, torch.ones((), device="cuda"))
    assert not loss.any() and lse.isfinite().all() and not dx.any() and not dw.any()


FIRST = r"""
import sys
import torch
sys.path.insert(0, sys.argv[1])
import paper_2609_39350_b200 as hap
x, w, off = torch.ones(200, 64, device="cuda", dtype=torch.bfloat16), torch.ones(1, 72, 64, device="cuda", dtype=torch.bfloat16), torch.tensor([0, 200], device="cuda")
t, lse, one = torch.zeros(200, device="cuda", dtype=torch.int64), torch.full((200,), 70.0, device="cuda"), torch.ones((), device="cuda")
space = hap.hap_linear_cross_entropy_workspace(x, w[0])
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    if sys.argv[2] == "product":
        y = hap.hap_expert_matmul(x, w, off)
    elif sys.argv[2] == "weight":
        y = hap.hap_expert_matmul(x, x, off, hap.EXPERT_GRAD_WEIGHT)
    else:
        y, _ = hap.hap_linear_cross_entropy(x, w[0], t, workspace=space)
y.zero_()
graph.replay()
torch.cuda.synchronize()
want = dict(product=64.0, weight=200.0, loss=4.276666)[sys.argv[2]]         # (the last: log 72)
assert ((y.float() - want).abs() < 1e-4).all(), y
assert hap.hap_operator_status() == 0
print("DONE")
"""


@pytest.mark.parametrize("what", ["product", "weight", "loss"])
def test_a_process_whose_first_call_is_captured(what):
    r = subprocess.run([sys.executable, "-c", FIRST, ROOT, what], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "DONE" in r.stdout, r.stderr[-2000:]
