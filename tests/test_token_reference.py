"""The references of the operators on a token's way: their gradients against differences, and hand-made rows."""
import math

import numpy as np
import pytest
import torch

import token_reference as ref

D = torch.float64


def normal(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=D)


def differences(f, x, h=1e-5):
    """The gradient of a sum by central differences: off by h^2 of the third derivatives and 1e-16 / h."""
    out = torch.zeros_like(x)
    for i in range(x.numel()):
        d = torch.zeros_like(x)
        d.view(-1)[i] = h
        out.view(-1)[i] = (f(x + d) - f(x - d)) / (2 * h)
    return out


@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [True, False])
def test_route_gradients_against_differences(scores, renormalise):
    z, g = normal(4, 9), normal(4, 3, seed=1)
    experts = torch.tensor([[8, 0, 3], [1, 2, -1], [-1, -1, -1], [4, 5, 6]])
    got = ref.route_gradients(z, experts, g, scores, renormalise, 2.5)
    want = differences(lambda x: (ref.weights_of(x, experts, scores, renormalise, 2.5) * torch.where(experts >= 0, g, 0)).sum(), z)
    assert torch.allclose(got, want, atol=1e-8, rtol=1e-7)


@pytest.mark.parametrize("centred", [True, False])
def test_norm_gradients_against_differences(centred):
    x, w, b, dy = normal(3, 7), normal(7, seed=1), normal(7, seed=2), normal(3, 7, seed=3)
    _, mean, rstd = ref.norm(x, w, b, 1e-3, centred)
    dx, dw, db = ref.norm_gradients(dy, x, w, mean, rstd, centred)
    f = lambda x, w, b: (ref.norm(x, w, b, 1e-3, centred)[0] * dy).sum()  # noqa: E731
    assert torch.allclose(dx, differences(lambda t: f(t, w, b), x), atol=1e-8, rtol=1e-7)
    assert torch.allclose(dw, differences(lambda t: f(x, t, b), w), atol=1e-8, rtol=1e-7)
    assert torch.allclose(db, differences(lambda t: f(x, w, t), b), atol=1e-8, rtol=1e-7)


def test_rows_worked_by_hand():
    inf = math.inf
    e, w = ref.route([0.0, math.log(3), 0.0, -inf], None, 2)
    assert e == [1, 0] and np.allclose(w, [0.75, 0.25])                 # equal ones in the order of their index
    e, w = ref.route([0.0, math.log(3), 0.0, -inf], None, 4, renormalise=False)
    assert e == [1, 0, 2, -1] and np.allclose(w, [0.6, 0.2, 0.2, 0])
    e, w = ref.route([0.0, 0.0, 0.0, 0.0], [0.0, 0.1, 0.3, 0.2], 2, scores="sigmoid", scale=2.0)
    assert e == [2, 3] and np.allclose(w, [1, 1])                       # the bias decides, the scores weigh
    # groups (0.5, 0.5) and (0.9, 0): by their best the second, by the sum of two the first
    z = [0.0, 0.0, math.log(9), -50.0]
    assert ref.route(z, None, 1, scores="sigmoid", groups=2, kept=1, best=1)[0] == [2]
    assert ref.route(z, None, 2, scores="sigmoid", groups=2, kept=1, best=2)[0] == [0, 1]
    assert ref.route([-inf] * 3, None, 2) == ([-1, -1], [0.0, 0.0])
    e, w = ref.route([-300.0, -301.0], None, 2, scores="sigmoid")
    assert e == [0, 1] and np.allclose(w, [1 / (1 + math.exp(-1)), 1 / (1 + math.e)])
    offsets, places = ref.order(np.array([[2, 0], [5, 2], [0, 0]]), 0, 3)
    assert offsets.tolist() == [0, 3, 3, 5] and places.tolist() == [[3, 0], [-1, 4], [1, 2]]
