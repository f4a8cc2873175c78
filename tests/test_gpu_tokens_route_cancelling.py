"""Groups whose two values cancel: their sum is small, what it is off by goes with the values."""
import pytest
import torch

from test_gpu_operators import F32, normal
from test_gpu_tokens import check_route

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("size", [2, 5, 16])
@pytest.mark.parametrize("every", [2, 8])
@pytest.mark.parametrize("B", [64.0, 256.0, 65536.0, 1e20])
def test_groups_of_values_that_cancel(B, every, size, scores):
    """Biases of B and -B in some groups and of 0 in the rest; sums of the two are about 1e-5 apart, so that few are near in 32 bits."""
    rows, groups, E = 3000, 8, 8 * size
    z = normal(rows, E, seed=6, dtype=F32, scale=0.5).view(rows, groups, size)
    if scores == "softmax":                                 # (all groups of a row alike)
        z[:, :, 0] = normal(rows, 1, seed=8, dtype=F32, scale=0.5)
    z[:, :, 1] = -z[:, :, 0] + normal(rows, groups, seed=7, dtype=F32, scale=4e-5 if scores == "sigmoid" else 1.6e-4)
    z[:, :, 2:] = -float("inf")
    bias = torch.zeros(groups, size, device="cuda")
    bias[::every, 0], bias[::every, 1] = B, -B
    spec = dict(k=4, scores=scores, groups=groups, kept=3, best=2, renormalise=True, scale=1.0)
    check_route(z.reshape(rows, E), bias.reshape(E), **spec)


def test_groups_whose_sums_are_beyond_the_largest_number():
    """In 64 bits they are numbers like others."""
    z = normal(200, 16, seed=6, dtype=F32)
    bias = torch.tensor([3e38, 3.1e38, 3e38, 3.2e38, -3e38, -3e38, 3.3e38, -3.3e38, 0.0, 1.0, -3.1e38, -3.3e38, 3e38, 2.9e38, 0.0, 0.0], device="cuda")
    for kept in (1, 2, 3, 5, 6, 7):
        check_route(z, bias, k=2, scores="sigmoid", groups=8, kept=kept, best=2, renormalise=True, scale=1.0)
