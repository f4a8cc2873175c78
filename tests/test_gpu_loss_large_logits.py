"""The head's loss of logits that are known to the last bit, the largest of them far above the others."""
import pytest
import torch

import paper_2609_39350_b200 as hap
from test_gpu_operators import BF, D, FP

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("V,at", [(128, 0), (128, 100), (1000, 300), (77, 5)])
@pytest.mark.parametrize("H", [64, 27], ids=["tiles", "plain"])
def test_loss_of_large_logits(H, V, at, dtype):
    """One logit is x_i, the others are 0.  Half a unit of x log2 e in the exponents' common part, half a unit of lse, two units
    of the exponential and as many of the logarithm; and for each addition of an e^-x, 128 in a part, its 32 slices and the parts,
    half a unit of the sum, or all that is added where that is less."""
    top = torch.arange(1, 241, device="cuda", dtype=torch.float32)
    x, w = torch.zeros(240, H, device="cuda", dtype=dtype), torch.zeros(V, H, device="cuda", dtype=dtype)
    x[:, 0], w[at, 0] = top.to(dtype), 1
    target = torch.full((240,), at, device="cuda")
    loss, lse = hap.hap_linear_cross_entropy(x, w, target)
    z = top.to(D)
    rest = (V - 1) * torch.exp(-z)
    want = torch.log1p(rest)
    off = (2 * z + 16) * 2.0 ** -24 + torch.clamp(rest, max=(192 + V / 128) * 2.0 ** -24)
    assert ((lse.to(D) - z - want).abs() <= off).all(), float(((lse.to(D) - z - want).abs() / off).max())
    assert ((loss.to(D) - want).abs() <= off + want * 2.0 ** -24).all(), float(((loss.to(D) - want).abs() / off).max())
    other = torch.full((240,), (at + 1) % V, device="cuda")
    loss, again = hap.hap_linear_cross_entropy(x, w, other)
    assert torch.equal(again, lse) and ((loss.to(D) - z - want).abs() <= off).all()
