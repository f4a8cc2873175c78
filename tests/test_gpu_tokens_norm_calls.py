"""Calls of the norms that their description allows and that are easily forgotten."""
import pytest
import torch

import paper_2609_39350_b200 as hap
from test_gpu_operators import BF, D, F32, U, close, normal, wide

pytestmark = pytest.mark.gpu


def test_a_mean_without_centring_is_none():
    """A tensor that is given for it is left as it was, and not handed on to the backward pass as a mean."""
    x, given = normal(40, 264), torch.full((40,), 7.0, device="cuda")
    y, mean, rstd = hap.hap_layer_norm(x, centred=False, mean=given)
    assert mean is None and (given == 7).all()
    assert torch.equal(y, hap.hap_layer_norm(x, centred=False)[0])
    dx, dw, db = hap.hap_layer_norm_backward(y, x, None, rstd, mean=mean)
    assert db is None and torch.equal(dx, hap.hap_layer_norm_backward(y, x, None, rstd)[0])
    assert hap.hap_layer_norm(x, mean=given)[1] is given
