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


def test_sums_are_added_to_all_that_is_wanted():
    """A gradient that is wanted is not left out because no tensor is given for it."""
    x, dy = normal(40, 264), normal(40, 264, seed=1)
    _, mean, rstd = hap.hap_layer_norm(x)
    sums = lambda: torch.zeros(264, device="cuda")  # noqa: E731
    for given in (dict(dw=sums()), dict(db=sums()), {}):
        with pytest.raises(hap.HapError):
            hap.hap_layer_norm_backward(dy, x, None, rstd, mean=mean, accumulate=True, **given)
    with pytest.raises(hap.HapError):
        hap.hap_layer_norm_backward(dy, x, None, rstd, accumulate=True)
    _, dw, db = hap.hap_layer_norm_backward(dy, x, None, rstd, mean=mean)
    for given in (dict(dw=sums(), db=sums()), dict(dw=sums(), want_dw=False), dict(db=sums(), want_dw=False)):
        got = hap.hap_layer_norm_backward(dy, x, None, rstd, mean=mean, accumulate=True, **given)
        for name, i, want in (("dw", 1, dw), ("db", 2, db)):
            assert got[i] is given.get(name) and (got[i] is None or torch.equal(got[i], want))
    only = sums()
    assert torch.equal(hap.hap_layer_norm_backward(dy, x, None, rstd, dw=only, accumulate=True)[1], hap.hap_layer_norm_backward(dy, x, None, rstd)[1])
