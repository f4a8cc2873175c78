"""What the bindings ask of tensors, without a GPU: every answer to what does not fit is a HapError."""
import pytest
import torch

import paper_2609_39350_b200 as hap
from paper_2609_39350_b200 import operators, tokens

CHECKS = [
    lambda t: operators._matrix("t", t, 0, (torch.float32,)), lambda t: operators._matrices("t", t, 0, (torch.float32,), 3), lambda t: operators._vector("t", t, 0, torch.float32),
    lambda t: tokens._table("t", t, 0, torch.float32),
]


@pytest.mark.parametrize("check", CHECKS)
def test_tensors_without_strides(check):
    for t in (torch.zeros(3, 8).to_sparse(), torch.zeros(8).to_sparse(), torch.eye(8).to_sparse_csr(), torch.zeros(3, 8, device="meta"), torch.zeros(8), torch.zeros(3, 8), None, 5):
        with pytest.raises(hap.HapError):
            check(t)


@pytest.mark.gpu
def test_tensors_without_strides_on_the_device():
    x = torch.ones(3, 8, device="cuda")
    for t in (x.to_sparse(), x.to_sparse_csr()):
        for call in (lambda: hap.hap_route(hap.hap_routing(8, 2), t), lambda: hap.hap_expert_dispatch(x, t), lambda: hap.hap_layer_norm(x, w=t[0] if t.layout == torch.sparse_coo else t),
                     lambda: hap.hap_expert_matmul(x.half(), t, torch.tensor([0, 3], device="cuda"))):
            with pytest.raises(hap.HapError):
                call()
