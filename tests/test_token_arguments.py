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


class Long:
    """What the checks ask of a tensor of one row."""
    dtype = torch.float32

    def __init__(self, *shape):
        self.shape = torch.Size(shape)

    def stride(self):
        return (self.shape[-1], 1)

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20


def test_rows_whose_length_32_bits_do_not_hold():
    """A row of 2^32 + 64 values would be taken for one of 64."""
    for check in (CHECKS[0], CHECKS[3]):
        assert check(Long(1, 64))
        for c in (1 << 31, (1 << 32) + 64):
            for rows in (1, 2):
                with pytest.raises(hap.HapError):
                    check(Long(rows, c))
    for E in (0, 1025, (1 << 32) + 8):
        with pytest.raises(hap.HapError):
            tokens._order_bytes(100, 4, E)
    with pytest.raises(hap.HapError):
        tokens._embedding_bytes(100, (1 << 32) + 8, 100)


@pytest.mark.gpu
def test_rows_whose_length_32_bits_do_not_hold_on_the_device():
    x = torch.empty(1, (1 << 32) + 64, dtype=torch.bfloat16, device="cuda")
    places, one = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    offsets = torch.tensor([0, 1], device="cuda")
    for call in (lambda: hap.hap_layer_norm(x, y=x), lambda: hap.hap_expert_dispatch(x, places, out=x), lambda: hap.hap_expert_combine(x, places, out=x), lambda: hap.hap_embedding(one, x, out=x),
                 lambda: hap.hap_expert_matmul(x, x[None], offsets)):
        with pytest.raises(hap.HapError):
            call()


@pytest.mark.gpu
def test_tensors_without_strides_on_the_device():
    x = torch.ones(3, 8, device="cuda")
    for t in (x.to_sparse(), x.to_sparse_csr()):
        for call in (lambda: hap.hap_route(hap.hap_routing(8, 2), t), lambda: hap.hap_expert_dispatch(x, t), lambda: hap.hap_layer_norm(x, w=t[0] if t.layout == torch.sparse_coo else t),
                     lambda: hap.hap_expert_matmul(x.half(), t, torch.tensor([0, 3], device="cuda"))):
            with pytest.raises(hap.HapError):
                call()
