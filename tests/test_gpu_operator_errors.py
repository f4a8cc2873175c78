"""A call that failed leaves nothing behind that a later, good call would be blamed for."""
import ctypes as C

import pytest
import torch

import paper_2609_39350_b200 as hap

pytestmark = pytest.mark.gpu


def test_status_asked_for_during_a_capture():
    """Waiting for the device is refused while a stream is captured; the step behind it is made, and says so."""
    runtime = C.CDLL("libcudart.so.12")                 # (the one that torch has loaded)
    side, graph = torch.cuda.Stream(), C.c_void_p()
    p, g, m, v = torch.zeros(300, device="cuda"), torch.ones(300, device="cuda"), torch.zeros(300, device="cuda"), torch.zeros(300, device="cuda")
    tensors = hap.hap_adamw_tensors([p], [g], [m], [v])
    x, w, off = torch.ones(9, 13, device="cuda", dtype=torch.bfloat16), torch.ones(1, 5, 13, device="cuda", dtype=torch.bfloat16), torch.tensor([0, 9], device="cuda")
    torch.cuda.synchronize()
    assert runtime.cudaStreamBeginCapture(C.c_void_p(side.cuda_stream), 1) == 0
    try:
        with pytest.raises(hap.HapError):
            hap.hap_operator_status()
    finally:
        runtime.cudaStreamEndCapture(C.c_void_p(side.cuda_stream), C.byref(graph))
        runtime.cudaGetLastError()
    hap.hap_adamw_step(tensors, 1, 0.5)
    assert (p < -0.49).all()
    assert (hap.hap_expert_matmul(x, w, off) == 13).all()
    assert hap.hap_operator_status() == 0


def test_the_same_tensor_twice_is_refused():
    """Tied weights listed twice, and states shared by two parameters, would be stepped twice at once."""
    p, q = torch.zeros(300, device="cuda"), torch.zeros(300, device="cuda")
    g, none = torch.ones(300, device="cuda"), torch.zeros(0, device="cuda")
    m, v, n, w = (torch.zeros(300, device="cuda") for _ in range(4))
    c = torch.zeros(300, device="cuda", dtype=torch.bfloat16)
    for args in (([p, p], [g, g], [m, n], [v, w]), ([p, q], [g, g], [m, m], [v, w]), ([p, q], [g, g], [m, n], [w, w])):
        with pytest.raises(hap.HapError):
            hap.hap_adamw_tensors(*args)
    with pytest.raises(hap.HapError):
        hap.hap_adamw_tensors([p, q], [g, g], [m, n], [v, w], copies=[c, c])
    hap.hap_adamw_step(hap.hap_adamw_tensors([p, none, q, none], [g, none, g, none], [m, none, n, none], [v, none, w, none]), 1, 0.5)
    assert torch.equal(p, q) and (p < -0.49).all()
