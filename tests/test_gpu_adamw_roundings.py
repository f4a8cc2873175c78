"""AdamW's update of parameters that are held in 32 bits: what its own roundings leave."""
import pytest
import torch

import paper_2609_39350_b200 as hap
from test_gpu_operators import D, F32, FP, BF, adamw_reference, normal, read8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gtype", [F32, BF, FP])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("n,shift", [(300000, 0), (4099, 1)])
def test_update_of_parameters_at_zero(n, shift, bits, gtype):
    """Parameters at 0 are the update and nothing else.  With factors that are powers of two and without eps it is one root and
    one quotient of the moments, each rounded once: half a unit in the last place each, (1 + 2^-24)^2 - 1 in all."""
    p, g = torch.zeros(n + shift, device="cuda")[shift:], normal(n + shift, seed=1, dtype=gtype, scale=1e-2)[shift:]
    copy = torch.zeros(n + shift, dtype=BF, device="cuda")[shift:]
    if bits == 32:
        m, v, more = normal(n + shift, seed=2, dtype=F32, scale=1e-2)[shift:], normal(n + shift, seed=3, dtype=F32, scale=1e-2).square()[shift:], {}
        rm, rv = m.to(D), v.to(D)
    else:
        m, v = torch.zeros(n, dtype=torch.int8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
        more = dict(m_scale=[torch.zeros(-(-n // 256), device="cuda")], v_scale=[torch.zeros(-(-n // 256), device="cuda")])
        rm, rv = torch.zeros(n, dtype=D, device="cuda"), torch.zeros(n, dtype=D, device="cuda")
    g.masked_fill_(g == 0, 1e-2)
    _, rm, rv, _ = adamw_reference(p, g, rm, rv, 1, lr=2.0 ** -10, beta1=0.5, beta2=0.75, eps=0.0, weight_decay=0.0)
    hap.hap_adamw_step(hap.hap_adamw_tensors([p], [g], [m], [v], copies=[copy], **more), 1, 2.0 ** -10, 0.5, 0.75, 0.0, 0.0)
    want = -2.0 ** -9 * rm / (2 * rv.sqrt())
    off = (p.to(D) - want).abs() / want.abs().clamp(min=1e-30)
    assert off.max() <= 2.0 ** -23 * (1 + 2.0 ** -20), float(off.max() / 2.0 ** -24)
    assert torch.equal(copy, p.to(BF))


def test_update_of_small_moments():
    """Gradients whose squares are subnormal or 0 in 32 bits: the same definition, no value that is not finite."""
    g = torch.tensor([1e-19, -1e-20, 3e-21, 1e-23, 0.0], device="cuda")
    p, m, v = torch.zeros(5, device="cuda"), torch.zeros(5, device="cuda"), torch.zeros(5, device="cuda")
    hap.hap_adamw_step(hap.hap_adamw_tensors([p], [g], [m], [v]), 1, 1e-3, 0.9, 0.95, 1e-8, 0.0)
    z = torch.zeros(5, dtype=D, device="cuda")
    ref, rm, rv, off = adamw_reference(z, g, z, z, 1, weight_decay=0.0)
    assert torch.equal(m.to(D), rm) and torch.equal(v.to(D), rv) and ((p.to(D) - ref).abs() <= off + 1e-45).all()
