"""Operators on matrices whose rows are a distance apart, on paths that only those or long contractions reach."""
import pytest
import torch

import paper_2609_39350_b200 as hap
from test_gpu_loss_leads import reference
from test_gpu_operators import BF, D, F32, FP, U, close, gated_reference, loss_reference, normal, offsets_of, wide

pytestmark = pytest.mark.gpu


def beside(t, pad):
    """What lies between the rows of a matrix made by wide()."""
    full = torch.as_strided(t, (*t.shape[:-1], t.shape[-1] + pad), t.stride())
    return full[..., t.shape[-1]:]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("pads", [(8, 8), (8, 3), (3, 8), (3, 5)], ids=str)         # of the operands, of what is kept and written
@pytest.mark.parametrize("loads,F,H", [([70, 0, 133], 136, 200), ([3, 260], 64, 72), ([1, 1], 40, 48)], ids=str)
def test_gated_of_slices(loads, F, H, pads, dtype):
    off, o = offsets_of(loads)
    rows, E, (pi, po) = o[-1], len(loads), pads
    x, w = wide(normal(rows, H, dtype=dtype), pi), wide(normal(E, 2 * F, H, seed=1, dtype=dtype, scale=2.0 * H ** -0.5), pi)
    gu, h = wide(torch.zeros(rows, 2 * F, dtype=dtype, device="cuda"), po), wide(torch.zeros(rows, F, dtype=dtype, device="cuda"), po)
    hap.hap_expert_gated(x, w, off, gu=gu, h=h)
    dy, w2 = wide(normal(rows, H, seed=2, dtype=dtype), pi), wide(normal(E, H, F, seed=3, dtype=dtype, scale=H ** -0.5), pi)
    dgu, h2 = wide(torch.zeros(rows, 2 * F, dtype=dtype, device="cuda"), po), wide(torch.zeros(rows, F, dtype=dtype, device="cuda"), po)
    hap.hap_expert_gated_backward(dy, w2, off, gu, dgu=dgu, h=h2)
    for t in (gu, h, dgu, h2):
        assert beside(t, po).isnan().all()
    same = wide(gu.contiguous(), po)
    hap.hap_expert_gated_backward(dy, w2, off, same, dgu=same, want_h=False)
    assert torch.equal(same, dgu) and beside(same, po).isnan().all()
    for e in range(E):
        i, j = o[e], o[e + 1]
        z, zoff, ref, hoff = gated_reference(x[i:j], w[e], F)
        close(gu[i:j], z, zoff, dtype)
        close(h[i:j], ref, hoff, dtype)
        g, u = gu[i:j, :F].to(D), gu[i:j, F:].to(D)
        dh, s = dy[i:j].to(D) @ w2[e].to(D), dy[i:j].to(D).abs() @ w2[e].to(D).abs()
        doff, sig = (H + 8) * U * s, torch.sigmoid(g)
        close(dgu[i:j, :F], dh * u * (sig + g * sig * (1 - sig)), 1.1 * u.abs() * doff + (dh * u).abs() * (12 + 6 * g.abs()) * U, dtype)
        close(dgu[i:j, F:], dh * g * sig, g.abs() * doff + (dh * g).abs() * (12 + 2 * g.abs()) * U, dtype)
        close(h2[i:j], g * sig * u, (12 + 2 * g.abs()) * U * (g * u).abs(), dtype)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("pads", [(8, 8), (8, 3), (3, 8)], ids=str)
@pytest.mark.parametrize("rows,H,V", [(1, 64, 300), (5, 33, 77), (100, 200, 1003), (129, 72, 511), (300, 264, 1030)])
def test_loss_of_slices(rows, H, V, pads, dtype):
    pi, po = pads
    x, w = wide(normal(rows, H, dtype=dtype), pi), wide(normal(V, H, seed=1, dtype=dtype, scale=2.0 * H ** -0.5), pi)
    target = torch.randint(0, V, (rows,), generator=torch.Generator(device="cuda").manual_seed(7), device="cuda")
    if rows > 2:
        target[1::9] = -100
    grad = torch.full((), 0.75, device="cuda")
    dx, dw = wide(torch.zeros(rows, H, dtype=dtype, device="cuda"), po), wide(torch.zeros(V, H, dtype=dtype, device="cuda"), po)
    loss, lse = hap.hap_linear_cross_entropy(x, w, target)
    hap.hap_linear_cross_entropy_backward(x, w, target, lse, grad, dx=dx, dw=dw)
    for got, (ref, off), t in zip((loss, lse, dx, dw), loss_reference(x, w, target, grad.to(D), dtype), (F32, F32, dtype, dtype)):
        close(got, ref, off, t)
    if rows > 1:
        assert beside(dx, po).isnan().all()
    assert beside(dw, po).isnan().all()


def test_dx_in_parts_and_in_pieces():
    """Few rows and a vocabulary of more than one piece: dx's contraction is split in each of them."""
    rows, H, V = 900, 264, 120000
    x, w = normal(rows, H), normal(V, H, seed=1, scale=2.0 * H ** -0.5)
    target = torch.randint(0, V, (rows,), generator=torch.Generator(device="cuda").manual_seed(7), device="cuda")
    target[0], target[1], target[2] = 0, V - 1, 111615
    grad = torch.full((), 1.0, device="cuda")
    loss, lse = hap.hap_linear_cross_entropy(x, w, target)
    dx, dw = hap.hap_linear_cross_entropy_backward(x, w, target, lse, grad)
    zoff = (H + 8) * U * (x.to(D).abs() @ w.to(D).abs().T)
    for got, (ref, off), t in zip((loss, lse, dx, dw), reference(x, w, target, grad, BF, zoff, None), (F32, F32, BF, BF)):
        close(got, ref, off, t)


def whole(*shape, seed, dtype, most=3):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=gen, device="cuda").to(dtype)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("loads", [[130, 0, 3], [1], [400]], ids=str)
@pytest.mark.parametrize("N,K", [(136, 1025), (1032, 200), (264, 2056), (2049, 72), (72, 5000), (5000, 40)])
def test_long_products_of_whole_numbers(loads, N, K, dtype):
    """Sums of whole numbers below 2^24 are exact in fp32 in any order: no step may be missing, and no step be taken twice."""
    off, o = offsets_of(loads)
    rows, E = o[-1], len(loads)
    x, dy, w = whole(rows, K, seed=1, dtype=dtype), whole(rows, N, seed=2, dtype=dtype), whole(E, N, K, seed=3, dtype=dtype)
    of = torch.repeat_interleave(torch.arange(E, device="cuda"), torch.tensor(loads, device="cuda"))
    refs = [torch.cat([x[of == e].to(D) @ w[e].to(D).T for e in range(E)]), torch.cat([dy[of == e].to(D) @ w[e].to(D) for e in range(E)])]
    for form, a, ref in zip((hap.EXPERT_FORWARD, hap.EXPERT_GRAD_INPUT), (x, dy), refs):
        out = hap.hap_expert_matmul(a, w, off, form, out_dtype=F32)
        assert torch.equal(out.to(D), ref)
        hap.hap_expert_matmul(a, w, off, form, out=out, accumulate=True)
        assert torch.equal(out.to(D), 2 * ref)
        assert torch.equal(hap.hap_expert_matmul(a, w, off, form), ref.to(F32).to(dtype))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("pad", [0, 4, 3])
@pytest.mark.parametrize("loads", [[40000, 1], [1500, 0, 63, 2049]], ids=str)
def test_long_weight_gradients_of_whole_numbers(loads, pad, dtype):
    """pad 3: an output that no tensor map describes, from operands that have one."""
    off, o = offsets_of(loads)
    rows, E, N, K = o[-1], len(loads), 136, 264
    a, b = whole(rows, N, seed=1, dtype=dtype), whole(rows, K, seed=2, dtype=dtype)
    ref = torch.stack([a[o[e]:o[e + 1]].to(D).T @ b[o[e]:o[e + 1]].to(D) for e in range(E)])
    assert ref.abs().max() < 2 ** 24
    out = torch.zeros(E, N, K, device="cuda")
    out = wide(out, pad) if pad else out
    hap.hap_expert_matmul(a, b, off, hap.EXPERT_GRAD_WEIGHT, out=out)
    assert torch.equal(out.to(D), ref)
    hap.hap_expert_matmul(a, b, off, hap.EXPERT_GRAD_WEIGHT, out=out, accumulate=True)
    assert torch.equal(out.to(D), 2 * ref)
    assert not pad or beside(out, pad).isnan().all()
    assert torch.equal(hap.hap_expert_matmul(a, b, off, hap.EXPERT_GRAD_WEIGHT), ref.to(F32).to(dtype))
