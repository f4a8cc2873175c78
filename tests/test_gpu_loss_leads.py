"""The head's loss where its two passes have to agree: rows whose target leads by far, and long rows with exact logits.

The loss of a row whose target leads by L over V classes has the gradient p - 1 = -(sum of the other p), about V e^-L: whatever
the two passes form differently of the same logit stands beside that."""
import pytest
import torch

import paper_2609_39350_b200 as hap
from test_gpu_operators import BF, D, F32, FP, U, close, normal, rounding

pytestmark = pytest.mark.gpu


def reference(x, w, target, grad, dtype, zoff, at_target):
    """loss, lse, dx, dw and how far each may be off, for logits that are off by zoff and, in both passes, by the same.

    at_target: what p of the target may be off beside that (see below); None: as the others' p."""
    x, w, n, V = x.to(D), w.to(D), x.shape[0], w.shape[0]
    z = x @ w.T
    lse = torch.logsumexp(z, 1)
    rows = torch.arange(n, device="cuda")
    # a common error of all terms from forming exponents of logits, one of each term, sums over tiles and of tiles
    lse_off = zoff.amax(1) + (z.abs().amax(1) + lse.abs() + 4) * 2 * U + (256 + V / 256) * U
    loss = lse - z[rows, target]
    p = torch.exp(z - lse[:, None])
    poff = p * (zoff + lse_off[:, None] + (z.abs() + lse.abs()[:, None] + 4) * 2 * U) * 1.01
    d = p.clone()
    d[rows, target] = 0
    d[rows, target] = -d.sum(1)
    if at_target is not None:
        poff[rows, target] = at_target(z[rows, target], lse) + d[rows, target].abs() * 2 * zoff.amax(1)
    doff = poff + rounding(d, dtype) + 2.0 ** -24 * 2.0 ** -15
    g = float(grad)
    dx, dx_off = g * (d @ w), g * (doff @ w.abs() + (V + 8) * U * (d.abs() @ w.abs()))
    dw, dw_off = g * (d.T @ x), g * (doff.T @ x.abs() + (n + 8) * U * (d.abs().T @ x.abs()))
    return (loss, lse_off + zoff[rows, target] + U * loss.abs()), (lse, lse_off), (dx, dx_off), (dw, dw_off)


def both_passes(x, w, target, grad):
    loss, lse = hap.hap_linear_cross_entropy(x, w, target)
    return loss, lse, *hap.hap_linear_cross_entropy_backward(x, w, target, lse, grad)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("rows", [24, 160])
@pytest.mark.parametrize("H", [4096, 8192])
def test_gradients_of_rows_whose_target_leads(rows, H, dtype):
    """A logit that both passes form alike, and is off by whatever, leaves in lse - z only: the target's part of the exponent in
    lse and in p (half a unit of z log2 e and of lse log2 e each), lse's own rounding, two units of each exponential, two of
    the logarithm: (|z| + 2 |lse| + 16) 2^-24 in all.  And the additions to the row's sum, 128 in a part, its 32 slices and the
    parts, are off by half a unit each, or by all that is added (1 - p) where that is less."""
    V = 1000
    x, w = normal(rows, H, dtype=dtype), normal(V, H, seed=1, dtype=dtype, scale=0.5 * H ** -0.5)
    target = (torch.arange(rows, device="cuda") * 6) % V
    lead = torch.where(torch.arange(rows, device="cuda") % 2 == 0, 15.0, 25.0)[:, None]
    w[target] = (x.float() * lead / x.float().square().sum(1, keepdim=True)).to(dtype)
    grad = torch.full((), 1024.0, device="cuda")
    zoff = (H + 8) * U * (x.to(D).abs() @ w.to(D).abs().T)
    refs = reference(x, w, target, grad, dtype, zoff, lambda z, lse: (z.abs() + 2 * lse.abs() + 16) * U / 2 + torch.clamp(-torch.expm1(z - lse), max=(192 + V / 128) * U / 2))
    for got, (ref, off), t in zip(both_passes(x, w, target, grad), refs, (F32, F32, dtype, dtype)):
        close(got, ref, off, t)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("rows,H,V", [(3, 1032, 700), (130, 1025, 300), (129, 2056, 1001), (24, 5120, 777), (300, 5120, 520), (260, 8192, 300)])
def test_long_rows_with_exact_logits(rows, H, V, dtype):
    """Logits that are sums of sixteenths: exact in fp32 in any order and under truncation, so that no step may be missing."""
    gen = torch.Generator(device="cuda").manual_seed(rows + H)
    x = torch.randint(-1, 2, (rows, H), generator=gen, device="cuda").to(dtype)
    w = (torch.randint(-1, 2, (V, H), generator=gen, device="cuda") / 16).to(dtype)
    target = torch.randint(0, V, (rows,), generator=gen, device="cuda")
    grad = torch.full((), 1.0, device="cuda")
    refs = reference(x, w, target, grad, dtype, torch.zeros(rows, V, dtype=D, device="cuda"), None)
    for got, (ref, off), t in zip(both_passes(x, w, target, grad), refs, (F32, F32, dtype, dtype)):
        close(got, ref, off, t)
