"""Many rows, all different: blocks and warps that go on to further rows, in every layout of the router's lanes and for norms whose
buffers are used again and again."""
import math

import pytest
import torch

import paper_2609_39350_b200 as hap
import token_reference as ref
from test_gpu_operators import BF, D, F32, FP, U, close, normal, wide

pytestmark = pytest.mark.gpu
INF = math.inf


def route_of_all(z, bias, k, scores, groups, kept, best, renormalise, scale):
    """(experts, weights) of all rows at once in 64 bits, by sorts that keep the order of equal values."""
    z = z.to(D)
    rows, E = z.shape
    b = torch.zeros(E, dtype=D, device="cuda") if bias is None else bias.to(D)
    bad = (z.isnan() | (z == INF) if scores == "softmax" else z.isnan()).any(1)
    z = torch.where(bad.unsqueeze(1), 0, z)
    open_ = (z > -INF) & (b > -INF)
    s = torch.softmax(z, 1).nan_to_num(0) if scores == "softmax" else torch.sigmoid(z)
    v = torch.where(open_, z if bias is None else s + b, -INF)
    if groups > 1:
        of = torch.where(open_, s + b if bias is not None or best > 1 else z, -INF).view(rows, groups, -1)
        top = of.topk(min(best, of.shape[2]), 2).values
        total = torch.where(top > -INF, top, 0).sum(2).masked_fill(top[:, :, 0] == -INF, -INF)
        first = torch.sort(total, dim=1, descending=True, stable=True).indices[:, :kept]
        keep = torch.zeros(rows, groups, dtype=torch.bool, device="cuda").scatter_(1, first, True)
        v = v.masked_fill(~keep.repeat_interleave(E // groups, 1), -INF)
    v, at = torch.sort(v, dim=1, descending=True, stable=True)
    there, at = v[:, :k] > -INF, at[:, :k]
    c = torch.where(there, s.gather(1, at), 0)
    if renormalise:
        c = c / torch.where(there.any(1, keepdim=True), c.sum(1, keepdim=True), 1)
    return torch.where(bad.unsqueeze(1), torch.arange(k, device="cuda"), torch.where(there, at, -1)), torch.where(bad.unsqueeze(1), math.nan, scale * c)


# E, rows, what is asked for: lanes of a row 1, 2, 4, 8, 16 (8 and 16 experts each), 32 (16 and 32 each), with rows in whole eights and not,
# and layouts that are done by whole warps.  At least three turns of as many blocks as there may be.
MANY = [
    (8, 300_000, dict(k=2)), (7, 300_000, dict(k=3)), (16, 150_000, dict(k=4)), (13, 150_000, dict(k=3)), (32, 80_000, dict(k=6)), (30, 80_000, dict(k=4, groups=3, kept=2)),
    (64, 40_000, dict(k=6)), (60, 40_000, dict(k=4, groups=6, kept=3, best=2)), (128, 20_000, dict(k=8)), (100, 20_000, dict(k=8)), (160, 20_000, dict(k=6, groups=8, kept=3)),
    (250, 20_000, dict(k=8)), (512, 10_000, dict(k=8, groups=8, kept=4, best=2)), (500, 10_000, dict(k=9)), (1024, 10_000, dict(k=8)), (1022, 10_000, dict(k=32)),
    (544, 10_000, dict(k=8, groups=17, kept=5, best=2)),
    (96, 10_000, dict(k=6, groups=12, kept=2, best=3)), (24, 40_000, dict(k=6, groups=2, kept=1, best=20)), (1020, 10_000, dict(k=8, groups=17, kept=3, best=2)),
]


@pytest.mark.parametrize("scores,biased,dtype", [("softmax", False, BF), ("sigmoid", True, F32), ("softmax", True, F32), ("sigmoid", False, FP)], ids=str)
@pytest.mark.parametrize("E,rows,more", MANY, ids=lambda x: str(x) if isinstance(x, int) else "-".join(f"{k}{v}" for k, v in x.items()))
def test_route_of_rows_that_follow(E, rows, more, scores, biased, dtype):
    spec = dict(groups=1, kept=1, best=1, renormalise=scores == "softmax" or biased, scale=1.5, scores=scores) | more
    z = normal(rows, E, dtype=dtype, scale=1.5)
    z[normal(rows, E, seed=1, dtype=F32) > 1.7] = -INF
    z[::997, E // 2] = math.nan                             # rows without an order here and there, from the first on
    z[5::1009] = -INF
    bias = normal(E, seed=2, dtype=F32, scale=0.05) if biased else None
    routing = hap.hap_routing(E, spec["k"], hap.SOFTMAX if scores == "softmax" else hap.SIGMOID, spec["groups"], spec["kept"], spec["best"], spec["renormalise"], spec["scale"])
    e, w = hap.hap_route(routing, z, bias=bias)
    want_e, want_w = route_of_all(z, bias, **spec)
    assert torch.equal(e.long(), want_e)
    assert torch.equal(w.isnan(), want_w.isnan())
    good = ~want_w.isnan().any(1)
    # logits are within 16 of one another: an exponential is off by 16 2^-24 of itself and a few units, a sum by its terms
    close(w[good], want_w[good], (E + 40) * U * want_w[good].abs(), F32)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("centred", [True, False])
@pytest.mark.parametrize("rows,H", [(30_000, 72), (12_000, 264), (9_001, 1000), (9_001, 1001), (2_300, 5120), (2_301, 5121), (1_500, 8192), (900, 10_248), (800, 16_384)])
def test_norms_of_rows_that_follow(rows, H, centred, dtype):
    """Every row has a mean and a size of its own: a row of an earlier turn would be seen at once."""
    own = torch.arange(rows, device="cuda", dtype=F32).unsqueeze(1)
    x = (normal(rows, H, dtype=F32) * (1 + own % 7) + own % 11 - 5).to(dtype)
    dy, base = (normal(rows, H, seed=1, dtype=F32) * (1 + own % 5)).to(dtype), (normal(rows, H, seed=2, dtype=F32) + own % 13).to(dtype)
    w, b = normal(H, seed=3, dtype=dtype), normal(H, seed=4, dtype=dtype) if centred else None
    y, mean, rstd = hap.hap_layer_norm(x, w, b, centred=centred)
    X, W, DY = x.to(D), w.to(D), dy.to(D)
    Y, M, R = ref.norm(X, W, b.to(D) if centred else None, 1e-5, centred)
    diff = X - M.unsqueeze(1)
    var = (diff * diff).mean(1)
    em = (H + 8) * U * X.abs().mean(1) if centred else torch.zeros_like(M)
    rel = (2 * em * diff.abs().mean(1) + em * em + (H + 16) * U * var) / (var + 1e-5) + 8 * U
    if centred:
        close(mean, M, em, F32)
    close(rstd, R, rel * R, F32)
    xh = (diff * R.unsqueeze(1)).abs()
    close(y, Y, W.abs() * (xh * (rel + 8 * U).unsqueeze(1) + (em * R).unsqueeze(1) * (1 + rel).unsqueeze(1)) + U * (W.abs() * xh + (b.to(D).abs() if centred else 0)), dtype)
    m, r = mean.to(D) if centred else torch.zeros_like(M), rstd.to(D)
    xh, e = ((X - m.unsqueeze(1)) * r.unsqueeze(1)).abs(), (X.abs() + m.abs().unsqueeze(1)) * r.unsqueeze(1) * 2 * U
    g = (DY * W).abs()
    off = r.unsqueeze(1) * ((H + 16) * U * (g + g.mean(1, keepdim=True) + xh * (g * xh).mean(1, keepdim=True)) + e * (g * xh).mean(1, keepdim=True) + (xh + e) * (g * e).mean(1, keepdim=True))
    dx, dw, db = ref.norm_gradients(DY, X, W, m, r, centred)
    for add in (None, base):
        gdx, gdw, gdb = hap.hap_layer_norm_backward(dy, x, w, rstd, mean=mean, base=add)
        close(gdx, dx if add is None else dx + add.to(D), off if add is None else off + 2 * U * (add.to(D).abs() + dx.abs()), dtype)
        close(gdw, dw, (rows + 16) * U * (DY.abs() * xh).sum(0) + (DY.abs() * e).sum(0), dtype)
        if centred:
            close(gdb, db, (rows + 16) * U * DY.abs().sum(0), dtype)
