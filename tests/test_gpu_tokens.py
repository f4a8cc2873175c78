"""Operators on a token's way (routing, experts' rows, embedding, layer norm) against their definitions in 64 bits.

Tolerances are bounds from arithmetic.  An operation in 32 bits is off by at most 2^-24 of its result, an exponential or a
quotient counts as 2^-22; a sum of n terms by (n + 8) 2^-23 of the sum of magnitudes, whatever its order; rounding to a type t adds
finfo(t).eps / 2 of the value, and half of the smallest subnormal of fp16."""
import math

import numpy as np
import pytest
import torch

import paper_2609_39350_b200 as hap
import token_reference as ref
from test_gpu_operators import BF, D, F32, FP, U, close, normal, wide

pytestmark = pytest.mark.gpu
INF = math.inf


# ---- routing --------------------------------------------------------------------------------------------------------------
def check_route(z, bias=None, exact_rows=None, **spec):
    """Experts equal, weights and gradients near; returns the experts."""
    rows, E = z.shape
    k = spec["k"]
    kinds = dict(softmax=hap.SOFTMAX, sigmoid=hap.SIGMOID)
    routing = hap.hap_routing(E, k, kinds[spec["scores"]], spec["groups"], spec["kept"], spec["best"], spec["renormalise"], spec["scale"])
    experts, weights = hap.hap_route(routing, z, bias=bias)
    zl, bl = z.double().cpu().tolist(), bias.double().cpu().tolist() if bias is not None else None
    want = [ref.route(row, bl, **spec) for row in zl]
    assert experts.cpu().tolist() == [e for e, _ in want]
    w = torch.tensor([x for _, x in want], dtype=D, device="cuda")
    finite = torch.where(z.isfinite(), z.double(), 0)
    spread = (finite.amax(1, keepdim=True) - finite.amin(1, keepdim=True)).clamp(min=0)
    off = (E + 16 + spread) * U
    assert torch.equal(weights.isnan(), w.isnan())
    good = ~w.isnan().any(1)
    close(weights[good], w[good], (off * w.abs())[good], F32)
    # backwards, from what the forward pass chose
    g = normal(rows, k, seed=9, dtype=F32)
    dz = hap.hap_route_backward(routing, z, experts, g)
    want = ref.route_gradients(z.double(), experts, g.double(), spec["scores"], spec["renormalise"], spec["scale"])
    s = torch.softmax(z.double(), 1).nan_to_num(0) if spec["scores"] == "softmax" else torch.sigmoid(z.double())
    there, at = experts >= 0, experts.clamp(min=0).long()
    c = torch.where(there, s.gather(1, at), 0)
    if spec["renormalise"]:
        c = c / torch.where(c.sum(1, keepdim=True) > 0, c.sum(1, keepdim=True), 1)
    mean = (g.double().abs() * c).sum(1, keepdim=True)
    size = torch.zeros_like(s).scatter_add_(1, at, torch.where(there, c * (g.double().abs() + mean), 0))
    if spec["scores"] == "softmax" and not spec["renormalise"]:
        size = size + s * mean
    # (of a sigmoid: s in 1 - s is off by 2^-22 of what is left)
    good = good & z.double().abs().nan_to_num(posinf=0, neginf=0).amax(1).lt(80)        # (beyond, the reference's sums of scores vanish)
    close(dz[good], want[good], ((off + 32 * U) * spec["scale"] * size)[good], z.dtype)
    return experts


SPECS = [
    (1, dict(k=1)), (2, dict(k=2)), (7, dict(k=3)), (8, dict(k=2)), (8, dict(k=8)), (33, dict(k=5)), (64, dict(k=8)), (100, dict(k=32)), (160, dict(k=6)),
    (256, dict(k=8)), (300, dict(k=7)), (512, dict(k=8)), (1024, dict(k=9)),
    (8, dict(k=2, groups=2)), (20, dict(k=4, groups=5, kept=2)), (64, dict(k=4, groups=8, kept=3, best=2)), (160, dict(k=6, groups=8, kept=3)),
    (160, dict(k=6, groups=8, kept=3, best=2)), (256, dict(k=8, groups=8, kept=4, best=2)), (256, dict(k=8, groups=8, kept=8, best=2)), (96, dict(k=6, groups=32, kept=5, best=2)),
    (96, dict(k=6, groups=12, kept=2, best=3)), (1020, dict(k=8, groups=17, kept=3, best=2)), (32, dict(k=3, groups=32, kept=3)), (24, dict(k=12, groups=2, kept=1, best=20)),
]


@pytest.mark.parametrize("dtype", [BF, FP, F32])
@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,more", SPECS, ids=lambda x: str(x) if isinstance(x, int) else "-".join(f"{k}{v}" for k, v in x.items()))
def test_route(E, more, scores, dtype):
    for i, (renormalise, biased) in enumerate([(True, False), (False, False), (True, True), (False, True)]):
        spec = dict(groups=1, kept=1, best=1, renormalise=renormalise, scale=1.0 if i % 2 else 2.5, scores=scores) | more
        spec["k"] = min(spec["k"], E // spec["groups"] * spec["kept"])
        for rows in (1, 41):
            z = normal(rows, E, seed=i, dtype=dtype, scale=2.0)
            if rows > 1:
                hide = normal(rows, E, seed=i + 50, dtype=F32)
                z[hide > 1.5] = -INF                        # single experts, whole rows, all but a few
                z[5] = -INF
                z[6, E // 2 + 1:] = -INF
                z[7, 1:] = -INF
                z[8] = z[8, 0].clone()                          # a row of ties
            check_route(z, normal(E, seed=i, dtype=F32, scale=0.1) if biased else None, **spec)


def test_route_rows_that_have_no_order():
    for scores, bad in (("softmax", [math.nan, INF]), ("sigmoid", [math.nan])):
        for x in bad:
            z = normal(6, 40, dtype=F32)
            z[1, 17], z[4, 39] = x, x
            z[5, 3:] = -INF
            spec = dict(k=4, scores=scores, groups=1, kept=1, best=1, renormalise=True, scale=1.0)
            routing = hap.hap_routing(40, 4, hap.SOFTMAX if scores == "softmax" else hap.SIGMOID)
            e, w = hap.hap_route(routing, z)
            assert e[1].tolist() == e[4].tolist() == [0, 1, 2, 3] and w[[1, 4]].isnan().all() and not w[[0, 2, 3, 5]].isnan().any()
            assert e[5, 3].item() == -1 and w[5, 3] == 0
            check_route(z, **spec)
    z = normal(3, 40, dtype=F32)
    z[1, 5] = INF                                           # a sigmoid's score of 1
    e, w = hap.hap_route(hap.hap_routing(40, 2, hap.SIGMOID, renormalise=False), z)
    assert e[1, 0] == 5 and w[1, 0] == 1
    bias = torch.zeros(40, device="cuda")
    bias[7] = -INF                                          # an expert that is off
    e, _ = hap.hap_route(hap.hap_routing(40, 32, hap.SIGMOID), normal(30, 40, dtype=F32), bias=bias)
    assert not (e == 7).any()
    for x in (math.nan, INF):
        bias[7] = x
        e, w = hap.hap_route(hap.hap_routing(40, 3, hap.SIGMOID, groups=4, kept_groups=2), normal(30, 40, dtype=F32), bias=bias)
        assert w.isnan().all() and (e == torch.arange(3, device="cuda")).all()


@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups,best", [(1, 1), (4, 1), (4, 2)])
def test_route_of_values_that_32_bits_cannot_tell_apart(scores, groups, best):
    """Biases that bring all values of a row to one number but for the bias's own rounding: the order is that in 64 bits."""
    E = 64
    z = normal(1, E, seed=3, dtype=F32)
    s = np.array(ref.score(z[0].double().cpu().tolist(), scores))
    bias = torch.tensor((0.75 - s).astype(np.float32), device="cuda")
    spec = dict(k=8, scores=scores, groups=groups, kept=max(1, groups // 2), best=best, renormalise=True, scale=1.0)
    check_route(z.repeat(5, 1), bias, **spec)
    rows = z.repeat(40, 1)
    rows[:, ::3] += normal(40, 22, seed=4, dtype=F32, scale=1e-7)      # and some that it can
    check_route(rows, bias, **spec)


@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
def test_route_of_many_rows(scores):
    """Enough rows for neighbours in the order that are a few units of 2^-24 apart: all against a stable sort in 64 bits."""
    rows, E, k = 40000, 256, 8
    z, bias = normal(rows, E, dtype=F32, scale=1.5), normal(E, seed=1, dtype=F32, scale=0.05)
    s = torch.softmax(z.double(), 1) if scores == "softmax" else 1 / (1 + torch.exp(-z.double()))
    v = s + bias.double()
    kind = hap.SOFTMAX if scores == "softmax" else hap.SIGMOID
    e, w = hap.hap_route(hap.hap_routing(E, k, kind, scale=2.5), z, bias=bias)
    want = torch.sort(v, dim=1, descending=True, stable=True).indices[:, :k]
    assert torch.equal(e.long(), want)
    c = s.gather(1, want)
    close(w, 2.5 * c / c.sum(1, keepdim=True), 64 * U * w.double(), F32)
    best = v.view(rows, 8, 32).topk(2, 2).values.sum(2)
    kept = torch.zeros(rows, 8, dtype=torch.bool, device="cuda").scatter_(1, best.topk(4, 1).indices, True)
    e, _ = hap.hap_route(hap.hap_routing(E, k, kind, groups=8, kept_groups=4, group_best=2), z, bias=bias)
    assert torch.equal(e.long(), torch.sort(v.masked_fill(~kept.repeat_interleave(32, 1), -INF), dim=1, descending=True, stable=True).indices[:, :k])


def test_route_of_large_and_small_logits():
    spec = dict(groups=1, kept=1, best=1, renormalise=True, scale=1.0)
    z = torch.tensor([[-300.0, -301.0, -1000.0, -299.5], [300.0, 301.0, 1000.0, 299.5], [-90.0, 5.0, -200.0, 80.0], [-3e38, -3.1e38, -3.3e38, -2e38]], device="cuda")
    for scores in ("softmax", "sigmoid"):
        for k in (1, 2, 4):
            routing = hap.hap_routing(4, k, hap.SOFTMAX if scores == "softmax" else hap.SIGMOID)
            e, w = hap.hap_route(routing, z)
            for row, ge, gw in zip(z.double().cpu().tolist(), e.tolist(), w.tolist()):
                we, ww = ref.route(row, None, k=k, scores=scores, **spec)
                assert ge == we and np.allclose(gw, ww, rtol=1e-4, atol=1e-37)          # (the logits' own differences are rounded: 1e-4 of e^0.5)
            dz = hap.hap_route_backward(routing, z, e, torch.ones_like(w))
            assert dz.isfinite().all() and dz.abs().max() < 1e-6                        # weights that add up to 1, all pulled alike


@pytest.mark.parametrize("pad", [3, 8])
def test_route_of_slices(pad):
    for dtype, E in ((BF, 64), (F32, 160), (FP, 8)):
        z, g = normal(50, E, dtype=dtype), normal(50, 4, seed=1, dtype=F32)
        for scores in (hap.SOFTMAX, hap.SIGMOID):
            for renormalise in (True, False):
                routing = hap.hap_routing(E, 4, scores, groups=4, kept_groups=2, group_best=2, renormalise=renormalise)
                e, w = hap.hap_route(routing, z)
                e2, w2 = hap.hap_route(routing, wide(z, pad))
                out = wide(torch.zeros(50, E, dtype=dtype, device="cuda"), pad)
                hap.hap_route_backward(routing, wide(z, pad), e2, g, dlogits=out)
                assert torch.equal(e, e2) and (w - w2).abs().max() <= 16 * U
                assert torch.allclose(out.float(), hap.hap_route_backward(routing, z, e, g).float(), rtol=0.01, atol=1e-6)
                assert torch.as_strided(out, (50, E + pad), out.stride())[:, E:].isnan().all()


def test_route_backward_of_given_experts():
    """Experts twice in a row add both gradients; numbers that are no experts add nothing."""
    z, g = normal(5, 40, dtype=F32), normal(5, 3, seed=1, dtype=F32)
    e = torch.tensor([[3, 3, 9], [-1, 40, 7], [-5, 1000, -1], [39, 39, 39], [0, 1, 2]], dtype=torch.int32, device="cuda")
    for scores in ("softmax", "sigmoid"):
        for renormalise in (True, False):
            routing = hap.hap_routing(40, 3, hap.SOFTMAX if scores == "softmax" else hap.SIGMOID, renormalise=renormalise)
            inside = torch.where((e >= 0) & (e < 40), e, -1)
            dz = hap.hap_route_backward(routing, z, e, g)
            want = ref.route_gradients(z.double(), inside, g.double(), scores, renormalise, 1.0)
            assert (dz.double() - want).abs().max() <= 64 * U * 3 * g.abs().max()       # |dz| <= s (|g| + mean |g|) of up to three entries
            assert not dz[2].any()


# ---- experts' rows ----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows,k", [(0, 2), (1, 1), (1, 32), (5, 8), (1365, 3), (4096, 1), (4097, 1), (1000, 6), (40000, 8), (2048, 32)])
@pytest.mark.parametrize("E,first", [(1, 0), (3, 7), (8, 0), (20, 40), (257, 0), (1024, 100)])
def test_expert_order(rows, k, E, first):
    gen = np.random.default_rng(rows + k + E)
    experts = gen.integers(first - 1, first + E + max(1, E // 8), (rows, k)).astype(np.int32)
    experts[gen.random((rows, k)) < 0.02] = -1
    if rows > 2:
        experts[rows // 2:rows // 2 + rows // 4] = first    # a busy one
        experts[0, 0], experts[1, 0] = np.iinfo(np.int32).max, np.iinfo(np.int32).min
    offsets, places = hap.hap_expert_order(torch.tensor(experts, device="cuda"), E, first=first)
    want = ref.order(experts, first, E)
    assert np.array_equal(offsets.cpu().numpy(), want[0]) and np.array_equal(places.cpu().numpy(), want[1])


def places_of(rows, k, spare, seed=0, away=0.2):
    """Places of (row, j) in some order, a fifth of them none."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = rows * k
    places = torch.randperm(n + spare, generator=gen, device="cuda")[:n].to(torch.int32).view(rows, k)
    places[torch.rand(rows, k, generator=gen, device="cuda") < away] = -1
    if rows > 2:
        places[1] = -1
        places[2, 0] = n + spare                            # behind the last row
    return places


ROW_SIZES = [(1, 1), (1, 8), (3, 7), (5, 2056), (300, 264), (70, 1000), (9, 250), (3000, 64), (2, 9001)]


@pytest.mark.parametrize("dtype", [BF, FP, F32])
@pytest.mark.parametrize("pads", [(0, 0), (8, 16), (3, 1)], ids=str)
@pytest.mark.parametrize("k", [1, 2, 6, 9, 32])
@pytest.mark.parametrize("rows,H", ROW_SIZES)
def test_rows_there_and_back(rows, H, k, pads, dtype):
    n = rows * k + 5
    at = lambda t, i: wide(t, pads[i]) if pads[i] else t  # noqa: E731
    places = places_of(rows, k, 5, seed=H)
    there = (places >= 0) & (places < n)
    x, y, w = normal(rows, H, dtype=dtype), normal(n, H, seed=1, dtype=dtype), normal(rows, k, seed=2, dtype=F32)
    idx = places.clamp(0, n - 1).long()
    # there
    out = at(torch.full((n, H), 7.0, dtype=dtype, device="cuda"), 1)
    assert hap.hap_expert_dispatch(at(x, 0), places, out=out) is out
    want = torch.full((n, H), 7.0, dtype=dtype, device="cuda")
    want[idx[there]] = x.unsqueeze(1).expand(rows, k, H)[there]
    assert torch.equal(out, want)
    # and back: rows that no place names may hold anything
    named = torch.zeros(n, dtype=torch.bool, device="cuda")
    named[idx[there]] = True
    y[~named] = float("nan")
    terms = torch.where(there.unsqueeze(2), y.to(D)[idx], 0)
    for weights, base in ((None, None), (w, None), (w, x)):
        got = hap.hap_expert_combine(at(y, 0), places, weights=weights, base=base)
        t = terms if weights is None else terms * w.to(D).unsqueeze(2)
        close(got, t.sum(1) + (base.to(D) if base is not None else 0), (k + 8) * U * (t.abs().sum(1) + (base.to(D).abs() if base is not None else 0)), dtype)
    again = x.clone()
    assert torch.equal(hap.hap_expert_combine(at(y, 0), places, weights=w, base=again, out=again), got)     # base may be out
    # gradients
    dout = normal(rows, H, seed=3, dtype=dtype)
    dy = at(torch.full((n, H), 7.0, dtype=dtype, device="cuda"), 1)
    hap.hap_expert_combine_backward(at(dout, 0), at(y, 1), places, weights=w, dy=dy, dweights=(dw := torch.full((rows, k), 7.0, device="cuda")))
    want = torch.full((n, H), 7.0, dtype=D, device="cuda")
    want[idx[there]] = (dout.to(D).unsqueeze(1) * w.to(D).unsqueeze(2))[there]
    close(dy, want, U * want.abs(), dtype)
    assert torch.equal(dy[~named], torch.full_like(dy[~named], 7.0))
    d = terms * dout.to(D).unsqueeze(1)
    close(dw, d.sum(2), (H + 8) * U * d.abs().sum(2), F32)
    assert not dw[~there].any()
    only = hap.hap_expert_combine_backward(dout, y, places, want_dweights=False, dy=torch.zeros(n, H, dtype=dtype, device="cuda"))
    assert only[1] is None and torch.equal(only[0][idx[there]], dout.unsqueeze(1).expand(rows, k, H)[there])
    assert torch.equal(hap.hap_expert_combine_backward(dout, y.contiguous(), places, want_dy=False)[1][~there], torch.zeros_like(dw[~there]))


def test_gradient_in_place_of_the_rows():
    places, y, dout, w = places_of(200, 4, 3), normal(803, 520), normal(200, 520, seed=1), normal(200, 4, seed=2, dtype=F32)
    dy, dw = hap.hap_expert_combine_backward(dout, y, places, weights=w, dy=torch.zeros_like(y))
    same = y.clone()
    got = hap.hap_expert_combine_backward(dout, same, places, weights=w, dy=same)
    there = (places >= 0) & (places < 803)
    assert torch.equal(got[1], dw) and torch.equal(same[places[there].long()], dy[places[there].long()])


# ---- embedding ----------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,out", [(BF, BF), (FP, F32), (F32, F32), (BF, F32)], ids=str)
@pytest.mark.parametrize("n,V,H", [(0, 5, 8), (1, 1, 1), (33, 5, 7), (31, 1000, 264), (4096, 3, 40), (4097, 32003, 64), (10000, 700, 72), (5000, (1 << 20) + 7, 8), (300, 50, 2056),
                                   (64, 2, 4104), (70000, 1023, 8)])
def test_embedding(n, V, H, dtype, out):
    gen = torch.Generator(device="cuda").manual_seed(n + V)
    first = 17
    tokens = first + torch.randint(-2, V + 2, (n,), generator=gen, device="cuda")
    if n > 40:
        tokens[n // 3:n // 2] = first + V // 2              # a frequent word
        tokens[3], tokens[4], tokens[5] = -(1 << 63), (1 << 63) - 1, -100
    there = (tokens >= first) & (tokens - first < V) & (tokens < 1 << 40)
    at = torch.where(there, tokens - first, 0)
    w, dy = normal(V, H, dtype=dtype), normal(n, H, seed=1, dtype=dtype)
    for pad in (0, 3, 8):
        place = lambda t: wide(t, pad) if pad else t  # noqa: E731
        got = hap.hap_embedding(tokens, place(w), first=first, scale=1.5, out=place(torch.zeros(n, H, dtype=dtype, device="cuda")))
        want = torch.where(there.unsqueeze(1), w.to(D)[at] * 1.5, 0)
        close(got, want, 0 * want, dtype)
        sums = torch.zeros(V, H, dtype=D, device="cuda").index_add_(0, at[there], dy.to(D)[there])
        size = torch.zeros(V, H, dtype=D, device="cuda").index_add_(0, at[there], dy.to(D)[there].abs())
        count = torch.zeros(V, device="cuda", dtype=D).index_add_(0, at[there], torch.ones_like(at[there], dtype=D)).unsqueeze(1)
        dw = place(torch.full((V, H), 7.0, dtype=out, device="cuda"))
        assert hap.hap_embedding_backward(tokens, place(dy), dw, first=first, scale=0.75) is dw
        close(dw, 0.75 * sums, (count + 8) * U * size, out)
        assert not dw[count[:, 0] == 0].any()
        before = normal(V, H, seed=2, dtype=out)
        dw = place(before.clone())
        hap.hap_embedding_backward(tokens, place(dy), dw, first=first, scale=0.75, accumulate=True)
        close(dw, before.to(D) + 0.75 * sums, (count + 8) * U * size + U * before.to(D).abs(), out)
        assert torch.equal(dw[count[:, 0] == 0], before[count[:, 0] == 0])
        if pad:
            assert torch.as_strided(dw, (V, H + pad), dw.stride())[:, H:].isnan().all()


def test_embedding_gradient_is_the_same_again():
    tokens = torch.randint(0, 900, (20000,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).square() // 900
    dy = normal(20000, 136)
    first = hap.hap_embedding_backward(tokens, dy, torch.empty(900, 136, device="cuda"))
    for _ in range(3):
        assert torch.equal(hap.hap_embedding_backward(tokens, dy, torch.empty(900, 136, device="cuda")), first)


# ---- layer norm ------------------------------------------------------------------------------------------------------------------
NORMS = [(1, 1), (3, 2), (5, 7), (130, 8), (33, 100), (700, 256), (9, 1000), (600, 1024), (3, 2056), (40, 5000), (5, 8192), (3, 8200), (2, 16384), (2000, 72), (601, 4096)]


@pytest.mark.parametrize("dtype,params", [(BF, BF), (BF, F32), (FP, FP), (F32, F32)], ids=str)
@pytest.mark.parametrize("centred", [True, False])
@pytest.mark.parametrize("rows,H", NORMS)
def test_layer_norm(rows, H, centred, dtype, params):
    eps = 1e-5
    x, dy, base = normal(rows, H, dtype=dtype, scale=2.0), normal(rows, H, seed=1, dtype=dtype), normal(rows, H, seed=2, dtype=dtype)
    x += 3.0
    w, b = normal(H, seed=3, dtype=params), normal(H, seed=4, dtype=params) if centred else None
    for pad in (0, 8, 3):
        at = lambda t: wide(t, pad) if pad else t  # noqa: E731
        y, mean, rstd = hap.hap_layer_norm(at(x), w, b, eps=eps, centred=centred, y=at(torch.zeros_like(x)))
        X, W = x.to(D), w.to(D)
        Y, M, R = ref.norm(X, W, b.to(D) if centred else None, eps, centred)
        diff = X - M.unsqueeze(1)
        var = (diff * diff).mean(1)
        em = (H + 8) * U * X.abs().mean(1) if centred else torch.zeros_like(M)
        # the variance: of differences that are off by em, a sum of H squares; its share in var + eps
        rel = (2 * em * diff.abs().mean(1) + em * em + (H + 16) * U * var) / (var + eps) + 8 * U
        if centred:
            close(mean, M, em, F32)
        else:
            assert mean is None
        close(rstd, R, rel * R, F32)
        xh = (diff * R.unsqueeze(1)).abs()
        off = W.abs() * (xh * (rel + 8 * U).unsqueeze(1) + (em * R).unsqueeze(1) * (1 + rel).unsqueeze(1)) + U * (W.abs() * xh + (b.to(D).abs() if centred else 0))
        close(y, Y, off, dtype)
        # backwards, from the kept mean and rstd
        m, r = mean.to(D) if centred else torch.zeros_like(M), rstd.to(D)
        DY = dy.to(D)
        dx, dw, db = ref.norm_gradients(DY, X, W, m, r, centred)
        xh, e = ((X - m.unsqueeze(1)) * r.unsqueeze(1)).abs(), ((X.abs() + m.abs().unsqueeze(1)) * r.unsqueeze(1)) * 2 * U      # xh, and what it is off by
        g = (DY * W).abs()
        off = r.unsqueeze(1) * ((H + 16) * U * (g + g.mean(1, keepdim=True) + xh * (g * xh).mean(1, keepdim=True))
                                + e * (g * xh).mean(1, keepdim=True) + (xh + e) * (g * e).mean(1, keepdim=True))
        gdx, gdw, gdb = hap.hap_layer_norm_backward(at(dy), at(x), w, rstd, mean=mean, dx=at(torch.zeros_like(x)))
        close(gdx, dx, off, dtype)
        offw, offb = (rows + 16) * U * (DY.abs() * xh).sum(0) + (DY.abs() * e).sum(0), (rows + 16) * U * DY.abs().sum(0)
        close(gdw, dw, offw, params)
        assert gdw.dtype == params and (gdb is None) == (not centred)
        if centred:
            close(gdb, db, offb, params)
        again, none, _ = hap.hap_layer_norm_backward(at(dy), at(x), w, rstd, mean=mean, base=at(base), want_dw=False)
        close(again, base.to(D) + dx, off + 2 * U * (base.to(D).abs() + dx.abs()), dtype)
        assert none is None
        start = normal(H, seed=5, dtype=F32)
        sums = (start.clone(), start.clone() if centred else None)
        hap.hap_layer_norm_backward(at(dy), at(x), w, rstd, mean=mean, want_dx=False, dw=sums[0], db=sums[1], accumulate=True)
        close(sums[0], start.to(D) + dw, offw + U * (start.to(D).abs() + dw.abs()), F32)
        if centred:
            close(sums[1], start.to(D) + db, offb + U * (start.to(D).abs() + db.abs()), F32)


def test_layer_norm_without_weights_and_of_constant_rows():
    x = torch.full((4, 264), 5.0, dtype=BF, device="cuda")
    x[1] = 0
    y, mean, rstd = hap.hap_layer_norm(x, eps=1e-6)
    assert not y.any() and torch.equal(mean, torch.tensor([5.0, 0, 5, 5], device="cuda")) and ((rstd - 1000).abs() < 0.01).all()
    dx, dw, db = hap.hap_layer_norm_backward(torch.ones_like(x), x, None, rstd, mean=mean)
    assert not dx.any() and not dw.any() and dw.dtype == F32 and (db == 4).all()
    y, none, _ = hap.hap_layer_norm(x, centred=False, eps=0.0)
    assert none is None and (y[0] == 1).all() and y[1].isnan().all()                # 0 / 0, as it is written
    none = torch.zeros(0, 264, dtype=BF, device="cuda")
    y, mean, rstd = hap.hap_layer_norm(none)
    dx, dw, db = hap.hap_layer_norm_backward(none, none, None, rstd, mean=mean)
    assert y.shape == dx.shape == (0, 264) and not dw.any() and not db.any()


def test_layer_norm_of_a_far_mean():
    """The variance is that of differences: it does not drown in the mean's square."""
    x = (normal(50, 1000, dtype=F32) * 2.0 ** -6 + 1000.0)
    y, mean, rstd = hap.hap_layer_norm(x, eps=0.0)
    Y, M, R = ref.norm(x.to(D), None, None, 0.0, True)
    # the mean is off by up to 1008 2^-23 of 1000, in practice a few units of 2^-24 of it: 1000 * 2^-20 against differences of 2^-6
    assert ((mean.to(D) - M).abs() < 1000 * 1008 * U).all()
    assert ((rstd.to(D) / R - 1).abs() < 0.02).all() and ((y.to(D) - Y).abs() < 0.15).all()
