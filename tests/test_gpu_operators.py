"""Training operators against their definitions in 64 bits.

Tolerances are bounds from arithmetic.  A sum of n products kept in fp32, each addition off by at most 2^-23 of the running
magnitude whatever its order and rounding, is off by at most (n + 8) 2^-23 S with S the sum of magnitudes; rounding to a type t
adds finfo(t).eps / 2 of the value, and half of the smallest subnormal of fp16."""
import pytest
import torch

import paper_2609_39350_b200 as hap

pytestmark = pytest.mark.gpu
BF, FP, F32, D = torch.bfloat16, torch.float16, torch.float32, torch.float64
U = 2.0 ** -23


def normal(*shape, seed=0, dtype=BF, scale=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed * 1000003 + sum((i + 1) * s for i, s in enumerate(shape)))
    return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dtype)


def rounding(ref, dtype):
    return torch.finfo(dtype).eps / 2 * ref.abs() + (2.0 ** -25 if dtype == FP else 0.0)


def close(got, ref, off, dtype):
    """|got - ref| within `off` and one rounding to dtype."""
    bound = off + rounding(ref, dtype) * (1 + 2.0 ** -6) + torch.finfo(dtype).eps * off + 1e-37
    bad = (got.to(D) - ref).abs() > bound
    assert not bad.any(), (int(bad.sum()), float(((got.to(D) - ref).abs() / bound).max()))


def offsets_of(loads, first=0):
    o = [first]
    for n in loads:
        o.append(o[-1] + n)
    return torch.tensor(o, dtype=torch.int64, device="cuda"), o


def wide(t, pad):
    """The same matrix as a slice of a wider one, whose other columns hold NaN."""
    shape = (*t.shape[:-1], t.shape[-1] + pad)
    full = torch.full(shape, float("nan"), dtype=t.dtype, device="cuda")
    full[..., :t.shape[-1]] = t
    return full[..., :t.shape[-1]]


LOADS = [[1], [2], [0, 1, 0], [128], [127, 129, 1], [0, 0, 300, 5, 64, 65, 63, 0], [1] * 40, [257, 0, 511]]
SIZES = [(256, 64), (8, 8), (136, 72), (264, 520), (1000, 200), (7, 13), (33, 250), (512, 1024)]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("loads", LOADS, ids=lambda x: "-".join(map(str, x[:8])))
@pytest.mark.parametrize("N,K", SIZES)
def test_expert_matmul(loads, N, K, dtype):
    off, o = offsets_of(loads, first=2)
    rows, E = o[-1] + 3, len(loads)
    x, dy, w = normal(rows, K, dtype=dtype), normal(rows, N, seed=1, dtype=dtype), normal(E, N, K, seed=2, dtype=dtype, scale=0.25)
    for t in (x, dy):                               # what the rows outside of the experts hold does not matter
        t[:2], t[o[-1]:] = float("nan"), float("inf")
    y = torch.full((rows, N), 7.0, dtype=dtype, device="cuda")
    dx = torch.full((rows, K), 7.0, dtype=F32, device="cuda")
    assert hap.hap_expert_matmul(x, w, off, out=y) is y
    hap.hap_expert_matmul(dy, w, off, hap.EXPERT_GRAD_INPUT, out=dx)
    dw = hap.hap_expert_matmul(dy, x, off, hap.EXPERT_GRAD_WEIGHT)
    start = normal(E, N, K, seed=3, dtype=F32)
    dw32 = hap.hap_expert_matmul(dy, x, off, hap.EXPERT_GRAD_WEIGHT, out=start.clone(), accumulate=True)
    for t in (y, dx):
        assert (t[:2] == 7).all() and (t[o[-1]:] == 7).all()
    for e in range(E):
        i, j = o[e], o[e + 1]
        a, g, m = x[i:j].to(D), dy[i:j].to(D), w[e].to(D)
        close(y[i:j], a @ m.T, (K + 8) * U * (a.abs() @ m.abs().T), dtype)
        close(dx[i:j], g @ m, (N + 8) * U * (g.abs() @ m.abs()), F32)
        ref, s = g.T @ a, g.abs().T @ a.abs()
        close(dw[e], ref, (j - i + 8) * U * s, dtype)
        close(dw32[e], ref + start[e].to(D), (j - i + 8) * U * s + U * (ref.abs() + s * U), F32)


@pytest.mark.parametrize("pad", [8, 3])
def test_expert_matmul_of_slices(pad):
    """Row distances other than the row's length, and outputs that are slices: nothing beside them is written."""
    off, o = offsets_of([70, 0, 133])
    E, N, K, rows = 3, 200, 328, o[-1]
    x, dy = wide(normal(rows, K), pad), wide(normal(rows, N, seed=1), pad)
    w = wide(normal(E, N, K, seed=2), pad)
    for form, a, b, shape in ((hap.EXPERT_FORWARD, x, w, (rows, N)), (hap.EXPERT_GRAD_INPUT, dy, w, (rows, K)), (hap.EXPERT_GRAD_WEIGHT, dy, x, (E, N, K))):
        out = wide(torch.zeros(shape, dtype=BF, device="cuda"), pad)
        hap.hap_expert_matmul(a, b, off, form, out=out)
        again = hap.hap_expert_matmul(a.contiguous(), b.contiguous(), off, form)
        if pad % 8 == 0:
            assert torch.equal(out, again)
        else:                                       # another variant: another order of additions
            assert (out.float() - again.float()).abs().max() <= 0.02 * again.float().abs().max()
        full = torch.as_strided(out, (*shape[:-1], shape[-1] + pad), out.stride())
        assert full[..., shape[-1]:].isnan().all()


def test_expert_matmul_of_offsets_out_of_order():
    """Offsets from a broken router lead nowhere: they are clamped and made ascending."""
    x, w = normal(100, 64), normal(3, 128, 64, seed=1)
    out = torch.full((100, 128), 7.0, dtype=BF, device="cuda")
    hap.hap_expert_matmul(x, w, torch.tensor([-5, 40, 20, 1 << 40], device="cuda"), out=out)
    ref = torch.cat([x[:40].float() @ w[0].float().T, x[40:].float() @ w[2].float().T])
    assert (out.float() - ref).abs().max() < 0.05 * ref.abs().max()


def test_expert_matmul_without_rows():
    w = normal(2, 64, 32)
    off = torch.zeros(3, dtype=torch.int64, device="cuda")
    none = torch.zeros(0, 32, dtype=BF, device="cuda")
    assert hap.hap_expert_matmul(none, w, off).shape == (0, 64)
    dw = hap.hap_expert_matmul(torch.zeros(0, 64, dtype=BF, device="cuda"), none, off, hap.EXPERT_GRAD_WEIGHT, out=torch.full((2, 64, 32), 5.0, dtype=BF, device="cuda"))
    assert not dw.any()
    kept = hap.hap_expert_matmul(normal(9, 64), normal(9, 32), off, hap.EXPERT_GRAD_WEIGHT, out=torch.full((2, 64, 32), 5.0, device="cuda"), accumulate=True)
    assert (kept == 5).all()


def test_many_experts_and_long_groups():
    E, N, K = 1024, 64, 64
    loads = [(7 * e) % 5 for e in range(E)]
    off, o = offsets_of(loads)
    x, w = normal(o[-1], K), normal(E, N, K, seed=1)
    of = torch.repeat_interleave(torch.arange(E, device="cuda"), torch.tensor(loads, device="cuda"))
    ref = torch.einsum("rk,rnk->rn", x.to(D), w[of].to(D))
    close(hap.hap_expert_matmul(x, w, off), ref, (K + 8) * U * torch.einsum("rk,rnk->rn", x.to(D).abs(), w[of].to(D).abs()), BF)
    off, _ = offsets_of([40000, 1])                 # one long contraction, one of a single row
    a, b = normal(40001, 136), normal(40001, 264, seed=1)
    dw = hap.hap_expert_matmul(a, b, off, hap.EXPERT_GRAD_WEIGHT, out_dtype=F32)
    close(dw[0], a[:40000].to(D).T @ b[:40000].to(D), 40008 * U * (a[:40000].to(D).abs().T @ b[:40000].to(D).abs()), F32)
    assert torch.equal(dw[1], a[40000:].float().T @ b[40000:].float())


def test_more_row_tiles_than_a_band():
    """A group of many tiles beside short ones, in all three forms."""
    loads, N, K = [5000, 3, 0, 700, 260], 520, 264
    off, o = offsets_of(loads, first=5)
    rows, E = o[-1] + 9, len(loads)
    x, dy, w = normal(rows, K), normal(rows, N, seed=1), normal(E, N, K, seed=2, scale=0.25)
    y, dx, dw = hap.hap_expert_matmul(x, w, off), hap.hap_expert_matmul(dy, w, off, hap.EXPERT_GRAD_INPUT), hap.hap_expert_matmul(dy, x, off, hap.EXPERT_GRAD_WEIGHT, out_dtype=F32)
    for e in range(E):
        i, j = o[e], o[e + 1]
        a, g, m = x[i:j].to(D), dy[i:j].to(D), w[e].to(D)
        close(y[i:j], a @ m.T, (K + 8) * U * (a.abs() @ m.abs().T), BF)
        close(dx[i:j], g @ m, (N + 8) * U * (g.abs() @ m.abs()), BF)
        close(dw[e], g.T @ a, (j - i + 8) * U * (g.abs().T @ a.abs()), F32)


@pytest.mark.parametrize("out_dtype", [BF, F32])
@pytest.mark.parametrize("loads", [[1, 1], [90, 0, 300]], ids=str)
def test_products_added_to_what_is_there(loads, out_dtype):
    off, o = offsets_of(loads)
    E, N, K, rows = len(loads), 264, 328, o[-1]
    x, dy, w = normal(rows, K), normal(rows, N, seed=1), normal(E, N, K, seed=2, scale=0.1)
    of = torch.repeat_interleave(torch.arange(E, device="cuda"), torch.tensor(loads, device="cuda"))
    for form, a, cols, terms in ((hap.EXPERT_FORWARD, x, N, "rk,rnk->rn"), (hap.EXPERT_GRAD_INPUT, dy, K, "rn,rnk->rk")):
        out = normal(rows, cols, seed=3, dtype=out_dtype)
        before = out.to(D)
        hap.hap_expert_matmul(a, w, off, form, out=out, accumulate=True)
        ref, s = torch.einsum(terms, a.to(D), w[of].to(D)), torch.einsum(terms, a.to(D).abs(), w[of].to(D).abs())
        close(out, before + ref, (a.shape[1] + 8) * U * s + U * (before.abs() + s), out_dtype)


def gated_reference(x, w, F):
    z, s = x.to(D) @ w.to(D).T, x.to(D).abs() @ w.to(D).abs().T
    g, u = z[:, :F], z[:, F:]
    off = (x.shape[1] + 8) * U * s
    h = g * torch.sigmoid(g) * u
    return z, off, h, 1.1 * u.abs() * off[:, :F] + g.abs() * off[:, F:] + 2 * off[:, :F] * off[:, F:] + (8 + 1.2 * g.abs()) * U * h.abs()


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("loads", LOADS[2:], ids=lambda x: "-".join(map(str, x[:8])))
@pytest.mark.parametrize("F,H", [(128, 64), (8, 8), (136, 200), (264, 512), (13, 27)])
def test_expert_gated(loads, F, H, dtype):
    off, o = offsets_of(loads, first=1)
    rows, E = o[-1] + 2, len(loads)
    x, w = normal(rows, H, dtype=dtype), normal(E, 2 * F, H, seed=1, dtype=dtype, scale=2.0 * H ** -0.5)
    gu, h = torch.full((rows, 2 * F), 7.0, dtype=dtype, device="cuda"), torch.full((rows, F), 7.0, dtype=dtype, device="cuda")
    hap.hap_expert_gated(x, w, off, gu=gu, h=h)
    only, none = hap.hap_expert_gated(x, w, off, keep=False)
    assert none is None and torch.equal(only[o[0]:o[-1]], h[o[0]:o[-1]])
    for t in (gu, h):
        assert (t[:1] == 7).all() and (t[o[-1]:] == 7).all()
    dy, w2 = normal(rows, H, seed=2, dtype=dtype), normal(E, H, F, seed=3, dtype=dtype, scale=H ** -0.5)
    dgu, h2 = hap.hap_expert_gated_backward(dy, w2, off, gu)
    in_place = gu.clone()
    hap.hap_expert_gated_backward(dy, w2, off, in_place, dgu=in_place, want_h=False)
    assert torch.equal(in_place[o[0]:o[-1]], dgu[o[0]:o[-1]])
    for e in range(E):
        i, j = o[e], o[e + 1]
        z, zoff, ref, hoff = gated_reference(x[i:j], w[e], F)
        close(gu[i:j], z, zoff, dtype)
        close(h[i:j], ref, hoff, dtype)
        g, u = gu[i:j, :F].to(D), gu[i:j, F:].to(D)             # as they were kept
        dh, s = dy[i:j].to(D) @ w2[e].to(D), dy[i:j].to(D).abs() @ w2[e].to(D).abs()
        doff, sig = (H + 8) * U * s, torch.sigmoid(g)
        slope = sig + g * sig * (1 - sig)
        close(dgu[i:j, :F], dh * u * slope, 1.1 * u.abs() * doff + (dh * u).abs() * (12 + 6 * g.abs()) * U, dtype)
        close(dgu[i:j, F:], dh * g * sig, g.abs() * doff + (dh * g).abs() * (12 + 2 * g.abs()) * U, dtype)
        close(h2[i:j], g * sig * u, (12 + 2 * g.abs()) * U * (g * u).abs(), dtype)


def test_gated_of_large_values():
    """silu at the ends of its range: no NaN where the exponential overflows."""
    off, _ = offsets_of([3])
    x = torch.zeros(3, 8, dtype=BF, device="cuda")
    x[0, 0], x[1, 0], x[2, 0] = 200, -200, 0
    w = torch.zeros(1, 16, 8, dtype=BF, device="cuda")
    w[:, :, 0] = 1
    h, gu = hap.hap_expert_gated(x, w, off)
    assert (h[0] == 40000).all() or (h[0].float() - 40000).abs().max() <= 128
    assert (h[1] == 0).all() and (h[2] == 0).all()
    dgu, _ = hap.hap_expert_gated_backward(torch.ones(3, 8, dtype=BF, device="cuda"), torch.ones(1, 8, 8, dtype=BF, device="cuda"), off, gu)
    assert dgu.isfinite().all()


def loss_reference(x, w, target, grad, dtype):
    """loss, lse, dx, dw and how far each may be off."""
    x, w, n, H, V = x.to(D), w.to(D), x.shape[0], x.shape[1], w.shape[0]
    z, zs = x @ w.T, x.abs() @ w.abs().T
    lse = torch.logsumexp(z, 1)
    zoff = (H + 8) * U * zs
    # a common error of all terms from forming exponents of logits, one of each term, sums over tiles and of tiles
    lse_off = zoff.amax(1) + (z.abs().amax(1) + lse.abs() + 4) * 2 * U + (256 + V / 256) * U
    ok = (target >= 0) & (target < V)
    at = torch.where(ok, target, 0)
    rows = torch.arange(n, device="cuda")
    loss = torch.where(ok, lse - z[rows, at], 0.0)
    p = torch.exp(z - lse[:, None])
    d = p.clone()
    d[rows, at] -= 1
    d = torch.where(ok[:, None], d, 0.0)
    poff = p * (zoff + lse_off[:, None] + (z.abs() + lse.abs()[:, None] + 4) * 2 * U)
    doff = torch.where(ok[:, None], poff * 1.01 + rounding(d, dtype) + 2.0 ** -24 * 2.0 ** -15, 0.0)
    g = abs(float(grad))
    dx, dx_off = grad * (d @ w), g * (doff @ w.abs() + (V + 8) * U * (d.abs() @ w.abs()))
    dw, dw_off = grad * (d.T @ x), g * (doff.T @ x.abs() + (n + 8) * U * (d.abs().T @ x.abs()))
    return (loss, lse_off + zoff[rows, at] + U * loss.abs()), (lse, lse_off), (dx, dx_off), (dw, dw_off)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("rows,H,V", [(1, 8, 1), (1, 64, 1000), (3, 128, 257), (129, 72, 511), (128, 64, 256), (200, 264, 3001), (5, 33, 77), (300, 64, 8200), (4, 264, 76033), (260, 320, 9001)])
def test_linear_cross_entropy(rows, H, V, dtype):
    x, w = normal(rows, H, dtype=dtype), normal(V, H, seed=1, dtype=dtype, scale=2.0 * H ** -0.5)
    target = torch.randint(0, V, (rows,), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    target[0], target[-1] = V - 1, V - 1
    target[rows // 3::7] = -100
    grad = torch.full((), 1.0 / rows if dtype == BF else 0.75, device="cuda")
    loss, lse = hap.hap_linear_cross_entropy(x, w, target)
    dx, dw = hap.hap_linear_cross_entropy_backward(x, w, target, lse, grad)
    for got, (ref, off), t in zip((loss, lse, dx, dw), loss_reference(x, w, target, grad.to(D), dtype), (F32, F32, dtype, dtype)):
        close(got, ref, off, t)
    assert not loss[target == -100].any() and not dx[target == -100].any()
    only, none = hap.hap_linear_cross_entropy_backward(x, w, target, lse, grad, want_dw=False)
    assert none is None and torch.equal(only, dx)
    none, only = hap.hap_linear_cross_entropy_backward(x, w, target, lse, grad, want_dx=False)
    assert none is None and torch.equal(only, dw)


def test_loss_in_pieces_against_differences():
    """More than one piece of the vocabulary, and the gradients against differences of the loss."""
    rows, H, V = 24700, 64, 4500                    # pieces are of 3840 columns here
    x, w = normal(rows, H, dtype=FP), normal(V, H, seed=1, dtype=FP, scale=2.0 * H ** -0.5)
    target = torch.randint(0, V, (rows,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    target[::11] = -1
    grad = torch.full((), 2.0, device="cuda")
    loss, lse = hap.hap_linear_cross_entropy(x, w, target, ignore_index=-1)
    dx, dw = hap.hap_linear_cross_entropy_backward(x, w, target, lse, grad, ignore_index=-1)
    for got, (ref, off), t in zip((loss, lse, dx, dw), loss_reference(x, w, target, grad.to(D), FP), (F32, F32, FP, FP)):
        close(got, ref, off, t)
    step = torch.randn(rows, H, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3), dtype=D)

    def total(t):
        z = (x.to(D) + t * step) @ w.to(D).T
        keep = target >= 0
        return 2.0 * (torch.logsumexp(z, 1) - z.gather(1, target.clamp(min=0)[:, None])[:, 0])[keep].sum()

    h = 1e-4
    slope = (total(h) - total(-h)) / (2 * h)        # off by h^2 / 6 of a third derivative, below 1e-6 of the slope's terms
    along = (dx.to(D) * step).sum()
    assert (slope - along).abs() <= 2.0 ** -11 * 4 * (dx.to(D) * step).square().sum().sqrt() + 1e-5 * (dx.to(D) * step).abs().sum()


def test_loss_without_rows():
    x, w, t = torch.zeros(0, 64, dtype=BF, device="cuda"), normal(300, 64), torch.zeros(0, dtype=torch.int64, device="cuda")
    loss, lse = hap.hap_linear_cross_entropy(x, w, t)
    dx, dw = hap.hap_linear_cross_entropy_backward(x, w, t, lse, torch.ones((), device="cuda"), dw=torch.full((300, 64), 3.0, dtype=BF, device="cuda"))
    assert loss.shape == (0,) and dx.shape == (0, 64) and not dw.any()


def test_loss_of_bad_targets_and_infinite_logits():
    x, w = normal(6, 64), normal(500, 64, seed=1)
    target = torch.tensor([3, 500, -2, -100, 499, 0], device="cuda")
    loss, lse = hap.hap_linear_cross_entropy(x, w, target)
    assert loss.isnan().tolist() == [False, True, True, False, False, False] and loss[3] == 0
    dx, _ = hap.hap_linear_cross_entropy_backward(x, w, target, lse, torch.ones((), device="cuda"))
    assert not dx[1:4].any() and dx[0].any()
    x[2, 0], target[2] = float("nan"), 1
    loss, lse = hap.hap_linear_cross_entropy(x, w, target)
    assert loss.isnan().tolist() == [False, True, True, False, False, False] and lse[2].isnan()


def adamw_reference(p, g, m, v, step, lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, scale=1.0):
    """The step with the moments' 32-bit operations as they are defined, the parameter in 64 bits."""
    c = lambda x: torch.tensor(x, dtype=D).to(F32).item()  # noqa: E731
    r = lambda x: x.to(F32).to(D)  # noqa: E731
    g = r(g.to(D) * scale)
    m = r(r(m * c(beta1)) + r(g * c(1 - beta1)))
    v = r(r(v * c(beta2)) + r(r(g * g) * c(1 - beta2)))
    p = p.to(D)
    move = lr / (1 - beta1 ** step) * m / (torch.sqrt(v / (1 - beta2 ** step)) + eps)
    return p * (1 - lr * weight_decay) - move, m, v, 16 * U * (p.abs() + move.abs())


def read8(code, scale, signed):
    r = lambda x: x.to(F32).to(D)  # noqa: E731
    n = code.numel()
    s = scale.to(D).repeat_interleave(256)[:n]
    t = r(code.to(D) * torch.tensor(1 / (127 if signed else 255), dtype=D).to(F32).item())
    return r(r(t * t.abs()) * s) if signed else r(r(r(t * t) * r(t * t)) * s)


def codes8(x, signed):
    r = lambda y: y.to(F32).to(D)  # noqa: E731
    n = x.numel()
    b = torch.cat([x, torch.zeros(-n % 256, dtype=D, device=x.device)]).view(-1, 256)
    s = b.abs().amax(1)
    q = r(b.abs() / torch.where(s > 0, s, 1.0)[:, None])
    if signed:
        c = torch.sign(b) * torch.round(r(r(torch.sqrt(q)) * 127))
    else:
        c = torch.where(b > 0, torch.round(r(r(torch.sqrt(r(torch.sqrt(q)))) * 255)).clamp(min=1), 0.0)
    return c.view(-1)[:n], s


SIZES_OF_TENSORS = [1, 2, 7, 255, 256, 257, 4095, 4096, 4097, 12288 + 5, 40000]


@pytest.mark.parametrize("ptype,gtype", [(BF, BF), (FP, FP), (BF, F32), (F32, F32), (F32, BF), (F32, FP), (FP, F32)])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("shift", [0, 1])
def test_adamw(ptype, gtype, bits, shift):
    """shift: tensors that follow one another in one buffer, so that most start at odd places."""
    sizes = SIZES_OF_TENSORS
    total = sum(sizes)

    def parts(flat):
        if shift:
            return list(flat.split(sizes))
        return [t.clone() for t in flat.split(sizes)]

    p, g = parts(normal(total, dtype=ptype, scale=0.1)), parts(normal(total, seed=1, dtype=gtype, scale=1e-2))
    g[5].zero_()
    scale = torch.full((), 0.37, device="cuda")
    copies = parts(torch.zeros(total, dtype=BF if gtype != FP else FP, device="cuda")) if ptype == F32 else None
    if bits == 32:
        m, v = parts(normal(total, seed=2, dtype=F32, scale=1e-3)), parts(normal(total, seed=3, dtype=F32, scale=1e-2).square())
        more = {}
    else:
        m, v = parts(torch.zeros(total, dtype=torch.int8, device="cuda")), parts(torch.zeros(total, dtype=torch.uint8, device="cuda"))
        ms = [torch.zeros(-(-n // 256), device="cuda") for n in sizes]
        vs = [torch.zeros(-(-n // 256), device="cuda") for n in sizes]
        more = dict(m_scale=ms, v_scale=vs)
    tensors = hap.hap_adamw_tensors(p, g, m, v, copies=copies, **more)
    for step in (1, 2, 3):
        before = [(a.clone(), x.clone(), y.clone()) for a, x, y in zip(p, m, v)]
        if bits == 8:
            before = [(a, read8(x, s, True), read8(y, q, False)) for (a, x, y), s, q in zip(before, ms, vs)]
        hap.hap_adamw_step(tensors, step, 1e-3, 0.9, 0.95, 1e-8, 0.1, grad_scale=scale)
        for i in range(len(sizes)):
            a, x, y = before[i]
            ref, rm, rv, off = adamw_reference(a, g[i], x.to(D), y.to(D), step, scale=torch.full((), 0.37).to(D).item())
            close(p[i], ref, off, ptype)
            if copies is not None:
                assert torch.equal(copies[i], p[i].to(copies[i].dtype))
            if bits == 32:                          # two roundings, or fewer where operations are fused
                assert ((m[i].to(D) - rm).abs() <= 2 * U * (x.to(D).abs() + g[i].to(D).abs())).all()
                assert ((v[i].to(D) - rv).abs() <= 3 * U * rv.abs() + 1e-44).all()
            else:
                for code, s, val, signed in ((m[i], ms[i], rm, True), (v[i], vs[i], rv, False)):
                    want, ws = codes8(val, signed)
                    assert torch.equal(s.to(D), ws) and torch.equal(code.to(D), want)
    if bits == 8:
        for i, (x, y) in enumerate(zip(*hap.hap_adamw_state(tensors))):
            assert torch.equal(x.to(D).view(-1), read8(m[i], ms[i], True)) and torch.equal(y.to(D).view(-1), read8(v[i], vs[i], False))


def test_adamw_of_values_at_the_ends():
    """Magnitudes near both ends of fp32 in blocks of 8-bit states, squares that are not finite, and gradients that are not."""
    tops = [1e-38, 1e-30, 1e-19, 1e-10, 1.0, 1e9, 1e18, 1.5e19, 6e19]
    blocks = len(tops) + 1
    n = 256 * blocks
    g = torch.zeros(n, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(2)
    for b, top in enumerate(tops):
        g[256 * b:256 * b + 256] = top * torch.exp2(-24 * torch.rand(256, generator=gen, device="cuda")) * torch.sign(torch.randn(256, generator=gen, device="cuda"))
    p = torch.zeros(n, device="cuda")
    m, v = torch.zeros(n, dtype=torch.int8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    ms, vs = torch.zeros(blocks, device="cuda"), torch.zeros(blocks, device="cuda")
    t = hap.hap_adamw_tensors([p], [g], [m], [v], [ms], [vs])
    hap.hap_adamw_step(t, 1, 1e-3, 0.9, 0.95)
    _, rm, rv, _ = adamw_reference(torch.zeros(n, device="cuda"), g, torch.zeros(n, dtype=D, device="cuda"), torch.zeros(n, dtype=D, device="cuda"), 1)
    for code, s, val, signed in ((m, ms, rm, True), (v, vs, rv, False)):
        want, ws = codes8(val, signed)
        held = ws.isfinite()                        # codes under a scale that is not finite mean nothing
        assert held.tolist() == [True] * 8 + [signed, True]
        of = held.repeat_interleave(256)
        assert torch.equal(s.to(D), ws) and torch.equal(code.to(D)[of], want[of])
    assert p.isfinite().all() and not p[256 * len(tops):].any()
    assert not hap.hap_adamw_state(t)[1][0][256 * 8:256 * 9].isfinite().any()
    g[0], g[256] = float("nan"), float("inf")
    hap.hap_adamw_step(t, 2, 1e-3, 0.9, 0.95)
    x, y = hap.hap_adamw_state(t)
    assert not x[0][:512].isfinite().any() and x[0][512:].isfinite().all()
    assert not y[0][:512].isfinite().any() and y[0][512:256 * 8].isfinite().all() and y[0][256 * 9:].isfinite().all()


def test_adamw_of_more_tensors_than_a_launch_holds():
    sizes = [1 + (37 * i) % 700 for i in range(900)]
    sizes[3] = 0
    p, g, m, v = ([normal(n, seed=s, dtype=F32) for n in sizes] for s in range(4))
    v = [t.square() for t in v]
    want = [adamw_reference(*(t.to(D) for t in x), 5) for x in zip(p, g, m, v)]
    hap.hap_adamw_step(hap.hap_adamw_tensors(p, g, m, v), 5, 1e-3, 0.9, 0.95, 1e-8, 0.1)
    for a, (ref, _, _, off) in zip(p, want):
        close(a, ref, off, F32)


def test_step_of_an_expert_layer_and_head():
    """The operators as a training step uses them: gated experts, their gradients, the head's loss, the optimizer; gradients
    against autograd in 64 bits from the same 16-bit inputs.  Intermediate values are held in 16 bits, each off by half a step:
    a gradient that passes through r such roundings is off by about sqrt(r) 2^-9 of its norm, and by no more than r 2^-8."""
    E, H, F, V = 4, 128, 192, 777
    off, o = offsets_of([50, 0, 131, 76])
    rows = o[-1]
    x, w13, w2 = normal(rows, H), normal(E, 2 * F, H, seed=1, scale=H ** -0.5), normal(E, H, F, seed=2, scale=F ** -0.5)
    head, target = normal(V, H, seed=3, scale=H ** -0.5), torch.randint(0, V, (rows,), device="cuda")
    grad = torch.full((), 1.0 / rows, device="cuda")
    h, gu = hap.hap_expert_gated(x, w13, off)
    y = hap.hap_expert_matmul(h, w2, off)
    loss, lse = hap.hap_linear_cross_entropy(y, head, target)
    dy, dhead = hap.hap_linear_cross_entropy_backward(y, head, target, lse, grad)
    dgu, h2 = hap.hap_expert_gated_backward(dy, w2, off, gu)
    dw2 = hap.hap_expert_matmul(dy, h2, off, hap.EXPERT_GRAD_WEIGHT)
    dw13 = hap.hap_expert_matmul(dgu, x, off, hap.EXPERT_GRAD_WEIGHT)
    dx = hap.hap_expert_matmul(dgu, w13, off, hap.EXPERT_GRAD_INPUT)
    leaves = [t.to(D).requires_grad_() for t in (x, w13, w2, head)]
    X, W13, W2, HEAD = leaves
    ys = []
    for e in range(E):
        z = X[o[e]:o[e + 1]] @ W13[e].T
        ys.append((z[:, :F] * torch.sigmoid(z[:, :F]) * z[:, F:]) @ W2[e].T)
    total = torch.nn.functional.cross_entropy(torch.cat(ys) @ HEAD.T, target, reduction="sum") / rows
    refs = torch.autograd.grad(total, leaves)
    assert abs(loss.to(D).mean() - total) < 1e-3 * total
    for got, ref, r in zip((dx, dw13, dw2, dhead), refs, (8, 8, 7, 5)):
        assert torch.linalg.vector_norm(got.to(D) - ref) <= r * 2.0 ** -8 * torch.linalg.vector_norm(ref)
    params, grads = [w13, w2, head], [dw13, dw2, dhead]
    m, v = [torch.zeros(t.shape, device="cuda") for t in params], [torch.zeros(t.shape, device="cuda") for t in params]
    old = [t.to(D) for t in params]
    hap.hap_adamw_step(hap.hap_adamw_tensors(params, grads, m, v), 1, 1e-2)
    for t, a, g in zip(params, old, grads):         # the first step moves every value by lr against its gradient's sign
        want = a - 1e-2 * g.to(D) / (g.to(D).abs() + 1e-8)
        close(t, want, 16 * U * (a.abs() + 1e-2), BF)


def calls():
    off, o = offsets_of([100, 3, 0, 200])
    x, dy, w, w13 = normal(303, 256), normal(303, 320, seed=1), normal(4, 320, 256, seed=2), normal(4, 640, 256, seed=3)
    w2, head = normal(4, 320, 128, seed=4), normal(2003, 256, seed=5, scale=0.1)
    gu = normal(303, 256, seed=6)
    target = torch.arange(303, device="cuda") * 5
    grad = torch.full((), 0.01, device="cuda")
    lse = hap.hap_linear_cross_entropy(x, head, target)[1]
    space = hap.hap_linear_cross_entropy_workspace(x, head)
    one = torch.tensor([0, 1, 1, 2, 2], device="cuda")
    return {
        "forward": lambda: hap.hap_expert_matmul(x, w, off),
        "grad_input": lambda: hap.hap_expert_matmul(dy, w, off, hap.EXPERT_GRAD_INPUT),
        "grad_weight": lambda: hap.hap_expert_matmul(dy, x, off, hap.EXPERT_GRAD_WEIGHT),
        "gated": lambda: hap.hap_expert_gated(x, w13, off),
        "gated_backward": lambda: hap.hap_expert_gated_backward(dy, w2, off, gu),
        "loss": lambda: hap.hap_linear_cross_entropy(x, head, target, workspace=space),
        "loss_backward": lambda: hap.hap_linear_cross_entropy_backward(x, head, target, lse, grad, workspace=space),
        "loss_backward_few": lambda: hap.hap_linear_cross_entropy_backward(x[:5], head, target[:5], lse[:5], grad, workspace=space),
        "one_row": lambda: hap.hap_expert_matmul(x[:2], w, one),
    }


@pytest.mark.parametrize("name", ["forward", "grad_input", "grad_weight", "gated", "gated_backward", "loss", "loss_backward", "loss_backward_few", "one_row"])
def test_repeated_captured_and_on_another_stream(name):
    """The same bits from a second call, from a call on another stream, and from a graph that is replayed twice."""
    call = calls()[name]
    flat = lambda r: [r] if isinstance(r, torch.Tensor) else list(r)  # noqa: E731
    first = [t.clone() for t in flat(call())]
    assert all(torch.equal(a, b) for a, b in zip(first, flat(call())))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there = flat(call())
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, there))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = flat(call())
    for _ in range(2):
        for t in kept:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, kept))
    assert hap.hap_operator_status() == 0


def test_calls_on_two_streams_at_once():
    """Kernels that fill the device, side by side on two streams with work of their own, small ones among them."""
    table = calls()
    flat = lambda r: [r] if isinstance(r, torch.Tensor) else list(r)  # noqa: E731
    names = [n for n in table if not n.startswith("loss")]          # (the two loss calls share a workspace)
    want = {n: [t.clone() for t in flat(table[n]())] for n in names}
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for turn in range(6):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                for n in names if (turn + k) % 2 else names[::-1]:
                    got.append((n, flat(table[n]())))
    torch.cuda.synchronize()
    for n, r in got:
        assert all(torch.equal(a, b) for a, b in zip(want[n], r))
    assert hap.hap_operator_status() == 0


def test_stream_argument_and_captured_step():
    side = torch.cuda.Stream()
    x, w = normal(64, 128), normal(1, 64, 128, seed=1)
    off, _ = offsets_of([64])
    torch.cuda.synchronize()
    there = hap.hap_expert_matmul(x, w, off, stream=side)
    side.synchronize()
    assert torch.equal(there, hap.hap_expert_matmul(x, w, off))
    p, g, m, v = normal(5000), normal(5000, seed=1), torch.zeros(5000, device="cuda"), torch.zeros(5000, device="cuda")
    q = p.clone()
    t = hap.hap_adamw_tensors([p], [g], [m], [v])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hap.hap_adamw_step(t, 1, 1e-3)
    graph.replay()
    torch.cuda.synchronize()
    u = hap.hap_adamw_tensors([q], [g], [torch.zeros(5000, device="cuda")], [torch.zeros(5000, device="cuda")])
    hap.hap_adamw_step(u, 1, 1e-3)
    assert torch.equal(p, q)


def test_refusals_of_the_binding():
    x, w, off = normal(10, 64), normal(2, 32, 64), torch.tensor([0, 4, 10], device="cuda")
    bad = [
        lambda: hap.hap_expert_matmul(x.float(), w.float(), off),
        lambda: hap.hap_expert_matmul(x, w.half(), off),
        lambda: hap.hap_expert_matmul(x, w, off.int()),
        lambda: hap.hap_expert_matmul(x, w, off[:2]),
        lambda: hap.hap_expert_matmul(x[:, :32], w, off),
        lambda: hap.hap_expert_matmul(x, w.transpose(1, 2), off),
        lambda: hap.hap_expert_matmul(x, w, off, form=7),
        lambda: hap.hap_expert_matmul(x, w, off, accumulate=True),
        lambda: hap.hap_expert_matmul(x, w, off, out=torch.empty(10, 33, dtype=BF, device="cuda")),
        lambda: hap.hap_expert_matmul(x.cpu(), w, off),
        lambda: hap.hap_expert_matmul(x, w[:, :31], off),
        lambda: hap.hap_expert_gated(x, w[:, :31], off),
        lambda: hap.hap_expert_gated_backward(x, w.transpose(1, 2).contiguous(), off, x[:, :63]),
        lambda: hap.hap_linear_cross_entropy(x, w[0], torch.zeros(9, dtype=torch.int64, device="cuda")),
        lambda: hap.hap_linear_cross_entropy(x, w[0], torch.zeros(10, dtype=torch.int32, device="cuda")),
        lambda: hap.hap_linear_cross_entropy(x, w[0], torch.zeros(10, dtype=torch.int64, device="cuda"), workspace=torch.empty(16, dtype=torch.uint8, device="cuda")),
        lambda: hap.hap_linear_cross_entropy_backward(x, w[0], torch.zeros(10, dtype=torch.int64, device="cuda"), torch.zeros(10, device="cuda"), 1.0),
        lambda: hap.hap_adamw_tensors([x], [x.float()[:9]], [x.float()], [x.float()]),
        lambda: hap.hap_adamw_tensors([x], [x], [x], [x.float()]),
        lambda: hap.hap_adamw_tensors([x.t()], [x], [x.float()], [x.float()]),
        lambda: hap.hap_adamw_tensors([x], [x.half()], [x.float()], [x.float()]),
        lambda: hap.hap_adamw_step(hap.hap_adamw_tensors([x], [x], [x.float()], [x.float()]), 0, 1e-3),
        lambda: hap.hap_adamw_step(hap.hap_adamw_tensors([x], [x], [x.float()], [x.float()]), 1, 1e-3, beta1=1.0),
    ]
    for call in bad:
        with pytest.raises(hap.HapError):
            call()
