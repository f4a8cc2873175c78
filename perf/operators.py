"""Performance cases of the training operators beside the planner, through the package's public entry points.

The planner's cost model is fed by profiled times: of an expert's feed-forward products, of the output head, of the
optimizer's work per parameter.  These are the operators whose times they are, at the model shapes of the repository's five
configurations and what lies between them:

  matmul    products of rows sorted by expert with their expert's matrix, and the two gradients:
              forward      Y_i  = X_i W_e^T           X [rows][K], W [E][N][K], rows of expert e at offsets[e] .. offsets[e+1]
              grad_input   dX_i = dY_i W_e
              grad_weight  dW_e = sum over e's rows of dY_i^T X_i, added to what dW holds where the case says so
  gated     the first half of a gated feed-forward block, [g | u]_i = X_i W_e^T with W [E][2F][H] and h = silu(g) u, both
            kept for the backward pass; and the product in front of it backwards: dh = dY_i W2_e with W2 [E][H][F],
            dg = dh u (s + g s (1 - s)), du = dh g s with s = 1 / (1 + exp(-g)), and h again for W2's gradient
  loss      cross entropy of the output head: logits z = X W^T over the vocabulary, loss_i = log(sum_j exp z_ij) - z_i,t(i),
            0 where t(i) is -100, and with it the gradients of grad * sum_i loss_i
  adamw     one step of AdamW over a list of tensors, states in 32 bits or in 8

States in 8 bits: blocks of 256 values of a tensor share a scale, the largest magnitude s of the block.  A first moment is
held as c in -127 .. 127 and stands for s t |t| with t = c / 127; a second moment as c in 0 .. 255 and stands for s t^4 with
t = c / 255.  c is the nearest whole number of 127 sqrt(|m| / s), with m's sign, and of 255 sqrt(sqrt(v / s)), ties to even,
and at least 1 where v is not 0 (a second moment that was rounded to 0 under a first that was not would make a step of
m / eps).  The parameter is updated from the moments before they are rounded.  So that the codes are the same wherever they
are computed, what leads to them is defined in 32-bit operations, each rounded to nearest: t as c times the rounded 1 / 127
or 1 / 255; the moments read as (t |t|) s and ((t t) (t t)) s; m = m b1 + g (1 - b1) and v = v b2 + (g g) (1 - b2) with the
four factors rounded to 32 bits; c as written above.
"""
import math

import torch

own = False

IGNORE = -100
BLOCK = 256
_DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def listed():
    return [
        # one token's two experts of the smallest model: latency, and weights that are read for a single row each
        dict(name="matmul_one_token", op="matmul", form="forward", dtype="bf16", out="bf16", E=8, rows=2, spare=0, zipf=0.0, N=1024, K=4096, accumulate=False),
        # down projection of 64 experts, loads by Zipf's law, some experts with few rows; buffer longer than the rows
        dict(name="matmul_64_experts", op="matmul", form="forward", dtype="bf16", out="bf16", E=64, rows=32768, spare=117, zipf=1.2, N=2048, K=1024, accumulate=False),
        # gradient of the input for a rank's 20 of 160 experts, uneven rows
        dict(name="matmul_grad_input", op="matmul", form="grad_input", dtype="fp16", out="fp16", E=20, rows=6141, spare=3, zipf=1.4, N=5120, K=1536, accumulate=False),
        # gradient of the weights, added to the step's gradient in 32 bits as over the micro-batches of a pipeline
        dict(name="matmul_grad_weight", op="matmul", form="grad_weight", dtype="bf16", out="fp32", E=8, rows=8192, spare=0, zipf=1.2, N=4096, K=14336, accumulate=True),
        # a rank's 32 of 256 experts of the largest model, one micro-batch
        dict(name="gated_32_experts", op="gated", backward=False, dtype="bf16", E=32, rows=8190, spare=2, zipf=1.2, H=8192, F=2048),
        # backward through the gate, an ordinary micro-batch of 64 experts
        dict(name="gated_backward", op="gated", backward=True, dtype="bf16", E=64, rows=32760, spare=8, zipf=1.2, H=2048, F=1024),
        # the head's loss alone (evaluation), a vocabulary that no tile divides
        dict(name="loss_short", op="loss", backward=False, dtype="bf16", rows=129, H=1024, V=32003, ignored=0.1),
        # the head of the 256-device configuration in training: loss and both gradients
        dict(name="loss_gradients", op="loss", backward=True, dtype="bf16", rows=4096, H=5120, V=102400, ignored=0.05),
        # the largest vocabulary's slice of one of 8 tensor-parallel ranks, a whole sequence, in fp16
        dict(name="loss_slice_gradients", op="loss", backward=True, dtype="fp16", rows=8192, H=8192, V=16000, ignored=0.0),
        # norms, biases and a router only: launches count
        dict(name="adamw_small", op="adamw", dtype="bf16", bits=32, tensors=33, total=91001, largest=32768, step=7),
        # a rank's dense share of a model in 32-bit states
        dict(name="adamw_32", op="adamw", dtype="bf16", bits=32, tensors=61, total=201_000_003, largest=58_720_256, step=1000),
        # the same with states in 8 bits, read out as values afterwards (a check of the run, a checkpoint in 32 bits)
        dict(name="adamw_8", op="adamw", dtype="bf16", bits=8, tensors=61, total=150_000_001, largest=58_720_256, step=1000),
    ]


def _spread(rng, low, high, multiple=1):
    v = math.exp(rng.uniform(math.log(low), math.log(high)))
    return max(multiple, int(round(v / multiple)) * multiple)


def draw(rng):
    """Any of the operators: hidden sizes of 256 to 8192, experts of 256 to 14336, 1 to 64 of them, 1 to 32768 rows; 1 to
    8192 rows against vocabularies of 1000 to 128000; 1 to 80 tensors of 1000 to 150 million values in all."""
    op = rng.choice(["matmul", "matmul", "gated", "loss", "adamw"])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    if op in ("matmul", "gated"):
        while True:
            E, rows, wide, ffn = _spread(rng, 1, 64), _spread(rng, 1, 32768), _spread(rng, 256, 8192, 8), _spread(rng, 256, 14336, 8)
            if rows * wide * ffn < 4.0e11 and E * wide * ffn < 6.0e8:
                break
        zipf, spare = rng.choice([0.0, 1.2, 1.4]), rng.choice([0, 0, rng.randint(1, 200)])
        if op == "gated":
            return dict(op=op, backward=rng.random() < 0.5, dtype=dtype, E=E, rows=rows, spare=spare, zipf=zipf, H=wide, F=ffn)
        form = rng.choice(["forward", "forward", "grad_input", "grad_weight"])
        N, K = (wide, ffn) if rng.random() < 0.5 else (ffn, wide)
        out = "fp32" if form == "grad_weight" and rng.random() < 0.5 else dtype
        return dict(op=op, form=form, dtype=dtype, out=out, E=E, rows=rows, spare=spare, zipf=zipf, N=N, K=K, accumulate=out == "fp32" and rng.random() < 0.5)
    if op == "loss":
        while True:
            rows, H, V = _spread(rng, 1, 8192), _spread(rng, 256, 8192, 8), _spread(rng, 1000, 128000)
            if rows * H * V < 1.0e12:
                break
        return dict(op=op, backward=rng.random() < 0.6, dtype=dtype, rows=rows, H=H, V=V, ignored=rng.choice([0.0, 0.1, 0.5]))
    total = _spread(rng, 1000, 150_000_000)
    return dict(op=op, dtype=rng.choice(["bf16", "fp16", "fp32"]), bits=rng.choice([32, 8]), tensors=rng.randint(1, 80), total=total,
                largest=max(1, int(total * rng.uniform(0.1, 0.9))), step=rng.choice([1, 10, 5000]))


def _loads(case):
    """Rows of each expert by Zipf's law, largest first; the seed shuffles them over the experts."""
    weights = [(r + 1.0) ** -case["zipf"] for r in range(case["E"])]
    total = sum(weights)
    loads = [int(case["rows"] * w / total) for w in weights]
    short = case["rows"] - sum(loads)
    for r in range(short):
        loads[r % case["E"]] += 1
    return loads


def _sizes(case):
    """Tensor sizes: the largest, then pieces that halve down to odd little ones; they add up to the total."""
    left, sizes = case["total"], []
    for i in range(case["tensors"]):
        if i == case["tensors"] - 1:
            n = left
        else:
            n = min(case["largest"] >> (i // 3), max(1, left // 2)) - (i % 2)
        n = max(1, min(n, left - (case["tensors"] - 1 - i)))
        if n < 1 or left < 1:
            break
        sizes.append(n)
        left -= n
    return sizes


def _inputs(case, seed):
    """Inputs of a case, from the seed alone."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, dt = case["op"], _DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0, dtype=dt):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=dtype).mul_(scale)

    if op in ("matmul", "gated"):
        perm = torch.randperm(case["E"], generator=torch.Generator().manual_seed(seed)).tolist()
        loads = [_loads(case)[p] for p in perm]
        bounds = [0]
        for n in loads:
            bounds.append(bounds[-1] + n)
        s = dict(bounds=bounds, offsets=torch.tensor(bounds, dtype=torch.int64, device="cuda"))
        E, length = case["E"], case["rows"] + case["spare"]
        if op == "gated":
            H, F = case["H"], case["F"]
            if case["backward"]:
                s.update(dy=normal(length, H), w=normal(E, H, F, scale=H ** -0.5), gu=normal(length, 2 * F),
                         dgu=torch.zeros(length, 2 * F, dtype=dt, device="cuda"), h=torch.zeros(length, F, dtype=dt, device="cuda"))
            else:
                s.update(x=normal(length, H), w=normal(E, 2 * F, H, scale=H ** -0.5),
                         gu=torch.zeros(length, 2 * F, dtype=dt, device="cuda"), h=torch.zeros(length, F, dtype=dt, device="cuda"))
            return s
        N, K, out = case["N"], case["K"], _DTYPES[case["out"]]
        if case["form"] == "forward":
            s.update(a=normal(length, K), b=normal(E, N, K, scale=K ** -0.5), out=torch.zeros(length, N, dtype=out, device="cuda"))
        elif case["form"] == "grad_input":
            s.update(a=normal(length, N), b=normal(E, N, K, scale=N ** -0.5), out=torch.zeros(length, K, dtype=out, device="cuda"))
        else:
            s.update(a=normal(length, N), b=normal(length, K, scale=0.1))
            s["out"] = normal(E, N, K, dtype=out) if case["accumulate"] else torch.zeros(E, N, K, dtype=out, device="cuda")
        return s
    if op == "loss":
        rows, H, V = case["rows"], case["H"], case["V"]
        x = normal(rows, H)
        target = torch.randint(0, V, (rows,), generator=gen, device="cuda")
        target[torch.rand(rows, generator=gen, device="cuda") < case["ignored"]] = IGNORE
        scale = 512.0 if dt == torch.float16 else 1.0                # loss scaling, as training in fp16 has
        return dict(x=x, w=normal(V, H, scale=2.0 * H ** -0.5), target=target, grad=torch.full((), scale / rows, device="cuda"))
    sizes = _sizes(case)
    total = sum(sizes)
    s = dict(sizes=sizes, p=normal(total, scale=0.02), g=normal(total, scale=1e-3))
    m, v = normal(total, scale=1e-4, dtype=torch.float32), normal(total, scale=1e-3, dtype=torch.float32).square_()
    if case["bits"] == 8:
        blocks = [-(-n // BLOCK) for n in sizes]
        at = torch.arange(total, device="cuda")            # where each value is when every tensor begins a block of its own
        start = 0
        first = 0
        for n, b in zip(sizes, blocks):
            at[start:start + n] += first * BLOCK - start
            start, first = start + n, first + b
        padded = torch.zeros(2, first * BLOCK, device="cuda")
        padded[0, at], padded[1, at] = m, v
        (mc, ms), (vc, vs) = _to_8_bits(padded[0].view(-1, BLOCK), True), _to_8_bits(padded[1].view(-1, BLOCK), False)
        s.update(blocks=blocks, at=at, m=mc.view(-1)[at].to(torch.int8), v=vc.view(-1)[at].to(torch.uint8), m_scale=ms, v_scale=vs,
                 m_value=torch.empty(total, device="cuda"), v_value=torch.empty(total, device="cuda"))
    else:
        s.update(m=m, v=v)
    return s


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if own:
        import paper_2609_39350_b200 as hap
        if case["op"] == "adamw":
            split = lambda t: list(t.split(s["sizes"]))  # noqa: E731
            more = {}
            if case["bits"] == 8:
                more = dict(m_scale=list(s["m_scale"].split(s["blocks"])), v_scale=list(s["v_scale"].split(s["blocks"])))
                s["values"] = split(s["m_value"]), split(s["v_value"])
            s["tensors"] = hap.hap_adamw_tensors(split(s["p"]), split(s["g"]), split(s["m"]), split(s["v"]), **more)
        elif case["op"] == "loss":
            s["workspace"] = hap.hap_linear_cross_entropy_workspace(s["x"], s["w"])
    return s


_HYPER = dict(lr=3e-4, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1)


def run(s):
    case = s["case"]
    if own:
        import paper_2609_39350_b200 as hap
        if case["op"] == "matmul":
            form = {"forward": hap.EXPERT_FORWARD, "grad_input": hap.EXPERT_GRAD_INPUT, "grad_weight": hap.EXPERT_GRAD_WEIGHT}[case["form"]]
            return hap.hap_expert_matmul(s["a"], s["b"], s["offsets"], form, out=s["out"], accumulate=case["accumulate"])
        if case["op"] == "gated":
            if case["backward"]:
                return hap.hap_expert_gated_backward(s["dy"], s["w"], s["offsets"], s["gu"], dgu=s["dgu"], h=s["h"])
            return hap.hap_expert_gated(s["x"], s["w"], s["offsets"], gu=s["gu"], h=s["h"])
        if case["op"] == "loss":
            loss, lse = hap.hap_linear_cross_entropy(s["x"], s["w"], s["target"], ignore_index=IGNORE, workspace=s["workspace"])
            if not case["backward"]:
                return loss, lse
            return loss, lse, *hap.hap_linear_cross_entropy_backward(s["x"], s["w"], s["target"], lse, s["grad"], ignore_index=IGNORE, workspace=s["workspace"])
        hap.hap_adamw_step(s["tensors"], step=case["step"], **_HYPER)
        if case["bits"] == 8:
            hap.hap_adamw_state(s["tensors"], *s["values"])
            return s["p"], s["m_value"], s["v_value"]
        return s["p"], s["m"], s["v"]
    if case["op"] == "matmul":
        return _matmul(s, case)
    if case["op"] == "gated":
        return _gated_backward(s) if case["backward"] else _gated(s)
    if case["op"] == "loss":
        return _loss(s, case["backward"])
    return _adamw_8(s, case) if case["bits"] == 8 else _adamw_32(s, case)


def _groups(s):
    """(expert, its first row, the row behind its last) of the experts with rows: a product each is the plain way, since a
    batched product over padded groups would do many times the work under uneven loads."""
    return [(e, a, b) for e, (a, b) in enumerate(zip(s["bounds"], s["bounds"][1:])) if b > a]


def _matmul(s, case):
    a, b, out = s["a"], s["b"], s["out"]
    if case["form"] == "grad_weight":
        if not case["accumulate"]:
            out.zero_()
        for e, i, j in _groups(s):
            d = a[i:j].float().t() @ b[i:j].float()
            out[e].copy_(out[e] + d if case["accumulate"] else d)
        return out
    for e, i, j in _groups(s):
        w = b[e].float()
        out[i:j].copy_(a[i:j].float() @ (w.t() if case["form"] == "forward" else w))
    return out


def _gated(s):
    x, w, gu, h = s["x"], s["w"], s["gu"], s["h"]
    F = h.shape[1]
    for e, i, j in _groups(s):
        z = x[i:j].float() @ w[e].float().t()
        gu[i:j].copy_(z)
        g, u = z[:, :F], z[:, F:]
        h[i:j].copy_(g / (1 + torch.exp(-g)) * u)
    return h, gu


def _gated_backward(s):
    dy, w, gu, dgu, h = s["dy"], s["w"], s["gu"], s["dgu"], s["h"]
    F = h.shape[1]
    for e, i, j in _groups(s):
        dh = dy[i:j].float() @ w[e].float()
        g, u = gu[i:j, :F].float(), gu[i:j, F:].float()
        sig = 1 / (1 + torch.exp(-g))
        dgu[i:j, :F].copy_(dh * u * (sig + g * sig * (1 - sig)))
        dgu[i:j, F:].copy_(dh * g * sig)
        h[i:j].copy_(g * sig * u)
    return dgu, h


def _loss(s, backward):
    x, w, target = s["x"].float(), s["w"].float(), s["target"]
    z = x @ w.t()
    top = z.amax(1, keepdim=True)
    lse = (top + torch.log(torch.exp(z - top).sum(1, keepdim=True))).squeeze(1)
    valid = target != IGNORE
    at = torch.where(valid, target, 0).unsqueeze(1)
    loss = torch.where(valid, lse - z.gather(1, at).squeeze(1), 0)
    if not backward:
        return loss, lse
    d = z.sub_(lse.unsqueeze(1)).exp_()
    d.scatter_add_(1, at, torch.full_like(lse, -1).unsqueeze(1))
    d.mul_((valid * s["grad"]).unsqueeze(1))
    return loss, lse, (d @ w).to(s["x"].dtype), (d.t() @ x).to(s["w"].dtype)


def _corrections(case):
    return 1 - _HYPER["beta1"] ** case["step"], 1 - _HYPER["beta2"] ** case["step"]


def _adamw_32(s, case):
    b1, b2, lr = _HYPER["beta1"], _HYPER["beta2"], _HYPER["lr"]
    c1, c2 = _corrections(case)
    p, g, m, v = s["p"], s["g"].float(), s["m"], s["v"]
    m.mul_(b1).add_(g * (1 - b1))
    v.mul_(b2).add_(g * g * (1 - b2))
    p.copy_(p.float() * (1 - lr * _HYPER["weight_decay"]) - lr / c1 * m / (torch.sqrt(v) * c2 ** -0.5 + _HYPER["eps"]))
    return p, m, v


def _to_8_bits(x, signed):
    """Codes and scales of blocks (the last dimension), as the head of this file defines them."""
    s = x.abs().amax(-1)
    r = torch.where(s > 0, s, 1).unsqueeze(-1)
    if signed:
        return torch.copysign(torch.round(torch.sqrt(x.abs() / r) * 127), x), s
    return torch.round(torch.sqrt(torch.sqrt(x / r)) * 255).clamp_(min=1).where(x > 0, 0), s


def _from_8_bits(code, scale, signed):
    t = code * torch.full((), 1.0, device="cuda", dtype=scale.dtype).div(127 if signed else 255)
    return t * t.abs() * scale if signed else (t * t) * (t * t) * scale


def _adamw_8(s, case):
    b1, b2, lr = _HYPER["beta1"], _HYPER["beta2"], _HYPER["lr"]
    c1, c2 = _corrections(case)
    p, g, at, blocks = s["p"], s["g"].float(), s["at"], s["m_scale"].numel()
    one = lambda x: torch.full((), x, device="cuda")  # noqa: E731  (factors in 32 bits, as the states' values are)
    of = at // BLOCK
    m = _from_8_bits(s["m"].float(), s["m_scale"][of], True) * one(b1) + g * one(1 - b1)
    v = _from_8_bits(s["v"].float(), s["v_scale"][of], False) * one(b2) + (g * g) * one(1 - b2)
    p.copy_(p.float() * (1 - lr * _HYPER["weight_decay"]) - lr / c1 * m / (torch.sqrt(v) * c2 ** -0.5 + _HYPER["eps"]))
    padded = torch.zeros(2, blocks * BLOCK, device="cuda")
    padded[0, at], padded[1, at] = m, v
    (mc, ms), (vc, vs) = _to_8_bits(padded[0].view(-1, BLOCK), True), _to_8_bits(padded[1].view(-1, BLOCK), False)
    mc, vc = mc.view(-1)[at], vc.view(-1)[at]
    s["m"].copy_(mc), s["v"].copy_(vc), s["m_scale"].copy_(ms), s["v_scale"].copy_(vs)
    s["m_value"].copy_(_from_8_bits(mc, ms[of], True)), s["v_value"].copy_(_from_8_bits(vc, vs[of], False))
    return p, s["m_value"], s["v_value"]


def work(case):
    op = case["op"]
    size = {"bf16": 2, "fp16": 2, "fp32": 4}
    if op in ("matmul", "gated"):
        rows, z = case["rows"], size[case["dtype"]]
        used = sum(n > 0 for n in _loads(case))
        if op == "gated":
            H, F = case["H"], case["F"]
            if case["backward"]:
                return {"bytes": z * (rows * (H + 5 * F) + used * H * F), "flops": 2.0 * rows * H * F}
            return {"bytes": z * (rows * (H + 3 * F) + used * 2 * H * F), "flops": 4.0 * rows * H * F}
        N, K = case["N"], case["K"]
        flops = 2.0 * rows * N * K
        if case["form"] == "grad_weight":
            return {"bytes": z * rows * (N + K) + size[case["out"]] * (2 * used if case["accumulate"] else case["E"]) * N * K, "flops": flops}
        return {"bytes": z * (rows * (N + K) + used * N * K), "flops": flops}
    if op == "loss":
        rows, H, V = case["rows"], case["H"], case["V"]
        z = size[case["dtype"]] * (rows + V) * H
        if case["backward"]:                    # three products; the logits are not kept, but that is the kernel's choice
            return {"bytes": 2 * z + 16 * rows, "flops": 6.0 * rows * H * V}
        return {"bytes": z + 16 * rows, "flops": 2.0 * rows * H * V}
    n, z = case["total"], size[case["dtype"]]
    if case["bits"] == 8:
        return {"bytes": n * (3 * z + 4 + 8) + n // BLOCK * 16, "flops": 30.0 * n}
    return {"bytes": n * (3 * z + 16), "flops": 15.0 * n}


def exact(case, seed):
    """The operators' definitions in 64 bits, written apart from run()'s plain forms."""
    s = _inputs(case, seed)
    d = torch.float64
    if case["op"] in ("matmul", "gated"):
        spans = list(zip(s["bounds"][:-1], s["bounds"][1:]))
        if case["op"] == "matmul":
            got = s["out"].to(d)
            for e, (i, j) in enumerate(spans):
                a = s["a"][i:j].to(d)
                if case["form"] == "grad_weight":
                    got[e] += torch.einsum("rn,rk->nk", a, s["b"][i:j].to(d))
                elif j > i:
                    got[i:j] = torch.einsum("rk,nk->rn" if case["form"] == "forward" else "rn,nk->rk", a, s["b"][e].to(d))
            return got
        F = case["F"]
        gu, h = torch.zeros(s["gu"].shape, dtype=d, device="cuda"), torch.zeros(s["h"].shape, dtype=d, device="cuda")
        for e, (i, j) in enumerate(spans):
            if j == i:
                continue
            if case["backward"]:
                g, u = s["gu"][i:j].to(d).split(F, dim=1)
                dh = torch.einsum("rn,nk->rk", s["dy"][i:j].to(d), s["w"][e].to(d))
                with torch.enable_grad():
                    g, u = g.clone().requires_grad_(), u.clone().requires_grad_()
                    y = g * torch.sigmoid(g) * u
                    gu[i:j] = torch.cat(torch.autograd.grad(y, (g, u), dh), 1)
                h[i:j] = y.detach()
            else:
                gu[i:j] = torch.einsum("rk,nk->rn", s["x"][i:j].to(d), s["w"][e].to(d))
                g, u = gu[i:j].split(F, dim=1)
                h[i:j] = g * torch.sigmoid(g) * u
        return (gu, h) if case["backward"] else (h, gu)
    if case["op"] == "loss":
        x, w, t = s["x"].to(d), s["w"].to(d), s["target"]
        z = torch.einsum("rh,vh->rv", x, w)
        lse = torch.logsumexp(z, 1)
        rows = torch.arange(t.numel(), device="cuda")
        kept = t >= 0
        loss = torch.zeros_like(lse)
        loss[kept] = lse[kept] - z[rows[kept], t[kept]]
        if not case["backward"]:
            return loss, lse
        z = torch.softmax(z, 1)
        z[rows[kept], t[kept]] -= 1
        z[~kept] = 0
        z *= s["grad"].item()
        return loss, lse, torch.einsum("rv,vh->rh", z, w), torch.einsum("rv,rh->vh", z, x)
    y = _HYPER
    m, v, g, p = (s[k].to(d) for k in "mvgp")
    if case["bits"] == 8:
        # the definition's 32-bit operations: computed in 64 bits and rounded to 32 after each, which is the correctly rounded
        # 32-bit result (53 bits are more than twice 24 and two)
        r = lambda x: x.to(torch.float32).to(d)  # noqa: E731
        c = lambda x: torch.tensor(x, dtype=d).to(torch.float32).item()  # noqa: E731
        of, n = s["at"] // BLOCK, s["m_scale"].numel()

        def read(m, v, ms, vs):
            t, u = r(m * c(1 / 127)), r(v * c(1 / 255))
            u = r(u * u)
            return r(r(t * t.abs()) * ms), r(r(u * u) * vs)

        m, v = read(m, v, s["m_scale"].to(d)[of], s["v_scale"].to(d)[of])
        m = r(r(m * c(y["beta1"])) + r(g * c(1 - y["beta1"])))
        v = r(r(v * c(y["beta2"])) + r(r(g * g) * c(1 - y["beta2"])))
    else:
        m = torch.lerp(g, m, y["beta1"])
        v = torch.lerp(g ** 2, v, y["beta2"])
    p = p - y["lr"] * (m / (1 - y["beta1"] ** case["step"]) / (torch.sqrt(v / (1 - y["beta2"] ** case["step"])) + y["eps"]) + y["weight_decay"] * p)
    if case["bits"] == 32:
        return p, m, v
    ms = torch.zeros(n, dtype=d, device="cuda").scatter_reduce_(0, of, m.abs(), "amax")[of]
    vs = torch.zeros(n, dtype=d, device="cuda").scatter_reduce_(0, of, v, "amax")[of]
    t = torch.round(r(r(torch.sqrt(r(m.abs() / ms.clamp(min=1e-300)))) * 127))
    u = torch.round(r(r(torch.sqrt(r(torch.sqrt(r(v / vs.clamp(min=1e-300)))))) * 255))
    return p, *read(torch.sign(m) * t, torch.where(v > 0, u.clamp(min=1), 0), ms, vs)
