"""Performance cases of the operators on a token's way through a layer of experts, through the package's public entry points.

What stands between the products by expert that perf/operators.py measures: the router's choice, the rows' way to the experts
and back, the embedding in front of the first layer and the norms in front of each block, at the model shapes of the
repository's five configurations and what lies between them:

  route      k of E experts for every row from its logits z: scores s = softmax(z) or 1 / (1 + exp(-z)), values v = s + bias
             (z itself without a bias); of `groups` groups of experts that follow one another the `kept` with the largest sums of
             their `best` largest v; in these the k largest v, descending, ties to the lowest index.  Weights are scale s, or scale
             times s over the sum of the chosen.  An expert of logit -inf is never chosen; -1 and weight 0 where none are left.
             Values are compared as the numbers they are, so in 64 bits.  Backwards: the logits' gradient from the weights'
  rows       the places of the chosen (row, j) sorted by expert, equal ones in their order, -1 where the expert is not among
             first .. first + E - 1, with the experts' offsets; dispatch, out[place] = x[row]; combine, out[row] = base[row] +
             sum_j weight_j y[place_j]; and combine's gradients, dy[place_j] = weight_j dout[row], dweight_j = <dout[row], y[place_j]>
  embedding  out_i = scale w[t_i - first], 0 where t_i - first is not a row of w; and its gradient
             dw_v = scale sum of dy_i over t_i - first = v, added to what dw holds where the case says so
  norm       y = (x - mean) r w + b with r = 1 / sqrt(variance + eps), or without mean and b; and its gradients
             dx = base + r (g - mean(g) - xh mean(g xh)) with g = dy w, xh = (x - mean) r; dw = sum dy xh; db = sum dy
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-5


def listed():
    return [
        # one token and the router of the smallest model: latency
        dict(name="route_one_token", op="route", dtype="bf16", rows=1, E=8, k=2, scores="softmax", groups=1, kept=1, best=1, renormalise=True, scale=1.0, bias=False, masked=0.0, backward=False),
        # the router of 160 experts in training, 8 groups of which 3 are kept, all scores in the gradient
        dict(name="route_groups", op="route", dtype="fp32", rows=4095, E=160, k=6, scores="softmax", groups=8, kept=3, best=1, renormalise=False, scale=16.0, bias=False, masked=0.02, backward=True),
        # the largest router: sigmoid scores, chosen with a bias that balances the experts, padded rows masked; with its gradient
        dict(name="route_bias", op="route", dtype="fp32", rows=32768, E=256, k=8, scores="sigmoid", groups=8, kept=4, best=2, renormalise=True, scale=2.5, bias=True, masked=0.05, backward=True),
        # a few tokens on their way to 64 experts: launches count
        dict(name="rows_few", op="rows", way="dispatch", dtype="bf16", rows=5, k=8, experts=64, first=0, E=64, H=2048, weights=False, base=False),
        # a micro-batch to a rank's 20 of 160 experts: an eighth of the chosen are its own
        dict(name="rows_to_rank", op="rows", way="dispatch", dtype="bf16", rows=32767, k=6, experts=160, first=40, E=20, H=5120, weights=False, base=False),
        # back from all experts, weighted, added to the residual stream
        dict(name="rows_back", op="rows", way="combine", dtype="bf16", rows=8192, k=8, experts=256, first=0, E=256, H=8192, weights=True, base=True),
        # the same way backwards: the experts' gradients and the router's weights' own
        dict(name="rows_back_gradients", op="rows", way="combine_backward", dtype="fp16", rows=4001, k=6, experts=160, first=0, E=160, H=5120, weights=True, base=False),
        # lookup alone, a vocabulary that no tile divides
        dict(name="embedding_short", op="embedding", way="lookup", dtype="bf16", rows=129, H=1024, V=32003, first=0, vocabulary=32003, scale=32.0, out="bf16", accumulate=False),
        # lookup and the whole gradient of the 256-device configuration, words by Zipf's law
        dict(name="embedding_gradient", op="embedding", way="both", dtype="bf16", rows=16384, H=5120, V=102400, first=0, vocabulary=102400, scale=1.0, out="bf16", accumulate=False),
        # one of 8 ranks' slice of the largest vocabulary, added to the step's gradient in 32 bits
        dict(name="embedding_slice", op="embedding", way="gradient", dtype="bf16", rows=32768, H=8192, V=16000, first=0, vocabulary=128000, scale=1.0, out="fp32", accumulate=True),
        # a few rows through a norm without mean, weights in 32 bits
        dict(name="norm_few", op="norm", dtype="bf16", params="fp32", rows=17, H=4096, centred=False, base=False, backward=False),
        # a micro-batch forwards and backwards, a length that no tile divides, the residual stream's gradient added
        dict(name="norm_gradients", op="norm", dtype="bf16", params="bf16", rows=32760, H=5120, centred=True, base=True, backward=True),
    ]


def _spread(rng, low, high, multiple=1):
    v = math.exp(rng.uniform(math.log(low), math.log(high)))
    return max(multiple, int(round(v / multiple)) * multiple)


def draw(rng):
    """Any of the operators: 1 to 32768 rows, 4 to 512 experts of which 1 to 8 are chosen, hidden sizes of 256 to 8192 (one in
    four odd), vocabularies of 1000 to 128000 in up to 8 slices."""
    op = rng.choice(["route", "rows", "embedding", "norm"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    size = 4 if dtype == "fp32" else 2
    rows = _spread(rng, 1, 32768)
    H = _spread(rng, 256, 8192, rng.choice([8, 8, 8, 1]))
    if op == "route":
        groups = rng.choice([1, 1, 4, 8])
        E = groups * _spread(rng, 4 if groups == 1 else 2, 512 // groups)
        kept = groups if groups == 1 else rng.randint(2, groups)
        bias = rng.random() < 0.5
        return dict(op=op, dtype=dtype, rows=rows, E=E, k=rng.randint(1, min(8, E // groups * kept)), scores=rng.choice(["softmax", "sigmoid"]), groups=groups, kept=kept,
                    best=1 if groups == 1 else rng.choice([1, 2]), renormalise=rng.random() < 0.6, scale=rng.choice([1.0, 2.5, 16.0]), bias=bias, masked=rng.choice([0.0, 0.1]),
                    backward=rng.random() < 0.5)
    if op == "rows":
        way = rng.choice(["dispatch", "combine", "combine_backward"])
        experts, k = _spread(rng, 4, 512), rng.choice([1, 2, 2, 4, 6, 8])
        k = min(k, experts)
        while rows * k * H * size > (5.5e8 if way == "combine_backward" else 1.1e9):
            rows = max(1, rows // 2)
        ranks = rng.choice([1, 1, 2, 4])
        E = max(1, experts // ranks)
        return dict(op=op, way=way, dtype=dtype, rows=rows, k=k, experts=experts, first=rng.choice([0, experts - E]), E=E, H=H, weights=rng.random() < 0.7 if way != "dispatch" else False,
                    base=way == "combine" and rng.random() < 0.5)
    if op == "embedding":
        vocabulary, ranks = _spread(rng, 1000, 128000), rng.choice([1, 1, 2, 8])
        V = vocabulary // ranks
        way = rng.choice(["lookup", "both", "gradient"])
        out = "fp32" if rng.random() < 0.4 else dtype
        while V * H * max(size, 4 if out == "fp32" else 2) > 9.0e8 or rows * H * size > 2.8e8:
            H, rows = max(256, H // 2), max(1, rows // 2)
        return dict(op=op, way=way, dtype=dtype, rows=rows, H=H, V=V, first=V * rng.randrange(ranks), vocabulary=vocabulary, scale=rng.choice([1.0, 32.0]), out=out,
                    accumulate=way == "gradient" and out == "fp32" and rng.random() < 0.6)
    while rows * H * size > 3.3e8:
        rows = max(1, rows // 2)
    backward = rng.random() < 0.6
    return dict(op=op, dtype=dtype, params=rng.choice([dtype, "fp32"]), rows=rows, H=H, centred=rng.random() < 0.6, base=backward and rng.random() < 0.5, backward=backward)


def _normal(gen, *shape, dtype, scale=1.0, shift=0.0):
    t = torch.randn(*shape, generator=gen, device="cuda", dtype=dtype).mul_(scale)
    return t.add_(shift) if shift else t


def _chosen(case, gen):
    """int32 [rows][k]: different experts of a row, popular ones more often."""
    popular = -1.2 * torch.log(1.0 + torch.randperm(case["experts"], generator=gen, device="cuda").float())
    noise = torch.rand(case["rows"], case["experts"], generator=gen, device="cuda").clamp_(min=1e-20)
    return (popular - torch.log((-torch.log(noise)).clamp_(min=1e-20))).topk(case["k"], 1).indices.to(torch.int32)


def _order(experts, first, E):
    """(offsets, places) of the chosen experts, by a sort."""
    flat = experts.reshape(-1).long() - first
    flat = torch.where((flat >= 0) & (flat < E), flat, E)
    order = torch.sort(flat, stable=True).indices
    places = torch.empty_like(order)
    places[order] = torch.arange(order.numel(), device=order.device)
    loads = torch.zeros(E + 2, dtype=torch.int64, device=order.device).index_add_(0, flat + 1, torch.ones_like(flat))
    return loads.cumsum(0)[:E + 1], torch.where(flat < E, places, -1).to(torch.int32).view(experts.shape)


def _inputs(case, seed):
    """Inputs of a case, from the seed alone."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, dt, rows = case["op"], _DTYPES[case["dtype"]], case["rows"]
    if op == "route":
        z = _normal(gen, rows, case["E"], dtype=dt, scale=1.5)
        padded = torch.rand(rows, generator=gen, device="cuda") < case["masked"]
        z[padded] = -math.inf
        s = dict(logits=z, bias=_normal(gen, case["E"], dtype=torch.float32, scale=0.05) if case["bias"] else None,
                 experts=torch.zeros(rows, case["k"], dtype=torch.int32, device="cuda"), weights=torch.zeros(rows, case["k"], device="cuda"))
        if case["backward"]:
            s.update(dweights=_normal(gen, rows, case["k"], dtype=torch.float32), dlogits=torch.zeros(rows, case["E"], dtype=dt, device="cuda"))
        return s
    if op == "rows":
        k, H, way = case["k"], case["H"], case["way"]
        s = dict(experts=_chosen(case, gen))
        if way == "dispatch":
            return dict(s, x=_normal(gen, rows, H, dtype=dt), offsets=torch.zeros(case["E"] + 1, dtype=torch.int64, device="cuda"),
                        places=torch.zeros(rows, k, dtype=torch.int32, device="cuda"), out=torch.zeros(rows * k, H, dtype=dt, device="cuda"))
        s["places"] = _order(s["experts"], case["first"], case["E"])[1]
        s["y"] = _normal(gen, rows * k, H, dtype=dt)
        s["weights"] = torch.softmax(_normal(gen, rows, k, dtype=torch.float32), 1) if case["weights"] else None
        if way == "combine":
            return dict(s, base=_normal(gen, rows, H, dtype=dt) if case["base"] else None, out=torch.zeros(rows, H, dtype=dt, device="cuda"))
        return dict(s, dout=_normal(gen, rows, H, dtype=dt, scale=0.1), dy=torch.zeros(rows * k, H, dtype=dt, device="cuda"),
                    dweights=torch.zeros(rows, k, device="cuda"))
    H = case["H"]
    if op == "embedding":
        n, V = case["vocabulary"], case["V"]
        often = (1.0 / (10.0 + torch.arange(n, device="cuda", dtype=torch.float64))).cumsum(0)      # Zipf's law, its first ranks flattened
        word = torch.searchsorted(often, often[-1] * torch.rand(rows, generator=gen, device="cuda", dtype=torch.float64)).clamp_(max=n - 1)
        s = dict(tokens=torch.randperm(n, generator=gen, device="cuda")[word])
        if case["way"] != "gradient":
            s.update(w=_normal(gen, V, H, dtype=dt, scale=H ** -0.5), out=torch.zeros(rows, H, dtype=dt, device="cuda"))
        if case["way"] != "lookup":
            out = _DTYPES[case["out"]]
            s.update(dy=_normal(gen, rows, H, dtype=dt, scale=0.1),
                     dw=_normal(gen, V, H, dtype=out, scale=0.1) if case["accumulate"] else torch.zeros(V, H, dtype=out, device="cuda"))
        return s
    pt = _DTYPES[case["params"]]
    s = dict(x=_normal(gen, rows, H, dtype=dt, scale=2.0, shift=0.25), w=_normal(gen, H, dtype=pt, scale=0.1, shift=1.0),
             b=_normal(gen, H, dtype=pt, scale=0.1) if case["centred"] else None, y=torch.zeros(rows, H, dtype=dt, device="cuda"),
             mean=torch.zeros(rows, device="cuda") if case["centred"] else None, rstd=torch.zeros(rows, device="cuda"))
    if case["backward"]:
        s.update(dy=_normal(gen, rows, H, dtype=dt, scale=0.1), base=_normal(gen, rows, H, dtype=dt, scale=0.1) if case["base"] else None,
                 dx=torch.zeros(rows, H, dtype=dt, device="cuda"), dw=torch.zeros(H, dtype=pt, device="cuda"), db=torch.zeros(H, dtype=pt, device="cuda") if case["centred"] else None)
    return s


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if own:
        import paper_2609_39350_b200 as hap
        if case["op"] == "route":
            s["routing"] = hap.hap_routing(case["E"], case["k"], scores=hap.SOFTMAX if case["scores"] == "softmax" else hap.SIGMOID, groups=case["groups"], kept_groups=case["kept"],
                                           group_best=case["best"], renormalise=case["renormalise"], scale=case["scale"])
        elif case["op"] == "rows" and case["way"] == "dispatch":
            s["workspace"] = hap.hap_expert_order_workspace(s["experts"], case["E"])
        elif case["op"] == "embedding" and case["way"] != "lookup":
            s["workspace"] = hap.hap_embedding_backward_workspace(s["tokens"], s["dw"])
        elif case["op"] == "norm" and case["backward"]:
            s["workspace"] = hap.hap_layer_norm_backward_workspace(s["x"])
    return s


def run(s):
    return _run_own(s, s["case"]) if own else {"route": _route, "rows": _rows, "embedding": _embedding, "norm": _norm}[s["case"]["op"]](s, s["case"])


def _run_own(s, case):
    import paper_2609_39350_b200 as hap
    op = case["op"]
    if op == "route":
        hap.hap_route(s["routing"], s["logits"], bias=s["bias"], experts=s["experts"], weights=s["weights"])
        if not case["backward"]:
            return s["experts"], s["weights"]
        hap.hap_route_backward(s["routing"], s["logits"], s["experts"], s["dweights"], dlogits=s["dlogits"])
        return s["experts"], s["weights"], s["dlogits"]
    if op == "rows":
        if case["way"] == "dispatch":
            hap.hap_expert_order(s["experts"], case["E"], first=case["first"], offsets=s["offsets"], places=s["places"], workspace=s["workspace"])
            hap.hap_expert_dispatch(s["x"], s["places"], out=s["out"])
            return s["offsets"], s["places"], s["out"]
        if case["way"] == "combine":
            return hap.hap_expert_combine(s["y"], s["places"], weights=s["weights"], base=s["base"], out=s["out"])
        return hap.hap_expert_combine_backward(s["dout"], s["y"], s["places"], weights=s["weights"], dy=s["dy"], dweights=s["dweights"])
    if op == "embedding":
        got = []
        if case["way"] != "gradient":
            got.append(hap.hap_embedding(s["tokens"], s["w"], first=case["first"], scale=case["scale"], out=s["out"]))
        if case["way"] != "lookup":
            got.append(hap.hap_embedding_backward(s["tokens"], s["dy"], s["dw"], first=case["first"], scale=case["scale"], accumulate=case["accumulate"], workspace=s["workspace"]))
        return got
    hap.hap_layer_norm(s["x"], s["w"], s["b"], eps=EPS, centred=case["centred"], y=s["y"], mean=s["mean"], rstd=s["rstd"])
    if not case["backward"]:
        return [s[key] for key in ("y", "mean", "rstd") if s[key] is not None]
    hap.hap_layer_norm_backward(s["dy"], s["x"], s["w"], s["rstd"], mean=s["mean"], base=s["base"], dx=s["dx"], dw=s["dw"], db=s["db"], workspace=s["workspace"])
    return [s[key] for key in ("y", "mean", "rstd", "dx", "dw", "db") if s[key] is not None]


def _first_by(values, n):
    """Indices of the n largest of each row, descending, ties to the lowest."""
    return torch.sort(values, dim=1, descending=True, stable=True).indices[:, :n]


def _route(s, case):
    z, bias, k, groups = s["logits"].double(), s["bias"], case["k"], case["groups"]
    rows, E = z.shape
    closed = z == -math.inf
    if case["scores"] == "softmax":
        top = z.amax(1, keepdim=True)
        t = torch.exp(z - torch.where(closed.all(1, keepdim=True), 0, top))
        score = t / t.sum(1, keepdim=True).clamp(min=1e-300)
    else:
        score = 1 / (1 + torch.exp(-z))
    value = (score + bias).masked_fill(closed, -math.inf) if bias is not None else z
    if groups > 1:
        by_value = torch.where(closed, -math.inf, score) if bias is None else value
        best = torch.sort(by_value.view(rows, groups, E // groups), dim=2, descending=True).values[:, :, :case["best"]]
        total = torch.where(best[:, :, 0] > -math.inf, torch.where(best > -math.inf, best, 0).sum(2), -math.inf)
        kept = torch.zeros(rows, groups, dtype=torch.bool, device="cuda").scatter_(1, _first_by(total, case["kept"]), True)
        value = value.masked_fill(~kept.repeat_interleave(E // groups, 1), -math.inf)
    experts = _first_by(value, k)
    there = value.gather(1, experts) > -math.inf
    chosen = torch.where(there, score.gather(1, experts), 0).float()
    total = chosen.sum(1, keepdim=True).clamp(min=1e-30) if case["renormalise"] else 1.0
    weights = chosen / total * case["scale"]
    s["experts"].copy_(torch.where(there, experts, -1)), s["weights"].copy_(weights)
    if not case["backward"]:
        return s["experts"], s["weights"]
    g = torch.where(there, s["dweights"], 0) * case["scale"]
    if case["renormalise"]:
        g = (g - (g * chosen / total).sum(1, keepdim=True)) / total
    d = torch.zeros(rows, E, device="cuda").scatter_add_(1, experts, torch.where(there, g, 0))
    score = score.float()
    if case["scores"] == "softmax":
        d = score * (d - (d * score).sum(1, keepdim=True))
    else:
        d = d * score * (1 - score)
    s["dlogits"].copy_(d)
    return s["experts"], s["weights"], s["dlogits"]


def _rows(s, case):
    if case["way"] == "dispatch":
        offsets, places = _order(s["experts"], case["first"], case["E"])
        there = places >= 0
        of = torch.arange(case["rows"], device="cuda").unsqueeze(1).expand_as(places)[there]
        s["offsets"].copy_(offsets), s["places"].copy_(places)
        s["out"][places[there].long()] = s["x"][of]
        return s["offsets"], s["places"], s["out"]
    places, weights = s["places"], s["weights"]
    there = (places >= 0).unsqueeze(1)
    at = places.clamp(min=0).long()
    if case["way"] == "combine":
        total = s["base"].float() if case["base"] else torch.zeros(s["out"].shape, device="cuda")
        for j in range(case["k"]):
            row = torch.where(there[:, :, j], s["y"][at[:, j]].float(), 0)
            total = total + (row * weights[:, j:j + 1] if weights is not None else row)
        return s["out"].copy_(total)
    dout = s["dout"].float()
    for j in range(case["k"]):
        row = torch.where(there[:, :, j], s["y"][at[:, j]].float(), 0)
        s["dweights"][:, j] = (row * dout).sum(1)
        put = there[:, 0, j]
        s["dy"][at[put, j]] = (dout[put] * weights[put, j:j + 1] if weights is not None else dout[put]).to(s["dy"].dtype)
    return s["dy"], s["dweights"]


def _embedding(s, case):
    at, V = s["tokens"] - case["first"], case["V"]
    there = (at >= 0) & (at < V)
    got = []
    if case["way"] != "gradient":
        row = s["w"][at.clamp(0, V - 1)].float() * case["scale"]
        got.append(s["out"].copy_(torch.where(there.unsqueeze(1), row, 0)))
    if case["way"] != "lookup":
        total = s["dw"].float() if case["accumulate"] else torch.zeros(s["dw"].shape, device="cuda")
        total.index_add_(0, at[there], s["dy"][there].float() * case["scale"])
        got.append(s["dw"].copy_(total))
    return got


def _norm(s, case):
    x, w = s["x"].float(), s["w"].float()
    mean = x.mean(1, keepdim=True) if case["centred"] else 0.0
    rstd = 1 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + EPS)
    xh = (x - mean) * rstd
    s["y"].copy_(xh * w + s["b"].float() if case["centred"] else xh * w)
    s["rstd"].copy_(rstd.squeeze(1))
    if case["centred"]:
        s["mean"].copy_(mean.squeeze(1))
    if case["backward"]:
        dy = s["dy"].float()
        g = dy * w
        d = g - xh * (g * xh).mean(1, keepdim=True)
        if case["centred"]:
            d = d - g.mean(1, keepdim=True)
            s["db"].copy_(dy.sum(0))
        s["dx"].copy_(s["base"].float() + d * rstd if case["base"] else d * rstd)
        s["dw"].copy_((dy * xh).sum(0))
    return [s[key] for key in ("y", "mean", "rstd", "dx", "dw", "db") if s.get(key) is not None]


def work(case):
    op, rows = case["op"], case["rows"]
    size = {"bf16": 2, "fp16": 2, "fp32": 4}
    z = size[case["dtype"]]
    if op == "route":
        E, k = case["E"], case["k"]
        moved, flops = rows * (E * z + 8 * k), rows * E * 8.0
        if case["backward"]:                    # the logits again, which are the same input; the weights' gradient in, the logits' out
            moved, flops = moved + rows * (4 * k + E * z), flops * 2
        return {"bytes": moved + (4 * E if case["bias"] else 0), "flops": flops}
    if op == "rows":
        H, k, n = case["H"], case["k"], rows * case["k"]
        here = n * case["E"] / case["experts"]  # places of this rank, were the experts chosen alike
        if case["way"] == "dispatch":
            return {"bytes": 8 * n + 8 * (case["E"] + 1) + z * H * (min(rows, here) + here), "flops": 4.0 * n}
        if case["way"] == "combine":
            return {"bytes": n * (8 if case["weights"] else 4) + z * H * (here + rows * (2 if case["base"] else 1)), "flops": 2.0 * here * H}
        return {"bytes": n * (12 if case["weights"] else 8) + z * H * (rows + 2 * here), "flops": 3.0 * here * H}
    H = case["H"]
    if op == "embedding":
        V, moved, flops = case["V"], 8 * rows, 0.0
        here = rows * V / case["vocabulary"]
        share = sum(1 - math.exp(-rows * p) for p in _shares(case["vocabulary"])) * V / case["vocabulary"]      # different words of the slice
        if case["way"] != "gradient":
            moved, flops = moved + z * H * (share + rows), flops + rows * H
        if case["way"] != "lookup":
            out = size[case["out"]]
            moved, flops = moved + z * H * here + out * H * (2 * share if case["accumulate"] else V), flops + here * H
        return {"bytes": moved, "flops": flops}
    p = size[case["params"]]
    moved, flops = rows * (2 * H * z + (8 if case["centred"] else 4)) + 2 * H * p, 7.0 * rows * H
    if case["backward"]:
        moved, flops = moved + rows * H * z * (3 if case["base"] else 2) + 2 * H * p, flops + 12.0 * rows * H
    return {"bytes": moved, "flops": flops}


def _shares(n):
    """The words' shares of a text, by the law that the tokens are drawn from."""
    weights = [1.0 / (10.0 + r) for r in range(n)]
    total = sum(weights)
    return [w / total for w in weights]


def exact(case, seed):
    """The operators' definitions in 64 bits, written apart from run()'s plain forms."""
    s, d = _inputs(case, seed), torch.float64
    return {"route": _exact_route, "rows": _exact_rows, "embedding": _exact_embedding, "norm": _exact_norm}[case["op"]](s, case, d)


def _exact_route(s, case, d):
    z = s["logits"].to(d)
    rows, E, k = case["rows"], case["E"], case["k"]
    open_ = z > -math.inf
    score = torch.where(open_, z, -1e300).softmax(1) * open_ if case["scores"] == "softmax" else torch.sigmoid(z)
    # the values' places in each row, from the front: 0 for the largest, ties to the lowest index
    value = score + s["bias"].to(d) if case["bias"] else z
    value = torch.where(open_, value, -math.inf)
    allowed = open_.clone()
    if case["groups"] > 1:
        of = (value if case["bias"] else torch.where(open_, score, -math.inf)).unflatten(1, (case["groups"], -1))
        best = of.topk(min(case["best"], of.shape[2]), 2).values
        any_ = best[:, :, 0] > -math.inf
        total = torch.where(any_, best.clamp(min=-1e6).mul(best > -math.inf).sum(2), -math.inf)
        ahead = (total.unsqueeze(2) > total.unsqueeze(1)) | ((total.unsqueeze(2) == total.unsqueeze(1)) & (
            torch.arange(case["groups"], device="cuda").unsqueeze(1) < torch.arange(case["groups"], device="cuda")))
        kept = ahead.sum(1) < case["kept"]
        allowed &= kept.unsqueeze(2).expand(-1, -1, E // case["groups"]).flatten(1)
    experts = torch.full((rows, k), -1, dtype=torch.int64, device="cuda")
    chosen = torch.zeros(rows, k, dtype=d, device="cuda")
    every = torch.arange(rows, device="cuda")
    for j in range(k):                          # one after the other: the first of the largest that are left
        left = torch.where(allowed, value, -math.inf)
        top = left.amax(1, keepdim=True)
        e = (left == top).to(torch.uint8).argmax(1)
        some = allowed.any(1)
        experts[:, j] = torch.where(some, e, -1)
        chosen[:, j] = torch.where(some, score[every, e], 0)
        allowed[every, e] = False
    there = experts >= 0
    w = chosen.clone().requires_grad_()
    weights = w * case["scale"]
    if case["renormalise"]:
        weights = weights / torch.where(there.any(1, keepdim=True), w.sum(1, keepdim=True), 1)
    if not case["backward"]:
        return experts.to(torch.int32), weights.detach()
    (dscore,) = torch.autograd.grad(weights, w, torch.where(there, s["dweights"].to(d), 0))
    full = torch.zeros(rows, E + 1, dtype=d, device="cuda").scatter_(1, torch.where(there, experts, E), torch.where(there, dscore, 0))[:, :E]
    if case["scores"] == "softmax":
        dz = score * full - score * torch.einsum("re,re->r", score, full).unsqueeze(1)
    else:
        dz = full * score * torch.sigmoid(-z)
        dz = torch.where(open_, dz, 0)
    return experts.to(torch.int32), weights.detach(), dz


def _exact_rows(s, case, d):
    rows, k, first, E = case["rows"], case["k"], case["first"], case["E"]
    e = s["experts"].long().flatten()
    mine = (e >= first) & (e < first + E)
    of = torch.nonzero(mine).flatten()                          # numbers row * k + j, ascending
    key = (e[of] - first) * (rows * k) + of                     # different for all: any sort is the stable one
    of = of[key.argsort()]
    places = torch.full((rows * k,), -1, dtype=torch.int64, device="cuda")
    places[of] = torch.arange(of.numel(), device="cuda")
    if case["way"] == "dispatch":
        offsets = torch.tensor([0, *torch.bincount(e[of] - first, minlength=E).cumsum(0).tolist()], dtype=torch.int64, device="cuda")
        out = s["out"].to(d)
        out[:of.numel()] = s["x"].to(d)[of // k]
        return offsets, places.to(torch.int32).view(rows, k), out
    w = torch.ones(rows * k, dtype=d, device="cuda") if s["weights"] is None else s["weights"].to(d).flatten()
    if case["way"] == "combine":
        out = s["base"].to(d) if case["base"] else torch.zeros(rows, case["H"], dtype=d, device="cuda")
        return out.index_add_(0, of // k, s["y"][:of.numel()].to(d) * w[of].unsqueeze(1))
    dout = s["dout"].to(d)[of // k]
    dy, dw = s["dy"].to(d), torch.zeros(rows * k, dtype=d, device="cuda")
    dy[:of.numel()] = dout * w[of].unsqueeze(1)
    dw[of] = torch.einsum("nh,nh->n", dout, s["y"][:of.numel()].to(d))
    return dy, dw.view(rows, k)


def _exact_embedding(s, case, d):
    at = s["tokens"] - case["first"]
    mine = torch.nonzero((at >= 0) & (at < case["V"])).flatten()
    got = []
    if case["way"] != "gradient":
        out = torch.zeros(case["rows"], case["H"], dtype=d, device="cuda")
        out[mine] = s["w"].to(d)[at[mine]] * case["scale"]
        got.append(out)
    if case["way"] != "lookup":
        # sorted by word, running sums, differences at the words' ends would cancel: a product with the words' rows instead
        words, of = at[mine].unique(return_inverse=True)
        sums = torch.zeros(words.numel(), case["H"], dtype=d, device="cuda").index_add_(0, of, s["dy"].to(d)[mine])
        dw = s["dw"].to(d) if case["accumulate"] else torch.zeros(case["V"], case["H"], dtype=d, device="cuda")
        dw[words] += sums * case["scale"]
        got.append(dw)
    return got


def _exact_norm(s, case, d):
    with torch.enable_grad():
        x, w = s["x"].to(d).requires_grad_(), s["w"].to(d).requires_grad_()
        if case["centred"]:
            b = s["b"].to(d).requires_grad_()
            var, mean = torch.var_mean(x, 1, correction=0)
            rstd = (var + EPS).rsqrt()
            y = (x - mean.unsqueeze(1)) * rstd.unsqueeze(1) * w + b
            got, leaves = [y, mean, rstd], (x, w, b)
        else:
            rstd = (x.square().mean(1) + EPS).rsqrt()
            y = x * rstd.unsqueeze(1) * w
            got, leaves = [y, rstd], (x, w)
        if case["backward"]:
            dx, *rest = torch.autograd.grad(y, leaves, s["dy"].to(d))
            got += [dx + s["base"].to(d) if case["base"] else dx, *rest]
    return [t.detach() for t in got]
