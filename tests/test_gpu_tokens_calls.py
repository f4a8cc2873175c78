"""The operators on a token's way as they are used: a layer of experts from the embedding to the gradients, captured and replayed calls,
streams, and calls that their description allows and that are easily forgotten."""
import os
import subprocess
import sys

import pytest
import torch

import paper_2609_39350_b200 as hap
import token_reference as ref
from test_gpu_operators import BF, D, F32, normal, wide
from test_gpu_tokens import places_of

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Layer:
    """Embedding, norm, router, gated experts, residual: forwards and backwards in 16 bits, through the package's functions."""

    def __init__(self, tokens=700, V=500, H=256, E=16, k=4, F=128):
        self.routing = hap.hap_routing(E, k, hap.SIGMOID, groups=4, kept_groups=2, group_best=2, renormalise=True, scale=1.5)
        gen = torch.Generator(device="cuda").manual_seed(5)
        self.tokens = torch.randint(0, V, (tokens,), device="cuda", generator=gen)
        self.table, self.w, self.b = normal(V, H, scale=1.0), normal(H, seed=1, scale=0.1) + 1, normal(H, seed=2, scale=0.1)
        self.router, self.bias = normal(E, H, seed=3, scale=H ** -0.5), normal(E, seed=4, dtype=F32, scale=0.05)
        self.w13, self.w2 = normal(E, 2 * F, H, seed=5, scale=H ** -0.5), normal(E, H, F, seed=6, scale=F ** -0.5)
        self.dout = normal(tokens, H, seed=7)
        self.all = torch.tensor([0, tokens], device="cuda")
        self.E, self.k, self.H, self.V = E, k, H, V

    def run(self):
        x = hap.hap_embedding(self.tokens, self.table, scale=2.0)
        n, mean, rstd = hap.hap_layer_norm(x, self.w, self.b)
        logits = hap.hap_expert_matmul(n, self.router[None], self.all)
        experts, weights = hap.hap_route(self.routing, logits, bias=self.bias)
        offsets, places = hap.hap_expert_order(experts, self.E)
        rows = hap.hap_expert_dispatch(n, places)
        h, gu = hap.hap_expert_gated(rows, self.w13, offsets)
        y = hap.hap_expert_matmul(h, self.w2, offsets)
        out = hap.hap_expert_combine(y, places, weights, base=x)
        # backwards
        dy, dweights = hap.hap_expert_combine_backward(self.dout, y, places, weights)
        dgu, h = hap.hap_expert_gated_backward(dy, self.w2, offsets, gu)
        dw2 = hap.hap_expert_matmul(dy, h, offsets, hap.EXPERT_GRAD_WEIGHT)
        dw13 = hap.hap_expert_matmul(dgu, rows, offsets, hap.EXPERT_GRAD_WEIGHT)
        drows = hap.hap_expert_matmul(dgu, self.w13, offsets, hap.EXPERT_GRAD_INPUT)
        dlogits = hap.hap_route_backward(self.routing, logits, experts, dweights)
        dn = hap.hap_expert_combine(drows, places)
        hap.hap_expert_matmul(dlogits, self.router[None], self.all, hap.EXPERT_GRAD_INPUT, out=dn, accumulate=True)
        drouter = hap.hap_expert_matmul(dlogits, n, self.all, hap.EXPERT_GRAD_WEIGHT)
        dx, dnw, dnb = hap.hap_layer_norm_backward(dn, x, self.w, rstd, mean=mean, base=self.dout)
        dtable = hap.hap_embedding_backward(self.tokens, dx, torch.empty(self.V, self.H, device="cuda"), scale=2.0)
        return dict(experts=experts, out=out, dw2=dw2, dw13=dw13, drouter=drouter[0], dnw=dnw, dnb=dnb, dtable=dtable)

    def reference(self, experts):
        """The same in 64 bits, differentiated by autograd, for given experts."""
        with torch.enable_grad():
            leaves = dict(dtable=self.table, dnw=self.w, dnb=self.b, drouter=self.router, dw13=self.w13, dw2=self.w2)
            p = {k: t.to(D).requires_grad_() for k, t in leaves.items()}
            x = p["dtable"][self.tokens] * 2.0
            n, _, _ = ref.norm(x, p["dnw"], p["dnb"], 1e-5, True)
            weights = ref.weights_of(n @ p["drouter"].T, experts, "sigmoid", True, 1.5)
            out = x
            for e in range(self.E):
                i, j = torch.nonzero(experts == e, as_tuple=True)
                g, u = (n[i] @ p["dw13"][e].T).chunk(2, dim=1)
                out = out.index_add(0, i, weights[i, j, None] * ((g * torch.sigmoid(g) * u) @ p["dw2"][e].T))
            grads = torch.autograd.grad(out, list(p.values()), self.dout.to(D))
        return dict(out=out.detach(), **dict(zip(p, grads)))


def test_a_layer_of_experts_forwards_and_backwards():
    layer = Layer()
    got = layer.run()
    want = layer.reference(got["experts"].long())
    # each tensor between two calls is rounded to 16 bits, by up to 2^-8 of a value, by 2^-9 in the mean; the gradients have some ten such
    # roundings behind them, each of which is passed on by linear maps of about its own size: 10 times 2^-8 of the norms
    for name, w in want.items():
        assert torch.linalg.norm(got[name].to(D) - w) <= 10 * 2.0 ** -8 * torch.linalg.norm(w), name
    logits = hap.hap_expert_matmul(hap.hap_layer_norm(hap.hap_embedding(layer.tokens, layer.table, scale=2.0), layer.w, layer.b)[0], layer.router[None], layer.all)
    for row, chosen in zip(logits[:50].double().cpu().tolist(), got["experts"][:50].cpu().tolist()):
        assert chosen == ref.route(row, layer.bias.double().cpu().tolist(), 4, "sigmoid", 4, 2, 2)[0]


def test_a_layer_gives_the_same_again_and_captured():
    layer = Layer()
    first = layer.run()
    for name, t in layer.run().items():
        assert torch.equal(t, first[name]), name
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = layer.run()
    # other inputs at the same places
    other = Layer()
    layer.tokens.copy_((layer.tokens * 7 + 3) % layer.V)
    other.tokens.copy_(layer.tokens)
    layer.bias.neg_(), other.bias.neg_()
    graph.replay()
    want = other.run()
    for name, t in kept.items():
        assert torch.equal(t, want[name]), name
    assert hap.hap_operator_status() == 0


def test_a_graph_is_captured_while_gradients_of_the_same_leaf_are_alive():
    """The functions record nothing: leaves that require gradients may be used eagerly and in a capture side by side."""
    w = normal(264, dtype=F32).requires_grad_()
    x = normal(40, 264, dtype=F32)
    eager = (x * w).sum()
    y, mean, rstd = hap.hap_layer_norm(x, w)
    assert not y.requires_grad
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dx, dw, _ = hap.hap_layer_norm_backward(x, x, w, rstd, mean=mean)
    graph.replay()
    eager.backward()
    assert torch.allclose(w.grad, x.sum(0), atol=1e-3) and torch.equal(dw, hap.hap_layer_norm_backward(x, x, w, rstd, mean=mean)[1])


def test_two_streams_at_once():
    a, b = Layer(), Layer(tokens=900, H=512, E=8, k=2)
    b.routing = hap.hap_routing(8, 2)
    want = a.run(), b.run()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(s):
            x = a.run()
        with torch.cuda.stream(t):
            y = b.run()
        torch.cuda.synchronize()
        for got, w in zip((x, y), want):
            assert all(torch.equal(got[k], w[k]) for k in w)
    # the stream argument
    logits = normal(300, 64)
    torch.cuda.synchronize()
    e, w = hap.hap_route(hap.hap_routing(64, 4), logits, stream=s)
    s.synchronize()
    assert torch.equal(e, hap.hap_route(hap.hap_routing(64, 4), logits)[0])


def test_what_is_refused():
    x, cpu = normal(8, 64), torch.zeros(8, 64, dtype=BF)
    places, tokens = torch.zeros(8, 2, dtype=torch.int32, device="cuda"), torch.zeros(8, dtype=torch.int64, device="cuda")
    r = hap.hap_routing(64, 2)
    mean = torch.zeros(8, device="cuda")
    bad = [
        lambda: hap.hap_route(r, cpu), lambda: hap.hap_route(r, x[:, :32]), lambda: hap.hap_route(r, x.double()), lambda: hap.hap_route(r, x, bias=x[0]),
        lambda: hap.hap_route(r, x, experts=places.long()), lambda: hap.hap_route(r, x, experts=places[:4]), lambda: hap.hap_route(r, x.t()),
        lambda: hap.hap_route_backward(r, x, places, places), lambda: hap.hap_route_backward(r, x, places, mean[:, None].expand(8, 2)),
        lambda: hap.hap_expert_order(places.long(), 4), lambda: hap.hap_expert_order(places, 0), lambda: hap.hap_expert_order(places, 4, offsets=tokens),
        lambda: hap.hap_expert_order(torch.zeros(8, 33, dtype=torch.int32, device="cuda"), 4),
        lambda: hap.hap_expert_dispatch(x, places[:4]), lambda: hap.hap_expert_dispatch(x, places, out=x[:, :32]), lambda: hap.hap_expert_dispatch(x, places, out=x.float()),
        lambda: hap.hap_expert_combine(x, places, weights=x[:, :2]), lambda: hap.hap_expert_combine(x, places, base=x[:4]), lambda: hap.hap_expert_combine(cpu, places),
        lambda: hap.hap_expert_combine_backward(x[:4], x, places), lambda: hap.hap_expert_combine_backward(x, x.float(), places),
        lambda: hap.hap_embedding(tokens.int(), x), lambda: hap.hap_embedding(tokens, x, out=x[:4]), lambda: hap.hap_embedding(tokens[:, None], x),
        lambda: hap.hap_embedding_backward(tokens, x, x[:, :32]), lambda: hap.hap_embedding_backward(tokens, x, normal(9, 64, dtype=torch.float16)),
        lambda: hap.hap_embedding_backward(tokens, x[:4], x), lambda: hap.hap_embedding_backward(tokens, x, x, workspace=torch.empty(1, dtype=torch.uint8, device="cuda")),
        lambda: hap.hap_layer_norm(x, w=x[0].half()), lambda: hap.hap_layer_norm(x, w=mean), lambda: hap.hap_layer_norm(x, y=x.float()), lambda: hap.hap_layer_norm(x, eps=-1.0),
        lambda: hap.hap_layer_norm_backward(x, x, None, mean[:4]), lambda: hap.hap_layer_norm_backward(x, x, None, mean, db=torch.zeros(64, device="cuda")),
        lambda: hap.hap_layer_norm_backward(x, x, x[0], mean, dw=x[0].half()), lambda: hap.hap_layer_norm_backward(x, x, None, mean, accumulate=True),
        lambda: hap.hap_expert_order(places, 4, first=1 << 31), lambda: hap.hap_expert_order(places, 1025),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(hap.HapError):
            call()
            print(i)
    assert hap.hap_route(r, x)[0].shape == (8, 2)


def test_addresses_behind_2_to_the_31():
    """Matrices of more than 2^32 bytes and 2^31 values: the last rows are reached."""
    H, n = 8192, 270_000
    big = torch.zeros(n, H, dtype=BF, device="cuda")
    tokens = torch.tensor([n - 1, 0, n - 2, n - 1, 5], device="cuda")
    big[n - 1], big[n - 2], big[0], big[5] = 3, 2, 1, 4
    assert hap.hap_embedding(tokens, big)[:, 0].tolist() == [3, 1, 2, 3, 4]
    places = torch.tensor([[n - 1, 0], [n - 2, 5]], dtype=torch.int32, device="cuda")
    assert hap.hap_expert_combine(big, places)[:, H - 1].tolist() == [4, 6]
    dw = hap.hap_expert_combine_backward(normal(2, H) * 0 + 1, big, places, want_dy=False)[1]
    assert dw.tolist() == [[3 * H, H], [2 * H, 4 * H]]
    dy = torch.ones(5, H, dtype=BF, device="cuda")
    hap.hap_embedding_backward(tokens, dy, big)
    assert big[n - 1, 7] == 2 and big[n - 2, H - 1] == 1 and big[n - 3].sum() == 0 and big.float().sum().item() == 5 * H
    hap.hap_expert_dispatch(dy[:2] * 9, places, out=big)
    assert (big[n - 1] == 9).all() and (big[n - 2] == 9).all() and (big[5] == 9).all() and not big[n - 3].any()
    rows = torch.zeros(n, H, dtype=BF, device="cuda")
    rows[n - 1] = torch.arange(H, device="cuda") % 2
    y, mean, rstd = hap.hap_layer_norm(rows, y=big)
    assert mean[n - 1] == 0.5 and not mean[:n - 1].any() and (y[n - 1].abs() - 1).abs().max() < 0.01
    dx, dw, db = hap.hap_layer_norm_backward(y, rows, None, rstd, mean=mean, dx=rows)
    assert abs(dw[0].item() - 1) < 0.01 and dx[n - 1].abs().max() < 0.01


@pytest.mark.parametrize("rows", [1, 2, 7])
def test_single_tokens(rows):
    """What a step of decoding does: as many rows as are answered at once."""
    layer = Layer(tokens=rows)
    got = layer.run()
    want = layer.reference(got["experts"].long())
    assert torch.linalg.norm(got["out"].to(D) - want["out"]) <= 10 * 2.0 ** -8 * torch.linalg.norm(want["out"])


def test_nothing_to_do():
    none, places = torch.zeros(0, 64, dtype=BF, device="cuda"), torch.zeros(0, 2, dtype=torch.int32, device="cuda")
    r = hap.hap_routing(64, 2)
    e, w = hap.hap_route(r, none)
    assert e.shape == w.shape == (0, 2) and hap.hap_route_backward(r, none, e, w).shape == (0, 64)
    offsets, p = hap.hap_expert_order(places, 5)
    assert not offsets.any() and offsets.numel() == 6 and p.shape == (0, 2)
    assert hap.hap_expert_dispatch(none, places).shape == (0, 64) and hap.hap_expert_combine(none, places).shape == (0, 64)
    # rows without a place, and no rows of experts at all
    x, none_of = normal(6, 64), torch.full((6, 2), -1, dtype=torch.int32, device="cuda")
    assert not hap.hap_expert_combine(none, none_of).any() and torch.equal(hap.hap_expert_combine(none, none_of, base=x), x)
    dy, dw = hap.hap_expert_combine_backward(x, none, none_of)
    assert dy.shape == (0, 64) and not dw.any()
    tokens = torch.zeros(0, dtype=torch.int64, device="cuda")
    assert hap.hap_embedding(tokens, x).shape == (0, 64)
    assert not hap.hap_embedding_backward(tokens, none, x.clone()).any() and torch.equal(hap.hap_embedding_backward(tokens, none, x.clone(), accumulate=True), x)


def test_workspaces_are_not_read_before_they_are_written():
    """A workspace that holds anything gives the same, and stays within its bytes."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    experts = torch.randint(0, 40, (3000, 4), device="cuda", generator=gen, dtype=torch.int32)
    tokens, dy = torch.randint(0, 3000, (9000,), device="cuda", generator=gen), normal(9000, 136)
    x = normal(900, 136)
    _, mean, rstd = hap.hap_layer_norm(x)
    calls = [
        (hap.hap_expert_order_workspace(experts, 40), lambda ws: hap.hap_expert_order(experts, 40, workspace=ws)),
        (hap.hap_embedding_backward_workspace(tokens, dy[:3000]), lambda ws: (hap.hap_embedding_backward(tokens, dy, torch.empty(3000, 136, device="cuda"), workspace=ws),)),
        (hap.hap_layer_norm_backward_workspace(x), lambda ws: hap.hap_layer_norm_backward(x, x, None, rstd, mean=mean, workspace=ws)),
    ]
    for ws, call in calls:
        want = call(None)
        for fill in (0, 0x7F, 0xFF):
            room = torch.full((ws.numel() + 4096,), fill, dtype=torch.uint8, device="cuda")
            for a, b in zip(call(room[:ws.numel()]), want):
                assert torch.equal(a, b)
            assert (room[ws.numel():] == fill).all()


FIRST = r"""
import sys
import torch
sys.path.insert(0, sys.argv[1])
import paper_2609_39350_b200 as hap
x = torch.ones(3000, 5000, device="cuda")
x[:, ::2] = 3
tokens, r = torch.arange(3000, device="cuda") % 7, hap.hap_routing(64, 8)
z = torch.arange(64, device="cuda").float().repeat(3000, 1)
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    y, mean, rstd = hap.hap_layer_norm(x)
    dx, dw, db = hap.hap_layer_norm_backward(y, x, None, rstd, mean=mean)
    e, w = hap.hap_route(r, z)
    offsets, places = hap.hap_expert_order(e, 64)
    g = hap.hap_embedding_backward(tokens, x, torch.empty(7, 5000, device="cuda"))
y.zero_()
graph.replay()
torch.cuda.synchronize()
assert (mean == 2).all() and ((dw - 3000).abs() < 1).all() and e[5].tolist() == list(range(63, 55, -1)) and offsets[-1] == 24000 and g[0, 0] == 3 * 429
print("DONE")
"""


def test_a_process_whose_first_calls_are_captured():
    r = subprocess.run([sys.executable, "-c", FIRST, ROOT], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "DONE" in r.stdout, r.stderr[-2000:]
