"""Binding of the operators on a token's way through a layer of experts: routing, the rows' way to the experts and back, embedding,
layer norm.  As in operators.py: torch tensors in, same names as the C ABI, argument marshalling only; every function enqueues on
`stream` (default: the current one), returns without waiting and records nothing, the gradients are functions of their own.

One layer, forwards:

    experts, weights = hap_route(routing, logits)
    offsets, places = hap_expert_order(experts, E)
    rows = hap_expert_dispatch(x, places)
    h, gu = hap_expert_gated(rows, w13, offsets)
    y = hap_expert_combine(hap_expert_matmul(h, w2, offsets), places, weights, base=x)
"""
from __future__ import annotations

import copy
import ctypes as C

import numpy as np
import torch

from . import operators
from .operators import _HALVES, _MOST, _TYPES, _check, _here, _matrix, _now, _on_stream, _refuse, _vector

SOFTMAX, SIGMOID = 0, 1
_FLOATS = (torch.float32, *_HALVES)


class _Routing(C.Structure):
    _fields_ = [*[(n, C.c_int32) for n in ("E", "k", "scores", "groups", "kept_groups", "group_best", "renormalise")], ("scale", C.c_float)]


_typed = None


def _lib():
    global _typed
    if _typed is None:
        L = operators._lib()
        i, l, u, p, f = C.c_int32, C.c_int64, C.c_uint64, C.c_void_p, C.c_float
        L.hap_route.argtypes = [p, i, l, p, l, p, p, p, p]
        L.hap_route_backward.argtypes = [p, i, l, p, l, p, p, p, l, p]
        L.hap_expert_order_workspace.argtypes = [l, i, i, p]
        L.hap_expert_order.argtypes = [l, i, i, i, p, p, p, p, u, p]
        L.hap_expert_dispatch.argtypes = [i, l, i, i, l, p, l, p, p, l, p]
        L.hap_expert_combine.argtypes = [i, l, i, i, l, p, l, p, p, p, l, p, l, p]
        L.hap_expert_combine_backward.argtypes = [i, l, i, i, l, p, l, p, l, p, p, p, l, p, p]
        L.hap_embedding.argtypes = [i, l, i, l, l, p, p, l, f, p, l, p]
        L.hap_embedding_backward_workspace.argtypes = [l, i, l, p]
        L.hap_embedding_backward.argtypes = [i, i, i, l, i, l, l, p, p, l, f, p, l, p, u, p]
        L.hap_layer_norm.argtypes = [i, i, i, l, i, p, l, p, p, f, p, l, p, p, p]
        L.hap_layer_norm_backward_workspace.argtypes = [l, i, p]
        L.hap_layer_norm_backward.argtypes = [i, i, i, i, i, l, i, p, l, p, l, p, p, p, p, l, p, l, p, p, p, u, p]
        _typed = L
    return _typed


def _table(name, t, here, dtype, rows=None, cols=None):
    """Address of a table [rows][cols] whose rows follow one another."""
    try:
        r, c = t.shape
        if t.get_device() == here and t.dtype == dtype and c <= _MOST and (rows is None or r == rows) and (cols is None or c == cols) and t.is_contiguous():
            return t.data_ptr()
    except (AttributeError, TypeError, ValueError, RuntimeError):
        pass
    _here(name, t, here, (dtype,), 2)
    if (rows is not None and t.shape[0] != rows) or (cols is not None and t.shape[1] != cols):
        _refuse(f"{name}: shape {tuple(t.shape)} where {(rows, cols)} is needed")
    if t.shape[1] > _MOST:
        _refuse(f"{name}: rows of {t.shape[1]} values")
    if not t.is_contiguous():
        _refuse(f"{name}: rows must follow one another")
    return t.data_ptr()


def _space(name, need, workspace, here):
    """(address, bytes) of a workspace, made here where none is given."""
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=here)
    return _vector(name, workspace, here, torch.uint8), workspace.numel(), workspace


class HapRouting:
    """How a router chooses: see hap_routing."""

    def __init__(self, E, k, scores=SOFTMAX, groups=1, kept_groups=1, group_best=1, renormalise=True, scale=1.0):
        if not 1 <= E <= 1024 or not 1 <= k <= min(E, 32):
            _refuse(f"k: {k} of {E} experts (1 to 1024 of them, up to 32 chosen)")
        if scores not in (SOFTMAX, SIGMOID):
            _refuse("scores: SOFTMAX or SIGMOID")
        if not 1 <= groups <= 32 or E % groups or not 1 <= kept_groups <= groups or group_best < 1:
            _refuse(f"groups: {kept_groups} of {groups} groups (up to 32 of equal sizes), {group_best} experts of each")
        self.k, self.E = k, E
        self.struct = _Routing(E, k, scores, groups, kept_groups, group_best, bool(renormalise), scale)
        self.at = C.addressof(self.struct)


def hap_routing(E, k, scores=SOFTMAX, groups=1, kept_groups=1, group_best=1, renormalise=True, scale=1.0) -> HapRouting:
    """k of E experts by SOFTMAX or SIGMOID scores; from the kept_groups of `groups` groups with the largest sums of their group_best
    largest values; weights are the scores, over their sum where renormalise is set, times scale."""
    return HapRouting(E, k, scores, groups, kept_groups, group_best, renormalise, scale)


@_on_stream
def hap_route(routing: HapRouting, logits, bias=None, experts=None, weights=None):
    """(experts, weights): int32 and fp32 [rows][k], best first, from logits [rows][E].  bias: fp32 [E], added to the scores for the
    choice alone.  Experts of logit -inf are never chosen; -1 with weight 0 where none are left."""
    here, stream = _now()
    pz, ld = _matrix("logits", logits, here, _FLOATS, None, routing.E)
    rows = logits.shape[0]
    pb = _vector("bias", bias, here, torch.float32, routing.E) if bias is not None else None
    if experts is None:
        experts = torch.empty((rows, routing.k), dtype=torch.int32, device=logits.device)
    if weights is None:
        weights = torch.empty((rows, routing.k), dtype=torch.float32, device=logits.device)
    pe, pw = _table("experts", experts, here, torch.int32, rows, routing.k), _table("weights", weights, here, torch.float32, rows, routing.k)
    _check(_lib().hap_route(routing.at, _TYPES[logits.dtype], rows, pz, ld, pb, pe, pw, stream), "hap_route")
    return experts, weights


@_on_stream
def hap_route_backward(routing: HapRouting, logits, experts, dweights, dlogits=None):
    """dlogits [rows][E], of the logits' type, from the weights' gradients: fp32 [rows][k]."""
    here, stream = _now()
    pz, ld = _matrix("logits", logits, here, _FLOATS, None, routing.E)
    rows = logits.shape[0]
    pe, pg = _table("experts", experts, here, torch.int32, rows, routing.k), _table("dweights", dweights, here, torch.float32, rows, routing.k)
    if dlogits is None:
        dlogits = torch.empty((rows, routing.E), dtype=logits.dtype, device=logits.device)
    pd, ldd = _matrix("dlogits", dlogits, here, (logits.dtype,), rows, routing.E)
    _check(_lib().hap_route_backward(routing.at, _TYPES[logits.dtype], rows, pz, ld, pe, pg, pd, ldd, stream), "hap_route_backward")
    return dlogits


def _order_bytes(rows, k, E):
    if not 1 <= E <= 1024:
        _refuse(f"E: {E} experts")
    n = C.c_uint64()
    _check(_lib().hap_expert_order_workspace(rows, k, E, C.byref(n)), "hap_expert_order_workspace")
    return n.value


def hap_expert_order_workspace(experts, E):
    """A workspace for hap_expert_order of as many rows and experts; needed during a call only."""
    _table("experts", experts, torch.cuda.current_device(), torch.int32)
    return torch.empty(max(256, _order_bytes(*experts.shape, E)), dtype=torch.uint8, device=experts.device)


@_on_stream
def hap_expert_order(experts, E, first=0, offsets=None, places=None, workspace=None):
    """(offsets, places): the places of the chosen (row, j) sorted by expert, of the experts first .. first + E - 1 (-1 for others), int32
    [rows][k]; and where each expert's rows begin, int64 [E + 1]."""
    here, stream = _now()
    pe = _table("experts", experts, here, torch.int32)
    rows, k = experts.shape
    if not -(1 << 31) <= first < 1 << 31 or not 1 <= E <= 1024:
        _refuse(f"first, E: {E} experts from {first} on")
    if offsets is None:
        offsets = torch.empty(E + 1, dtype=torch.int64, device=experts.device)
    if places is None:
        places = torch.empty((rows, k), dtype=torch.int32, device=experts.device)
    po, pp = _vector("offsets", offsets, here, torch.int64, E + 1), _table("places", places, here, torch.int32, rows, k)
    ps, n, workspace = _space("workspace", 0 if workspace is not None else max(256, _order_bytes(rows, k, E)), workspace, here)
    _check(_lib().hap_expert_order(rows, k, first, E, pe, po, pp, ps, n, stream), "hap_expert_order")
    return offsets, places


@_on_stream
def hap_expert_dispatch(x, places, out=None):
    """out[places[i][j]] = x[i]: rows on their way to the experts.  out [n][H], rows * k of them unless given; rows that no place
    names, and so what lies behind the last expert's, are left as they are (unset in an output made here)."""
    here, stream = _now()
    px, ldx = _matrix("x", x, here, _FLOATS)
    rows, H = x.shape
    pp = _table("places", places, here, torch.int32, rows)
    k = places.shape[1]
    if out is None:
        out = torch.empty((rows * k, H), dtype=x.dtype, device=x.device)
    po, ldo = _matrix("out", out, here, (x.dtype,), None, H)
    _check(_lib().hap_expert_dispatch(_TYPES[x.dtype], rows, k, H, out.shape[0], px, ldx, pp, po, ldo, stream), "hap_expert_dispatch")
    return out


@_on_stream
def hap_expert_combine(y, places, weights=None, base=None, out=None):
    """out[i] = base[i] + sum_j weights[i][j] y[places[i][j]].  Without weights it is the gradient of hap_expert_dispatch."""
    here, stream = _now()
    py, ldy = _matrix("y", y, here, _FLOATS)
    placed, H = y.shape
    pp = _table("places", places, here, torch.int32)
    rows, k = places.shape
    kind = (y.dtype,)
    pw = _table("weights", weights, here, torch.float32, rows, k) if weights is not None else None
    pb, ldb = _matrix("base", base, here, kind, rows, H) if base is not None else (None, 0)
    if out is None:
        out = torch.empty((rows, H), dtype=y.dtype, device=y.device)
    po, ldo = _matrix("out", out, here, kind, rows, H)
    _check(_lib().hap_expert_combine(_TYPES[y.dtype], rows, k, H, placed, py, ldy, pp, pw, pb, ldb, po, ldo, stream), "hap_expert_combine")
    return out


@_on_stream
def hap_expert_combine_backward(dout, y, places, weights=None, dy=None, dweights=None, want_dy=True, want_dweights=True):
    """(dy, dweights): dy[places[i][j]] = weights[i][j] dout[i], other rows left as they are; dweights[i][j] = <dout[i], y[places[i][j]]>."""
    here, stream = _now()
    py, ldy = _matrix("y", y, here, _FLOATS)
    placed, H = y.shape
    pp = _table("places", places, here, torch.int32)
    rows, k = places.shape
    kind = (y.dtype,)
    pd, ldd = _matrix("dout", dout, here, kind, rows, H)
    pw = _table("weights", weights, here, torch.float32, rows, k) if weights is not None else None
    if dy is None and want_dy:
        dy = torch.empty((placed, H), dtype=y.dtype, device=y.device)
    if dweights is None and want_dweights:
        dweights = torch.empty((rows, k), dtype=torch.float32, device=y.device)
    pdy, lddy = _matrix("dy", dy, here, kind, placed, H) if dy is not None else (None, 0)
    pdw = _table("dweights", dweights, here, torch.float32, rows, k) if dweights is not None else None
    _check(_lib().hap_expert_combine_backward(_TYPES[y.dtype], rows, k, H, placed, pd, ldd, py, ldy, pp, pw, pdy, lddy, pdw, stream), "hap_expert_combine_backward")
    return dy, dweights


@_on_stream
def hap_embedding(tokens, w, first=0, scale=1.0, out=None):
    """out[i] = scale w[tokens[i] - first], 0 where that is not a row of w.  tokens: int64 [n]."""
    here, stream = _now()
    pt = _vector("tokens", tokens, here, torch.int64)
    pw, ldw = _matrix("w", w, here, _FLOATS)
    n, (V, H) = tokens.numel(), w.shape
    if out is None:
        out = torch.empty((n, H), dtype=w.dtype, device=w.device)
    po, ldo = _matrix("out", out, here, (w.dtype,), n, H)
    _check(_lib().hap_embedding(_TYPES[w.dtype], n, H, V, first, pt, pw, ldw, scale, po, ldo, stream), "hap_embedding")
    return out


def _embedding_bytes(n, H, V):
    if H > _MOST:
        _refuse(f"dw: rows of {H} values")
    b = C.c_uint64()
    _check(_lib().hap_embedding_backward_workspace(n, H, V, C.byref(b)), "hap_embedding_backward_workspace")
    return b.value


def hap_embedding_backward_workspace(tokens, dw):
    """A workspace for the gradient of as many tokens and a weight of this size; needed during a call only."""
    _vector("tokens", tokens, torch.cuda.current_device(), torch.int64)
    V, H = dw.shape
    return torch.empty(max(256, _embedding_bytes(tokens.numel(), H, V)), dtype=torch.uint8, device=tokens.device)


@_on_stream
def hap_embedding_backward(tokens, dy, dw, first=0, scale=1.0, accumulate=False, workspace=None):
    """dw[v] = scale sum of dy[i] over the tokens[i] - first = v; added to what dw [V][H] holds with accumulate, else all of dw is
    written.  dw: of dy's type, or fp32."""
    here, stream = _now()
    pt = _vector("tokens", tokens, here, torch.int64)
    n = tokens.numel()
    pd, ldd = _matrix("dy", dy, here, _FLOATS, n)
    H = dy.shape[1]
    pw, ldw = _matrix("dw", dw, here, (dy.dtype, torch.float32), None, H)
    V = dw.shape[0]
    ps, b, workspace = _space("workspace", 0 if workspace is not None else max(256, _embedding_bytes(n, H, V)), workspace, here)
    _check(_lib().hap_embedding_backward(_TYPES[dy.dtype], _TYPES[dw.dtype], bool(accumulate), n, H, V, first, pt, pd, ldd, scale, pw, ldw, ps, b, stream), "hap_embedding_backward")
    return dw


def _params(x, here, H, named):
    """(parameters' type, their addresses): vectors of x's type or fp32, all of one type."""
    kind, at = x.dtype, []
    for name, t in named:
        if isinstance(t, torch.Tensor) and t.dtype == torch.float32:
            kind = torch.float32
    for name, t in named:
        at.append(_vector(name, t, here, kind, H) if t is not None else None)
    return kind, at


@_on_stream
def hap_layer_norm(x, w=None, b=None, eps=1e-5, centred=True, y=None, mean=None, rstd=None, keep=True):
    """(y, mean, rstd): y = (x - mean) rstd w + b over the rows of x; with centred false without the mean, which is None then.
    w, b: of x's type or fp32.  mean, rstd: fp32 [rows], for the backward pass (None where keep is false).  A mean that is given with
    centred false is not written."""
    here, stream = _now()
    px, ldx = _matrix("x", x, here, _FLOATS)
    rows, H = x.shape
    kind, (pw, pb) = _params(x, here, H, (("w", w), ("b", b)))
    if y is None:
        y = torch.empty((rows, H), dtype=x.dtype, device=x.device)
    py, ldy = _matrix("y", y, here, (x.dtype,), rows, H)
    if mean is None and keep and centred:
        mean = torch.empty(rows, dtype=torch.float32, device=x.device)
    if rstd is None and keep:
        rstd = torch.empty(rows, dtype=torch.float32, device=x.device)
    pm = _vector("mean", mean, here, torch.float32, rows) if mean is not None else None
    pr = _vector("rstd", rstd, here, torch.float32, rows) if rstd is not None else None
    _check(_lib().hap_layer_norm(_TYPES[x.dtype], _TYPES[kind], bool(centred), rows, H, px, ldx, pw, pb, eps, py, ldy, pm, pr, stream), "hap_layer_norm")
    return y, mean if centred else None, rstd


def _norm_bytes(rows, H):
    n = C.c_uint64()
    _check(_lib().hap_layer_norm_backward_workspace(rows, H, C.byref(n)), "hap_layer_norm_backward_workspace")
    return n.value


def hap_layer_norm_backward_workspace(x):
    """A workspace for the gradients of a norm of x; needed during a call only."""
    _matrix("x", x, torch.cuda.current_device(), _FLOATS)
    return torch.empty(max(256, _norm_bytes(*x.shape)), dtype=torch.uint8, device=x.device)


@_on_stream
def hap_layer_norm_backward(dy, x, w, rstd, mean=None, base=None, dx=None, dw=None, db=None, want_dx=True, want_dw=True, accumulate=False, workspace=None):
    """(dx, dw, db) of hap_layer_norm: centred where a mean is given.  base: added to dx.  dw and db are made, of w's type (fp32 without
    one), where want_dw is set; given ones are of w's type or fp32.  With accumulate they are added to, and none is made: those that
    are wanted have to be given (one alone: with want_dw false).  db is None without a mean."""
    here, stream = _now()
    px, ldx = _matrix("x", x, here, _FLOATS)
    rows, H = x.shape
    same = (x.dtype,)
    pd, ldd = _matrix("dy", dy, here, same, rows, H)
    kind, (pw,) = _params(x, here, H, (("w", w),))
    pr = _vector("rstd", rstd, here, torch.float32, rows)
    pm = _vector("mean", mean, here, torch.float32, rows) if mean is not None else None
    pb, ldb = _matrix("base", base, here, same, rows, H) if base is not None else (None, 0)
    if dx is None and want_dx:
        dx = torch.empty((rows, H), dtype=x.dtype, device=x.device)
    pdx, lddx = _matrix("dx", dx, here, same, rows, H) if dx is not None else (None, 0)
    given = dw if dw is not None else db
    grads = given.dtype if given is not None else kind if w is not None else torch.float32
    if accumulate and want_dw and (dw is None or (db is None and mean is not None)):
        _refuse("dw, db: needed where sums are added to them")
    if want_dw and not accumulate:
        dw = torch.empty(H, dtype=grads, device=x.device) if dw is None else dw
        db = torch.empty(H, dtype=grads, device=x.device) if db is None and mean is not None else db
    if grads not in (kind, torch.float32):
        _refuse(f"dw, db: {grads} where {kind} or torch.float32 is needed")
    at = [_vector(name, t, here, grads, H) if t is not None else None for name, t in (("dw", dw), ("db", db))]
    ps = n = None
    if dw is not None or db is not None:
        ps, n, workspace = _space("workspace", 0 if workspace is not None else max(256, _norm_bytes(rows, H)), workspace, here)
    _check(_lib().hap_layer_norm_backward(_TYPES[x.dtype], _TYPES[kind], _TYPES[grads], bool(accumulate), mean is not None, rows, H, pd, ldd, px, ldx, pw, pm, pr, pb, ldb, pdx, lddx,
                                          *at, ps, n or 0, stream), "hap_layer_norm_backward")
    return dx, dw, db


class _MeasuredTokens(C.Structure):
    _fields_ = [("tpre", C.c_void_p), ("tnorm", C.c_void_p), ("croute", C.c_double)]


def hap_measure_tokens_workspace(pb) -> int:
    """Bytes of device memory that hap_measure_tokens needs for a problem."""
    model, profile, keep = operators._measured_parts(pb)
    n = C.c_uint64()
    _check(_lib().hap_measure_tokens_workspace(model, profile, C.byref(n)), "hap_measure_tokens_workspace")
    return int(n.value)


@_on_stream
def hap_measure_tokens(pb, device_type, workspace=None):
    """Times embedding, norms and router on the current device and returns (problem, measured): a copy of the problem whose tpre and
    croute of one device type are these times, and what was measured as a dict; the norms' times (tnorm, forward and backward) are a
    part of tdf and tdb, which are not changed."""
    T = int(pb.P.shape[0])
    if not 0 <= device_type < T:
        _refuse(f"device_type: {device_type} of {T}")
    if workspace is None:
        workspace = torch.empty(hap_measure_tokens_workspace(pb), dtype=torch.uint8, device="cuda")
    here, stream = _now()
    ps = _vector("workspace", workspace, here, torch.uint8)
    n = tuple(len(x) for x in (pb.tp_list, pb.cp_list, pb.mb_list))
    tpre, tnorm = np.zeros(n), np.zeros((*n, 2))
    out = _MeasuredTokens(tpre.ctypes.data, tnorm.ctypes.data)
    model, profile, keep = operators._measured_parts(pb)
    _check(_lib().hap_measure_tokens(model, profile, C.byref(out), C.c_void_p(ps), C.c_uint64(workspace.numel()), C.c_void_p(stream)), "hap_measure_tokens")
    new = copy.copy(pb)
    for name in ("tpre", "croute"):
        setattr(new, name, np.array(getattr(pb, name), dtype=np.float64))
    new.tpre[device_type], new.croute[device_type] = tpre, out.croute
    return new, dict(tpre=tpre, tnorm=tnorm, croute=out.croute)
