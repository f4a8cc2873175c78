"""Binding of the training operators: torch tensors in, same names as the C ABI, argument marshalling only.

Every function enqueues on `stream` (default: the current stream of the current device) and returns without waiting.  Tensors
live on the current device; rows may be a distance apart (a slice of a wider matrix), elements of a row are side by side.

The functions read and write memory and record nothing: an output does not require a gradient even where an input does.  The
gradients are functions of their own here, to be called from the backward of whatever the caller differentiates.  A kernel whose
wait ran out ends early with its outputs unfinished, which only hap_operator_status tells, since it has to wait for the device.
"""
from __future__ import annotations

import copy
import ctypes as C
import functools

import numpy as np
import torch

from . import binding
from .binding import HapError, load_library

EXPERT_FORWARD, EXPERT_GRAD_INPUT, EXPERT_GRAD_WEIGHT = 0, 1, 2
_TYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
_HALVES = (torch.bfloat16, torch.float16)
_MOST = (1 << 31) - 1           # values of a row: row lengths are passed in 32 bits


class _AdamWTensor(C.Structure):
    _fields_ = [*[(n, C.c_void_p) for n in ("param", "grad", "m", "v", "m_scale", "v_scale", "copy")], ("count", C.c_uint64)]


class _AdamWOptions(C.Structure):
    _fields_ = [*[(n, C.c_double) for n in ("lr", "beta1", "beta2", "eps", "weight_decay")], ("step", C.c_int64)]


def _on_stream(call):
    """With `stream` given the whole call is made there: what it allocates belongs to that stream too."""
    @functools.wraps(call)
    def on_stream(*args, stream=None, **more):
        if stream is None:
            return call(*args, **more)
        with torch.cuda.stream(stream):
            return call(*args, **more)
    return on_stream


def _refuse(what: str):
    raise HapError(1, what)


def _lib():
    """The library with the operators' argument types set: plain numbers and addresses are passed."""
    global _typed
    if _typed is None:
        L = load_library()
        i, l, u, p = C.c_int32, C.c_int64, C.c_uint64, C.c_void_p
        L.hap_expert_matmul.argtypes = [i] * 5 + [l, i, i, p, p, l, p, l, p, l, p]
        L.hap_expert_gated.argtypes = [i, i, l, i, i, p, p, l, p, l, p, l, p, l, p]
        L.hap_expert_gated_backward.argtypes = [i, i, l, i, i, p, p, l, p, l, p, l, p, l, p, l, p]
        L.hap_linear_cross_entropy_workspace.argtypes = [l, i, l, p]
        L.hap_linear_cross_entropy.argtypes = [i, l, i, l, p, l, p, l, p, l, p, p, p, u, p]
        L.hap_linear_cross_entropy_backward.argtypes = [i, l, i, l, p, l, p, l, p, l, p, p, p, l, p, l, p, u, p]
        L.hap_adamw_step.argtypes = [p, i, i, i, i, i, p, p, p]
        L.hap_adamw_state.argtypes = [p, i, p, p, p]
        L.hap_operator_status.argtypes = [p]
        _typed = L
    return _typed


_typed = None


def _here(name, t, here, dtypes, dims):
    """Checks what every tensor argument has to be."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _refuse(f"{name}: must be a CUDA tensor")
    if t.layout != torch.strided:
        _refuse(f"{name}: must be a strided tensor")
    if t.get_device() != here:
        _refuse(f"{name}: must live on the current CUDA device")
    if t.dtype not in dtypes:
        _refuse(f"{name}: {t.dtype} where one of {[str(d) for d in dtypes]} is needed")
    if t.dim() != dims:
        _refuse(f"{name}: {t.dim()} dimensions where {dims} are needed")


def _matrix(name, t, here, dtypes, rows=None, cols=None):
    """(address, distance of two rows) of a matrix."""
    try:                                            # what is usual, asked for in as few steps as there are; the rest below
        (r, c), (ld, one) = t.shape, t.stride()
        if t.get_device() == here and t.dtype in dtypes and one == 1 and r > 0 and (rows is None or r == rows) and (cols is None or c == cols):
            if r == 1 and c <= _MOST:
                return t.data_ptr(), (c + 7) & ~7
            if _MOST >= c <= ld:
                return t.data_ptr(), ld
    except (AttributeError, TypeError, ValueError, RuntimeError):
        pass
    _here(name, t, here, dtypes, 2)
    (r, c), (ld, one) = t.shape, t.stride()
    if (rows is not None and r != rows) or (cols is not None and c != cols):
        _refuse(f"{name}: shape {tuple(t.shape)} where {(rows, cols)} is needed")
    if c > _MOST:
        _refuse(f"{name}: rows of {c} values")
    if one != 1 and c > 1:
        _refuse(f"{name}: elements of a row must lie side by side")
    if r < 2:
        ld = (c + 7) & ~7
    if ld < c:
        _refuse(f"{name}: rows overlap")
    return t.data_ptr(), ld


def _matrices(name, t, here, dtypes, batch, rows=None, cols=None):
    """The same of matrices that follow one another."""
    _here(name, t, here, dtypes, 3)
    (n, r, c), (far, ld, one) = t.shape, t.stride()
    if n != batch or (rows is not None and r != rows) or (cols is not None and c != cols):
        _refuse(f"{name}: shape {tuple(t.shape)} where {(batch, rows, cols)} is needed")
    if max(r, c) > _MOST:
        _refuse(f"{name}: matrices of {r} rows of {c} values")
    if one != 1 and c > 1:
        _refuse(f"{name}: elements of a row must lie side by side")
    if r < 2:
        ld = (c + 7) & ~7 if n < 2 else far
    if ld < c or (n > 1 and far != r * ld):
        _refuse(f"{name}: rows overlap, or matrices do not follow one another")
    return t.data_ptr(), ld


def _vector(name, t, here, dtype, n=None):
    try:
        (m,), (one,) = t.shape, t.stride()
        if t.get_device() == here and t.dtype == dtype and one == 1 and (n is None or m == n):
            return t.data_ptr()
    except (AttributeError, TypeError, ValueError, RuntimeError):
        pass
    _here(name, t, here, (dtype,), 1)
    if n is not None and t.numel() != n:
        _refuse(f"{name}: {t.numel()} elements where {n} are needed")
    if t.stride(0) != 1 and t.numel() > 1:
        _refuse(f"{name}: elements must lie side by side")
    return t.data_ptr()


def _check(status, what):
    if status != 0:
        raise HapError(status, what)


def _now():
    """(current device, address of its current stream)"""
    here = torch.cuda.current_device()
    return here, torch._C._cuda_getCurrentRawStream(here)           # (the address alone: a microsecond less than a Stream object)


def _offsets(offsets, here):
    at = _vector("offsets", offsets, here, torch.int64)
    if offsets.numel() < 2:
        _refuse("offsets: one more than there are experts are needed")
    if offsets.numel() > _MOST:
        _refuse(f"offsets: of {offsets.numel() - 1} experts")
    return at, offsets.numel() - 1


@_on_stream
def hap_expert_matmul(a, b, offsets, form=EXPERT_FORWARD, out=None, out_dtype=None, accumulate=False):
    """Products of rows sorted by expert with their expert's matrix (offsets: int64 [E + 1] on the device).

    EXPERT_FORWARD      a [rows][K], b [E][N][K] -> out [rows][N] = a w_e^T
    EXPERT_GRAD_INPUT   a [rows][N], b [E][N][K] -> out [rows][K] = a w_e
    EXPERT_GRAD_WEIGHT  a [rows][N], b [rows][K] -> out [E][N][K] = sum over the expert's rows of a^T b

    Rows of `out` outside of every expert's are left as they are (unset in an output made here)."""
    here, stream = _now()
    at, E = _offsets(offsets, here)
    if form not in (EXPERT_FORWARD, EXPERT_GRAD_INPUT, EXPERT_GRAD_WEIGHT):
        _refuse("form")
    if not isinstance(a, torch.Tensor) or not isinstance(b, torch.Tensor) or a.dim() != 2:
        _refuse("a, b: matrices are needed")
    halves = (a.dtype,) if a.dtype in _HALVES else _HALVES
    rows = a.shape[0]
    if form == EXPERT_GRAD_WEIGHT:
        pa, lda = _matrix("a", a, here, halves)
        pb, ldb = _matrix("b", b, here, halves, rows)
        N, K = a.shape[1], b.shape[1]
        shape = (E, N, K)
    else:
        pb, ldb = _matrices("b", b, here, halves, E)
        N, K = b.shape[1:]
        pa, lda = _matrix("a", a, here, halves, None, K if form == EXPERT_FORWARD else N)
        shape = (rows, N if form == EXPERT_FORWARD else K)
    if out is None:
        if accumulate:
            _refuse("out: needed where the product is added to it")
        out = torch.empty(shape, dtype=out_dtype or a.dtype, device=a.device)
    elif out_dtype is not None and out.dtype != out_dtype:
        _refuse("out: is not of out_dtype")
    kinds = (a.dtype, torch.float32)
    po, ldo = _matrices("out", out, here, kinds, *shape) if form == EXPERT_GRAD_WEIGHT else _matrix("out", out, here, kinds, *shape)
    _check(_lib().hap_expert_matmul(form, _TYPES[a.dtype], _TYPES[out.dtype], bool(accumulate), E, rows, N, K, at, pa, lda, pb, ldb, po, ldo, stream), "hap_expert_matmul")
    return out


@_on_stream
def hap_expert_gated(x, w, offsets, gu=None, h=None, keep=True):
    """(h, gu): [g | u] = x w_e^T with w [E][2F][H] and h = silu(g) u.  gu is None where keep is false."""
    here, stream = _now()
    at, E = _offsets(offsets, here)
    pw, ldw = _matrices("w", w, here, _HALVES, E)
    F2, H = w.shape[1:]
    if F2 % 2:
        _refuse("w: the gate's rows and as many others are needed")
    kind = (w.dtype,)
    px, ldx = _matrix("x", x, here, kind, None, H)
    rows, F = x.shape[0], F2 // 2
    if gu is None and keep:
        gu = torch.empty((rows, F2), dtype=x.dtype, device=x.device)
    if h is None:
        h = torch.empty((rows, F), dtype=x.dtype, device=x.device)
    pg, ldg = _matrix("gu", gu, here, kind, rows, F2) if gu is not None else (None, 0)
    ph, ldh = _matrix("h", h, here, kind, rows, F)
    _check(_lib().hap_expert_gated(_TYPES[w.dtype], E, rows, H, F, at, px, ldx, pw, ldw, pg, ldg, ph, ldh, stream), "hap_expert_gated")
    return h, gu


@_on_stream
def hap_expert_gated_backward(dy, w2, offsets, gu, dgu=None, h=None, want_h=True):
    """(dgu, h): dh = dy w2_e with w2 [E][H][F], the gradients of g and u from it and the kept gu, and h again.  dgu may be gu."""
    here, stream = _now()
    at, E = _offsets(offsets, here)
    pw, ldw = _matrices("w2", w2, here, _HALVES, E)
    H, F = w2.shape[1:]
    kind = (w2.dtype,)
    py, ldy = _matrix("dy", dy, here, kind, None, H)
    rows = dy.shape[0]
    pg, ldg = _matrix("gu", gu, here, kind, rows, 2 * F)
    if dgu is None:
        dgu = torch.empty((rows, 2 * F), dtype=dy.dtype, device=dy.device)
    if h is None and want_h:
        h = torch.empty((rows, F), dtype=dy.dtype, device=dy.device)
    pd, ldd = _matrix("dgu", dgu, here, kind, rows, 2 * F)
    ph, ldh = _matrix("h", h, here, kind, rows, F) if h is not None else (None, 0)
    _check(_lib().hap_expert_gated_backward(_TYPES[w2.dtype], E, rows, H, F, at, py, ldy, pw, ldw, pg, ldg, pd, ldd, ph, ldh, stream), "hap_expert_gated_backward")
    return dgu, h


def hap_linear_cross_entropy_workspace(x, w):
    """A workspace for the forward and the backward pass of x [rows][H] and w [V][H]; needed during a call only."""
    here = torch.cuda.current_device()
    _matrix("x", x, here, _HALVES)
    _matrix("w", w, here, (x.dtype,), None, x.shape[1])
    n = C.c_uint64()
    _check(_lib().hap_linear_cross_entropy_workspace(x.shape[0], x.shape[1], w.shape[0], C.byref(n)), "hap_linear_cross_entropy_workspace")
    return torch.empty(max(256, n.value), dtype=torch.uint8, device=x.device)


def _loss_args(x, w, target, workspace, here):
    px, ldx = _matrix("x", x, here, _HALVES)
    pw, ldw = _matrix("w", w, here, (x.dtype,), None, x.shape[1])
    pt = _vector("target", target, here, torch.int64, x.shape[0])
    if workspace is None:
        workspace = hap_linear_cross_entropy_workspace(x, w)
    ps = _vector("workspace", workspace, here, torch.uint8)
    return (_TYPES[x.dtype], x.shape[0], x.shape[1], w.shape[0], px, ldx, pw, ldw, pt), ps, workspace


@_on_stream
def hap_linear_cross_entropy(x, w, target, ignore_index=-100, loss=None, lse=None, workspace=None):
    """(loss, lse), fp32 [rows]: cross entropy of the logits x w^T against int64 targets, without keeping the logits."""
    here, stream = _now()
    head, ps, workspace = _loss_args(x, w, target, workspace, here)
    rows = x.shape[0]
    loss = torch.empty(rows, device=x.device) if loss is None else loss
    lse = torch.empty(rows, device=x.device) if lse is None else lse
    pl, pe = _vector("loss", loss, here, torch.float32, rows), _vector("lse", lse, here, torch.float32, rows)
    _check(_lib().hap_linear_cross_entropy(*head, ignore_index, pl, pe, ps, workspace.numel(), stream), "hap_linear_cross_entropy")
    return loss, lse


@_on_stream
def hap_linear_cross_entropy_backward(x, w, target, lse, grad, ignore_index=-100, dx=None, dw=None, want_dx=True, want_dw=True, workspace=None):
    """(dx, dw): gradients of grad * sum(loss); grad: fp32 scalar on the device."""
    here, stream = _now()
    head, ps, workspace = _loss_args(x, w, target, workspace, here)
    pe = _vector("lse", lse, here, torch.float32, x.shape[0])
    if not isinstance(grad, torch.Tensor) or grad.numel() != 1:
        _refuse("grad: one fp32 value on the device is needed")
    pg = _vector("grad", grad.reshape(1), here, torch.float32)
    if dx is None and want_dx:
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    if dw is None and want_dw:
        dw = torch.empty(w.shape, dtype=w.dtype, device=w.device)
    pdx = _matrix("dx", dx, here, (x.dtype,), *x.shape) if dx is not None else (None, 0)
    pdw = _matrix("dw", dw, here, (x.dtype,), *w.shape) if dw is not None else (None, 0)
    _check(_lib().hap_linear_cross_entropy_backward(*head, ignore_index, pe, pg, *pdx, *pdw, ps, workspace.numel(), stream), "hap_linear_cross_entropy_backward")
    return dx, dw


class HapAdamWTensors:
    """The descriptors of an optimizer's tensors, and the tensors they point to."""

    def __init__(self, params, grads, m, v, m_scale=None, v_scale=None, copies=None):
        n = len(params)
        lists = [("grads", grads), ("m", m), ("v", v), ("m_scale", m_scale), ("v_scale", v_scale), ("copies", copies)]
        if n < 1:
            _refuse("params: empty")
        if any(x is not None and len(x) != n for _, x in lists):
            _refuse("lists of different lengths")
        if (m_scale is None) != (v_scale is None):
            _refuse("m_scale, v_scale: both or neither")
        self.bits = 32 if m_scale is None else 8
        self.kept = [list(params), *[list(x) for _, x in lists if x is not None]]
        self.device = params[0].device
        here = torch.cuda.current_device()
        types = dict(params=(torch.float32, *_HALVES), grads=(torch.float32, *_HALVES), copies=_HALVES,
                     m=(torch.float32,) if self.bits == 32 else (torch.int8,), v=(torch.float32,) if self.bits == 32 else (torch.uint8,),
                     m_scale=(torch.float32,), v_scale=(torch.float32,))
        self.array = (_AdamWTensor * n)()
        at = {}
        for name, tensors in [("params", params), *lists]:
            if tensors is None:
                at[name] = [0] * n
                continue
            for p, t in zip(params, tensors):
                _here(name, t, here, types[name][:1] if len(types[name]) == 1 else (tensors[0].dtype,), t.dim() if isinstance(t, torch.Tensor) else 0)
                if t.dtype not in types[name]:
                    _refuse(f"{name}: {t.dtype}")
                if not t.is_contiguous():
                    _refuse(f"{name}: tensors must be contiguous")
                if t.numel() != (-(-p.numel() // 256) if name.endswith("scale") else p.numel()):
                    _refuse(f"{name}: of another size than its parameter asks for")
            at[name] = [t.data_ptr() for t in tensors]
            if name != "grads":                         # (weights that are tied are one tensor; two steps at once on it would race)
                used = [a for a, t in zip(at[name], tensors) if t.numel()]
                if len(set(used)) != len(used):
                    _refuse(f"{name}: the same tensor twice")
        for i, p in enumerate(params):
            d = self.array[i]
            d.param, d.grad, d.m, d.v, d.m_scale, d.v_scale, d.copy = (at[k][i] for k in ("params", "grads", "m", "v", "m_scale", "v_scale", "copies"))
            d.count = p.numel()
        self.types = (_TYPES[params[0].dtype], _TYPES[grads[0].dtype], _TYPES[copies[0].dtype] if copies is not None else 0)
        if self.types[1] != self.types[0] and 2 not in self.types[:2]:
            _refuse("grads: of the parameters' type or in fp32")

    def __len__(self):
        return len(self.array)


def hap_adamw_tensors(params, grads, m, v, m_scale=None, v_scale=None, copies=None) -> HapAdamWTensors:
    """Descriptors for hap_adamw_step: contiguous tensors, one gradient and two states each; states are fp32, or int8 and uint8
    with fp32 scales of ceil(n / 256) values.  copies: 16-bit tensors that get fp32 parameters rounded.  The object holds the
    addresses, and the tensors: make it again when a gradient is another tensor (6 us a parameter).  Only gradients may be listed twice."""
    return HapAdamWTensors(params, grads, m, v, m_scale, v_scale, copies)


@_on_stream
def hap_adamw_step(tensors: HapAdamWTensors, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, grad_scale=None):
    """One step over all tensors; step counts from 1.  grad_scale: fp32 scalar on the device (loss scaling, clipping)."""
    if tensors.device.index != torch.cuda.current_device():
        _refuse("tensors: must live on the current CUDA device")
    here, stream = _now()
    pg = None
    if grad_scale is not None:
        if not isinstance(grad_scale, torch.Tensor) or grad_scale.numel() != 1:
            _refuse("grad_scale: one fp32 value on the device is needed")
        pg = _vector("grad_scale", grad_scale.reshape(1), here, torch.float32)
    options = _AdamWOptions(lr, beta1, beta2, eps, weight_decay, step)
    _check(_lib().hap_adamw_step(tensors.array, len(tensors.array), *tensors.types, tensors.bits, C.byref(options), pg, stream), "hap_adamw_step")


@_on_stream
def hap_adamw_state(tensors: HapAdamWTensors, m=None, v=None):
    """(m, v): lists of fp32 tensors with the values that 8-bit states stand for."""
    if tensors.bits != 8:
        _refuse("tensors: states are in 32 bits")
    if tensors.device.index != torch.cuda.current_device():
        _refuse("tensors: must live on the current CUDA device")
    got = []
    for name, values in (("m", m), ("v", v)):
        if values is None:
            values = [torch.empty(p.shape, device=p.device) for p in tensors.kept[0]]
        if len(values) != len(tensors):
            _refuse(f"{name}: lists of different lengths")
        for t, d in zip(values, tensors.array):
            if t.numel() != d.count or t.dtype != torch.float32 or not t.is_contiguous() or t.device != tensors.device:
                _refuse(f"{name}: contiguous fp32 tensors of the parameters' sizes are needed")
        got.append((values, (C.c_void_p * len(values))(*[t.data_ptr() for t in values])))
    _check(_lib().hap_adamw_state(tensors.array, len(tensors), got[0][1], got[1][1], _now()[1]), "hap_adamw_state")
    return got[0][0], got[1][0]


def hap_operator_status() -> int:
    """0, or the bits of waits that ran out in an operator's kernel since the last call (waits for the current device)."""
    bits = C.c_uint32()
    _check(_lib().hap_operator_status(C.byref(bits)), "hap_operator_status")
    return int(bits.value)


class _Measured(C.Structure):
    _fields_ = [*[(n, C.c_void_p) for n in ("tff", "tfb", "tpost")], *[(n, C.c_double) for n in ("eta", "gamma", "copt")]]


def _measured_parts(pb):
    descriptors, keep = binding._descriptors(pb, 0, 0)
    return C.byref(descriptors, binding._OFFSETS[0]), C.byref(descriptors, binding._OFFSETS[2]), (descriptors, keep)


def hap_measure_workspace(pb) -> int:
    """Bytes of device memory that hap_measure_profile needs for a problem."""
    model, profile, keep = _measured_parts(pb)
    n = C.c_uint64()
    _check(_lib().hap_measure_workspace(model, profile, C.byref(n)), "hap_measure_workspace")
    return int(n.value)


@_on_stream
def hap_measure_profile(pb, device_type, workspace=None):
    """Times the training operators on the current device and returns (problem, measured): a copy of the problem whose entries of
    one device type are these times, and what was measured as a dict.  Replaced: tff, tfb, tpost, eta and copt of the type; tdf
    and tdb keep their difference to tff and tfb (attention and the rest of a layer, which are not measured).  gamma, which all
    types share, is in the dict only."""
    T = int(pb.P.shape[0])
    if not 0 <= device_type < T:
        _refuse(f"device_type: {device_type} of {T}")
    if workspace is None:
        workspace = torch.empty(hap_measure_workspace(pb), dtype=torch.uint8, device="cuda")
    here, stream = _now()
    ps = _vector("workspace", workspace, here, torch.uint8)
    n = tuple(len(x) for x in (pb.tp_list, pb.cp_list, pb.mb_list))
    tff, tfb, tpost = np.zeros((*n, 2)), np.zeros((*n, 2)), np.zeros(n)
    out = _Measured(tff.ctypes.data, tfb.ctypes.data, tpost.ctypes.data)
    model, profile, keep = _measured_parts(pb)
    _check(_lib().hap_measure_profile(model, profile, C.byref(out), C.c_void_p(ps), C.c_uint64(workspace.numel()), C.c_void_p(stream)), "hap_measure_profile")
    new = copy.copy(pb)
    for name in ("tdf", "tdb", "tff", "tfb", "tpost", "eta", "copt"):
        setattr(new, name, np.array(getattr(pb, name), dtype=np.float64))
    kind = np.asarray(pb.kind)
    for total, part, times in ((new.tdf, new.tff, tff), (new.tdb, new.tfb, tfb)):
        measured = times[..., kind]                     # [ntp][ncp][nmb][N]
        total[device_type] = np.maximum(total[device_type] - part[device_type], 0.0) + measured
        part[device_type] = measured
    new.tpost[device_type], new.eta[device_type], new.copt[device_type] = tpost, out.eta, out.copt
    return new, dict(tff=tff, tfb=tfb, tpost=tpost, eta=out.eta, gamma=out.gamma, copt=out.copt)
