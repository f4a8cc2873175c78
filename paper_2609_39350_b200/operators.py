"""Binding of the training operators: torch tensors in, same names as the C ABI, argument marshalling only.

Every function enqueues on `stream` (default: the current stream of the current device) and returns without waiting.  Tensors
live on the current device; rows may be a distance apart (a slice of a wider matrix), elements of a row are side by side.
"""
from __future__ import annotations

import ctypes as C
import functools

import torch

from .binding import HapError, load_library

EXPERT_FORWARD, EXPERT_GRAD_INPUT, EXPERT_GRAD_WEIGHT = 0, 1, 2
_TYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
_HALVES = (torch.bfloat16, torch.float16)


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


def _here(name, t, dtypes, dims):
    """Checks what every tensor argument has to be."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _refuse(f"{name}: must be a CUDA tensor")
    if t.device.index != torch.cuda.current_device():
        _refuse(f"{name}: must live on the current CUDA device")
    if t.dtype not in dtypes:
        _refuse(f"{name}: {t.dtype} where one of {[str(d) for d in dtypes]} is needed")
    if t.dim() != dims:
        _refuse(f"{name}: {t.dim()} dimensions where {dims} are needed")


def _matrix(name, t, dtypes, rows=None, cols=None, batch=None):
    """(address, distance of two rows) of a matrix, or of matrices that follow one another."""
    _here(name, t, dtypes, 2 if batch is None else 3)
    shape = tuple(t.shape)
    want = ((batch,) if batch is not None else ()) + (rows, cols)
    if any(w is not None and w != s for w, s in zip(want, shape)):
        _refuse(f"{name}: shape {shape} where {want} is needed")
    r, c = shape[-2:]
    if c > 1 and t.stride(-1) != 1:
        _refuse(f"{name}: elements of a row must lie side by side")
    ld = t.stride(-2) if r > 1 else -(-c // 8) * 8 if batch is None or shape[0] < 2 else t.stride(0)
    if ld < c or (batch is not None and shape[0] > 1 and t.stride(0) != r * ld):
        _refuse(f"{name}: rows overlap, or matrices do not follow one another")
    return C.c_void_p(t.data_ptr()), C.c_int64(ld)


def _vector(name, t, dtype, n=None):
    _here(name, t, (dtype,), 1)
    if n is not None and t.numel() != n:
        _refuse(f"{name}: {t.numel()} elements where {n} are needed")
    if t.numel() > 1 and t.stride(0) != 1:
        _refuse(f"{name}: elements must lie side by side")
    return C.c_void_p(t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _check(status, what):
    if status != 0:
        raise HapError(status, what)


def _offsets(offsets):
    at = _vector("offsets", offsets, torch.int64)
    if offsets.numel() < 2:
        _refuse("offsets: one more than there are experts are needed")
    return at, offsets.numel() - 1


@_on_stream
def hap_expert_matmul(a, b, offsets, form=EXPERT_FORWARD, out=None, out_dtype=None, accumulate=False):
    """Products of rows sorted by expert with their expert's matrix (offsets: int64 [E + 1] on the device).

    EXPERT_FORWARD      a [rows][K], b [E][N][K] -> out [rows][N] = a w_e^T
    EXPERT_GRAD_INPUT   a [rows][N], b [E][N][K] -> out [rows][K] = a w_e
    EXPERT_GRAD_WEIGHT  a [rows][N], b [rows][K] -> out [E][N][K] = sum over the expert's rows of a^T b

    Rows of `out` outside of every expert's are left as they are (unset in an output made here)."""
    at, E = _offsets(offsets)
    if form not in (EXPERT_FORWARD, EXPERT_GRAD_INPUT, EXPERT_GRAD_WEIGHT):
        _refuse("form")
    if not isinstance(a, torch.Tensor) or not isinstance(b, torch.Tensor) or a.dim() != 2:
        _refuse("a, b: matrices are needed")
    halves = (a.dtype,) if a.dtype in _HALVES else _HALVES
    rows = a.shape[0]
    if form == EXPERT_GRAD_WEIGHT:
        pa, lda = _matrix("a", a, halves)
        pb, ldb = _matrix("b", b, halves, rows=rows)
        N, K = a.shape[1], b.shape[1]
        shape = (E, N, K)
    else:
        pb, ldb = _matrix("b", b, halves, batch=E)
        N, K = b.shape[1:]
        pa, lda = _matrix("a", a, halves, cols=K if form == EXPERT_FORWARD else N)
        shape = (rows, N if form == EXPERT_FORWARD else K)
    if out is None:
        if accumulate:
            _refuse("out: needed where the product is added to it")
        out = torch.empty(shape, dtype=out_dtype or a.dtype, device=a.device)
    elif out_dtype is not None and out.dtype != out_dtype:
        _refuse("out: is not of out_dtype")
    po, ldo = _matrix("out", out, (a.dtype, torch.float32), *shape[-2:], batch=E if form == EXPERT_GRAD_WEIGHT else None)
    _check(load_library().hap_expert_matmul(C.c_int32(form), C.c_int32(_TYPES[a.dtype]), C.c_int32(_TYPES[out.dtype]), C.c_int32(bool(accumulate)), C.c_int32(E),
                                            C.c_int64(rows), C.c_int32(N), C.c_int32(K), at, pa, lda, pb, ldb, po, ldo, _stream()), "hap_expert_matmul")
    return out


@_on_stream
def hap_expert_gated(x, w, offsets, gu=None, h=None, keep=True):
    """(h, gu): [g | u] = x w_e^T with w [E][2F][H] and h = silu(g) u.  gu is None where keep is false."""
    at, E = _offsets(offsets)
    pw, ldw = _matrix("w", w, _HALVES, batch=E)
    F2, H = w.shape[1:]
    if F2 % 2:
        _refuse("w: the gate's rows and as many others are needed")
    px, ldx = _matrix("x", x, (w.dtype,), cols=H)
    rows, F = x.shape[0], F2 // 2
    if gu is None and keep:
        gu = torch.empty((rows, F2), dtype=x.dtype, device=x.device)
    if h is None:
        h = torch.empty((rows, F), dtype=x.dtype, device=x.device)
    pg, ldg = _matrix("gu", gu, (w.dtype,), rows, F2) if gu is not None else (C.c_void_p(0), C.c_int64(0))
    ph, ldh = _matrix("h", h, (w.dtype,), rows, F)
    _check(load_library().hap_expert_gated(C.c_int32(_TYPES[w.dtype]), C.c_int32(E), C.c_int64(rows), C.c_int32(H), C.c_int32(F), at, px, ldx, pw, ldw, pg, ldg,
                                           ph, ldh, _stream()), "hap_expert_gated")
    return h, gu


@_on_stream
def hap_expert_gated_backward(dy, w2, offsets, gu, dgu=None, h=None, want_h=True):
    """(dgu, h): dh = dy w2_e with w2 [E][H][F], the gradients of g and u from it and the kept gu, and h again.  dgu may be gu."""
    at, E = _offsets(offsets)
    pw, ldw = _matrix("w2", w2, _HALVES, batch=E)
    H, F = w2.shape[1:]
    py, ldy = _matrix("dy", dy, (w2.dtype,), cols=H)
    rows = dy.shape[0]
    pg, ldg = _matrix("gu", gu, (w2.dtype,), rows, 2 * F)
    if dgu is None:
        dgu = torch.empty((rows, 2 * F), dtype=dy.dtype, device=dy.device)
    if h is None and want_h:
        h = torch.empty((rows, F), dtype=dy.dtype, device=dy.device)
    pd, ldd = _matrix("dgu", dgu, (w2.dtype,), rows, 2 * F)
    ph, ldh = _matrix("h", h, (w2.dtype,), rows, F) if h is not None else (C.c_void_p(0), C.c_int64(0))
    _check(load_library().hap_expert_gated_backward(C.c_int32(_TYPES[w2.dtype]), C.c_int32(E), C.c_int64(rows), C.c_int32(H), C.c_int32(F), at, py, ldy, pw, ldw,
                                                    pg, ldg, pd, ldd, ph, ldh, _stream()), "hap_expert_gated_backward")
    return dgu, h


def hap_linear_cross_entropy_workspace(x, w):
    """A workspace for the forward and the backward pass of x [rows][H] and w [V][H]; needed during a call only."""
    _matrix("x", x, _HALVES)
    _matrix("w", w, (x.dtype,), cols=x.shape[1])
    n = C.c_uint64()
    _check(load_library().hap_linear_cross_entropy_workspace(C.c_int64(x.shape[0]), C.c_int32(x.shape[1]), C.c_int64(w.shape[0]), C.byref(n)), "hap_linear_cross_entropy_workspace")
    return torch.empty(max(256, n.value), dtype=torch.uint8, device=x.device)


def _loss_args(x, w, target, workspace):
    px, ldx = _matrix("x", x, _HALVES)
    pw, ldw = _matrix("w", w, (x.dtype,), cols=x.shape[1])
    pt = _vector("target", target, torch.int64, x.shape[0])
    if workspace is None:
        workspace = hap_linear_cross_entropy_workspace(x, w)
    ps = _vector("workspace", workspace, torch.uint8)
    head = (C.c_int32(_TYPES[x.dtype]), C.c_int64(x.shape[0]), C.c_int32(x.shape[1]), C.c_int64(w.shape[0]), px, ldx, pw, ldw, pt)
    return head, ps, C.c_uint64(workspace.numel()), workspace


@_on_stream
def hap_linear_cross_entropy(x, w, target, ignore_index=-100, loss=None, lse=None, workspace=None):
    """(loss, lse), fp32 [rows]: cross entropy of the logits x w^T against int64 targets, without keeping the logits."""
    head, ps, n, workspace = _loss_args(x, w, target, workspace)
    loss = torch.empty(x.shape[0], device=x.device) if loss is None else loss
    lse = torch.empty(x.shape[0], device=x.device) if lse is None else lse
    pl, pe = _vector("loss", loss, torch.float32, x.shape[0]), _vector("lse", lse, torch.float32, x.shape[0])
    _check(load_library().hap_linear_cross_entropy(*head, C.c_int64(ignore_index), pl, pe, ps, n, _stream()), "hap_linear_cross_entropy")
    return loss, lse


@_on_stream
def hap_linear_cross_entropy_backward(x, w, target, lse, grad, ignore_index=-100, dx=None, dw=None, want_dx=True, want_dw=True, workspace=None):
    """(dx, dw): gradients of grad * sum(loss); grad: fp32 scalar on the device."""
    head, ps, n, workspace = _loss_args(x, w, target, workspace)
    pe = _vector("lse", lse, torch.float32, x.shape[0])
    if not isinstance(grad, torch.Tensor) or grad.numel() != 1:
        _refuse("grad: one fp32 value on the device is needed")
    pg = _vector("grad", grad.reshape(1), torch.float32)
    none = C.c_void_p(0), C.c_int64(0)
    if dx is None and want_dx:
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    if dw is None and want_dw:
        dw = torch.empty(w.shape, dtype=w.dtype, device=w.device)
    pdx = _matrix("dx", dx, (x.dtype,), *x.shape) if dx is not None else none
    pdw = _matrix("dw", dw, (x.dtype,), *w.shape) if dw is not None else none
    _check(load_library().hap_linear_cross_entropy_backward(*head, C.c_int64(ignore_index), pe, pg, *pdx, *pdw, ps, n, _stream()), "hap_linear_cross_entropy_backward")
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
        self.kept = [params, *[x for _, x in lists if x is not None]]
        self.device = params[0].device
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
                _here(name, t, types[name][:1] if len(types[name]) == 1 else (tensors[0].dtype,), t.dim() if isinstance(t, torch.Tensor) else 0)
                if t.dtype not in types[name]:
                    _refuse(f"{name}: {t.dtype}")
                if not t.is_contiguous():
                    _refuse(f"{name}: tensors must be contiguous")
                if t.numel() != (-(-p.numel() // 256) if name.endswith("scale") else p.numel()):
                    _refuse(f"{name}: of another size than its parameter asks for")
            at[name] = [t.data_ptr() for t in tensors]
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
    addresses, and the tensors: make it again when a gradient is another tensor."""
    return HapAdamWTensors(params, grads, m, v, m_scale, v_scale, copies)


@_on_stream
def hap_adamw_step(tensors: HapAdamWTensors, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, grad_scale=None):
    """One step over all tensors; step counts from 1.  grad_scale: fp32 scalar on the device (loss scaling, clipping)."""
    if tensors.device.index != torch.cuda.current_device():
        _refuse("tensors: must live on the current CUDA device")
    pg = C.c_void_p(0)
    if grad_scale is not None:
        if not isinstance(grad_scale, torch.Tensor) or grad_scale.numel() != 1:
            _refuse("grad_scale: one fp32 value on the device is needed")
        pg = _vector("grad_scale", grad_scale.reshape(1), torch.float32)
    options = _AdamWOptions(lr, beta1, beta2, eps, weight_decay, step)
    _check(load_library().hap_adamw_step(tensors.array, C.c_int32(len(tensors.array)), *(C.c_int32(t) for t in tensors.types), C.c_int32(tensors.bits),
                                         C.byref(options), pg, _stream()), "hap_adamw_step")


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
    _check(load_library().hap_adamw_state(tensors.array, C.c_int32(len(tensors)), got[0][1], got[1][1], _stream()), "hap_adamw_state")
    return got[0][0], got[1][0]


def hap_operator_status() -> int:
    """0, or the bits of waits that ran out in an operator's kernel since the last call (waits for the current device)."""
    bits = C.c_uint32()
    _check(load_library().hap_operator_status(C.byref(bits)), "hap_operator_status")
    return int(bits.value)
