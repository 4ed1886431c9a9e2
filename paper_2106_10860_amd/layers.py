"""What stands around exact layers and layers of experts: binding of the calls that ``include/maddness.h`` describes under that heading.
Argument marshalling only, as in the package's other calls; no CPU fallback.

A matrix in 8-bit integers is an ``IntegerMatrix``: values and one fp32 scale for each row.  A layer of weight [outputs, inputs], as it is served,
behind its norm:

    W = maddness_quantise_rows(weight)
    y = maddness_integer_product(maddness_layer_norm(x, norm_weight, norm_bias, integer=True), W, bias=b)

A training step of a layer of experts (``ExpertLayer`` makes the balance's calls by itself):

    h, mean, rstd = maddness_layer_norm(x, norm_weight, norm_bias, training=True)
    ...                                                        # the layer on h, back to the gradient dh of h
    dx, dnorm_weight, dnorm_bias = maddness_layer_norm_gradient(dh, x, mean, rstd, norm_weight)
    norm = maddness_clip_gradients([dW, dgate, dnorm_weight, dnorm_bias], 1.0)

The calls are no part of torch's autograd: an operand that requires a gradient is refused while gradients are recorded.
"""
from __future__ import annotations

import ctypes as C

import paper_2106_10860_amd as _m

from .blocks import _code, _flat, _float_code, _no_gradient, _on, _same_device, _scores, _up

MADDNESS_I8 = 17


def _here(t) -> None:
    """The kernels go to the current device's stream: that has to be the tensors' device."""
    torch = _m._torch or _m._torch_module()
    if t.device.index != torch.cuda.current_device():
        raise ValueError(f"tensors are on {t.device}, the current device is cuda:{torch.cuda.current_device()}")


class IntegerMatrix:
    """8-bit integers ``q`` [rows, cols] of dtype int8 with unit column stride, rows 16-byte aligned, and their ``scale`` fp32 [rows]:
    row r stands for q[r] * scale[r].  Both may be replaced; every call checks what it finds."""

    __slots__ = ("q", "scale")

    def __init__(self, q, scale):
        self.q, self.scale = q, scale
        self._check()

    def _check(self) -> None:
        torch, q, scale = _m._torch or _m._torch_module(), self.q, self.scale
        if not isinstance(q, torch.Tensor) or not isinstance(scale, torch.Tensor) or not q.is_cuda or not scale.is_cuda:
            raise TypeError("q and scale must be device tensors")
        if q.dtype is not torch.int8 or scale.dtype is not torch.float32:
            raise TypeError(f"q must have dtype int8 and scale float32, have {q.dtype} and {scale.dtype}")
        if q.dim() != 2 or tuple(scale.shape) != (q.shape[0],):
            raise ValueError(f"q must be 2-D and scale [rows], have {tuple(q.shape)} and {tuple(scale.shape)}")
        _same_device(q, scale)
        if q.shape[1] > 1 and q.stride(1) != 1:
            raise ValueError("q must have unit column stride")
        if not scale.is_contiguous():
            raise ValueError("scale must be contiguous")
        _no_gradient(scale, "scale")

    @classmethod
    def _made(cls, q, scale) -> "IntegerMatrix":
        """Of tensors that this package made."""
        b = cls.__new__(cls)
        b.q, b.scale = q, scale
        return b

    @classmethod
    def empty(cls, rows: int, cols: int, device="cuda") -> "IntegerMatrix":
        torch = _m._torch or _m._torch_module()
        return cls._made(torch.empty((rows, _up(cols, 16)), dtype=torch.int8, device=device)[:, :cols],
                         torch.empty(rows, dtype=torch.float32, device=device))

    @property
    def shape(self):
        return tuple(self.q.shape)

    @property
    def device(self):
        return self.q.device

    @property
    def _struct(self):
        self._check()
        rows, cols = self.q.shape
        ld = self.q.stride(0) if rows > 1 else _up(max(cols, self.q.stride(0)), 16)
        return _m._IntegerMatrix(self.q.data_ptr(), MADDNESS_I8, rows, cols, ld, self.scale.data_ptr())

    def values(self):
        """What the matrix stands for, in fp32 (elementary torch operations; for checks)."""
        return self.q.float() * self.scale.unsqueeze(1)


def maddness_quantise_rows(x, stream=None) -> IntegerMatrix:
    """x (float, [rows, cols] with unit column stride) as an IntegerMatrix: every row over its largest magnitude / 127, to the nearest
    integer.  A row with a NaN or an infinity has the scale NaN."""
    if stream is not None:
        with _on(stream):
            return maddness_quantise_rows(x)
    r = _m._native.quantise_rows(x)
    if r is not NotImplemented:
        return IntegerMatrix._made(*_m._done(r))
    code = _code(x, "x")
    _here(x)
    rows, cols, ldx = _m._rows(x, "x")
    out = IntegerMatrix.empty(rows, cols, x.device)
    s = out._struct
    _m._check(_m.lib().maddness_quantise_rows(x.data_ptr(), code, rows, cols, ldx, s.data, s.ld, s.scale, _m._stream(None)))
    return out


def maddness_integer_product(A, B: IntegerMatrix, bias=None, out_dtype=None, out=None, workspace=None, stream=None):
    """A @ B.T + bias in ``out_dtype`` (bfloat16).  A: an IntegerMatrix or a float tensor [M, K], whose rows are then rounded within the call;
    B: an IntegerMatrix [N, K]; bias: fp32 [N].  Sums are exact, the scales and the bias come in as fp32."""
    if not isinstance(B, IntegerMatrix):
        raise TypeError("B must be an IntegerMatrix")
    if stream is not None:
        with _on(stream):
            return maddness_integer_product(A, B, bias, out_dtype, out, workspace)
    r = _m._native.integer_product(isinstance(A, IntegerMatrix), A, B, bias, out_dtype, out, workspace)
    if r is not NotImplemented:
        return _m._done(r)
    torch = _m._torch or _m._torch_module()
    b = B._struct
    if isinstance(A, IntegerMatrix):
        a, (M, K), device = A._struct, A.shape, A.device
    else:
        code = _code(A, "A")
        M, K, lda = _m._rows(A, "A")
        a, device = _m._IntegerMatrix(A.data_ptr(), code, M, K, lda, None), A.device
    N = B.shape[0]
    bias_p = _flat(bias, torch.float32, (N,), "bias")
    if out is None:
        out = torch.empty((M, N), dtype=out_dtype or torch.bfloat16, device=device)
    elif tuple(out.shape) != (M, N) or (out_dtype is not None and out.dtype is not out_dtype):
        raise ValueError(f"out must have shape {(M, N)}{'' if out_dtype is None else f' and dtype {out_dtype}'}")
    _same_device(A.q if isinstance(A, IntegerMatrix) else A, B.q, bias, out, workspace)
    out_code = _code(out, "out")
    _here(out)
    L = _m.lib()
    need = L.maddness_integer_product_workspace(M, K, a.dtype)
    if workspace is None and need:
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
    if workspace is not None and not workspace.is_contiguous():              # (its size in bytes is then not what it has room for)
        raise ValueError("workspace must be contiguous")
    _m._check(L.maddness_integer_product(C.byref(a), C.byref(b), bias_p, out.data_ptr(), out_code, _m._rows(out, "out")[2],
                                         _m._ptr(workspace, torch.uint8, "workspace"), 0 if workspace is None else workspace.numel(),
                                         _m._stream(None)))
    return out


def _parameters(weight, bias, cols: int):
    """(pointers of weight and bias, their type)."""
    torch = _m._torch or _m._torch_module()
    dtypes = {t.dtype for t in (weight, bias) if t is not None}
    if len(dtypes) > 1:
        raise TypeError(f"weight and bias must have one dtype, have {weight.dtype} and {bias.dtype}")
    dtype = dtypes.pop() if dtypes else torch.float32
    return _flat(weight, dtype, (cols,), "weight"), _flat(bias, dtype, (cols,), "bias"), _float_code(dtype, "weight")


def maddness_layer_norm(x, weight=None, bias=None, eps: float = 1e-5, training: bool = False, integer: bool = False, out_dtype=None, out=None,
                        stream=None):
    """The layer norm of the rows of x (float, [rows, cols]), times ``weight`` and plus ``bias`` ([cols], of any float type): y in
    ``out_dtype`` (x's), or with ``integer`` as an IntegerMatrix.  With ``training`` (y, mean, rstd), the latter fp32 [rows] for the gradient."""
    if stream is not None:
        with _on(stream):
            return maddness_layer_norm(x, weight, bias, eps, training, integer, out_dtype, out)
    if integer and (out is not None or out_dtype is not None):
        raise ValueError("integer goes without out and out_dtype")
    r = _m._native.layer_norm(x, weight, bias, eps, training, integer, out_dtype, out)
    if r is not NotImplemented:
        r = _m._done(r)
        return r if not integer else (IntegerMatrix._made(r[0], r[1]), *r[2:]) if training else IntegerMatrix._made(*r)
    torch = _m._torch or _m._torch_module()
    code = _code(x, "x")
    rows, cols, ldx = _m._rows(x, "x")
    weight_p, bias_p, parameter_code = _parameters(weight, bias, cols)
    _same_device(x, weight, bias, out)
    _here(x)
    mean, rstd = (torch.empty(rows, dtype=torch.float32, device=x.device) for _ in range(2)) if training else (None, None)
    if integer:
        y = IntegerMatrix.empty(rows, cols, x.device)
        s = y._struct
        out_p, out_code, ldo, scale_p = s.data, MADDNESS_I8, s.ld, s.scale
    else:
        if out is None:
            out = torch.empty((rows, cols), dtype=out_dtype or x.dtype, device=x.device)
        elif tuple(out.shape) != (rows, cols) or (out_dtype is not None and out.dtype is not out_dtype):
            raise ValueError(f"out must have shape {(rows, cols)}{'' if out_dtype is None else f' and dtype {out_dtype}'}")
        y, out_p, out_code, ldo, scale_p = out, out.data_ptr(), _code(out, "out"), _m._rows(out, "out")[2], None
    _m._check(_m.lib().maddness_layer_norm(x.data_ptr(), code, rows, cols, ldx, weight_p, bias_p, parameter_code, eps, out_p, out_code, ldo, scale_p,
                                           mean.data_ptr() if training else None, rstd.data_ptr() if training else None, _m._stream(None)))
    return (y, mean, rstd) if training else y


def maddness_layer_norm_gradient(gradient, x, mean, rstd, weight=None, parameters=None, stream=None):
    """From the gradient of maddness_layer_norm's y: (dx of x's dtype, dweight, dbias), the latter fp32 [cols], or None without
    ``parameters`` (by default with a weight)."""
    if parameters is None:
        parameters = weight is not None
    if stream is not None:
        with _on(stream):
            return maddness_layer_norm_gradient(gradient, x, mean, rstd, weight, parameters)
    r = _m._native.layer_norm_gradient(gradient, x, mean, rstd, weight, parameters)
    if r is not NotImplemented:
        return _m._done(r)
    torch = _m._torch or _m._torch_module()
    gradient_code, code = _code(gradient, "gradient"), _code(x, "x")
    rows, cols, ldx = _m._rows(x, "x")
    if tuple(gradient.shape) != (rows, cols):
        raise ValueError(f"gradient must have shape {(rows, cols)}, has {tuple(gradient.shape)}")
    mean_p, rstd_p = _flat(mean, torch.float32, (rows,), "mean"), _flat(rstd, torch.float32, (rows,), "rstd")
    weight_p, _, parameter_code = _parameters(weight, None, cols)
    _same_device(gradient, x, mean, rstd, weight)
    _here(x)
    dx = torch.empty((rows, cols), dtype=x.dtype, device=x.device)
    dweight = dbias = workspace = None
    need, L = 0, _m.lib()
    if parameters:
        dweight, dbias = (torch.empty(cols, dtype=torch.float32, device=x.device) for _ in range(2))
        need = L.maddness_layer_norm_gradient_workspace(rows, cols)
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
    _m._check(L.maddness_layer_norm_gradient(
        gradient.data_ptr(), gradient_code, _m._rows(gradient, "gradient")[2], x.data_ptr(), code, rows, cols, ldx, mean_p, rstd_p, weight_p, parameter_code,
        dx.data_ptr(), max(cols, 1), dweight.data_ptr() if parameters else None, dbias.data_ptr() if parameters else None,
        workspace.data_ptr() if parameters else None, need, _m._stream(None)))
    return dx, dweight, dbias


def maddness_balance(logits, ids, scores: str = "softmax", factor: float = 1.0, stream=None):
    """How evenly maddness_route's tokens fall on the experts: (loss, fp32 scalar tensor: ``factor`` where all experts have as many, more
    otherwise; counts int32 [E]; push fp32 [E], for the gradient)."""
    if stream is not None:
        with _on(stream):
            return maddness_balance(logits, ids, scores, factor)
    r = _m._native.balance(logits, ids, _scores(scores) == 1, factor)
    if r is not NotImplemented:
        return _m._done(r)
    torch = _m._torch or _m._torch_module()
    code = _code(logits, "logits")
    T, E, ldl = _m._rows(logits, "logits")
    if ids.dim() != 2 or ids.shape[1] < 1:
        raise ValueError("ids must be [T, k]")
    _same_device(logits, ids)
    _here(logits)
    k, L = ids.shape[1], _m.lib()
    ids_p = _flat(ids, torch.int32, (T, k), "ids")
    loss = torch.empty((), dtype=torch.float32, device=logits.device)
    counts = torch.empty(E, dtype=torch.int32, device=logits.device)
    push = torch.empty(E, dtype=torch.float32, device=logits.device)
    need = L.maddness_balance_workspace(T, E)
    workspace = torch.empty(need, dtype=torch.uint8, device=logits.device)
    _m._check(L.maddness_balance(logits.data_ptr(), code, T, E, ldl, _scores(scores), ids_p, k, factor, loss.data_ptr(), counts.data_ptr(), push.data_ptr(),
                                 workspace.data_ptr(), need, _m._stream(None)))
    return loss, counts, push


def maddness_balance_gradient(logits, push, scores: str = "softmax", loss_gradient=None, add=None, out=None, stream=None):
    """The gradient of the logits (their dtype, [T, E]) of maddness_balance's loss, times ``loss_gradient`` (an fp32 tensor of one element)
    and plus ``add`` ([T, E] of the logits' dtype: the gradient that they have already; it may be ``out`` too)."""
    if stream is not None:
        with _on(stream):
            return maddness_balance_gradient(logits, push, scores, loss_gradient, add, out)
    r = _m._native.balance_gradient(logits, push, _scores(scores) == 1, loss_gradient, add, out)
    if r is not NotImplemented:
        return _m._done(r)
    torch = _m._torch or _m._torch_module()
    code = _code(logits, "logits")
    T, E, ldl = _m._rows(logits, "logits")
    push_p = _flat(push, torch.float32, (E,), "push")
    times_p = None if loss_gradient is None else _flat(loss_gradient.reshape(-1), torch.float32, (1,), "loss_gradient")
    if out is None:
        out = torch.empty((T, E), dtype=logits.dtype, device=logits.device)
    for t, name in ((add, "add"), (out, "out")):
        if t is not None and (tuple(t.shape) != (T, E) or t.dtype is not logits.dtype):
            raise ValueError(f"{name} must have shape {(T, E)} and dtype {logits.dtype}")
        if t is not None:
            _code(t, name)
    _same_device(logits, push, loss_gradient, add, out)
    _here(logits)
    _m._check(_m.lib().maddness_balance_gradient(logits.data_ptr(), code, T, E, ldl, _scores(scores), push_p, times_p, None if add is None else add.data_ptr(),
                                                 0 if add is None else _m._rows(add, "add")[2], out.data_ptr(), _m._rows(out, "out")[2], _m._stream(None)))
    return out


def _dense(t, name: str) -> int:
    """The type code of a tensor whose elements fill one run of memory, each once, in whatever order."""
    code = _code(t, name)
    if not t.is_contiguous():
        run = 1
        for stride, size in sorted((s, n) for s, n in zip(t.stride(), t.shape) if n != 1):
            if stride != run:
                raise ValueError(f"{name} must fill its memory without gaps")
            run *= size
    return code


def _listed(tensors, name: str) -> list:
    torch = _m._torch or _m._torch_module()
    if isinstance(tensors, torch.Tensor):
        raise TypeError(f"{name} must be a list of tensors")
    return list(tensors)


def _table(tensors, outs, which: str):
    table = (_m._Tensor * max(len(tensors), 1))()
    for i, t in enumerate(tensors):
        code = _dense(t, f"{which}[{i}]")
        table[i] = _m._Tensor(t.data_ptr(), None, t.numel(), code, code)
        if outs is None:
            continue
        o = outs[i]
        if o is not t:
            if o.shape != t.shape or (t.stride() != o.stride() and not (t.is_contiguous() and o.is_contiguous())):
                raise ValueError(f"out[{i}] must have the shape and strides of {which}[{i}]")
            table[i].out_dtype = _dense(o, f"out[{i}]")
        table[i].out = o.data_ptr()
    _same_device(*tensors, *(outs or ()))
    return table


def _norm_like(tensors):
    torch = _m._torch or _m._torch_module()
    device = tensors[0].device if len(tensors) else torch.device("cuda", torch.cuda.current_device())
    if len(tensors):
        _here(tensors[0])
    return (torch.empty((), dtype=torch.float32, device=device),
            torch.empty(_m.lib().maddness_gradient_norm_workspace(), dtype=torch.uint8, device=device))


def maddness_gradient_norm(tensors, stream=None):
    """The norm over all elements of a list of float tensors, an fp32 scalar tensor; summed in fp64."""
    if stream is not None:
        with _on(stream):
            return maddness_gradient_norm(tensors)
    tensors = _listed(tensors, "tensors")
    r = _m._native.clip_gradients(tensors, None, None, None)
    if r is not NotImplemented:
        return _m._done(r)
    table = _table(tensors, None, "tensors")
    norm, workspace = _norm_like(tensors)
    _m._check(_m.lib().maddness_gradient_norm(table, len(tensors), norm.data_ptr(), workspace.data_ptr(), workspace.numel(), _m._stream(None)))
    return norm


def maddness_clip_gradients(tensors, max_norm: float, norm=None, out=None, stream=None):
    """Scales a list of float tensors down to the norm ``max_norm`` where theirs is larger, in place or into the list ``out`` (their shapes, any float
    types); returns the norm as it was.  ``norm`` (fp32, one element): that instead of theirs, say of the tensors of all processes.  A
    norm that is not finite scales nothing."""
    if stream is not None:
        with _on(stream):
            return maddness_clip_gradients(tensors, max_norm, norm, out)
    tensors = _listed(tensors, "tensors")
    out = None if out is None else _listed(out, "out")
    max_norm = float(max_norm)
    r = _m._native.clip_gradients(tensors, max_norm, norm, out)
    if r is not NotImplemented:
        return _m._done(r)
    torch = _m._torch or _m._torch_module()
    if out is not None and len(out) != len(tensors):
        raise ValueError(f"out must have {len(tensors)} tensors, has {len(out)}")
    table = _table(tensors, tensors if out is None else out, "tensors")
    workspace = None
    given = norm is not None
    if given:
        norm_p = _flat(norm.reshape(-1), torch.float32, (1,), "norm")
        _same_device(norm, *tensors[:1])
        _here(norm)
    else:
        norm, workspace = _norm_like(tensors)
        norm_p = norm.data_ptr()
    _m._check(_m.lib().maddness_clip_gradients(table, len(tensors), max_norm, norm_p, int(given), None if given else workspace.data_ptr(),
                                               0 if given else workspace.numel(), _m._stream(None)))
    return norm
