"""The exact product at 8 bits, and the parts of a layer of experts: binding of the calls that ``include/maddness.h`` describes under
that heading.  Argument marshalling only, as in the package's other calls; no CPU fallback.

A matrix at 8 bits is a ``BlockMatrix``: values in E4M3 and one power of two for 128 of them along a row (``tile=1``) or for a tile of
128 x 128 (``tile=128``, what weights are kept in).  ``maddness_block_product(A, B)`` is ``A @ B.T`` of two of them; A may also be
float, its rows are then rounded within the call.  With W of shape [outputs, inputs] a layer and its gradients are

    W, Wt = maddness_quantise_blocks(weight, tile=128, both=True)
    y = maddness_block_product(x, W)
    dy, dy_t = maddness_quantise_blocks(grad, both=True)
    dx = maddness_block_product(dy, Wt)
    dw = maddness_block_product(dy_t, maddness_quantise_blocks(x, transposed=True), out_dtype=torch.float32)

The calls are no part of torch's autograd: an operand that requires a gradient is refused while gradients are recorded.  A program calls
the gradients' own calls, as above, or makes a torch.autograd.Function of both.
"""
from __future__ import annotations

import ctypes as C

import paper_2106_10860_amd as _m

BLOCK = 128
MADDNESS_E4M3 = 16
MADDNESS_DENSE, MADDNESS_BY_ROWS, MADDNESS_BY_DEPTH, MADDNESS_BY_CHOICE = 0, 1, 2, 4
MAX_CHOSEN = 512
_BY = {"rows": MADDNESS_BY_ROWS, "depth": MADDNESS_BY_DEPTH, "choice": MADDNESS_BY_CHOICE}
_SCORES = {"softmax": 0, "sigmoid": 1}
_INT_MAX = 2 ** 31 - 1


def _up(n: int, to: int) -> int:
    return -(-n // to) * to


def _on(stream):
    """A call with ``stream`` runs with that as the current one, so that its results and workspace are that stream's memory too: nothing
    else gets it before the call's kernels are done with it."""
    torch = _m._torch or _m._torch_module()
    return torch.cuda.stream(stream)


def _fits(**numbers) -> None:
    for name, v in numbers.items():
        if not -_INT_MAX - 1 <= v <= _INT_MAX:
            raise ValueError(f"{name} = {v} does not fit 32 bits")


def _no_gradient(t, name: str) -> None:
    if t.requires_grad and _m._torch.is_grad_enabled():
        raise ValueError(f"{name} requires a gradient, which these calls do not record: give {name}.detach(), or call under torch.no_grad() "
                         "or in a torch.autograd.Function, whose backward makes the gradients' calls")


def _code(t, name: str) -> int:
    """The dtype code of a floating device tensor."""
    torch = _m._torch or _m._torch_module()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    _no_gradient(t, name)
    return _float_code(t.dtype, name)


def _float_code(dtype, name: str) -> int:
    torch = _m._torch or _m._torch_module()
    code = (_m.MADDNESS_BF16 if dtype is torch.bfloat16 else _m.MADDNESS_F32 if dtype is torch.float32 else
            _m.MADDNESS_F16 if dtype is torch.float16 else None)
    if code is None:
        raise TypeError(f"{name} has dtype {dtype}; supported: float32, float16, bfloat16")
    return code


def _same_device(*tensors) -> None:
    devices = {t.device for t in tensors if t is not None}
    if len(devices) > 1:
        raise ValueError(f"tensors on several devices: {sorted(map(str, devices))}")


def _flat(t, dtype, shape, name: str):
    """Pointer of a contiguous device tensor of this type and shape (None: NULL)."""
    if t is None:
        return None
    p = _m._ptr(t, dtype, name)
    _no_gradient(t, name)
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, has {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return p


class BlockMatrix:
    """8-bit values ``q`` [rows, cols] (or [experts, rows, cols]) of dtype float8_e4m3fn with unit column stride, and their exponents
    ``scale``, uint8 [rows / tile, cols / 128] each rounded up, the byte b for 2^(b - 127).  All may be replaced; every call checks what it finds."""

    __slots__ = ("q", "scale", "tile")

    def __init__(self, q, scale, tile: int = 1):
        self.q, self.scale, self.tile = q, scale, tile
        self._check()

    def _check(self) -> None:
        torch, q, scale, tile = _m._torch or _m._torch_module(), self.q, self.scale, self.tile
        if not isinstance(q, torch.Tensor) or not isinstance(scale, torch.Tensor) or not q.is_cuda or not scale.is_cuda:
            raise TypeError("q and scale must be device tensors")
        if q.dtype is not torch.float8_e4m3fn or scale.dtype is not torch.uint8:
            raise TypeError(f"q must have dtype float8_e4m3fn and scale uint8, have {q.dtype} and {scale.dtype}")
        if tile not in (1, BLOCK):
            raise ValueError("tile must be 1 or 128")
        if q.dim() not in (2, 3) or scale.dim() != q.dim():
            raise ValueError("q and scale must both be 2-D, or both 3-D with the experts first")
        rows, cols = q.shape[-2:]
        need = (*q.shape[:-2], -(-rows // tile), -(-cols // BLOCK))
        if tuple(scale.shape[:-1]) != need[:-1] or scale.shape[-1] < need[-1]:
            raise ValueError(f"scale must have shape {need} (or wider rows) for q of shape {tuple(q.shape)}, has {tuple(scale.shape)}")
        _same_device(q, scale)
        for t, name in ((q, "q"), (scale, "scale")):
            if t.shape[-1] > 1 and t.stride(-1) != 1:
                raise ValueError(f"{name} must have unit column stride")

    @classmethod
    def _made(cls, q, scale, tile: int) -> "BlockMatrix":
        """Of tensors that this package made."""
        b = cls.__new__(cls)
        b.q, b.scale, b.tile = q, scale, tile
        return b

    @property
    def shape(self):
        return tuple(self.q.shape)

    @property
    def _struct(self):
        self._check()

        def strides(t, unit):
            ld = t.stride(-2) if t.shape[-2] > 1 else _up(max(t.shape[-1], t.stride(-2)), unit)
            return ld, (t.stride(0) if t.dim() == 3 and t.shape[0] > 1 else 0)

        (ld, stride), (lds, scale_stride) = strides(self.q, 16), strides(self.scale, 4)
        rows, cols = self.q.shape[-2:]
        return _m._BlockMatrix(self.q.data_ptr(), MADDNESS_E4M3, self.tile, rows, cols, ld, stride, self.scale.data_ptr(), lds, scale_stride)

    @property
    def device(self):
        return self.q.device

    @classmethod
    def empty(cls, shape, tile: int = 1, device="cuda") -> "BlockMatrix":
        torch = _m._torch or _m._torch_module()
        *lead, rows, cols = shape
        q = torch.empty((*lead, rows, _up(cols, 16)), dtype=torch.float8_e4m3fn, device=device)[..., :cols]
        scale = torch.empty((*lead, -(-rows // tile), _up(-(-cols // BLOCK), 4)), dtype=torch.uint8, device=device)
        return cls(q, scale, tile)

    def values(self):
        """What the matrix stands for, in fp32 (elementary torch operations; for checks)."""
        torch = _m._torch or _m._torch_module()
        rows, cols = self.shape[-2:]
        e = self.scale.to(torch.int32)[..., : -(-cols // BLOCK)].repeat_interleave(BLOCK, -1)[..., :cols]
        if self.tile != 1:
            e = e.repeat_interleave(self.tile, -2)[..., :rows, :]
        return (self.q.double() * torch.exp2(e.double() - 127)).float()


def maddness_quantise_blocks(x, tile: int = 1, transposed: bool = False, both: bool = False, source=None, repeat: int = 1, factors=None,
                             stream=None):
    """x (float, [rows, cols] or [experts, rows, cols] with unit column stride) as a BlockMatrix; with ``transposed`` its transpose,
    with ``both`` the pair of them from one pass.

    ``source`` (int32 [rows']): row r of the result is x[source[r] // repeat] (times factors[source[r]] where ``factors``, fp32, is
    given), zeros where source[r] is negative; x is 2-D then."""
    if stream is not None:
        with _on(stream):
            return maddness_quantise_blocks(x, tile, transposed, both, source, repeat, factors)
    r = _m._native.quantise_blocks(x, tile, transposed, both, source, repeat, factors)
    if r is not NotImplemented:
        r = _m._done(r)
        return (BlockMatrix._made(r[0], r[1], tile), BlockMatrix._made(r[2], r[3], tile)) if both else BlockMatrix._made(r[0], r[1], tile)
    torch = _m._torch or _m._torch_module()
    code = _code(x, "x")
    if x.dim() == 2:
        x_rows, cols, ldx = _m._rows(x, "x")
        lead, count, stride_x = (), 1, 0
    elif x.dim() == 3 and source is None:
        _, cols, ldx = _m._rows(x[0], "x") if x.shape[0] else (0, x.shape[2], x.shape[2])
        x_rows, count = x.shape[1], x.shape[0]
        lead, stride_x = (count,), x.stride(0)
    else:
        raise ValueError("x must be 2-D, or 3-D with the experts first (not with source)")
    rows = x_rows
    if source is None:
        source_p = factors_p = None
        if factors is not None:
            raise ValueError("factors go with source")
    else:
        if source.dim() != 1 or repeat < 1:
            raise ValueError("source must be 1-D and repeat >= 1")
        _fits(repeat=repeat)
        _same_device(x, source, factors)
        rows = source.shape[0]
        source_p = _flat(source, torch.int32, (rows,), "source")
        factors_p = None if factors is None else _flat(factors.view(-1), torch.float32, (x_rows * repeat,), "factors")
    a = BlockMatrix.empty((*lead, rows, cols), tile, x.device) if both or not transposed else None
    b = BlockMatrix.empty((*lead, cols, rows), tile, x.device) if both or transposed else None
    s, t = (a._struct if a else None), (b._struct if b else None)
    _m._check(_m.lib().maddness_quantise_blocks(
        x.data_ptr(), code, count, rows, cols, ldx, stride_x, tile, source_p, x_rows, repeat, factors_p,
        s and s.data, s.ld if s else 0, s and s.scale, s.lds if s else 0, t and t.data, t.ld if t else 0, t and t.scale, t.lds if t else 0,
        _m._stream(None)))
    return (a, b) if both else (b if transposed else a)


def maddness_block_product(A, B: BlockMatrix, offsets=None, by: str = "rows", source=None, repeat: int = 1, out_dtype=None, out=None, workspace=None, stream=None):
    """A @ B.T.  A: a BlockMatrix or a float tensor [M, K]; B: a BlockMatrix [N, K].  Sums are fp32, rounded once to ``out_dtype`` (bfloat16); for
    bfloat16 results of many rows the products of every eight neighbours are cut off at 2^-13 of the largest before, with float32 never.

    With ``offsets`` (int32 [experts + 1]) by experts: by="rows" multiplies rows offsets[e] .. offsets[e + 1] - 1 of A with B[e]
    (B [experts, N, K]) into out [M, N], rows that no expert has are left as they are; by="depth" gives out [experts, M, N] from the
    columns offsets[e] .. offsets[e + 1] - 1 of A [M, K] and B [N, K] (multiples of 128).

    With ``source`` (int32 [slots], by="rows") out is [slots, N] and its row r that of A's row source[r] // repeat; rows whose source is
    negative are left as they are.

    by="choice" takes the experts' ids themselves as ``source`` (int32 [slots] or [M, k], slots up to 512) in place of an order: out is
    [slots, N] and its row r that of A's row r // repeat (k of a source [M, k]) with B[source[r]], zeros for an id of no expert."""
    if not isinstance(B, BlockMatrix):
        raise TypeError("B must be a BlockMatrix")
    how = _BY.get(by)
    if how is None:
        raise ValueError(f"by must be 'rows', 'depth' or 'choice', is {by!r}")
    if how == MADDNESS_BY_DEPTH and offsets is None:
        raise ValueError("by='depth' needs offsets")
    if how == MADDNESS_BY_CHOICE:
        if source is None or offsets is not None:
            raise ValueError("by='choice' goes with source, and without offsets")
        if source.dim() == 2:
            repeat, source = max(source.shape[1], 1), source.view(-1)
    if stream is not None:
        with _on(stream):
            return maddness_block_product(A, B, offsets, by, source, repeat, out_dtype, out, workspace)
    r = _m._native.block_product(isinstance(A, BlockMatrix), A, B, offsets, how, source, repeat, out_dtype, out, workspace)
    if r is not NotImplemented:
        return _m._done(r)
    torch = _m._torch or _m._torch_module()
    b = B._struct
    if isinstance(A, BlockMatrix):
        A._check()
        if len(A.shape) != 2:
            raise ValueError("A must be 2-D")
        a, a_dtype, (M, K), device = A._struct, MADDNESS_E4M3, A.shape, A.device
    else:
        a_dtype = _code(A, "A")
        M, K, lda = _m._rows(A, "A")
        a, device = _m._BlockMatrix(A.data_ptr(), a_dtype, 1, M, K, lda, 0, None, 0, 0), A.device
    N, a_rows, source_p = B.shape[-2], M, None
    if source is not None:
        if how != MADDNESS_BY_CHOICE and (offsets is None or how != MADDNESS_BY_ROWS) or source.dim() != 1 or repeat < 1:
            raise ValueError("source must be 1-D, with offsets, by='rows' and repeat >= 1, or with by='choice'")
        _fits(repeat=repeat)
        M = source.shape[0]
        source_p = _flat(source, torch.int32, (M,), "source") if M or offsets is None else offsets.data_ptr()      # (an empty one may have no address, and is not read)
    if how == MADDNESS_BY_CHOICE:
        if len(B.shape) != 3:
            raise ValueError(f"B must be [experts, N, K], has shape {B.shape}")
        groups, offsets_p, lead = B.shape[0], None, ()
    elif offsets is None:
        how, groups, offsets_p, lead = MADDNESS_DENSE, 1, None, ()
        if len(B.shape) != 2:
            raise ValueError("B of several experts needs offsets, or by='choice'")
    else:
        groups = offsets.shape[0] - 1 if offsets.dim() == 1 else -1
        if groups < 1:
            raise ValueError("offsets must be 1-D with one entry more than there are experts")
        offsets_p = _flat(offsets, torch.int32, (groups + 1,), "offsets")
        lead = () if by == "rows" else (groups,)
        if by == "rows" and (len(B.shape) != 3 or B.shape[0] != groups):
            raise ValueError(f"B must be [experts, N, K] with {groups} experts, has shape {B.shape}")
        if by == "depth" and len(B.shape) != 2:
            raise ValueError("B must be 2-D for by='depth'")
    if out is None:
        out = torch.empty((*lead, M, N), dtype=out_dtype or torch.bfloat16, device=device)
    elif tuple(out.shape) != (*lead, M, N) or (out_dtype is not None and out.dtype is not out_dtype):
        raise ValueError(f"out must have shape {(*lead, M, N)}{'' if out_dtype is None else f' and dtype {out_dtype}'}")
    elif lead and not out.is_contiguous():
        raise ValueError("out must be contiguous")
    _same_device(B.q, out, offsets, source, A.q if isinstance(A, BlockMatrix) else A, workspace)
    ldo = _m._rows(out.view(-1, N) if lead and N else out[0] if lead else out, "out")[2]
    L = _m.lib()
    need = L.maddness_block_product_workspace(a_rows, K, how, a_dtype) if a_dtype != MADDNESS_E4M3 else 0
    if workspace is None and need:
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
    if workspace is not None and not workspace.is_contiguous():              # (its size in bytes is then not what it has room for)
        raise ValueError("workspace must be contiguous")
    _m._check(L.maddness_block_product(C.byref(a), C.byref(b), how, groups, offsets_p, source_p, M, repeat, out.data_ptr(), _code(out, "out"), ldo,
                                       _m._ptr(workspace, torch.uint8, "workspace"), 0 if workspace is None else workspace.numel(),
                                       _m._stream(None)))
    return out


def _scores(scores: str) -> int:
    if scores not in _SCORES:
        raise ValueError(f"scores must be 'softmax' or 'sigmoid', is {scores!r}")
    return _SCORES[scores]


def maddness_route(logits, k: int, scores: str = "softmax", bias=None, groups: int = 1, kept_groups: int = 1, renormalise: bool = True,
                   factor: float = 1.0, stream=None):
    """Which k experts each token goes to, and with which weights: (ids int32 [T, k], -1 where there is none; weights fp32 [T, k])."""
    if stream is not None:
        with _on(stream):
            return maddness_route(logits, k, scores, bias, groups, kept_groups, renormalise, factor)
    r = _m._native.route(logits, k, _scores(scores) == 1, bias, groups, kept_groups, renormalise, factor)
    if r is not NotImplemented:
        return _m._done(r)
    torch = _m._torch or _m._torch_module()
    code = _code(logits, "logits")
    T, E, ldl = _m._rows(logits, "logits")
    _same_device(logits, bias)
    bias_p = _flat(bias, torch.float32, (E,), "bias")
    _fits(k=k, groups=groups, kept_groups=kept_groups)
    if k < 1:
        raise ValueError(f"k must be positive, is {k}")
    ids = torch.empty((T, k), dtype=torch.int32, device=logits.device)
    weights = torch.empty((T, k), dtype=torch.float32, device=logits.device)
    _m._check(_m.lib().maddness_route(logits.data_ptr(), code, T, E, ldl, bias_p, _scores(scores), groups, kept_groups, k,
                                      1 if renormalise else 0, factor, ids.data_ptr(), weights.data_ptr(), _m._stream(None)))
    return ids, weights


def maddness_route_gradient(logits, ids, weights_gradient, scores: str = "softmax", renormalise: bool = True, factor: float = 1.0, stream=None):
    """The gradient of the logits (their dtype, [T, E]) from that of the weights that maddness_route gave with these ids."""
    if stream is not None:
        with _on(stream):
            return maddness_route_gradient(logits, ids, weights_gradient, scores, renormalise, factor)
    r = _m._native.route_gradient(logits, ids, weights_gradient, _scores(scores) == 1, renormalise, factor)
    if r is not NotImplemented:
        return _m._done(r)
    torch = _m._torch or _m._torch_module()
    code = _code(logits, "logits")
    T, E, ldl = _m._rows(logits, "logits")
    if ids.dim() != 2:
        raise ValueError("ids must be [T, k]")
    k = ids.shape[1]
    _same_device(logits, ids, weights_gradient)
    ids_p = _flat(ids, torch.int32, (T, k), "ids")
    dw_p = _flat(weights_gradient, torch.float32, (T, k), "weights_gradient")
    out = torch.empty((T, E), dtype=logits.dtype, device=logits.device)
    _m._check(_m.lib().maddness_route_gradient(logits.data_ptr(), code, T, E, ldl, _scores(scores), k, 1 if renormalise else 0, factor, ids_p,
                                               dw_p, out.data_ptr(), E, _m._stream(None)))
    return out


def maddness_order(ids, experts: int, align: int = 1, stream=None):
    """The slots (choice j of token t is slot t * k + j) in the order of their experts: (offsets int32 [experts + 1], each expert's places
    a multiple of ``align``; counts int32 [experts]; source int32 [places], the slot at each place or -1; place int32 of ids' shape, or -1)."""
    if stream is not None:
        with _on(stream):
            return maddness_order(ids, experts, align)
    r = _m._native.order(ids, experts, align)
    if r is not NotImplemented:
        return _m._done(r)
    torch = _m._torch or _m._torch_module()
    ids_p = _flat(ids, torch.int32, ids.shape, "ids")
    slots, dev, L = ids.numel(), ids.device, _m.lib()
    if not 0 < experts <= _INT_MAX or not 0 < align <= _INT_MAX:
        raise ValueError("experts and align must be positive")
    capacity = L.maddness_order_capacity(slots, experts, align)
    need = max(4, L.maddness_order_workspace(slots, experts))
    ints = torch.empty(experts + 1 + experts + capacity + need // 4, dtype=torch.int32, device=dev)
    offsets, counts, source, workspace = ints.split([experts + 1, experts, capacity, need // 4])
    place = torch.empty(ids.shape, dtype=torch.int32, device=dev)
    _m._check(L.maddness_order(ids_p, slots, experts, align, offsets.data_ptr(), counts.data_ptr(), source.data_ptr(), capacity,
                               place.data_ptr(), workspace.data_ptr(), need, _m._stream(None)))
    return offsets, counts, source, place


def maddness_combine(y, place=None, weights=None, out_dtype=None, out=None, stream=None):
    """out[t] = sum over j of weights[t, j] * y[place[t, j]]; a negative place adds nothing, weights None are 1.  place None, with weights
    [T, k]: y[t * k + j]."""
    if stream is not None:
        with _on(stream):
            return maddness_combine(y, place, weights, out_dtype, out)
    r = _m._native.combine(y, place, weights, out_dtype, out)
    if r is not NotImplemented:
        return _m._done(r)
    torch = _m._torch or _m._torch_module()
    code = _code(y, "y")
    rows, N, ldy = _m._rows(y, "y")
    slots = weights if place is None else place
    if slots is None or slots.dim() != 2:
        raise ValueError("place must be [T, k], or None and weights [T, k]")
    T, k = slots.shape
    if out is None:
        out = torch.empty((T, N), dtype=out_dtype or y.dtype, device=y.device)
    elif tuple(out.shape) != (T, N) or (out_dtype is not None and out.dtype is not out_dtype):
        raise ValueError(f"out must have shape {(T, N)}{'' if out_dtype is None else f' and dtype {out_dtype}'}")
    _same_device(y, place, weights, out)
    _m._check(_m.lib().maddness_combine(y.data_ptr(), code, rows, N, ldy, _flat(place, torch.int32, (T, k), "place"),
                                        _flat(weights, torch.float32, (T, k), "weights"), T, k, out.data_ptr(), _code(out, "out"),
                                        _m._rows(out, "out")[2], _m._stream(None)))
    return out


def maddness_combine_gradient(gradient, y, place, stream=None):
    """The gradient of maddness_combine's weights, fp32 [T, k].  (That of y: maddness_quantise_blocks of the gradient with ``source``
    and ``factors``, or the gradient's rows times the weights.)"""
    if stream is not None:
        with _on(stream):
            return maddness_combine_gradient(gradient, y, place)
    r = _m._native.combine_gradient(gradient, y, place)
    if r is not NotImplemented:
        return _m._done(r)
    torch = _m._torch or _m._torch_module()
    code, y_code = _code(gradient, "gradient"), _code(y, "y")
    rows, N, ldy = _m._rows(y, "y")
    T, n, ldg = _m._rows(gradient, "gradient")
    if place.dim() != 2 or place.shape[0] != T or n != N:
        raise ValueError("gradient must be [T, N] and place [T, k] for y [rows, N]")
    k = place.shape[1]
    _same_device(gradient, y, place)
    out = torch.empty((T, k), dtype=torch.float32, device=y.device)
    _m._check(_m.lib().maddness_combine_gradient(gradient.data_ptr(), code, ldg, y.data_ptr(), y_code, rows, N, ldy,
                                                 _flat(place, torch.int32, (T, k), "place"), T, k, out.data_ptr(), _m._stream(None)))
    return out
