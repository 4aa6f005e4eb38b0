"""Operators of an 8-bit linear layer: quantiser, product, norm, and the layer with
its gradients (C ABI in ``include/prm.h``).

The functions marshal tensors and allocate outputs; the arithmetic runs in libprm's
kernels, on the tensors' device and its current torch stream, and nothing waits for
the GPU: every call may be captured into a HIP graph.  Activations are float32,
bfloat16 or float16, with any number of leading dimensions and any strides (a tensor
whose rows are not contiguous is copied first).

The 8-bit form of a matrix is a pair: int8 ``q`` and a float32 ``scale`` for each of its
rows, ``s = max|v| / 127``, ``q = rn(127 v / max|v|)``.  A row of zeros has scale 0, a row
with an infinity or a NaN has scale NaN.

Gradients are those of backward passes.  Forward-mode derivatives, and traces (``torch.jit.trace``,
``make_fx``), do not see what runs here: both are refused.
"""
from __future__ import annotations

import torch
from torch.autograd import forward_ad

from . import BF16, F16, F32, _check, load

load()  # libprm.so, or a loud error
try:  # the plain calls, natively where _operators.so is built; None: not a plain call
    from . import _operators as _native
except ImportError:
    class _native:
        quantize_rows = quantize_cols = int8_matmul = int8_linear = rms_norm = staticmethod(lambda *a: None)

__all__ = ["quantize_rows", "int8_matmul", "int8_linear", "rms_norm"]

_CODE = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}


def _float_code(x, what):
    code = _CODE.get(x.dtype)
    if code is None:
        raise ValueError(f"{what}: need float32, bfloat16 or float16, got {x.dtype}")
    return code


def _on_device(x, what):
    if not x.is_cuda:
        raise ValueError(f"{what}: need a device tensor, got one on {x.device}")


def _seen(call, *inputs):
    """Refuses what would be lost without a word: a call under a tracer, which records the outputs'
    allocation alone, and inputs with a tangent."""
    if torch.jit.is_tracing() or torch._C._get_dispatch_mode(torch._C._TorchDispatchModeKey.PROXY) is not None:
        raise RuntimeError(f"{call}: a trace does not see its kernels; call it outside of one")
    if forward_ad._current_level >= 0:
        for x in inputs:
            if isinstance(x, torch.Tensor) and forward_ad.unpack_dual(x).tangent is not None:
                raise RuntimeError(f"{call}: no forward-mode derivative")


def _same(x, like, shape, what):
    """x has the type and device of `like`, and this shape."""
    if tuple(x.shape) != tuple(shape) or x.dtype != like.dtype or x.device != like.device:
        raise ValueError(f"{what}: need {like.dtype} {tuple(shape)} on {like.device}, got {x.dtype} {tuple(x.shape)} on {x.device}")


def _rows(x):
    """(matrix of the last dimension's rows, its leading dimension): a view where the
    rows are contiguous and evenly spaced, else a copy.  Its memory holds its values: a view
    that stands for the negative (conj().imag) is copied."""
    x = x.resolve_neg()
    c = x.shape[-1]
    if x.dim() != 2:
        x = x.reshape(-1, c) if x.numel() else x.new_empty((x.numel() // max(c, 1), c))
    if (x.stride(1) != 1 and c > 1) or (x.stride(0) < c and x.shape[0] > 1):
        x = x.contiguous()
    return x, (x.stride(0) if x.shape[0] > 1 else max(c, 1))


def _vector(x):
    x = x.resolve_neg()
    return x if x.dim() == 1 and (x.stride(0) == 1 or x.shape[0] <= 1) else x.contiguous()


class _device_of:
    """The tensor's device as the current one; its current stream."""

    __slots__ = ("_guard", "stream")

    def __init__(self, x):
        i = x.device.index
        self._guard = None if i == torch.cuda.current_device() else torch.cuda.device(i)

    def __enter__(self):
        if self._guard is not None:
            self._guard.__enter__()
        self.stream = torch.cuda.current_stream().cuda_stream
        return self.stream

    def __exit__(self, *exc):
        if self._guard is not None:
            self._guard.__exit__(*exc)


def _count(x):
    """Leading rows of x, and its last dimension."""
    if x.dim() < 1:
        raise ValueError("need at least one dimension")
    c = x.shape[-1]
    if c < 1:
        raise ValueError("need a last dimension of one or more")
    return x.numel() // c, c


def _eight_bits(lead, cols, device):
    """An int8 tensor whose rows start on 16-byte boundaries (the product's fast loads)."""
    ld = (cols + 15) // 16 * 16
    q = torch.empty((*lead, ld), dtype=torch.int8, device=device)
    return (q if ld == cols else q[..., :cols]), ld


def quantize_rows(x, transpose: bool = False):
    """``(q, scale)``: the rows of ``x`` (``[..., cols]``) in 8 bits, a scale for each
    (``scale`` has the leading dimensions).  ``transpose`` (2-D ``x`` only): the columns
    instead, ``q`` is ``[cols, rows]`` and ``scale`` ``[cols]``, what
    ``quantize_rows(x.t())`` gives without a transposed copy.  Not differentiable."""
    if transpose:
        r = _native.quantize_cols(x)
        if r is not None:
            return r if type(r) is tuple else _check(r)
        _seen("quantize_rows")
        return _quantize_cols(x, False)[:2]
    r = _native.quantize_rows(x)
    if r is not None:
        return r if type(r) is tuple else _check(r)
    _seen("quantize_rows")
    _on_device(x, "x")
    code = _float_code(x, "x")
    x = x.detach()
    rows, cols = _count(x)
    with _device_of(x) as stream:
        q, ldq = _eight_bits(x.shape[:-1], cols, x.device)
        scale = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
        m, ldx = _rows(x)
        _check(load().prm_quantize_rows(m.data_ptr(), code, rows, cols, ldx, q.data_ptr(), ldq, scale.data_ptr(), stream))
    return q, scale


def _quantize_cols(x, with_sum):
    _on_device(x, "x")
    code = _float_code(x, "x")
    x = x.detach()
    if x.dim() != 2:
        raise ValueError(f"x: the transposed form needs a matrix, got {tuple(x.shape)}")
    rows, cols = _count(x)
    L = load()
    with _device_of(x) as stream:
        m, ldx = _rows(x)
        q, ldq = _eight_bits((cols,), max(rows, 1), x.device)
        scale = torch.empty(cols, dtype=torch.float32, device=x.device)
        total = torch.empty(cols, dtype=x.dtype, device=x.device) if with_sum else None
        need = L.prm_quantize_cols_workspace(rows, cols)
        ws = torch.empty(need, dtype=torch.uint8, device=x.device)
        _check(L.prm_quantize_cols(m.data_ptr(), code, rows, cols, ldx, q.data_ptr(), ldq, scale.data_ptr(),
                                   total.data_ptr() if with_sum else None, ws.data_ptr(), need, stream))
    return q, scale, total


def int8_matmul(a, a_scale, b, b_scale, bias=None, dtype=torch.bfloat16):
    """``a_scale a (b_scale b)^T + bias``: the product of 8-bit operands, ``a``
    ``[..., k]`` with a scale for each row (token) and ``b`` ``[n, k]`` with one for each
    row (output channel, as a linear layer's weight is kept; rows on 16-byte boundaries, as
    ``quantize_rows`` gives them, are the fast ones); ``bias`` ``[n]`` and the result ``[..., n]`` are
    of type ``dtype``.  The sum over k (at most 2^20) is exact; ``a_scale``, ``b_scale`` and
    bias are applied in this order in fp32 and the result rounded once.  Not differentiable
    (``int8_linear`` is)."""
    r = _native.int8_matmul(a, a_scale, b, b_scale, bias, _CODE.get(dtype, -1))
    if r is not None:
        return _check(r) if type(r) is int else r
    _seen("int8_matmul")
    for t, what in ((a, "a"), (b, "b")):
        _on_device(t, what)
        if t.dtype != torch.int8:
            raise ValueError(f"{what}: need int8, got {t.dtype}")
    if b.dim() != 2 or b.device != a.device:
        raise ValueError(f"b: need a matrix on {a.device}, got {tuple(b.shape)} on {b.device}")
    if dtype not in _CODE:
        raise ValueError(f"dtype: need float32, bfloat16 or float16, got {dtype}")
    rows, k = _count(a)
    n = b.shape[0]
    if b.shape[1] != k:
        raise ValueError(f"b: need rows of {k}, as a's, got {b.shape[1]}")
    for t, shape, what in ((a_scale, a.shape[:-1], "a_scale"), (b_scale, (n,), "b_scale")):
        if t.dtype != torch.float32 or tuple(t.shape) != tuple(shape) or t.device != a.device:
            raise ValueError(f"{what}: need float32 {tuple(shape)} on {a.device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    if bias is not None and (bias.dtype != dtype or tuple(bias.shape) != (n,) or bias.device != a.device):
        raise ValueError(f"bias: need {dtype} {(n,)} on {a.device}, got {bias.dtype} {tuple(bias.shape)} on {bias.device}")
    with _device_of(a) as stream:
        out = torch.empty((*a.shape[:-1], n), dtype=dtype, device=a.device)
        m, lda = _rows(a)
        bm, ldb = _rows(b)
        sa, sb = a_scale.resolve_neg().contiguous(), b_scale.resolve_neg().contiguous()
        bv = None if bias is None else _vector(bias.detach())
        L = load()
        need = L.prm_int8_matmul_workspace(m.data_ptr(), lda, bm.data_ptr(), ldb, rows, n, k)
        ws = torch.empty(need, dtype=torch.uint8, device=a.device) if need else None
        _check(L.prm_int8_matmul(m.data_ptr(), lda, sa.data_ptr(), bm.data_ptr(), ldb, sb.data_ptr(),
                                 None if bv is None else bv.data_ptr(), _CODE[dtype], out.data_ptr(), max(n, 1),
                                 rows, n, k, ws.data_ptr() if need else None, need, stream))
    return out


# ---- gradients of gradients: refused where they are asked for, and not before --------
class _Refuse(torch.autograd.Function):
    @staticmethod
    def forward(ctx, *grads):
        return tuple(g.detach() for g in grads)

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("these gradients are not differentiable")


def _once(backward):
    def wrapped(ctx, *grads):
        recording = torch.is_grad_enabled()
        with torch.no_grad():
            out = backward(ctx, *grads)
        if not recording:
            return out
        kept = [g.detach().requires_grad_() for g in out if g is not None]
        refusing = iter(_Refuse.apply(*kept)) if kept else iter(())
        return tuple(None if g is None else next(refusing) for g in out)
    return wrapped


# ---- norm ------------------------------------------------------------------
def _norm(x, weight, residual, eps, quantize):
    code = _float_code(x, "x")
    rows, cols = _count(x)
    with _device_of(x) as stream:
        m, ldx = _rows(x)
        h = q = scale = y = None
        rp = hp = yp = qp = sp = None
        ldr = ldq = 0
        if residual is not None:
            r, ldr = _rows(residual)
            rp = r.data_ptr()
            h = torch.empty(x.shape, dtype=x.dtype, device=x.device)
            hp = h.data_ptr()
        if quantize:
            q, ldq = _eight_bits(x.shape[:-1], cols, x.device)
            scale = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
            qp, sp = q.data_ptr(), scale.data_ptr()
        else:
            y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
            yp = y.data_ptr()
        w = None if weight is None else _vector(weight)
        if rows:
            _check(load().prm_rms_norm(m.data_ptr(), ldx, rp, ldr, None if w is None else w.data_ptr(), code, rows, cols,
                                       eps, hp, cols, yp, cols, qp, ldq, sp, stream))
    return y, q, scale, h


class _RmsNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, residual, eps):
        y, _, _, h = _norm(x, weight, residual, eps, False)
        ctx.save_for_backward(x if h is None else h, weight)
        ctx.eps = eps
        ctx.set_materialize_grads(False)
        return y if h is None else (y, h)

    @staticmethod
    @_once
    def backward(ctx, gy, gh=None):
        h, weight = ctx.saved_tensors
        need_dw = weight is not None and ctx.needs_input_grad[1]
        if gy is None:  # only the kept sum has a gradient, in which the weight takes no part
            return (gh if ctx.needs_input_grad[0] else None), None, (gh if ctx.needs_input_grad[2] else None), None
        _same(h, gy, gy.shape, "saved input")  # hooks may bring back something else
        if weight is not None:
            _same(weight, gy, gy.shape[-1:], "saved weight")
        rows, cols = _count(h)
        L = load()
        with _device_of(h) as stream:
            dx = torch.empty(h.shape, dtype=h.dtype, device=h.device)
            dw = torch.empty(cols, dtype=h.dtype, device=h.device) if need_dw else None
            mg, ldg = _rows(gy)
            mh, ldh = _rows(h)
            ms, lds = _rows(gh) if gh is not None else (None, 0)
            w = None if weight is None else _vector(weight)
            need = L.prm_rms_norm_backward_workspace(rows, cols) if need_dw else 0
            ws = torch.empty(need, dtype=torch.uint8, device=h.device) if need else None
            _check(L.prm_rms_norm_backward(mg.data_ptr(), ldg, None if ms is None else ms.data_ptr(), lds, mh.data_ptr(),
                                           ldh, None if w is None else w.data_ptr(), _CODE[h.dtype], rows, cols, ctx.eps,
                                           dx.data_ptr(), cols, dw.data_ptr() if need_dw else None,
                                           ws.data_ptr() if need else None, need, stream))
        return (dx if ctx.needs_input_grad[0] else None), dw, (dx if ctx.needs_input_grad[2] else None), None


def rms_norm(x, weight=None, residual=None, eps: float = 1e-6, quantize: bool = False):
    """Root-mean-square norm of the last dimension, ``h weight / sqrt(mean(h^2) + eps)``
    with ``h = x + residual`` (kept in x's type; the norm is that of the kept sum).

    Returns ``y``, or ``(y, h)`` with a residual; with ``quantize`` the norm in 8 bits,
    ``(q, scale)`` or ``(q, scale, h)``, for ``int8_matmul``.  ``weight`` ``[cols]`` and
    ``residual`` (shaped as x) have x's type.  The plain outputs are differentiable in
    x, weight and residual; the 8-bit ones are not.  Sums over a row are taken in fp32, where
    they leave its range in fp64 or scaled."""
    eps = float(eps)
    r = _native.rms_norm(x, weight, residual, eps, quantize)
    if r is not None:
        return _check(r) if type(r) is int else r
    _seen("rms_norm", x, weight, residual)
    _on_device(x, "x")
    _float_code(x, "x")
    _, cols = _count(x)
    if residual is not None:
        _same(residual, x, x.shape, "residual")
    if weight is not None:
        _same(weight, x, (cols,), "weight")
    grad = torch.is_grad_enabled() and (x.requires_grad or (weight is not None and weight.requires_grad)
                                        or (residual is not None and residual.requires_grad))
    if quantize:
        if grad:
            raise ValueError("the 8-bit output has no gradient: call under torch.no_grad(), or quantize=False and int8_linear")
        _, q, scale, h = _norm(x, weight, residual, eps, True)
        return (q, scale) if residual is None else (q, scale, h)
    if grad:
        return _RmsNorm.apply(x, weight, residual, eps)
    y, _, _, h = _norm(x, weight, residual, eps, False)
    return y if residual is None else (y, h)


# ---- linear layer ------------------------------------------------------------
class _Int8Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias):
        # each serves the other's gradient alone
        ctx.save_for_backward(x if ctx.needs_input_grad[1] else None, weight if ctx.needs_input_grad[0] else None)
        ctx.shape = x.shape
        return int8_matmul(*quantize_rows(x), *quantize_rows(weight), bias=bias, dtype=x.dtype)

    @staticmethod
    @_once
    def backward(ctx, gy):
        x, weight = ctx.saved_tensors
        need_x, need_w, need_b = ctx.needs_input_grad
        g = gy.reshape(-1, gy.shape[-1])
        dx = dw = db = None
        n, k = g.shape[1], ctx.shape[-1]
        if g.shape[0] == 0:
            return (g.new_zeros(ctx.shape) if need_x else None, g.new_zeros(n, k) if need_w else None, g.new_zeros(n) if need_b else None)
        if need_x:  # hooks may bring back something else
            _same(weight, g, (n, k), "saved weight")
            wq, ws, _ = _quantize_cols(weight, False)
            dx = int8_matmul(*quantize_rows(g), wq, ws, dtype=g.dtype).reshape(ctx.shape)
        if need_w:
            _same(x, g, ctx.shape, "saved input")
            gq, gs, db = _quantize_cols(g, need_b)
            xq, xs, _ = _quantize_cols(x.reshape(-1, x.shape[-1]), False)
            dw = int8_matmul(gq, gs, xq, xs, dtype=g.dtype)
        elif need_b:
            db = _quantize_cols(g, True)[2]
        return dx, dw, db


def int8_linear(x, weight, bias=None):
    """``x weight^T + bias`` with the product in 8 bits: ``x`` ``[..., k]`` quantised for
    each token, ``weight`` ``[n, k]`` for each output channel, all of one type, which the
    result ``[..., n]`` has.  Its gradients are those of the unquantised layer, their
    products in 8 bits too, each operand quantised along the sum it enters:
    ``dx = Q(gy) Q(weight^T)^T``, ``dweight = Q(gy^T) Q(x^T)^T``, ``dbias`` the sum of
    ``gy`` in fp32.  At most 2^24 tokens and outputs; a sum of at most 2^20: ``k`` in the
    result, the outputs in ``dx``, the tokens in ``dweight`` (in ``dbias`` 2^22).  Each rounding
    to 8 bits is off by at most half of 1/127 of its row's (column's) largest value."""
    r = _native.int8_linear(x, weight, bias)
    if r is not None:
        return _check(r) if type(r) is int else r
    _seen("int8_linear", x, weight, bias)
    _on_device(x, "x")
    _float_code(x, "x")
    _, k = _count(x)
    if weight.dim() != 2:
        raise ValueError(f"weight: need a matrix, got {tuple(weight.shape)}")
    n = weight.shape[0]
    if n < 1:
        raise ValueError("weight: need one output or more")
    _same(weight, x, (n, k), "weight")
    if bias is not None:
        _same(bias, x, (n,), "bias")
    return _Int8Linear.apply(x, weight, bias)
