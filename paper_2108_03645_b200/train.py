"""Training-step operators: binding of ``ones_train.h`` (argument checks and marshalling only).

Layer norm, the cross entropy of a projection on a large vocabulary, both with their gradients, and the orthogonalised
update of matrix parameters, for CUDA tensors.  Work goes to torch's current stream of the tensors' device; outputs and
workspaces come from torch's allocator on that stream.  Nothing synchronises except `check`.

The functions take rows with any stride between them (a slice of a wider buffer is read in place).  Other layouts, and
for the cross entropy rows that do not start on 16-byte boundaries, are copied first.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import binding as _b

F32, BF16, F16 = 0, 1, 2
_TYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
MAX_NORM_COLS = 65536

_SIGNATURES = {
    "ones_layer_norm": (C.c_int, [C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_float, C.c_int32,
                                  C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p]),
    "ones_layer_norm_workspace_bytes": (C.c_size_t, [C.c_int32, C.c_int32]),
    "ones_layer_norm_backward": (C.c_int, [C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p,
                                           C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p,
                                           C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "ones_linear_ce_workspace_bytes": (C.c_size_t, [C.c_int32, C.c_int32]),
    "ones_linear_ce": (C.c_int, [C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_int32, C.c_int32, C.c_int32,
                                 C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "ones_linear_ce_backward_workspace_bytes": (C.c_size_t, [C.c_int32, C.c_int32, C.c_int32, C.c_int32]),
    "ones_linear_ce_backward": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p,
                                          C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p,
                                          C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_size_t, C.c_void_p]),
    "ones_orthogonalize_workspace_bytes": (C.c_size_t, [C.c_int32, C.c_int32, C.c_int32]),
    "ones_orthogonalize": (C.c_int, [C.c_void_p, C.c_int64, C.c_int64, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                     C.c_float, C.c_float, C.c_float, C.c_float, C.c_void_p, C.c_void_p, C.c_size_t,
                                     C.c_void_p]),
    "ones_train_status": (C.c_int, [C.c_void_p]),
}

_lib = None


def lib() -> C.CDLL:
    """The loaded library; raises if it is missing (there is no fallback)."""
    global _lib
    if _lib is None:
        L = _b.lib()
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def _device(t: torch.Tensor, call):
    """The result of `call` made with the tensor's device current."""
    with torch.cuda.device(t.device):
        return call()


def _rows(t: torch.Tensor, align: int = 0) -> tuple[torch.Tensor, int]:
    """`t` [..][cols] as rows that can be read, and the distance between two of them in values.  align: 8 for rows that
    have to start on 16-byte boundaries (16-bit types)."""
    if t.dim() != 2:
        t = t.reshape(-1, t.shape[-1])
    n, c = t.shape
    ld, inner = t.stride()
    if n <= 1:  # there is no second row
        ld = (max(c, 1) + align - 1) // align * align if align else max(c, 1)
    if (inner != 1 and c > 1) or ld < c:
        t = t.contiguous()
        ld = c
    if align and (ld % align or t.data_ptr() % 16):
        ld = (c + align - 1) // align * align
        wide = torch.empty(n, ld, dtype=t.dtype, device=t.device)
        wide[:, :c] = t
        t = wide
    return t, ld


def _like(t: torch.Tensor) -> torch.Tensor:
    return torch.empty_like(t) if t.is_contiguous() else torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _vector(n: int, dtype, device) -> torch.Tensor:
    return torch.empty_strided((n,), (1,), dtype=dtype, device=device)


_stream_of = torch._C._cuda_getCurrentRawStream  # current_stream(device).cuda_stream without the Stream object
_current = torch.cuda.current_device


def _done(rc: int, where: str):
    if rc:
        raise _b.OnesError(rc, where)


def _is_param(t, cols, x) -> bool:
    return (t.dim() == 1 and t.size(0) == cols and t.device == x.device and t.is_contiguous() and
            (t.dtype is torch.float32 or t.dtype is x.dtype))


def layer_norm(x: torch.Tensor, weight=None, bias=None, eps: float = 1e-5):
    """Layer norm over the last dimension (``ones_layer_norm``): (y, mean, rstd), mean and rstd in float32 with x's
    leading dimensions.  weight and bias: None, or vectors of x's type or of float32 (both of one type)."""
    kind = _TYPES.get(x.dtype) if x.is_cuda and x.dim() else None
    if kind is None:
        raise ValueError("x: a float32, bfloat16 or float16 CUDA tensor is needed")
    lead, cols, device = x.shape[:-1], x.shape[-1], x.device
    wkind = F32
    wp = bp = None
    if bias is not None:
        if not _is_param(bias, cols, x):
            raise ValueError(f"bias: a contiguous vector of {cols} values of float32 or x's type on {device} is needed")
        wkind, bp = _TYPES[bias.dtype], bias.data_ptr()
    if weight is not None:
        if not _is_param(weight, cols, x) or (bias is not None and bias.dtype is not weight.dtype):
            raise ValueError(f"weight: a contiguous vector of {cols} values of float32 or x's type on {device} is needed, "
                             "of one type with bias")
        wkind, wp = _TYPES[weight.dtype], weight.data_ptr()
    index = device.index
    if index != _current():
        return _device(x, lambda: layer_norm(x, weight, bias, eps))
    p, ld = _rows(x)
    rows = p.size(0)
    y = _like(x)
    mean = _vector(rows, torch.float32, device)
    rstd = torch.empty_like(mean)
    _done((_lib or lib()).ones_layer_norm(p.data_ptr(), ld, wp, bp, rows, cols, eps, kind, wkind, y.data_ptr(), cols,
                                          mean.data_ptr(), rstd.data_ptr(), _stream_of(index)), "ones_layer_norm")
    if len(lead) != 1:
        mean, rstd = mean.view(lead), rstd.view(lead)
    return y, mean, rstd


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, weight=None, *,
                        parameters: bool = True):
    """Gradients of `layer_norm` (``ones_layer_norm_backward``): (dx, dweight, dbias), the latter two in the type of
    weight (float32 where it is None), or None both with parameters=False."""
    kind = _TYPES.get(x.dtype) if x.is_cuda and x.dim() else None
    if kind is None:
        raise ValueError("x: a float32, bfloat16 or float16 CUDA tensor is needed")
    shape, device = x.shape, x.device
    cols = shape[-1]
    if dy.shape != shape or dy.dtype is not x.dtype or dy.device != device:
        raise ValueError("dy needs x's shape, type and device")
    wt, wp = torch.float32, None
    if weight is not None:
        if not _is_param(weight, cols, x):
            raise ValueError(f"weight: a contiguous vector of {cols} values of float32 or x's type on {device} is needed")
        wt, wp = weight.dtype, weight.data_ptr()
    for s in (mean, rstd):
        if s.dtype is not torch.float32 or s.device != device or s.shape != shape[:-1] or not s.is_contiguous():
            raise ValueError("mean, rstd: what layer_norm returned is needed")
    index = device.index
    if index != _current():
        return _device(x, lambda: layer_norm_backward(dy, x, mean, rstd, weight, parameters=parameters))
    L = _lib or lib()
    p, ld = _rows(x)
    q, ldq = _rows(dy)
    rows = p.size(0)
    dx = _like(x)
    dw = db = dwp = dbp = sp = None
    nbytes = 0
    if parameters:
        dw = torch.empty_like(weight) if weight is not None else _vector(cols, wt, device)
        db = torch.empty_like(dw)
        nbytes = L.ones_layer_norm_workspace_bytes(rows, cols)
        space = _vector(nbytes, torch.uint8, device)
        dwp, dbp, sp = dw.data_ptr(), db.data_ptr(), space.data_ptr()
    _done(L.ones_layer_norm_backward(q.data_ptr(), ldq, p.data_ptr(), ld, mean.data_ptr(), rstd.data_ptr(), wp, rows, cols, kind,
                                     _TYPES[wt], dx.data_ptr(), cols, dwp, dbp, sp, nbytes, _stream_of(index)),
          "ones_layer_norm_backward")
    return dx, dw, db


def _ce_args(hidden, weight, target):
    if not hidden.is_cuda or hidden.dtype not in (torch.bfloat16, torch.float16) or not hidden.dim():
        raise ValueError("hidden: a bfloat16 or float16 CUDA tensor is needed")
    if (weight.dim() != 2 or weight.dtype is not hidden.dtype or weight.device != hidden.device or
            weight.size(1) != hidden.size(-1)):
        raise ValueError("weight: [vocab][cols] of hidden's type and device is needed")
    if target.dtype is not torch.int64 or target.device != hidden.device or target.shape != hidden.shape[:-1]:
        raise ValueError("target: int64 with hidden's leading dimensions is needed")


def linear_cross_entropy(hidden: torch.Tensor, weight: torch.Tensor, target: torch.Tensor):
    """Cross entropy of ``hidden @ weight.T`` at `target` without keeping the logits (``ones_linear_ce``): (loss, lse),
    float32 with hidden's leading dimensions.  Rows whose target is outside [0, vocab) have loss 0."""
    _ce_args(hidden, weight, target)
    device = hidden.device
    index = device.index
    if index != _current():
        return _device(hidden, lambda: linear_cross_entropy(hidden, weight, target))
    L = _lib or lib()
    h, ldh = _rows(hidden, 8)
    w, ldw = _rows(weight, 8)
    t = target.contiguous()
    rows, vocab, lead = h.size(0), w.size(0), target.shape
    loss = _vector(rows, torch.float32, device)
    lse = torch.empty_like(loss)
    nbytes = L.ones_linear_ce_workspace_bytes(rows, vocab)
    space = _vector(nbytes, torch.uint8, device)
    _done(L.ones_linear_ce(h.data_ptr(), ldh, w.data_ptr(), ldw, t.data_ptr(), rows, hidden.size(-1), vocab, _TYPES[hidden.dtype],
                           loss.data_ptr(), lse.data_ptr(), space.data_ptr(), nbytes, _stream_of(index)), "ones_linear_ce")
    if len(lead) != 1:
        loss, lse = loss.view(lead), lse.view(lead)
    return loss, lse


def linear_cross_entropy_backward(dloss: torch.Tensor, hidden: torch.Tensor, weight: torch.Tensor, target: torch.Tensor,
                                  lse: torch.Tensor, *, weight_gradient: torch.dtype | None = None, piece: int = 0):
    """Gradients of `linear_cross_entropy` for the gradient `dloss` of its loss (``ones_linear_ce_backward``):
    (dhidden, dweight).  weight_gradient: float32 for dweight in 32 bits (default: weight's type).  piece: entries of the
    vocabulary that are taken at a time (a multiple of 256; 0: the library's choice)."""
    _ce_args(hidden, weight, target)
    wt = weight_gradient or weight.dtype
    if wt is not torch.float32 and wt is not weight.dtype:
        raise ValueError("weight_gradient: float32 or weight's type is needed")
    device = hidden.device
    for s in (dloss, lse):
        if s.dtype is not torch.float32 or s.device != device or s.shape != target.shape:
            raise ValueError("dloss, lse: float32 with target's shape is needed")
    index = device.index
    if index != _current():
        return _device(hidden, lambda: linear_cross_entropy_backward(dloss, hidden, weight, target, lse,
                                                                     weight_gradient=weight_gradient, piece=piece))
    L = _lib or lib()
    h, ldh = _rows(hidden)
    w, ldw = _rows(weight, 8)
    t, g, l = target.contiguous(), dloss.contiguous(), lse.contiguous()
    rows, cols, vocab = h.size(0), hidden.size(-1), w.size(0)
    dh = _like(hidden)
    dw = torch.empty(weight.shape, dtype=wt, device=device)
    nbytes = L.ones_linear_ce_backward_workspace_bytes(rows, cols, vocab, piece)
    space = _vector(nbytes, torch.uint8, device)
    _done(L.ones_linear_ce_backward(g.data_ptr(), h.data_ptr(), ldh, w.data_ptr(), ldw, t.data_ptr(), l.data_ptr(), rows, cols,
                                    vocab, _TYPES[hidden.dtype], _TYPES[wt], piece, dh.data_ptr(), cols, dw.data_ptr(), cols,
                                    space.data_ptr(), nbytes, _stream_of(index)), "ones_linear_ce_backward")
    return dh, dw


def orthogonalize(g: torch.Tensor, *, steps: int = 5, coefficients=(3.4445, -4.7750, 2.0315), eps: float = 1e-7) -> torch.Tensor:
    """Newton-Schulz orthogonalised update (``ones_orthogonalize``) of a matrix [m][n], or of several [count][m][n], in
    bfloat16."""
    kind = _TYPES.get(g.dtype) if g.is_cuda and g.dim() in (2, 3) else None
    if kind is None:
        raise ValueError("g: a float32, bfloat16 or float16 CUDA matrix is needed, or several")
    a, b, c = coefficients
    device = g.device
    index = device.index
    if index != _current():
        return _device(g, lambda: orthogonalize(g, steps=steps, coefficients=coefficients, eps=eps))
    L = _lib or lib()
    s = g if g.dim() == 3 else g[None]
    count, m, n = s.shape
    if (s.stride(2) != 1 and n > 1) or (s.stride(1) < n and m > 1):
        s = s.contiguous()
    out = torch.empty(g.shape, dtype=torch.bfloat16, device=device)
    if count * m * n == 0:
        return out
    nbytes = L.ones_orthogonalize_workspace_bytes(count, m, n)
    if nbytes == 0:
        raise _b.OnesError(-3, "ones_orthogonalize_workspace_bytes")
    space = _vector(nbytes, torch.uint8, device)
    _done(L.ones_orthogonalize(s.data_ptr(), s.stride(1) if m > 1 else n, s.stride(0), count, m, n, kind, steps, a, b, c, eps,
                               out.data_ptr(), space.data_ptr(), nbytes, _stream_of(index)), "ones_orthogonalize")
    return out


def check() -> None:
    """Waits for the current stream and raises if a kernel gave up waiting since the last check (``ones_train_status``)."""
    _done(lib().ones_train_status(torch.cuda.current_stream().cuda_stream), "ones_train_status")


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        y, mean, rstd = layer_norm(x, weight, bias, eps)
        ctx.save_for_backward(x, weight, mean, rstd)
        ctx.has_bias = bias is not None
        return y

    @staticmethod
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        dx, dw, db = layer_norm_backward(dy, x, mean, rstd, weight, parameters=weight is not None or ctx.has_bias)
        return dx, dw if weight is not None else None, db if ctx.has_bias else None, None


class _LinearCrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, hidden, weight, target):
        loss, lse = linear_cross_entropy(hidden, weight, target)
        ctx.save_for_backward(hidden, weight, target, lse)
        return loss

    @staticmethod
    def backward(ctx, dloss):
        hidden, weight, target, lse = ctx.saved_tensors
        return (*linear_cross_entropy_backward(dloss, hidden, weight, target, lse), None)


def layer_norm_autograd(x, weight=None, bias=None, eps: float = 1e-5) -> torch.Tensor:
    """`layer_norm` as a differentiable function of x, weight and bias: y."""
    return _LayerNorm.apply(x, weight, bias, eps)


def linear_cross_entropy_autograd(hidden, weight, target) -> torch.Tensor:
    """`linear_cross_entropy` as a differentiable function of hidden and weight: the loss of each row."""
    return _LinearCrossEntropy.apply(hidden, weight, target)
