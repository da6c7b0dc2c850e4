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


def _need(ok, what, *args):
    if not ok:
        raise ValueError(what.format(*args))


def _device(t: torch.Tensor, call):
    """None when the tensor's device is current; otherwise the result of `call` made with it current."""
    if t.device.index == torch.cuda.current_device():
        return None
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


def _space(nbytes: int, device) -> torch.Tensor:
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


_stream_of = torch._C._cuda_getCurrentRawStream  # current_stream(device).cuda_stream without the Stream object


def _done(rc: int, where: str):
    if rc:
        raise _b.OnesError(rc, where)


def _param(t, cols, x, name):
    _need(t.dim() == 1 and t.shape[0] == cols and t.device == x.device and t.is_contiguous(),
          "{}: a contiguous vector of {} values on {} is needed", name, cols, x.device)
    _need(t.dtype is x.dtype or t.dtype is torch.float32, "{}: float32 or the type of x ({}) is needed, not {}", name, x.dtype, t.dtype)


def layer_norm(x: torch.Tensor, weight=None, bias=None, eps: float = 1e-5):
    """Layer norm over the last dimension (``ones_layer_norm``): (y, mean, rstd), mean and rstd in float32 with x's
    leading dimensions.  weight and bias: None, or vectors of x's type or of float32 (both of one type)."""
    kind = _TYPES.get(x.dtype)
    _need(kind is not None and x.is_cuda and x.dim() >= 1, "x: a float32, bfloat16 or float16 CUDA tensor is needed")
    shape = x.shape
    cols = shape[-1]
    wkind = F32
    wp = bp = None
    if bias is not None:
        _param(bias, cols, x, "bias")
        wkind, bp = _TYPES[bias.dtype], bias.data_ptr()
    if weight is not None:
        _param(weight, cols, x, "weight")
        _need(bias is None or bias.dtype is weight.dtype, "weight and bias need one type")
        wkind, wp = _TYPES[weight.dtype], weight.data_ptr()
    if (other := _device(x, lambda: layer_norm(x, weight, bias, eps))) is not None:
        return other
    device = x.device
    p, ld = _rows(x)
    y = torch.empty(shape, dtype=x.dtype, device=device)
    mean = torch.empty(shape[:-1], dtype=torch.float32, device=device)
    rstd = torch.empty_like(mean)
    _done(lib().ones_layer_norm(p.data_ptr(), ld, wp, bp, p.shape[0], cols, eps, kind, wkind, y.data_ptr(), cols, mean.data_ptr(),
                                rstd.data_ptr(), _stream_of(device.index)), "ones_layer_norm")
    return y, mean, rstd


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, weight=None, *,
                        parameters: bool = True):
    """Gradients of `layer_norm` (``ones_layer_norm_backward``): (dx, dweight, dbias), the latter two in the type of
    weight (float32 where it is None), or None both with parameters=False."""
    kind = _TYPES.get(x.dtype)
    _need(kind is not None and x.is_cuda and x.dim() >= 1, "x: a float32, bfloat16 or float16 CUDA tensor is needed")
    _need(dy.shape == x.shape and dy.dtype is x.dtype and dy.device == x.device, "dy needs x's shape, type and device")
    cols = x.shape[-1]
    wt, wp = torch.float32, None
    if weight is not None:
        _param(weight, cols, x, "weight")
        wt, wp = weight.dtype, weight.data_ptr()
    for s in (mean, rstd):
        _need(s.dtype is torch.float32 and s.device == x.device and s.shape == x.shape[:-1] and s.is_contiguous(),
              "mean, rstd: what layer_norm returned is needed")
    if (other := _device(x, lambda: layer_norm_backward(dy, x, mean, rstd, weight, parameters=parameters))) is not None:
        return other
    device = x.device
    p, ld = _rows(x)
    q, ldq = _rows(dy)
    rows = p.shape[0]
    dx = torch.empty(x.shape, dtype=x.dtype, device=device)
    dw = db = dwp = dbp = sp = None
    nbytes = 0
    if parameters:
        dw = torch.empty(cols, dtype=wt, device=device)
        db = torch.empty_like(dw)
        nbytes = lib().ones_layer_norm_workspace_bytes(rows, cols)
        space = _space(nbytes, device)
        dwp, dbp, sp = dw.data_ptr(), db.data_ptr(), space.data_ptr()
    _done(lib().ones_layer_norm_backward(q.data_ptr(), ldq, p.data_ptr(), ld, mean.data_ptr(), rstd.data_ptr(), wp, rows, cols, kind,
                                         _TYPES[wt], dx.data_ptr(), cols, dwp, dbp, sp, nbytes, _stream_of(device.index)),
          "ones_layer_norm_backward")
    return dx, dw, db


def _ce_args(hidden, weight, target):
    _need(hidden.is_cuda and (hidden.dtype is torch.bfloat16 or hidden.dtype is torch.float16) and hidden.dim() >= 1,
          "hidden: a bfloat16 or float16 CUDA tensor is needed")
    _need(weight.dim() == 2 and weight.dtype is hidden.dtype and weight.device == hidden.device and
          weight.shape[1] == hidden.shape[-1], "weight: [vocab][cols] of hidden's type and device is needed")
    _need(target.dtype is torch.int64 and target.device == hidden.device and target.shape == hidden.shape[:-1],
          "target: int64 with hidden's leading dimensions is needed")


def linear_cross_entropy(hidden: torch.Tensor, weight: torch.Tensor, target: torch.Tensor):
    """Cross entropy of ``hidden @ weight.T`` at `target` without keeping the logits (``ones_linear_ce``): (loss, lse),
    float32 with hidden's leading dimensions.  Rows whose target is outside [0, vocab) have loss 0."""
    _ce_args(hidden, weight, target)
    if (other := _device(hidden, lambda: linear_cross_entropy(hidden, weight, target))) is not None:
        return other
    device = hidden.device
    h, ldh = _rows(hidden, 8)
    w, ldw = _rows(weight, 8)
    t = target.contiguous()
    rows, vocab = h.shape[0], weight.shape[0]
    loss = torch.empty(target.shape, dtype=torch.float32, device=device)
    lse = torch.empty_like(loss)
    nbytes = lib().ones_linear_ce_workspace_bytes(rows, vocab)
    space = _space(nbytes, device)
    _done(lib().ones_linear_ce(h.data_ptr(), ldh, w.data_ptr(), ldw, t.data_ptr(), rows, hidden.shape[-1], vocab,
                               _TYPES[hidden.dtype], loss.data_ptr(), lse.data_ptr(), space.data_ptr(), nbytes,
                               _stream_of(device.index)), "ones_linear_ce")
    return loss, lse


def linear_cross_entropy_backward(dloss: torch.Tensor, hidden: torch.Tensor, weight: torch.Tensor, target: torch.Tensor,
                                  lse: torch.Tensor, *, weight_gradient: torch.dtype | None = None, piece: int = 0):
    """Gradients of `linear_cross_entropy` for the gradient `dloss` of its loss (``ones_linear_ce_backward``):
    (dhidden, dweight).  weight_gradient: float32 for dweight in 32 bits (default: weight's type).  piece: entries of the
    vocabulary that are taken at a time (a multiple of 256; 0: the library's choice)."""
    _ce_args(hidden, weight, target)
    wt = weight_gradient or weight.dtype
    _need(wt is torch.float32 or wt is weight.dtype, "weight_gradient: float32 or weight's type is needed")
    for s in (dloss, lse):
        _need(s.dtype is torch.float32 and s.device == hidden.device and s.shape == target.shape,
              "dloss, lse: float32 with target's shape is needed")
    if (other := _device(hidden, lambda: linear_cross_entropy_backward(dloss, hidden, weight, target, lse,
                                                                       weight_gradient=weight_gradient, piece=piece))) is not None:
        return other
    device = hidden.device
    h, ldh = _rows(hidden)
    w, ldw = _rows(weight, 8)
    t, g, l = target.contiguous(), dloss.contiguous(), lse.contiguous()
    rows, cols, vocab = h.shape[0], hidden.shape[-1], weight.shape[0]
    dh = torch.empty(hidden.shape, dtype=hidden.dtype, device=device)
    dw = torch.empty(weight.shape, dtype=wt, device=device)
    nbytes = lib().ones_linear_ce_backward_workspace_bytes(rows, cols, vocab, piece)
    space = _space(nbytes, device)
    _done(lib().ones_linear_ce_backward(g.data_ptr(), h.data_ptr(), ldh, w.data_ptr(), ldw, t.data_ptr(), l.data_ptr(), rows, cols,
                                        vocab, _TYPES[hidden.dtype], _TYPES[wt], piece, dh.data_ptr(), cols, dw.data_ptr(), cols,
                                        space.data_ptr(), nbytes, _stream_of(device.index)), "ones_linear_ce_backward")
    return dh, dw


def orthogonalize(g: torch.Tensor, *, steps: int = 5, coefficients=(3.4445, -4.7750, 2.0315), eps: float = 1e-7) -> torch.Tensor:
    """Newton-Schulz orthogonalised update (``ones_orthogonalize``) of a matrix [m][n], or of several [count][m][n], in
    bfloat16."""
    kind = _TYPES.get(g.dtype)
    _need(kind is not None and g.is_cuda and g.dim() in (2, 3), "g: a float32, bfloat16 or float16 CUDA matrix is needed, or several")
    a, b, c = coefficients
    if (other := _device(g, lambda: orthogonalize(g, steps=steps, coefficients=coefficients, eps=eps))) is not None:
        return other
    device = g.device
    s = g if g.dim() == 3 else g[None]
    count, m, n = s.shape
    if (s.stride(2) != 1 and n > 1) or (s.stride(1) < n and m > 1):
        s = s.contiguous()
    out = torch.empty(g.shape, dtype=torch.bfloat16, device=device)
    if count * m * n == 0:
        return out
    nbytes = lib().ones_orthogonalize_workspace_bytes(count, m, n)
    if nbytes == 0:
        raise _b.OnesError(-3, "ones_orthogonalize_workspace_bytes")
    space = _space(nbytes, device)
    _done(lib().ones_orthogonalize(s.data_ptr(), s.stride(1) if m > 1 else n, s.stride(0), count, m, n, kind, steps, a, b, c, eps,
                                   out.data_ptr(), space.data_ptr(), nbytes, _stream_of(device.index)), "ones_orthogonalize")
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
