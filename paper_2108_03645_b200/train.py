"""Training-step operators: binding of ``ones_train.h`` and ``ones_attention.h``.

`lib()` is the C ABI through ctypes.  The functions below take torch tensors and go through ``_train_torch``, a small
compiled module that checks arguments, allocates outputs and workspaces and calls the same C ABI: small calls are bound
by the host, and the same marshalling in Python costs 9 us a call.

Layer norm, the cross entropy of a projection on a large vocabulary, norms of queries and keys with their rotation, causal
attention over packed sequences, all with their gradients, the orthogonalised update of matrix parameters and the clipping of
gradients, for CUDA tensors.  Work goes to torch's current stream of the tensors' device; outputs and
workspaces come from torch's allocator on that stream.  Nothing synchronises except `check`.

The functions take rows with any stride between them (a slice of a wider buffer is read in place).  Other layouts, and
for the cross entropy rows that do not start on 16-byte boundaries, are copied first.

Their results have no graph, so they refuse inputs that require a gradient while gradients are recorded, and tangents of
forward mode; `layer_norm_autograd`, `linear_cross_entropy_autograd`, `qk_norm_autograd` and `attention_autograd` are
differentiable, once.
"""
from __future__ import annotations

import ctypes as C

import torch
from torch.autograd.function import once_differentiable

from . import binding as _b

F32, BF16, F16 = 0, 1, 2  # ONES_F32, ONES_BF16, ONES_F16
MAX_NORM_COLS = 65536

_SIGNATURES = {
    "ones_layer_norm": (C.c_int, [C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_float, C.c_int32,
                                  C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p]),
    "ones_layer_norm_workspace_bytes": (C.c_size_t, [C.c_int32, C.c_int32]),
    "ones_layer_norm_backward": (C.c_int, [C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p,
                                           C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p,
                                           C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "ones_align_rows": (C.c_int, [C.c_void_p, C.c_int64, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p]),
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



class Heads(C.Structure):
    """``ones_heads``: vectors of a head for each token, strides in values."""
    _fields_ = [("data", C.c_void_p), ("token", C.c_int64), ("head", C.c_int64), ("heads", C.c_int32)]


_HEADS = C.POINTER(Heads)

_ATTENTION_SIGNATURES = {
    "ones_qk_norm": (C.c_int, [_HEADS, _HEADS, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32,
                               C.c_int32, C.c_float, C.c_int32, C.c_int32, _HEADS, _HEADS, C.c_void_p]),
    "ones_qk_norm_workspace_bytes": (C.c_size_t, [C.c_int32]),
    "ones_qk_norm_backward": (C.c_int, [_HEADS, _HEADS, _HEADS, _HEADS, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32,
                                        C.c_int32, C.c_int32, C.c_int32, C.c_float, C.c_int32, C.c_int32, _HEADS, _HEADS, C.c_void_p,
                                        C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "ones_attention_workspace_bytes": (C.c_size_t, [C.c_int32] * 4),
    "ones_attention": (C.c_int, [_HEADS, _HEADS, _HEADS, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_float, C.c_int32, _HEADS,
                                 C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "ones_attention_backward_workspace_bytes": (C.c_size_t, [C.c_int32] * 5),
    "ones_attention_backward": (C.c_int, [_HEADS, _HEADS, _HEADS, _HEADS, _HEADS, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32,
                                          C.c_int32, C.c_float, C.c_int32, _HEADS, _HEADS, _HEADS, C.c_void_p, C.c_size_t, C.c_void_p]),
    "ones_gradient_norm_workspace_bytes": (C.c_size_t, [C.c_int32]),
    "ones_gradient_norm": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "ones_clip_gradients": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_double, C.c_double, C.c_void_p,
                                      C.c_void_p, C.c_size_t, C.c_void_p]),
}

_lib = None


def lib() -> C.CDLL:
    """The loaded library; raises if it is missing (there is no fallback)."""
    global _lib
    if _lib is None:
        L = _b.lib()
        for name, (res, args) in (_SIGNATURES | _ATTENTION_SIGNATURES).items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


_ops = None


def _load():
    """The marshalling module; raises if it is missing (there is no fallback)."""
    global _ops
    if _ops is None:
        lib()
        try:
            from . import _train_torch
        except ImportError as e:
            raise ImportError("_train_torch.so is missing or does not fit this torch: run paper_2108_03645_b200/build.py") from e
        _ops = _train_torch
    return _ops


def _done(r, where: str):
    if type(r) is int:
        raise _b.OnesError(r, where)
    return r


def layer_norm(x: torch.Tensor, weight=None, bias=None, eps: float = 1e-5):
    """Layer norm over the last dimension (``ones_layer_norm``): (y, mean, rstd), mean and rstd in float32 with x's
    leading dimensions.  weight and bias: None, or vectors of x's type or of float32 (both of one type)."""
    return _done((_ops or _load()).layer_norm(x, weight, bias, eps), "ones_layer_norm")


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, weight=None, *,
                        parameters: bool = True):
    """Gradients of `layer_norm` (``ones_layer_norm_backward``): (dx, dweight, dbias), the latter two in the type of
    weight (float32 where it is None), or None both with parameters=False."""
    return _done((_ops or _load()).layer_norm_backward(dy, x, mean, rstd, weight, parameters), "ones_layer_norm_backward")


def linear_cross_entropy(hidden: torch.Tensor, weight: torch.Tensor, target: torch.Tensor):
    """Cross entropy of ``hidden @ weight.T`` at `target` without keeping the logits (``ones_linear_ce``): (loss, lse),
    float32 with hidden's leading dimensions.  Rows whose target is outside [0, vocab) have loss 0."""
    return _done((_ops or _load()).linear_cross_entropy(hidden, weight, target), "ones_linear_ce")


def linear_cross_entropy_backward(dloss: torch.Tensor, hidden: torch.Tensor, weight: torch.Tensor, target: torch.Tensor,
                                  lse: torch.Tensor, *, weight_gradient: torch.dtype | None = None, piece: int = 0):
    """Gradients of `linear_cross_entropy` for the gradient `dloss` of its loss (``ones_linear_ce_backward``):
    (dhidden, dweight).  weight_gradient: float32 for dweight in 32 bits (default: weight's type).  piece: entries of the
    vocabulary that are taken at a time (a multiple of 256; 0: the library's choice)."""
    if weight_gradient is not None and weight_gradient not in (torch.float32, weight.dtype):
        raise ValueError("weight_gradient: float32 or weight's type is needed")
    return _done((_ops or _load()).linear_cross_entropy_backward(dloss, hidden, weight, target, lse, weight_gradient is torch.float32, piece),
                 "ones_linear_ce_backward")


def orthogonalize(g: torch.Tensor, *, steps: int = 5, coefficients=(3.4445, -4.7750, 2.0315), eps: float = 1e-7) -> torch.Tensor:
    """Newton-Schulz orthogonalised update (``ones_orthogonalize``) of a matrix [m][n], or of several [count][m][n], in
    bfloat16."""
    a, b, c = coefficients
    return _done((_ops or _load()).orthogonalize(g, steps, a, b, c, eps), "ones_orthogonalize")


def qk_norm(q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor, frequencies: torch.Tensor, q_weight=None, k_weight=None, *,
            eps: float = 1e-6, interleaved: bool = False):
    """Root-mean-square norm of every head's query and key, and the rotation of its position (``ones_qk_norm``): (q, k), new
    tensors.  q, k [..][heads][dim]; positions int64 [..]; frequencies float64 (`rotary_frequencies`): the first twice as many
    values of a head turn, pairs being i and i + rotary / 2, or neighbours where interleaved.  Weights: None, or vectors of q's
    type or of float32."""
    return _done((_ops or _load()).qk_norm(q, k, positions, frequencies, q_weight, k_weight, eps, interleaved), "ones_qk_norm")


def qk_norm_backward(dq: torch.Tensor, dk: torch.Tensor, q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor,
                     frequencies: torch.Tensor, q_weight=None, k_weight=None, *, eps: float = 1e-6, interleaved: bool = False,
                     parameters: bool = True):
    """Gradients of `qk_norm` (``ones_qk_norm_backward``) for the gradients dq, dk of its results: (dq, dk, dq_weight, dk_weight),
    the latter two in the type of the weights (float32 where both are None), or None both with parameters=False."""
    return _done((_ops or _load()).qk_norm_backward(dq, dk, q, k, positions, frequencies, q_weight, k_weight, eps, interleaved, parameters),
                 "ones_qk_norm_backward")


def rotary_frequencies(rotary: int, base: float = 10000.0, *, device="cuda") -> torch.Tensor:
    """The frequencies base^(-2 i / rotary), i < rotary / 2, in float64, for `qk_norm`."""
    if rotary < 0 or rotary % 2:
        raise ValueError("rotary: an even number of values is needed")
    return base ** (torch.arange(rotary // 2, dtype=torch.float64, device=device) * (-2.0 / max(rotary, 1)))


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, offsets=None, *, scale: float | None = None):
    """Causal attention (``ones_attention``): (out, lse), out with q's shape, lse float32 without its last dimension.
    q [tokens][heads][dim], k and v [tokens][kv heads][dim] with the sequences packed one behind the other, bounds in `offsets`
    (int64, on the device; None: one sequence), or all [batch][tokens][..] without offsets.  scale: None for 1 / sqrt(dim).
    Tokens of no sequence have out = 0 and lse = 0."""
    return _done((_ops or _load()).attention(q, k, v, offsets, scale), "ones_attention")


def attention_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, lse: torch.Tensor,
                       offsets=None, *, scale: float | None = None):
    """Gradients of `attention` (``ones_attention_backward``) for the gradient dout of out: (dq, dk, dv)."""
    return _done((_ops or _load()).attention_backward(dout, q, k, v, out, lse, offsets, scale), "ones_attention_backward")


def gradient_norm(gradients) -> torch.Tensor:
    """Euclidean norm of all values of a list of tensors (``ones_gradient_norm``): float32, 0-d, on the device."""
    return _done((_ops or _load()).clip(list(gradients), None, None, 0.0), "ones_gradient_norm")


def clip_gradients(gradients, max_norm: float, *, out=None, eps: float = 1e-6) -> torch.Tensor:
    """Scales all gradients by min(1, max_norm / (norm + eps)) (``ones_clip_gradients``), in place or into the tensors `out` (of the
    same shapes, strides and types); returns the norm before, float32, 0-d.  Nothing synchronises."""
    return _done((_ops or _load()).clip(list(gradients), None if out is None else list(out), max_norm, eps), "ones_clip_gradients")


def check(device=None) -> None:
    """Waits for the current stream of `device` (None: the current one) and raises if a kernel on it gave up waiting since the
    last check (``ones_train_status``). Such a kernel's results are void, and nothing else says so: a program calls this before it
    trusts what it computed, at a step that it waits for anyway."""
    with torch.cuda.device(device):
        rc = lib().ones_train_status(torch.cuda.current_stream().cuda_stream)
    if rc:
        raise _b.OnesError(rc, "ones_train_status")


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        y, mean, rstd = layer_norm(x, weight, bias, eps)
        ctx.save_for_backward(x, weight, mean, rstd)
        ctx.has_bias = bias is not None
        return y

    @staticmethod
    @once_differentiable
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
    @once_differentiable
    def backward(ctx, dloss):
        hidden, weight, target, lse = ctx.saved_tensors
        return (*linear_cross_entropy_backward(dloss, hidden, weight, target, lse), None)


class _QkNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, positions, frequencies, q_weight, k_weight, eps, interleaved):
        ctx.save_for_backward(q, k, positions, frequencies, q_weight, k_weight)
        ctx.form = (eps, interleaved)
        return qk_norm(q, k, positions, frequencies, q_weight, k_weight, eps=eps, interleaved=interleaved)

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk):
        q, k, positions, frequencies, q_weight, k_weight = ctx.saved_tensors
        eps, interleaved = ctx.form
        dq, dk, dqw, dkw = qk_norm_backward(dq, dk, q, k, positions, frequencies, q_weight, k_weight, eps=eps, interleaved=interleaved,
                                            parameters=q_weight is not None or k_weight is not None)
        return dq, dk, None, None, dqw if q_weight is not None else None, dkw if k_weight is not None else None, None, None


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, offsets, scale):
        out, lse = attention(q, k, v, offsets, scale=scale)
        ctx.save_for_backward(q, k, v, out, lse, offsets)
        ctx.scale = scale
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        q, k, v, out, lse, offsets = ctx.saved_tensors
        return (*attention_backward(dout, q, k, v, out, lse, offsets, scale=ctx.scale), None, None)


def layer_norm_autograd(x, weight=None, bias=None, eps: float = 1e-5) -> torch.Tensor:
    """`layer_norm` as a (once) differentiable function of x, weight and bias: y."""
    return _LayerNorm.apply(x, weight, bias, eps)


def linear_cross_entropy_autograd(hidden, weight, target) -> torch.Tensor:
    """`linear_cross_entropy` as a (once) differentiable function of hidden and weight: the loss of each row."""
    return _LinearCrossEntropy.apply(hidden, weight, target)


def qk_norm_autograd(q, k, positions, frequencies, q_weight=None, k_weight=None, *, eps: float = 1e-6, interleaved: bool = False):
    """`qk_norm` as a (once) differentiable function of q, k and the weights: (q, k). Frequencies that require a gradient are refused: they
    get none."""
    if frequencies.requires_grad and torch.is_grad_enabled():
        raise ValueError("frequencies require a gradient, but qk_norm_autograd has none for them: detach them, or call it under torch.no_grad()")
    return _QkNorm.apply(q, k, positions, frequencies, q_weight, k_weight, eps, interleaved)


def attention_autograd(q, k, v, offsets=None, *, scale: float | None = None) -> torch.Tensor:
    """`attention` as a (once) differentiable function of q, k and v: out."""
    return _Attention.apply(q, k, v, offsets, scale)
