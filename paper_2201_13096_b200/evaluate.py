"""Thin ctypes binding of ``include/spdy_eval.h``: the operators around the search.

SPDY's search asks its caller for the calibration loss of a stitched model (Section 3.4), and the pruned model is tuned
against the dense one afterwards.  ``linear`` and ``layer_norm`` carry a block of such a model, ``token_logprobs`` scores it
(and takes the dense model's most probable tokens), ``distill_loss`` compares it with them; the ``..._backward`` and
``..._with_grad`` calls give the gradients.

Every call runs in the CUDA library on ``stream`` (default: torch's current stream of the tensors' device); PyTorch supplies
memory and streams.  Matrices are 2-D CUDA tensors with unit column stride and any row stride.  There is no CPU fallback.
"""
from __future__ import annotations

import contextlib
import ctypes
from typing import NamedTuple, Optional

from . import binding

EXPORTS = (
    "spdy_linear", "spdy_linear_workspace_bytes", "spdy_linear_check_status", "spdy_layer_norm", "spdy_layer_norm_backward",
    "spdy_layer_norm_backward_workspace_bytes", "spdy_token_logprobs", "spdy_token_logprobs_backward",
    "spdy_token_logprobs_with_grad", "spdy_distill_loss", "spdy_distill_loss_backward", "spdy_distill_loss_with_grad",
)
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
SPDY_TOP_MAX, SPDY_DISTILL_MAX = 128, 256

__all__ = ["TokenLogprobs", "DistillLoss", "linear", "linear_check_status", "layer_norm", "layer_norm_backward", "token_logprobs",
           "token_logprobs_backward", "token_logprobs_with_grad", "distill_loss", "distill_loss_backward",
           "distill_loss_with_grad"]


class TokenLogprobs(NamedTuple):
    """Per row: log probability of the given token, entropy, log of the sum of exponentials, and the alternatives."""

    logprob: object
    entropy: object
    lse: object
    top_ids: Optional[object] = None
    top_logprobs: Optional[object] = None


class DistillLoss(NamedTuple):
    """Per row: loss, log of the sum of exponentials over all ids, and over the ids outside the teacher's (``tail`` only)."""

    loss: object
    lse: object
    rest: Optional[object] = None


_lib = None


def _load():
    """The product library, whichever build ``binding`` has selected for the solver."""
    global _lib
    if _lib is None:
        lib = binding.open_library(binding.LIB_PATH)
        vp, i32, i64, f32, size, cint = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t,
                                         ctypes.c_int)
        rows = [vp, i64, cint, vp, cint]
        for name, result, args in (
            ("spdy_linear_workspace_bytes", size, [vp, i64, vp, i64, cint, i64, i64, i64]),
            ("spdy_linear", cint, [vp, i64, vp, i64, cint, vp, cint, vp, i64, cint, i64, i64, i64, vp, i64, cint, vp, size, vp]),
            ("spdy_linear_check_status", cint, [vp]),
            ("spdy_layer_norm", cint, [vp, i64, cint, vp, vp, cint, i64, i64, f32, vp, i64, vp, vp, vp]),
            ("spdy_layer_norm_backward_workspace_bytes", size, [i64, i64, cint]),
            ("spdy_layer_norm_backward", cint, [vp, i64, vp, i64, cint, vp, cint, vp, vp, i64, i64, vp, i64, vp, vp, vp, size, vp]),
            ("spdy_token_logprobs", cint, rows + [i64, i64, f32, i32, vp, vp, vp, vp, vp, vp]),
            ("spdy_token_logprobs_backward", cint, rows + [i64, i64, f32, vp, vp, vp, vp, vp, i64, vp]),
            ("spdy_token_logprobs_with_grad", cint, rows + [i64, i64, f32, vp, vp, vp, vp, vp, vp, i64, vp]),
            ("spdy_distill_loss", cint, rows + [vp, i64, i64, i32, f32, cint, vp, vp, vp, vp]),
            ("spdy_distill_loss_backward", cint, rows + [vp, i64, i64, i32, f32, cint, vp, vp, vp, vp, i64, vp]),
            ("spdy_distill_loss_with_grad", cint, rows + [vp, i64, i64, i32, f32, cint, vp, vp, vp, vp, vp, i64, vp]),
        ):
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = result, args
        _lib = lib
    return _lib


def library():
    """The loaded library with the evaluation entries typed (raises if it has not been built)."""
    return _load()


_TYPES = None


def _dtype(t, what: str) -> int:
    global _TYPES
    if _TYPES is None:
        import torch

        _TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
    code = _TYPES.get(t.dtype)
    if code is None:
        raise ValueError(f"{what} must be float32, bfloat16 or float16")
    return code


def _matrix(t, what: str, rows: Optional[int] = None, cols: Optional[int] = None, dtype=None, device=None) -> int:
    """Checks a 2-D CUDA tensor with unit column stride; its row stride in elements."""
    if not t.is_cuda or t.dim() != 2:
        raise ValueError(f"{what} must be a 2-D CUDA tensor")
    r, c = t.shape
    if (rows is not None and r != rows) or (cols is not None and c != cols):
        raise ValueError(f"{what} must be [{'*' if rows is None else rows}][{'*' if cols is None else cols}]")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{what} must be {dtype}")
    if device is not None and t.device != device:
        raise ValueError(f"{what} must be on {device}")
    s0, s1 = t.stride()
    if c > 1 and s1 != 1:
        raise ValueError(f"{what} must have unit column stride")
    if r <= 1:
        return c if s0 < c else s0
    if s0 < c:
        raise ValueError(f"{what} must not have overlapping rows")
    return s0


def _vector(t, what: str, n: int, device, dtype=None):
    if not t.is_cuda or t.dim() != 1 or t.shape[0] != n or t.device != device or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{what} must be a contiguous [{n}] tensor on {device}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{what} must be {dtype}")
    return t.data_ptr()


def _ids(t, what: str, shape, device) -> int:
    import torch

    if t.dtype not in (torch.int64, torch.int32):
        raise ValueError(f"{what} must be int32 or int64")
    if tuple(t.shape) != shape or t.device != device or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous {list(shape)} tensor on {device}")
    return 64 if t.dtype == torch.int64 else 32


class _Scope:
    """Current device and stream for the duration of a call: memory comes from the stream the work runs on."""

    def __init__(self, device, stream):
        import torch

        self._stack = None
        if torch.cuda.current_device() != device.index or stream is not None:
            self._stack = contextlib.ExitStack()
            self._stack.enter_context(torch.cuda.device(device))
            if stream is not None:
                if stream.device != device:
                    self._stack.close()
                    raise ValueError("the stream must be on the tensors' device")
                self._stack.enter_context(torch.cuda.stream(stream))
        self.handle = torch.cuda.current_stream().cuda_stream

    def __enter__(self):
        return self.handle

    def __exit__(self, *exc):
        if self._stack is not None:
            self._stack.close()


def _ptr(t):
    return None if t is None else t.data_ptr()


def _workspace(nbytes: int, device):
    import torch

    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def linear(x, weight, bias=None, residual=None, activation: str = "none", out=None, out_dtype=None, stream=None):
    """``spdy_linear``: ``act(x @ weight.T + bias) + residual``.

    ``x`` [M][K] and ``weight`` [N][K] bfloat16 or float16 (the same), ``bias`` [N] of that type or float32, ``residual``
    [M][N] of that type; ``activation`` one of "none", "relu", "gelu" (with erf), "silu".  The result is ``out`` if given,
    else a new tensor of ``out_dtype`` (default: ``x``'s type; float32 is the other choice).  ``out`` may be ``residual``."""
    import torch

    if activation not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {sorted(ACTIVATIONS)}")
    if x.dtype not in (torch.bfloat16, torch.float16):
        raise ValueError("x must be bfloat16 or float16")
    ldx = _matrix(x, "x")
    M, K = x.shape
    dev = x.device
    ldw = _matrix(weight, "weight", cols=K, dtype=x.dtype, device=dev)
    N = weight.shape[0]
    if bias is not None:
        _vector(bias, "bias", N, dev)
        if bias.dtype not in (x.dtype, torch.float32):
            raise ValueError("bias must have x's type or be float32")
    ldres = 0 if residual is None else _matrix(residual, "residual", M, N, x.dtype, dev)
    lib, code = _load(), _dtype(x, "x")
    with _Scope(dev, stream) as handle:
        if out is None:
            out = torch.empty((M, N), dtype=x.dtype if out_dtype is None else out_dtype, device=dev)
        elif out_dtype is not None and out.dtype != out_dtype:
            raise ValueError("out must have out_dtype")
        if out.dtype not in (x.dtype, torch.float32):
            raise ValueError("the result must have x's type or be float32")
        ldy = _matrix(out, "out", M, N, device=dev)
        px, pw = x.data_ptr(), weight.data_ptr()
        need = lib.spdy_linear_workspace_bytes(px, ldx, pw, ldw, code, M, N, K)
        ws = _workspace(need, dev)
        binding._check(lib.spdy_linear(px, ldx, pw, ldw, code, _ptr(bias), 0 if bias is None else _dtype(bias, "bias"),
                                       _ptr(residual), ldres, ACTIVATIONS[activation], M, N, K, out.data_ptr(), ldy,
                                       _dtype(out, "out"), _ptr(ws), need, handle), "spdy_linear")
    return out


def linear_check_status(stream=None):
    """``spdy_linear_check_status``: raises if a wait inside the linear kernels ever ran out of time (waits for the stream)."""
    binding._check(_load().spdy_linear_check_status(binding._stream_handle(stream)), "spdy_linear_check_status")


def _norm_params(x, weight, bias):
    import torch

    kind = None
    for name, p in (("weight", weight), ("bias", bias)):
        if p is None:
            continue
        _vector(p, name, x.shape[1], x.device)
        if p.dtype not in (x.dtype, torch.float32) or (kind is not None and p.dtype != kind):
            raise ValueError("weight and bias must both have x's type or both be float32")
        kind = p.dtype
    return 0 if kind is None else (0 if kind == torch.float32 else _dtype(x, "x"))


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, out=None, stream=None):
    """``spdy_layer_norm``: (y, mean, rstd) of ``x`` [R][D] (float32, bfloat16 or float16); ``weight`` and ``bias`` [D] of
    ``x``'s type or float32, or None.  ``mean`` and ``rstd`` [R] are float32.  ``out`` may be ``x``."""
    import torch

    code, ldx = _dtype(x, "x"), _matrix(x, "x")
    R, D = x.shape
    kind = _norm_params(x, weight, bias)
    lib = _load()
    with _Scope(x.device, stream) as handle:
        if out is None:
            out = torch.empty((R, D), dtype=x.dtype, device=x.device)
        ldy = _matrix(out, "out", R, D, x.dtype, x.device)
        stats = torch.empty((2, R), dtype=torch.float32, device=x.device)
        mean, rstd = stats.unbind(0)
        binding._check(lib.spdy_layer_norm(x.data_ptr(), ldx, code, _ptr(weight), _ptr(bias), kind, R, D, eps, out.data_ptr(), ldy,
                                           mean.data_ptr(), rstd.data_ptr(), handle), "spdy_layer_norm")
    return out, mean, rstd


def layer_norm_backward(dy, x, weight, mean, rstd, out=None, params: bool = True, stream=None):
    """``spdy_layer_norm_backward``: (dx, dweight, dbias) from the gradient ``dy`` [R][D] of ``layer_norm``'s result, its input
    ``x`` and its ``mean`` and ``rstd``.  ``dx`` has ``x``'s type, ``dweight`` and ``dbias`` [D] are float32 (None with
    ``params=False``).  ``out`` receives ``dx`` and may be ``dy`` or ``x``."""
    import torch

    code, ldx = _dtype(x, "x"), _matrix(x, "x")
    R, D = x.shape
    dev = x.device
    lddy = _matrix(dy, "dy", R, D, x.dtype, dev)
    kind = _norm_params(x, weight, None)
    pm, pr = _vector(mean, "mean", R, dev, torch.float32), _vector(rstd, "rstd", R, dev, torch.float32)
    lib = _load()
    with _Scope(dev, stream) as handle:
        if out is None:
            out = torch.empty((R, D), dtype=x.dtype, device=dev)
        lddx = _matrix(out, "out", R, D, x.dtype, dev)
        dw = db = ws = None
        need = 0
        if params:
            dw, db = torch.empty((2, D), dtype=torch.float32, device=dev).unbind(0)
            need = lib.spdy_layer_norm_backward_workspace_bytes(R, D, code)
            ws = _workspace(need, dev)
        binding._check(lib.spdy_layer_norm_backward(dy.data_ptr(), lddy, x.data_ptr(), ldx, code, _ptr(weight), kind, pm, pr, R, D,
                                                    out.data_ptr(), lddx, _ptr(dw), _ptr(db), _ptr(ws), need, handle),
                       "spdy_layer_norm_backward")
    return out, dw, db


def _logits(logits):
    code, ld = _dtype(logits, "logits"), _matrix(logits, "logits")
    return code, ld, logits.shape[0], logits.shape[1], logits.device


def _grads_out(out, logits, R, V, dev):
    import torch

    if out is None:
        out = torch.empty((R, V), dtype=logits.dtype, device=dev)
    return out, _matrix(out, "out", R, V, logits.dtype, dev)


def token_logprobs(logits, tokens, top_k: int = 0, temperature: float = 1.0, stream=None) -> TokenLogprobs:
    """``spdy_token_logprobs``: log probability of ``tokens`` [R] (int32 or int64; negative = none) under
    softmax(``logits`` [R][V] / ``temperature``), entropy and lse of each row, and with ``top_k`` > 0 the ids (int32) and log
    probabilities of its most probable ids, best first, equal logits by ascending id."""
    import torch

    code, ld, R, V, dev = _logits(logits)
    bits = _ids(tokens, "tokens", (R,), dev)
    top_k = int(top_k)
    lib = _load()
    with _Scope(dev, stream) as handle:
        logprob, entropy, lse = torch.empty((3, R), dtype=torch.float32, device=dev).unbind(0)
        ids = lps = None
        if top_k > 0:
            ids = torch.empty((R, top_k), dtype=torch.int32, device=dev)
            lps = torch.empty((R, top_k), dtype=torch.float32, device=dev)
        binding._check(lib.spdy_token_logprobs(logits.data_ptr(), ld, code, tokens.data_ptr(), bits, R, V, temperature, top_k,
                                               logprob.data_ptr(), entropy.data_ptr(), lse.data_ptr(), _ptr(ids), _ptr(lps),
                                               handle), "spdy_token_logprobs")
    return TokenLogprobs(logprob, entropy, lse, ids, lps)


def token_logprobs_backward(logits, tokens, lse, entropy=None, grad_logprob=None, grad_entropy=None, temperature: float = 1.0,
                            out=None, stream=None):
    """``spdy_token_logprobs_backward``: the gradient [R][V] (``logits``' type) of ``sum(grad_logprob * logprob + grad_entropy *
    entropy)``, from the forward call's ``lse`` and (with ``grad_entropy``) ``entropy``.  ``out`` may be ``logits``."""
    import torch

    code, ld, R, V, dev = _logits(logits)
    bits = _ids(tokens, "tokens", (R,), dev)
    for name, t in (("lse", lse), ("entropy", entropy), ("grad_logprob", grad_logprob), ("grad_entropy", grad_entropy)):
        if t is not None:
            _vector(t, name, R, dev, torch.float32)
    lib = _load()
    with _Scope(dev, stream) as handle:
        out, ldo = _grads_out(out, logits, R, V, dev)
        binding._check(lib.spdy_token_logprobs_backward(logits.data_ptr(), ld, code, tokens.data_ptr(), bits, R, V, temperature,
                                                        _ptr(lse), _ptr(entropy), _ptr(grad_logprob), _ptr(grad_entropy),
                                                        out.data_ptr(), ldo, handle), "spdy_token_logprobs_backward")
    return out


def token_logprobs_with_grad(logits, tokens, grad_logprob=None, grad_entropy=None, temperature: float = 1.0, out=None,
                             stream=None):
    """``spdy_token_logprobs_with_grad``: (``TokenLogprobs``, gradient) in one call, for a loss whose weights per row are known
    beforehand.  ``out`` receives the gradient and may be ``logits``."""
    import torch

    code, ld, R, V, dev = _logits(logits)
    bits = _ids(tokens, "tokens", (R,), dev)
    for name, t in (("grad_logprob", grad_logprob), ("grad_entropy", grad_entropy)):
        if t is not None:
            _vector(t, name, R, dev, torch.float32)
    lib = _load()
    with _Scope(dev, stream) as handle:
        out, ldo = _grads_out(out, logits, R, V, dev)
        logprob, entropy, lse = torch.empty((3, R), dtype=torch.float32, device=dev).unbind(0)
        binding._check(lib.spdy_token_logprobs_with_grad(logits.data_ptr(), ld, code, tokens.data_ptr(), bits, R, V, temperature,
                                                         _ptr(grad_logprob), _ptr(grad_entropy), logprob.data_ptr(),
                                                         entropy.data_ptr(), lse.data_ptr(), out.data_ptr(), ldo, handle),
                       "spdy_token_logprobs_with_grad")
    return TokenLogprobs(logprob, entropy, lse), out


def _teacher(top_ids, top_logprobs, R, dev):
    import torch

    if top_ids.dim() != 2:
        raise ValueError("top_ids must be [R][K]")
    K = top_ids.shape[1]
    bits = _ids(top_ids, "top_ids", (R, K), dev)
    if tuple(top_logprobs.shape) != (R, K) or top_logprobs.dtype != torch.float32 or top_logprobs.device != dev or not top_logprobs.is_contiguous():
        raise ValueError("top_logprobs must be a contiguous float32 tensor like top_ids")
    return bits, K


def distill_loss(logits, top_ids, top_logprobs, temperature: float = 1.0, tail: bool = True, stream=None) -> DistillLoss:
    """``spdy_distill_loss``: the divergence of softmax(``logits`` [R][V] / ``temperature``) from a teacher known by its top log
    probabilities [R][K] (float32, at the same temperature) at ``top_ids`` [R][K] (negative = no entry).  With ``tail`` the
    teacher's remaining mass is compared with the student's mass outside the ids; without, the teacher is renormalised over
    them.  Rows are not averaged."""
    import torch

    code, ld, R, V, dev = _logits(logits)
    bits, K = _teacher(top_ids, top_logprobs, R, dev)
    lib = _load()
    with _Scope(dev, stream) as handle:
        loss, lse, rest = torch.empty((3, R), dtype=torch.float32, device=dev).unbind(0)
        binding._check(lib.spdy_distill_loss(logits.data_ptr(), ld, code, top_ids.data_ptr(), bits, top_logprobs.data_ptr(), R, V, K,
                                             temperature, bool(tail), loss.data_ptr(), lse.data_ptr(),
                                             rest.data_ptr() if tail else None, handle), "spdy_distill_loss")
    return DistillLoss(loss, lse, rest if tail else None)


def distill_loss_backward(logits, top_ids, top_logprobs, lse, rest, grad_loss, temperature: float = 1.0, tail: bool = True,
                          out=None, stream=None):
    """``spdy_distill_loss_backward``: the gradient [R][V] (``logits``' type) of ``sum(grad_loss * loss)`` from the forward call's
    ``lse`` and ``rest`` (None without ``tail``).  ``out`` may be ``logits``."""
    import torch

    code, ld, R, V, dev = _logits(logits)
    bits, K = _teacher(top_ids, top_logprobs, R, dev)
    if tail and rest is None:
        raise ValueError("rest is needed with tail")
    for name, t in (("lse", lse), ("rest", rest if tail else None), ("grad_loss", grad_loss)):
        if t is not None:
            _vector(t, name, R, dev, torch.float32)
    lib = _load()
    with _Scope(dev, stream) as handle:
        out, ldo = _grads_out(out, logits, R, V, dev)
        binding._check(lib.spdy_distill_loss_backward(logits.data_ptr(), ld, code, top_ids.data_ptr(), bits, top_logprobs.data_ptr(), R,
                                                      V, K, temperature, bool(tail), _ptr(lse), _ptr(rest) if tail else None,
                                                      _ptr(grad_loss), out.data_ptr(), ldo, handle), "spdy_distill_loss_backward")
    return out


def distill_loss_with_grad(logits, top_ids, top_logprobs, grad_loss, temperature: float = 1.0, tail: bool = True, out=None,
                           stream=None):
    """``spdy_distill_loss_with_grad``: (``DistillLoss``, gradient) in one call.  ``out`` receives the gradient and may be
    ``logits``."""
    import torch

    code, ld, R, V, dev = _logits(logits)
    bits, K = _teacher(top_ids, top_logprobs, R, dev)
    _vector(grad_loss, "grad_loss", R, dev, torch.float32)
    lib = _load()
    with _Scope(dev, stream) as handle:
        out, ldo = _grads_out(out, logits, R, V, dev)
        loss, lse, rest = torch.empty((3, R), dtype=torch.float32, device=dev).unbind(0)
        binding._check(lib.spdy_distill_loss_with_grad(logits.data_ptr(), ld, code, top_ids.data_ptr(), bits, top_logprobs.data_ptr(),
                                                       R, V, K, temperature, bool(tail), grad_loss.data_ptr(), loss.data_ptr(),
                                                       lse.data_ptr(), rest.data_ptr() if tail else None, out.data_ptr(), ldo,
                                                       handle), "spdy_distill_loss_with_grad")
    return DistillLoss(loss, lse, rest if tail else None), out
