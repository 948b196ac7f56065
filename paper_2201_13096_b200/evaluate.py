"""Thin ctypes binding of ``include/spdy_eval.h``: the operators around the search.

SPDY's search asks its caller for the calibration loss of a stitched model (Section 3.4), and the pruned model is tuned
against the dense one afterwards.  ``linear`` and ``layer_norm`` carry a block of such a model, ``token_logprobs`` scores it
(and takes the dense model's most probable tokens), ``distill_loss`` compares it with them; ``linear_token_logprobs`` scores
an output layer without a table of logits.  The ``..._backward`` and ``..._with_grad`` calls give the gradients of the losses,
of ``layer_norm`` and of that output layer (``linear`` has no backward call: its input's gradient is ``linear`` with the weight
transposed, its weight's is not here), and ``adamw_step`` applies gradients to any number of tensors.

Every call runs in the CUDA library on ``stream`` (default: torch's current stream of the tensors' device); PyTorch supplies
memory and streams.  Matrices are 2-D CUDA tensors with unit column stride and any row stride.  There is no CPU fallback.
Nothing is recorded for autograd: with gradients enabled, tensors that require one are refused (detach them, and take the
gradient from the ``..._backward`` and ``..._with_grad`` calls; ``AdamW`` takes leaves, and changes them in place).  Tensors that a call
writes (``out`` and the like, what ``AdamW`` steps) get a new version, so that a graph that saved one raises, as it does for torch's own
operations in place.
"""
from __future__ import annotations

import contextlib
import ctypes
from typing import NamedTuple, Optional

import numpy as np

from . import binding

EXPORTS = (
    "spdy_linear", "spdy_linear_workspace_bytes", "spdy_linear_check_status", "spdy_layer_norm", "spdy_layer_norm_backward",
    "spdy_layer_norm_backward_workspace_bytes", "spdy_token_logprobs", "spdy_token_logprobs_backward",
    "spdy_token_logprobs_with_grad", "spdy_linear_token_logprobs", "spdy_linear_token_logprobs_backward",
    "spdy_linear_token_logprobs_with_grad", "spdy_linear_token_logprobs_workspace_bytes", "spdy_distill_loss", "spdy_distill_loss_backward", "spdy_distill_loss_with_grad",
    "spdy_adamw_step", "spdy_adamw_moments",
)
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
SPDY_TOP_MAX, SPDY_DISTILL_MAX = 128, 256

__all__ = ["TokenLogprobs", "LinearGrads", "DistillLoss", "linear", "linear_check_status", "layer_norm", "layer_norm_backward", "token_logprobs",
           "token_logprobs_backward", "token_logprobs_with_grad", "linear_token_logprobs", "linear_token_logprobs_backward",
           "linear_token_logprobs_with_grad", "distill_loss", "distill_loss_backward",
           "distill_loss_with_grad", "AdamW", "AdamWMoments", "adamw_step", "adamw_moments"]


class TokenLogprobs(NamedTuple):
    """Per row: log probability of the given token, entropy, log of the sum of exponentials, and the alternatives."""

    logprob: object
    entropy: object
    lse: object
    top_ids: Optional[object] = None
    top_logprobs: Optional[object] = None


class LinearGrads(NamedTuple):
    """Gradients by a linear layer's input, weight and bias; None where they were not asked for."""

    dhidden: object
    dweight: object
    dbias: Optional[object] = None


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
        _import_torch()
        lib = binding.open_library(binding.LIB_PATH)
        vp, i32, i64, f32, size, cint = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t,
                                         ctypes.c_int)
        rows = [vp, i64, cint, vp, cint]
        head = [vp, i64, vp, i64, cint, vp, cint, vp, cint, i64, i64, i64, f32]
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
            ("spdy_linear_token_logprobs_workspace_bytes", size, [vp, i64, vp, i64, cint, i64, i64, i64, cint, cint]),
            ("spdy_linear_token_logprobs", cint, head + [vp, vp, vp, vp, size, vp]),
            ("spdy_linear_token_logprobs_backward", cint, head + [vp, vp, vp, vp, vp, i64, vp, i64, vp, vp, size, vp]),
            ("spdy_linear_token_logprobs_with_grad", cint, head + [vp, vp, vp, vp, vp, vp, i64, vp, i64, vp, vp, size, vp]),
            ("spdy_distill_loss", cint, rows + [vp, i64, i64, i32, f32, cint, vp, vp, vp, vp]),
            ("spdy_distill_loss_backward", cint, rows + [vp, i64, i64, i32, f32, cint, vp, vp, vp, vp, i64, vp]),
            ("spdy_adamw_step", cint, [vp, i32, vp, vp]),
            ("spdy_adamw_moments", cint, [vp, i32, vp, vp, cint, vp]),
            ("spdy_distill_loss_with_grad", cint, rows + [vp, i64, i64, i32, f32, cint, vp, vp, vp, vp, vp, i64, vp]),
        ):
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = result, args
        _lib = lib
    return _lib


def library():
    """The loaded library with the evaluation entries typed (raises if it has not been built)."""
    return _load()


# PyTorch, imported with the library (the package itself imports without it).
torch = None
_TYPES = {}
_current_stream = _current_device = _empty_strided = _new_versions = None


def _checked(fast, plain, same):
    """``fast`` if it is there and ``same(fast, plain)``, else ``plain``: an entry of torch without a promise is used only as far as
    it answers like the public one."""
    try:
        return fast if fast is not None and same(fast, plain) else plain
    except Exception:
        return plain


def _same_memory(fast, plain):
    a, b = fast((2, 3), (4, 1), torch.float16), plain((2, 3), (4, 1), torch.float16)
    return all(f(a) == f(b) for f in (type, lambda t: t.shape, lambda t: t.stride(), lambda t: t.dtype, lambda t: t.device, lambda t: t.requires_grad))


def _same_versions(fast, plain):
    a, b = torch.zeros(2), torch.zeros(2)
    fast([a, b]), plain([b])
    return a._version == 1 and b._version == 2


def _import_torch():
    global torch, _current_stream, _current_device, _empty_strided, _new_versions
    import torch as t

    torch = t
    _TYPES.update({t.float32: 0, t.bfloat16: 1, t.float16: 2})
    # Small calls are bound by the host: the handle of the current stream as a number, without an object around it, and
    # uninitialised memory on the current device by (shape, strides, type), without the general call's argument parsing.
    _current_stream, _current_device = lambda i: t.cuda.current_stream(i).cuda_stream, t.cuda.current_device
    _empty_strided = lambda shape, strides, dtype: t.empty_strided(shape, strides, dtype=dtype, device="cuda")  # noqa: E731
    # A list of tensors that have been changed in place, without a test of what it is.
    _new_versions = _checked(getattr(t._C, "_increment_version", None), t.autograd.graph.increment_version, _same_versions)
    if t.cuda.is_available():
        _current_device = _checked(getattr(t._C, "_cuda_getDevice", None), _current_device, lambda f, p: f() == p())
        _current_stream = _checked(getattr(t._C, "_cuda_getCurrentRawStream", None), _current_stream, lambda f, p: f(_current_device()) == p(_current_device()))
        guards = getattr(getattr(t._C, "_dynamo", None), "guards", None)
        _empty_strided = _checked(getattr(guards, "_empty_strided_cuda", None), _empty_strided, _same_memory)


def _matrix(rows: int, cols: int, dtype):
    return _empty_strided((rows, cols), (cols, 1), dtype)


def _vectors(count: int, n: int):
    """``count`` float32 vectors of ``n``."""
    f32 = torch.float32
    return [_empty_strided((n,), (1,), f32) for _ in range(count)]


def _dtype(t, what: str) -> int:
    code = _TYPES.get(t.dtype)
    if code is None:
        raise ValueError(f"{what} must be float32, bfloat16 or float16")
    return code


def _refuse_gradient(what: str):
    if torch.is_grad_enabled():
        raise ValueError(f"{what} requires a gradient, which this call does not record: pass {what}.detach() or call under torch.no_grad()")


def _rows(t, what: str):
    """(rows, columns, row stride in elements, device index) of a 2-D CUDA tensor with unit column stride."""
    if t.requires_grad:
        _refuse_gradient(what)
    if not t.is_cuda or t.ndim != 2:
        raise ValueError(f"{what} must be a 2-D CUDA tensor")
    (r, c), (s0, s1) = t.shape, t.stride()
    if s1 != 1 and c > 1:
        raise ValueError(f"{what} must have unit column stride")
    if s0 < c:
        if r > 1:
            raise ValueError(f"{what} must not have overlapping rows")
        s0 = c
    return r, c, s0, t.get_device()


def _like(t, what: str, rows: int, cols: int, dtype, device: int) -> int:
    """The row stride of a matrix that has to have this shape, type and device."""
    r, c, ld, dev = _rows(t, what)
    if r != rows or c != cols or dev != device or t.dtype != dtype:
        raise ValueError(f"{what} must be [{rows}][{cols}] of {dtype} on cuda:{device}")
    return ld


def _out(t, what: str, rows: int, cols: int, dtype, device: int) -> int:
    """The same of a matrix that the caller gives to be written: a graph that saved it before must notice."""
    ld = _like(t, what, rows, cols, dtype, device)
    if not t.is_inference():
        _new_versions([t])
    return ld


def _vector(t, what: str, n: int, device: int, dtype=None):
    if t.requires_grad:
        _refuse_gradient(what)
    if t.ndim != 1 or t.shape[0] != n or t.get_device() != device or (n > 1 and not t.is_contiguous()):
        raise ValueError(f"{what} must be a contiguous [{n}] tensor on cuda:{device}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{what} must be {dtype}")
    return t.data_ptr()


def _ids(t, what: str, shape, device: int) -> int:
    bits = 64 if t.dtype == torch.int64 else 32 if t.dtype == torch.int32 else 0
    if not bits:
        raise ValueError(f"{what} must be int32 or int64")
    if t.shape != shape or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous {list(shape)} tensor on cuda:{device}")
    return bits


class _Scope:
    """Current device and stream for the duration of a call: memory comes from the stream the work runs on."""

    __slots__ = ("_stack", "handle")

    def __init__(self, device: int, stream):
        self._stack = None
        if stream is not None or _current_device() != device:
            if stream is not None and stream.device_index != device:
                raise ValueError("the stream must be on the tensors' device")
            self._stack = contextlib.ExitStack()
            self._stack.enter_context(torch.cuda.device(device) if stream is None else torch.cuda.stream(stream))
        self.handle = _current_stream(device)

    def __enter__(self):
        return self.handle

    def __exit__(self, *exc):
        if self._stack is not None:
            self._stack.close()


def _ptr(t):
    return None if t is None else t.data_ptr()


def linear(x, weight, bias=None, residual=None, activation: str = "none", out=None, out_dtype=None, stream=None):
    """``spdy_linear``: ``act(x @ weight.T + bias) + residual``.

    ``x`` [M][K] and ``weight`` [N][K] bfloat16 or float16 (the same), ``bias`` [N] of that type or float32, ``residual``
    [M][N] of that type; ``activation`` one of "none", "relu", "gelu" (with erf), "silu".  The result is ``out`` if given,
    else a new tensor of ``out_dtype`` (default: ``x``'s type; float32 is the other choice).  ``out`` may be ``residual``."""
    lib = _lib or _load()
    act = ACTIVATIONS.get(activation)
    if act is None:
        raise ValueError(f"activation must be one of {sorted(ACTIVATIONS)}")
    dtype = x.dtype
    code = _TYPES.get(dtype, 0)
    if not code:
        raise ValueError("x must be bfloat16 or float16")
    M, K, ldx, dev = _rows(x, "x")
    N, k, ldw, wdev = _rows(weight, "weight")
    if k != K or wdev != dev or weight.dtype != dtype:
        raise ValueError(f"weight must be [N][{K}] of {dtype} on cuda:{dev}")
    pb, bcode, pr, ldres = None, 0, None, 0
    if bias is not None:
        pb, bcode = _vector(bias, "bias", N, dev), _TYPES.get(bias.dtype, -1)
        if bcode and bcode != code:
            raise ValueError("bias must have x's type or be float32")
    if residual is not None:
        pr, ldres = residual.data_ptr(), _like(residual, "residual", M, N, dtype, dev)
    with _Scope(dev, stream) as handle:
        if out is None:
            out = _matrix(M, N, dtype if out_dtype is None else out_dtype)
            ldy = N
        else:
            if out_dtype is not None and out.dtype != out_dtype:
                raise ValueError("out must have out_dtype")
            ldy = _out(out, "out", M, N, out.dtype, dev)
        ocode = _TYPES.get(out.dtype, -1)
        if ocode and ocode != code:
            raise ValueError("the result must have x's type or be float32")
        px, pw = x.data_ptr(), weight.data_ptr()
        pws, need = None, 0
        if (px | pw | ldx * 2 | ldw * 2) & 15:
            need = lib.spdy_linear_workspace_bytes(px, ldx, pw, ldw, code, M, N, K)
            if need:
                ws = _empty_strided((need,), (1,), torch.uint8)
                pws = ws.data_ptr()
        rc = lib.spdy_linear(px, ldx, pw, ldw, code, pb, bcode, pr, ldres, act, M, N, K, out.data_ptr(), ldy, ocode, pws, need, handle)
    if rc:
        binding._check(rc, "spdy_linear")
    return out


def linear_check_status(stream=None):
    """``spdy_linear_check_status``: raises if a wait inside the linear kernels ever ran out of time (waits for the stream)."""
    binding._check(_load().spdy_linear_check_status(binding._stream_handle(stream)), "spdy_linear_check_status")


def _norm_params(x, weight, bias, D, dev, code):
    kind = None
    for name, p in (("weight", weight), ("bias", bias)):
        if p is None:
            continue
        _vector(p, name, D, dev)
        c = _TYPES.get(p.dtype, -1)
        if (c and c != code) or (kind is not None and c != kind):
            raise ValueError("weight and bias must both have x's type or both be float32")
        kind = c
    return kind or 0


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, out=None, stream=None):
    """``spdy_layer_norm``: (y, mean, rstd) of ``x`` [R][D] (float32, bfloat16 or float16); ``weight`` and ``bias`` [D] of
    ``x``'s type or float32, or None.  ``mean`` and ``rstd`` [R] are float32.  ``out`` may be ``x``."""
    lib = _lib or _load()
    R, D, ldx, dev = _rows(x, "x")
    code = _dtype(x, "x")
    kind = _norm_params(x, weight, bias, D, dev, code)
    with _Scope(dev, stream) as handle:
        if out is None:
            out, ldy = _matrix(R, D, x.dtype), D
        else:
            ldy = _out(out, "out", R, D, x.dtype, dev)
        mean, rstd = _vectors(2, R)
        rc = lib.spdy_layer_norm(x.data_ptr(), ldx, code, _ptr(weight), _ptr(bias), kind, R, D, eps, out.data_ptr(), ldy,
                                 mean.data_ptr(), rstd.data_ptr(), handle)
    if rc:
        binding._check(rc, "spdy_layer_norm")
    return out, mean, rstd


def layer_norm_backward(dy, x, weight, mean, rstd, out=None, params: bool = True, stream=None):
    """``spdy_layer_norm_backward``: (dx, dweight, dbias) from the gradient ``dy`` [R][D] of ``layer_norm``'s result, its input
    ``x`` and its ``mean`` and ``rstd``.  ``dx`` has ``x``'s type, ``dweight`` and ``dbias`` [D] are float32 (None with
    ``params=False``).  ``out`` receives ``dx`` and may be ``dy`` or ``x``."""
    lib = _lib or _load()
    R, D, ldx, dev = _rows(x, "x")
    code = _dtype(x, "x")
    lddy = _like(dy, "dy", R, D, x.dtype, dev)
    kind = _norm_params(x, weight, None, D, dev, code)
    pm, pr = _vector(mean, "mean", R, dev, torch.float32), _vector(rstd, "rstd", R, dev, torch.float32)
    with _Scope(dev, stream) as handle:
        if out is None:
            out, lddx = _matrix(R, D, x.dtype), D
        else:
            lddx = _out(out, "out", R, D, x.dtype, dev)
        dw = db = pw = pb = pws = None
        need = 0
        if params:
            dw, db = _vectors(2, D)
            pw, pb = dw.data_ptr(), db.data_ptr()
            need = lib.spdy_layer_norm_backward_workspace_bytes(R, D, code)
            if need:
                ws = _empty_strided((need,), (1,), torch.uint8)
                pws = ws.data_ptr()
        rc = lib.spdy_layer_norm_backward(dy.data_ptr(), lddy, x.data_ptr(), ldx, code, _ptr(weight), kind, pm, pr, R, D, out.data_ptr(),
                                          lddx, pw, pb, pws, need, handle)
    if rc:
        binding._check(rc, "spdy_layer_norm_backward")
    return out, dw, db


def _logits(logits):
    """(pointer, row stride, type) as the C calls take them, and (rows, columns, device index)."""
    R, V, ld, dev = _rows(logits, "logits")
    return (logits.data_ptr(), ld, _dtype(logits, "logits")), R, V, dev


def _grads_out(out, logits, R, V, dev):
    if out is None:
        return _matrix(R, V, logits.dtype), V
    return out, _out(out, "out", R, V, logits.dtype, dev)


def _optional(R, dev, **vectors):
    return [None if t is None else _vector(t, name, R, dev, torch.float32) for name, t in vectors.items()]


def token_logprobs(logits, tokens, top_k: int = 0, temperature: float = 1.0, stream=None) -> TokenLogprobs:
    """``spdy_token_logprobs``: log probability of ``tokens`` [R] (int32 or int64; negative = none) under
    softmax(``logits`` [R][V] / ``temperature``), entropy and lse of each row, and with ``top_k`` > 0 the ids (int32) and log
    probabilities of its most probable ids, best first, equal logits by ascending id."""
    lib = _lib or _load()
    head, R, V, dev = _logits(logits)
    bits = _ids(tokens, "tokens", (R,), dev)
    top_k = int(top_k)
    with _Scope(dev, stream) as handle:
        logprob, entropy, lse = _vectors(3, R)
        ids = lps = pi = pl = None
        if top_k > 0:
            ids, lps = _matrix(R, top_k, torch.int32), _matrix(R, top_k, torch.float32)
            pi, pl = ids.data_ptr(), lps.data_ptr()
        rc = lib.spdy_token_logprobs(*head, tokens.data_ptr(), bits, R, V, temperature, top_k, logprob.data_ptr(), entropy.data_ptr(),
                                     lse.data_ptr(), pi, pl, handle)
    if rc:
        binding._check(rc, "spdy_token_logprobs")
    return TokenLogprobs(logprob, entropy, lse, ids, lps)


def token_logprobs_backward(logits, tokens, lse, entropy=None, grad_logprob=None, grad_entropy=None, temperature: float = 1.0,
                            out=None, stream=None):
    """``spdy_token_logprobs_backward``: the gradient [R][V] (``logits``' type) of ``sum(grad_logprob * logprob + grad_entropy *
    entropy)``, from the forward call's ``lse`` and (with ``grad_entropy``) ``entropy``.  ``out`` may be ``logits``."""
    lib = _lib or _load()
    head, R, V, dev = _logits(logits)
    bits = _ids(tokens, "tokens", (R,), dev)
    vectors = _optional(R, dev, lse=lse, entropy=entropy, grad_logprob=grad_logprob, grad_entropy=grad_entropy)
    with _Scope(dev, stream) as handle:
        out, ldo = _grads_out(out, logits, R, V, dev)
        rc = lib.spdy_token_logprobs_backward(*head, tokens.data_ptr(), bits, R, V, temperature, *vectors, out.data_ptr(), ldo, handle)
    if rc:
        binding._check(rc, "spdy_token_logprobs_backward")
    return out


def token_logprobs_with_grad(logits, tokens, grad_logprob=None, grad_entropy=None, temperature: float = 1.0, out=None,
                             stream=None):
    """``spdy_token_logprobs_with_grad``: (``TokenLogprobs``, gradient) in one call, for a loss whose weights per row are known
    beforehand.  ``out`` receives the gradient and may be ``logits``."""
    lib = _lib or _load()
    head, R, V, dev = _logits(logits)
    bits = _ids(tokens, "tokens", (R,), dev)
    vectors = _optional(R, dev, grad_logprob=grad_logprob, grad_entropy=grad_entropy)
    with _Scope(dev, stream) as handle:
        out, ldo = _grads_out(out, logits, R, V, dev)
        logprob, entropy, lse = _vectors(3, R)
        rc = lib.spdy_token_logprobs_with_grad(*head, tokens.data_ptr(), bits, R, V, temperature, *vectors, logprob.data_ptr(),
                                               entropy.data_ptr(), lse.data_ptr(), out.data_ptr(), ldo, handle)
    if rc:
        binding._check(rc, "spdy_token_logprobs_with_grad")
    return TokenLogprobs(logprob, entropy, lse), out


def _head(hidden, weight, tokens, bias, temperature):
    """The C calls' common arguments, and what the outputs are made from: rows, ids, width, device and the workspace query's share."""
    dtype = hidden.dtype
    code = _TYPES.get(dtype, 0)
    if not code:
        raise ValueError("hidden must be bfloat16 or float16")
    R, D, ldh, dev = _rows(hidden, "hidden")
    V, d, ldw, wdev = _rows(weight, "weight")
    if d != D or wdev != dev or weight.dtype != dtype:
        raise ValueError(f"weight must be [V][{D}] of {dtype} on cuda:{dev}")
    pb, bcode = None, 0
    if bias is not None:
        pb, bcode = _vector(bias, "bias", V, dev), _TYPES.get(bias.dtype, -1)
        if bcode and bcode != code:
            raise ValueError("bias must have hidden's type or be float32")
    bits = _ids(tokens, "tokens", (R,), dev)
    query = (hidden.data_ptr(), ldh, weight.data_ptr(), ldw, code)
    return (*query, pb, bcode, tokens.data_ptr(), bits, R, V, D, temperature), R, V, D, dev, query


def _head_workspace(lib, query, R, V, D, forward, gradients):
    need = lib.spdy_linear_token_logprobs_workspace_bytes(*query, R, V, D, forward, gradients)
    ws = _empty_strided((need,), (1,), torch.uint8) if need else None
    return _ptr(ws), need, ws


def _head_grads(hidden, weight, bias, R, V, D, dev, wanted, dhidden, dweight):
    """``LinearGrads`` to write, and the C calls' arguments for them."""
    unknown = set(wanted) - {"hidden", "weight", "bias"}
    if unknown:
        raise ValueError(f"wanted names hidden, weight and bias, not {sorted(unknown)}")
    if (dhidden is not None and "hidden" not in wanted) or (dweight is not None and "weight" not in wanted):
        raise ValueError("a gradient's tensor is given, and the gradient is not wanted")
    ldh = ldw = D
    if "hidden" in wanted:
        if dhidden is None:
            dhidden = _matrix(R, D, hidden.dtype)
        else:
            ldh = _out(dhidden, "dhidden", R, D, hidden.dtype, dev)
    if "weight" in wanted:
        if dweight is None:
            dweight = _matrix(V, D, hidden.dtype)
        else:
            ldw = _out(dweight, "dweight", V, D, hidden.dtype, dev)
    dbias = _vectors(1, V)[0] if "bias" in wanted and bias is not None else None
    return LinearGrads(dhidden, dweight, dbias), (_ptr(dhidden), ldh, _ptr(dweight), ldw, _ptr(dbias))


def linear_token_logprobs(hidden, weight, tokens, bias=None, temperature: float = 1.0, stream=None) -> TokenLogprobs:
    """``spdy_linear_token_logprobs``: ``token_logprobs(hidden @ weight.T + bias, tokens)`` without the table of logits.

    ``hidden`` [R][D] and ``weight`` [V][D] bfloat16 or float16 (the same), ``bias`` [V] of that type or float32 (-inf: id not
    allowed), ``tokens`` [R] int32 or int64 (negative = none).  ``logprob``, ``entropy`` and ``lse`` [R] are float32."""
    lib = _lib or _load()
    head, R, V, D, dev, query = _head(hidden, weight, tokens, bias, temperature)
    with _Scope(dev, stream) as handle:
        logprob, entropy, lse = _vectors(3, R)
        pws, need, ws = _head_workspace(lib, query, R, V, D, 1, 0)
        rc = lib.spdy_linear_token_logprobs(*head, logprob.data_ptr(), entropy.data_ptr(), lse.data_ptr(), pws, need, handle)
    if rc:
        binding._check(rc, "spdy_linear_token_logprobs")
    return TokenLogprobs(logprob, entropy, lse)


def linear_token_logprobs_backward(hidden, weight, tokens, lse, entropy=None, grad_logprob=None, grad_entropy=None, bias=None,
                                   temperature: float = 1.0, wanted=("hidden", "weight", "bias"), dhidden=None, dweight=None,
                                   stream=None) -> LinearGrads:
    """``spdy_linear_token_logprobs_backward``: the gradients of ``sum(grad_logprob * logprob + grad_entropy * entropy)`` by
    ``hidden``, ``weight`` (their type) and, where there is one, ``bias`` (float32), from the forward call's ``lse`` and (with
    ``grad_entropy``) ``entropy``.  ``wanted`` names the ones to compute; ``dhidden`` and ``dweight`` may be given, with rows of
    any stride, and are overwritten."""
    lib = _lib or _load()
    head, R, V, D, dev, query = _head(hidden, weight, tokens, bias, temperature)
    vectors = _optional(R, dev, lse=lse, entropy=entropy, grad_logprob=grad_logprob, grad_entropy=grad_entropy)
    with _Scope(dev, stream) as handle:
        grads, outs = _head_grads(hidden, weight, bias, R, V, D, dev, wanted, dhidden, dweight)
        pws, need, ws = _head_workspace(lib, query, R, V, D, 0, 1 if grads.dbias is None else 2)
        rc = lib.spdy_linear_token_logprobs_backward(*head, *vectors, *outs, pws, need, handle)
    if rc:
        binding._check(rc, "spdy_linear_token_logprobs_backward")
    return grads


def linear_token_logprobs_with_grad(hidden, weight, tokens, grad_logprob=None, grad_entropy=None, bias=None, temperature: float = 1.0,
                                    wanted=("hidden", "weight", "bias"), dhidden=None, dweight=None, stream=None):
    """``spdy_linear_token_logprobs_with_grad``: (``TokenLogprobs``, ``LinearGrads``) in one call, for a loss whose weights per row
    are known beforehand."""
    lib = _lib or _load()
    head, R, V, D, dev, query = _head(hidden, weight, tokens, bias, temperature)
    vectors = _optional(R, dev, grad_logprob=grad_logprob, grad_entropy=grad_entropy)
    with _Scope(dev, stream) as handle:
        logprob, entropy, lse = _vectors(3, R)
        grads, outs = _head_grads(hidden, weight, bias, R, V, D, dev, wanted, dhidden, dweight)
        pws, need, ws = _head_workspace(lib, query, R, V, D, 1, 1 if grads.dbias is None else 2)
        rc = lib.spdy_linear_token_logprobs_with_grad(*head, *vectors, logprob.data_ptr(), entropy.data_ptr(), lse.data_ptr(), *outs, pws,
                                                      need, handle)
    if rc:
        binding._check(rc, "spdy_linear_token_logprobs_with_grad")
    return TokenLogprobs(logprob, entropy, lse), grads


def _teacher(top_ids, top_logprobs, R, dev):
    """(ids' pointer, their bits, log probabilities' pointer) as the C calls take them, and K."""
    if top_ids.ndim != 2:
        raise ValueError("top_ids must be [R][K]")
    K = top_ids.shape[1]
    if top_logprobs.requires_grad:
        _refuse_gradient("top_logprobs")
    bits = _ids(top_ids, "top_ids", (R, K), dev)
    if (top_logprobs.shape != (R, K) or top_logprobs.dtype != torch.float32 or top_logprobs.get_device() != dev
            or not top_logprobs.is_contiguous()):
        raise ValueError("top_logprobs must be a contiguous float32 tensor like top_ids")
    return (top_ids.data_ptr(), bits, top_logprobs.data_ptr()), K


def distill_loss(logits, top_ids, top_logprobs, temperature: float = 1.0, tail: bool = True, stream=None) -> DistillLoss:
    """``spdy_distill_loss``: the divergence of softmax(``logits`` [R][V] / ``temperature``) from a teacher known by its top log
    probabilities [R][K] (float32, at the same temperature) at ``top_ids`` [R][K] (negative = no entry).  With ``tail`` the
    teacher's remaining mass is compared with the student's mass outside the ids; without, the teacher is renormalised over
    them.  Rows are not averaged."""
    lib = _lib or _load()
    head, R, V, dev = _logits(logits)
    teacher, K = _teacher(top_ids, top_logprobs, R, dev)
    with _Scope(dev, stream) as handle:
        out = _vectors(3 if tail else 2, R)
        rc = lib.spdy_distill_loss(*head, *teacher, R, V, K, temperature, bool(tail), out[0].data_ptr(), out[1].data_ptr(),
                                   out[2].data_ptr() if tail else None, handle)
    if rc:
        binding._check(rc, "spdy_distill_loss")
    return DistillLoss(*out)


def distill_loss_backward(logits, top_ids, top_logprobs, lse, rest, grad_loss, temperature: float = 1.0, tail: bool = True,
                          out=None, stream=None):
    """``spdy_distill_loss_backward``: the gradient [R][V] (``logits``' type) of ``sum(grad_loss * loss)`` from the forward call's
    ``lse`` and ``rest`` (None without ``tail``).  ``out`` may be ``logits``."""
    lib = _lib or _load()
    head, R, V, dev = _logits(logits)
    teacher, K = _teacher(top_ids, top_logprobs, R, dev)
    if tail and rest is None:
        raise ValueError("rest is needed with tail")
    vectors = _optional(R, dev, lse=lse, rest=rest if tail else None, grad_loss=grad_loss)
    with _Scope(dev, stream) as handle:
        out, ldo = _grads_out(out, logits, R, V, dev)
        rc = lib.spdy_distill_loss_backward(*head, *teacher, R, V, K, temperature, bool(tail), *vectors, out.data_ptr(), ldo, handle)
    if rc:
        binding._check(rc, "spdy_distill_loss_backward")
    return out


def distill_loss_with_grad(logits, top_ids, top_logprobs, grad_loss, temperature: float = 1.0, tail: bool = True, out=None,
                           stream=None):
    """``spdy_distill_loss_with_grad``: (``DistillLoss``, gradient) in one call.  ``out`` receives the gradient and may be
    ``logits``."""
    lib = _lib or _load()
    head, R, V, dev = _logits(logits)
    teacher, K = _teacher(top_ids, top_logprobs, R, dev)
    pg = _vector(grad_loss, "grad_loss", R, dev, torch.float32)
    with _Scope(dev, stream) as handle:
        out, ldo = _grads_out(out, logits, R, V, dev)
        sums = _vectors(3 if tail else 2, R)
        rc = lib.spdy_distill_loss_with_grad(*head, *teacher, R, V, K, temperature, bool(tail), pg, sums[0].data_ptr(), sums[1].data_ptr(),
                                             sums[2].data_ptr() if tail else None, out.data_ptr(), ldo, handle)
    if rc:
        binding._check(rc, "spdy_distill_loss_with_grad")
    return DistillLoss(*sums), out


class AdamWMoments(NamedTuple):
    """A tensor's moments: float32 [n], or bytes [n] with the bytes [ceil(n / 32)] that blocks of 32 elements share."""

    m: object
    v: object
    m_exp: Optional[object] = None
    v_exp: Optional[object] = None


_TENSOR = np.dtype([("param", "u8"), ("grad", "u8"), ("master", "u8"), ("m", "u8"), ("v", "u8"), ("m_exp", "u8"), ("v_exp", "u8"), ("n", "i8"),
                    ("weight_decay", "f4"), ("param_dtype", "i4"), ("grad_dtype", "i4"), ("state_bits", "i4"), ("keep_zeros", "i4"), ("reserved", "i4")])


class _AdamWOptions(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double), ("step", ctypes.c_int64),
                ("seed", ctypes.c_uint32), ("rounding", ctypes.c_int32), ("lr_device", ctypes.c_void_p), ("step_device", ctypes.c_void_p),
                ("grad_scale", ctypes.c_void_p), ("skip", ctypes.c_void_p)]


def _per_tensor(value, count: int, what: str):
    values = list(value) if isinstance(value, (list, tuple)) else [value] * count
    if len(values) != count:
        raise ValueError(f"{what} must be one value or one for each of the {count} parameters")
    return values


class AdamW:
    """What ``adamw_step`` keeps of a list of parameters: their moments, master copies and settings (``spdy_adamw_tensor``).

    ``params``: contiguous float32, bfloat16 or float16 CUDA tensors of one device, changed in place by the steps.  ``bits``: 32 or 8
    bits for each moment.  ``masters``: None, True (float32 copies of the 16-bit parameters are made here), or a list of float32
    tensors (None where there is no copy).  ``moments``: None (zeros), or a list of ``AdamWMoments`` to go on with, which the steps
    change in place.  ``weight_decay`` and ``keep_zeros`` (elements whose weight is 0 stay 0): one value, or one for each parameter.
    The tensors must keep their memory as long as the plan is used.  ``rounding`` of 16-bit parameters without a master: "nearest" or "stochastic"."""

    def __init__(self, params, bits: int = 32, masters=None, moments=None, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay=0.01, keep_zeros=False,
                 rounding: str = "nearest"):
        _load()
        self.params = list(params)
        if not self.params:
            raise ValueError("params must hold a tensor at least")
        if bits not in (32, 8):
            raise ValueError("bits must be 32 or 8")
        if rounding not in ("nearest", "stochastic"):
            raise ValueError("rounding must be nearest or stochastic")
        self.bits, self.betas, self.eps, self.rounding = bits, (float(betas[0]), float(betas[1])), float(eps), rounding
        if not (0.0 <= self.betas[0] < 1.0 and 0.0 <= self.betas[1] < 1.0 and 0.0 <= self.eps <= 1e30):
            raise ValueError("betas must be in [0, 1), eps at least 0")
        count = len(self.params)
        self.device = self.params[0].get_device()
        for i, p in enumerate(self.params):
            if not p.is_cuda or p.get_device() != self.device or not p.is_contiguous():
                raise ValueError(f"params[{i}] must be a contiguous CUDA tensor on cuda:{self.device}")
            _dtype(p, f"params[{i}]")
        decay, keep = _per_tensor(weight_decay, count, "weight_decay"), _per_tensor(keep_zeros, count, "keep_zeros")
        if not all(0.0 <= float(d) <= 3.4e38 for d in decay):
            raise ValueError("weight_decay must be finite and at least 0")
        with torch.cuda.device(self.device), torch.no_grad():
            if masters is True:
                masters = [None if p.dtype == torch.float32 else p.detach().float() for p in self.params]
            self.masters = _per_tensor(masters, count, "masters")
            if moments is None:
                moments = [self._fresh(p.numel()) for p in self.params]
            self.moments = _per_tensor(list(moments), count, "moments")
        self._table = np.zeros(count, dtype=_TENSOR)
        for i, (p, master, mom) in enumerate(zip(self.params, self.masters, self.moments)):
            n = p.numel()
            if master is not None:
                if p.dtype == torch.float32:
                    raise ValueError(f"params[{i}] is float32 and needs no master")
                self._flat(master, f"masters[{i}]", n, torch.float32)
            if bits == 32:
                parts = ((mom.m, "m", n, torch.float32), (mom.v, "v", n, torch.float32))
            else:
                blocks = (n + 31) // 32
                parts = ((mom.m, "m", n, torch.uint8), (mom.v, "v", n, torch.uint8), (mom.m_exp, "m_exp", blocks, torch.uint8),
                         (mom.v_exp, "v_exp", blocks, torch.uint8))
            for t, name, size, dtype in parts:
                self._flat(t, f"moments[{i}].{name}", size, dtype)
            if n and (mom.m.data_ptr() | mom.v.data_ptr()) & 15:
                raise ValueError(f"moments[{i}] must start on 16 bytes")
            row = self._table[i]
            row["param"], row["master"], row["n"] = p.data_ptr(), _ptr(master) or 0, n
            row["m"], row["v"] = mom.m.data_ptr(), mom.v.data_ptr()
            if bits == 8:
                row["m_exp"], row["v_exp"] = mom.m_exp.data_ptr(), mom.v_exp.data_ptr()
            row["weight_decay"], row["param_dtype"], row["grad_dtype"] = float(decay[i]), _TYPES[p.dtype], _TYPES[p.dtype]
            row["state_bits"], row["keep_zeros"] = bits, bool(keep[i])
        written = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in self._written() if t.numel())
        if any(a[1] > b[0] for a, b in zip(written, written[1:])):
            raise ValueError("params, masters and moments must not share memory")
        self._words = self._table.view(np.uint64).reshape(count, -1)
        self._pointers = [p.data_ptr() for p in self.params]
        self._shapes = [tuple(p.shape) for p in self.params]
        self._strides = [p.stride() for p in self.params]
        self._dtypes = [p.dtype for p in self.params]
        # What autograd may have saved, whether or not it requires a gradient itself: not the 8-bit codes, nor what inference mode made.
        self._seen = [[t for t in (p, master, *mom[:2]) if t is not None and t.is_floating_point() and not t.is_inference()]
                      for p, master, mom in zip(self.params, self.masters, self.moments)]
        self._all_seen = [t for tensors in self._seen for t in tensors]

    def _fresh(self, n: int) -> AdamWMoments:
        if self.bits == 32:
            return AdamWMoments(*(torch.zeros(n, device="cuda") for _ in range(2)))
        return AdamWMoments(*(torch.zeros(size, dtype=torch.uint8, device="cuda") for size in (n, n, (n + 31) // 32, (n + 31) // 32)))

    def _flat(self, t, what: str, n: int, dtype):
        if t is None or not t.is_cuda or t.get_device() != self.device or t.dtype != dtype or t.numel() != n or not t.is_contiguous():
            raise ValueError(f"{what} must be a contiguous tensor of {n} {dtype} on cuda:{self.device}")
        if t.requires_grad:
            raise ValueError(f"{what} must not require a gradient")

    def _written(self):
        for p, master, mom in zip(self.params, self.masters, self.moments):
            yield p
            yield from (t for t in (master, *mom) if t is not None)


def _scalar(t, what: str, dtype, device: int) -> int:
    if not t.is_cuda or t.get_device() != device or t.dtype != dtype or t.numel() != 1:
        raise ValueError(f"{what} must be one {dtype} on cuda:{device}")
    if t.requires_grad:
        _refuse_gradient(what)
    return t.data_ptr()


def adamw_step(plan: AdamW, grads, lr, step, seed: int = 0, grad_scale=None, skip=None, stream=None) -> None:
    """``spdy_adamw_step``: one step on all of ``plan``'s parameters, in place.

    ``grads``: one contiguous tensor of its parameter's shape for each, of its type or float32 (None: the parameter is left alone).
    ``step`` counts from 1.  ``lr`` and ``step`` are numbers, or (for captured steps, which read them when they are replayed) a
    float32 and an int64 CUDA tensor of one element; with ``lr`` a tensor ``step`` has to be one.  ``seed`` (32 bits) drives
    stochastic rounding.  ``grad_scale``: a float32 CUDA tensor of one element that the gradients are multiplied by; ``skip``: one
    that leaves everything unchanged if it is not 0."""
    lib = _lib or _load()
    if len(grads) != len(plan.params):
        raise ValueError(f"grads must hold one entry for each of the {len(plan.params)} parameters")
    dev, f32 = plan.device, torch.float32
    pointers, wide = [], []
    for g, shape, dtype in zip(grads, plan._shapes, plan._dtypes):
        if g is None:
            pointers.append(0)
            continue
        if g.requires_grad:
            _refuse_gradient(f"grads[{len(pointers)}]")
        if g.shape != shape or g.get_device() != dev or not g.is_contiguous():
            raise ValueError(f"grads[{len(pointers)}] must be a contiguous {list(shape)} tensor on cuda:{dev}")
        if g.dtype is not dtype:
            if g.dtype is not f32:
                raise ValueError(f"grads[{len(pointers)}] must be {dtype} or float32")
            wide.append(len(pointers))
        pointers.append(g.data_ptr())
    if plan._pointers != [p.data_ptr() for p in plan.params]:
        raise ValueError("params must stay where they were when the plan was made")
    words = plan._words.copy()  # the plan's own stays as it is: calls of several threads do not meet
    words[:, 1] = pointers
    if wide:
        words.view(_TENSOR)["grad_dtype"][wide] = 0
    o = _AdamWOptions(0.0, *plan.betas, plan.eps, 1, seed & 0xFFFFFFFF, plan.rounding == "stochastic")
    if isinstance(lr, torch.Tensor):
        o.lr_device = _scalar(lr, "lr", f32, dev)
        if not isinstance(step, torch.Tensor):
            raise ValueError("step must be a tensor where lr is one")
    else:
        o.lr = lr
    if isinstance(step, torch.Tensor):
        o.step_device = _scalar(step, "step", torch.int64, dev)
    else:
        o.step = step
    if grad_scale is not None:
        o.grad_scale = _scalar(grad_scale, "grad_scale", f32, dev)
    if skip is not None:
        o.skip = _scalar(skip, "skip", f32, dev)
    with _Scope(dev, stream) as handle:
        rc = lib.spdy_adamw_step(words.ctypes.data, len(pointers), ctypes.byref(o), handle)
    if rc:
        binding._check(rc, "spdy_adamw_step")
    # A graph that was recorded before must notice, as with every operation in place.
    seen = plan._all_seen if 0 not in pointers else [t for tensors, g in zip(plan._seen, grads) if g is not None for t in tensors]
    if seen:
        _new_versions(seen)


def adamw_moments(plan: AdamW, dtype=None, stream=None):
    """The moments of all parameters as numbers: a list of (m, v), in the parameters' shapes.  With 32 bits they are the plan's own
    tensors; with 8 bits ``spdy_adamw_moments`` writes new ones of ``dtype``, float32 (the default) or bfloat16 (as exact)."""
    lib = _lib or _load()
    if plan.bits == 32:
        if dtype not in (None, torch.float32):
            raise ValueError("moments of 32 bits are float32")
        return [(mom.m.view(p.shape), mom.v.view(p.shape)) for p, mom in zip(plan.params, plan.moments)]
    dtype = torch.float32 if dtype is None else dtype
    if dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("dtype must be float32 or bfloat16")
    with _Scope(plan.device, stream) as handle:
        out = [(_empty_strided(shape, strides, dtype), _empty_strided(shape, strides, dtype)) for shape, strides in zip(plan._shapes, plan._strides)]
        firsts, seconds = (np.array([pair[k].data_ptr() for pair in out], dtype=np.uint64) for k in (0, 1))
        rc = lib.spdy_adamw_moments(plan._table.ctypes.data, len(out), firsts.ctypes.data, seconds.ctypes.data, _TYPES[dtype], handle)
    if rc:
        binding._check(rc, "spdy_adamw_moments")
    return out
