"""The evaluation operators (include/spdy_eval.h) against their formulas in 64 bits, their special values and refusals."""
import ctypes
import math
import os
import re

import pytest
import torch

import eval_reference as ref
from paper_2201_13096_b200 import binding, build as build_mod, evaluate

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INF = math.inf
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
gpu = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    build_mod.build()


def rand(*shape, seed=0, dtype=F32, scale=1.0, pad=0, shift=0):
    """Normal values on the GPU; with ``pad`` a view of a buffer whose rows are longer, ``shift`` elements in."""
    g = torch.Generator().manual_seed(seed)
    v = (torch.randn(*shape, generator=g) * scale).to(dtype)
    if not pad and not shift:
        return v.cuda()
    buf = torch.full((shape[0], shape[1] + pad + shift), 7.0, dtype=dtype, device="cuda")
    view = buf[:, shift:shift + shape[1]]
    view.copy_(v)
    return view


def twin(x):
    """A copy with the same strides and alignment: sums over its rows run in the same order."""
    if x._base is None:
        return x.clone()
    return x._base.clone().as_strided(x.shape, x.stride(), x.storage_offset())


# ------------------------------------------------------------------------------------------------ without a GPU

def test_library_exports_every_declared_operator():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "spdy_eval.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(spdy_[a-z_0-9]+)\s*\(", text)))
    lib = evaluate.library()
    assert names == sorted(evaluate.EXPORTS)
    for name in names:
        assert hasattr(lib, name), name


def test_c_entries_refuse_bad_arguments_before_any_gpu_work():
    lib = evaluate.library()
    P = 1 << 20  # a pointer that is never followed
    lin = lib.spdy_linear
    good = [P, 64, P, 64, 1, None, 1, None, 0, 0, 9, 8, 64, P, 8, 1, None, 0, None]

    def bad(fn, args, *changes):
        args = list(args)
        for at, v in changes:
            args[at] = v
        return fn(*args)

    for change in ((0, None), (0, P + 1), (1, 63), (2, None), (3, 63), (4, 0), (4, 3), (9, 4), (9, -1), (10, -1), (11, -1), (12, -1),
                   (13, None), (13, P + 1), (14, 7), (15, 2), (10, 1 << 31), (12, 1 << 31)):
        assert bad(lin, good, change) == -1, change
    assert bad(lin, good, (5, P), (6, 2)) == -1            # bias of another 16-bit type
    assert bad(lin, good, (7, P), (8, 7)) == -1            # residual rows overlap
    assert bad(lin, good, (1, 65)) == -1                   # needs a workspace and has none
    assert bad(lin, good, (1, 65), (16, P + 8), (17, 1 << 20)) == -1   # misaligned workspace
    assert bad(lin, good, (1, 65), (16, P), (17, 16)) == -2
    assert bad(lin, good, (10, 0)) == 0 and bad(lin, good, (11, 0)) == 0
    assert lib.spdy_linear_workspace_bytes(P, 64, P, 64, 1, 9, 8, 64) == 0
    assert lib.spdy_linear_workspace_bytes(P, 65, P, 64, 1, 9, 8, 64) == 9 * 64 * 2 // 256 * 256 + 256
    assert lib.spdy_linear_workspace_bytes(P, 65, P, 65, 1, 1, 8, 64) == 0  # few rows need none

    norm = [P, 8, 0, P, P, 0, 4, 8, 1e-5, P, 8, P, P, None]
    for change in ((0, None), (1, 7), (2, 5), (5, 1), (6, -1), (7, 0), (8, -1.0), (8, math.nan), (8, INF), (9, None), (10, 7), (0, P + 2)):
        assert bad(lib.spdy_layer_norm, norm, change) == -1, change
    assert bad(lib.spdy_layer_norm, norm, (6, 0)) == 0
    back = [P, 8, P, 8, 0, P, 0, P, P, 4, 8, P, 8, P, P, P, 1 << 20, None]
    for change in ((0, None), (1, 7), (2, None), (3, 7), (4, 9), (6, 2), (7, None), (8, None), (9, -1), (10, 0), (11, None), (12, 7), (15, None),
                   (15, P + 16)):
        assert bad(lib.spdy_layer_norm_backward, back, change) == -1, change
    assert bad(lib.spdy_layer_norm_backward, back, (16, 8)) == -2
    assert lib.spdy_layer_norm_backward_workspace_bytes(0, 8, 0) == 0

    lp = [P, 16, 1, P, 64, 2, 16, 1.0, 4, P, P, P, P, P, None]
    for change in ((0, None), (0, P + 1), (1, 15), (2, 7), (3, None), (3, P + 4), (4, 16), (5, -1), (6, 0), (7, 0.0), (7, -1.0), (7, math.nan),
                   (7, INF), (8, -1), (8, 17), (12, None), (13, None)):
        assert bad(lib.spdy_token_logprobs, lp, change) == -1, change
    assert bad(lib.spdy_token_logprobs, lp, (6, 1000), (1, 1000), (8, evaluate.SPDY_TOP_MAX + 1)) == -1
    assert bad(lib.spdy_token_logprobs, lp, (5, 0)) == 0
    lb = [P, 16, 1, P, 64, 2, 16, 1.0, P, P, P, P, P, 16, None]
    for change in ((8, None), (9, None), (12, None), (13, 15), (3, None)):
        assert bad(lib.spdy_token_logprobs_backward, lb, change) == -1, change
    lg = [P, 16, 1, P, 64, 2, 16, 1.0, P, P, P, P, P, P, 16, None]
    for change in ((3, None), (11, None), (12, None), (13, None), (14, 15)):
        assert bad(lib.spdy_token_logprobs_with_grad, lg, change) == -1, change

    di = [P, 16, 1, P, 64, P, 2, 16, 4, 1.0, 1, P, P, P, None]
    for change in ((0, None), (1, 15), (3, None), (3, P + 4), (4, 8), (5, None), (5, P + 2), (7, 0), (8, 0), (8, evaluate.SPDY_DISTILL_MAX + 1), (9, 0.0)):
        assert bad(lib.spdy_distill_loss, di, change) == -1, change
    db = [P, 16, 1, P, 64, P, 2, 16, 4, 1.0, 1, P, P, P, P, 16, None]
    for change in ((11, None), (12, None), (13, None), (14, None), (15, 15)):
        assert bad(lib.spdy_distill_loss_backward, db, change) == -1, change
    dg = [P, 16, 1, P, 64, P, 2, 16, 4, 1.0, 1, P, P, P, P, P, 16, None]
    for change in ((11, None), (13, None), (14, None), (15, None), (16, 15)):
        assert bad(lib.spdy_distill_loss_with_grad, dg, change) == -1, change


def test_python_calls_refuse_cpu_tensors():
    x = torch.zeros(2, 8)
    with pytest.raises(ValueError, match="CUDA"):
        evaluate.layer_norm(x)
    with pytest.raises(ValueError, match="bfloat16"):
        evaluate.linear(x, x)
    with pytest.raises(ValueError, match="CUDA"):
        evaluate.linear(x.bfloat16(), x.bfloat16())
    with pytest.raises(ValueError, match="activation"):
        evaluate.linear(x.bfloat16(), x.bfloat16(), activation="tanh")
    with pytest.raises(ValueError, match="CUDA"):
        evaluate.token_logprobs(x, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError, match="CUDA"):
        evaluate.distill_loss(x, torch.zeros(2, 1, dtype=torch.int64), torch.zeros(2, 1))


# ------------------------------------------------------------------------------------------------ linear

LINEAR = [
    # M, K, N, dtype, activation, bias, residual, pad of x, pad of w
    (1, 1, 1, BF16, "none", None, False, 0, 0), (1, 768, 96, BF16, "gelu", "same", False, 0, 0), (1, 77, 5, F16, "silu", F32, True, 3, 1),
    (2, 256, 3, BF16, "relu", "same", True, 0, 0), (4, 264, 130, F16, "gelu", None, True, 8, 0), (5, 1001, 33, BF16, "silu", F32, False, 5, 2),
    (8, 512, 64, F16, "none", "same", True, 0, 0), (8, 100, 17, BF16, "gelu", "same", True, 4, 4),
    (9, 8, 1, BF16, "none", None, False, 0, 0), (9, 64, 64, F16, "relu", "same", True, 0, 0), (17, 1, 9, BF16, "gelu", F32, False, 0, 0),
    (33, 63, 65, F16, "silu", "same", True, 1, 0), (128, 64, 64, BF16, "none", None, False, 0, 0), (128, 768, 2, BF16, "gelu", "same", True, 0, 0),
    (129, 1024, 200, F16, "gelu", F32, True, 8, 16), (300, 2048, 64, BF16, "relu", "same", False, 0, 0), (100, 4096, 72, F16, "none", "same", True, 0, 0),
    (257, 1000, 127, BF16, "silu", "same", True, 22, 5), (2048, 72, 1280, BF16, "gelu", "same", True, 0, 0), (2050, 200, 1281, F16, "silu", F32, False, 0, 0),
    (4096, 64, 1280, F16, "relu", None, True, 0, 0), (4100, 136, 1300, BF16, "gelu", "same", True, 8, 0), (640, 320, 2000, BF16, "none", "same", False, 0, 0),
]


@gpu
@pytest.mark.parametrize("M,K,N,dtype,kind,bias,residual,padx,padw", LINEAR)
def test_linear_against_the_formula(M, K, N, dtype, kind, bias, residual, padx, padw):
    x, w = rand(M, K, seed=1, dtype=dtype, pad=padx), rand(N, K, seed=2, dtype=dtype, scale=K ** -0.5, pad=padw)
    b = None if bias is None else rand(N, seed=3, dtype=dtype if bias == "same" else bias)
    res = rand(M, N, seed=4, dtype=dtype, pad=padx) if residual else None
    want, err = ref.linear(x, w, b, res, kind)
    ref.close(evaluate.linear(x, w, b, res, kind), want, err, "16-bit result")
    ref.close(evaluate.linear(x, w, b, res, kind, out_dtype=F32), want, err, "fp32 result")
    out = rand(M, N, seed=5, dtype=dtype, pad=3, shift=1)  # rows that start anywhere, neighbours left alone
    whole = out._base.clone()
    assert evaluate.linear(x, w, b, res, kind, out=out) is out
    ref.close(out, want, err, "into a wider buffer")
    whole[:, 1:1 + N] = out
    assert torch.equal(whole, out._base)
    if residual:
        again = res.clone()
        evaluate.linear(x, w, b, again, kind, out=again)
        ref.close(again, want, err, "over the residual")
    evaluate.linear_check_status()


@gpu
@pytest.mark.parametrize("M", [0, 1, 8, 9, 40])
@pytest.mark.parametrize("K", [0, 24])
@pytest.mark.parametrize("N", [0, 5])
def test_linear_of_nothing(M, K, N):
    x, w, b, res = rand(M, K, dtype=BF16), rand(N, K, seed=1, dtype=BF16), rand(N, seed=2, dtype=BF16), rand(M, N, seed=3, dtype=BF16)
    want, err = ref.linear(x, w, b, res, "gelu")
    ref.close(evaluate.linear(x, w, b, res, "gelu"), want, err)


@gpu
@pytest.mark.parametrize("M", [3, 20])
@pytest.mark.parametrize("kind", ["none", "relu", "gelu", "silu"])
def test_linear_carries_special_values(M, kind):
    x, w = torch.zeros(M, 16, dtype=F16, device="cuda"), torch.eye(16, dtype=F16, device="cuda")
    x[0, :4] = torch.tensor([INF, -INF, math.nan, 60000.0])
    x[1, :4] = torch.tensor([-60000.0, -20.0, 20.0, 1e-7])
    z = x.float().cpu()
    z[0, torch.arange(16) != 0] = math.nan  # an infinity times 0 in the other columns
    z[0, 0] = math.nan                      # and a NaN in its row
    y = evaluate.linear(x, w, activation=kind).float().cpu()
    assert torch.isnan(y[0]).all()
    want = ref.activation(z[1:].double(), kind)
    ref.close(evaluate.linear(x[1:], w, activation=kind), want, 2.0 ** -20 * z[1:].double().abs())
    ends = torch.tensor([INF, -INF], dtype=F32, device="cuda").repeat(8)
    y = evaluate.linear(torch.zeros(M, 16, dtype=F16, device="cuda"), w, bias=ends, activation=kind, out_dtype=F32).cpu()
    assert (y[:, 0] == INF).all()
    if kind == "gelu":
        assert (torch.isnan(y[:, 1]) | (y[:, 1] == 0)).all()
    else:
        assert (y[:, 1] == {"none": -INF, "relu": 0.0, "silu": 0.0}[kind]).all()


# ------------------------------------------------------------------------------------------------ layer norm

def norm_bounds(x, w, b, y, rstd):
    """fp32 error of y: the mean is off by at most 2^-20 of the mean magnitude (sums of D values in about log D + D / 512
    levels), the deviations and rstd by a few units, relative to the larger of |x| and the deviation."""
    xd = ref.d64(x)
    size = xd.abs().mean(1, keepdim=True) + xd.abs()
    ww = torch.ones(x.shape[1], dtype=torch.float64) if w is None else ref.d64(w).abs()
    return 2.0 ** -20 * (size * rstd[:, None] * ww) + 2.0 ** -20 * y.abs() + (0 if b is None else 2.0 ** -22 * ref.d64(b).abs())


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("R,D,pad", [(1, 1, 0), (3, 2, 0), (5, 7, 0), (9, 8, 8), (4, 31, 1), (130, 64, 0), (33, 256, 3), (7, 768, 0), (5, 999, 0), (300, 1024, 0),
                                     (3, 1025, 0), (2, 2048, 8), (6, 2049, 0), (3, 4096, 0), (4, 4100, 5), (2, 8192, 0), (3, 8193, 0), (2, 16384, 0),
                                     (2, 40000, 0), (2, 40001, 1)])
def test_layer_norm_and_its_gradients(dtype, R, D, pad):
    x = rand(R, D, seed=1, dtype=dtype, pad=pad, scale=2.0)
    x += 0.5
    dy = rand(R, D, seed=2, dtype=dtype, pad=pad)
    for params in ("same", F32, None):
        w = None if params is None else (1.0 + 0.2 * rand(D, seed=3)).to(dtype if params == "same" else F32)
        b = None if params is None else (0.3 * rand(D, seed=4)).to(dtype if params == "same" else F32)
        want, mean64, rstd64 = ref.layer_norm(x, w, b, 1e-5)
        y, mean, rstd = evaluate.layer_norm(x, w, b)
        size = ref.d64(x).abs().mean(1)
        ref.close(mean, mean64, 2.0 ** -20 * size, "mean")
        ref.close(rstd, rstd64, 2.0 ** -20 * rstd64 * (1 + (mean64 * rstd64) ** 2 * 2.0 ** -10), "rstd")
        ref.close(y, want, norm_bounds(x, w, b, want, rstd64), "y")
        over = twin(x)
        assert torch.equal(evaluate.layer_norm(over, w, b, out=over)[0], y)
        dx64, dw64, db64 = ref.layer_norm_backward(dy, x, w, mean, rstd)
        dx, dw, db = evaluate.layer_norm_backward(dy, x, w, mean, rstd)
        h = (ref.d64(x) - ref.d64(mean)[:, None]) * ref.d64(rstd)[:, None]
        u = ref.d64(dy) * (1.0 if w is None else ref.d64(w))
        # h is off by 2^-22 of (|x| + |mean|) rstd; the row's two means and the columns' sums by 2^-20 of their magnitudes
        eh = 2.0 ** -22 * (ref.d64(x).abs() + ref.d64(mean).abs()[:, None]) * ref.d64(rstd)[:, None]
        part = u.abs() + u.abs().mean(1, keepdim=True) + (h.abs() + 1) * (u * h).abs().mean(1, keepdim=True)
        ref.close(dx, dx64, ref.d64(rstd)[:, None] * (2.0 ** -19 * part + eh * (u * h).abs().mean(1, keepdim=True) + h.abs() * (u.abs() * eh).mean(1, keepdim=True)), "dx")
        ref.close(dw, dw64, (2.0 ** -20 * (ref.d64(dy) * h).abs() + ref.d64(dy).abs() * eh).sum(0), "dweight")
        ref.close(db, db64, 2.0 ** -20 * ref.d64(dy).abs().sum(0), "dbias")
        over, _, none = evaluate.layer_norm_backward(same := twin(dy), x, w, mean, rstd, out=same, params=False)
        assert none is None and torch.equal(over, dx)
        again = evaluate.layer_norm_backward(dy, x, w, mean, rstd)
        assert torch.equal(again[1], dw) and torch.equal(again[2], db)


@gpu
def test_layer_norm_of_many_rows_adds_every_row_once():
    R, D = 5000, 40
    x = rand(R, D, seed=1)
    dy = torch.ones(R, D, device="cuda")
    _, mean, rstd = evaluate.layer_norm(x)
    _, dw, db = evaluate.layer_norm_backward(dy, x, None, mean, rstd)
    assert torch.equal(db.cpu(), torch.full((D,), float(R)))
    _, dw64, _ = ref.layer_norm_backward(dy, x, None, mean, rstd)
    ref.close(dw, dw64, 2.0 ** -20 * R)


@gpu
@pytest.mark.parametrize("D", [1, 5, 64, 3000])
def test_layer_norm_of_constant_rows_and_of_none(D):
    x = torch.full((4, D), 3.25, device="cuda")
    y, mean, rstd = evaluate.layer_norm(x, bias=torch.full((D,), 0.5, device="cuda"), eps=1e-3)
    assert torch.equal(mean, x[:, 0]) and torch.equal(y, torch.full_like(y, 0.5))
    ref.close(rstd, torch.full((4,), 1e-3, dtype=torch.float64) ** -0.5, 2.0 ** -21 * 40)
    y, mean, rstd = evaluate.layer_norm(x[:0])
    assert y.shape == (0, D) and mean.shape == (0,)
    dx, dw, db = evaluate.layer_norm_backward(x[:0], x[:0], None, mean, rstd)
    assert dx.shape == (0, D) and not dw.any() and not db.any()


def difference(f, x, direction, step):
    return (f(x + step * direction) - f(x - step * direction)) / (2 * step)


@gpu
def test_layer_norm_gradient_against_differences():
    R, D = 6, 37
    x, w, b, dy = rand(R, D, seed=1), rand(D, seed=2), rand(D, seed=3), rand(R, D, seed=4)
    _, mean, rstd = evaluate.layer_norm(x, w, b)
    dx, dw, db = evaluate.layer_norm_backward(dy, x, w, mean, rstd)
    f = lambda xx, ww, bb: (ref.layer_norm(xx, ww, bb, 1e-5)[0] * ref.d64(dy)).sum()  # noqa: E731
    for k, (grad, at) in enumerate(((dx, x), (dw, w), (db, b))):
        v = torch.randn(at.shape, generator=torch.Generator().manual_seed(9 + k), dtype=torch.float64)
        args = [ref.d64(t) for t in (x, w, b)]
        slope = difference(lambda t: f(*[t if i == k else a for i, a in enumerate(args)]), args[k], v, 1e-5)
        # the quotient is good to 1e-8 here; the fp32 gradient to 2^-18 of the sum of magnitudes
        assert abs(float((ref.d64(grad) * v).sum() - slope)) <= 2.0 ** -18 * float((ref.d64(grad) * v).abs().sum()) + 1e-6


# ------------------------------------------------------------------------------------------------ token log probabilities

def logits_of(R, V, dtype, seed=0, pad=0, shift=0, masked=0.0):
    x = rand(R, V, seed=seed, dtype=dtype, scale=3.0, pad=pad, shift=shift)
    if masked:
        g = torch.Generator().manual_seed(seed + 1)
        x[(torch.rand(R, V, generator=g) < masked).cuda()] = -INF
    return x


def sizes_of(x, temperature):
    """The largest finite |x| / T of each row: what the exponents' roundings are relative to."""
    v = ref.d64(x).abs() / temperature
    return torch.where(torch.isfinite(v), v, torch.zeros_like(v)).amax(1)


ROWS = [(1, 1, 0, 0), (2, 2, 0, 0), (3, 7, 1, 0), (5, 8, 0, 0), (4, 9, 0, 0), (3, 127, 0, 1), (200, 130, 0, 0), (3, 1000, 8, 0), (4, 4099, 0, 0), (2, 16384, 0, 0),
        (1, 32768, 0, 0), (2, 50001, 3, 1), (1, 140001, 0, 0), (1, 300007, 0, 0)]


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("R,V,pad,shift", ROWS)
@pytest.mark.parametrize("masked", [0.0, 0.9])
def test_token_logprobs_against_the_formula(dtype, R, V, pad, shift, masked):
    x = logits_of(R, V, dtype, seed=V, pad=pad, shift=shift, masked=masked)
    tokens = torch.randint(-1, V, (R,), generator=torch.Generator().manual_seed(1)).cuda()
    for temperature, k in ((1.0, min(V, 20)), (0.7, min(V, 128)), (3.0, 0)):
        got = evaluate.token_logprobs(x, tokens, top_k=k, temperature=temperature)
        lp, h, lse = ref.token_logprobs(x, tokens, temperature)
        a = sizes_of(x, temperature)
        # every exponent x c - m is rounded once relative to |x c| (2^-24) and c itself once; the sums add 2^-22 or less, so
        # the logarithms are good to 2^-21 of (|x| / T + log V); the entropy multiplies that by the spread of the row at most
        err = 2.0 ** -21 * (a + 14)
        ref.close(got.lse, lse, err, "lse")
        ref.close(got.logprob, lp, err, "logprob")
        ref.close(got.entropy, h, 4 * err, "entropy")
        if k:
            ids = ref.top(x, k)
            assert torch.equal(got.top_ids.cpu().long(), ids)
            logp, _, _ = ref.softmax_row(x, temperature)
            ref.close(got.top_logprobs, logp.gather(1, ids), err[:, None].expand(R, k), "alternatives")
        else:
            assert got.top_ids is None
        same = evaluate.token_logprobs(x, tokens.int(), top_k=k, temperature=temperature)
        assert all(a is None or torch.equal(a.view(torch.int32), b.view(torch.int32)) for a, b in zip(got, same))


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("kind", ["constant", "rising", "falling", "two values", "few left", "nothing left", "lowest value", "zeros of both signs", "NaN", "all NaN"])
@pytest.mark.parametrize("R,V", [(2, 700), (1, 20011), (300, 9000)])
def test_alternatives_where_the_order_is_against_them(dtype, kind, R, V):
    x = torch.zeros(R, V, dtype=dtype, device="cuda")
    ramp = torch.arange(V, device="cuda", dtype=F32)
    if kind == "rising":
        x += (ramp / V * 20).to(dtype)
    elif kind == "falling":
        x -= (ramp / V * 20).to(dtype)
    elif kind == "two values":
        x[:, ::3] = 1.0
    elif kind == "few left":
        x.fill_(-INF)
        x[:, 5::V // 7] = 2.0
    elif kind == "nothing left":
        x.fill_(-INF)
    elif kind == "lowest value":
        x.fill_(torch.finfo(dtype).min)
        x[:, V // 2:] = -INF
    elif kind == "zeros of both signs":
        x[:, ::2] = -0.0
    elif kind == "NaN":
        x += (ramp / V).to(dtype)
        x[:, 3::5] = math.nan
    elif kind == "all NaN":
        x.fill_(math.nan)
    tokens = torch.full((R,), V - 1, device="cuda")
    for k in (1, 20, 128):
        got = evaluate.token_logprobs(x, tokens, top_k=k)
        ids = ref.top(x[:1], k)
        assert torch.equal(got.top_ids.cpu().long(), ids.expand(R, k))
    lp, h, lse = ref.token_logprobs(x[:1], tokens[:1], 1.0)
    logp, _, _ = ref.softmax_row(x[:1], 1.0)
    err = 2.0 ** -21 * (sizes_of(x[:1], 1.0) + 14)
    for name, a, b, e in (("lse", got.lse, lse, err), ("logprob", got.logprob, lp, err), ("entropy", got.entropy, h, 4 * err)):
        ref.close(a, b.expand(R), e, name)
    ref.close(got.top_logprobs, logp.gather(1, ids).expand(R, 128), err, "alternatives")


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("R,V,pad,shift", ROWS)
def test_token_logprobs_gradients_against_the_formula(dtype, R, V, pad, shift):
    x = logits_of(R, V, dtype, seed=V + 1, pad=pad, shift=shift, masked=0.3 if V > 8 else 0.0)
    tokens = torch.randint(-1, V, (R,), generator=torch.Generator().manual_seed(2)).cuda()
    gl, gh = rand(R, seed=5, scale=8.0), rand(R, seed=6)
    for temperature, l, h in ((1.0, gl, None), (0.7, gl, gh), (2.0, None, gh)):
        want = ref.token_logprobs_grad(x, tokens, l, h, temperature)
        fwd = evaluate.token_logprobs(x, tokens, temperature=temperature)
        got = evaluate.token_logprobs_backward(x, tokens, fwd.lse, fwd.entropy, l, h, temperature=temperature)
        logp, p, _ = ref.softmax_row(x, temperature)
        # p is good to the exponent's error, 2^-21 (|x| / T + 14) relative; the factor beside it likewise
        lp = torch.where(p > 0, logp.abs(), torch.zeros_like(p))
        rel = 2.0 ** -21 * (sizes_of(x, temperature)[:, None] + 14)
        scale = (0 if l is None else ref.d64(l).abs()[:, None]) + (0 if h is None else ref.d64(h).abs()[:, None] * (2 * lp + 14))
        err = 2 * rel * p * scale / temperature + 2.0 ** -22 * want.abs()
        ref.close(got, want, err, "backward")
        both, grad = evaluate.token_logprobs_with_grad(x, tokens, l, h, temperature=temperature)
        ref.close(grad, want, err, "with_grad")
        e = 2.0 ** -21 * (sizes_of(x, temperature) + 14)
        for name, a, b, bound in zip(("logprob", "entropy", "lse"), both[:3], ref.token_logprobs(x, tokens, temperature), (e, 4 * e, e)):
            ref.close(a, b, bound, name)
        over = twin(x)
        evaluate.token_logprobs_backward(over, tokens, fwd.lse, fwd.entropy, l, h, temperature=temperature, out=over)
        assert torch.equal(over, got)
        over = twin(x)
        evaluate.token_logprobs_with_grad(over, tokens, l, h, temperature=temperature, out=over)
        assert torch.equal(over, grad)


@gpu
@pytest.mark.parametrize("V", [40, 3000, 70000])
@pytest.mark.parametrize("dtype", [F32, F16])
def test_token_logprobs_gradients_of_special_rows(dtype, V):
    x = logits_of(6, V, dtype, seed=3)
    x[0] = -INF
    x[1, 5] = math.nan
    x[2, 6] = INF
    tokens = torch.tensor([3, 3, 3, V, -100, 1 << 40], device="cuda")
    gl, gh = torch.ones(6, device="cuda"), torch.ones(6, device="cuda")
    fwd = evaluate.token_logprobs(x, tokens, top_k=4)
    assert fwd.lse[0] == -INF and fwd.logprob[0] == -INF and fwd.entropy[0] == 0
    assert torch.isnan(torch.stack([fwd.lse[1:3], fwd.logprob[1:3], fwd.entropy[1:3]])).all()
    assert torch.isnan(fwd.logprob[[3, 5]]).all() and fwd.logprob[4] == 0 and torch.isfinite(fwd.lse[3:]).all()
    for h in (None, gh):
        for grad in (evaluate.token_logprobs_backward(x, tokens, fwd.lse, fwd.entropy, gl, h),
                     evaluate.token_logprobs_with_grad(x, tokens, gl, h)[1]):
            assert not grad[0].any() and torch.isnan(grad[[1, 2, 3, 5]]).all()
            assert torch.isfinite(grad[4]).all() and (h is not None or not grad[4].any())


@gpu
def test_token_logprobs_gradient_against_differences():
    R, V = 5, 61
    x, tokens = rand(R, V, seed=1, scale=2.0), torch.arange(R).cuda() * 7
    gl, gh = rand(R, seed=2), rand(R, seed=3)
    for temperature in (1.0, 1.7):
        def f(t):
            lp, h, _ = ref.token_logprobs(t, tokens, temperature)
            return (lp * ref.d64(gl) + h * ref.d64(gh)).sum()

        grad = evaluate.token_logprobs_with_grad(x, tokens, gl, gh, temperature=temperature)[1]
        v = torch.randn(R, V, generator=torch.Generator().manual_seed(4), dtype=torch.float64)
        slope = difference(f, ref.d64(x), v, 1e-5)
        assert abs(float((ref.d64(grad) * v).sum() - slope)) <= 2.0 ** -17 * float((ref.d64(grad) * v).abs().sum()) + 1e-6


# ------------------------------------------------------------------------------------------------ distillation

def teacher_of(x, K, temperature, seed, absent=False):
    g = torch.Generator().manual_seed(seed)
    t = ref.d64(x) * 0.8 / temperature + torch.randn(x.shape, generator=g, dtype=torch.float64)
    t = torch.where(torch.isfinite(t), t, torch.full_like(t, -INF))
    best = t.topk(K, dim=1)
    ids, lps = best.indices, (best.values - torch.logsumexp(t, 1, keepdim=True)).float()
    if absent and K > 2:
        ids[::2, 1] = -1
    return ids.cuda(), lps.cuda()


DISTILL = [(1, 1, 1), (3, 2, 1), (4, 7, 3), (3, 64, 64), (2, 129, 100), (200, 300, 5), (3, 1000, 32), (2, 4099, 256), (2, 20000, 16), (1, 50001, 64), (1, 140001, 40)]


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("R,V,K", DISTILL)
@pytest.mark.parametrize("tail", [True, False])
def test_distillation_against_the_formula(dtype, R, V, K, tail):
    for temperature, masked, pad, absent in ((1.0, 0.0, 0, False), (2.0, 0.3 if V > 40 and K < V // 3 else 0.0, 5, True)):
        x = logits_of(R, V, dtype, seed=V + K, pad=pad, masked=masked)
        ids, lps = teacher_of(x, K, temperature, 11, absent)
        g = rand(R, seed=8, scale=4.0)
        loss, lse, rest, grad = ref.distill(x, ids, lps, temperature, tail, g.cpu())
        got = evaluate.distill_loss(x, ids, lps, temperature=temperature, tail=tail)
        a = sizes_of(x, temperature)
        e = 2.0 ** -21 * (a + 14)
        ref.close(got.lse, lse, e, "lse")
        # log p is good to e, log q to 2^-22 of itself; q to 2^-21, 1 - sum q to 2^-22 (K / 32 + 5) in all: with the logarithms'
        # sizes (at most lse - log p's range, about a + 30) as slopes
        el = (e + 2.0 ** -20 * (a + 30) * (1 + K / 64))
        if tail:
            ref.close(got.rest, rest, e, "rest")
        ref.close(got.loss, loss, el * 2, "loss")
        back = evaluate.distill_loss_backward(x, ids, lps, got.lse, got.rest, g, temperature=temperature, tail=tail)
        _, p, _ = ref.softmax_row(x, temperature)
        rel = 2 * e[:, None] + 2.0 ** -20
        outside = torch.exp(ref.d64(x) / temperature - rest[:, None])
        outside = torch.where(torch.isfinite(outside), outside, torch.zeros_like(outside))
        inside = torch.zeros(R, V + 1, dtype=torch.float64).scatter_(1, torch.where(ids.cpu() < 0, V, ids.cpu().long()), 1.0)[:, :V]
        # outside the ids the factor A p_rest - left is off by 2^-21 (K / 32 + 8) beside p_rest's own relative error
        err = ref.d64(g).abs()[:, None] / temperature * (
            rel * (p + inside) + (1 - inside) * outside * (2.0 ** -21 * (K / 32 + 8) + rel * 2 * torch.exp(rest - lse).nan_to_num()[:, None]) * float(tail))
        err = err + rel * grad.abs()
        ref.close(back, grad, err, "backward")
        both, once = evaluate.distill_loss_with_grad(x, ids, lps, g, temperature=temperature, tail=tail)
        ref.close(once, grad, err, "with_grad")
        ref.close(both.loss, loss, el * 2, "with_grad's loss")
        ref.close(both.lse, lse, e, "with_grad's lse")
        assert (both.rest is None) == (not tail)
        over = twin(x)
        assert torch.equal(evaluate.distill_loss_with_grad(over, ids, lps, g, temperature=temperature, tail=tail, out=over)[1], once)
        over = twin(x)
        assert torch.equal(evaluate.distill_loss_backward(over, ids, lps, got.lse, got.rest, g, temperature=temperature, tail=tail, out=over), back)
        same = evaluate.distill_loss(x, ids.int(), lps, temperature=temperature, tail=tail)
        assert torch.equal(same.loss, got.loss)


@gpu
@pytest.mark.parametrize("V", [60, 5000, 70001])
@pytest.mark.parametrize("tail", [True, False])
def test_distillation_of_special_rows(V, tail):
    K = 6
    x = logits_of(9, V, F32, seed=2)
    ids, lps = teacher_of(x, K, 1.0, 5)
    x[0] = -INF                                                 # no id is allowed
    ids[1] = -1                                                 # no teacher
    lps[2] = -INF                                               # a teacher without mass on its ids
    ids[3, 2] = V                                               # an id beyond the vocabulary
    x[4, ids[4, 0]] = -INF                                      # the student excludes what the teacher wants
    mask = torch.ones(V, dtype=torch.bool, device="cuda")
    mask[ids[5]] = False
    x[5, mask] = -INF                                           # nothing left outside the ids
    ids[6, 1] = ids[6, 0]                                       # an id twice
    x[7, 0] = math.nan
    g = torch.ones(9, device="cuda")
    loss, lse, rest, grad = ref.distill(x, ids, lps, 1.0, tail, g.cpu())
    loss[0] = INF
    got = evaluate.distill_loss(x, ids, lps, tail=tail)
    both, once = evaluate.distill_loss_with_grad(x, ids, lps, g, tail=tail)
    back = evaluate.distill_loss_backward(x, ids, lps, got.lse, got.rest, g, tail=tail)
    grad[7] = math.nan
    for values in (got, both):
        ref.close(values.loss, loss, 1e-4, "loss")
        ref.close(values.lse, lse, 1e-4, "lse")
        if tail:
            ref.close(values.rest, rest, 1e-4, "rest")
    for d in (once, back):
        rows = [0, 1, 2, 3, 4, 5, 6, 8]
        ref.close(d[rows], grad[rows], 2e-5, "gradient")
        assert torch.isnan(d[7]).any()
    assert not once[0].any() and (tail or not once[1].any())


@gpu
@pytest.mark.parametrize("tail", [True, False])
def test_distillation_gradient_against_differences(tail):
    R, V, K = 4, 53, 6
    x = rand(R, V, seed=1, scale=2.0)
    ids, lps = teacher_of(x, K, 1.5, 3)
    g = rand(R, seed=2)
    f = lambda t: (ref.distill(t, ids, lps, 1.5, tail)[0] * ref.d64(g)).sum()  # noqa: E731
    grad = evaluate.distill_loss_with_grad(x, ids, lps, g, temperature=1.5, tail=tail)[1]
    v = torch.randn(R, V, generator=torch.Generator().manual_seed(4), dtype=torch.float64)
    slope = difference(f, ref.d64(x), v, 1e-5)
    assert abs(float((ref.d64(grad) * v).sum() - slope)) <= 2.0 ** -17 * float((ref.d64(grad) * v).abs().sum()) + 1e-6


@gpu
def test_the_dense_models_alternatives_feed_the_distillation():
    """A student equal to its teacher has loss 0 and no gradient, whatever part of the vocabulary was kept."""
    x = logits_of(7, 4000, F32, seed=9)
    tokens = torch.zeros(7, dtype=torch.int64, device="cuda")
    top = evaluate.token_logprobs(x, tokens, top_k=50, temperature=2.0)
    got, grad = evaluate.distill_loss_with_grad(x, top.top_ids, top.top_logprobs, torch.ones(7, device="cuda"), temperature=2.0)
    assert got.loss.abs().max() < 2.0 ** -20 * 40 and grad.abs().max() < 2.0 ** -20


# ------------------------------------------------------------------------------------------------ calls

@gpu
def test_rows_of_none():
    e = torch.empty(0, 50, device="cuda")
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    got = evaluate.token_logprobs(e, none, top_k=3)
    assert got.logprob.shape == (0,) and got.top_ids.shape == (0, 3)
    assert evaluate.token_logprobs_with_grad(e, none)[1].shape == (0, 50)
    got = evaluate.distill_loss(e, torch.empty(0, 4, dtype=torch.int32, device="cuda"), torch.empty(0, 4, device="cuda"))
    assert got.loss.shape == (0,)


@gpu
def test_other_streams_and_graphs():
    x, w, b = rand(64, 128, dtype=BF16), rand(96, 128, seed=1, dtype=BF16), rand(96, seed=2, dtype=BF16)
    odd = rand(64, 128, dtype=BF16, pad=1)
    logits, tokens = rand(5, 3000, seed=3, dtype=BF16), torch.arange(5, device="cuda")
    ones = torch.ones(5, device="cuda")

    def everything(stream=None):
        y = evaluate.linear(x, w, b, activation="gelu", stream=stream)
        y2 = evaluate.linear(odd, w, b, activation="gelu", stream=stream)
        n, mean, rstd = evaluate.layer_norm(y, stream=stream)
        grads = evaluate.layer_norm_backward(y, y, None, mean, rstd, stream=stream)
        top = evaluate.token_logprobs(logits, tokens, top_k=9, stream=stream)
        dist, grad = evaluate.distill_loss_with_grad(logits, top.top_ids, top.top_logprobs, ones, stream=stream)
        return [y, y2, n, mean, rstd, *grads, *top, dist.loss, grad]

    want = everything()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = everything(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    assert torch.cuda.current_stream() != side
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = everything()
    for t in captured:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, captured))


@gpu
def test_python_calls_refuse_what_does_not_fit():
    x, w = rand(4, 16, dtype=BF16), rand(8, 16, dtype=BF16)
    logits, tokens = rand(4, 16), torch.zeros(4, dtype=torch.int64, device="cuda")
    ids, lps = torch.zeros(4, 2, dtype=torch.int64, device="cuda"), torch.zeros(4, 2, device="cuda")
    bad = [
        lambda: evaluate.linear(x, w[:, :8]), lambda: evaluate.linear(x, w.half()), lambda: evaluate.linear(x.t(), w), lambda: evaluate.linear(x, w, bias=rand(7, dtype=BF16)),
        lambda: evaluate.linear(x, w, bias=rand(8, dtype=F16)), lambda: evaluate.linear(x, w, residual=x), lambda: evaluate.linear(x, w, out_dtype=F16),
        lambda: evaluate.linear(x, w, out=rand(4, 8)[:, :7]), lambda: evaluate.linear(x[:1].expand(4, 16), w), lambda: evaluate.linear(x[0], w),
        lambda: evaluate.layer_norm(x, weight=rand(15, dtype=BF16)), lambda: evaluate.layer_norm(x, weight=rand(16, dtype=BF16), bias=rand(16)),
        lambda: evaluate.layer_norm(x.int()), lambda: evaluate.layer_norm(x, eps=-1.0), lambda: evaluate.layer_norm_backward(x, x, None, rand(3), rand(4)),
        lambda: evaluate.layer_norm_backward(x.half(), x, None, rand(4), rand(4)),
        lambda: evaluate.token_logprobs(logits, tokens[:3]), lambda: evaluate.token_logprobs(logits, tokens.float()), lambda: evaluate.token_logprobs(logits, tokens, top_k=17),
        lambda: evaluate.token_logprobs(logits, tokens, top_k=-1), lambda: evaluate.token_logprobs(logits, tokens, temperature=0.0),
        lambda: evaluate.token_logprobs(logits, tokens, temperature=math.nan), lambda: evaluate.token_logprobs(logits.double(), tokens),
        lambda: evaluate.token_logprobs(rand(4, 300), tokens, top_k=200), lambda: evaluate.token_logprobs_with_grad(logits, tokens, grad_logprob=rand(3)),
        lambda: evaluate.token_logprobs_backward(logits, tokens, rand(4), None, None, rand(4)), lambda: evaluate.token_logprobs(logits, tokens.cpu()),
        lambda: evaluate.distill_loss(logits, ids, lps[:, :1]), lambda: evaluate.distill_loss(logits, ids[:3], lps), lambda: evaluate.distill_loss(logits, ids[0], lps),
        lambda: evaluate.distill_loss(logits, ids, lps.half()), lambda: evaluate.distill_loss_backward(logits, ids, lps, rand(4), None, rand(4)),
        lambda: evaluate.distill_loss_with_grad(logits, ids, lps, rand(4), out=rand(4, 15)), lambda: evaluate.distill_loss(logits, ids.float(), lps),
    ]
    for k, call in enumerate(bad):
        with pytest.raises((ValueError, binding.SpdyError)):
            call()
            pytest.fail(f"call {k} was accepted")
    torch.cuda.synchronize()
