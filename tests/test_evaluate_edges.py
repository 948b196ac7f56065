"""The evaluation operators at the ends of their ranges: alignments, magnitudes, counts, and what they refuse."""
import math

import pytest
import torch

import eval_reference as ref
import test_evaluate
from paper_2201_13096_b200 import build as build_mod, evaluate
from test_evaluate import BF16, F16, F32, norm_bounds, rand

INF = math.inf
gpu = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    build_mod.build()


# ------------------------------------------------------------------------------------------------ layer norm

@gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("R,D", [(7, 768), (5, 8), (300, 96)])
@pytest.mark.parametrize("lead", range(8))
def test_layer_norm_of_rows_that_start_anywhere_with_fp32_parameters(dtype, R, D, lead):
    """A row's first granule may begin before the row: the parameters are not read there."""
    x = rand(R, D, seed=1, dtype=dtype, pad=12 - lead, shift=lead)
    w, b = 1.0 + 0.2 * rand(D, seed=2), 0.3 * rand(D, seed=3)
    want, mean64, rstd64 = ref.layer_norm(x, w, b, 1e-5)
    y, mean, rstd = evaluate.layer_norm(x, w, b)
    ref.close(y, want, norm_bounds(x, w, b, want, rstd64), "y")


# ------------------------------------------------------------------------------------------------ large finite logits

def lowered(x):
    """(64-bit logits less each row's largest, that largest): beside -1e30 not even 64 bits resolve the log of a count."""
    top = ref.d64(x).amax(1, keepdim=True)
    return ref.d64(x) - top, top[:, 0]


def distill_lowered(x, ids, lps, temperature, tail, weight):
    """``ref.distill`` for rows of distinct ids, some logits allowed outside them, every sum relative to its own largest term: (loss,
    lse, rest, gradient, log p, p, the softmax outside the ids and its log)."""
    low, top = lowered(x)
    t, teacher, ids = low / temperature, ref.d64(lps), ids.cpu()
    if not tail:
        teacher = torch.log_softmax(teacher, 1)
    q = teacher.exp()
    inside = torch.zeros(t.shape, dtype=torch.bool).scatter(1, ids, True)
    left = (1.0 - q.sum(1)).clamp(min=0.0) if tail else torch.zeros(len(t), dtype=torch.float64)
    logp = torch.log_softmax(t, 1)
    best_out = t.masked_fill(inside, -INF).amax(1, keepdim=True)
    out_log = torch.log_softmax((t - best_out).masked_fill(inside, -INF), 1)
    log_rest = torch.logsumexp((t - best_out).masked_fill(inside, -INF), 1) + best_out[:, 0] - torch.logsumexp(t, 1)  # of p outside
    loss = (q * (teacher - logp.gather(1, ids))).sum(1) + torch.where(left > 0, left * (left.log() - log_rest), torch.zeros_like(left))
    grad = (q.sum(1) + left)[:, None] * logp.exp() - left[:, None] * out_log.exp()
    grad = grad.scatter_add(1, ids, -q) * ref.d64(weight)[:, None] / temperature
    lse = torch.logsumexp(t, 1) + top / temperature
    return loss, lse, lse + log_rest, grad, logp, logp.exp(), out_log.exp(), out_log


def magnitudes(x, temperature):
    """The magnitude of each row's largest logit over T, which lse is rounded relative to."""
    return (ref.d64(x).amax(1) / temperature).abs()


def masked_rows(V, dtype, value, seed):
    """Seven rows of ordinary logits in which ``value`` marks ids that are not allowed: all of them, all but one, the first half, the
    second half, 95 in 100, every second, none."""
    x = rand(7, V, seed=seed, dtype=dtype, scale=3.0)
    few = (torch.rand(V, generator=torch.Generator().manual_seed(seed)) < 0.95).cuda()
    few[:2] = False  # some stay
    x[0] = value
    x[1, torch.arange(V, device="cuda") != V // 3] = value
    x[2, :V // 2] = value
    x[3, V // 2:] = value
    x[4, few] = value
    x[5, ::2] = value
    return x


def gradient_bound(p, logp, size):
    """p is off by its exponent's rounding, which is relative to |log p| (and 2^-20 for the sum it is divided by); below 2^-126 it is 0."""
    rel = 2.0 ** -20 * (14 + torch.where(p > 0, logp.abs(), torch.zeros_like(p)))
    return (rel * p + 2.0 ** -126) * size


LARGE = [(F32, -1e9), (F32, -5e9), (F32, -1e10), (F32, -3e10), (F32, -1e20), (F32, -1e30), (BF16, -1e9), (BF16, -1e10), (BF16, -3e10), (BF16, -1e30), (F16, -6e4)]


@gpu
@pytest.mark.parametrize("V", [40, 1500, 3000, 30000])
@pytest.mark.parametrize("dtype,value", LARGE)
def test_token_logprobs_where_large_finite_numbers_mask(dtype, value, V):
    x = masked_rows(V, dtype, value, V)
    tokens = torch.tensor([1, V // 3, V - 1, 0, 2, 1, -1], device="cuda")
    gl, gh = rand(7, seed=5), rand(7, seed=6)
    for temperature in (1.0, 0.7, 0.1):
        low, top = lowered(x)
        lp, h, lse = ref.token_logprobs(low, tokens, temperature)
        lse = lse + top / temperature
        err = 2.0 ** -21 * (magnitudes(x, temperature) + 14)
        # beside the largest logit nothing of a row's size comes in: its sums are relative to it
        flat = 2.0 ** -19 * 14 * torch.ones(7, dtype=torch.float64)
        logp, p, _ = ref.softmax_row(low, temperature)
        want = ref.token_logprobs_grad(low, tokens, gl, gh, temperature)
        size = ref.d64(gl).abs()[:, None] + ref.d64(gh).abs()[:, None] * (2 * torch.where(p > 0, logp.abs(), torch.zeros_like(p)) + 14)
        got = evaluate.token_logprobs(x, tokens, top_k=min(20, V), temperature=temperature)
        both, grad = evaluate.token_logprobs_with_grad(x, tokens, gl, gh, temperature=temperature)
        for values in (got, both):
            ref.close(values.lse, lse, err, "lse")
            ref.close(values.logprob, lp, flat + 2.0 ** -21 * lp.abs(), "logprob")
            ref.close(values.entropy, h, flat, "entropy")
        assert torch.equal(got.top_ids.cpu().long(), ref.top(x, min(20, V)))
        ref.close(got.top_logprobs, logp.gather(1, got.top_ids.cpu().long()), 2.0 ** -19 * 14 + 2.0 ** -21 * logp.gather(1, got.top_ids.cpu().long()).abs(), "alternatives")
        ref.close(grad, want, 2 * gradient_bound(p, logp, size) / temperature + 2.0 ** -21 * want.abs(), "with_grad")
        back = evaluate.token_logprobs_backward(x, tokens, got.lse, got.entropy, gl, gh, temperature=temperature)
        small = magnitudes(x, temperature) < 1e4
        assert torch.equal(small, torch.arange(7) > 0)
        e = 2 * (err[:, None] * p * size + gradient_bound(p, logp, size)) / temperature + 2.0 ** -21 * want.abs()
        ref.close(back[1:], want[1:], e[1:], "backward")
        # an lse of that size names no row's sum: p is between 0 and 1 all the same
        most = (ref.d64(gl).abs() + ref.d64(gh).abs() * (14 + 1))[0] / temperature
        assert bool(torch.isfinite(back[0]).all()) and float(back[0].float().abs().max()) <= float(most) * 1.01


@gpu
@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("V", [40, 1500, 3000, 30000])
@pytest.mark.parametrize("dtype,value", LARGE)
def test_distillation_where_large_finite_numbers_mask(dtype, value, V, tail):
    K = 6
    x = masked_rows(V, dtype, value, V + 1)
    g = torch.Generator().manual_seed(V)
    scores = torch.where(ref.d64(x) < -1e4, torch.full((7, V), -20.0, dtype=torch.float64), ref.d64(x)) + torch.randn(7, V, generator=g, dtype=torch.float64)
    best = torch.log_softmax(scores, 1).topk(K, dim=1)
    ids, lps = best.indices.cuda(), best.values.float().cuda()
    weight = rand(7, seed=8)
    for temperature in (1.0, 0.7, 0.1):
        loss, lse, rest, grad, logp, p, outside, out_log = distill_lowered(x, ids, lps, temperature, tail, weight)
        err = 2.0 ** -21 * (magnitudes(x, temperature) + 14)
        # log p within 2^-21 of itself and 2^-19 * 14, q and 1 - sum q within 2^-20, the latter times the tail's logarithm
        bound = 2.0 ** -19 * 44 + 2.0 ** -20 * loss.abs() + 2.0 ** -20 * (torch.exp(ref.d64(lps)) * logp.gather(1, ids.cpu()).abs()).sum(1)
        if tail:
            bound = bound + 2.0 ** -20 * (rest - lse).abs()
        got = evaluate.distill_loss(x, ids, lps, temperature=temperature, tail=tail)
        both, once = evaluate.distill_loss_with_grad(x, ids, lps, weight, temperature=temperature, tail=tail)
        inside = torch.zeros(7, V, dtype=torch.float64).scatter(1, ids.cpu(), 1.0)
        e = gradient_bound(p, logp, 4.0) + 2.0 ** -20 * inside
        if tail:
            e = e + gradient_bound(outside, out_log, 4.0)
        e = e * ref.d64(weight).abs()[:, None] / temperature + 2.0 ** -20 * grad.abs()
        for values in (got, both):
            ref.close(values.lse, lse, err, "lse")
            ref.close(values.loss, loss, bound, "loss")
            if tail:
                ref.close(values.rest, rest, 2.0 ** -21 * (rest.abs() + 14), "rest")
        ref.close(once, grad, e, "with_grad")
        back = evaluate.distill_loss_backward(x, ids, lps, got.lse, got.rest, weight, temperature=temperature, tail=tail)
        rows = [r for r in range(7) if lse[r].abs() < 1e4 and (not tail or rest[r].abs() < 1e4)]
        assert len(rows) >= 4  # with few ids all of those allowed may be the teacher's
        extra = 4 * (err[:, None] * (p + inside) + (2.0 ** -21 * (rest.abs() + 14))[:, None] * outside * float(tail)) * ref.d64(weight).abs()[:, None] / temperature
        ref.close(back[rows], grad[rows], (e + extra)[rows], "backward")
        assert bool(torch.isfinite(back).all()) and bool((back.float().abs().cpu() <= 3.01 * weight.abs().cpu()[:, None] / temperature).all())


@gpu
@pytest.mark.parametrize("V", [40, 1500, 3000, 30000])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("temperature", [1e-9, 1e-6, 1e6])
def test_token_logprobs_at_extreme_temperatures(dtype, V, temperature):
    x = rand(5, V, seed=V, dtype=dtype, scale=3.0)
    x[0] = 13.7
    x[1, V // 2:] = 20.3
    tokens = x.argmax(1)
    gl, gh = rand(5, seed=5), rand(5, seed=6)
    low, top = lowered(x)
    lp, h, lse = ref.token_logprobs(low, tokens, temperature)
    lse = lse + top / temperature
    logp, p, _ = ref.softmax_row(low, temperature)
    flat = 2.0 ** -19 * 14 * torch.ones(5, dtype=torch.float64)
    got = evaluate.token_logprobs(x, tokens, temperature=temperature)
    both, grad = evaluate.token_logprobs_with_grad(x, tokens, gl, gh, temperature=temperature)
    for values in (got, both):
        ref.close(values.lse, lse, 2.0 ** -21 * (magnitudes(x, temperature) + 14), "lse")
        ref.close(values.logprob, lp, flat + 2.0 ** -21 * lp.abs(), "logprob")
        ref.close(values.entropy, h, flat, "entropy")
    want = ref.token_logprobs_grad(low, tokens, gl, gh, temperature)
    size = ref.d64(gl).abs()[:, None] + ref.d64(gh).abs()[:, None] * (2 * torch.where(p > 0, logp.abs(), torch.zeros_like(p)) + 14)
    ref.close(grad, want, 2 * gradient_bound(p, logp, size) / temperature + 2.0 ** -21 * want.abs(), "with_grad")


# ------------------------------------------------------------------------------------------------ activations

@gpu
@pytest.mark.parametrize("M", [1, 16, 300])
@pytest.mark.parametrize("kind", ["gelu", "silu"])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_activations_are_accurate_relative_to_themselves(dtype, kind, M):
    """Down to where they underflow: a value formed from 1 + erf would lose the negative tail."""
    z = torch.cat([torch.linspace(-13, 13, 4001), torch.linspace(-6, -2, 2001), rand(2000, seed=3).cpu(), torch.tensor([0.0, -0.0, 1e-6, -1e-6, 40.0, 1e4, -60.0, -1e3, INF])]).cuda()
    x, w = torch.zeros(M, 16, dtype=dtype, device="cuda"), torch.zeros(z.numel(), 16, dtype=dtype, device="cuda")
    zd = ref.d64(z)
    want = 0.5 * zd * torch.special.erfc(-zd / math.sqrt(2.0)) if kind == "gelu" else zd * torch.sigmoid(zd)
    # the exponential's argument, z^2 log2(e) / 2 or z log2(e), is rounded to 24 bits; some ten roundings beside it
    err = 2.0 ** -20 * want.abs() * (1 + (zd ** 2 / 16 if kind == "gelu" else zd.abs() / 8).clamp(max=100.0))
    err[zd == INF] = 0.0
    got = evaluate.linear(x, w, bias=z, activation=kind, out_dtype=F32)
    ref.close(got, want.expand(M, -1), err.expand(M, -1), "fp32")
    ref.close(evaluate.linear(x, w, bias=z, activation=kind), want.expand(M, -1), err.expand(M, -1), "16 bits")
    assert torch.isnan(evaluate.linear(x, w, bias=torch.full_like(z, math.nan), activation=kind)).all()


# ------------------------------------------------------------------------------------------------ linear

@gpu
@pytest.mark.parametrize("M", [262140, 262141, 600001])
@pytest.mark.parametrize("out_dtype", [BF16, F32])
def test_linear_without_products_has_as_many_rows_as_any(M, out_dtype):
    N = 3
    x, w = torch.empty(M, 0, dtype=BF16, device="cuda"), torch.empty(N, 0, dtype=BF16, device="cuda")
    b, res = rand(N, seed=1), rand(M, N, seed=2, dtype=BF16, pad=2)
    want, err = ref.linear(x, w, b, res, "silu")
    ref.close(evaluate.linear(x, w, b, res, "silu", out_dtype=out_dtype), want, err)
    want, err = ref.linear(x, w, b, None, "none")
    ref.close(evaluate.linear(x, w, b, out_dtype=out_dtype), want, err)


# ------------------------------------------------------------------------------------------------ gradients that autograd expects

def test_tensors_that_require_a_gradient_are_refused():
    x = torch.zeros(2, 8, requires_grad=True)
    evaluate.library()
    with pytest.raises(ValueError, match="gradient"):
        evaluate.layer_norm(x)
    with torch.no_grad(), pytest.raises(ValueError, match="CUDA"):
        evaluate.layer_norm(x)


@gpu
def test_every_tensor_that_requires_a_gradient_is_refused():
    """Nothing is recorded, so that a result without history would lose it in silence."""
    x, w, b = rand(4, 16, dtype=BF16), rand(16, 16, seed=1, dtype=BF16), rand(16, seed=2, dtype=BF16)
    logits, tokens, v = rand(4, 16, seed=3), torch.zeros(4, dtype=torch.int64, device="cuda"), rand(4, seed=4)
    ids, lps = torch.arange(2, device="cuda").expand(4, 2).contiguous(), torch.full((4, 2), -2.0, device="cuda")
    calls = [
        (evaluate.linear, (x, w, b, x)), (evaluate.layer_norm, (x, b, b)), (evaluate.layer_norm_backward, (x, x, b, v, v)),
        (evaluate.token_logprobs, (logits, tokens)), (evaluate.token_logprobs_backward, (logits, tokens, v, v, v, v)),
        (evaluate.token_logprobs_with_grad, (logits, tokens, v, v)), (evaluate.distill_loss, (logits, ids, lps)),
        (evaluate.distill_loss_backward, (logits, ids, lps, v, v, v)), (evaluate.distill_loss_with_grad, (logits, ids, lps, v)),
    ]
    for call, args in calls:
        call(*args)
        for k, t in enumerate(args):
            if not t.is_floating_point():
                continue
            tracked = [*args[:k], t.detach().clone().requires_grad_(), *args[k + 1:]]
            with pytest.raises(ValueError, match="gradient"):
                call(*tracked)
            with torch.no_grad():
                call(*tracked)
    torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------------ what torch does not promise

def test_an_entry_of_torch_that_answers_otherwise_is_not_used():
    evaluate.library()
    plain = lambda shape, strides, dtype: torch.empty_strided(shape, strides, dtype=dtype)  # noqa: E731
    for fast in (None, lambda *a: 1 / 0, lambda shape, strides: plain(shape, strides, F16), lambda shape, strides, dtype: plain(shape, strides, F32),
                 lambda shape, strides, dtype: torch.empty(shape, dtype=dtype), lambda *a: None):
        assert evaluate._checked(fast, plain, evaluate._same_memory) is plain
    good = lambda shape, strides, dtype: plain(shape, strides, dtype)  # noqa: E731
    assert evaluate._checked(good, plain, evaluate._same_memory) is good


@gpu
def test_results_lie_in_memory_of_the_kind_asked_for():
    evaluate.library()
    t = evaluate._empty_strided((3, 5), (5, 1), BF16)
    assert t.is_cuda and t.shape == (3, 5) and t.is_contiguous() and t.dtype == BF16
    assert evaluate._current_device() == torch.cuda.current_device()
    assert evaluate._current_stream(0) == torch.cuda.current_stream(0).cuda_stream


# ------------------------------------------------------------------------------------------------ linear: large products

def tiles_of(M, N, K, sms=148):
    """The tile shape with the least estimated time, as the library estimates it for products too large to share a tile's K."""
    up, k = (lambda a, b: -(-a // b)), -(-K // 128)
    assert up(M, 128) * up(N, 64) * 2 > sms
    options = {"pair": (256, 256, sms // 2, 1040, 4000), "128": (128, 128, sms, 620, 2500), "64": (128, 64, sms, 540, 2000)}
    time = {name: up(up(M, r) * up(N, w), units) * per * k + fixed for name, (r, w, units, per, fixed) in options.items()}
    return min(time, key=time.get), up(up(M, 256) * up(N, 256), sms // 2)


# M, K, N, dtype, activation, bias, residual, pad of x, pad of w, tiles, tiles of 256 x 256 that a pair of multiprocessors has at most
PRODUCTS = [
    (2304, 1536, 2048, BF16, "none", None, False, 0, 0, "pair", 1), (2290, 1001, 1793, BF16, "gelu", "same", True, 0, 0, "pair", 1),
    (4097, 520, 2999, F16, "silu", "same", True, 8, 16, "pair", 3), (4100, 384, 3000, BF16, "relu", F32, True, 0, 0, "pair", 3),
    (8191, 700, 2559, BF16, "gelu", "same", True, 5, 3, "pair", 5), (16390, 400, 765, F16, "none", "same", True, 0, 8, "pair", 3),
    (2305, 1000, 2311, F16, "gelu", "same", True, 0, 0, "128", 2), (16390, 640, 60, BF16, "none", None, True, 8, 0, "64", 1),
]


@gpu
@pytest.mark.parametrize("M,K,N,dtype,kind,bias,residual,padx,padw,tiles,rounds", PRODUCTS)
def test_large_products_against_the_formula(M, K, N, dtype, kind, bias, residual, padx, padw, tiles, rounds):
    """Pairs of multiprocessors on a tile: rings that wrap around, accumulators used again, ends of rows, columns and K, strided operands,
    both result types, over the residual, into a wider buffer."""
    assert tiles_of(M, N, K) == (tiles, rounds)
    test_evaluate.test_linear_against_the_formula(M, K, N, dtype, kind, bias, residual, padx, padw)


# ------------------------------------------------------------------------------------------------ offsets beyond 32 bits

def filled(R, C, seed):
    """bf16 values whose last rows lie beyond 2^31 elements."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(R, C, dtype=BF16, device="cuda").normal_(generator=g)


@gpu
def test_rows_beyond_the_first_2_to_the_31_elements():
    R, C = 66000, 33001
    assert (R - 2) * C > 2 ** 31
    x = filled(R, C, 1)
    at = torch.tensor([0, 1, R - 2, R - 1])
    xs = x[at.cuda()].clone()
    tokens = torch.arange(R, device="cuda") % C
    ids = (torch.arange(4, device="cuda")[None, :] * 7919 + torch.arange(R, device="cuda")[:, None]) % C
    lps = torch.full((R, 4), -2.0, device="cuda")
    g = torch.ones(R, device="cuda")
    lp, h, lse = ref.token_logprobs(xs, tokens[at.cuda()], 1.0)
    flat = 2.0 ** -19 * 14
    got = evaluate.token_logprobs(x, tokens, top_k=5)
    ref.close(got.logprob[at.cuda()], lp, flat)
    assert torch.equal(got.top_ids[at.cuda()].cpu().long(), ref.top(xs, 5))
    y, mean, rstd = evaluate.layer_norm(x)
    want, mean64, rstd64 = ref.layer_norm(xs, None, None, 1e-5)
    ref.close(y[at.cuda()], want, norm_bounds(xs, None, None, want, rstd64), "y")
    dx, _, _ = evaluate.layer_norm_backward(y, x, None, mean, rstd, out=y, params=False)
    dx64, _, _ = ref.layer_norm_backward(want.bfloat16(), xs, None, mean64, rstd64)
    ref.close(dx[at.cuda()], dx64, 0.02 * (1 + want.abs()))  # y was rounded to 16 bits, the gradient of which is nearly all cancelled
    del y, dx
    loss, _, _, grad = ref.distill(xs, ids[at.cuda()], lps[at.cuda()], 1.0, True, g[at.cuda()].cpu())
    out, dlogits = evaluate.distill_loss_with_grad(x, ids, lps, g, out=x)
    ref.close(out.loss[at.cuda()], loss, 1e-4)
    ref.close(dlogits[at.cuda()], grad, 1e-6)


@gpu
@pytest.mark.parametrize("K", [64, 61])
def test_products_beyond_the_first_2_to_the_31_elements(K):
    M, N = 1100000, 2000
    assert (M - 2) * N > 2 ** 31
    x, w, b = rand(300, K, seed=1, dtype=BF16).repeat(-(-M // 300), 1)[:M], rand(N, K, seed=2, dtype=BF16, scale=K ** -0.5), rand(N, seed=3)
    at = torch.tensor([0, 1, M // 2, M - 2, M - 1])
    want, err = ref.linear(x[at.cuda()], w, b, None, "gelu")
    ref.close(evaluate.linear(x, w, b, activation="gelu")[at.cuda()], want, err)
