"""A head's log probabilities and gradients: single outputs, and how exact logits are (include/spdy_eval.h, spdy_linear_token_logprobs*)."""
import pytest
import torch

from paper_2201_13096_b200 import build as build_mod, evaluate
import tune_reference as tune
from test_linear_logprobs import head, weights

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
gpu = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    build_mod.build()


@gpu
@pytest.mark.parametrize("R,V,D,dtype,entropy", [
    (130, 520, 520, BF16, False), (3, 700, 512, F16, True), (300, 5003, 1030, F16, True), (9000, 40000, 512, BF16, False), (600, 9000, 128, BF16, True),
])
def test_each_gradient_alone_is_the_one_of_a_call_for_several(R, V, D, dtype, entropy):
    # without dbias kept logits have 16 bits, with it 23: each call has its match among those of as many
    h, w, tokens, b = head(R, V, D, dtype, F32)
    gl, gh = weights(R, dtype, entropy)
    for call in (lambda wanted: evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl, gh, b, wanted=wanted)[1],
                 lambda wanted: evaluate.linear_token_logprobs_backward(h, w, tokens, saved.lse, saved.entropy, gl, gh, b, wanted=wanted)):
        saved = evaluate.linear_token_logprobs(h, w, tokens, b)
        two, three = call(("hidden", "weight")), call(("hidden", "weight", "bias"))
        for wanted, want in ((("hidden",), two), (("weight",), two), (("bias",), three), (("bias", "hidden"), three), (("weight", "bias"), three)):
            got = call(wanted)
            for name in ("hidden", "weight", "bias"):
                t = getattr(got, "d" + name)
                assert (t is None) == (name not in wanted)
                assert t is None or torch.equal(t, getattr(want, "d" + name)), (wanted, name)


# Logits are fp32 sums of the tensor core's sums of up to 384 products, twice, and 256 from there on.  Those are cut, 16 products at a time, by less than one
# unit in fp32's last place each: 24 2^-23 of the magnitudes; the additions round by 2^-24 of them each.
def cut_of(D):
    return min(D, 384) / 16 * 2.0 ** -23 + D / 256 * 2.0 ** -24


def against(h, w, b, tokens, cut, dtype):
    """Values, and dbias of both calls (fp32 all of them), against the formula with logits off by ``cut`` of their magnitudes."""
    gl, _ = weights(h.shape[0], dtype, False)
    want = tune.head(h, w, b, tokens, 1.0, gl, None, on="cuda", cut=cut)
    out, grads = evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl, None, b)
    alone = evaluate.linear_token_logprobs(h, w, tokens, b)
    for name in ("logprob", "entropy", "lse"):
        tune.close(getattr(out, name), want, name)
        tune.close(getattr(alone, name), want, name)
    again = evaluate.linear_token_logprobs_backward(h, w, tokens, want["lse"].float(), None, gl, None, b, wanted=("bias",))
    # An exponential below 2^-126 counts as 0 (the special-function unit gives no smaller numbers), each row's by as much times its weight.
    flushed = gl.abs().double().sum() * 2.0 ** -126
    want["dbias_err"] += flushed
    tune.close(again.dbias, want, "dbias")
    if h.shape[1] >= 512:
        want = tune.head(h, w, b, tokens, 1.0, gl, None, on="cuda", cut=cut, kept=23)
        want["dbias_err"] += flushed
    tune.close(grads.dbias, want, "dbias")


@gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("R,D", [(5, 4096), (33, 640), (300, 4096), (300, 20000)])
def test_logits_of_single_products_are_exact(R, D, dtype):
    # as rows of an embedding have them, and channels that pruning left at 0: nothing is cut from sums that fp32 holds
    V = 1003
    g = torch.Generator().manual_seed(1)
    h = torch.zeros(R, D, dtype=dtype)
    h[torch.arange(R), torch.randint(0, D, (R,), generator=g)] = 20.0
    w = torch.randn(V, D, generator=g).to(dtype).cuda()
    tokens = torch.randint(0, V, (R,), generator=g).cuda()
    against(h.cuda(), w, torch.zeros(V, device="cuda"), tokens, 0.0, dtype)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("R,D", [(5, 4096), (32, 1000), (33, 1000), (300, 768), (300, 4096), (300, 16384)])
def test_logits_of_positive_products(R, D, dtype):
    V = 1003
    g = torch.Generator().manual_seed(2)
    h, w = torch.rand(R, D, generator=g).to(dtype).cuda(), (torch.rand(V, D, generator=g) * (40.0 / D)).to(dtype).cuda()
    against(h, w, torch.zeros(V, device="cuda"), torch.randint(0, V, (R,), generator=g).cuda(), cut_of(D), dtype)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("R", [3, 20, 300])
@pytest.mark.parametrize("D,wide", [(64, 4096), (200, 400), (512, 1536)])
def test_columns_of_zeros_change_nothing(R, D, wide, dtype):
    V = 2000
    h, w, tokens, b = head(R, V, D, dtype, F32)
    gl, gh = weights(R, dtype, True)
    hz, wz = (torch.nn.functional.pad(t, (0, wide - D)) for t in (h, w))
    narrow, padded = evaluate.linear_token_logprobs(h, w, tokens, b), evaluate.linear_token_logprobs(hz, wz, tokens, b)
    for name in ("logprob", "entropy", "lse"):
        assert torch.equal(getattr(narrow, name), getattr(padded, name)), name
    one, other = (evaluate.linear_token_logprobs_backward(x, y, tokens, narrow.lse, narrow.entropy, gl, gh, b) for x, y in ((h, w), (hz, wz)))
    assert torch.equal(one.dbias, other.dbias)
    assert (other.dhidden[:, D:] == 0).all() and (other.dweight[:, D:] == 0).all()


@gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("R,V,D", [(5, 3840, 2624), (11, 3840, 2624), (11, 1000, 8192), (16, 1000, 4096), (40, 1000, 8192)])
def test_dbias_of_few_wide_rows_from_a_saved_lse(R, V, D, dtype):
    # Nothing cancels here: lse comes from elsewhere, and p is off by what its logit lacks.  That is followed sum by sum: every 16 products the
    # accumulator loses half a unit of its last place (of the largest number in it) on average; of some hundred cuts the sum stays within a fifth of that.
    # The additions of the pieces round by half a unit of the logit's place at most, evenly: a standard deviation of 12^-1/2 units each, four of them
    # allowed.  The exponent's roundings and lse's own are 2^-22 of lse together.
    h, w, tokens, b = head(R, V, D, dtype, F32, seed=3)
    gl, _ = weights(R, dtype, False)
    h64, w64 = h.double(), w.double()
    x = h64 @ w64.T + b.double()
    lse = torch.logsumexp(x, 1)
    p = (x - lse[:, None]).exp()
    named = tokens >= 0
    g = -p * torch.where(named, gl.double(), 0.0)[:, None]
    g[torch.arange(R, device="cuda")[named], tokens[named]] += gl.double()[named]

    def unit(t):
        return torch.exp2(torch.floor(torch.log2(t.abs().clamp(min=1e-30))) - 23)

    lost, acc = torch.zeros_like(x), torch.zeros_like(x)
    for k in range(0, D, 16):
        if k in (384, 768) or (k > 768 and k % 256 == 0):
            acc.zero_()
        products = h64[:, None, k:k + 16] * w64[None, :, k:k + 16]
        before = acc.abs()
        acc = acc + products.sum(2)
        lost += 0.6 * unit(torch.maximum(torch.maximum(before, acc.abs()), products.abs().amax(2)))
    off = lost + 4 * (D / 256 / 12) ** 0.5 * unit(x) + 2.0 ** -22 * lse.abs()[:, None]
    bound = (p * gl.double().abs()[:, None] * off).sum(0).norm() + 2.0 ** -22 * g.sum(0).norm()
    got = evaluate.linear_token_logprobs_backward(h, w, tokens, lse.float(), None, gl, None, b).dbias
    assert (got.double() - g.sum(0)).norm() <= bound


@gpu
@pytest.mark.parametrize("R,V,D,dtype,bias,entropy", [
    (5, 3000, 72, BF16, None, True), (6, 1764, 826, F16, None, False), (44, 1536, 1536, F16, None, False), (63, 777, 200, F16, F32, True), (64, 5003, 512, BF16, F32, False),
    (33, 2001, 640, F16, F32, True), (32, 9000, 64, BF16, "same", True), (61, 999, 1030, BF16, None, True), (64, 4096, 256, F16, None, True), (64, 700, 1100, BF16, F32, True),
])
def test_gradients_of_few_rows_are_rounded_once(R, V, D, dtype, bias, entropy):
    # up to 64 rows the gradient by the logits is the sum of two numbers of 16 bits: dhidden and dweight are as exact as their own last rounding, and what
    # kept logits and the sums' cuts take
    h, w, tokens, b = head(R, V, D, dtype, bias, padh=3, padw=0)
    gl, gh = weights(R, dtype, entropy)
    saved = evaluate.linear_token_logprobs(h, w, tokens, b)
    again = evaluate.linear_token_logprobs_backward(h, w, tokens, saved.lse, saved.entropy, gl, gh, b)
    want = tune.head(h, w, b, tokens, 1.0, gl, gh, on="cuda", halves=2)
    for name in ("dhidden", "dweight"):
        tune.close(getattr(again, name), want, name)
    for wanted in (("hidden", "weight"), ("hidden", "weight", "bias")):
        kept = 0 if D < 512 else 23 if b is not None and "bias" in wanted else 16
        want = tune.head(h, w, b, tokens, 1.0, gl, gh, on="cuda", kept=kept, halves=2)
        grads = evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl, gh, b, wanted=wanted)[1]
        for name in ("dhidden", "dweight"):
            tune.close(getattr(grads, name), want, name)
        if grads.dbias is not None:
            tune.close(grads.dbias, want, "dbias")


@gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_few_rows_over_pieces_of_a_vocabulary(dtype):
    R, V, D = 10, 2_200_001, 24  # the gradient in two halves, for 1.8 million ids at a time
    h, w, tokens, b = head(R, V, D, dtype, F32)
    gl, gh = weights(R, dtype, True)
    want = tune.head(h, w, b, tokens, 1.0, gl, gh, on="cuda", halves=2)
    saved = evaluate.linear_token_logprobs(h, w, tokens, b)
    for grads in (evaluate.linear_token_logprobs_backward(h, w, tokens, saved.lse, saved.entropy, gl, gh, b),
                  evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl, gh, b)[1]):
        for name in ("dhidden", "dweight", "dbias"):
            tune.close(getattr(grads, name), want, name)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("D", [64, 520])
def test_few_rows_that_are_not_finite_stay_alone(D, dtype):
    R, V = 40, 777
    h, w, tokens, b = head(R, V, D, dtype, F32)
    gl, gh = weights(R, dtype, True)

    def calls():
        saved = evaluate.linear_token_logprobs(h, w, tokens, b)  # the backward call takes what the forward call gave for the same rows
        return (evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl, gh, b, wanted=("hidden", "weight"))[1], evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl, gh, b)[1],
                evaluate.linear_token_logprobs_backward(h, w, tokens, saved.lse, saved.entropy, gl, gh, b))

    clean = calls()
    h[5, 3], h[39, 0] = float("nan"), float("inf")
    rest = torch.ones(R, dtype=torch.bool, device="cuda")
    rest[5] = rest[39] = False
    for got, want in zip(calls(), clean):
        assert torch.isnan(got.dhidden[5]).all() and not torch.isfinite(got.dhidden[39]).any()
        assert torch.equal(got.dhidden[rest], want.dhidden[rest])
    tokens.fill_(-1)  # padding: rows without a token and without a gradient, finite ones
    h[5, 3], h[39, 0] = 1.0, 1.0
    saved = evaluate.linear_token_logprobs(h, w, tokens, b)
    for grads in (evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl, None, b)[1], evaluate.linear_token_logprobs_backward(h, w, tokens, saved.lse, None, gl, None, b)):
        assert (grads.dhidden == 0).all() and (grads.dweight == 0).all() and (grads.dbias == 0).all()
