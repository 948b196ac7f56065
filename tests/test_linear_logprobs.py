"""A head's log probabilities without a table of logits, and their gradients (include/spdy_eval.h, spdy_linear_token_logprobs*)."""
import math

import pytest
import torch

import eval_reference as ref
import tune_reference as tune
from paper_2201_13096_b200 import binding, build as build_mod, evaluate
from test_evaluate import rand

INF = math.inf
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
gpu = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    build_mod.build()


def head(R, V, D, dtype, bias=None, padh=0, padw=0, seed=0, named=0.7):
    """Hidden states, weight, bias and tokens as a model has them: most tokens are likely, some rows have none."""
    h, w = rand(R, D, seed=seed, dtype=dtype, pad=padh), rand(V, D, seed=seed + 1, dtype=dtype, scale=3.0 * D ** -0.5, pad=padw)
    g = torch.Generator().manual_seed(seed + 2)
    tokens = torch.randint(0, V, (R,), generator=g)
    push = (torch.rand(R, 1, generator=g) < named).float().cuda()
    h.copy_((h.float() + push * w[tokens.cuda()].float() * (4.0 / 3.0)).to(dtype))
    tokens[torch.rand(R, generator=g) < 0.1] = -100
    b = None if bias is None else rand(V, seed=seed + 3, dtype=dtype if bias == "same" else F32, scale=0.5)
    return h, w, tokens.cuda(), b


def weights(R, dtype, entropy, seed=7):
    scale = 4096.0 if dtype == F16 else 1.0
    gl = -rand(R, seed=seed).abs() * scale / max(R, 1)
    return gl, rand(R, seed=seed + 1) * (0.05 * scale / max(R, 1)) if entropy else None


def check(h, w, b, tokens, temperature, gl, gh, on="cpu"):
    want = tune.head(h, w, b, tokens, temperature, gl, gh, on)
    alone = evaluate.linear_token_logprobs(h, w, tokens, b, temperature)
    out, grads = evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl, gh, b, temperature)
    again = evaluate.linear_token_logprobs_backward(h, w, tokens, out.lse, out.entropy, gl, gh, b, temperature)
    # from a width of 512 on the logits are kept, in 23 bits with dbias and in 16 without
    other, kept = evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl, gh, b, temperature, wanted=("hidden", "weight"))
    for name in ("logprob", "entropy", "lse"):
        tune.close(getattr(out, name), want, name)
        tune.close(getattr(other, name), want, name)
        tune.close(getattr(alone, name), want, name)  # up to four rows go their own way
    tune.close(again.dhidden, want, "dhidden")
    tune.close(again.dweight, want, "dweight")
    wide = w.shape[1] >= 512
    if b is not None:
        tune.close(again.dbias, want, "dbias")
        assert kept.dbias is None
        fine = tune.head(h, w, b, tokens, temperature, gl, gh, on, kept=23) if wide else want  # (from 1024 on where the logits are many)
        tune.close(grads.dhidden, fine, "dhidden")
        tune.close(grads.dweight, fine, "dweight")
        tune.close(grads.dbias, fine, "dbias")
    else:
        assert torch.equal(kept.dhidden, grads.dhidden) and torch.equal(kept.dweight, grads.dweight) and grads.dbias is None
    if wide:
        want = tune.head(h, w, b, tokens, temperature, gl, gh, on, kept=16)
    tune.close(kept.dhidden, want, "dhidden")
    tune.close(kept.dweight, want, "dweight")
    evaluate.linear_check_status()


HEADS = [
    # R, V, D, dtype, bias, temperature, entropy, pad of hidden, pad of weight
    (1, 1, 1, BF16, None, 1.0, False, 0, 0), (1, 1000, 64, BF16, None, 1.0, False, 0, 0), (2, 255, 8, F16, "same", 1.0, True, 0, 0),
    (1, 257, 72, F16, F32, 0.7, True, 0, 0), (31, 256, 128, BF16, "same", 1.0, False, 8, 0), (33, 511, 100, BF16, F32, 2.0, True, 4, 4),
    (128, 512, 256, F16, None, 1.0, False, 0, 0), (129, 700, 65, BF16, "same", 1.0, True, 3, 5), (255, 1025, 200, F16, F32, 1.3, False, 0, 8),
    (256, 2048, 64, BF16, None, 1.0, True, 0, 0), (257, 2049, 136, F16, None, 0.5, False, 1, 1), (513, 999, 264, BF16, F32, 1.0, True, 0, 0),
    (1000, 3001, 96, BF16, "same", 1.0, False, 0, 0), (700, 64, 1000, F16, F32, 1.0, True, 22, 0), (3, 5000, 520, BF16, F32, 1.0, True, 0, 0),
    (2000, 3, 16, F16, "same", 1.0, True, 0, 0), (40, 4100, 1, BF16, None, 1.0, True, 0, 0),
    (1, 30001, 768, BF16, F32, 1.0, False, 0, 0), (4, 20003, 264, F16, "same", 0.9, True, 8, 0), (4, 1003, 77, BF16, None, 1.0, True, 0, 3), (2, 5003, 1030, F16, F32, 0.7, True, 1, 0), (5, 1003, 77, BF16, None, 1.0, False, 0, 3),
]


@gpu
@pytest.mark.parametrize("R,V,D,dtype,bias,temperature,entropy,padh,padw", HEADS)
def test_against_the_formula(R, V, D, dtype, bias, temperature, entropy, padh, padw):
    h, w, tokens, b = head(R, V, D, dtype, bias, padh, padw)
    check(h, w, b, tokens, temperature, *weights(R, dtype, entropy))


@gpu
@pytest.mark.parametrize("R,V,D,dtype", [
    (70000, 4500, 64, BF16),      # pieces of the least width
    (9000, 33000, 72, F16),       # pieces that the budget sets, the last one shorter
    (300, 20000, 520, BF16),      # the summed index of dhidden shared among multiprocessors
    (20000, 300, 40, F16),        # that of dweight
    (9000, 40000, 1024, BF16),    # two pieces of rows (three with dbias)
    (9001, 70001, 520, F16),      # three, odd ends
    (5000, 70001, 1032, F16),     # two with dbias
    (700, 5003, 600, F16),        # all rows at once
    (5, 3000, 640, BF16),
    (512, 30001, 96, BF16),
    (11000, 70001, 40, BF16),     # two pieces of rows for the values
    (512, 30001, 512, F16),
])
@pytest.mark.parametrize("entropy", [False, True])
def test_pieces_and_shares(R, V, D, dtype, entropy):
    h, w, tokens, b = head(R, V, D, dtype, F32)
    check(h, w, b, tokens, 1.0, *weights(R, dtype, entropy), on="cuda")


@gpu
def test_rows_that_are_not_finite_in_one_of_several_pieces():
    R, V, D = 9000, 40000, 512  # two pieces of rows
    h, w, tokens, b = head(R, V, D, BF16)
    gl, _ = weights(R, BF16, False)
    clean = evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl)
    h[8000, 5] = math.nan
    out, grads = evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl)
    rest = torch.arange(R, device="cuda") != 8000
    assert torch.equal(out.lse[rest], clean[0].lse[rest]) and torch.equal(grads.dhidden[rest], clean[1].dhidden[rest])
    assert torch.isnan(out.lse[8000]) and torch.isnan(grads.dhidden[8000]).all()


@gpu
@pytest.mark.parametrize("bits", [torch.int32, torch.int64])
def test_tokens_that_are_none_or_beyond(bits):
    h, w, tokens, b = head(50, 300, 64, BF16)
    tokens[0], tokens[1], tokens[2], tokens[3] = 299, 300, 2 ** 31 - 1, -1
    gl, gh = weights(50, BF16, False)
    tokens = tokens.to(bits)
    want = tune.head(h, w, None, tokens, 1.0, gl, gh)
    out, grads = evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl, gh)
    tune.close(out.logprob, want, "logprob")
    tune.close(grads.dhidden, want, "dhidden")
    assert torch.isnan(grads.dhidden[1:3]).all() and torch.isnan(grads.dweight).all()
    assert (grads.dhidden[3] == 0).all() and out.logprob[3] == 0


@gpu
@pytest.mark.parametrize("entropy", [False, True])
@pytest.mark.parametrize("low", [-INF, -1e9, -1e30, float(torch.finfo(F32).min)])
@pytest.mark.parametrize("D,dtype", [(96, BF16), (512, BF16), (520, F16)])
def test_ids_that_are_not_allowed(low, entropy, D, dtype):
    h, w, tokens, b = head(100, 777, D, dtype, F32)
    allowed = torch.rand(777, generator=torch.Generator().manual_seed(3)) < 0.3
    allowed[256:512] = False  # a tile without any
    b = torch.where(allowed.cuda(), b, torch.full_like(b, low))
    ids = allowed.nonzero()[:, 0].cuda()
    tokens = torch.where(tokens >= 0, ids[tokens.clamp(min=0) % ids.numel()], tokens)
    gl, gh = weights(100, dtype, entropy)
    check(h, w, torch.where(allowed.cuda(), b, torch.full_like(b, -INF)) if low < -1e8 else b, tokens, 1.0, gl, gh)
    got, grads = evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl, gh, b)
    want = tune.head(h, w, torch.where(allowed.cuda(), b, torch.full_like(b, -INF)), tokens, 1.0, gl, gh)
    for name in ("logprob", "entropy", "lse"):
        tune.close(getattr(got, name), want, name)
    if D >= 512:
        want = tune.head(h, w, torch.where(allowed.cuda(), b, torch.full_like(b, -INF)), tokens, 1.0, gl, gh, kept=23)
    for name in ("dhidden", "dweight", "dbias"):
        tune.close(getattr(grads, name), want, name)
    kept = evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl, gh, b, wanted=("hidden", "weight"))[1]
    for g in (grads, kept):
        assert (g.dweight[~allowed.cuda()] == 0).all()
    assert (grads.dbias[~allowed.cuda()] == 0).all()


@gpu
@pytest.mark.parametrize("D", [64, 512])
def test_rows_with_nothing_left(D):
    h, w, tokens, _ = head(40, 300, D, F16)
    b = torch.full((300,), -INF, device="cuda")
    gl, gh = weights(40, F16, True)
    out, grads = evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl, gh, b)
    again = evaluate.linear_token_logprobs_backward(h, w, tokens, out.lse, out.entropy, gl, gh, b)
    assert (out.lse == -INF).all() and (out.entropy == 0).all()
    assert (out.logprob[tokens >= 0] == -INF).all() and (out.logprob[tokens < 0] == 0).all()
    kept = evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl, gh, b, wanted=("hidden", "weight"))[1]
    for g in (grads, again, kept):
        assert (g.dhidden == 0).all() and (g.dweight == 0).all() and (g.dbias is None or (g.dbias == 0).all())


@gpu
def test_all_ids_under_a_finite_mask():
    h, w, tokens, _ = head(40, 300, 64, BF16)
    tokens = tokens.clamp(min=0)
    b = torch.full((300,), -1e30, device="cuda")  # every logit is the same number
    out, grads = evaluate.linear_token_logprobs_with_grad(h, w, tokens, torch.ones(40, device="cuda"), None, b)
    assert torch.allclose(out.logprob.cpu(), torch.full((40,), -math.log(300.0)), rtol=1e-6, atol=0)
    assert torch.allclose(out.entropy.cpu(), torch.full((40,), math.log(300.0)), rtol=1e-6, atol=0)
    assert (grads.dbias.sum().abs() < 1e-4).item() and torch.isfinite(grads.dhidden).all()


@gpu
@pytest.mark.parametrize("D", [64, 512])
def test_values_that_are_not_finite_stay_in_their_rows(D):
    h, w, tokens, b = head(70, 600, D, BF16)
    gl, gh = weights(70, BF16, True)
    clean = evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl, gh)
    h[5, 3], h[40, 0] = math.nan, INF
    out, grads = evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl, gh)
    rest = torch.ones(70, dtype=torch.bool, device="cuda")
    rest[5] = rest[40] = False
    for name in ("lse", "entropy", "logprob"):
        a, c = getattr(out, name), getattr(clean[0], name)
        assert torch.equal(a[rest], c[rest]), name
        assert torch.isnan(a[5]) or (name == "logprob" and tokens[5] < 0)
        assert torch.isnan(a[40]) or (name == "logprob" and tokens[40] < 0)
    assert torch.isnan(grads.dhidden[5]).all() and torch.isnan(grads.dhidden[40]).all()
    assert torch.equal(grads.dhidden[rest], clean[1].dhidden[rest])
    b = torch.zeros(600, device="cuda")
    b[599] = INF
    assert torch.isnan(evaluate.linear_token_logprobs(h, w, tokens, b).lse).all()
    few = evaluate.linear_token_logprobs(h[4:7], w, tokens[4:7])
    assert torch.isnan(few.lse).tolist() == [False, True, False] and torch.isnan(few.entropy).tolist() == [False, True, False]
    assert torch.isnan(evaluate.linear_token_logprobs(h[4:7], w, tokens[4:7], b).lse).all()
    b.fill_(-INF)
    few = evaluate.linear_token_logprobs(h[6:8], w, tokens[6:8].clamp(min=0), b)
    assert (few.lse == -INF).all() and (few.logprob == -INF).all() and (few.entropy == 0).all()


@gpu
@pytest.mark.parametrize("D", [64, 72, 100, 520])
def test_outputs_with_strides_leave_their_neighbours(D):
    R, V = 130, 520
    h, w, tokens, b = head(R, V, D, BF16, F32)
    gl, gh = weights(R, BF16, False)
    want = evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl, gh, b)[1]
    dh, dw = rand(R, D, dtype=BF16, pad=5, shift=1), rand(V, D, dtype=BF16, pad=3, shift=1)
    whole = [t._base.clone() for t in (dh, dw)]
    got = evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl, gh, b, dhidden=dh, dweight=dw)[1]
    assert got.dhidden is dh and got.dweight is dw
    assert torch.equal(dh, want.dhidden) and torch.equal(dw, want.dweight) and torch.equal(got.dbias, want.dbias)
    for before, t in zip(whole, (dh, dw)):
        before[:, 1:1 + D] = t
        assert torch.equal(before, t._base)
    for wanted in (("hidden",), ("weight",), ("bias",), ()):
        some = evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl, gh, b, wanted=wanted)[1]
        for name in ("hidden", "weight", "bias"):
            a, c = getattr(some, "d" + name), getattr(want, "d" + name)
            assert (a is None) if name not in wanted else torch.equal(a, c) or (D >= 512 and "bias" not in wanted)
    for out in ({}, {"dhidden": dh, "dweight": dw}):
        kept = evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl, gh, b, wanted=("hidden", "weight"), **out)[1]
        want = tune.head(h, w, b, tokens, 1.0, gl, gh, kept=16 if D >= 512 else 0)
        tune.close(kept.dhidden, want, "dhidden")
        tune.close(kept.dweight, want, "dweight")


@gpu
@pytest.mark.parametrize("R,dtype", [(1, BF16), (3, F16), (4, BF16)])
def test_few_rows_with_all_but_certain_tokens(R, dtype):
    # 1 - p is all that is left of the gradient at the token: p itself has to be right to fp32's last places
    V, D = 3001, 2048
    h, w, tokens, b = head(R, V, D, dtype, F32)
    tokens = tokens.clamp(min=0)
    h.copy_((0.5 * rand(R, D, seed=5) + 1.5 * w[tokens].float()).to(dtype))
    gl, _ = weights(R, dtype, False)
    want = tune.head(h, w, b, tokens, 0.7, gl, None)
    out, grads = evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl, None, b, 0.7)
    assert (want["logprob"] > -0.02).all()
    exact = (torch.exp(want["logprob"]) - 1).abs() * gl.cpu().double().abs() / 0.7
    got = grads.dbias[tokens].cpu().double().abs()
    # products added in fp32 by 32 lanes, 64 each: within 80 roundings of magnitudes that sum to about 30 a logit, twice, and lse's own
    assert ((got - exact).abs() <= gl.cpu().double().abs() * (200 * 2.0 ** -24 * 40 + 2.0 ** -20)).all()
    tune.close(out.logprob, want, "logprob")


@gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("entropy", [False, True])
def test_many_rows_with_all_but_certain_tokens(dtype, entropy):
    # the gradient at the token is 1 - p, which kept logits would not hold
    R, V, D = 100, 3001, 512
    h, w, tokens, b = head(R, V, D, dtype, F32)
    tokens = tokens.clamp(min=0)
    h.copy_((0.5 * rand(R, D, seed=5) + 1.5 * w[tokens].float()).to(dtype))
    gl, gh = weights(R, dtype, entropy)
    want = tune.head(h, w, b, tokens, 0.7, gl, gh)
    assert want["logprob"].median() > -0.01
    check(h, w, b, tokens, 0.7, gl, gh)
    check(h, w, None, tokens, 0.7, gl, gh)
    kept = evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl, gh, b, 0.7, wanted=("hidden", "weight"))[1]
    off = (kept.dhidden.cpu().double() - want["dhidden"]).norm() / want["dhidden"].norm()
    assert off < 2.5 * ref.HALF_ULP[dtype]  # two roundings and the kept logits'


@gpu
def test_no_rows():
    h, w, tokens, b = head(5, 30, 16, BF16, F32)
    none = torch.zeros(0, device="cuda")
    out, grads = evaluate.linear_token_logprobs_with_grad(h[:0], w, tokens[:0], none, None, b)
    assert out.lse.shape == (0,) and grads.dhidden.shape == (0, 16)
    assert (grads.dweight == 0).all() and (grads.dbias == 0).all()


@gpu
@pytest.mark.parametrize("D,wanted,dtype", [(128, ("hidden", "weight", "bias"), BF16), (512, ("hidden", "weight"), BF16), (520, ("weight", "hidden"), F16)])
def test_the_same_call_gives_the_same_bits_on_any_stream_and_in_a_graph(D, wanted, dtype):
    h, w, tokens, b = head(600, 9000, D, dtype, F32)
    gl, gh = weights(600, dtype, True)

    def call(stream=None):
        out, grads = evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl, gh, b, wanted=wanted, stream=stream)
        more = evaluate.linear_token_logprobs_backward(h, w, tokens, out.lse, out.entropy, gl, gh, b, wanted=wanted, stream=stream)
        return [t for t in (out.logprob, out.entropy, out.lse, *grads, *more) if t is not None]

    want = call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = call(side)
    side.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    graphs = []
    for _ in range(2):  # two graphs, replayed in turn, each with its own workspace
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            kept = call()
        graphs.append((g, kept))
    for _ in range(2):
        for g, kept in graphs:
            for t in kept:
                t.zero_()
            g.replay()
    torch.cuda.synchronize()
    for _, kept in graphs:
        assert all(torch.equal(a, c) for a, c in zip(kept, want))


@gpu
def test_gradients_against_differences():
    R, V, D = 60, 500, 64
    h, w, tokens, b = head(R, V, D, BF16, F32)
    tokens = tokens.clamp(min=0)
    gl, gh = torch.ones(R, device="cuda"), torch.full((R,), 0.5, device="cuda")
    _, grads = evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl, gh, b)

    def value(h, w, b):
        out = evaluate.linear_token_logprobs(h, w, tokens, b)
        return (gl * out.logprob + gh * out.entropy).double().sum()

    # Steps uphill that 16 bits hold: every eighth element moves by 2^-6 of its power of two.
    for name, key, t in (("dhidden", "h", h), ("dweight", "w", w), ("dbias", "b", b)):
        grad = getattr(grads, name).double()
        size = torch.exp2(torch.floor(torch.log2(t.float().abs().clamp(min=2.0 ** -20))) - 6) * torch.sign(grad).float()
        size = torch.where(rand(*t.shape, seed=9) > 1.15, size, torch.zeros_like(size))
        up, down = (t.float() + size).to(t.dtype), (t.float() - size).to(t.dtype)
        step = (up.double() - down.double()) / 2
        args = {"h": h, "w": w, "b": b}
        change = (value(**{**args, key: up}) - value(**{**args, key: down})) / 2
        along, size = (grad * step).sum(), (grad * step).abs().sum()
        if key == "h":
            dz = (step @ w.double().T).abs().amax(1)
        elif key == "w":
            dz = (h.double() @ step.T).abs().amax(1)
        else:
            dz = step.abs().amax().expand(R)
        # Left over: the third derivative of lse along the step (at most (2 dz)^3 a row, the entropy's within three times that), the gradient's
        # 16 bits, and the values' own fp32 (the tensor core's sums among them).
        bound = (2.5 * (2 * dz) ** 3 / 6).sum() + 2.0 ** -7 * size + R * 2e-5
        assert (change - along).abs() < bound, (name, float(change), float(along), float(bound))
        assert bound < along.abs(), (name, float(along), float(bound))


@gpu
def test_python_refusals_on_the_device():
    h, w, tokens, b = head(8, 30, 16, BF16, F32)
    call = evaluate.linear_token_logprobs_with_grad
    with pytest.raises(ValueError, match="weight"):
        call(h, w.half(), tokens)
    with pytest.raises(ValueError, match="weight"):
        call(h, w[:, :8], tokens)
    with pytest.raises(ValueError, match="bias"):
        call(h, w, tokens, bias=b.half())
    with pytest.raises(ValueError, match="bias"):
        call(h, w, tokens, bias=b[:5])
    with pytest.raises(ValueError, match="tokens"):
        call(h, w, tokens[:4])
    with pytest.raises(ValueError, match="tokens"):
        call(h, w, tokens.float())
    with pytest.raises(ValueError, match="grad_logprob"):
        call(h, w, tokens, torch.ones(8, device="cuda", dtype=BF16))
    with pytest.raises(ValueError, match="wanted"):
        call(h, w, tokens, wanted=("head",))
    with pytest.raises(ValueError, match="wanted"):
        call(h, w, tokens, wanted=("weight",), dhidden=torch.empty_like(h))
    with pytest.raises(ValueError, match="dweight"):
        call(h, w, tokens, dweight=torch.empty(30, 16, device="cuda"))
    with pytest.raises(ValueError, match="requires a gradient"):
        call(h.clone().requires_grad_(), w, tokens)
    for t in (0.0, -1.0, math.nan, INF):
        with pytest.raises(binding.SpdyError):
            call(h, w, tokens, temperature=t)
    with pytest.raises(binding.SpdyError):
        evaluate.linear_token_logprobs_backward(h, w, tokens, torch.zeros(8, device="cuda"), grad_entropy=torch.ones(8, device="cuda"))
    with pytest.raises(binding.SpdyError):
        call(h, w, tokens, torch.ones(8, device="cuda"), dhidden=h)


# ------------------------------------------------------------------------------------------------ without a GPU

def test_c_entries_refuse_bad_arguments_before_any_gpu_work():
    lib = evaluate.library()
    P, Q = 1 << 20, 1 << 30  # pointers that are never followed
    first = [P, 64, P + (1 << 16), 64, 1, None, 1, P, 64, 9, 100, 64, 1.0]
    forward = first + [P, P, P, P, 1 << 40, None]
    backward = first + [P, P, P, P, Q, 64, Q + (1 << 20), 64, P, P, 1 << 40, None]
    both = first + [P, P, P, P, P, Q, 64, Q + (1 << 20), 64, P, P, 1 << 40, None]

    def bad(fn, args, *changes):
        args = list(args)
        for at, v in changes:
            args[at] = v
        return fn(*args)

    for fn, args in ((lib.spdy_linear_token_logprobs, forward), (lib.spdy_linear_token_logprobs_backward, backward),
                     (lib.spdy_linear_token_logprobs_with_grad, both)):
        for change in ((0, None), (0, P + 1), (1, 63), (2, None), (2, P + 1), (3, 63), (4, 0), (4, 3), (7, P + 4), (8, 16), (9, -1), (10, 0), (11, 0),
                       (9, 1 << 31), (10, 1 << 31), (11, 1 << 31), (12, 0.0), (12, -1.0), (12, math.nan), (12, INF), (7, None)):
            assert bad(fn, args, change) == -1, (fn, change)
        assert bad(fn, args, (5, P), (6, 2)) == -1      # bias of another 16-bit type
        assert bad(fn, args, (5, P + 2), (6, 0)) == -1  # misaligned bias
        assert bad(fn, args, (-3, None)) == -1 and bad(fn, args, (-3, P + 8)) == -1 and bad(fn, args, (-2, 8)) == -2
    for change in ((13, None), (17, Q + 1), (18, 63), (19, Q + 1), (20, 63), (14, None)):
        assert bad(lib.spdy_linear_token_logprobs_backward, backward, change) == -1, change
    for change in ((18, Q + 1), (19, 63), (20, Q + 1), (21, 63)):
        assert bad(lib.spdy_linear_token_logprobs_with_grad, both, change) == -1, change
    for change in ((18, P), (20, P), (18, P + (1 << 16)), (20, P + (1 << 16) + 100)):  # gradients over the inputs
        assert bad(lib.spdy_linear_token_logprobs_with_grad, both, change) == -1, change
    assert bad(lib.spdy_linear_token_logprobs, forward, (9, 0)) == 0


def test_workspace_stays_bounded():
    lib = evaluate.library()
    P = 1 << 20

    def need(R, V, D, forward, gradients, ld=None):
        return lib.spdy_linear_token_logprobs_workspace_bytes(P, ld or D, P, ld or D, 1, R, V, D, forward, gradients)

    assert need(0, 100, 64, 1, 1) == 0 and need(10, 0, 64, 1, 1) == 0
    assert need(8192, 131072, 4096, 1, 0) < 40 << 20                    # forward: 12 bytes per row and tile of 256 ids, of some rows
    assert need(1 << 20, 131072, 4096, 1, 0) < 40 << 20
    assert need(8192, 131072, 4096, 0, 1) < (256 + 200) << 20           # a piece of 256 MB and dhidden's fp32 sums
    assert need(8192, 65536, 4096, 1, 1) < (512 + 1024 + 200) << 20     # some rows' logits and gradient, fp32 sums of dweight
    assert need(4096, 65536, 4096, 1, 1) < (512 + 250) << 20            # all rows at once
    assert need(8192, 65536, 4096, 1, 2) < (512 + 1024 + 250) << 20     # with dbias
    assert need(8192, 200000, 4096, 1, 1) < (256 + 200 + 80) << 20      # fewer than 2048 rows would fit: the same
    assert need(1 << 20, 131072, 64, 0, 1) < (4096 + 700) << 20         # 2048 ids at least
    assert need(64, 5000, 100, 1, 0, ld=101) >= need(64, 5000, 104, 1, 0) + 5000 * 100 * 2  # copies of rows that TMA cannot read


def test_cpu_tensors_are_refused():
    x = torch.zeros(2, 8, dtype=BF16)
    t = torch.zeros(2, dtype=torch.int64)
    with pytest.raises(ValueError, match="CUDA"):
        evaluate.linear_token_logprobs(x, x, t)
    with pytest.raises(ValueError, match="bfloat16"):
        evaluate.linear_token_logprobs(x.float(), x.float(), t)
