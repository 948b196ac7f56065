"""The evaluation operators where many or long rows take other ways through the kernels than a few: persistent blocks, rings
that wrap around, one block per long row, several segments of the teacher's bitmap.  All rows are worked on, some are compared."""

import pytest
import torch

import eval_reference as ref
from paper_2201_13096_b200 import build as build_mod, evaluate
from test_evaluate import BF16, F16, F32, norm_bounds, sizes_of, teacher_of, twin

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.fixture(scope="module", autouse=True)
def built():
    build_mod.build()


def rand(R, C, seed, dtype, pad=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((R, C + pad), 7.0, dtype=dtype, device="cuda")
    buf[:, :C] = torch.randn(R, C, generator=g, device="cuda") * scale
    return buf[:, :C] if pad else buf


def some_rows(R, count, seed):
    rows = torch.randperm(R, generator=torch.Generator().manual_seed(seed))[:count].tolist()
    return torch.tensor(sorted({0, 1, R - 2, R - 1, *rows}))


# rows of 26 MB or more in all, of every length class, starting on 16 bytes or anywhere
NORMS = [(100001, 136, 0), (100000, 131, 0), (33000, 401, 3), (33001, 512, 0), (18001, 768, 0), (18000, 761, 0), (13001, 1024, 8), (14000, 999, 0), (7001, 2000, 0), (7000, 2047, 0),
         (3300, 4096, 0), (3301, 4093, 1), (1700, 8192, 0), (1701, 8190, 3), (900, 16000, 0), (901, 15999, 0)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("R,D,pad", NORMS)
def test_layer_norm_of_many_rows(dtype, R, D, pad):
    x = rand(R, D, 1, dtype, pad, 2.0)
    x += 0.5
    dy = rand(R, D, 2, dtype)
    at = some_rows(R, 300, 3)
    xs, dys = x[at.cuda()], dy[at.cuda()]
    for params in (dtype, F32, None):
        w = None if params is None else (1.0 + 0.2 * rand(1, D, 3, F32)[0]).to(params)
        b = None if params is None else (0.3 * rand(1, D, 4, F32)[0]).to(params)
        y, mean, rstd = evaluate.layer_norm(x, w, b)
        want, mean64, rstd64 = ref.layer_norm(xs, w, b, 1e-5)
        ref.close(mean[at.cuda()], mean64, 2.0 ** -20 * ref.d64(xs).abs().mean(1), "mean")
        ref.close(rstd[at.cuda()], rstd64, 2.0 ** -20 * rstd64 * (1 + (mean64 * rstd64) ** 2 * 2.0 ** -10), "rstd")
        ref.close(y[at.cuda()], want, norm_bounds(xs, w, b, want, rstd64), "y")
        over = twin(x)
        assert torch.equal(evaluate.layer_norm(over, w, b, out=over)[0], y)
        if pad:
            assert bool((over._base[:, D:] == x._base[:, D:]).all())
        dx, dw, db = evaluate.layer_norm_backward(dy, x, w, mean, rstd)
        m, s = mean[at.cuda()], rstd[at.cuda()]
        dx64, _, _ = ref.layer_norm_backward(dys, xs, w, m, s)
        h = (ref.d64(xs) - ref.d64(m)[:, None]) * ref.d64(s)[:, None]
        u = ref.d64(dys) * (1.0 if w is None else ref.d64(w))
        # as for few rows: h within 2^-22 of (|x| + |mean|) rstd, the row's two means within 2^-20 of their magnitudes
        eh = 2.0 ** -22 * (ref.d64(xs).abs() + ref.d64(m).abs()[:, None]) * ref.d64(s)[:, None]
        part = u.abs() + u.abs().mean(1, keepdim=True) + (h.abs() + 1) * (u * h).abs().mean(1, keepdim=True)
        assert bool(torch.isfinite(dx).all())  # nothing left out
        ref.close(dx[at.cuda()], dx64, ref.d64(s)[:, None] * (2.0 ** -19 * part + eh * (u * h).abs().mean(1, keepdim=True) + h.abs() * (u.abs() * eh).mean(1, keepdim=True)), "dx")
        # the columns' sums over all rows, in 64 bits on the device: a thread's chain of R / (rows in flight) additions, then the
        # groups' and blocks', each within 2^-24 of the sum of magnitudes
        hd = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
        d = dy.double()
        levels = R / 148 + 40
        eh_sum = (d.abs() * 2.0 ** -22 * (x.double().abs() + mean.double().abs()[:, None]) * rstd.double()[:, None]).sum(0).cpu()
        ref.close(dw, (d * hd).sum(0).cpu(), 2.0 ** -24 * levels * (d * hd).abs().sum(0).cpu() + eh_sum, "dweight")
        ref.close(db, d.sum(0).cpu(), 2.0 ** -24 * levels * d.abs().sum(0).cpu(), "dbias")
        over = twin(x)
        assert torch.equal(evaluate.layer_norm_backward(dy, over, w, mean, rstd, out=over, params=False)[0], dx)


LONG = [(700, 3000, 0), (601, 9001, 0), (300, 34001, 3), (301, 66000, 0), (300, 140003, 0)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("R,V,pad", LONG)
def test_token_logprobs_of_many_long_rows(dtype, R, V, pad):
    x = rand(R, V, 5, dtype, pad, 3.0)
    x[3, V // 2:] = -INF
    tokens = torch.randint(-1, V, (R,), generator=torch.Generator().manual_seed(1)).cuda()
    at = torch.unique(torch.cat([some_rows(R, 8, 2), torch.tensor([3])]))
    k = 20
    got = evaluate.token_logprobs(x, tokens, top_k=k, temperature=0.7)
    xs, ts = x[at.cuda()], tokens[at.cuda()]
    lp, h, lse = ref.token_logprobs(xs, ts, 0.7)
    a = sizes_of(xs, 0.7)
    err = 2.0 ** -21 * (a + 14)
    ref.close(got.lse[at.cuda()], lse, err, "lse")
    ref.close(got.logprob[at.cuda()], lp, err, "logprob")
    ref.close(got.entropy[at.cuda()], h, 4 * err, "entropy")
    assert torch.equal(got.top_ids[at.cuda()].cpu().long(), ref.top(xs, k))
    gl, gh = rand(1, R, 6, F32)[0], rand(1, R, 7, F32)[0]
    both, grad = evaluate.token_logprobs_with_grad(x, tokens, gl, gh, temperature=0.7)
    for u, v in zip(both[:3], evaluate.token_logprobs(x, tokens, temperature=0.7)[:3]):
        ref.close(u[at.cuda()], ref.d64(v[at.cuda()]), 4 * err * 2, "with_grad's sums")
    want = ref.token_logprobs_grad(xs, ts, gl[at.cuda()], gh[at.cuda()], 0.7)
    _, p, _ = ref.softmax_row(xs, 0.7)
    logp = torch.where(p == 0, torch.zeros_like(p), p.log().abs())
    # p within 2 err of itself, log p + H within 5 err; the products' terms one by one
    size = ref.d64(gl[at.cuda()]).abs()[:, None] * p + ref.d64(gh[at.cuda()]).abs()[:, None] * p * (logp + h[:, None])
    bound = (8 * err[:, None] * (size + ref.d64(gh[at.cuda()]).abs()[:, None] * p) + 2.0 ** -20 * (size + want.abs())) / 0.7
    ref.close(grad[at.cuda()], want, bound, "gradient")
    assert bool(torch.isfinite(grad).all())
    over = twin(x)
    assert torch.equal(evaluate.token_logprobs_with_grad(over, tokens, gl, gh, temperature=0.7, out=over)[1], grad)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("R,V,pad", LONG)
@pytest.mark.parametrize("tail", [True, False])
def test_distillation_of_many_long_rows(dtype, R, V, pad, tail):
    x = rand(R, V, 8, dtype, pad, 3.0)
    K = 40
    at = some_rows(R, 6, 4)
    xs = x[at.cuda()]
    top_ids, top_lps = evaluate.token_logprobs(x, torch.zeros(R, dtype=torch.int64, device="cuda"), top_k=K)[3:]
    ids, lps = top_ids.long(), top_lps.clone()
    some, some_lps = teacher_of(xs, K, 1.0, 11)
    ids[at.cuda()], lps[at.cuda()] = some, some_lps
    g = rand(1, R, 9, F32)[0]
    loss, lse, rest, want = ref.distill(xs, ids[at.cuda()], lps[at.cuda()], 1.0, tail, g[at.cuda()].cpu())
    e = 2.0 ** -21 * (sizes_of(xs, 1.0) + 14)
    el = e + 2.0 ** -20 * (sizes_of(xs, 1.0) + 30) * (1 + K / 64)
    got = evaluate.distill_loss(x, ids, lps, tail=tail)
    ref.close(got.loss[at.cuda()], loss, el * 2, "loss")
    ref.close(got.lse[at.cuda()], lse, e, "lse")
    if tail:
        ref.close(got.rest[at.cuda()], rest, e, "rest")
    both, grad = evaluate.distill_loss_with_grad(x, ids, lps, g, tail=tail)
    ref.close(both.loss[at.cuda()], loss, el * 2, "with_grad's loss")
    _, p, _ = ref.softmax_row(xs, 1.0)
    rel = 2 * e[:, None] + 2.0 ** -20
    outside = torch.exp(ref.d64(xs) - rest[:, None])
    inside = torch.zeros(len(at), V, dtype=torch.float64).scatter_(1, ids[at.cuda()].cpu(), 1.0)
    err = ref.d64(g[at.cuda()]).abs()[:, None] * (
        rel * (p + inside) + (1 - inside) * outside * (2.0 ** -21 * (K / 32 + 8) + rel * 2 * torch.exp(rest - lse)[:, None]) * float(tail))
    ref.close(grad[at.cuda()], want, err + rel * want.abs(), "gradient")
    assert bool(torch.isfinite(grad).all())
    over = twin(x)
    assert torch.equal(evaluate.distill_loss_with_grad(over, ids, lps, g, tail=tail, out=over)[1], grad)
