"""AdamW steps at the edges of their formats and of autograd (include/spdy_eval.h, spdy_adamw_*)."""
import math

import pytest
import torch

import eval_reference as ref
import tune_reference as tune
from paper_2201_13096_b200 import build as build_mod, evaluate
from test_adamw import gradient, snapshot, values

gpu = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    build_mod.build()


@gpu
@pytest.mark.parametrize("large,small", [(1.0, 1e-12), (1e6, 1e-3), (1e6, 1e-12), (1e8, 1e-5), (1e12, 1e-1), (1e18, 1e-3), (1e20, 1e-18)])
def test_second_moments_beside_large_ones_have_a_floor(large, small):
    # 0.001 g^2 of the large one is 2^10 to 2^126: the conversion's power of two is no float of one step from 2^30 on.  The small one's is a positive
    # number, 2^-32 of the largest or less, and has to stay one.
    g = torch.zeros(64, device="cuda")
    g[0], g[1], g[17], g[40] = large, small, small, small  # the last in a block of its own
    plan = evaluate.AdamW([torch.ones(64, device="cuda")], bits=8)
    evaluate.adamw_step(plan, [g], lr=0.0, step=1)
    v = evaluate.adamw_moments(plan)[0][1].double()
    assert abs(float(v[0]) / (0.001 * float(g[0].double()) ** 2) - 1) <= 2.0 ** -3  # a step of the mantissa's three bits
    unit = 2.0 ** (math.floor(math.log2(0.001 * float(g[0].double()) ** 2)) - 32)
    assert float(v[1]) == float(v[17]) == unit  # the least number of the block
    assert float(v[40]) > 0 and int((v > 0).sum()) == 4


@gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype,master", [(torch.float32, False), (torch.bfloat16, True), (torch.float16, False)])
@pytest.mark.parametrize("rate,decay,eps", [(math.inf, 0.0, 1e-8), (math.nan, 0.1, 1e-8), (1e30, 3e38, 1e-8), (math.inf, 0.1, 0.0), (1e30, 3e38, 0.0), (0.1, 0.1, 0.0)])
def test_zeros_are_kept_whatever_the_rate(rate, decay, eps, dtype, master, bits):
    for n in (77, 4096):
        w = (values(n, 1) * (values(n, 2) > 0)).cuda().to(dtype)
        gone = w == 0
        plan = evaluate.AdamW([w], bits=bits, masters=True if master else None, weight_decay=decay, eps=eps, keep_zeros=True)
        lr, step = torch.full((1,), rate, device="cuda"), torch.ones(1, dtype=torch.int64, device="cuda")
        for given in ((lr, step), (rate, 1)) if math.isfinite(rate) else ((lr, step),):
            evaluate.adamw_step(plan, [gradient(n, 3).cuda().to(dtype)], lr=given[0], step=given[1])
            assert (w[gone] == 0).all() and 0 < int(gone.sum()) < n
            for t in plan.masters + [m for pair in evaluate.adamw_moments(plan) for m in pair]:
                assert t is None or (t[gone] == 0).all()


@gpu
@pytest.mark.parametrize("eps", [1e-60, 1e-45, 1e-39, 1e-37, 1e-30, 1e-12])
def test_an_eps_below_the_normal_numbers(eps):
    # no gradient and no moments: 0 / eps is 0, and the weights stay
    w = values(100, 1).cuda()
    before = w.clone()
    plan = evaluate.AdamW([w], weight_decay=0.0, eps=eps)
    evaluate.adamw_step(plan, [torch.zeros(100, device="cuda")], lr=0.1, step=1)
    assert torch.equal(w, before)
    # a moment of eps's size beside a second one of 0: m / eps, where fp32 has it.  Roundings of 0.9 m and of it times the rate, at least 2^-150 of fp32's
    # least normal numbers each, quotient and decay as the header has them.
    small = float(torch.tensor(eps, dtype=torch.float64).float())
    if small < 1e-39:
        return
    m = torch.full((100,), 10.0, dtype=torch.float64).mul(small).float()
    plan = evaluate.AdamW([w], weight_decay=0.0, eps=eps, moments=[evaluate.AdamWMoments(m.cuda(), torch.zeros(100, device="cuda"))])
    evaluate.adamw_step(plan, [torch.zeros(100, device="cuda")], lr=1.0, step=100000)
    change = 0.9 * m.double() / small
    cut = 2 * 2.0 ** -150 / (9 * small) + 2.0 ** -21 + 2.0 ** -22
    assert ((ref.d64(w) - (ref.d64(before) - change)).abs() <= change * cut + 2.0 ** -23 * 10).all()


@gpu
@pytest.mark.parametrize("beta2", [0.999, 1 - 1e-9, 1 - 1e-12])
def test_second_moments_below_the_normal_numbers(beta2):
    # a first step from 0: m / (1 - beta1) = g, and sqrt(v / (1 - beta2)) = |g| shows beside eps although v itself is below 2^-126
    g = torch.logspace(-16, -11, 200, dtype=torch.float64).float()
    w = torch.zeros(200, device="cuda")
    plan = evaluate.AdamW([w], weight_decay=0.0, eps=1e-9, betas=(0.9, beta2))
    evaluate.adamw_step(plan, [g.cuda()], lr=1.0, step=1)
    want = -g.double() / (g.double() + 1e-9)
    v = (1 - beta2) * g.double() ** 2
    # v is off by up to 2^-149 (its factor's product and its own) beside the relative errors, at most all of it; the rest as in tune_reference.adamw
    off = (2.0 ** -149 / v).clamp(max=1.0) * g.double() / (g.double() + 1e-9)
    assert ((ref.d64(w) - want).abs() <= want.abs() * (off + 2.0 ** -18)).all()


def _frozen(w):
    return w


def _detached(w):
    return w.detach()


@gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("taken", [_frozen, _detached])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_graphs_notice_steps_on_weights_that_require_no_gradient(dtype, taken, bits):
    w = torch.randn(64, 8, device="cuda").to(dtype)
    plan = evaluate.AdamW([taken(w), torch.ones(5, device="cuda")], bits=bits, masters=[torch.zeros(64 * 8, device="cuda") if dtype != torch.float32 else None, None])
    grads = [torch.ones(64, 8, device="cuda", dtype=dtype), None]
    x = torch.randn(3, 8, device="cuda").to(dtype).requires_grad_()
    saved = [w, plan.params[1]] + ([plan.masters[0]] if plan.masters[0] is not None else []) + ([plan.moments[0].m, plan.moments[0].v] if bits == 32 else [])
    for t in saved:
        y = (x @ t.T).sum() if t is w else (t * torch.ones_like(t).requires_grad_()).sum()
        before = t._version
        evaluate.adamw_step(plan, grads, lr=0.1, step=1)
        if t is plan.params[1]:  # no gradient, no step
            assert t._version == before
            y.backward()
            continue
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()


@gpu
def test_graphs_notice_steps_on_a_weight_unfrozen_later():
    w = torch.randn(64, device="cuda")
    plan = evaluate.AdamW([w])
    w.requires_grad_()
    y = (w * w).sum()
    evaluate.adamw_step(plan, [torch.ones(64, device="cuda")], lr=0.1, step=1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    (w * w).sum().backward()  # and after the step it is a leaf like any other
    assert torch.equal(w.grad, 2 * w.detach())


@gpu
def test_tensors_of_inference_mode_can_be_stepped():
    with torch.inference_mode():
        w = torch.ones(64, device="cuda")
        plan = evaluate.AdamW([w])
        evaluate.adamw_step(plan, [torch.ones(64, device="cuda")], lr=0.1, step=1)
    evaluate.adamw_step(plan, [torch.ones(64, device="cuda")], lr=0.1, step=2)
    assert (w < 0.9).all()
