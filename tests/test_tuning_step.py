"""The operators of tuning run together, as a user does: a normalisation, a head without a table of logits, their gradients, and AdamW."""
import os
import sys

import pytest
import torch

import eval_reference as ref
import tune_reference as tune
from paper_2201_13096_b200 import build as build_mod, evaluate
from test_evaluate import rand

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module", autouse=True)
def built():
    build_mod.build()


class Tail:
    """The last normalisation and the output layer of a model, half of whose weights are pruned away."""

    def __init__(self, R, V, D, seed=0):
        self.x = rand(R, D, seed=seed, dtype=BF16)
        self.head = rand(V, D, seed=seed + 1, dtype=BF16, scale=2.0 * D ** -0.5)
        self.head[rand(V, D, seed=seed + 2) > 0] = 0
        self.weight, self.bias = 1.0 + 0.1 * rand(D, seed=seed + 3), 0.1 * rand(D, seed=seed + 4)
        self.tokens = torch.randint(0, V, (R,), generator=torch.Generator().manual_seed(seed)).cuda()
        self.tokens[::7] = -1
        self.per_row = torch.full((R,), -1.0 / R, device="cuda")

    def gradients(self):
        h, mean, rstd = evaluate.layer_norm(self.x, self.weight, self.bias)
        out, grads = evaluate.linear_token_logprobs_with_grad(h, self.head, self.tokens, self.per_row)
        dx, dweight, dbias = evaluate.layer_norm_backward(grads.dhidden, self.x, self.weight, mean, rstd)
        return out, h, dx, [grads.dweight, dweight, dbias]

    def params(self):
        return [self.head, self.weight, self.bias]


@pytest.mark.parametrize("R,V,D", [(300, 2000, 64), (300, 2000, 512)])
def test_gradients_of_the_whole_against_autograd_in_64_bits(R, V, D):
    tail = Tail(R, V, D)
    out, h, dx, grads = tail.gradients()
    x, head, weight, bias = (t.detach().double().requires_grad_() for t in (tail.x, *tail.params()))
    normed = torch.nn.functional.layer_norm(x, (D,), weight, bias)
    logp = torch.log_softmax(normed @ head.T, 1)
    named = tail.tokens >= 0
    picked = torch.where(named, logp.gather(1, tail.tokens.clamp(min=0)[:, None])[:, 0], torch.zeros_like(logp[:, 0]))
    (picked * tail.per_row.double()).sum().backward()
    assert (out.logprob.double() - picked).abs().max() < 0.05  # h is rounded to 16 bits: logits of up to 8 move by 2^-8 of their terms
    # 16 bits hold h (in the head's gradient a factor), g and dhidden: three roundings of at most 2^-8 each, whose signs do not agree
    for got, want in zip([dx, *grads], (x.grad, head.grad, weight.grad, bias.grad)):
        assert ((got.double() - want).norm() / want.norm()).item() < 3 * 2.0 ** -8


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_eager_and_replayed_give_the_same_bits(bits):
    def run(graphed):
        tail = Tail(200, 1500, 512)
        plan = evaluate.AdamW(tail.params(), bits=bits, keep_zeros=[True, False, False], weight_decay=[0.01, 0.0, 0.0], rounding="stochastic")
        step, lr = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.full((1,), 2.0 ** -10, device="cuda")
        source = tail.x.clone()
        side = torch.cuda.Stream()

        def once():
            tail.x.copy_(source)  # a copy before, and work on another stream that this waits for
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                step.add_(1)
            torch.cuda.current_stream().wait_stream(side)
            _, _, _, grads = tail.gradients()
            evaluate.adamw_step(plan, grads, lr=lr, step=step, seed=11)
            return grads

        if graphed:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                kept = once()
            step.zero_()
            for _ in range(4):
                g.replay()
            del kept
        else:
            for _ in range(4):
                once()
        torch.cuda.synchronize()
        return tail, list(plan._written())

    pruned = Tail(200, 1500, 512).head == 0
    (tail, eager), (_, replayed) = run(False), run(True)
    for a, b in zip(eager, replayed):
        assert torch.equal(a, b)
    assert (tail.head[pruned] == 0).all() and (tail.head[~pruned] != Tail(200, 1500, 512).head[~pruned]).any()
    evaluate.linear_check_status()


def test_two_streams_at_once():
    tails = [Tail(700, 9000, 512, seed) for seed in (0, 20)]
    want = [t.gradients() for t in tails]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in tails]
    for _ in range(3):
        got = []
        for t, s in zip(tails, streams):
            with torch.cuda.stream(s):
                got.append(t.gradients())
        torch.cuda.synchronize()
        for (a, _, adx, ag), (b, _, bdx, bg) in zip(got, want):
            assert torch.equal(a.lse, b.lse) and torch.equal(adx, bdx) and all(torch.equal(x, y) for x, y in zip(ag, bg))
    evaluate.linear_check_status()


def test_the_example_tunes_on_answers_and_its_gradients():
    import stitched_search

    out = stitched_search.main(["--trials", "4", "--tune-steps", "2", "--answer-steps", "3"])
    assert len(out["answers"]) == 3 and all(0.0 < v < 20.0 for v in out["answers"])
    model = stitched_search.StitchedModel(1, 128, 256, 1000, 64, [0.0, 0.5], 4)
    logprob, (dhead, dweight, dbias) = model.answer_gradients([0, 1])
    h, (x, mean, rstd) = model.hidden([0, 1])
    want = tune.head(h, model.head, None, model.top_ids[:, 0], 1.0, torch.full((64,), -1.0 / 64.0), None)
    assert abs(float(logprob) - float(want["logprob"].mean())) < 1e-3
    tune.close(dhead, want, "dweight")
    dh = evaluate.linear_token_logprobs_with_grad(h, model.head, model.top_ids[:, 0].contiguous(), torch.full((64,), -1.0 / 64.0, device="cuda"))[1].dhidden
    _, ndw, ndb = ref.layer_norm_backward(dh, x, model.norms[-1][0], mean, rstd)
    for got, exact in ((dweight, ndw), (dbias, ndb)):
        assert ((ref.d64(got) - exact).norm() / exact.norm()).item() < 1e-5
