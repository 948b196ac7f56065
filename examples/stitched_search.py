"""SPDY's search with a real evaluation: the calibration loss of a stitched model, computed by this package's operators.

The model is a stack of BERT-style feed-forward blocks over a small vocabulary with random weights:

    h = embedding(tokens);  per block  h = layer_norm(linear(gelu(linear(h, W1) + b1), W2) + b2 + h);  logits = linear(h, W_out)

Every linear layer of the blocks can be pruned to each sparsity of the grid of Section 4 (the database holds its weights with the
smallest magnitudes removed), and the search picks one sparsity per layer within a time budget.  A profile's loss
(``eval_fn``, Section 3.4) is the distillation loss of the model stitched together for it against the dense model's most
probable tokens.  Afterwards the last normalisation of the chosen model is tuned against the dense model for a few steps, and with
``--answer-steps`` it is tuned on the dense model's best tokens together with the output layer, by AdamW with moments in 8 bits.

    python examples/stitched_search.py [--blocks 2] [--hidden 256] [--speedup 2.5] ...
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2201_13096_b200 import binding, evaluate, search, workloads  # noqa: E402


class StitchedModel:
    """The dense model, its database of pruned layers, and the calibration batch."""

    def __init__(self, blocks: int, hidden: int, ffn: int, vocabulary: int, tokens: int, sparsities, top_k: int, seed: int = 0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def randn(*shape, scale):
            return (torch.randn(*shape, generator=g, device="cuda") * scale).to(torch.bfloat16)

        self.embedding = randn(vocabulary, hidden, scale=1.0)
        self.head = randn(vocabulary, hidden, scale=3.0 * hidden ** -0.5)
        self.head_by_input = self.head.t().contiguous()  # laid out once for the gradient's product
        self.norms, self.biases, self.database = [], [], []  # per block; per layer; per layer and choice
        for _ in range(blocks):
            self.norms.append((torch.ones(hidden, device="cuda"), torch.zeros(hidden, device="cuda")))
            for n, k in ((ffn, hidden), (hidden, ffn)):
                dense = randn(n, k, scale=1.5 * k ** -0.5)
                order = dense.float().abs().flatten().sort().values
                self.biases.append(randn(n, scale=0.1))
                self.database.append([torch.where(dense.float().abs() < order[int(s * (order.numel() - 1))], 0, dense) if s > 0 else dense
                                      for s in sparsities])
        self.ids = torch.randint(0, vocabulary, (tokens,), generator=g, device="cuda")
        logits, _ = self.forward([0] * len(self.database))
        dense = evaluate.token_logprobs(logits, logits.argmax(dim=1), top_k=top_k)
        self.top_ids, self.top_logprobs = dense.top_ids, dense.top_logprobs  # the dense model's answers, kept for good

    def hidden(self, profile):
        """What the output layer sees in the model stitched together for ``profile`` (a choice per layer), and the last normalisation's
        input and statistics."""
        h = self.embedding[self.ids]
        for b, (weight, bias) in enumerate(self.norms):
            up, down = 2 * b, 2 * b + 1
            inner = evaluate.linear(h, self.database[up][profile[up]], bias=self.biases[up], activation="gelu")
            last = evaluate.linear(inner, self.database[down][profile[down]], bias=self.biases[down], residual=h)
            h, mean, rstd = evaluate.layer_norm(last, weight, bias)
        return h, (last, mean, rstd)

    def forward(self, profile):
        """Logits of the stitched model, and the last normalisation's input and statistics."""
        h, last = self.hidden(profile)
        return evaluate.linear(h, self.head), last

    def loss(self, profile) -> float:
        """The search's ``eval_fn``: +inf for an infeasible profile (bytes 0xFF)."""
        if (np.asarray(profile) >= len(self.database[0])).any():
            return float("inf")
        logits, _ = self.forward([int(c) for c in profile])
        return float(evaluate.distill_loss(logits, self.top_ids, self.top_logprobs).loss.mean())

    def tune(self, profile, steps: int, rate: float):
        """Gradient steps on the last normalisation's weight and bias; the loss before each."""
        profile, losses = [int(c) for c in profile], []
        per_row = torch.full((self.ids.numel(),), 1.0 / self.ids.numel(), device="cuda")
        for _ in range(steps):
            logits, (x, mean, rstd) = self.forward(profile)
            weight, bias = self.norms[-1]
            out, dlogits = evaluate.distill_loss_with_grad(logits, self.top_ids, self.top_logprobs, per_row, out=logits)
            losses.append(float(out.loss.mean()))
            dh = evaluate.linear(dlogits, self.head_by_input)
            _, dweight, dbias = evaluate.layer_norm_backward(dh, x, weight, mean, rstd)
            self.norms[-1] = (weight - rate * dweight, bias - rate * dbias)
        return losses

    def answer_gradients(self, profile):
        """Mean log probability of the dense model's best tokens, and the gradients of its negative by the output layer's weight and the last
        normalisation's weight and bias.  No table of logits is made."""
        h, (x, mean, rstd) = self.hidden([int(c) for c in profile])
        weight, _ = self.norms[-1]
        tokens = self.top_ids[:, 0].contiguous()
        per_row = torch.full((self.ids.numel(),), -1.0 / self.ids.numel(), device="cuda")
        out, grads = evaluate.linear_token_logprobs_with_grad(h, self.head, tokens, per_row)
        _, dweight, dbias = evaluate.layer_norm_backward(grads.dhidden, x, weight, mean, rstd)
        return out.logprob.mean(), [grads.dweight, dweight, dbias]

    def tune_on_answers(self, profile, steps: int, rate: float):
        """AdamW steps on the output layer and the last normalisation; the loss before each."""
        weight, bias = (t.clone() for t in self.norms[-1])
        self.norms[-1] = (weight, bias)
        plan = evaluate.AdamW([self.head, weight, bias], bits=8, weight_decay=[0.01, 0.0, 0.0], rounding="stochastic")
        losses = []
        for step in range(1, steps + 1):
            logprob, grads = self.answer_gradients(profile)
            losses.append(-float(logprob))
            evaluate.adamw_step(plan, grads, lr=rate, step=step, seed=step)
        self.head_by_input = self.head.t().contiguous()
        return losses


def main(argv=None) -> dict:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--blocks", type=int, default=2)
    ap.add_argument("--hidden", type=int, default=256)
    ap.add_argument("--ffn", type=int, default=1024)
    ap.add_argument("--vocabulary", type=int, default=8000)
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--choices", type=int, default=8, help="sparsities per layer, the dense one among them")
    ap.add_argument("--top-k", type=int, default=32)
    ap.add_argument("--speedup", type=float, default=2.5)
    ap.add_argument("--budget", type=int, default=1000, help="time buckets")
    ap.add_argument("--trials", type=int, default=30)
    ap.add_argument("--tune-steps", type=int, default=10)
    ap.add_argument("--answer-steps", type=int, default=0)
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args(argv)

    sparsities = workloads.sparsity_levels(a.choices, 0.95)
    model = StitchedModel(a.blocks, a.hidden, a.ffn, a.vocabulary, a.tokens, sparsities, a.top_k, a.seed)
    macs = np.asarray([a.hidden * a.ffn] * (2 * a.blocks), dtype=np.float64)
    times = workloads.make_times(macs / macs.sum() * (a.speedup * a.budget), sparsities)
    L = times.shape[0]
    samples = workloads.sensitivity_samples(a.seed, L, a.trials + 1)
    found = search.search(times, a.budget, samples[0], samples[1:], workloads.mutation_draws(a.seed, L), model.loss, trials=a.trials)
    uniform, _ = binding.uniform_profile(times, a.budget)
    out = {"dense": model.loss([0] * L), "uniform": model.loss([uniform] * L), "searched": found["loss"],
           "profile": [int(c) for c in found["profile"]], "time": int(sum(times[i][c] for i, c in enumerate(found["profile"]))),
           "budget": a.budget, "evals": found["evals"]}
    out["tuning"] = model.tune(found["profile"], a.tune_steps, rate=0.5)
    out["tuned"] = model.loss(found["profile"])
    if a.answer_steps:
        out["answers"] = model.tune_on_answers(found["profile"], a.answer_steps, rate=1e-3)
    return out


if __name__ == "__main__":
    result = main()
    for key, value in result.items():
        print(f"{key:>9}: {value}")
