"""Tensors that callers give to be written (paper_2201_13096_b200/evaluate.py): a graph that saved one notices."""
import pytest
import torch

from paper_2201_13096_b200 import build as build_mod, evaluate

gpu = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def built():
    build_mod.build()


def randn(*shape, dtype=BF16):
    return torch.randn(*shape, device="cuda").to(dtype)


def calls():
    x, w, logits = randn(6, 16), randn(6, 16), randn(6, 16)
    tokens, gl = torch.arange(6, device="cuda"), torch.ones(6, device="cuda")
    top = evaluate.token_logprobs(logits, tokens, top_k=4)
    ids, lps, lse = top.top_ids, top.top_logprobs, top.lse
    rest = evaluate.distill_loss(logits, ids, lps).rest
    _, mean, rstd = evaluate.layer_norm(x)
    return {
        "linear": lambda t: evaluate.linear(x, randn(16, 16), out=t),
        "layer_norm": lambda t: evaluate.layer_norm(x, out=t),
        "layer_norm_backward": lambda t: evaluate.layer_norm_backward(x, x, None, mean, rstd, out=t),
        "token_logprobs_backward": lambda t: evaluate.token_logprobs_backward(logits, tokens, lse, grad_logprob=gl, out=t),
        "token_logprobs_with_grad": lambda t: evaluate.token_logprobs_with_grad(logits, tokens, gl, out=t),
        "distill_loss_backward": lambda t: evaluate.distill_loss_backward(logits, ids, lps, lse, rest, gl, out=t),
        "distill_loss_with_grad": lambda t: evaluate.distill_loss_with_grad(logits, ids, lps, gl, out=t),
        "dhidden": lambda t: evaluate.linear_token_logprobs_with_grad(x, w, tokens, gl, dhidden=t),
        "dweight": lambda t: evaluate.linear_token_logprobs_backward(x, w, tokens, lse, grad_logprob=gl, dweight=t),
    }


@gpu
@pytest.mark.parametrize("name", ["linear", "layer_norm", "layer_norm_backward", "token_logprobs_backward", "token_logprobs_with_grad", "distill_loss_backward",
                                  "distill_loss_with_grad", "dhidden", "dweight"])
def test_a_graph_notices_that_a_tensor_it_saved_was_written(name):
    call, t = calls()[name], randn(6, 16)
    x = randn(6, 16).requires_grad_()
    y = (x * t).sum()
    call(t)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    (x * t).sum().backward()
    assert torch.equal(x.grad, t)
    with torch.inference_mode():
        u = randn(6, 16)
    call(u)  # has no versions
    assert torch.isfinite(u).all()
