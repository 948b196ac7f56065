"""A head's log probabilities and gradients: single outputs, and how exact logits are (include/spdy_eval.h, spdy_linear_token_logprobs*)."""
import pytest
import torch

from paper_2201_13096_b200 import build as build_mod, evaluate
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
