"""An output layer whose weight, hidden states or gradients hold more than 2^31 elements."""
import pytest
import torch

import tune_reference as tune
from paper_2201_13096_b200 import build as build_mod, evaluate

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def built():
    build_mod.build()


def normal(rows, columns, scale, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = torch.empty(rows, columns, dtype=BF16, device="cuda")
    for a in range(0, rows, 65536):
        out[a:a + 65536] = torch.randn(min(65536, rows - a), columns, generator=g, device="cuda") * scale
    return out


@pytest.mark.parametrize("R", [3, 40])
def test_weights_beyond_32_bits(R):
    V, D, tail = 530_000, 4096, 2000
    assert V * D > 1 << 31
    h, w = normal(R, D, 1.0, 0), normal(V, D, 2.0 / 64.0, 1)
    tokens = torch.randint(V - tail, V, (R,), device="cuda")  # their rows' gradients lie at the far end
    gl = -torch.rand(R, device="cuda") - 0.5
    out, grads = evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl)
    logits = torch.cat([h.double() @ w[a:a + 40000].double().T for a in range(0, V, 40000)], 1)
    lse = torch.logsumexp(logits, 1)
    # 4096 products of magnitudes that sum to about 80: see tune_reference.head
    error = (4096 / 8 + 16) * 2.0 ** -23 * 80
    assert ((out.lse.double() - lse).abs() < error).all()
    assert ((out.logprob.double() - (logits.gather(1, tokens[:, None])[:, 0] - lse)).abs() < 2 * error).all()
    d = -torch.exp(logits - lse[:, None]) * gl.double()[:, None]
    d.scatter_add_(1, tokens[:, None], gl.double()[:, None])
    for part in (slice(V - tail, V), slice(0, 500), slice(V // 2, V // 2 + 500)):
        want = d[:, part].T @ h.double()
        assert (grads.dweight[part].double() - want).norm() < 2 * 2.0 ** -8 * want.norm()  # two roundings to 16 bits
    want = sum(d[:, a:a + 40000] @ w[a:a + 40000].double() for a in range(0, V, 40000))
    assert (grads.dhidden.double() - want).norm() < 2 * 2.0 ** -8 * want.norm()
    evaluate.linear_check_status()


def test_rows_beyond_32_bits():
    R, V, D, tail = 530_000, 300, 4096, 300
    assert R * D > 1 << 31
    h, w = normal(R, D, 1.0, 2), normal(V, D, 2.0 / 64.0, 3)
    tokens = torch.randint(0, V, (R,), device="cuda")
    gl = torch.zeros(R, device="cuda")
    gl[-tail:] = -1.0 / tail  # only the far rows count, so that dweight is theirs alone
    gl[:50] = -1.0 / tail
    for wanted in (("hidden", "weight"), ("hidden", "weight", "bias")):
        b = torch.zeros(V, device="cuda") if "bias" in wanted else None
        out, grads = evaluate.linear_token_logprobs_with_grad(h, w, tokens, gl, None, b, wanted=wanted)
        rows = torch.cat([torch.arange(50, device="cuda"), torch.arange(R - tail, R, device="cuda")])
        want = tune.head(h[rows], w, b, tokens[rows], 1.0, gl[rows], None, "cuda", kept=16 if b is None else 23)
        for name in ("lse", "logprob", "entropy"):
            tune.close(getattr(out, name)[rows], want, name)
        tune.close(grads.dhidden[rows], want, "dhidden")
        # R products are added up, nearly all of them 0
        want["dweight_err"] = want["dweight_err"] + (R / 8 + 16) * 2.0 ** -23 * want["dweight"].abs()
        tune.close(grads.dweight, want, "dweight")
        assert (grads.dhidden[50:R - tail] == 0).all()
    evaluate.linear_check_status()
