"""The operators of tuning (a head's log probabilities with gradients, the AdamW step) from their formulas in 64 bits, with the error that
their kernels may make: what the tests compare with."""
import math

import torch

import eval_reference as ref

F16 = torch.float16


def head(hidden, weight, bias, tokens, temperature, gl=None, gh=None, on="cpu"):
    """A dict of values and, under the same name with ``_err``, of bounds on the fp32 error before the last rounding."""
    h, w = (t.detach().to(on).double() for t in (hidden, weight))
    R, D = h.shape
    V = w.shape[0]
    x, size = h @ w.T, h.abs() @ w.abs().T
    if bias is not None:
        b = bias.detach().to(on).double()
        x, size = x + b, size + torch.where(torch.isfinite(b), b.abs(), torch.zeros_like(b))
    tokens = tokens.to(on).long()
    logp, p, lse = ref_softmax(x, temperature)
    # Logits: D products added in fp32, see eval_reference.linear.  Only ids with a share count: an id's error moves lse by p times itself.
    ez = ((D / 8 + 16) * 2.0 ** -23 * size / temperature)
    ez = torch.where(p > 0, ez, torch.zeros_like(ez)).nan_to_num(0.0).amax(1)
    named = (tokens >= 0) & (tokens < V)
    at = tokens.clamp(0, V - 1)[:, None]
    lp = logp.gather(1, at)[:, 0]
    ez_token = ((D / 8 + 16) * 2.0 ** -23 * size / temperature).gather(1, at)[:, 0]
    lp = torch.where(tokens < 0, torch.zeros_like(lp), torch.where(tokens >= V, torch.full_like(lp, math.nan), lp))
    spread = torch.where(p == 0, torch.zeros_like(p), p * logp)
    entropy = -spread.sum(1)
    # Sums over V terms: 64 in a row in a warp, joined over 4 warps, 16 shares of the tiles, 16 warps; terms from the special-function unit
    # (2^-22) with arguments rounded twice (2^-23 of themselves, at most 0.37 after weighting by the term).
    adds = (64 + 4 + V / 4096 + 16 + 16) * 2.0 ** -24 + 2.0 ** -21
    out = {"logprob": lp, "entropy": entropy, "lse": lse}
    out["lse_err"] = ez + adds + 2.0 ** -22 * lse.abs().nan_to_num(0.0, posinf=0.0, neginf=0.0)
    out["logprob_err"] = torch.where(named, ez + ez_token + adds + 2.0 ** -21 * lp.abs().nan_to_num(0.0, posinf=0.0, neginf=0.0), torch.zeros_like(ez))
    out["entropy_err"] = (2 * entropy.nan_to_num(0.0) + 2) * (ez + adds)
    if gl is None and gh is None:
        return out
    a = torch.zeros(R, dtype=torch.float64, device=h.device) if gl is None else torch.where(tokens < 0, 0.0, gl.to(on).double())
    b = torch.zeros(R, dtype=torch.float64, device=h.device) if gh is None else gh.to(on).double()
    empty = torch.isneginf(lse)
    a, b = torch.where(empty, 0.0, a), torch.where(empty, 0.0, b)
    dead = p == 0
    logs = torch.where(dead, torch.zeros_like(logp), logp)
    p = torch.where(empty[:, None], torch.zeros_like(p), p)
    g = -p * (a[:, None] + b[:, None] * (logs + entropy[:, None]))
    g[torch.arange(R, device=h.device)[named], tokens[named]] += a[named]
    if gl is not None:
        g[tokens >= V] = math.nan
    g = g / temperature
    # p is off by the errors of its logit and of lse (as saved, in fp32), and by the roundings of the exponent
    off = 3 * ez + adds + 2.0 ** -22 * (lse.abs().nan_to_num(0.0, posinf=0.0, neginf=0.0) + 4)
    share = p * (a.abs()[:, None] + b.abs()[:, None] * (logs.abs() + entropy[:, None] + 1)) / temperature
    eg = share * (off[:, None] + 2.0 ** -21 * logs.abs()) + 2.0 ** -23 * g.abs()
    most = float(((a.abs() + b.abs() * (0.37 + entropy)) / temperature).nan_to_num(0.0).max()) if R else 0.0
    rounded = eg + ref.HALF_ULP[hidden.dtype] * 1.01 * (g.abs() + eg) + (2.0 ** -38 * most if hidden.dtype == F16 else 2.0 ** -134)
    out["dhidden"], out["dweight"], out["dbias"] = g @ w, g.T @ h, g.sum(0)
    out["dhidden_err"] = rounded @ w.abs() + (V / 8 + 16 + V / 1024) * 2.0 ** -23 * (g.abs() @ w.abs())
    out["dweight_err"] = rounded.T @ h.abs() + (R / 8 + 16 + 64) * 2.0 ** -23 * (g.abs().T @ h.abs())
    out["dbias_err"] = eg.sum(0) + (R / 256 + 16) * 2.0 ** -24 * g.abs().sum(0)
    return out


def ref_softmax(x, temperature):
    t = x / temperature
    lse = torch.logsumexp(t, 1)
    logp = torch.where(torch.isneginf(lse)[:, None], torch.full_like(t, -math.inf), t - lse[:, None])
    bad = torch.isnan(t).any(1) | torch.isposinf(t).any(1)
    lse = torch.where(bad, torch.full_like(lse, math.nan), lse)
    logp = torch.where(bad[:, None], torch.full_like(logp, math.nan), logp)
    return logp, logp.exp(), lse


def close(got, want, name):
    ref.close(got, want[name].cpu(), want[name + "_err"].cpu(), name)
