"""The evaluation operators from their formulas in 64 bits (PyTorch on the CPU, no fused calls): what the tests of
``paper_2201_13096_b200.evaluate`` compare with."""
import math

import torch

HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}
INF = math.inf


def d64(t):
    return t.detach().cpu().double()


def activation(z, kind):
    if kind == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if kind == "gelu":
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))
    if kind == "silu":
        return torch.where(z == -INF, torch.zeros_like(z), z * torch.sigmoid(z))
    return z


def linear(x, w, b, res, kind):
    """(y, bound on the fp32 error before the last rounding)."""
    x, w = d64(x), d64(w)
    K = x.shape[1]
    z, size = x @ w.T, x.abs() @ w.abs().T
    if b is not None:
        z, size = z + d64(b), size + d64(b).abs()
    y = activation(z, kind)
    # K products added in fp32 in some order (the tensor core keeps at least 24 bits of each partial sum and may cut rather
    # than round): each of about K / 8 + 16 additions loses at most 2^-23 of the sum of magnitudes; the activations' slopes
    # stay below 1.2 and their own evaluation within 2^-20 of |z|
    err = 1.2 * (K / 8 + 16) * 2.0 ** -23 * size + 2.0 ** -20 * z.abs()
    if res is not None:
        y = y + d64(res)
        err = err + 2.0 ** -23 * y.abs()
    return y, err


def layer_norm(x, w, b, eps):
    x = d64(x)
    mean = x.mean(1, keepdim=True)
    var = ((x - mean) ** 2).mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt(var + eps)
    y = (x - mean) * rstd
    if w is not None:
        y = y * d64(w)
    if b is not None:
        y = y + d64(b)
    return y, mean[:, 0], rstd[:, 0]


def layer_norm_backward(dy, x, w, mean, rstd):
    dy, x, mean, rstd = d64(dy), d64(x), d64(mean)[:, None], d64(rstd)[:, None]
    h = (x - mean) * rstd
    u = dy if w is None else dy * d64(w)
    dx = rstd * (u - u.mean(1, keepdim=True) - h * (u * h).mean(1, keepdim=True))
    return dx, (dy * h).sum(0), dy.sum(0)


def softmax_row(x, temperature):
    """(log p, p, lse) of rows; a row of -inf alone has lse -inf, p 0 and log p -inf."""
    t = d64(x) / temperature
    lse = torch.logsumexp(t, 1)
    logp = torch.where(torch.isneginf(lse)[:, None], torch.full_like(t, -INF), t - lse[:, None])
    bad = torch.isnan(t).any(1) | torch.isposinf(t).any(1)
    lse = torch.where(bad, torch.full_like(lse, math.nan), lse)
    logp = torch.where(bad[:, None], torch.full_like(logp, math.nan), logp)
    return logp, logp.exp(), lse


def token_logprobs(x, tokens, temperature):
    logp, p, lse = softmax_row(x, temperature)
    tokens = tokens.cpu().long()
    V = x.shape[1]
    lp = logp.gather(1, tokens.clamp(0, V - 1)[:, None])[:, 0]
    lp = torch.where(tokens < 0, torch.zeros_like(lp), torch.where(tokens >= V, torch.full_like(lp, math.nan), lp))
    entropy = -torch.where(p == 0, torch.zeros_like(p), p * logp).sum(1)
    return lp, entropy, lse


def top(x, k):
    """Ids of the k largest logits of each row, equal ones by ascending id, NaN below -inf."""
    x = d64(x)
    rows = []
    for row in x.tolist():
        rows.append(sorted(range(len(row)), key=lambda i: (row[i] != row[i], -row[i] if row[i] == row[i] else 0.0, i))[:k])
    return torch.tensor(rows, dtype=torch.int64).reshape(x.shape[0], k)


def token_logprobs_grad(x, tokens, gl, gh, temperature):
    logp, p, _ = softmax_row(x, temperature)
    V = x.shape[1]
    tokens = tokens.cpu().long()
    entropy = -torch.where(p == 0, torch.zeros_like(p), p * logp).sum(1, keepdim=True)
    gl = torch.zeros(x.shape[0], dtype=torch.float64) if gl is None else torch.where(tokens < 0, 0.0, d64(gl))
    gh = torch.zeros(x.shape[0], dtype=torch.float64) if gh is None else d64(gh)
    hit = (torch.arange(V)[None, :] == tokens[:, None]).double()
    d = gl[:, None] * (hit - p) - gh[:, None] * torch.where(p == 0, torch.zeros_like(p), p * (logp + entropy))
    d = torch.where(torch.isneginf(d64(x)).all(1)[:, None], torch.zeros_like(d), d)
    if gl is not None:
        d = torch.where((tokens >= V)[:, None], torch.full_like(d, math.nan), d)
    return d / temperature


def distill(x, ids, lps, temperature, tail, g=None):
    """(loss, lse, rest, gradient or None) row by row from the definition."""
    logp, p, lse = softmax_row(x, temperature)
    t = d64(x) / temperature
    ids, lps = ids.cpu().long(), d64(lps)
    R, V = t.shape
    loss, rest = torch.zeros(R, dtype=torch.float64), torch.full((R,), -INF, dtype=torch.float64)
    grad = torch.zeros(R, V, dtype=torch.float64)
    for r in range(R):
        here = [j for j in range(ids.shape[1]) if ids[r, j] >= 0]
        if any(int(ids[r, j]) >= V for j in here):
            loss[r], grad[r] = math.nan, math.nan
            inside = sorted({int(ids[r, j]) for j in here if int(ids[r, j]) < V})
            outside = [v for v in range(V) if v not in set(inside)]
            rest[r] = torch.logsumexp(t[r, outside], 0) if outside else -INF
            continue
        if tail:
            q = {j: math.exp(lps[r, j]) for j in here}
            logq = {j: float(lps[r, j]) for j in here}
            left = max(0.0, 1.0 - sum(q.values()))
        else:
            finite = [float(lps[r, j]) for j in here if lps[r, j] > -INF]
            top_lp = max(finite) if finite else 0.0
            total = sum(math.exp(v - top_lp) for v in finite)
            logq = {j: (float(lps[r, j]) - top_lp - math.log(total)) if total > 0 else -INF for j in here}
            q = {j: math.exp(logq[j]) for j in here}
            left = 0.0
        inside = sorted({int(ids[r, j]) for j in here})
        mask = torch.ones(V, dtype=torch.bool)
        mask[inside] = False
        rest[r] = torch.logsumexp(t[r, mask], 0) if mask.any() else -INF
        value = sum(q[j] * (logq[j] - float(logp[r, int(ids[r, j])])) for j in here if q[j] > 0)
        if torch.isnan(lse[r]):
            rest[r] = math.nan if (torch.isnan(t[r, mask]) | torch.isposinf(t[r, mask])).any() else rest[r]
        if not tail or torch.isneginf(rest[r]):
            left = 0.0
        elif left > 0:
            value += left * (math.log(left) - float(rest[r] - lse[r]))
        loss[r] = value
        mass = sum(q.values()) + left
        if g is not None and not torch.isneginf(lse[r]):
            d = mass * p[r]
            if tail and left > 0:
                d = d - torch.where(mask, left * torch.exp(t[r] - rest[r]), torch.zeros(V, dtype=torch.float64))
            for j in here:
                d[int(ids[r, j])] -= q[j]
            grad[r] = d * float(g[r]) / temperature
    return loss, lse, rest, grad


def same_special(a, b):
    """Equal positions of NaN and of the infinities."""
    return bool(torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.isinf(a), torch.isinf(b))
                and torch.equal(a[torch.isinf(a)], b[torch.isinf(b)]))


def close(got, want, err, what=""):
    """Every element within ``err`` plus half a unit in the last place of the result's type."""
    t = got.dtype
    got = d64(got)
    big = want.abs() > (3.3e38 if t != torch.float16 else 65520.0)
    assert same_special(torch.where(big, torch.zeros_like(got), got), torch.where(big, torch.zeros_like(want), want)), f"{what}: special values differ"
    ok = torch.isfinite(want) & ~big
    off = (got - want).abs()[ok]
    bound = (torch.as_tensor(err, dtype=torch.float64).expand(want.shape)[ok] * 1.0 + 1.01 * HALF_ULP[t] * want.abs()[ok] + TINY[t])
    worst = (off - bound).max() if off.numel() else torch.tensor(-1.0)
    assert worst <= 0, f"{what}: off by {float(off.max()):.3g}, {float((off / bound).max()):.3g} times the bound"
