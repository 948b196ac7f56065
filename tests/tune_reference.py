"""The operators of tuning (a head's log probabilities with gradients, the AdamW step) from their formulas in 64 bits, with the error that
their kernels may make: what the tests compare with."""
import math

import torch

import eval_reference as ref

F16 = torch.float16


def head(hidden, weight, bias, tokens, temperature, gl=None, gh=None, on="cpu", kept=0, cut=None, halves=1):
    """A dict of values and, under the same name with ``_err``, of bounds on the fp32 error before the last rounding.
    ``kept``: the gradient comes from logits kept in so many bits, as a call that gives values and gradients keeps them: 16, or 23 with
    dbias; the token's own is not among them.
    ``halves``: in how many numbers of 16 bits the gradient by the logits goes into the products.
    ``cut``: by how much of its magnitudes a logit may be off, where that is known better than from the number of products."""
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
    cut = (D / 8 + 16) * 2.0 ** -23 if cut is None else cut
    ez = (cut * size / temperature)
    ez = torch.where(p > 0, ez, torch.zeros_like(ez)).nan_to_num(0.0).amax(1)
    named = (tokens >= 0) & (tokens < V)
    at = tokens.clamp(0, V - 1)[:, None]
    lp = logp.gather(1, at)[:, 0]
    ez_token = (cut * size / temperature).gather(1, at)[:, 0]
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
    if kept:  # log2 p in steps of 2^-10 (half precision 2^-11), or 2^-7 of that, off by half a step; 64 (32) octaves below a neighbour p counts as 0
        steps, octaves = (2.0 ** -11, 32) if hidden.dtype == F16 else (2.0 ** -10, 64)
        more = share * (steps * 2.0 ** (16 - kept) / 2 * math.log(2) * 1.001)
        more = more + 2.0 ** -octaves * (a.abs() + b.abs() * (octaves + entropy)).nan_to_num(0.0)[:, None] / temperature
        more[torch.arange(R, device=h.device)[named], tokens[named]] = 0.0
        eg = eg + more
    # Half precision: a power of two brings the largest bound on a row's gradient, |a| + |b| (0.37 + log V), to 2^13 .. 2^14, where numbers below the
    # normal ones are rounded by 2^-25: 2^-38 of that bound.
    most = float(((a.abs() + b.abs() * (0.37 + math.log(V))) / temperature).nan_to_num(0.0).max()) if R else 0.0
    rounded = eg + ref.HALF_ULP[hidden.dtype] ** halves * 1.01 * (g.abs() + eg) + (2.0 ** -38 * most if hidden.dtype == F16 else 2.0 ** -134)
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


# ------------------------------------------------------------------------------------------------ AdamW

def mix(x):
    """The hash, on uint64 arrays that hold 32 bits."""
    import numpy as np
    m = np.uint64(0xFFFFFFFF)
    x = np.asarray(x, dtype=np.uint64) & m
    x = ((x ^ (x >> np.uint64(16))) * np.uint64(0x7FEB352D)) & m
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0x846CA68B)) & m
    return x ^ (x >> np.uint64(16))


def random_bits(seed, step, tensor, n, first=0):
    import numpy as np
    key = int(mix(int(mix(int(mix(seed)) + step)) + tensor))
    e = np.arange(first, first + n, dtype=np.uint64)
    return torch.from_numpy(mix((e & np.uint64(0xFFFFFFFF)) + np.uint64(key) + (e >> np.uint64(32)) * np.uint64(0x9E3779B9)).astype(np.int64))


def by_blocks(t):
    return torch.nn.functional.pad(t, (0, -t.numel() % 32)).view(-1, 32)


def decode(mom, signed):
    """A moment of 8 bits as numbers, from the layout's definition."""
    codes, E = ref_ints(mom.m if signed else mom.v), ref_ints(mom.m_exp if signed else mom.v_exp)
    size = codes & 127 if signed else codes
    field, mantissa = size >> 3, (size & 7).double()
    top = 14 if signed else 30
    value = torch.where(field > 0, torch.ldexp(1 + mantissa / 8, field - top), torch.ldexp(mantissa / 8, torch.full_like(field, 1 - top)))
    value = torch.where((codes > 127) & torch.tensor(signed), -value, value)
    per = E.repeat_interleave(32)[:codes.numel()]
    value = torch.ldexp(value, per - 127)
    return torch.where(per == 255, torch.full_like(value, math.nan), value)


def ref_ints(t):
    return t.detach().cpu().to(torch.int64)


def check_codes(mom, signed, y, err, bits, what):
    """Whether the moment is ``y`` (64 bits, off by ``err`` in the kernel) rounded with the random ``bits``: where the sum of the part cut
    off and the random number is within the error of 1, either neighbour will do."""
    got = decode(mom, signed)
    E = ref_ints(mom.m_exp if signed else mom.v_exp)
    rows, erows = by_blocks(y), by_blocks(err)
    amax = rows.abs().amax(1)
    bad = ~torch.isfinite(amax) | (amax >= 2.0 ** 127)
    want_e = torch.where(bad, torch.tensor(255), (torch.frexp(amax)[1] - 1 + 127).clamp(min=1))
    sure = ((torch.frexp(amax * (1 - 2.0 ** -20))[1] == torch.frexp(amax * (1 + 2.0 ** -20))[1]) | bad) & (amax > 2.0 ** -120)
    assert torch.equal(E[sure], want_e[sure].long()), what
    assert torch.isnan(got[E.repeat_interleave(32)[:got.numel()] == 255]).all(), what
    e = E.repeat_interleave(32).view(-1, 32)
    top, lowest = (14, -13) if signed else (30, -29)
    fine = e != 255
    binade = torch.maximum(torch.frexp(rows)[1] - 1, e - 127 + lowest)
    unit = torch.ldexp(torch.ones_like(rows), binade - 3)
    u = by_blocks(((bits & 0xFFFFF) if signed else bits >> 12).double() * 2.0 ** -20)
    steps = rows.abs() / unit
    slack = erows / unit + 2.0 ** -18
    low, high = torch.floor(steps + u - slack), torch.floor(steps + u + slack)
    if not signed:
        low, high = (torch.where(rows > 0, t.clamp(min=1), t) for t in (low, high))
    have = by_blocks(torch.nan_to_num(got, nan=0.0)).abs() / unit
    ok = (have >= low) & (have <= high) | ~fine
    assert ok.all(), (what, int((~ok).sum()))
    assert (slack[fine & (rows.abs() > 0)] < 0.01).float().mean() > 0.9 or not (rows.abs() > 0).any(), what  # the test says something
    neg = by_blocks(got) < 0
    assert not (neg & (rows > 0) & fine).any(), what


def adamw(old, g, m, v, lr, decay, betas, eps, t, keep):
    """(param, m, v) in 64 bits and the errors of their fp32 evaluation."""
    b1, b2 = betas
    m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    em = 2.0 ** -21 * (b1 * m.abs() + (1 - b1) * g.abs())  # two roundings of each product (its factor's and its own), one of the sum, one of g
    ev = 2.0 ** -21 * v1 + 2.0 ** -149
    denom = (v1 / (1 - b2 ** t)).sqrt() + eps
    rate = lr / (1 - b1 ** t)
    change = rate * m1 / denom
    new = old * (1 - lr * decay) - change
    # sqrt and quotient within 2^-21 each, half of v's error, factors
    ep = rate * em / denom + change.abs() * (2.0 ** -19 + torch.where(v1 > 0, ev / (2 * v1), torch.zeros_like(v1))) + 2.0 ** -22 * old.abs()
    if keep:
        zero = old == 0
        m1, v1, new, em, ev, ep = (torch.where(zero, torch.zeros_like(x), x) for x in (m1, v1, new, em, ev, ep))
    return new, m1, v1, ep, em, ev


def check_random_rounding(got, want, err, bits, what):
    """16-bit params rounded stochastically: floor(|y| / unit + u) units, either neighbour within the error of the border."""
    t = got.dtype
    shift, digits, least = (16, 7, -126) if t == torch.bfloat16 else (13, 10, -14)
    u = (((bits * 0x9E3779B1) & 0xFFFFFFFF) >> (32 - shift)).double() * 2.0 ** -shift
    binade = (torch.frexp(want)[1] - 1).clamp(min=least)
    unit = torch.ldexp(torch.ones_like(want), binade - digits)
    slack = err / unit + 2.0 ** -shift
    low, high = torch.floor(want.abs() / unit + u - slack), torch.floor(want.abs() / unit + u + slack)
    have = ref.d64(got).abs() / unit
    ok = (have >= low) & (have <= high)  # where the update takes the weight to almost 0, the error is more than a unit of what is left
    assert ok.all(), (what, int((~ok).sum()))
