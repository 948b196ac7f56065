"""What the evaluation and fine-tuning operators are measured on.

The search of this package asks its caller for the calibration loss of a stitched model, and a pruned model is
then tuned against the dense one.  Four operators carry that work: the linear layers of a block with bias,
activation and residual (``linear``), the normalisation between them (``layer_norm``), the log probabilities of
given tokens with entropy and top alternatives (``token_logprobs``), and distillation from the dense model's top
log probabilities (``distill``).  Each is given here in its plain form (elementary torch operations in 32 bits,
rounded once at the end), as the calls a user makes of the package, and from its definition in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
LARGEST_LOGITS = 1 << 28      # elements of the largest 16-bit logits table
LARGEST_PRODUCT = 1 << 36     # 2 m n k of the largest linear layer
LARGEST_ROWS = 1 << 25        # elements of the largest normalised matrix


def listed():
    return [
        # One token through the up projection of a BERT-base block: an interactive answer, where latency counts.
        {"name": "linear one token", "op": "linear", "m": 1, "k": 768, "n": 3072, "dtype": "bf16",
         "activation": "gelu", "bias": True, "residual": False, "pad": 0},
        # A calibration batch of 32 sequences of 128 tokens through the same layer.
        {"name": "linear BERT-base up", "op": "linear", "m": 4096, "k": 768, "n": 3072, "dtype": "bf16",
         "activation": "gelu", "bias": True, "residual": False, "pad": 0},
        # The down projection of a BERT-large block, whose output joins the residual stream: the largest product.
        {"name": "linear BERT-large down", "op": "linear", "m": 8192, "k": 4096, "n": 1024, "dtype": "f16",
         "activation": "none", "bias": True, "residual": True, "pad": 0},
        # A layer left with odd widths by structured pruning, on a batch of whatever sentences came, out of a wider buffer.
        {"name": "linear odd widths", "op": "linear", "m": 333, "k": 1001, "n": 517, "dtype": "bf16",
         "activation": "silu", "bias": True, "residual": True, "pad": 22},
        # One sequence normalised while the search evaluates a profile.
        {"name": "layer norm one sequence", "op": "layer_norm", "mode": "forward", "r": 128, "d": 768,
         "dtype": "bf16", "pad": 0},
        # A fine-tuning batch through a BERT-large normalisation, forward and backward.
        {"name": "layer norm BERT-large step", "op": "layer_norm", "mode": "train", "r": 32768, "d": 1024,
         "dtype": "bf16", "pad": 0},
        # The log probability, entropy and 8 alternatives of one next token, in 32 bits.
        {"name": "log probs one token", "op": "token_logprobs", "mode": "forward", "r": 1, "v": 32768,
         "dtype": "f32", "top": 8, "temperature": 1.0, "masked": 0.0, "pad": 0},
        # The dense model's answers on a calibration set, with the 20 alternatives kept for later.
        {"name": "log probs calibration set", "op": "token_logprobs", "mode": "forward", "r": 2048, "v": 131072,
         "dtype": "bf16", "top": 20, "temperature": 1.0, "masked": 0.0, "pad": 0},
        # Cross entropy with an entropy bonus over a vocabulary of odd size, with its gradient.
        {"name": "log probs odd step", "op": "token_logprobs", "mode": "train", "r": 1024, "v": 50001,
         "dtype": "bf16", "top": 0, "temperature": 1.0, "masked": 0.0, "pad": 0},
        # A short evaluation against the dense model's 32 best tokens, in 32 bits: a candidate profile's loss.
        {"name": "distill profile loss", "op": "distill", "mode": "forward", "r": 37, "v": 30001, "dtype": "f32",
         "top": 32, "temperature": 1.0, "tail": True, "masked": 0.0, "pad": 0},
        # A fine-tuning step on the dense model's 64 best tokens and the mass of the rest: the most bytes.
        {"name": "distill large step", "op": "distill", "mode": "train", "r": 4096, "v": 65536, "dtype": "bf16",
         "top": 64, "temperature": 2.0, "tail": True, "masked": 0.0, "pad": 0},
        # A step on renormalised alternatives, half precision, part of the vocabulary not allowed.
        {"name": "distill masked step", "op": "distill", "mode": "train", "r": 640, "v": 32768, "dtype": "f16",
         "top": 16, "temperature": 1.0, "tail": False, "masked": 0.5, "pad": 64},
    ]


def _log_uniform(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["linear", "linear", "layer_norm", "token_logprobs", "token_logprobs", "distill", "distill"])
    if op == "linear":
        k, n = _log_uniform(rng, 64, 4096), _log_uniform(rng, 2, 4096)
        if rng.random() < 0.6:  # most layers keep widths that are multiples of 64
            k, n = max(64, k // 64 * 64), max(64, n // 64 * 64)
        m = _log_uniform(rng, 1, max(1, min(16384, LARGEST_PRODUCT // (2 * k * n))))
        return {"op": op, "m": m, "k": k, "n": n, "dtype": rng.choice(["bf16", "f16"]),
                "activation": rng.choice(["none", "relu", "gelu", "silu"]), "bias": rng.random() < 0.8,
                "residual": rng.random() < 0.5, "pad": rng.choice([0, 0, 8, 13])}
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    size = 4 if dtype == "f32" else 2
    if op == "layer_norm":
        d = _log_uniform(rng, 16, 8192)
        if rng.random() < 0.6:
            d = max(16, d // 16 * 16)
        return {"op": op, "mode": rng.choice(["forward", "backward", "train"]),
                "r": _log_uniform(rng, 1, LARGEST_ROWS * 2 // size // d), "d": d, "dtype": dtype,
                "pad": rng.choice([0, 0, 8, 13])}
    v = _log_uniform(rng, 1000, 200000)
    if rng.random() < 0.6:
        v = max(1024, v // 64 * 64)
    case = {"op": op, "mode": rng.choice(["forward", "backward", "train"]),
            "r": _log_uniform(rng, 1, LARGEST_LOGITS * 2 // size // v), "v": v, "dtype": dtype,
            "temperature": rng.choice([1.0, 1.0, 0.7, 2.0, 4.0]), "masked": rng.choice([0.0, 0.0, 0.5, 0.95]),
            "pad": rng.choice([0, 0, 64, 5])}
    case["top"] = _log_uniform(rng, 1, max(1, min(64, int(v * (1.0 - case["masked"])) // 4)))
    if op == "token_logprobs":
        if case["mode"] != "forward" or rng.random() < 0.3:
            case["top"] = 0
    else:
        case["tail"] = rng.random() < 0.6
    return case


# ------------------------------------------------------------------------------------------------ inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _rand(g, *shape):
    return torch.rand(*shape, generator=g, device="cuda", dtype=torch.float32)


def _padded(values, pad, dtype):
    """``values`` as the first columns of a buffer that is ``pad`` columns wider (a view with its own row stride)."""
    r, c = values.shape
    buffer = torch.zeros(r, c + pad, dtype=dtype, device="cuda")
    buffer[:, :c] = values
    return buffer[:, :c]


def prepare(case, seed):
    g = _generator(seed)
    dtype = DTYPES[case["dtype"]]
    if case["op"] == "linear":
        m, k, n = case["m"], case["k"], case["n"]
        w = _randn(g, n, k) / math.sqrt(k)
        w = torch.where(w.abs() < 0.6745 / math.sqrt(k), torch.zeros_like(w), w * 1.4)  # half the weights pruned away
        return {"case": case, "x": _padded(_randn(g, m, k), case["pad"], dtype), "w": w.to(dtype),
                "b": (0.2 * _randn(g, n)).to(dtype) if case["bias"] else None,
                "res": _randn(g, m, n).to(dtype) if case["residual"] else None}
    if case["op"] == "layer_norm":
        r, d = case["r"], case["d"]
        scale = torch.where(_rand(g, d) < 0.01, 12.0, 1.0)  # a few channels are much larger than the rest
        x = _padded(_randn(g, r, d) * scale + 0.3 * _randn(g, d) + 0.2 * _randn(g, r, 1), case["pad"], dtype)
        state = {"case": case, "x": x, "w": (1.0 + 0.1 * _randn(g, d)).to(dtype), "b": (0.1 * _randn(g, d)).to(dtype),
                 "dy": (_randn(g, r, d) * 0.1).to(dtype), "eps": 1e-5}
        if case["mode"] == "backward":
            xf = x.float()
            state["mean"] = xf.mean(dim=1)
            state["rstd"] = torch.rsqrt(((xf - state["mean"][:, None]) ** 2).mean(dim=1) + state["eps"])
        return state
    r, v = case["r"], case["v"]
    common = 1.5 * _randn(g, v)                                    # how frequent a token is
    logits = torch.empty(r, v + case["pad"], dtype=dtype, device="cuda")[:, :v]
    step = max(1, (1 << 26) // v)
    for a in range(0, r, step):
        rows = _randn(g, min(step, r - a), v).mul_(2.0).add_(common)
        hot = torch.randint(0, v, (rows.shape[0], 4), generator=g, device="cuda")  # what the context asks for
        rows.scatter_add_(1, hot, 8.0 + 4.0 * _rand(g, rows.shape[0], 4))
        if case["masked"]:
            rows.masked_fill_(_rand(g, rows.shape[0], v) < case["masked"], -math.inf)
        logits[a:a + step] = rows
    state = {"case": case, "logits": logits, "temperature": case["temperature"]}
    scale = 8192.0 if case["dtype"] == "f16" else 1.0  # half precision trains with a scaled loss
    if case["op"] == "token_logprobs":
        best = logits.argmax(dim=1)
        tokens = torch.where(_rand(g, r) < 0.6, best, torch.randint(0, v, (r,), generator=g, device="cuda"))
        if r > 8:
            tokens = torch.where(_rand(g, r) < 0.1, torch.full_like(tokens, -100), tokens)  # padding: no token
        state["tokens"] = tokens
        state["g_logprob"] = -scale * _rand(g, r) / r
        state["g_entropy"] = -0.01 * scale * _rand(g, r) / r
        if case["mode"] == "backward":
            saved = _plain_token_logprobs(dict(state, case=dict(case, mode="forward", top=0)))
            state["lse"], state["entropy"] = saved["lse"], saved["entropy"]
        return state
    top = min(case["top"], v)
    ids, lps = [], []
    for a in range(0, r, step):  # the dense model's answers: the same tokens allowed, other scores
        t = logits[a:a + step].float()
        t = (t * 1.1 + 1.5 * _randn(g, *t.shape)) / case["temperature"]
        best = t.topk(top, dim=1)
        ids.append(best.indices)
        lps.append(best.values - torch.logsumexp(t, dim=1, keepdim=True))
    state["ids"], state["lps"] = torch.cat(ids), torch.cat(lps)
    state["g"] = scale * (0.5 + _rand(g, r)) / r
    if case["mode"] == "backward":
        saved = _plain_distill(dict(state, case=dict(case, mode="forward")))
        state["lse"], state["rest"] = saved["lse"], saved.get("rest")
    return state


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    case = state["case"]
    if own:
        return _OWN[case["op"]](state)
    return _PLAIN[case["op"]](state)


def _own_linear(s):
    from paper_2201_13096_b200 import evaluate
    return {"y": evaluate.linear(s["x"], s["w"], bias=s["b"], residual=s["res"], activation=s["case"]["activation"])}


def _own_layer_norm(s):
    from paper_2201_13096_b200 import evaluate
    mode, out = s["case"]["mode"], {}
    if mode == "backward":
        mean, rstd = s["mean"], s["rstd"]
    else:
        out["y"], mean, rstd = evaluate.layer_norm(s["x"], s["w"], s["b"], eps=s["eps"])
        out["mean"], out["rstd"] = mean, rstd
    if mode != "forward":
        out["dx"], out["dw"], out["db"] = evaluate.layer_norm_backward(s["dy"], s["x"], s["w"], mean, rstd)
    return out


def _own_token_logprobs(s):
    from paper_2201_13096_b200 import evaluate
    mode, temperature = s["case"]["mode"], s["temperature"]
    if mode == "backward":
        return {"dlogits": evaluate.token_logprobs_backward(s["logits"], s["tokens"], s["lse"], s["entropy"],
                                                            s["g_logprob"], s["g_entropy"], temperature=temperature)}
    if mode == "train":
        got, dlogits = evaluate.token_logprobs_with_grad(s["logits"], s["tokens"], s["g_logprob"], s["g_entropy"],
                                                         temperature=temperature)
        return {"logprob": got.logprob, "entropy": got.entropy, "lse": got.lse, "dlogits": dlogits}
    got = evaluate.token_logprobs(s["logits"], s["tokens"], top_k=s["case"]["top"], temperature=temperature)
    out = {"logprob": got.logprob, "entropy": got.entropy, "lse": got.lse}
    if s["case"]["top"]:
        out["top_ids"], out["top_logprobs"] = got.top_ids, got.top_logprobs
    return out


def _own_distill(s):
    from paper_2201_13096_b200 import evaluate
    mode, kind = s["case"]["mode"], {"temperature": s["temperature"], "tail": s["case"]["tail"]}
    if mode == "backward":
        return {"dlogits": evaluate.distill_loss_backward(s["logits"], s["ids"], s["lps"], s["lse"], s["rest"], s["g"], **kind)}
    if mode == "train":
        got, dlogits = evaluate.distill_loss_with_grad(s["logits"], s["ids"], s["lps"], s["g"], **kind)
    else:
        got, dlogits = evaluate.distill_loss(s["logits"], s["ids"], s["lps"], **kind), None
    out = {"loss": got.loss, "lse": got.lse}
    if s["case"]["tail"]:
        out["rest"] = got.rest
    if dlogits is not None:
        out["dlogits"] = dlogits
    return out


_OWN = {"linear": _own_linear, "layer_norm": _own_layer_norm, "token_logprobs": _own_token_logprobs, "distill": _own_distill}


def _plain_linear(s):
    z = torch.matmul(s["x"].float(), s["w"].float().t())
    if s["b"] is not None:
        z = z + s["b"].float()
    kind = s["case"]["activation"]
    if kind == "relu":
        z = torch.maximum(z, torch.zeros_like(z))
    elif kind == "gelu":
        z = 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    elif kind == "silu":
        z = z / (1.0 + torch.exp(-z))
    if s["res"] is not None:
        z = z + s["res"].float()
    return {"y": z.to(s["x"].dtype)}


def _plain_layer_norm(s):
    mode, out = s["case"]["mode"], {}
    x, w = s["x"].float(), s["w"].float()
    if mode == "backward":
        mean, rstd = s["mean"], s["rstd"]
        hat = (x - mean[:, None]) * rstd[:, None]
    else:
        mean = x.sum(dim=1) / x.shape[1]
        rstd = 1.0 / torch.sqrt(((x - mean[:, None]) ** 2).sum(dim=1) / x.shape[1] + s["eps"])
        hat = (x - mean[:, None]) * rstd[:, None]
        out.update(y=(hat * w + s["b"].float()).to(s["x"].dtype), mean=mean, rstd=rstd)
    if mode != "forward":
        dy = s["dy"].float()
        dhat = dy * w
        a = dhat.sum(dim=1, keepdim=True) / x.shape[1]
        b = (dhat * hat).sum(dim=1, keepdim=True) / x.shape[1]
        out.update(dx=((dhat - a - hat * b) * rstd[:, None]).to(s["x"].dtype), dw=(dy * hat).sum(dim=0), db=dy.sum(dim=0))
    return out


def _ordered_top(x, k):
    """The k largest of each row of ``x`` (32 bits), the lowest index first where values are equal: ids and values."""
    bits = (x + 0.0).view(torch.int32)
    key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() * (1 << 32) + (
        (1 << 32) - 1 - torch.arange(x.shape[1], device=x.device))
    ids = ((1 << 32) - 1) - (key.topk(k, dim=1).values & ((1 << 32) - 1))
    return ids, x.gather(1, ids)


def _plain_token_logprobs(s):
    mode, dtype = s["case"]["mode"], s["logits"].dtype
    x = s["logits"].float()
    z = x / s["temperature"]
    if mode == "backward":
        lse, entropy, out = s["lse"], s["entropy"], {}
    else:
        m = z.amax(dim=1, keepdim=True)
        e = torch.exp(z - m)
        total = e.sum(dim=1)
        lse = torch.log(total) + m[:, 0]
        entropy = torch.log(total) - torch.where(e > 0, e * (z - m), torch.zeros_like(e)).sum(dim=1) / total
        named = s["tokens"] >= 0
        picked = z.gather(1, torch.where(named, s["tokens"], torch.zeros_like(s["tokens"]))[:, None])[:, 0] - lse
        out = {"logprob": torch.where(named, picked, torch.zeros_like(picked)), "entropy": entropy, "lse": lse}
        if s["case"]["top"]:
            ids, values = _ordered_top(x, s["case"]["top"])
            out["top_ids"], out["top_logprobs"] = ids.to(torch.int32), values / s["temperature"] - lse[:, None]
    if mode != "forward":
        logp = z - lse[:, None]
        p = torch.exp(logp)
        grad = -p * s["g_logprob"][:, None] * (s["tokens"] >= 0)[:, None]
        grad = grad - s["g_entropy"][:, None] * torch.where(p > 0, p * (logp + entropy[:, None]), torch.zeros_like(p))
        hit = torch.arange(x.shape[1], device=x.device)[None, :] == s["tokens"][:, None]
        grad = grad + torch.where(hit, s["g_logprob"][:, None], torch.zeros_like(grad))
        out["dlogits"] = (grad / s["temperature"]).to(dtype)
    return out


def _plain_distill(s):
    mode, dtype, tail = s["case"]["mode"], s["logits"].dtype, s["case"]["tail"]
    z = s["logits"].float() / s["temperature"]
    lps = s["lps"].float()
    if tail:
        q = torch.exp(lps)
        left = torch.clamp(1.0 - q.sum(dim=1), min=0.0)
        logq = lps
    else:
        e = torch.exp(lps - lps.amax(dim=1, keepdim=True))
        total = e.sum(dim=1, keepdim=True)
        q, logq, left = e / total, lps - lps.amax(dim=1, keepdim=True) - torch.log(total), None
    out = {}
    if mode == "backward":
        lse, rest = s["lse"], s["rest"]
    else:
        m = z.amax(dim=1)
        log_total = torch.log(torch.exp(z - m[:, None]).sum(dim=1))
        lse = log_total + m
        logp = z.gather(1, s["ids"]) - m[:, None] - log_total[:, None]
        loss = torch.where(q > 0, q * (logq - logp), torch.zeros_like(q)).sum(dim=1)
        out = {"loss": loss, "lse": lse}
        rest = None
        if tail:
            outside = z.scatter(1, s["ids"], -math.inf)
            rest_m = outside.amax(dim=1)
            log_rest = torch.log(torch.exp(outside - rest_m[:, None]).sum(dim=1))
            rest = log_rest + rest_m
            log_ratio = torch.log(left) - (rest_m - m) - (log_rest - log_total)
            out["loss"] = loss + torch.where(left > 0, left * log_ratio, torch.zeros_like(left))
            out["rest"] = rest
    if mode != "forward":
        mass = q.sum(dim=1) + (left if tail else 0.0)
        grad = torch.exp(z - lse[:, None]) * mass[:, None]
        if tail:
            grad = grad - left[:, None] * torch.exp(z - rest[:, None]).scatter(1, s["ids"], 0.0)
        grad = grad.scatter_add(1, s["ids"], -q)
        out["dlogits"] = (grad * s["g"][:, None] / s["temperature"]).to(dtype)
    return out


_PLAIN = {"linear": _plain_linear, "layer_norm": _plain_layer_norm, "token_logprobs": _plain_token_logprobs,
          "distill": _plain_distill}


# ------------------------------------------------------------------------------------------------ work

def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "linear":
        m, k, n = case["m"], case["k"], case["n"]
        elements = m * k + n * k + m * n + (n if case["bias"] else 0) + (m * n if case["residual"] else 0)
        return {"bytes": size * elements, "flops": 2 * m * n * k}
    if case["op"] == "layer_norm":
        r, d = case["r"], case["d"]
        tables = {"forward": 2, "backward": 3, "train": 4}[case["mode"]]
        extra = 2 * d * size + 8 * r + (8 * d if case["mode"] != "forward" else 0)
        return {"bytes": tables * r * d * size + extra, "flops": {"forward": 8, "backward": 12, "train": 20}[case["mode"]] * r * d}
    r, v, top = case["r"], case["v"], case["top"]
    tables = 1 if case["mode"] == "forward" else 2
    per_row = 32 + 12 * top
    return {"bytes": tables * r * v * size + r * per_row, "flops": {"forward": 6, "backward": 6, "train": 12}[case["mode"]] * r * v}


# ------------------------------------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_linear, "layer_norm": _exact_layer_norm, "token_logprobs": _exact_token_logprobs,
            "distill": _exact_distill}[case["op"]](s)


def _exact_linear(s):
    f = {"none": lambda t: t, "relu": lambda t: t.clamp(min=0), "silu": lambda t: t * torch.sigmoid(t),
         "gelu": lambda t: t * 0.5 * torch.special.erfc(-t / math.sqrt(2.0))}[s["case"]["activation"]]
    y = s["x"].double() @ s["w"].double().T
    y = f(y if s["b"] is None else y + s["b"].double())
    return {"y": y if s["res"] is None else y + s["res"].double()}


def _exact_layer_norm(s):
    x, w, b, dy = (s[n].double() for n in ("x", "w", "b", "dy"))
    mode, out = s["case"]["mode"], {}
    var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
    rstd = (var + s["eps"]).pow(-0.5)
    if mode == "backward":
        mean, rstd = s["mean"].double()[:, None], s["rstd"].double()[:, None]
    hat = (x - mean) * rstd
    if mode != "backward":
        out = {"y": torch.addcmul(b, hat, w), "mean": mean[:, 0], "rstd": rstd[:, 0]}
    if mode != "forward":
        u = w * dy
        out["dx"] = rstd * (u - u.mean(1, keepdim=True) - hat * (u * hat).mean(1, keepdim=True))
        out["dw"], out["db"] = torch.einsum("rd,rd->d", dy, hat), dy.sum(0)
    return out


def _by_rows(s, v, names, one):
    """``one`` on blocks of rows of the state's tensors ``names``, its outputs joined: 64-bit tables of all rows would not fit."""
    r, step, parts = s["logits"].shape[0], max(1, (1 << 27) // v), []
    for a in range(0, r, step):
        parts.append(one({n: None if s.get(n) is None else s[n][a:a + step] for n in names}))
    return {k: None if parts[0][k] is None else torch.cat([p[k] for p in parts]) for k in parts[0]}


def _exact_token_logprobs(s):
    mode, top, temperature = s["case"]["mode"], s["case"]["top"], s["temperature"]

    def one(p):
        t = p["logits"].double() / temperature
        lse = torch.logsumexp(t, 1) if mode != "backward" else p["lse"].double()
        logp = t - lse[:, None]
        prob = logp.exp()
        entropy = torch.special.entr(prob).sum(1) if mode != "backward" else p["entropy"].double()
        rows, named = torch.arange(t.shape[0], device=t.device), p["tokens"] >= 0
        out = {}
        if mode != "backward":
            out = {"logprob": logp[rows, p["tokens"].clamp(min=0)].masked_fill(~named, 0.0), "entropy": entropy, "lse": lse}
            if top:
                out.update(top_ids=None, top_logprobs=logp.topk(top, dim=1).values)
        if mode != "forward":
            gl = p["g_logprob"].double() * named
            d = prob * -(gl + p["g_entropy"].double() * entropy)[:, None] + p["g_entropy"].double()[:, None] * torch.special.entr(prob)
            d[rows, p["tokens"].clamp(min=0)] += gl
            out["dlogits"] = d / temperature
        return out

    return _by_rows(s, s["case"]["v"], ("logits", "tokens", "lse", "entropy", "g_logprob", "g_entropy"), one)


def _exact_distill(s):
    mode, tail, temperature = s["case"]["mode"], s["case"]["tail"], s["temperature"]

    def one(p):
        t, ids, teacher = p["logits"].double() / temperature, p["ids"], p["lps"].double()
        if not tail:
            teacher = torch.log_softmax(teacher, dim=1)
        q = teacher.exp()
        inside = torch.zeros(t.shape, dtype=torch.bool, device=t.device).scatter(1, ids, True)
        left = (1.0 - q.sum(1)).clamp(min=0.0) if tail else torch.zeros_like(q[:, 0])
        lse = torch.logsumexp(t, 1) if mode != "backward" else p["lse"].double()
        rest = torch.logsumexp(t.masked_fill(inside, -math.inf), 1) if p["rest"] is None else p["rest"].double()
        out = {}
        if mode != "backward":
            loss = (torch.special.xlogy(q, q) - torch.where(q > 0, q * t.gather(1, ids), 0.0)).sum(1) + q.sum(1) * lse
            if tail:
                loss = loss + torch.special.xlogy(left, left) + torch.where(left > 0, left * (lse - rest), 0.0)
            out = {"loss": loss, "lse": lse}
            if tail:
                out["rest"] = rest
        if mode != "forward":
            d = torch.softmax(t, 1) if mode != "backward" else (t - lse[:, None]).exp()
            d = d * (q.sum(1) + left)[:, None]
            if tail:
                d = d - torch.where(inside, 0.0, (t - rest[:, None]).exp() * left[:, None])
            out["dlogits"] = d.scatter_add(1, ids, -q) * p["g"].double()[:, None] / temperature
        return out

    return _by_rows(s, s["case"]["v"], ("logits", "ids", "lps", "lse", "rest", "g"), one)
