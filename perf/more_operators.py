"""What the operators of tuning a pruned language model are measured on.

A pruned model is tuned with the gradient of its head's loss and a step on its weights.  Two operators carry that work: the log
probabilities of given tokens under a head's softmax, straight from the hidden states and the head's weight (``linear_token_logprobs``,
with its gradients; no table of logits is kept), and an AdamW step over many tensors at once, with moments in 32 or in 8 bits
(``adamw_step``).  Each is given here in its plain form (elementary torch operations in 32 bits, rounded once at the end), as the
calls a user makes of the package, and from its definition in 64 bits.

Moments in 8 bits: 32 consecutive elements of a tensor share a byte E, the exponent field (as in fp32, at least 1) of the largest
magnitude among them; E = 255 marks a block that holds anything not finite or from 2^127 on.  An element y is kept as a small
floating-point number relative to 2^(E - 127): the first moment with a sign, 4 bits of exponent and 3 of mantissa (the largest
magnitude's binade has exponent field 14), the second with 5 and 3 bits (exponent field 30), fields of 0 without the leading 1.
Rounding is stochastic, up with the probability of the part cut off (20 bits of it), from a hash of seed, step, tensor and element;
a positive second moment is never rounded to 0.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
LARGEST_LOSS = 1 << 41        # rows x vocabulary x width of the largest head
LARGEST_LOGITS = 1 << 29      # rows x vocabulary, which only the plain form keeps
LARGEST_WEIGHT = 1 << 28      # elements of the largest head's weight
LARGEST_TENSORS = 1 << 27     # elements that a drawn step updates at most
BETAS, EPS = (0.9, 0.999), 1e-8

BERT_LARGE_BLOCK = ["1024x1024", "1024"] * 4 + ["4096x1024", "4096", "1024x4096", "1024"] + ["1024"] * 4


def listed():
    return [
        # The log probability of one token after a prompt, a head of BERT-base's width: latency counts.
        {"name": "head one token", "op": "head", "mode": "forward", "r": 1, "v": 32768, "d": 768, "dtype": "bf16",
         "temperature": 1.0, "bias": False, "masked": 0.0, "entropy": False, "pad": 0},
        # The dense model's log probabilities and entropies on a calibration set: a large vocabulary, forward alone.
        {"name": "head calibration set", "op": "head", "mode": "forward", "r": 2048, "v": 131072, "d": 2048, "dtype": "bf16",
         "temperature": 1.0, "bias": False, "masked": 0.0, "entropy": False, "pad": 0},
        # A fine-tuning step of four sequences of 128 tokens through BERT-base's head, odd vocabulary, with its bias.
        {"name": "head BERT-base step", "op": "head", "mode": "train", "r": 512, "v": 30001, "d": 768, "dtype": "bf16",
         "temperature": 1.0, "bias": True, "masked": 0.0, "entropy": False, "pad": 0},
        # The gradients from the lse of an earlier forward call (a loss that is weighted once all log probabilities are known).
        {"name": "head backward", "op": "head", "mode": "backward", "r": 4096, "v": 32768, "d": 1024, "dtype": "bf16",
         "temperature": 1.0, "bias": False, "masked": 0.0, "entropy": False, "pad": 0},
        # Odd sizes out of wider buffers in half precision, an entropy bonus, a temperature, part of the ids not allowed.
        {"name": "head odd masked step", "op": "head", "mode": "train", "r": 1021, "v": 50001, "d": 1000, "dtype": "f16",
         "temperature": 0.7, "bias": True, "masked": 0.25, "entropy": True, "pad": 13},
        # A large training batch: the most work.
        {"name": "head large step", "op": "head", "mode": "train", "r": 8192, "v": 65536, "d": 4096, "dtype": "bf16",
         "temperature": 1.0, "bias": False, "masked": 0.0, "entropy": False, "pad": 0},
        # The last normalisation's weight and bias: the smallest step, where latency counts.
        {"name": "step last norm", "op": "step", "sizes": "1024 1024", "dtype": "f32", "grads": "f32", "bits": 32, "master": False,
         "rounding": "nearest", "keep_zeros": False, "scaled": False, "aligned": True, "step": 3},
        # The upper half of a pruned BERT-large: 16-bit weights with their copies in 32 bits, pruned weights stay pruned.
        {"name": "step pruned BERT-large", "op": "step", "sizes": " ".join(BERT_LARGE_BLOCK * 12),
         "dtype": "bf16", "grads": "bf16", "bits": 32, "master": True, "rounding": "nearest", "keep_zeros": True, "scaled": True,
         "aligned": True, "step": 1000},
        # One wide block with moments in 8 bits and 16-bit weights that are rounded stochastically: the least memory.
        {"name": "step wide block 8 bits", "op": "step", "sizes": "12288x4096 4096x4096 8192x4096 4096 4096", "dtype": "bf16",
         "grads": "bf16", "bits": 8, "master": False, "rounding": "stochastic", "keep_zeros": False, "scaled": False, "aligned": True, "step": 250},
        # Layers left with odd widths by structured pruning, one buffer of half-precision weights behind one another, a scaled loss.
        {"name": "step odd widths 8 bits", "op": "step", "sizes": "1001x517 517 333x1001 333 77x333 77 1 31", "dtype": "f16",
         "grads": "f32", "bits": 8, "master": True, "rounding": "nearest", "keep_zeros": True, "scaled": True, "aligned": False, "step": 17},
    ]


def _log_uniform(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    if rng.random() < 0.6:
        d = _log_uniform(rng, 64, 4096)
        v = _log_uniform(rng, 1000, min(200000, LARGEST_WEIGHT // d))
        if rng.random() < 0.6:  # most heads have widths and vocabularies that are multiples of 64
            d, v = max(64, d // 64 * 64), max(1024, v // 64 * 64)
        r = _log_uniform(rng, 1, min(16384, LARGEST_LOGITS // v, LARGEST_LOSS // (v * d)))
        bias = rng.random() < 0.4
        return {"op": "head", "mode": rng.choice(["forward", "backward", "train", "train"]), "r": r, "v": v, "d": d,
                "dtype": rng.choice(["bf16", "bf16", "f16"]), "temperature": rng.choice([1.0, 1.0, 0.7, 2.0]), "bias": bias,
                "masked": rng.choice([0.0, 0.5]) if bias else 0.0, "entropy": rng.random() < 0.3, "pad": rng.choice([0, 0, 8, 13])}
    bits, dtype = rng.choice([32, 8]), rng.choice(["bf16", "bf16", "f16", "f32"])
    left, sizes = _log_uniform(rng, 1000, LARGEST_TENSORS), []
    for _ in range(rng.randint(1, 24 if bits == 8 else 60)):
        n = _log_uniform(rng, 1, max(1, left))
        if rng.random() < 0.6:
            n = max(1, n // 64 * 64)
        sizes.append(n)
        left = max(1, left - n)
    master = dtype != "f32" and rng.random() < 0.5
    return {"op": "step", "sizes": " ".join(map(str, sizes)), "dtype": dtype, "grads": rng.choice([dtype, "f32"]), "bits": bits, "master": master,
            "rounding": rng.choice(["nearest", "stochastic"]) if dtype != "f32" and not master else "nearest", "keep_zeros": rng.random() < 0.4,
            "scaled": rng.random() < 0.5, "aligned": rng.random() < 0.7, "step": _log_uniform(rng, 1, 100000)}


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


def _sizes(case):
    """Elements of each tensor of a step."""
    return [math.prod(int(n) for n in t.split("x")) for t in case["sizes"].split()]


def _flat(case, dtype, apart):
    """A buffer of zeros for all tensors of a step, each ``apart`` elements after a multiple of 64 or right behind the last, and its parts."""
    starts, at = [], 0
    for n in _sizes(case):
        starts.append(at)
        at += (n + 63) // 64 * 64 if apart else n
    buffer = torch.zeros(at, dtype=dtype, device="cuda")
    return buffer, [buffer[a:a + n] for a, n in zip(starts, _sizes(case))]


def prepare(case, seed):
    g = _generator(seed)
    return _prepare_head(case, g) if case["op"] == "head" else _prepare_step(case, g, seed)


def _prepare_head(case, g):
    r, v, d, dtype = case["r"], case["v"], case["d"], DTYPES[case["dtype"]]
    weight = _randn(g, v, d) * (3.0 / math.sqrt(d))
    target = torch.randint(0, v, (r,), generator=g, device="cuda")
    hidden = _randn(g, r, d)
    hidden += weight[target] * (4.0 / 3.0) * (_rand(g, r, 1) < 0.7)   # most tokens are what the context asks for
    state = {"case": case, "hidden": _padded(hidden, case["pad"], dtype), "weight": _padded(weight, case["pad"], dtype),
             "temperature": case["temperature"], "bias": None}
    if case["bias"]:
        bias = 0.5 * _randn(g, v)
        allowed = _rand(g, v) >= case["masked"]
        allowed[target] = True
        state["bias"] = torch.where(allowed, bias, torch.full_like(bias, -math.inf))
    state["tokens"] = torch.where(_rand(g, r) < 0.1, torch.full_like(target, -100), target) if r > 8 else target  # padding: no token
    scale = 8192.0 if case["dtype"] == "f16" else 1.0  # half precision trains with a scaled loss
    state["g_logprob"] = -scale * (0.5 + _rand(g, r)) / r
    state["g_entropy"] = -0.01 * scale * _rand(g, r) / r if case["entropy"] else None
    if case["mode"] == "backward":
        saved = _plain_head(dict(state, case=dict(case, mode="forward")))
        state["lse"], state["saved_entropy"] = saved["lse"], saved["entropy"]
    return state


def _prepare_step(case, g, seed):
    dtype, gdtype, bits = DTYPES[case["dtype"]], DTYPES[case["grads"]], case["bits"]
    state = {"case": case, "lr": 1e-3, "seed": seed % (1 << 32)}
    state["params"], params = _flat(case, dtype, case["aligned"])
    _, grads = _flat(case, gdtype, case["aligned"])
    state["master"], masters = _flat(case, torch.float32, True) if case["master"] else (None, [None] * len(params))
    state["tensors"], state["decay"], state["keep"] = [], [], []
    loss_scale = 1024.0 if case["scaled"] else 1.0
    state["grad_scale"] = torch.full((1,), 1.0 / loss_scale, device="cuda") if case["scaled"] else None
    kept = []
    for n in _sizes(case):
        state["decay"].append(0.01 if n >= 4096 else 0.0)            # biases and normalisations do not decay
        state["keep"].append(bool(case["keep_zeros"] and n >= 4096))
    if bits == 32:
        state["m"], ms = _flat(case, torch.float32, True)
        state["v"], vs = _flat(case, torch.float32, True)
    else:
        ms, vs = _flat(case, torch.uint8, True)[1], _flat(case, torch.uint8, True)[1]
    for p, gr, mc, m, v, keep in zip(params, grads, masters, ms, vs, state["keep"]):
        n = p.numel()
        w = _randn(g, n) * 0.02
        if keep:
            w = torch.where(_rand(g, n) < 0.5, torch.zeros_like(w), w)  # half the weights pruned away
        if mc is not None:
            mc.copy_(w)
        p.copy_(w)
        size = 1e-4 * torch.exp(1.5 * _randn(g, n))                   # gradients of weights differ by orders of magnitude
        gr.copy_(size * _randn(g, n) * loss_scale)
        old_m, old_v = size * _randn(g, n) * 0.3, size * size * (0.2 + _rand(g, n))
        if bits == 32:
            m.copy_(old_m)
            v.copy_(old_v)
            kept.append((p, gr, mc, m, v, None, None))
        else:
            blocks = (n + 31) // 32
            exps = [torch.zeros(blocks, dtype=torch.uint8, device="cuda") for _ in range(2)]
            half = torch.full((n,), 1 << 19, dtype=torch.int64, device="cuda")
            _encode(old_m, half, 113, True, m, exps[0])
            _encode(old_v, half, 97, False, v, exps[1])
            kept.append((p, gr, mc, m, v, exps[0], exps[1]))
    state["tensors"] = kept
    return state


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    if own:
        return (_own_head if state["case"]["op"] == "head" else _own_step)(state)
    return (_plain_head if state["case"]["op"] == "head" else _plain_step)(state)


def _own_head(s):
    from paper_2201_13096_b200 import evaluate
    mode, kind = s["case"]["mode"], {"bias": s["bias"], "temperature": s["temperature"]}
    if mode == "forward":
        got, grads = evaluate.linear_token_logprobs(s["hidden"], s["weight"], s["tokens"], **kind), None
    elif mode == "backward":
        got, grads = None, evaluate.linear_token_logprobs_backward(s["hidden"], s["weight"], s["tokens"], s["lse"], s["saved_entropy"],
                                                                   s["g_logprob"], s["g_entropy"], **kind)
    else:
        got, grads = evaluate.linear_token_logprobs_with_grad(s["hidden"], s["weight"], s["tokens"], s["g_logprob"], s["g_entropy"], **kind)
    out = {} if got is None else {"logprob": got.logprob, "entropy": got.entropy, "lse": got.lse}
    if grads is not None:
        out["dhidden"], out["dweight"] = grads.dhidden, grads.dweight
        if s["bias"] is not None:
            out["dbias"] = grads.dbias
    return out


def _own_step(s):
    from paper_2201_13096_b200 import evaluate
    case = s["case"]
    if "plan" not in s:  # the handle that a training program keeps from its first step on
        moments = [evaluate.AdamWMoments(m, v, me, ve) for _, _, _, m, v, me, ve in s["tensors"]]
        s["plan"] = evaluate.AdamW([t[0] for t in s["tensors"]], bits=case["bits"], masters=[t[2] for t in s["tensors"]] if case["master"] else None,
                                   moments=moments, betas=BETAS, eps=EPS, weight_decay=s["decay"], keep_zeros=s["keep"], rounding=case["rounding"])
    evaluate.adamw_step(s["plan"], [t[1] for t in s["tensors"]], lr=s["lr"], step=case["step"], seed=s["seed"], grad_scale=s["grad_scale"])
    out = {"params": s["params"], "master": s["master"]}
    if case["bits"] == 32:
        out["m"], out["v"] = s["m"], s["v"]
    else:
        out["moments"] = evaluate.adamw_moments(s["plan"], dtype=torch.bfloat16)
    return out


def _plain_head(s):
    mode, hidden, weight = s["case"]["mode"], s["hidden"].float(), s["weight"].float()
    z = torch.matmul(hidden, weight.t())
    if s["bias"] is not None:
        z = z + s["bias"]
    z = z / s["temperature"]
    if mode == "backward":
        lse, entropy, out = s["lse"], s["saved_entropy"], {}
    else:
        top = z.amax(dim=1, keepdim=True)
        e = torch.exp(z - top)
        total = e.sum(dim=1)
        lse = torch.log(total) + top[:, 0]
        entropy = torch.log(total) - torch.where(e > 0, e * (z - top), torch.zeros_like(e)).sum(dim=1) / total
        named = s["tokens"] >= 0
        picked = z.gather(1, torch.where(named, s["tokens"], torch.zeros_like(s["tokens"]))[:, None])[:, 0] - lse
        out = {"logprob": torch.where(named, picked, torch.zeros_like(picked)), "entropy": entropy, "lse": lse}
        del e
    if mode != "forward":
        logp = z - lse[:, None]
        p = torch.exp(logp)
        grad = -p * (s["g_logprob"] * (s["tokens"] >= 0))[:, None]
        if s["g_entropy"] is not None:
            grad = grad - s["g_entropy"][:, None] * torch.where(p > 0, p * (logp + entropy[:, None]), torch.zeros_like(p))
        del p, logp
        hit = torch.arange(z.shape[1], device=z.device)[None, :] == s["tokens"][:, None]
        grad = (grad + torch.where(hit, s["g_logprob"][:, None], torch.zeros_like(grad))) / s["temperature"]
        del hit
        out["dhidden"] = torch.matmul(grad, weight).to(s["hidden"].dtype)
        out["dweight"] = torch.matmul(grad.t(), hidden).to(s["weight"].dtype)
        if s["bias"] is not None:
            out["dbias"] = grad.sum(dim=0)
    return out


_MASK = (1 << 32) - 1


def _mix(x):
    """A hash of 32 bits (of a number, or of int64 elements)."""
    x = x & _MASK
    x = ((x ^ (x >> 16)) * 0x7FEB352D) & _MASK
    x = ((x ^ (x >> 15)) * 0x846CA68B) & _MASK
    return x ^ (x >> 16)


def _random_bits(seed, step, tensor, n):
    """32 random bits for each of the n elements of a tensor."""
    key = _mix(_mix(_mix(seed) + step) + tensor)
    at = torch.arange(n, dtype=torch.int64, device="cuda")
    return _mix((at & _MASK) + key + (at >> 32) * 0x9E3779B9)


def _power(e):
    """2^e as fp32, for integer tensors -127 <= e <= 127."""
    return torch.where(e < -126, torch.full_like(e, 1 << 22), (e + 127) << 23).to(torch.int32).view(torch.float32)


def _blocks(t):
    """``t`` with zeros behind it, 32 elements to a row."""
    n = t.numel()
    return torch.cat([t, t.new_zeros(-n % 32)]).view(-1, 32)


def _decode(codes, exps, field, signed):
    c = _blocks(codes).long()
    magnitude = (((c & 127) if signed else c) << 20).to(torch.int32).view(torch.float32)
    e = exps.long()[:, None]
    y = magnitude * 2.0 ** field * _power(e - 127)
    if signed:
        y = torch.where(c > 127, -y, y)
    return torch.where(e == 255, torch.full_like(y, math.nan), y).view(-1)[:codes.numel()]


def _encode(y, random, field, signed, codes, exps):
    """``y`` (32 bits) into ``codes`` and ``exps``, rounded with the 20 random bits of each element."""
    n = y.numel()
    rows, random = _blocks(y), _blocks(random)
    size = rows.abs()
    e = (size.view(torch.int32).amax(dim=1, keepdim=True) >> 23).long().clamp(min=1)  # the bits of magnitudes are in order, NaN last
    bad = e >= 254
    safe = torch.where(bad, torch.full_like(e, 127), e)
    scaled = size * _power(127 - safe) * 2.0 ** -field
    code = (scaled.view(torch.int32).long() + random) >> 20
    if signed:
        code = code | (rows.view(torch.int32).long() >> 31 & 1) << 7
    else:
        code = torch.maximum(code, (size > 0).long())
    codes.copy_(torch.where(bad, torch.zeros_like(code), code).view(-1)[:n].to(torch.uint8))
    exps.copy_(torch.where(bad, torch.full_like(e, 255), e).view(-1).to(torch.uint8))


def _round_up_or_down(y, dtype, random):
    """``y`` rounded to 16 bits, up with the probability of the part cut off."""
    shift, field = (16, 0) if dtype == torch.bfloat16 else (13, 112)
    bits = (y.abs() * 2.0 ** -field).view(torch.int32).long()
    code = (bits + (random >> (32 - shift))) >> shift
    code = torch.minimum(code, torch.full_like(code, 0x7F80 if field == 0 else 0x7C00)) | (y.view(torch.int32).long() >> 31 & 1) << 15
    rounded = code.to(torch.int32).to(torch.int16).view(dtype)
    return torch.where(torch.isfinite(y), rounded, y.to(dtype))


def _plain_step(s):
    case, (b1, b2) = s["case"], BETAS
    t = case["step"]
    rate, root = s["lr"] / (1.0 - b1 ** t), 1.0 / math.sqrt(1.0 - b2 ** t)
    moments = []
    for i, (p, g, master, m, v, me, ve) in enumerate(s["tensors"]):  # every tensor has blocks and random numbers of its own
        old = p.float() if master is None else master
        g = g.float()
        if s["grad_scale"] is not None:
            g = g * s["grad_scale"]
        eight = case["bits"] == 8
        random = _random_bits(s["seed"], t, i, p.numel()) if eight or case["rounding"] == "stochastic" else None
        m0, v0 = (_decode(m, me, 113, True), _decode(v, ve, 97, False)) if eight else (m, v)
        m1 = m0 * b1 + g * (1.0 - b1)
        v1 = v0 * b2 + (g * (1.0 - b2)) * g
        new = old * (1.0 - s["lr"] * s["decay"][i]) - (m1 * rate) / (torch.sqrt(v1) * root + EPS)
        if s["keep"][i]:
            zero = old == 0
            m1, v1, new = (torch.where(zero, torch.zeros_like(x), x) for x in (m1, v1, new))
        if eight:
            _encode(m1, random & 0xFFFFF, 113, True, m, me)
            _encode(v1, random >> 12, 97, False, v, ve)
            moments.append((_decode(m, me, 113, True).bfloat16(), _decode(v, ve, 97, False).bfloat16()))
        else:
            m.copy_(m1)
            v.copy_(v1)
        if master is not None:
            master.copy_(new)
        p.copy_(_round_up_or_down(new, p.dtype, random * 0x9E3779B1 & _MASK) if case["rounding"] == "stochastic" else new)
    out = {"params": s["params"], "master": s["master"]}
    out.update({"m": s["m"], "v": s["v"]} if case["bits"] == 32 else {"moments": moments})
    return out


# ------------------------------------------------------------------------------------------------ work

def work(case):
    if case["op"] == "head":
        r, v, d = case["r"], case["v"], case["d"]
        once = 2 * (r * d + v * d) + (4 * v if case["bias"] else 0) + 8 * r
        if case["mode"] == "forward":
            return {"bytes": once + 12 * r, "flops": 2 * r * v * d}
        return {"bytes": 2 * once + 20 * r, "flops": 6 * r * v * d}
    n, size, gsize = sum(_sizes(case)), 4 if case["dtype"] == "f32" else 2, 4 if case["grads"] == "f32" else 2
    weights = 8 + size if case["master"] else 2 * size           # a copy in 32 bits is read in the weight's place
    moments = 16 if case["bits"] == 32 else 4 + 4 / 32 + 4       # in 8 bits: read, written, and read back as values of 16 bits
    return {"bytes": n * (weights + gsize + moments), "flops": 15 * n}


# ------------------------------------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return _exact_head(s) if case["op"] == "head" else _exact_step(s)


def _exact_head(s):
    case, temperature = s["case"], s["temperature"]
    mode, weight = case["mode"], s["weight"].double()
    step, parts = max(1, (1 << 28) // case["v"]), []
    dweight = torch.zeros_like(weight) if mode != "forward" else None
    dbias = torch.zeros(case["v"], dtype=torch.float64, device="cuda") if mode != "forward" else None
    for a in range(0, case["r"], step):
        h, tokens = s["hidden"][a:a + step].double(), s["tokens"][a:a + step]
        logits = h @ weight.T
        if s["bias"] is not None:
            logits += s["bias"].double()
        logits /= temperature
        rows, named, at = torch.arange(h.shape[0], device=h.device), tokens >= 0, tokens.clamp(min=0)
        part = {}
        if mode == "backward":
            lse, entropy = s["lse"][a:a + step].double(), s["saved_entropy"][a:a + step].double()
            prob = (logits - lse[:, None]).exp()
        else:
            lse = torch.logsumexp(logits, 1)
            prob = torch.softmax(logits, 1)
            entropy = torch.special.entr(prob).sum(1)
            part = {"logprob": (logits[rows, at] - lse).masked_fill(~named, 0.0), "entropy": entropy, "lse": lse}
        if mode != "forward":
            gl = s["g_logprob"][a:a + step].double() * named
            grad = prob * -gl[:, None]
            if s["g_entropy"] is not None:
                ge = s["g_entropy"][a:a + step].double()
                grad += ge[:, None] * (torch.special.entr(prob) - prob * entropy[:, None])
            grad[rows, at] += gl
            grad /= temperature
            part["dhidden"] = grad @ weight
            dweight += grad.T @ h
            dbias += grad.sum(0)
        parts.append(part)
    out = {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
    if mode != "forward":
        out["dweight"] = dweight
        if s["bias"] is not None:
            out["dbias"] = dbias
    return out


def _exact_lattice(y, u, lowest, floor=False):
    """``y`` (64 bits) on floating-point numbers of 3 bits of mantissa relative to the largest of each 32, whose binade is 0; ``lowest``
    is the last binade with a leading 1.  ``u`` in [0, 1) decides about the part cut off."""
    n = y.numel()
    pad = -n % 32
    rows = torch.nn.functional.pad(y, (0, pad)).view(-1, 32)
    u = torch.nn.functional.pad(u, (0, pad)).view(-1, 32)
    top = torch.frexp(rows.abs().amax(1, keepdim=True))[1] - 1
    binade = torch.maximum(torch.frexp(rows)[1] - 1, top + lowest)
    unit = torch.ldexp(torch.ones_like(rows), binade - 3)
    steps = torch.floor(rows.abs() / unit + u)
    if floor:
        steps = torch.where(rows > 0, steps.clamp(min=1), steps)
    return (torch.sign(rows) * steps * unit).view(-1)[:n]


def _exact_step(s):
    case, t = s["case"], s["case"]["step"]
    b1, b2 = BETAS
    eight, moments = case["bits"] == 8, []
    out = {"params": torch.zeros_like(s["params"], dtype=torch.float64), "master": None}
    base = {"params": s["params"]}
    if s["master"] is not None:
        out["master"], base["master"] = torch.zeros_like(s["master"], dtype=torch.float64), s["master"]
    if not eight:
        out.update(m=torch.zeros_like(s["m"], dtype=torch.float64), v=torch.zeros_like(s["v"], dtype=torch.float64))
    for i, (p, g, master, m, v, me, ve) in enumerate(s["tensors"]):
        w = (p if master is None else master).double()
        g = g.double() * (1.0 if s["grad_scale"] is None else s["grad_scale"].double())
        first, second = (_decode(m, me, 113, True), _decode(v, ve, 97, False)) if eight else (m, v)
        first = first.double().lerp(g, 1.0 - b1)
        second = second.double() * b2 + (1.0 - b2) * g.square()
        change = first / (1.0 - b1 ** t) / ((second / (1.0 - b2 ** t)).sqrt() + EPS) + s["decay"][i] * w
        new = w - s["lr"] * change
        if s["keep"][i]:
            there = (w != 0).double()
            first, second, new = first * there, second * there, new * there
        bits = _random_bits(s["seed"], t, i, p.numel()).double() if eight or case["rounding"] == "stochastic" else None
        if eight:
            u = bits / 2.0 ** 32
            moments.append((_exact_lattice(first, torch.remainder(bits, 2.0 ** 20) / 2.0 ** 20, -13),
                            _exact_lattice(second, u, -29, floor=True)))
        else:
            for name, value, at in (("m", first, m), ("v", second, v)):
                out[name][at.storage_offset():at.storage_offset() + at.numel()] = value
        if master is not None:
            out["master"][master.storage_offset():master.storage_offset() + master.numel()] = new
        out["params"][p.storage_offset():p.storage_offset() + p.numel()] = new
    if eight:
        out["moments"] = moments
    return out
