"""AdamW steps over many tensors (include/spdy_eval.h, spdy_adamw_*)."""
import ctypes
import math

import numpy as np
import pytest
import torch

import eval_reference as ref
import tune_reference as tune
from paper_2201_13096_b200 import binding, build as build_mod, evaluate

INF = math.inf
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
gpu = pytest.mark.gpu
SIZES = (1, 31, 32, 33, 255, 256, 2047, 2048, 2049, 5000)


@pytest.fixture(scope="module", autouse=True)
def built():
    build_mod.build()


def values(n, seed, scale=1.0):
    return torch.randn(n, generator=torch.Generator().manual_seed(seed)) * scale


def at(buffer_dtype, v, shift):
    """``v`` on the GPU, ``shift`` elements into a buffer."""
    buf = torch.full((v.numel() + shift + 3,), 7.0, dtype=buffer_dtype, device="cuda")
    part = buf[shift:shift + v.numel()]
    part.copy_(v)
    return part


def gradient(n, seed, scale=1.0):
    """Values over several orders of magnitude, zeros among them."""
    g = values(n, seed) * torch.exp(2.0 * values(n, seed + 1)) * 1e-3 * scale
    return torch.where(values(n, seed + 2) > 1.5, torch.zeros(n), g)


def snapshot(plan):
    old = [ref.d64(p if w is None else w).flatten() for p, w in zip(plan.params, plan.masters)]
    if plan.bits == 32:
        return old, [ref.d64(x.m) for x in plan.moments], [ref.d64(x.v) for x in plan.moments]
    return old, [tune.decode(x, True) for x in plan.moments], [tune.decode(x, False) for x in plan.moments]


def check_step(plan, grads, before, lr, step, seed, decay, keep, scale=1.0):
    for i, (p, w, mom) in enumerate(zip(plan.params, plan.masters, plan.moments)):
        old, m, v = (x[i] for x in before)
        new, m1, v1, ep, em, ev = tune.adamw(old, ref.d64(grads[i]).flatten() * scale, m, v, lr, decay[i], plan.betas, plan.eps, step, keep[i])
        bits = tune.random_bits(seed, step, i, p.numel())
        if plan.bits == 32:
            ref.close(mom.m, m1, em, f"m of {i}")
            ref.close(mom.v, v1, ev, f"v of {i}")
        else:
            tune.check_codes(mom, True, m1, em, bits, f"m of {i}")
            tune.check_codes(mom, False, v1, ev, bits, f"v of {i}")
        if w is not None:
            ref.close(w.flatten(), new, ep, f"master of {i}")
            assert torch.equal(p, w.to(p.dtype))
        elif plan.rounding == "stochastic" and p.dtype != F32:
            tune.check_random_rounding(p.flatten(), new, ep, bits, f"param {i}")
        else:
            ref.close(p.flatten(), new, ep, f"param {i}")


KINDS = [
    # param, gradient, master, rounding
    (F32, F32, False, "nearest"), (BF16, BF16, False, "nearest"), (BF16, BF16, False, "stochastic"), (BF16, F32, True, "nearest"),
    (F16, F16, True, "nearest"), (F16, F32, False, "stochastic"), (F16, F16, False, "nearest"), (BF16, BF16, True, "stochastic"),
]


@gpu
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("ptype,gtype,master,rounding", KINDS)
def test_steps_against_the_formula(ptype, gtype, master, rounding, bits, shift):
    params = [at(ptype, values(n, i) * (values(n, i + 50) > 0), shift) for i, n in enumerate(SIZES)]  # half of them 0
    neighbours = [p._base.clone() for p in params]
    decay, keep = [0.0 if i % 3 else 0.1 for i in range(len(SIZES))], [i % 2 == 0 for i in range(len(SIZES))]
    plan = evaluate.AdamW(params, bits=bits, masters=True if master else None, weight_decay=decay, keep_zeros=keep, rounding=rounding, eps=1e-6)
    scale = torch.full((1,), 1.0 / 512.0, device="cuda") if gtype == F16 else None
    for step in (1, 2, 900):
        grads = [at(gtype, gradient(n, 100 * step + i, 512.0 if scale is not None else 1.0), shift) for i, n in enumerate(SIZES)]
        before = snapshot(plan)
        evaluate.adamw_step(plan, grads, lr=0.01, step=step, seed=77, grad_scale=scale)
        check_step(plan, grads, before, 0.01, step, 77, decay, keep, 1.0 / 512.0 if scale is not None else 1.0)
    for p, before, k in zip(params, neighbours, keep):
        whole = before.clone()
        whole[shift:shift + p.numel()] = p
        assert torch.equal(whole, p._base)
        if k:
            assert (p[before[shift:shift + p.numel()] == 0] == 0).all()


@gpu
def test_pruned_weights_stay_pruned_and_leave_their_block():
    p = torch.randn(256, device="cuda")
    p[::2] = 0
    plan = evaluate.AdamW([p], bits=8, keep_zeros=True)
    g = torch.where(torch.arange(256, device="cuda") % 2 == 0, 1e6, 1e-3)  # large where it does not count
    evaluate.adamw_step(plan, [g], lr=0.1, step=1)
    m, v = evaluate.adamw_moments(plan)[0]
    assert (p[::2] == 0).all() and (m[::2] == 0).all() and (v[::2] == 0).all()
    assert torch.allclose(m[1::2], torch.full((128,), 1e-4, device="cuda"), rtol=0.13) and (v[1::2] > 0).all()


@gpu
@pytest.mark.parametrize("dtype", [None, F32, BF16])
def test_moments_as_numbers(dtype):
    params = [torch.randn(n, device="cuda") for n in SIZES] + [torch.randn(7, 9, device="cuda")]
    plan = evaluate.AdamW(params, bits=8)
    evaluate.adamw_step(plan, [gradient(p.numel(), i).view(p.shape).cuda() for i, p in enumerate(params)], lr=0.01, step=1)
    for (m, v), mom, p in zip(evaluate.adamw_moments(plan, dtype), plan.moments, params):
        assert m.shape == v.shape == p.shape and m.dtype == v.dtype == (dtype or F32)
        assert torch.equal(ref.d64(m).flatten(), tune.decode(mom, True)) and torch.equal(ref.d64(v).flatten(), tune.decode(mom, False))
    plan = evaluate.AdamW(params)
    assert evaluate.adamw_moments(plan)[0][0].data_ptr() == plan.moments[0].m.data_ptr()


@gpu
def test_averages_in_8_bits_keep_moving():
    # 400 steps of a constant gradient: v rises by 0.1 % of what is left each step, far below the distance of its neighbours.  Each step's rounding
    # has a standard deviation of at most half a unit (2^-3 of the value's power of two, at most 1/8 of the value), and the mean is over n
    # independent elements.
    n, steps = 8192, 400
    p = torch.zeros(n, device="cuda")
    plan = evaluate.AdamW([p], bits=8, weight_decay=0.0)
    g = torch.full((n,), 0.5, device="cuda")
    for t in range(1, steps + 1):
        evaluate.adamw_step(plan, [g], lr=0.0, step=t, seed=5)
    m, v = evaluate.adamw_moments(plan)[0]
    want = 0.25 * (1 - 0.999 ** steps)
    assert abs(float(v.double().mean()) - want) < 6 * want / 8 / 2 * math.sqrt(steps) / math.sqrt(n)
    assert abs(float(m.double().mean()) - 0.5) < 6 * 0.5 / 8 / 2 * math.sqrt(1 / (1 - 0.81)) / math.sqrt(n) + 1e-6


@gpu
def test_small_second_moments_have_a_floor():
    g = torch.zeros(32, device="cuda")
    g[0], g[1] = 1.0, 1e-12  # v of the second would be 1e-24 of the first's
    plan = evaluate.AdamW([torch.ones(32, device="cuda")], bits=8)
    evaluate.adamw_step(plan, [g], lr=0.0, step=1)
    m, v = evaluate.adamw_moments(plan)[0]
    assert 0 < float(v[1]) <= 2.0 ** -31 * 0.001 and (v[2:] == 0).all()


@gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [INF, -INF, math.nan, 3e38])
def test_gradients_that_are_not_finite(bits, bad):
    p = torch.ones(2100, device="cuda")
    plan, clean = (evaluate.AdamW([t], bits=bits) for t in (p, p.clone()))
    g = gradient(2100, 3).cuda()
    evaluate.adamw_step(clean, [g], lr=0.1, step=1)
    spoilt = g.clone()
    spoilt[70] = bad
    evaluate.adamw_step(plan, [spoilt], lr=0.1, step=1)
    others = torch.ones(2100, dtype=torch.bool, device="cuda")
    others[70] = False
    assert torch.equal(p[others], clean.params[0][others])
    v = evaluate.adamw_moments(plan)[0][1]
    block = torch.arange(2100, device="cuda") // 32 == 70 // 32
    assert torch.equal(v[~block], evaluate.adamw_moments(clean)[0][1][~block])
    if bits == 8:
        assert torch.isnan(v[block]).all()
    else:
        assert not torch.isfinite(v[70])


@gpu
@pytest.mark.parametrize("scale", [1e-30, 1e-19, 1e5, 1e15, 1e19])
def test_gradients_of_any_size(scale):
    n = 4096
    p = torch.ones(n, device="cuda")
    plan = evaluate.AdamW([p], bits=8, eps=0.0)
    for t in (1, 2):
        before = snapshot(plan)
        g = (values(n, t).abs() + 0.5) * scale
        evaluate.adamw_step(plan, [g.cuda()], lr=0.01, step=t, seed=1)
        if scale > 1e-20:
            check_step(plan, [g], before, 0.01, t, 1, [0.01], [False])
        else:  # squares are below fp32: m is still right
            _, m1, _, _, em, _ = tune.adamw(before[0][0], ref.d64(g), before[1][0], before[2][0], 0.01, 0.01, plan.betas, 0.0, t, False)
            tune.check_codes(plan.moments[0], True, m1, em, tune.random_bits(1, t, 0, n), "m")


@gpu
def test_more_tensors_than_a_launch_takes_and_kinds_together():
    types = (F32, BF16, F16)
    params = [values(1 + i % 70, i).cuda().to(types[i % 3]) for i in range(1200)]
    alone = [p.clone() for p in params]
    grads = [gradient(p.numel(), i).cuda().to(p.dtype) if i % 7 else None for i, p in enumerate(params)]
    plan = evaluate.AdamW(params, weight_decay=0.1)
    evaluate.adamw_step(plan, grads, lr=0.01, step=3)
    for i, (p, a) in enumerate(zip(params, alone)):
        if grads[i] is None:
            assert torch.equal(p, a) and (plan.moments[i].m == 0).all()
            continue
        one = evaluate.AdamW([a], weight_decay=0.1)
        evaluate.adamw_step(one, [grads[i]], lr=0.01, step=3)
        assert torch.equal(p, a) and torch.equal(one.moments[0].v, plan.moments[i].v), i


@gpu
def test_empty_tensors_and_lists_of_nothing():
    params = [torch.zeros(0, device="cuda"), torch.ones(5, device="cuda"), torch.zeros(3, 0, device="cuda")]
    plan = evaluate.AdamW(params, bits=8)
    evaluate.adamw_step(plan, [torch.zeros_like(p) + 1.0 for p in params], lr=0.1, step=1)
    assert (params[1] < 1).all()
    evaluate.adamw_step(plan, [None] * 3, lr=0.1, step=2)
    assert evaluate.adamw_moments(plan)[2][0].shape == (3, 0)


@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_numbers_on_the_device_skips_streams_and_graphs(bits):
    def fresh():
        params = [values(n, n).cuda().to(BF16) for n in SIZES]
        return evaluate.AdamW(params, bits=bits, rounding="stochastic"), [gradient(n, n + 1).cuda().to(BF16) for n in SIZES]

    def state(plan):
        return [t.clone() for t in plan._written()]

    host, grads = fresh()
    for t in range(1, 6):
        evaluate.adamw_step(host, grads, lr=0.01 / t, step=t, seed=9)
    graphed, grads = fresh()
    lr, step, skip = torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, device="cuda")
    first = state(graphed)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    skip.fill_(1.0)
    side.wait_stream(torch.cuda.current_stream())
    evaluate.adamw_step(graphed, grads, lr=lr, step=step, seed=9, skip=skip, stream=side)  # changes nothing
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, state(graphed)))
    skip.zero_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step.add_(1)
        evaluate.adamw_step(graphed, grads, lr=lr, step=step, seed=9, skip=skip)
    for t in range(1, 6):
        lr.fill_(0.01 / t)
        g.replay()
    torch.cuda.synchronize()
    for a, b in zip(host._written(), graphed._written()):
        # lr passes through fp32 here, which moves the last place of the update
        if a.dtype == torch.uint8:
            assert torch.equal(a, b)
        elif a.dtype == F32:
            assert torch.equal(a, b)
        else:
            assert ((a.float() - b.float()).abs() <= 2.0 ** -7 * a.float().abs()).all() and (a != b).float().mean() < 0.01


@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_numbers_on_the_device_with_more_chunks_than_blocks(bits):
    sizes = (6_000_001, 33, 3_000_000)  # blocks walk over several chunks, and from one tensor into the next

    def run(device):
        params = [values(n, n % 1000).cuda().to(BF16) for n in sizes]
        plan = evaluate.AdamW(params, bits=bits, rounding="stochastic")
        for t in (1, 2):
            grads = [gradient(n, t + n % 1000).cuda().to(BF16) for n in sizes]
            if device:
                evaluate.adamw_step(plan, grads, lr=torch.full((1,), 0.25, device="cuda"), step=torch.full((1,), t, dtype=torch.int64, device="cuda"), seed=4)
            else:
                evaluate.adamw_step(plan, grads, lr=0.25, step=t, seed=4)
        return list(plan._written())

    for a, b in zip(run(False), run(True)):  # 0.25 is the same in fp32
        assert torch.equal(a, b)


@gpu
def test_parameters_that_moved_are_refused():
    p = torch.ones(64, device="cuda")
    plan = evaluate.AdamW([p])
    p.data = torch.ones(64, device="cuda")
    with pytest.raises(ValueError, match="stay where"):
        evaluate.adamw_step(plan, [torch.ones(64, device="cuda")], lr=0.1, step=1)


@gpu
def test_leaves_of_autograd_notice_the_step():
    w = torch.nn.Parameter(torch.randn(64, device="cuda"))
    y = (w * w).sum()
    plan = evaluate.AdamW([w])
    evaluate.adamw_step(plan, [torch.ones(64, device="cuda")], lr=0.1, step=1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    with pytest.raises(ValueError, match="requires a gradient"):
        evaluate.adamw_step(plan, [torch.ones(64, device="cuda", requires_grad=True)], lr=0.1, step=2)


@gpu
def test_offsets_beyond_32_bits():
    n, tail = (1 << 32) + 4097, 4097 + 40
    p, g = torch.zeros(n, dtype=BF16, device="cuda"), torch.zeros(n, dtype=BF16, device="cuda")
    p[-tail:] = values(tail, 1).cuda()
    g[-tail:] = gradient(tail, 2).cuda()
    old, grad = ref.d64(p[-tail:]), ref.d64(g[-tail:])
    plan = evaluate.AdamW([p], bits=8, rounding="stochastic")
    evaluate.adamw_step(plan, [g], lr=0.01, step=1, seed=3)
    first = n - tail
    skip = -first % 32  # whole blocks of the tail
    zeros = torch.zeros(tail - skip, dtype=torch.float64)
    new, m1, v1, ep, em, ev = tune.adamw(old[skip:], grad[skip:], zeros, zeros, 0.01, 0.01, plan.betas, plan.eps, 1, False)
    bits = tune.random_bits(3, 1, 0, tail - skip, first + skip)
    mom = plan.moments[0]
    part = evaluate.AdamWMoments(mom.m[first + skip:], mom.v[first + skip:], mom.m_exp[(first + skip) // 32:], mom.v_exp[(first + skip) // 32:])
    tune.check_codes(part, True, m1, em, bits, "m")
    tune.check_codes(part, False, v1, ev, bits, "v")
    tune.check_random_rounding(p[first + skip:], new, ep, bits, "param")
    assert not p[:first].any() and not mom.v[:first].any()


@gpu
def test_python_refusals():
    p, q = torch.zeros(40, device="cuda"), torch.zeros(40, device="cuda", dtype=BF16)
    for bad, match in (({"bits": 16}, "bits"), ({"rounding": "up"}, "rounding"), ({"betas": (1.0, 0.9)}, "betas"), ({"eps": -1.0}, "eps"),
                       ({"weight_decay": -0.1}, "weight_decay"), ({"weight_decay": [0.1, 0.1]}, "weight_decay"), ({"masters": [torch.zeros(40, device="cuda")]}, "float32"),
                       ({"moments": [evaluate.AdamWMoments(p, p)]}, "share memory"), ({"keep_zeros": [True] * 3}, "keep_zeros")):
        with pytest.raises(ValueError, match=match):
            evaluate.AdamW([p], **bad)
    with pytest.raises(ValueError, match="share memory"):
        evaluate.AdamW([p, p[8:]])
    with pytest.raises(ValueError, match="contiguous"):
        evaluate.AdamW([p[::2]])
    with pytest.raises(ValueError, match="contiguous"):
        evaluate.AdamW([p.cpu()])
    with pytest.raises(ValueError, match="float32, bfloat16 or float16"):
        evaluate.AdamW([p.double()])
    with pytest.raises(ValueError, match="16 bytes"):
        buf = torch.zeros(90, device="cuda")
        evaluate.AdamW([p], moments=[evaluate.AdamWMoments(buf[1:41], buf[48:88])])
    with pytest.raises(ValueError, match="moments"):
        evaluate.AdamW([p], bits=8, moments=[evaluate.AdamWMoments(p, p)])
    with pytest.raises(ValueError, match="masters"):
        evaluate.AdamW([q], masters=[p[:8]])
    with pytest.raises(ValueError, match="at least"):
        evaluate.AdamW([])
    plan, small = evaluate.AdamW([p]), evaluate.AdamW([q], bits=8)
    one = torch.ones(1, device="cuda")
    for args, match in ((([p, p], 0.1, 1), "one entry"), (([p[:3]], 0.1, 1), r"grads\[0\]"), (([p.half()], 0.1, 1), r"grads\[0\]"), (([p], one, 1), "step"),
                        (([p], 0.1, one), "step"), (([p.cpu()], 0.1, 1), r"grads\[0\]")):
        with pytest.raises(ValueError, match=match):
            evaluate.adamw_step(plan, *args)
    with pytest.raises(ValueError, match="grad_scale"):
        evaluate.adamw_step(plan, [p], 0.1, 1, grad_scale=one.double())
    for lr, step in ((-0.1, 1), (math.nan, 1), (0.1, 0), (0.1, -3)):
        with pytest.raises(binding.SpdyError):
            evaluate.adamw_step(plan, [torch.zeros_like(p)], lr, step)
    with pytest.raises(ValueError, match="float32"):
        evaluate.adamw_moments(plan, dtype=BF16)
    with pytest.raises(ValueError, match="dtype"):
        evaluate.adamw_moments(small, dtype=F16)


# ------------------------------------------------------------------------------------------------ without a GPU

def test_c_entries_refuse_bad_arguments_before_any_gpu_work():
    lib = evaluate.library()
    assert evaluate._TENSOR.itemsize == 88 and ctypes.sizeof(evaluate._AdamWOptions) == 80
    P = 1 << 20

    def step(table=(), options=(), count=1):
        t = np.zeros(1, dtype=evaluate._TENSOR)
        t[0] = (P, P, 0, P, P, P, P, 100, 0.1, 1, 1, 8, 0, 0)
        for name, value in dict(table).items():
            t[name] = value
        o = evaluate._AdamWOptions(0.1, 0.9, 0.999, 1e-8, 1, 0, 0)
        for name, value in dict(options).items():
            setattr(o, name, value)
        return lib.spdy_adamw_step(t.ctypes.data, count, ctypes.byref(o), None)

    for name, value in (("param", 0), ("param", P + 1), ("grad", P + 1), ("m", 0), ("v", 0), ("m", P + 8), ("v", P + 4), ("m_exp", 0), ("v_exp", 0), ("n", -1),
                        ("n", 1 << 42), ("weight_decay", -1.0), ("weight_decay", math.nan), ("weight_decay", INF), ("param_dtype", 3), ("grad_dtype", 2),
                        ("state_bits", 16), ("master", P + 2)):
        assert step({name: value}) == -1, name
    assert step({"param_dtype": 0, "grad_dtype": 0, "master": P}) == -1
    for name, value in (("lr", -1.0), ("lr", math.nan), ("beta1", 1.0), ("beta2", -0.1), ("beta2", math.nan), ("eps", -1.0), ("eps", INF), ("step", 0), ("rounding", 2),
                        ("lr_device", P), ("step_device", P + 4), ("grad_scale", P + 1), ("skip", P + 2)):
        assert step((), {name: value}) == -1, name
    assert step(count=-1) == -1
    assert lib.spdy_adamw_step(None, 1, None, None) == -1 and lib.spdy_adamw_step(None, 1, ctypes.byref(evaluate._AdamWOptions(0.1, 0.9, 0.9, 0.0, 1)), None) == -1
    assert step(count=0) == 0 and step({"n": 0}) == 0 and step({"grad": 0}) == 0

    def moments(table=(), m=P, v=P, dtype=0):
        t = np.zeros(1, dtype=evaluate._TENSOR)
        t[0] = (0, 0, 0, P, P, P, P, 100, 0.1, 1, 1, 8, 0, 0)
        for name, value in dict(table).items():
            t[name] = value
        out = np.array([m, v], dtype=np.uint64)
        return lib.spdy_adamw_moments(t.ctypes.data, 1, out[:1].ctypes.data, out[1:].ctypes.data, dtype, None)

    assert moments(dtype=2) == -1 and moments({"state_bits": 32}) == -1 and moments(m=0) == -1 and moments(v=P + 2) == -1 and moments({"n": -1}) == -1
    assert moments({"n": 0}) == 0 and lib.spdy_adamw_moments(None, 1, None, None, 0, None) == -1


def test_the_hash_and_the_lattice_of_the_reference():
    # the reference's own parts, by hand: a block whose largest is 1.5, all its other fields
    import numpy as np
    E = 127
    codes = np.array([14 << 3 | 4, 128 | 14 << 3, 1, 7, 8] + [0] * 27, dtype=np.uint8)
    mom = evaluate.AdamWMoments(torch.from_numpy(codes), torch.from_numpy(np.array([30 << 3 | 4, 1, 8] + [0] * 29, dtype=np.uint8)),
                                torch.tensor([E], dtype=torch.uint8), torch.tensor([E], dtype=torch.uint8))
    assert tune.decode(mom, True)[:5].tolist() == [1.5, -1.0, 2.0 ** -16, 7 * 2.0 ** -16, 2.0 ** -13]
    assert tune.decode(mom, False)[:3].tolist() == [1.5, 2.0 ** -32, 2.0 ** -29]
    bits = tune.random_bits(1, 2, 3, 100000)
    assert 0 <= int(bits.min()) and int(bits.max()) < 1 << 32
    counts = torch.bincount(bits >> 28, minlength=16)  # sixteen equal shares: six standard deviations of a binomial count
    assert (counts - 6250).abs().max() < 6 * math.sqrt(100000 / 16)
