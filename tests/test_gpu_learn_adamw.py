"""GPU: the AdamW step against its formula in 64 bits, for 32- and 8-bit states.

Bounds: m has three roundings, v four, each of 2^-24 of the terms; the update
lr mhat / (sqrt(vhat) + eps) seven more; an 8-bit code is off by half a step,
2^-4 of the value or half the smallest code, 2^-10 of the block's scale."""
import math

import pytest

import learn_util as U
from gpu_util import need_gpu, note

pytestmark = pytest.mark.gpu
HYPER = dict(lr=1e-3, betas=(0.9, 0.99), eps=1e-6, weight_decay=0.05)


def tensors(sizes, bits, half, seed=0, shift=0):
    torch = need_gpu()
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        def buf(t, scale=1.0):
            x = (torch.randn(n + shift, device="cuda", generator=g) * scale).to(t)
            return x[shift:]
        t = dict(param=buf(torch.float32), grad=buf(torch.bfloat16 if half else torch.float32, 0.01), decay=i % 2 == 0)
        if bits == 32:
            t |= dict(m=buf(torch.float32, 0.01), v=buf(torch.float32, 0.01).square_())
        else:
            codes = torch.randint(0, 256, (2, n + shift), device="cuda", generator=g, dtype=torch.uint8)
            codes[codes % 128 == 127] = 0                  # no NaN codes
            codes[1] &= 127                                # sqrt(v) is not negative
            blocks = -(-n // 256)
            t |= dict(m=codes[0, shift:].view(torch.float8_e4m3fn), v=codes[1, shift:].view(torch.float8_e4m3fn),
                      m_scale=torch.rand(blocks, device="cuda", generator=g) * 1e-4,
                      v_scale=torch.rand(blocks, device="cuda", generator=g) * 1e-4)
        if i != 1:
            t["copy"] = torch.zeros(n + shift, dtype=torch.bfloat16, device="cuda")[shift:]
        out.append(t)
    return out


def spread(scale, n):
    return scale.double().repeat_interleave(256)[:n]


def expected(t, bits, step, scale, h=HYPER):
    n = t["param"].numel()
    b1, b2 = h["betas"]
    g = t["grad"].double() * scale
    if bits == 32:
        m, v = t["m"].double(), t["v"].double()
    else:
        m = t["m"].float().double() * spread(t["m_scale"], n)
        v = (t["v"].float().double() * spread(t["v_scale"], n)) ** 2
    em = 4 * U.U * ((b1 * m).abs() + (1 - b1) * g.abs())
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    ev = 8 * U.U * v
    mh, vh = m / (1 - b1 ** step), v / (1 - b2 ** step)
    den = vh.sqrt() + h["eps"]
    up = h["lr"] * mh / den
    keep = 1 - h["lr"] * h["weight_decay"] if t["decay"] else 1.0
    p = t["param"].double() * keep - up
    ep = 4 * U.U * (t["param"].double().abs() + up.abs()) + 16 * U.U * up.abs() + h["lr"] * em / (1 - b1 ** step) / den
    return dict(m=m, v=v, p=p, em=em, ev=ev, ep=ep)


def clone(ts):
    return [{k: (x.clone() if hasattr(x, "clone") else x) for k, x in t.items()} for t in ts]


def check(ts, old, bits, step, scale, h=HYPER):
    for i, (t, o) in enumerate(zip(ts, old)):
        r, n = expected(o, bits, step, scale, h), t["param"].numel()
        U.close(t["param"], r["p"], r["ep"], f"param {i}")
        if "copy" in t:
            assert bool((t["copy"] == t["param"].bfloat16()).all())
        if bits == 32:
            U.close(t["m"], r["m"], r["em"], f"m {i}")
            U.close(t["v"], r["v"], r["ev"], f"v {i}")
            continue
        for key, want, err in (("m", r["m"], r["em"]), ("v", r["v"].sqrt(), 8 * U.U * r["v"].sqrt())):
            s = t[key + "_scale"].double()
            pad = -n % 256
            import torch
            top = torch.nn.functional.pad(want.abs(), (0, pad)).view(-1, 256).amax(1)
            U.close(s, (top / 448).clamp_min(2.0 ** -126), 16 * U.U * top / 448, f"{key}_scale {i}")
            got, S = t[key].float().double() * spread(t[key + "_scale"], n), spread(t[key + "_scale"], n)
            tol = 2.0 ** -4 * want.abs() * (1 + 1e-5) + S * 2.0 ** -10 + err
            if key == "v":   # what is above zero has the smallest code at least
                tol = tol + S * 2.0 ** -9 * (want < S * 2.0 ** -9)
                assert bool((t["v"].float()[want > 0] > 0).all())
            U.close(got, want, tol, f"{key} {i}")


SIZES = [[1], [4096], [255, 256, 257, 0, 4095, 4097], [86 * 256, 256, 256 * 256, 256, 256 * 15, 15], [1000003, 7]]


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("sizes", SIZES)
def test_step(sizes, bits, half):
    import paper_2606_11440_amd as P
    torch = need_gpu()
    note(f"[adamw] {sizes} bits={bits} half={half}")
    ts = tensors(sizes, bits, half, seed=len(sizes))
    opt = P.AdamW(ts, bits=bits)
    step = torch.full((1,), 7, dtype=torch.int64, device="cuda")
    scale = torch.full((1,), 0.5, device="cuda")
    for k in range(3):
        old = clone(ts)
        for t in ts:
            t["grad"].mul_(0.9)
        old = clone(ts)
        opt.step(step, scale=scale if k else None, **HYPER)
        torch.cuda.synchronize()
        assert int(step) == 8 + k
        check(ts, old, bits, 8 + k, 0.5 if k else 1.0)
    opt.close()


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("shift", [1, 2, 3])
def test_any_alignment(shift, bits, half):
    import paper_2606_11440_amd as P
    torch = need_gpu()
    note(f"[adamw alignment] shift={shift} bits={bits} half={half}")
    ts = tensors([5000, 3], bits, half, seed=shift, shift=shift)
    old = clone(ts)
    opt = P.AdamW(ts, bits=bits)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    opt.step(step, **HYPER)
    torch.cuda.synchronize()
    check(ts, old, bits, 1, 1.0)


@pytest.mark.parametrize("bits", [32, 8])
def test_from_zero_states(bits):
    """The first step moves each parameter by lr against its gradient's sign
    (where the gradient is far above eps); a zero gradient moves nothing."""
    import paper_2606_11440_amd as P
    torch = need_gpu()
    t = tensors([1000], bits, False, seed=1)[0]
    for k in ("m", "v", "m_scale", "v_scale"):
        if k in t:
            t[k].view(torch.uint8).zero_() if t[k].dtype == torch.float8_e4m3fn else t[k].zero_()
    t["grad"] = torch.where(torch.arange(1000, device="cuda") % 3 == 0, torch.zeros_like(t["grad"]), t["grad"].sign())
    before = t["param"].clone()
    opt = P.AdamW([t], bits=bits)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    opt.step(step, lr=0.01, betas=(0.9, 0.999), eps=1e-12, weight_decay=0.0)
    torch.cuda.synchronize()
    # t = 1: mhat = g, vhat = g^2 up to the roundings of 1 - beta (2^-24 / (1 - beta2) of it) and the others
    moved = before.double() - t["param"].double()
    U.close(moved, 0.01 * t["grad"].double(), 0.01 * (2.0 ** -24 / 0.001 + 16 * U.U) + 2 * U.U * before.double().abs(), "moved")


def test_values_that_are_not_finite_stay_in_their_block():
    import paper_2606_11440_amd as P
    torch = need_gpu()
    t = tensors([1024], 8, False, seed=2)[0]
    t["grad"][300] = float("nan")
    t["grad"][600] = float("inf")
    opt = P.AdamW([t], bits=8)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    opt.step(step, **HYPER)
    torch.cuda.synchronize()
    m = t["m"].float() * t["m_scale"].repeat_interleave(256)
    for k, whole in enumerate((True, False, False, True)):
        assert bool(torch.isfinite(m[k * 256:(k + 1) * 256]).all()) == whole
        assert whole or bool(torch.isnan(m[k * 256:(k + 1) * 256]).all())
    assert int(torch.isnan(t["param"]).sum()) == 2


def test_no_tensors_counts_the_step():
    import paper_2606_11440_amd as P
    torch = need_gpu()
    opt = P.AdamW([])
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    opt.step(step, **HYPER)
    opt.step(step, **HYPER)
    torch.cuda.synchronize()
    assert int(step) == 2


def test_refusals():
    import paper_2606_11440_amd as P
    torch = need_gpu()
    t = tensors([100], 32, False)[0]
    for over in (dict(param=t["param"].half()), dict(grad=t["grad"][:50]), dict(grad=t["grad"].double()),
                 dict(m=t["m"].bfloat16()), dict(v=t["v"].cpu()), dict(copy=t["copy"].float()),
                 dict(param=torch.zeros(200, device="cuda")[::2])):
        with pytest.raises(P.IMError):
            P.AdamW([t | over])
    with pytest.raises(P.IMError):
        P.AdamW([t], bits=8)
    with pytest.raises(P.IMError):
        P.AdamW([t, t | dict(grad=t["grad"].bfloat16())])
    opt = P.AdamW([t])
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    for over in (dict(lr=-1.0), dict(lr=math.nan), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=-1e-8),
                 dict(weight_decay=-1.0)):
        with pytest.raises(P.IMError) as e:
            opt.step(step, **(HYPER | over))
        assert e.value.status == P._lib.IM_EINVAL
    with pytest.raises(P.IMError):
        opt.step(step.int(), **HYPER)
    opt.close()
    with pytest.raises(P.IMError):
        opt.step(step, **HYPER)


def test_a_plan_dropped_while_a_graph_is_captured():
    import gc

    import paper_2606_11440_amd as P
    torch = need_gpu()
    note("[adamw dropped]")
    ts = tensors([5000, 300], 32, False, seed=9)
    start, step = clone(ts), torch.zeros(1, dtype=torch.int64, device="cuda")
    opt, other = P.AdamW(ts), P.AdamW(tensors([100], 8, True, seed=10), bits=8)
    other.step(torch.zeros(1, dtype=torch.int64, device="cuda"), **HYPER)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step(step, **HYPER)
        del other
        gc.collect()
    for k in range(3):
        old = clone(ts)
        graph.replay()
        torch.cuda.synchronize()
        assert int(step) == k + 1
        check(ts, old, 32, k + 1, 1.0)
    again, count = clone(start), torch.zeros(1, dtype=torch.int64, device="cuda")
    eager = P.AdamW(again)
    for _ in range(3):
        eager.step(count, **HYPER)
    torch.cuda.synchronize()
    assert all(torch.equal(a["param"], b["param"]) for a, b in zip(again, ts))


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-45])
@pytest.mark.parametrize("bits", [32, 8])
def test_gradients_whose_squares_are_subnormal(bits, eps, half):
    """Gradients of 1e-20 to 1e-17 have v down to 1e-42, which the formula divides by
    like any other. There a rounding is half of 2^-149: up to four of those in v
    (the square, its product with 1 - beta2, the state's with beta2, a decoded
    state's square), half of their share of v in its root."""
    import paper_2606_11440_amd as P
    torch = need_gpu()
    note(f"[adamw subnormal] bits={bits} eps={eps} half={half}")
    t = tensors([3000], bits, half, seed=3)[0]
    g = torch.Generator(device="cuda").manual_seed(4)
    size = 10.0 ** (-20 + 3 * torch.rand(3000, device="cuda", generator=g, dtype=torch.float64))
    t["grad"] = (size * t["grad"].double().sign()).to(t["grad"].dtype)
    t["grad"][t["grad"] == 0] = 1e-18
    for k in ("m", "v", "m_scale", "v_scale"):
        if k in t:
            t[k].view(torch.uint8).zero_() if t[k].dtype == torch.float8_e4m3fn else t[k].zero_()
    opt, step, h = P.AdamW([t], bits=bits), torch.zeros(1, dtype=torch.int64, device="cuda"), HYPER | dict(eps=eps)
    lost = 4 * 2.0 ** -150
    for k in range(1, 4):
        old = clone([t])[0]
        opt.step(step, **h)
        torch.cuda.synchronize()
        r = expected(old, bits, k, 1.0, h)
        up = (r["p"] - old["param"].double() * (1 - h["lr"] * h["weight_decay"])).abs()
        U.close(t["param"], r["p"], r["ep"] + up * lost / (2 * r["v"] - lost), f"param, step {k}")
        if bits == 32:
            U.close(t["v"], r["v"], r["ev"] + lost, "v")
        else:
            assert bool((t["v"].float() > 0).all())


@pytest.mark.parametrize("bits", [32, 8])
def test_zero_states_and_gradients_with_the_least_eps(bits):
    """0 / eps is 0 for every eps above 0."""
    import paper_2606_11440_amd as P
    torch = need_gpu()
    for eps in (5e-324, 1e-45, 1e-39, 1e-38):
        t = tensors([600], bits, False, seed=5)[0]
        for k in ("m", "v", "m_scale", "v_scale", "grad"):
            if k in t:
                t[k].view(torch.uint8).zero_() if t[k].dtype == torch.float8_e4m3fn else t[k].zero_()
        before = t["param"].clone()
        P.AdamW([t], bits=bits).step(torch.zeros(1, dtype=torch.int64, device="cuda"), lr=0.01, eps=eps, weight_decay=0.0)
        torch.cuda.synchronize()
        assert torch.equal(t["param"], before), eps
