"""GPU: the softmax head and its gradient against 64 bits (bounds: learn_util)."""
import pytest

import learn_util as U
from gpu_util import need_gpu, note

pytestmark = pytest.mark.gpu
F32, BF16 = "float32", "bfloat16"


def make(n, d, V, sizes, dtype, seed=0, mask=True, pad=0, relu=True, scale=1.5):
    torch = need_gpu()
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = getattr(torch, dtype)
    G = len(sizes) if sizes else 1

    def normal(*s, scale=1.0, t=dt):
        return (torch.randn(*s, device="cuda", generator=g) * scale).to(t)
    h = normal(n, d + pad)[:, :d]
    if relu:
        h.relu_()
    off = None
    if sizes:
        off = [0]
        for s in sizes:
            off.append(off[-1] + s)
    words = (V + 31) // 32
    target = torch.randint(V, (n,), device="cuda", generator=g, dtype=torch.int32)
    valid = None
    if mask:
        bits = torch.rand(n, words * 32, device="cuda", generator=g) < 0.7
        bits[torch.arange(n), target.long()] = True
        none = torch.rand(n, device="cuda", generator=g) < 0.1
        one = torch.rand(n, device="cuda", generator=g) < 0.1     # only the target is valid
        bits[none | one] = False
        bits[one, target[one].long()] = True
        target[none] = -1
        w = (bits.view(n, words, 32).long() << torch.arange(32, device="cuda")).sum(2)
        valid = torch.where(w >= 2 ** 31, w - 2 ** 32, w).to(torch.int32)
    target[torch.rand(n, device="cuda", generator=g) < 0.1] = -1
    return dict(torch=torch, h=h, W=normal(G, V, d, scale=scale * d ** -0.5), b=normal(G, V, t=torch.float32), target=target,
                valid=valid, off=off, dev=None if off is None else torch.tensor(off, dtype=torch.int32, device="cuda"),
                G=G, dt=dt, dlogp=normal(n, t=torch.float32), dent=normal(n, scale=0.3, t=torch.float32))


def run_forward(c, b=True, entropy=True, lse=True):
    import paper_2606_11440_amd as P
    torch, n = c["torch"], c["h"].shape[0]
    o = {k: torch.full((n,), 77.0, device="cuda") for k in ("logp", "entropy", "lse")}
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    P.im_head_forward(c["h"], c["W"], c["b"] if b else None, c["target"], o["logp"], o["entropy"] if entropy else None,
                      o["lse"] if lse else None, valid=c["valid"], offsets=c["dev"], error=err)
    torch.cuda.synchronize()
    o["error"] = int(err)
    return o


def end_of(c):
    return c["off"][-1] if c["off"] else c["h"].shape[0]


def check_forward(c, b=True):
    o, e = run_forward(c, b), end_of(c)
    assert o["error"] == 0
    r = U.Head(c["h"], c["W"], c["b"] if b else None, c["valid"], c["target"], c["off"])
    U.close(o["logp"][:e], r.logp[:e], r.e_logp[:e], "logp")
    U.close(o["lse"][:e], r.lse[:e], r.e_logp[:e] + 2 * U.U * r.lse[:e].nan_to_num(0, 0, 0).abs(), "lse")
    U.close(o["entropy"][:e], r.H[:e], r.e_H[:e], "entropy")
    assert all(bool((o[k][e:] == 77.0).all()) for k in ("logp", "lse", "entropy"))
    return o, r


def run_backward(c, o, relu_in, ent=True, want=("dh", "dW", "db"), b=True):
    import paper_2606_11440_amd as P
    torch, (n, d), (G, V, _) = c["torch"], c["h"].shape, c["W"].shape
    q = dict(dh=torch.full((n, d + 3), 77.0, dtype=c["dt"], device="cuda")[:, :d],
             dW=torch.full((G, V, d), 77.0, dtype=c["dt"], device="cuda"), db=torch.full((G, V), 77.0, device="cuda"))
    q = {k: v if k in want else None for k, v in q.items()}
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    P.im_head_backward(c["h"], c["W"], c["b"] if b else None, c["target"], o["lse"], c["dlogp"], q["dh"], q["dW"], q["db"],
                       valid=c["valid"], entropy=o["entropy"] if ent else None, dentropy=c["dent"] if ent else None,
                       offsets=c["dev"], relu_in=relu_in, error=err)
    torch.cuda.synchronize()
    assert int(err) == c.get("error", 0)
    return q


def check_backward(c, o, r, relu_in, ent=True, want=("dh", "dW", "db"), b=True):
    q, e = run_backward(c, o, relu_in, ent, want, b), end_of(c)
    refs = dict(zip(("dh", "dW", "db"), r.grads(c["dlogp"], c["dent"] if ent else None, relu_in)))
    for k in want:
        ref, tol = refs[k]
        if k == "dh":
            assert bool((q[k][e:] == 77.0).all())
            U.close(q[k][:e], ref[:e], tol[:e], k)
        else:
            U.close(q[k], ref, tol, k)


SHAPES = [  # n, dim, classes, group sizes
    (1, 1, 1, None), (1, 64, 15, None), (2, 5, 2, [1, 1]), (50, 256, 15, None), (64, 64, 64, [64]), (65, 100, 65, [30, 35]),
    (129, 33, 33, [0, 100, 29]), (300, 128, 24, [1] * 100 + [199]), (500, 200, 300, [450]), (1000, 384, 1000, None),
    (257, 72, 4100, [200, 0, 57]), (3, 40, 10007, None), (20000, 64, 15, [7000, 0, 12990]), (40000, 96, 64, [15000, 25000]),
    (2000, 512, 257, [900, 1100]), (700, 600, 40, [300, 390]), (333, 300, 15, [10, 0, 320]), (9000, 512, 64, [4000, 5000]),
    (5000, 256, 24, None), (300, 7, 64, [299, 1]), (100, 1030, 9, None),
]


@pytest.mark.parametrize("relu_in", [False, True])
@pytest.mark.parametrize("n,d,V,sizes", [(20000, 512, 32, [9000, 11000]), (9000, 512, 31, None), (20000, 256, 32, None),
                                         (9000, 256, 33, [4000, 0, 5000]), (9000, 256, 64, None), (700, 511, 17, None)])
def test_narrow_heads_at_the_edges_of_their_blocks(n, d, V, sizes, relu_in):
    c = make(n, d, V, sizes, BF16, seed=V, relu=relu_in)
    o, r = check_forward(c)
    check_backward(c, o, r, relu_in)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("mask", [False, True])
@pytest.mark.parametrize("n,d,V,sizes", SHAPES)
def test_head(n, d, V, sizes, mask, dtype):
    note(f"[head] n={n} d={d} V={V} groups={sizes and len(sizes)} mask={mask} {dtype}")
    c = make(n, d, V, sizes, dtype, seed=n + V, mask=mask, pad=5)
    o, r = check_forward(c)
    check_backward(c, o, r, relu_in=True)
    check_backward(c, o, r, relu_in=False, ent=False)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_pieces(dtype):
    """Rows enough that the classes go in several pieces, the last one short."""
    note(f"[pieces] {dtype}")
    n = 60000 if dtype == BF16 else 50000
    c = make(n, 24, 2600, None, dtype, seed=3, mask=False)
    o, r = check_forward(c)
    check_backward(c, o, r, relu_in=True)


@pytest.mark.parametrize("want", [("dh",), ("dW",), ("db",), ("dh", "db")])
def test_some_outputs(want):
    c = make(600, 70, 130, [300, 290], BF16, seed=4)
    o, r = check_forward(c, b=False)
    check_backward(c, o, r, relu_in=False, want=want, b=False)
    p = run_forward(c, b=False, entropy=False, lse=False)
    assert c["torch"].equal(p["logp"], o["logp"]) and bool((p["lse"] == 77.0).all())


def test_no_rows():
    c = make(0, 20, 30, None, BF16, mask=False)
    o = run_forward(c)
    q = run_backward(c, o, True)
    assert bool((q["dW"] == 0).all()) and bool((q["db"] == 0).all())


@pytest.mark.parametrize("V", [15, 200])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_empty_and_ignored_rows_may_hold_anything(V, dtype):
    """Rows without a valid class, ignored rows and rows behind the last group
    hold not-a-numbers and infinities: nothing of them gets out."""
    note(f"[ignored rows] V={V} {dtype}")
    c = make(400, 48, V, [150, 220], dtype, seed=6)
    torch = c["torch"]
    clean = dict(c, h=c["h"].clone())
    ignored = torch.zeros(400, dtype=torch.bool, device="cuda")
    ignored[::7] = True
    c["target"][ignored] = -1
    c["dent"][ignored] = 0
    c["valid"][3::14] = 0
    c["target"][3::14] = -1
    ignored[3::14] = True
    ignored[370:] = True
    o, r = check_forward(c)
    dirty = dict(c, h=c["h"].clone())
    dirty["h"][ignored] = float("nan")
    dirty["h"][7] = float("inf")
    od = run_forward(dirty)
    keep = ~ignored
    for k in ("logp", "lse", "entropy"):
        assert torch.equal(od[k][keep], o[k][keep]), k
    empty = torch.zeros(400, dtype=torch.bool, device="cuda")
    empty[3::14] = True
    empty[370:] = False
    assert bool((od["logp"][empty] == 0).all()) and bool((od["entropy"][empty] == 0).all())
    assert bool(torch.isneginf(od["lse"][empty]).all())
    a, b = run_backward(c, o, False), run_backward(dirty, od, False)
    inside = keep.clone()
    inside[370:] = False
    assert torch.equal(a["dh"][inside], b["dh"][inside])
    assert bool((b["dh"][:370][ignored[:370]] == 0).all())
    assert torch.equal(a["dW"], b["dW"]) and torch.equal(a["db"], b["db"])
    check_backward(c, o, r, relu_in=False)


@pytest.mark.parametrize("V", [15, 300])
def test_extreme_biases(V):
    """Biases of -infinity, of the lowest float and large ones."""
    note(f"[biases] V={V}")
    c = make(200, 32, V, None, F32, seed=7, mask=False)
    torch = c["torch"]
    c["b"][0, 1::5] = float("-inf")
    c["b"][0, 2::5] = torch.finfo(torch.float32).min
    c["b"][0, 3::5] += 60.0
    c["target"][c["target"] % 5 == 1] = 0
    c["target"][c["target"] % 5 == 2] = 3
    o, r = check_forward(c)
    check_backward(c, o, r, relu_in=False)
    c["b"][:] = float("-inf")
    o = run_forward(c)
    assert bool((o["entropy"] == 0).all()) and bool(torch.isneginf(o["lse"]).all()) and bool((o["logp"] == 0).all())
    q = run_backward(c, o, False)
    assert all(bool((v == 0).all()) for v in q.values())


@pytest.mark.parametrize("V", [20, 150])
def test_targets_out_of_range_or_masked(V):
    """They count as none, and IM_ERR_ACTION is raised."""
    import paper_2606_11440_amd as P
    note(f"[targets] V={V}")
    c = make(300, 32, V, None, BF16, seed=8)
    torch = c["torch"]
    good = dict(c, target=c["target"].clone())
    bad = dict(c, target=c["target"].clone(), error=P._lib.IM_ERR_ACTION)
    bad["target"][5], bad["target"][6], bad["target"][7] = V, -2, 2 ** 31 - 1
    good["target"][5:8] = -1
    bits = U.unpack(c["valid"], 300, V)
    row = int(torch.nonzero(~bits.all(1) & (torch.arange(300) > 10))[0])
    bad["target"][row] = int(torch.nonzero(~bits[row])[0])
    good["target"][row] = -1
    a, b = run_forward(good), run_forward(bad)
    assert a["error"] == 0 and b["error"] == P._lib.IM_ERR_ACTION
    assert all(torch.equal(a[k], b[k]) for k in ("logp", "lse", "entropy"))
    x, y = run_backward(good, a, True), run_backward(bad, b, True)
    assert all(torch.equal(x[k], y[k]) for k in x)


def test_broken_offsets():
    import paper_2606_11440_amd as P
    c = make(100, 40, 150, [30, 70], BF16, seed=10)
    torch = c["torch"]
    c["dev"] = torch.tensor([0, 80, 70], dtype=torch.int32, device="cuda")
    o = run_forward(c)
    assert o["error"] == P._lib.IM_ERR_COUNT and bool((o["logp"] == 77.0).all())
    c["error"] = P._lib.IM_ERR_COUNT
    q = run_backward(c, o, False)
    assert all(bool((v == 77.0).all()) for v in q.values())


def test_gradient_against_differences():
    """The analytic gradient that the kernels follow, against central
    differences of the 64-bit logp and entropy; the kernels' against it."""
    torch = need_gpu()
    c = make(6, 5, 7, [2, 4], F32, seed=12, relu=False)
    o, r = check_forward(c)
    q = run_backward(c, o, False)

    def loss(h, W, b):
        s = U.Head(h, W, b, c["valid"], c["target"], c["off"])
        return float((c["dlogp"].double().cpu() * s.logp + c["dent"].double().cpu() * s.H).sum())
    base = [c["h"].double().cpu(), c["W"].double().cpu(), c["b"].double().cpu()]
    for i, name in enumerate(("dh", "dW", "db")):
        flat = q[name].double().cpu().reshape(-1)
        for j in range(base[i].numel()):
            ends = []
            for s in (1e-5, -1e-5):
                a = [t.clone() for t in base]
                a[i].view(-1)[j] += s
                ends.append(loss(*a))
            num = (ends[0] - ends[1]) / 2e-5
            # differences: third derivatives of order 10 times 1e-10, rounding 1e-15 / 1e-5; the kernel: fp32
            assert abs(float(flat[j]) - num) < 1e-5 * (1 + abs(num)), (name, j)


def test_same_bits_each_time():
    c = make(20000, 100, 300, [12000, 7000], BF16, seed=11)
    a, b = run_forward(c), run_forward(c)
    assert all(c["torch"].equal(a[k], b[k]) for k in ("logp", "lse", "entropy"))
    x, y = run_backward(c, a, True), run_backward(c, a, True)
    assert all(c["torch"].equal(x[k], y[k]) for k in x)


@pytest.mark.parametrize("n,d,V", [(40, 8, 15), (60, 8, 32), (40, 300, 24), (60, 8, 64), (40, 300, 50)])
def test_dz_of_narrow_heads_has_sixteen_bits(n, d, V):
    """Narrow heads' dz enters the products as two bf16 numbers: the first is off by
    2^-8 of dz, and the second by 2^-8 of that. Sums that cancel show it: there the
    results' own rounding hides neither a second number left out nor one subtracted."""
    note(f"[two numbers] n={n} d={d} V={V}")
    c = make(n, d, V, None, BF16, seed=V, mask=False, relu=False, scale=0.05)   # small products: fp32 errors far below 2^-16
    torch = c["torch"]
    o, r = check_forward(c)
    q = run_backward(c, o, False)
    (dh, eh), (dW, eW), _ = r.grads(c["dlogp"], c["dent"], False)
    dz, h, W = r.dz, r.h, r.W[0]
    less = U.ROUND[torch.bfloat16] - 2.0 ** -16
    eh = eh - less * (dz.abs() @ W.abs())
    eW = eW[0] - less * (dz.abs().T @ h.abs())
    U.close(q["dh"], dh, eh, "dh")
    U.close(q["dW"][0], dW[0], eW, "dW")
    first = dz.bfloat16().double()
    for wrong in (first, 2 * first - dz):       # without the second number, and with its sign turned
        assert int(((wrong @ W - dh).abs() > eh).sum()) >= 5
        assert int(((wrong.T @ h - dW[0]).abs() > eW).sum()) >= 5


@pytest.mark.parametrize("V,dtype", [(30, BF16), (30, F32), (300, BF16)])
def test_no_rows_whatever_the_offsets_hold(V, dtype):
    """Without rows offsets are not read: the gradients of every group are zero."""
    c = make(0, 20, V, [0, 0], dtype, mask=False)
    c["dev"] = c["torch"].tensor([0, 5, 3], dtype=c["torch"].int32, device="cuda")
    q = run_backward(c, run_forward(c), True)
    assert bool((q["dW"] == 0).all()) and bool((q["db"] == 0).all())
