"""GPU: rows in 8 bits, the layer that multiplies them and the gradients of a layer whose input was
kept so (bounds: experts_util, learn_util)."""
import pytest

import experts_util as X
import learn_util as U
from gpu_util import need_gpu, note

pytestmark = pytest.mark.gpu
F32, BF16 = "float32", "bfloat16"
DIMS = [1, 2, 3, 4, 5, 8, 9, 15, 17, 33, 64, 86, 130, 193, 256, 387, 512, 513, 1000, 1030, 2048, 2500, 4096, 4100, 8200, 65536]


def packed(x, keep=False, pad=0):
    import paper_2606_11440_amd as P
    import torch
    n, d = x.shape
    wide = torch.full((n, d + pad), 77, dtype=torch.int8, device="cuda")
    scale = torch.full((n,), 77.0, device="cuda")
    P.im_rows_pack(x, wide[:, :d], scale, keep=keep)
    assert bool((wide[:, d:] == 77).all())
    return wide[:, :d], scale


def same(a, b):
    a, b = a.cpu(), b.cpu()
    return bool(((a == b) | ((a != a) & (b != b))).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", DIMS)
def test_pack(dim, dtype):
    note(f"[pack] dim={dim} {dtype}")
    import paper_2606_11440_amd as P
    torch = need_gpu()
    g = torch.Generator().manual_seed(dim)
    for n, pad, keep in ((1, 0, False), (37, 3, True), (70, 8, False)):
        x = (torch.randn(n, dim + pad, generator=g) * torch.exp(4 * torch.randn(n, 1, generator=g))).to(getattr(torch, dtype))
        x = x.cuda()[:, pad // 2:pad // 2 + dim]
        if n > 30:
            x[3], x[4] = 0, torch.relu(x[4])
            x[5, 0], x[6, dim - 1], x[7, dim // 2] = float("nan"), float("inf"), -float("inf")
            x[8], x[9] = 3.3e38, x[9] * 1e-30
            x[10] = torch.randn(dim, generator=g) * 2e-38
            x[11, 0] = 1e30      # the rest rounds to 0
            x[12] = 1e-40
        q, s = packed(x, keep, pad)
        want_q, want_s = X.pack(x, keep)
        assert same(s, want_s) and same(q, want_q)
        back = torch.full((n, dim + pad), 77.0, dtype=x.dtype, device="cuda")
        P.im_rows_unpack(q, s, back[:, :dim])
        want = (want_s[:, None] * want_q.float()).to(x.dtype)
        assert same(back[:, :dim], want) and bool((back[:, dim:] == 77.0).all())


def test_pack_rows_far_apart():
    """Offsets past 32 bits: 70,000 rows, 65,536 elements apart."""
    note("[pack far rows]")
    import paper_2606_11440_amd as P
    torch = need_gpu()
    n, d = 70000, 40
    wide, codes = (torch.empty(n, 65536, dtype=t, device="cuda") for t in (torch.bfloat16, torch.int8))
    x = torch.randn(n, d, device="cuda").bfloat16()
    wide[:, :d] = x
    s, s2, q = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, d, dtype=torch.int8, device="cuda")
    P.im_rows_pack(x, q, s)
    P.im_rows_pack(wide[:, :d], codes[:, :d], s2)
    assert same(s, s2) and same(q, codes[:, :d])
    a, b = torch.empty_like(x), wide[:, 1000:1000 + d]
    P.im_rows_unpack(q, s, a)
    P.im_rows_unpack(codes[:, :d], s, b)
    assert same(a, b)


def make(n, k, m, sizes, dtype, seed, pad=0, relu=False):
    torch = need_gpu()
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, G = getattr(torch, dtype), len(sizes) if sizes else 1

    def normal(*s, scale=1.0, t=dt):
        return (torch.randn(*s, device="cuda", generator=g) * scale).to(t)
    x = normal(n, k)
    if relu:
        x.relu_()
    q, s = packed(x, relu, pad)
    W = normal(G, m, k, scale=k ** -0.5)
    Wq, Ws = packed(W.reshape(G * m, k))
    off = None
    if sizes:
        off = [0]
        for size in sizes:
            off.append(off[-1] + size)
    dev = None if off is None else torch.tensor(off, dtype=torch.int32, device="cuda")
    return dict(torch=torch, q=q, s=s, W=W, Wq=Wq.reshape(G, m, k), Ws=Ws.reshape(G, m), b=normal(G, m, t=torch.float32),
                dy=normal(n, m + pad)[:, :m], off=off, dev=dev, G=G, dt=dt)


def check_forward(c, relu, b=True, pad=0):
    import paper_2606_11440_amd as P
    torch, n, m = c["torch"], c["q"].shape[0], c["W"].shape[1]
    y = torch.full((n, m + pad), 77.0, dtype=c["dt"], device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    P.im_linear_forward_packed(c["q"], c["s"], c["Wq"], c["Ws"], c["b"] if b else None, y[:, :m], offsets=c["dev"],
                               relu=relu, error=err)
    assert int(err) == 0
    want, tol = X.packed_linear(c["q"], c["s"], c["Wq"], c["Ws"], c["b"] if b else None, c["off"], relu, c["dt"])
    end = c["off"][-1] if c["off"] else n
    X.same_or_close(y[:end, :m], want[:end], tol[:end], "y")
    assert bool((y[end:] == 77.0).all() and (y[:, m:] == 77.0).all())


def check_backward(c, relu_in, some=("dx", "dW", "db"), pad=0):
    import paper_2606_11440_amd as P
    torch, (n, k), (G, m, _) = c["torch"], c["q"].shape, c["W"].shape
    o = dict(dx=torch.full((n, k + pad), 77.0, dtype=c["dt"], device="cuda")[:, :k],
             dW=torch.full((G, m, k), 77.0, dtype=c["dt"], device="cuda"), db=torch.full((G, m), 77.0, device="cuda"))
    o = {key: v if key in some else None for key, v in o.items()}
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    P.im_linear_backward_packed(c["dy"], c["q"], c["s"], c["W"], o["dx"], o["dW"], o["db"], offsets=c["dev"],
                                relu_in=relu_in, error=err)
    assert int(err) == 0
    x = c["q"].double() * c["s"].double()[:, None]
    refs = dict(zip(("dx", "dW", "db"), U.linear_grad(c["dy"], x.float(), c["W"], c["off"], relu_in)))
    end = c["off"][-1] if c["off"] else n
    off = c["off"] or [0, n]
    for key in some:
        ref, tol = refs[key]
        R = X.ROUND[c["dt"]]
        tol = tol + R * ref.abs()
        if key == "dx":
            assert bool((o["dx"][end:] == 77.0).all())
            ref, tol = ref[:end], tol[:end]
            X.same_or_close(o["dx"][:end], ref, tol, key)
        elif key == "dW":   # scale times code is rounded to the products' type
            size = torch.stack([c["dy"][a:b].double().abs().T @ x[a:b].abs() for a, b in zip(off, off[1:])])
            X.same_or_close(o[key], ref, tol + (R + X.U) * size, key)
        else:
            X.same_or_close(o[key], ref, tol, key)


SHAPES = [  # n, in, out, group sizes (None: no offsets)
    (1, 1, 1, None), (1, 86, 256, None), (3, 7, 5, None), (48, 86, 256, None), (64, 64, 64, [64]), (65, 33, 65, [65]),
    (130, 193, 129, [0, 130]), (200, 8, 8, [50, 0, 0, 149, 1]), (257, 256, 15, [100, 157]), (300, 104, 24, [7] * 40),
    (513, 384, 128, [511]), (700, 72, 200, [0, 0, 0]), (1000, 513, 255, [1, 2, 997]),
    (4096, 193, 512, [1000, 0, 3000, 50, 13]), (70000, 64, 48, [30000, 39000]), (900, 40, 24, [3] * 299 + [1]),
    (40000, 520, 520, [39000, 1000]), (20000, 130, 300, None), (5000, 15, 17, [4000, 900]),
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,k,m,sizes", SHAPES)
def test_layer(n, k, m, sizes, dtype):
    note(f"[packed layer] n={n} k={k} m={m} groups={sizes and len(sizes)} {dtype}")
    c = make(n, k, m, sizes, dtype, seed=n + k)
    check_forward(c, relu=True)
    check_forward(c, relu=False, b=False)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,k,m,sizes", SHAPES)
def test_layer_gradient(n, k, m, sizes, dtype):
    note(f"[packed layer gradient] n={n} k={k} m={m} groups={sizes and len(sizes)} {dtype}")
    check_backward(make(n, k, m, sizes, dtype, seed=n + m), relu_in=False)
    check_backward(make(n, k, m, sizes, dtype, seed=n + m + 1, relu=True), relu_in=True)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pad", [1, 2, 3, 8, 10])
def test_strides(dtype, pad):
    note(f"[packed strides] pad={pad} {dtype}")
    for n, k, m, sizes in ((77, 45, 33, [70]), (600, 200, 130, [300, 299]), (300, 256, 256, None)):
        c = make(n, k, m, sizes, dtype, seed=pad, pad=pad, relu=True)
        check_forward(c, relu=True, pad=pad)
        check_backward(c, relu_in=True, pad=pad)


# large tiles of rows that are whole units of 16 bytes: from one stage of 64 bytes to many, ends inside one
LARGE = [(30000, 16, 777, None), (5000, 48, 5000, None), (70000, 64, 512, [33000, 36990]), (20000, 272, 1030, [7000, 0, 12999]),
         (40000, 528, 520, [1, 39999]), (9000, 1040, 2056, [100, 8000, 3, 800]), (30000, 320, 640, [300] * 100),
         (4096, 4096, 2048, None), (8192, 4096, 4096, None), (9000, 4112, 2050, [100, 8000, 899]), (5000, 4224, 4096, [0, 5000])]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,k,m,sizes", LARGE)
def test_large_tiles(n, k, m, sizes, dtype):
    note(f"[packed large] n={n} k={k} m={m} groups={sizes and len(sizes)} {dtype}")
    c = make(n, k, m, sizes, dtype, seed=k)
    check_forward(c, relu=True)
    check_forward(c, relu=False, b=False, pad=3)
    wide = make(n, k, m, sizes, dtype, seed=k, pad=32)   # rows of 16-byte units within wider ones
    wide["q"] = c["q"].new_empty(n, k + 32)[:, :k].copy_(c["q"])
    wide["s"] = c["s"]
    check_forward(wide, relu=True)


def test_large_tiles_and_rows_that_are_not_finite():
    """In large tiles too a row's NaN scale is its own, and one behind the last group reaches nothing."""
    note("[packed large: NaN]")
    import paper_2606_11440_amd as P
    c = make(70000, 64, 512, [33000, 36990], BF16, seed=3)
    torch = c["torch"]
    bad = torch.tensor([0, 255, 256, 33000, 69989], device="cuda")
    c["s"][bad] = float("nan")
    c["s"][69990:] = float("nan")
    y = torch.full((70000, 512), 77.0, dtype=torch.bfloat16, device="cuda")
    P.im_linear_forward_packed(c["q"], c["s"], c["Wq"], c["Ws"], c["b"], y, offsets=c["dev"], relu=True)
    rows = torch.isnan(y).all(1)
    assert int(rows.sum()) == 5 and bool(rows[bad].all()) and int(torch.isnan(y).sum()) == 5 * 512
    assert bool((y[69990:] == 77.0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_many_groups(dtype):
    """1024 groups, most of them empty or of some rows, one of most rows."""
    note(f"[packed groups] {dtype}")
    sizes = [(7 * g) % 5 if g % 3 else 0 for g in range(1024)]
    sizes[500] = 9000
    c = make(sum(sizes) + 11, 80, 48, sizes, dtype, seed=6, relu=True)
    check_forward(c, relu=True)
    check_backward(c, relu_in=True)


@pytest.mark.parametrize("some", [("dx",), ("dW",), ("db",), ("dW", "db")])
def test_some_gradients(some):
    note(f"[packed: some gradients] {some}")
    check_backward(make(500, 100, 70, [400, 90], BF16, seed=5), relu_in=False, some=some)
    check_backward(make(500, 100, 70, None, F32, seed=6, relu=True), relu_in=True, some=some)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,k,m,sizes", [(1, 4096, 200, None), (20, 5001, 130, [5, 0, 15]), (150, 8200, 70, [100]),
                                         (33, 20000, 20, None), (16, 65536, 48, None)])
def test_few_rows_and_a_long_sum(n, k, m, sizes, dtype):
    """The sum is cut into runs that a second kernel joins."""
    note(f"[packed long sum] n={n} k={k} m={m} {dtype}")
    c = make(n, k, m, sizes, dtype, seed=k)
    check_forward(c, relu=True)
    check_forward(c, relu=False, b=False)
    check_backward(make(n, m, k, sizes, dtype, seed=k, relu=True), relu_in=True)


def test_largest_sum():
    """All codes 127 over the longest row: 127^2 65536, exact in the sum, rounded once on its way out."""
    note("[packed largest sum]")
    import paper_2606_11440_amd as P
    torch = need_gpu()
    for n, m in ((3, 5), (300, 260)):
        q = torch.full((n, 65536), 127, dtype=torch.int8, device="cuda")
        W = torch.full((m, 65536), -127, dtype=torch.int8, device="cuda")
        W[0] = 127
        y = torch.empty(n, m, device="cuda")
        P.im_linear_forward_packed(q, torch.ones(n, device="cuda"), W, torch.ones(m, device="cuda"), None, y)
        big = float(torch.tensor(127.0 ** 2 * 65536, dtype=torch.float64).float())
        assert bool((y[:, 0] == big).all() and (y[:, 1:] == -big).all())


def test_rows_that_are_not_finite():
    """A row's NaN scale makes its y NaN (ReLU or not) and dW; other rows and dx do not see it."""
    note("[packed NaN]")
    import paper_2606_11440_amd as P
    torch = need_gpu()
    for dtype in (F32, BF16):
        c = make(100, 40, 30, None, dtype, seed=2, relu=True)
        c["s"][7] = float("nan")
        c["q"][7] = 0
        y = torch.empty(100, 30, dtype=c["dt"], device="cuda")
        P.im_linear_forward_packed(c["q"], c["s"], c["Wq"], c["Ws"], c["b"], y, relu=True)
        bad = torch.isnan(y).cpu()
        assert bool(bad[7].all()) and int(bad.sum()) == 30
        dx, dW = torch.empty(100, 40, dtype=c["dt"], device="cuda"), torch.empty_like(c["W"])
        P.im_linear_backward_packed(c["dy"], c["q"], c["s"], c["W"], dx, dW, relu_in=True)
        assert bool(torch.isfinite(dx).all() and (dx[7] == 0).all() and torch.isnan(dW).all())


def test_rows_behind_the_last_group_hold_nothing():
    """NaN scales and values behind the last group reach no output."""
    note("[packed rows behind]")
    for dtype in (F32, BF16):
        c = make(300, 70, 50, [100, 130], dtype, seed=8, relu=True)
        c["s"][230:] = float("nan")
        c["dy"][230:] = float("nan")
        check_forward(c, relu=False)
        check_backward(c, relu_in=True)


def test_broken_groups():
    note("[packed broken groups]")
    import paper_2606_11440_amd as P
    torch = need_gpu()
    c = make(50, 20, 30, [20, 30], F32, seed=1)
    for off in ([0, 60, 50], [1, 20, 50], [0, 30, 20], [0, 20, 51], [0, -1, 50]):
        off = torch.tensor(off, dtype=torch.int32, device="cuda")
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        y = torch.full((50, 30), 77.0, device="cuda")
        P.im_linear_forward_packed(c["q"], c["s"], c["Wq"], c["Ws"], None, y, offsets=off, error=err)
        assert int(err) == 2 and bool((y == 77.0).all())
        err.zero_()
        dx, dW = torch.full((50, 20), 77.0, device="cuda"), torch.full((2, 30, 20), 77.0, device="cuda")
        P.im_linear_backward_packed(c["dy"], c["q"], c["s"], c["W"], dx, dW, offsets=off, error=err)
        assert int(err) == 2 and bool((dx == 77.0).all() and (dW == 77.0).all())


def test_no_rows():
    note("[packed no rows]")
    import paper_2606_11440_amd as P
    torch = need_gpu()
    q, s = torch.empty(0, 16, dtype=torch.int8, device="cuda"), torch.empty(0, device="cuda")
    W = torch.randn(2, 8, 16, device="cuda")
    Wq, Ws = packed(W.reshape(16, 16))
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    y = torch.empty(0, 8, device="cuda")
    P.im_linear_forward_packed(q, s, Wq.reshape(2, 8, 16), Ws, None, y, offsets=off)
    dW, db = torch.full_like(W, 77.0), torch.full((2, 8), 77.0, device="cuda")
    P.im_linear_backward_packed(y, q, s, W, None, dW, db, offsets=off)
    assert bool((dW == 0).all() and (db == 0).all())
    P.im_rows_pack(torch.empty(0, 16, device="cuda"), q, s)
    P.im_rows_unpack(q, s, torch.empty(0, 16, device="cuda"))
