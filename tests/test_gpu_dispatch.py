"""GPU: the places of (row, expert) pairs, rows sent to them and the sums that return, against plain
forms (bounds count roundings, experts_util)."""
import pytest

import experts_util as X
from gpu_util import need_gpu, note

pytestmark = pytest.mark.gpu


def experts(torch, n, k, E, seed, drop=0.1):
    g = torch.Generator().manual_seed(seed)
    e = torch.randint(0, E, (n, k), generator=g, dtype=torch.int32)
    e[torch.rand(n, k, generator=g) < drop] = -1
    return e


def make_plan(torch, e, E, workspace=None):
    import paper_2606_11440_amd as P
    offsets = torch.full((E + 1,), 77, dtype=torch.int32, device="cuda")
    slot = torch.full(e.shape, 77, dtype=torch.int32, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    P.im_dispatch_plan(e.cuda(), offsets, slot, workspace=workspace, error=err)
    return offsets, slot, int(err)


@pytest.mark.parametrize("n,k,E", [(1, 1, 1), (1, 32, 1024), (3, 2, 5), (64, 1, 2), (65, 3, 7), (1000, 4, 64), (513, 8, 512),
                                   (2048, 2, 1000), (4097, 1, 3), (5000, 4, 64), (70001, 3, 193), (100000, 4, 257),
                                   (40000, 8, 1024), (9000, 1, 1), (300000, 4, 64), (12345, 5, 511)])
def test_plan(n, k, E):
    note(f"[plan] n={n} k={k} E={E}")
    torch = need_gpu()
    for drop, seed in ((0.0, 1), (0.3, 2)):
        e = experts(torch, n, k, E, seed, drop)
        if drop:   # one expert with most of the pairs, some with none
            e[e > E // 2] = E // 3
        offsets, slot, err = make_plan(torch, e, E)
        want = X.plan(e, E)
        assert err == 0 and bool((offsets.cpu() == want[0]).all()) and bool((slot.cpu() == want[1]).all())


def test_plan_without_pairs_and_with_wrong_ones():
    note("[plan: none, wrong]")
    torch = need_gpu()
    for n in (5, 20000):
        e = torch.full((n, 2), -1, dtype=torch.int32)
        offsets, slot, err = make_plan(torch, e, 9)
        assert err == 0 and bool((offsets == 0).all()) and bool((slot == -1).all())
        e[:, 0] = torch.arange(n) % 9
        e[1, 1], e[3, 1], e[4, 1] = 9, -2, 2 ** 31 - 1
        offsets, slot, err = make_plan(torch, e, 9)
        e[1, 1] = e[3, 1] = e[4, 1] = -1
        want = X.plan(e, 9)
        assert err == 16 and bool((offsets.cpu() == want[0]).all()) and bool((slot.cpu() == want[1]).all())
    offsets, slot, err = make_plan(torch, torch.empty(0, 3, dtype=torch.int32), 4)
    assert err == 0 and offsets.tolist() == [0] * 5


DIMS = [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 31, 64, 86, 193, 256, 387, 512, 520, 1030, 4096, 5001]


def rows(torch, n, d, dtype, seed, pad):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if dtype == "int8":
        t = torch.randint(-127, 128, (n, d + pad), device="cuda", generator=g, dtype=torch.int8)
    else:
        t = torch.randn(n, d + pad, device="cuda", generator=g).to(getattr(torch, dtype))
    return t[:, pad // 2:pad // 2 + d]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "int8"])
@pytest.mark.parametrize("dim", DIMS)
def test_rows_sent(dim, dtype):
    note(f"[sent] dim={dim} {dtype}")
    import paper_2606_11440_amd as P
    torch = need_gpu()
    for n, k, pad in ((1, 1, 0), (77, 3, 3), (130, 5, 8)):
        slot = X.plan(experts(torch, n, k, 6, n), 6)[1]
        x = rows(torch, n, dim, dtype, n, pad)
        wide = torch.full((n * k + 2, dim + pad), 77, dtype=x.dtype, device="cuda")
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        P.im_dispatch_forward(x, slot.cuda(), wide[:, :dim], error=err)
        want = torch.full_like(wide, 77).cpu()
        for i in range(n):
            for c in range(k):
                if slot[i, c] >= 0:
                    want[slot[i, c], :dim] = x[i].cpu()
        assert int(err) == 0 and bool((wide.cpu() == want).all())


def taken(torch, t, slot):
    got = t.cpu().double()[slot.long().clamp_min(0)]
    return torch.where((slot >= 0)[:, :, None], got, torch.zeros((), dtype=torch.float64))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("dim", DIMS)
def test_sums_of_rows(dim, dtype):
    note(f"[sums] dim={dim} {dtype}")
    import paper_2606_11440_amd as P
    torch = need_gpu()
    R = X.ROUND[getattr(torch, dtype)]
    for n, k, pad in ((1, 1, 0), (77, 3, 3), (130, 9, 8)):
        slot = X.plan(experts(torch, n, k, 6, n), 6)[1]
        ys = rows(torch, n * k, dim, dtype, n, pad)
        w = torch.randn(n, k, generator=torch.Generator().manual_seed(n))
        each = taken(torch, ys, slot)
        for weight in (w, None):
            wide = torch.full((n, dim + pad), 77.0, dtype=ys.dtype, device="cuda")
            err = torch.zeros(1, dtype=torch.int32, device="cuda")
            if weight is None:
                P.im_dispatch_backward(ys, slot.cuda(), wide[:, :dim], error=err)
                terms = each
            else:
                P.im_combine_forward(ys, slot.cuda(), w.cuda(), wide[:, :dim], error=err)
                terms = each * w.double()[:, :, None]
            want = terms.sum(1)
            assert int(err) == 0 and bool((wide[:, dim:] == 77.0).all())
            X.same_or_close(wide[:, :dim], want, (k + 1) * X.U * terms.abs().sum(1) + R * want.abs(), (n, k))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("dim", DIMS)
def test_combine_gradient(dim, dtype):
    note(f"[combine gradient] dim={dim} {dtype}")
    import paper_2606_11440_amd as P
    torch = need_gpu()
    R = X.ROUND[getattr(torch, dtype)]
    for n, k, pad in ((1, 1, 0), (77, 3, 3), (130, 9, 8)):
        slot = X.plan(experts(torch, n, k, 6, n), 6)[1]
        ys, dy = rows(torch, n * k, dim, dtype, n, pad), rows(torch, n, dim, dtype, n + 1, pad)
        w = torch.randn(n, k, generator=torch.Generator().manual_seed(n))
        each, D = taken(torch, ys, slot), dy.cpu().double()[:, None, :]
        want_w = (each * D).sum(2)
        tol_w = 2 * (dim + 8) * X.U * (each * D).abs().sum(2)
        want = torch.full((n * k, dim + pad), 77.0, dtype=torch.float64)
        for i in range(n):
            for c in range(k):
                if slot[i, c] >= 0:
                    want[slot[i, c], :dim] = w[i, c].double() * D[i, 0]
        for some in ("both", "dys", "dweight"):
            wide = torch.full((n * k, dim + pad), 77.0, dtype=ys.dtype, device="cuda")
            dw = torch.full((n, k), 77.0, device="cuda")
            err = torch.zeros(1, dtype=torch.int32, device="cuda")
            P.im_combine_backward(dy, ys if some != "dys" else None, slot.cuda(), w.cuda(),
                                  wide[:, :dim] if some != "dweight" else None, dw if some != "dys" else None, error=err)
            assert int(err) == 0
            if some != "dys":
                X.same_or_close(dw, want_w, tol_w, (n, k))
            if some != "dweight":
                X.same_or_close(wide, want, (X.U + R) * want.abs() * (want != 77.0), (n, k))


def test_wrong_slots():
    """Slots that are none are reported, and neither read nor written."""
    note("[wrong slots]")
    import paper_2606_11440_amd as P
    torch = need_gpu()
    x = torch.randn(4, 40, device="cuda")
    slot = torch.tensor([[0, 5], [-2, 1], [6, 2 ** 31 - 1], [-1, -2 ** 31]], dtype=torch.int32, device="cuda")
    xs = torch.full((6, 40), 77.0, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    P.im_dispatch_forward(x, slot, xs, error=err)
    assert int(err) == 16
    assert bool((xs[0] == x[0]).all() and (xs[5] == x[0]).all() and (xs[1] == x[1]).all() and (xs[2:5] == 77.0).all())
    w, y = torch.ones(4, 2, device="cuda"), torch.empty(4, 40, device="cuda")
    err.zero_()
    P.im_combine_forward(xs, slot, w, y, error=err)
    assert int(err) == 16 and bool((y[0] == 2 * x[0]).all() and (y[1] == x[1]).all() and (y[2:] == 0).all())
    err.zero_()
    dw, dys = torch.empty(4, 2, device="cuda"), torch.full((6, 40), 77.0, device="cuda")
    P.im_combine_backward(x, xs, slot, w, dys, dw, error=err)
    assert int(err) == 16 and bool((dw[2:] == 0).all() and dw[1, 0] == 0 and (dys[2:5] == 77.0).all())
    # no slots at all
    err.zero_()
    none = torch.empty(0, 40, device="cuda")
    P.im_dispatch_backward(none, torch.full_like(slot, -1), y, error=err)
    assert int(err) == 0 and bool((y == 0).all())


def test_rows_that_hold_no_numbers():
    """What no slot names is not read: NaN there reaches nothing; infinities go where they are sent."""
    note("[NaN elsewhere]")
    import paper_2606_11440_amd as P
    torch = need_gpu()
    for dim in (3, 70):
        ys = torch.full((6, dim), float("nan"), device="cuda")
        ys[2] = 1.0
        ys[3] = float("inf")
        slot = torch.tensor([[2, -1], [3, 2], [-1, -1]], dtype=torch.int32, device="cuda")
        w, y = torch.full((3, 2), 0.5, device="cuda"), torch.empty(3, dim, device="cuda")
        P.im_combine_forward(ys, slot, w, y)
        assert bool((y[0] == 0.5).all() and torch.isinf(y[1]).all() and (y[2] == 0).all())
        dw, dys = torch.empty(3, 2, device="cuda"), torch.zeros(6, dim, device="cuda")
        P.im_combine_backward(torch.ones(3, dim, device="cuda"), ys, slot, w, dys, dw)
        assert dw.tolist() == [[dim, 0], [float("inf"), dim], [0, 0]]


def test_slots_far_apart():
    """Offsets past 32 bits: 70,000 slots 65,536 elements apart."""
    note("[far slots]")
    import paper_2606_11440_amd as P
    torch = need_gpu()
    n, d = 35000, 48
    wide = torch.empty(2 * n, 65536, dtype=torch.bfloat16, device="cuda")
    slot = torch.randperm(2 * n, device="cuda").to(torch.int32).reshape(n, 2)
    x = torch.randn(n, d, device="cuda").bfloat16()
    P.im_dispatch_forward(x, slot, wide[:, :d])
    assert bool((wide[slot.long(), :d] == x[:, None]).all())
    w, y = torch.full((n, 2), 0.5, device="cuda"), torch.empty_like(x)
    P.im_combine_forward(wide[:, :d], slot, w, y)
    assert bool((y == x).all())
    dw = torch.empty_like(w)
    P.im_combine_backward(x, wide[:, :d], slot, w, wide[:, 1000:1000 + d], dw)
    assert bool((wide[slot.long(), 1000:1000 + d] == (x.float() * 0.5).bfloat16()[:, None]).all())
    assert bool((dw[:, 0] == dw[:, 1]).all())
