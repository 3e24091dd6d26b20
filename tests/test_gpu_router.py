"""GPU: routing to experts and its gradient against 64 bits (bounds: experts_util)."""
import numpy as np
import pytest

import experts_util as X
from gpu_util import need_gpu, note

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


def make(n, E, dtype, seed, mask=False, spread=1.5, pad=0):
    torch = need_gpu()
    g = torch.Generator().manual_seed(seed)
    wide = (torch.randn(n, E + pad, generator=g) * spread).to(getattr(torch, dtype)).cuda()
    z = wide[:, pad // 2:pad // 2 + E]
    ok = None
    if mask:
        ok = (torch.rand(n, E, generator=g) < 0.7).numpy()
        ok[torch.rand(n, generator=g).numpy() < 0.1] = False
    return torch, g, z, ok


def check(torch, z, ok, k, score, renorm, bias=None, sets=1, top_sets=1, best=1, scale=1.0, seed=0, pad=0):
    import paper_2606_11440_amd as P
    n, E = z.shape
    ref = X.Router(z.cpu(), score, ok)
    valid = None if ok is None else X.words(ok).cuda()
    expert = torch.full((n, k), 77, dtype=torch.int32, device="cuda")
    weight = torch.full((n, k), 77.0, device="cuda")
    P.im_router_forward(z, expert, weight, bias=None if bias is None else bias.cuda(), valid=valid, score=score,
                        renorm=renorm, scale=scale, n_sets=sets, top_sets=top_sets, set_best=best)
    want = ref.choose(k, bias, sets, top_sets, best)
    got = expert.cpu().numpy()
    assert (got == want).all(), (np.argwhere(got != want)[:4].tolist(), got[got != want][:4], want[got != want][:4])
    w, tol = ref.weights(want, renorm, scale)
    X.same_or_close(weight, w, tol, "weight")
    g = torch.Generator().manual_seed(seed + 1)
    dw = torch.randn(n, k, generator=g)
    full = torch.full((n, E + pad), 77.0, dtype=z.dtype, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    P.im_router_backward(z, expert, dw.cuda(), full[:, :E], valid=valid, score=score, renorm=renorm, scale=scale, error=err)
    assert int(err) == 0
    dz, tol = ref.grad(want, dw, renorm, scale)
    X.same_or_close(full[:, :E], dz, tol, "dz")
    assert bool((full[:, E:] == 77.0).all())
    return expert, weight


SIZES = [(1, 1, 1), (1, 8, 2), (2, 2, 2), (3, 3, 1), (5, 15, 4), (64, 8, 8), (65, 33, 6), (63, 64, 8), (100, 65, 3),
         (129, 100, 10), (40, 128, 32), (33, 193, 6), (50, 256, 8), (31, 257, 9), (20, 512, 16), (9, 1000, 32),
         (7, 1024, 5), (3000, 64, 4), (2000, 24, 3)]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,E,k", SIZES)
def test_router(n, E, k, dtype, score):
    note(f"[router] n={n} E={E} k={k} {dtype} {score}")
    for i, (renorm, bias, mask) in enumerate([(True, False, False), (False, True, True), (True, True, True),
                                              (False, False, True)]):
        torch, g, z, ok = make(n, E, dtype, seed=n + E + i, mask=mask)
        b = torch.randn(E, generator=g) * 0.1 if bias else None
        check(torch, z, ok, k, score, renorm, b, scale=1.0 if i % 2 else 2.5, seed=i)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,sets,top_sets,k", [(8, 2, 1, 2), (64, 8, 4, 4), (64, 64, 5, 5), (96, 3, 2, 8), (100, 10, 1, 7),
                                               (256, 8, 3, 8), (256, 2, 2, 8), (512, 16, 4, 10), (1024, 512, 300, 32),
                                               (65, 13, 6, 12)])
def test_sets(E, sets, top_sets, k, score):
    note(f"[sets] E={E} sets={sets} of {top_sets} k={k} {score}")
    for i, (best, bias, mask) in enumerate([(1, False, False), (2, False, True), (1, True, True), (2, True, True),
                                            (2, True, False)]):
        for dtype in ("float32", "bfloat16"):
            torch, g, z, ok = make(130, E, dtype, seed=E + i, mask=mask)
            b = torch.randn(E, generator=g) * 0.1 if bias else None
            check(torch, z, ok, k, score, True, b, sets, top_sets, best)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_equal_scores_go_to_the_lowest_index(score):
    note(f"[equal scores] {score}")
    torch = need_gpu()
    for E, k in ((8, 3), (64, 8), (200, 20), (1024, 32)):
        z = torch.zeros(20, E, device="cuda")
        z[5:10] = torch.randint(0, 3, (5, E)).float().cuda()   # few values
        z[10:15, E // 2:] = 1.0
        check(torch, z, None, k, score, True)
        check(torch, z, None, k, score, True, torch.zeros(E))
        check(torch, z.bfloat16(), None, k, score, False, torch.arange(E).remainder(3).float() * 0.25)
        check(torch, z, None, min(k, E // 4), score, True, torch.zeros(E), 4, 1, 2)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_scores_that_fp32_cannot_tell_apart(score):
    """Biases that bring every c to within some 1e-8 of one another."""
    note(f"[near ties] {score}")
    torch = need_gpu()
    E, n = 64, 300
    z = torch.randn(1, E, generator=torch.Generator().manual_seed(3)).expand(n, E).contiguous()
    ref = X.Router(z, score)
    b = torch.from_numpy((0.7 - ref.s[0]).astype(np.float32))
    check(torch, z.cuda(), None, 8, score, True, b)
    check(torch, z.cuda(), None, 8, score, True, b, 8, 2, 2)
    check(torch, z.cuda(), None, 8, score, True, b, 8, 3, 1)
    # scores near 1, and near 0
    for shift in (14.0, 30.0, 60.0, -20.0, -60.0):
        check(torch, (z + shift).cuda(), None, 6, score, True, torch.randn(E) * 1e-7)
        check(torch, (z + shift).cuda(), None, 6, score, True, None, 8, 4, 2)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_values_at_the_ends(score, dtype):
    note(f"[ends] {score} {dtype}")
    torch, g, z, _ = make(40, 48, dtype, seed=11)
    z = z.clone()
    ok = np.ones((40, 48), bool)
    z[0] = -INF                       # nothing to choose
    z[1, 3:] = -INF                   # three to choose
    z[2, ::2] = NAN
    ok[3] = False                     # masked whole, whatever it holds
    z[3] = NAN
    z[4, :10], ok[4, :10] = INF, False
    z[5, 7] = INF
    z[6, :20] = INF
    z[7] = -3e38
    z[8] = 3e38
    z[9] = torch.linspace(-3e38, 3e38, 48)
    z[10] = torch.linspace(-120, -100, 48)    # sigmoids below the smallest float
    z[11] = torch.linspace(-800, -740, 48)    # and below the smallest double
    z[12] = torch.linspace(30, 200, 48)
    z[13] = 1e-40
    ok[14, 1:] = False                # one to choose
    z[15, 0] = 1e4
    for renorm in (True, False):
        check(torch, z, ok, 5, score, renorm)
        check(torch, z, ok, 5, score, renorm, torch.randn(48, generator=g) * 0.1, 8, 4, 2)
        check(torch, z, ok, 5, score, renorm, None, 6, 2, 2)
        check(torch, z, ok, 5, score, renorm, None, 6, 2, 1)
    b = torch.randn(48, generator=g) * 0.1
    b[3], b[4], b[5], b[6] = -INF, NAN, INF, -1e30    # shut off, shut off, first, last
    check(torch, z, ok, 5, score, True, b)
    check(torch, z, ok, 5, score, False, b, 6, 3, 2)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_strides(dtype):
    note(f"[router strides] {dtype}")
    for pad in (1, 3, 8):
        for E in (7, 64, 130):
            torch, g, z, ok = make(77, E, dtype, seed=pad, mask=True, pad=pad)
            check(torch, z, ok, 4, "softmax", False, None, pad=pad)
            check(torch, z, ok, 4, "sigmoid", True, torch.randn(E, generator=g) * 0.1, pad=pad)


def test_rows_far_apart():
    """Element offsets past 32 bits: 70,000 rows of 40 logits, 65,536 apart."""
    note("[router far rows]")
    import paper_2606_11440_amd as P
    torch = need_gpu()
    n, E = 70000, 40
    wide = torch.empty(n, 65536, dtype=torch.bfloat16, device="cuda")
    z = wide[:, :E]
    z.copy_(torch.randn(n, E, device="cuda"))
    near = z.contiguous()
    out = []
    for t in (z, near):
        e, w = torch.empty(n, 4, dtype=torch.int32, device="cuda"), torch.empty(n, 4, device="cuda")
        P.im_router_forward(t, e, w, score="softmax", renorm=False)
        dz = torch.empty_like(near) if t is near else wide[:, 1000:1000 + E]
        P.im_router_backward(t, e, w, dz, renorm=False)
        out.append((e, w, dz))
    assert all(bool((a == b).all()) for a, b in zip(*out))


def test_experts_of_ones_own():
    """The gradient for any list of experts: twice the same, none, out of range, not valid."""
    note("[router lists]")
    import paper_2606_11440_amd as P
    torch, g, z, _ = make(6, 20, "float32", seed=4)
    ok = np.ones((6, 20), bool)
    ok[3, 5] = False
    e = torch.tensor([[1, 1, 1, 4], [0, -1, 0, -1], [-1, -1, -1, -1], [5, 6, 7, 5], [20, 3, -2, 4], [2 ** 31 - 1, -2 ** 31, 0, 1]],
                     dtype=torch.int32)
    dw = torch.randn(6, 4, generator=g)
    clean = e.clone()
    clean[(clean < 0) | (clean > 19)] = -1
    clean[3, 0] = clean[3, 3] = -1
    for score in ("softmax", "sigmoid"):
        for renorm in (True, False):
            ref = X.Router(z.cpu(), score, ok)
            dz = torch.empty_like(z)
            err = torch.zeros(1, dtype=torch.int32, device="cuda")
            P.im_router_backward(z, e.cuda(), dw.cuda(), dz, valid=X.words(ok).cuda(), score=score, renorm=renorm, error=err)
            assert int(err) == 16
            want, tol = ref.grad(clean.numpy(), dw, renorm)
            X.same_or_close(dz, want, tol, (score, renorm))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_gradient_against_differences(score, renorm):
    """The gradient is that of the weights: central differences of the forward call's own outputs in
    64 bits (the reference's weights, whose choice does not change)."""
    note(f"[router differences] {score} {renorm}")
    import paper_2606_11440_amd as P
    torch, g, z, _ = make(8, 12, "float32", seed=9)
    e, w = torch.empty(8, 3, dtype=torch.int32, device="cuda"), torch.empty(8, 3, device="cuda")
    P.im_router_forward(z, e, w, score=score, renorm=renorm, scale=1.5)
    dw = torch.randn(8, 3, generator=g)
    dz = torch.empty_like(z)
    P.im_router_backward(z, e, dw.cuda(), dz, score=score, renorm=renorm, scale=1.5)
    base, at, h = z.cpu().double(), e.cpu().numpy(), 1e-4
    for j in range(12):
        up, down = base.clone(), base.clone()
        up[:, j] += h
        down[:, j] -= h
        slope = [(X.Router(t, score).weights(at, renorm, 1.5)[0] * dw.double()).sum(1) for t in (up, down)]
        X.same_or_close(dz[:, j], (slope[0] - slope[1]) / (2 * h), torch.full((8,), 1e-5), j)   # h^2 and fp32
