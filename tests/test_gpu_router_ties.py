"""GPU: routing where values that decide something are equal, or as good as equal, and where they are not
finite; against 64 bits (bounds: experts_util)."""
import numpy as np
import pytest

import experts_util as X
from gpu_util import need_gpu, note
from test_gpu_router import check

pytestmark = pytest.mark.gpu
INF = float("inf")
SCORES = ["softmax", "sigmoid"]


def sets_of_equal_sum(E, sets, seed):
    """Biases whose two best of a set are some M + d and M - d, of few M and many d (multiples of 2^-6: all
    sums are exact), and whose others are far below."""
    r = np.random.default_rng(seed)
    each = E // sets
    b = -0.5 - r.integers(1, 33, (sets, each)) / 64
    for s in range(sets):
        i, j = r.permutation(each)[:2]
        m, d = r.integers(0, 2) / 32, r.integers(1, 17) / 64
        b[s, i], b[s, j] = m + d, m - d
    return b.reshape(E).astype(np.float32)


@pytest.mark.parametrize("score", SCORES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("E,sets", [(8, 2), (16, 4), (32, 4), (64, 16), (64, 8), (64, 4), (128, 4), (256, 8), (256, 64),
                                    (12, 4), (96, 8), (512, 16), (1024, 128)])
def test_sets_of_equal_sum(E, sets, dtype, score):
    """Sets of 2, 4, 8, .. experts worth the same whose members lie apart: of equal ones the lowest sets count."""
    note(f"[sets of equal sum] E={E} sets={sets} {dtype} {score}")
    torch = need_gpu()
    z = torch.zeros(70, E, dtype=getattr(torch, dtype), device="cuda")    # scores are 1 / 2, or 1 / E
    for seed in range(6):
        b = torch.from_numpy(sets_of_equal_sum(E, sets, seed))
        for top_sets in {1, 2, max(1, sets // 2), sets - 1}:
            k = min(E // sets * top_sets, 2 + 2 * (seed % 3), 32)
            check(torch, z, None, k, score, True, b, sets, top_sets, 2)


def test_two_sets_of_equal_sum():
    """Both sets are worth 1; their best experts lie in both."""
    note("[two sets of equal sum]")
    import paper_2606_11440_amd as P
    torch = need_gpu()
    z = torch.zeros(5, 8, device="cuda")
    b = torch.tensor([.25, -.25, -.4, -.4, .125, -.125, -.4, -.4], device="cuda")
    e, w = torch.empty(5, 2, dtype=torch.int32, device="cuda"), torch.empty(5, 2, device="cuda")
    P.im_router_forward(z, e, w, bias=b, score="sigmoid", n_sets=2, top_sets=1, set_best=2)
    assert e.tolist() == [[0, 1]] * 5


@pytest.mark.parametrize("E,sets,top_sets", [(16, 4, 1), (64, 8, 3), (64, 4, 2), (256, 16, 5)])
def test_sets_whose_sums_fp32_cannot_tell_apart(E, sets, top_sets):
    """Sums of two sigmoids some 1e-9 to 1e-7 apart, of members far apart: 3000 rows of their own."""
    note(f"[sets of near sums] E={E} sets={sets} of {top_sets}")
    torch = need_gpu()
    g = torch.Generator().manual_seed(E + sets)
    n, each = 3000, E // sets
    s = torch.rand(n, sets, generator=g, dtype=torch.float64) * 0.3 + 0.05
    z = torch.full((n, sets, each), -4.0, dtype=torch.float64) - torch.rand(n, sets, each, generator=g, dtype=torch.float64)
    z[:, :, 1] = torch.logit(s)
    z[:, :, 3] = torch.logit(0.9 - s)
    check(torch, z.reshape(n, E).float().cuda(), None, min(4, 2 * top_sets), "sigmoid", True, None, sets, top_sets, 2)


@pytest.mark.parametrize("score", SCORES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("E,sets,top_sets", [(8, 1, 1), (8, 2, 1), (24, 1, 1), (64, 1, 1), (64, 8, 3), (100, 10, 2),
                                             (200, 1, 1), (1024, 1, 1)])
def test_biases_of_infinity(E, sets, top_sets, dtype, score):
    """Two of them, and more than can be chosen: equal c, the lowest index first."""
    note(f"[infinite biases] E={E} sets={sets} {dtype} {score}")
    torch = need_gpu()
    g = torch.Generator().manual_seed(E)
    z = torch.randn(90, E, generator=g).to(getattr(torch, dtype)).cuda()
    for where in ([1, 4], [E - 1, 0], [0, 1, 2, 3], list(range(E // 2, E)), list(range(E))):
        for k in (1, 2, 4):
            for best in (1, 2):
                b = torch.randn(E, generator=g) * 0.1
                b[where] = INF
                check(torch, z, None, k, score, True, b, sets, top_sets, best)
    ok = (torch.rand(90, E, generator=g) < 0.6).numpy()
    b[:] = torch.where(torch.rand(E, generator=g) < 0.5, INF, -INF)
    check(torch, z, ok, 2, score, False, b, sets, top_sets, 2)


@pytest.mark.parametrize("score", SCORES)
@pytest.mark.parametrize("E", [16, 32, 64, 256, 1024])
def test_scores_next_to_large_biases(E, score):
    """Two experts whose c, a bias of 64 or so + a score of 1 / 2 or 1 / 4, lie some 1e-8 apart where fp32 rounds (half
    its unit of 2^-17 under a multiple of 16): what it makes of them is a unit apart, either way."""
    note(f"[large biases] E={E} {score}")
    torch = need_gpu()
    n, r = 20000 if E <= 64 else 3000, np.random.default_rng(E)
    unit, apart = 2.0 ** -17, 30000                  # of the biases, in units
    V = 4 if E <= 16 else (8 if E <= 32 else 16)
    L = E // V                                       # lanes of a row
    pair = [0, (V // 4 - 1) * 4 * L + 3]             # the first and the last number of the first lane
    for first, second in (pair, pair[::-1]):
        c = 0.5 - unit / 2 + r.uniform(-4e-8, 4e-8, (n, 2))
        s = c - np.array([0, apart * unit])
        z = torch.full((n, E), -60.0, dtype=torch.float64)
        z[:, [first, second]] = torch.from_numpy(np.log(s / (1 - s) if score == "sigmoid" else s))
        if score == "softmax":
            z[:, 5] = torch.from_numpy(np.log(1 - s.sum(1)))
        b = torch.full((E,), -100.0)
        b[first], b[second] = 64.0, 64.0 + apart * unit
        check(torch, z.float().cuda(), None, 1, score, True, b)


@pytest.mark.parametrize("score", SCORES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_no_expert_is_left(dtype, score):
    """Rows with as many experts to choose as are chosen, or fewer."""
    note(f"[none left] {dtype} {score}")
    torch = need_gpu()
    g = torch.Generator().manual_seed(8)
    for E, sets, top_sets, k in ((8, 1, 1, 8), (8, 2, 1, 4), (64, 8, 1, 8), (64, 16, 4, 16), (200, 1, 1, 32), (30, 10, 2, 6)):
        z = torch.randn(150, E, generator=g).to(getattr(torch, dtype)).cuda()
        ok = (torch.rand(150, E, generator=g) < 0.2).numpy()
        b = torch.randn(E, generator=g) * 0.1
        for mask in (None, ok):
            check(torch, z, mask, k, score, True, b, sets, top_sets, 2)
            check(torch, z, mask, k, score, False, None, sets, top_sets, 2)


@pytest.mark.parametrize("E,sets,top_sets", [(8, 2, 1), (64, 8, 3), (100, 10, 2), (256, 8, 4)])
def test_sigmoids_below_the_normal_floats(E, sets, top_sets):
    """Sums and biases of about the smallest normal float, which scores of logits near -88 have."""
    note(f"[tiny sigmoids] E={E} sets={sets}")
    torch = need_gpu()
    g = torch.Generator().manual_seed(E)
    z = (-86.3 - 2.5 * torch.rand(500, E, generator=g)).cuda()
    check(torch, z, None, 3, "sigmoid", True, None, sets, top_sets, 2)
    check(torch, z, None, 3, "sigmoid", True, torch.randn(E, generator=g) * 1e-38)
    check(torch, z, None, 3, "sigmoid", True, torch.randn(E, generator=g) * 1e-38, sets, top_sets, 2)
    check(torch, z, None, 3, "sigmoid", True, torch.randn(E, generator=g) * 1e-39, sets, top_sets, 1)


@pytest.mark.parametrize("score", SCORES)
@pytest.mark.parametrize("E,sets,top_sets", [(8, 1, 1), (30, 1, 1), (64, 1, 1), (64, 8, 4), (193, 1, 1), (1000, 10, 9)])
def test_infinity_is_above_the_largest_bf16(E, sets, top_sets, score):
    """A logit of +infinity counts as the largest float, which no bf16 number reaches."""
    note(f"[bf16 infinity] E={E} sets={sets} {score}")
    torch = need_gpu()
    g = torch.Generator().manual_seed(E)
    z = torch.randn(60, E, generator=g).bfloat16()
    top = torch.finfo(torch.bfloat16).max
    z[:30, 1], z[:30, 5] = top, INF
    z[30:, :4], z[30:, 4:7] = top, INF
    z[45:, 0], z[45:, 3] = -top, -INF
    z[50:, 2], z[50:, 7] = 0.0, -0.0
    z[55:, 8 - E:] = -top
    for k in (1, 2, 4):
        for renorm in (True, False):
            check(torch, z.cuda(), None, k, score, renorm, None, sets, top_sets, 1)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("E", [8, 40, 193, 1000])
def test_gradients_that_are_not_finite_stay_with_valid_experts(E, dtype):
    """dweight of NaN or infinity: dz of experts that are not valid is zero all the same, and other rows do not see it."""
    note(f"[dz of no expert] E={E} {dtype}")
    import paper_2606_11440_amd as P
    torch = need_gpu()
    g = torch.Generator().manual_seed(E)
    n, k = 70, 3
    z = torch.randn(n, E, generator=g).to(getattr(torch, dtype))
    ok = (torch.rand(n, E, generator=g) < 0.6).numpy()
    ok[:, 0] = True
    z[:, E // 2], z[:, E - 1] = -INF, float("nan")
    valid = torch.from_numpy(ok) & (z > -INF)
    for score in SCORES:
        for renorm in (False, True):
            ref = X.Router(z, score, ok)
            e = ref.choose(k)
            dw = torch.randn(n, k, generator=g)
            clean, tol = ref.grad(e, dw, renorm)
            bad = {4: float("nan"), 9: INF, 30: -INF, 69: float("nan")}
            for row, x in bad.items():
                dw[row, 0] = x
            dz = torch.full((n, E), 77.0, dtype=z.dtype, device="cuda")
            P.im_router_backward(z.cuda(), torch.from_numpy(e).int().cuda(), dw.cuda(), dz, valid=X.words(ok).cuda(),
                                 score=score, renorm=renorm)
            dz = dz.cpu()
            assert bool((dz[~valid] == 0).all()), (score, renorm)
            assert all(not bool(torch.isfinite(dz[row]).all()) for row in bad), (score, renorm)
            rows = [i for i in range(n) if i not in bad]
            X.same_or_close(dz[rows], clean[rows], tol[rows], (score, renorm))
