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
