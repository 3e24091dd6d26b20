"""GPU: the learner's operators at sizes where launches and offsets are largest."""
import pytest

import learn_util as U
from gpu_util import need_gpu, note

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _memory():
    """These tests take tens of GB: none is kept for the next."""
    torch = need_gpu()
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def test_statistics_of_more_rows_than_a_launch_has_threads_for():
    """2^28 rows and some, with classes in several tiles that are joined: 16
    threads a row would be 2^32. Every row repeats one of 61."""
    import paper_2606_11440_amd as P
    torch = need_gpu()
    n, d, V, kinds = 2 ** 28 + 37, 8, 300, 61
    note(f"[rows] n={n}")
    g = torch.Generator(device="cuda").manual_seed(1)
    h = torch.randn(kinds, d, device="cuda", generator=g).bfloat16()
    W, b = torch.randn(1, V, d, device="cuda", generator=g).bfloat16(), torch.randn(1, V, device="cuda", generator=g)
    y = torch.randint(-1, V, (kinds,), device="cuda", generator=g, dtype=torch.int32)
    kind = torch.arange(n, device="cuda", dtype=torch.int32) % kinds
    hs, ys, step = torch.zeros(n, d, dtype=h.dtype, device="cuda"), y.index_select(0, kind), kinds << 18
    for at in range(0, n, step):       # torch's own selection is wrong past 2^31 elements
        hs[at:at + step] = h.index_select(0, kind[at:at + step])
        assert torch.equal(hs[at:at + kinds], h[:min(kinds, n - at)])
    o = {k: torch.full((n,), 77.0, device="cuda") for k in ("logp", "entropy", "lse")}
    P.im_head_forward(hs, W, b, ys, o["logp"], o["entropy"], o["lse"])
    torch.cuda.synchronize()
    r = U.Head(h, W, b, None, y, None)
    tol = dict(logp=r.e_logp, entropy=r.e_H, lse=r.e_logp + 2 * U.U * r.lse.abs())
    for k, want in (("logp", r.logp), ("entropy", r.H), ("lse", r.lse)):
        first = o[k][:kinds]
        U.close(first, want, tol[k], k)
        assert torch.equal(o[k], first.index_select(0, kind)), k   # a row's bits do not depend on its place


def test_gradient_of_more_tiles_than_a_launch_has_blocks_across():
    """65536 x 65536 in tiles of 256: 65536 tiles for a group that has rows and for
    one that has none."""
    import paper_2606_11440_amd as P
    torch = need_gpu()
    n, k, m = 3, 65536, 65536
    note(f"[tiles] {m} x {k}")
    g = torch.Generator(device="cuda").manual_seed(2)
    x, dy = (torch.randn(n, w, device="cuda", generator=g).bfloat16() for w in (k, m))
    W = torch.empty(2, m, k, dtype=torch.bfloat16, device="cuda")      # read for dx only
    dW, db = torch.empty_like(W), torch.full((2, m), 77.0, device="cuda")
    for at in range(0, m, 4096):
        dW[:, at:at + 4096] = 77.0
    off = torch.tensor([0, n, n], dtype=torch.int32, device="cuda")
    P.im_linear_backward(dy, x, W, None, dW, db, offsets=off)
    torch.cuda.synchronize()
    for at in range(0, m, 4096):
        want = dy[:, at:at + 4096].float().T @ x.float()
        size = dy[:, at:at + 4096].float().abs().T @ x.float().abs()
        over = (dW[0, at:at + 4096].float() - want).abs() - 2 * U.gamma(n) * size - U.ROUND[torch.bfloat16] * want.abs()
        assert float(over.max()) <= 0, at
        assert int(torch.count_nonzero(dW[1, at:at + 4096])) == 0, at
    U.close(db[0], dy.double().sum(0), U.gamma(n) * dy.double().abs().sum(0) + U.U * dy.double().sum(0).abs(), "db")
    assert int(torch.count_nonzero(db[1])) == 0
