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
