"""GPU: outputs and inputs in one buffer: side by side they give what separate
buffers give, bit for bit; on one another the call is refused."""
import pytest

from gpu_util import need_gpu, note

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,k,m", [(1, 8, 24), (300, 86, 256), (1000, 256, 40)])
def test_columns_side_by_side(n, k, m, dtype):
    import paper_2606_11440_amd as P
    torch = need_gpu()
    note(f"[views] {n} x ({k}, {m}) {dtype}")
    g = torch.Generator(device="cuda").manual_seed(n)
    dt = getattr(torch, dtype)
    x, dy, W = (torch.randn(*s, device="cuda", generator=g).to(dt) for s in ((n, k), (n, m), (1, m, k)))
    b = torch.randn(1, m, device="cuda", generator=g)
    y, dx, dW, db = torch.empty_like(dy), torch.empty_like(x), torch.empty_like(W), torch.empty_like(b)
    P.im_linear_forward(x, W, b, y, relu=True)
    P.im_linear_backward(dy, x, W, dx, dW, db)
    one = torch.full((n, 2 * (k + m) + 3), 77.0, dtype=dt, device="cuda")
    X, Y, DY, DX = (one[:, a:a + w] for a, w in ((0, k), (k, m), (k + m + 1, m), (k + 2 * m + 1, k)))
    X.copy_(x)
    DY.copy_(dy)
    P.im_linear_forward(X, W, b, Y, relu=True)
    DW, DB = torch.empty_like(W), torch.empty_like(b)
    P.im_linear_backward(DY, X, W, DX, DW, DB)
    torch.cuda.synchronize()
    for got, want in ((X, x), (Y, y), (DY, dy), (DX, dx), (DW, dW), (DB, db)):
        assert torch.equal(got, want)
    assert bool((one[:, k + m] == 77).all()) and bool((one[:, 2 * (k + m) + 1:] == 77).all())


def test_overlaps_are_refused():
    import paper_2606_11440_amd as P
    torch = need_gpu()
    x, W = torch.ones(64, 32, device="cuda"), torch.ones(32, 32, device="cuda")
    t, v = torch.zeros(64, dtype=torch.int32, device="cuda"), [torch.zeros(64, device="cuda") for _ in range(4)]
    keep = x.clone()
    wide = torch.ones(64, 60, device="cuda")
    for call in (lambda: P.im_linear_forward(x, W, None, x), lambda: P.im_linear_backward(x, x, W, x),
                 lambda: P.im_linear_forward(x[:63], W, None, x[1:]), lambda: P.im_linear_forward(wide[:, :32], W, None, wide[:, 28:]),
                 lambda: P.im_linear_backward(x, keep, W, torch.empty_like(x), W), lambda: P.im_head_forward(x, W, None, t, v[0], v[0]),
                 lambda: P.im_head_forward(x, W, None, t, v[0], v[1], v[1]),
                 lambda: P.im_head_backward(x, W, None, t, v[0], v[1], x), lambda: P.im_head_backward(x, W, None, t, v[0], v[1], None, W),
                 lambda: P.im_linear_forward(x, W, None, torch.empty(64, 32, device="cuda"), error=x.view(torch.int32).view(-1)[5:6])):
        with pytest.raises(P.IMError) as e:
            call()
        assert e.value.status == P._lib.IM_EINVAL and "overlaps" in str(e.value)
    torch.cuda.synchronize()
    assert torch.equal(x, keep)
