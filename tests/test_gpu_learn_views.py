"""GPU: buffers that the caller lays out. Outputs and inputs in one buffer: side
by side they give what separate buffers give, bit for bit; on one another the
call is refused. Workspaces of just the size that a call asks for."""
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


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,G,k,V", [(16, 1, 4096, 256), (3000, 5, 256, 15), (900, 3, 200, 700)])
def test_workspaces_of_just_their_size(n, G, k, V, dtype):
    """One call of each after the other in one buffer: its end stays as it was, and
    a byte less is refused."""
    import paper_2606_11440_amd as P
    torch = need_gpu()
    note(f"[workspaces] n={n} G={G} {k} -> {V} {dtype}")
    g = torch.Generator(device="cuda").manual_seed(n)
    dt = getattr(torch, dtype)
    x, dy, W = (torch.randn(*s, device="cuda", generator=g).to(dt) for s in ((n, k), (n, V), (G, V, k)))
    b, target = torch.randn(G, V, device="cuda", generator=g), torch.randint(V, (n,), device="cuda", generator=g, dtype=torch.int32)
    off = torch.arange(G + 1, device="cuda", dtype=torch.int32) * (n // G)
    f = [torch.zeros(n, device="cuda") for _ in range(6)]
    f[3].normal_(generator=g)
    f[4].normal_(generator=g)
    out = {}

    def calls(tag, buffer):
        y, dx, dW, db, dh = (torch.zeros_like(t) for t in (dy, x, W, b, x))
        kw = lambda size: dict(offsets=off, workspace=buffer(size))  # noqa: E731
        P.im_linear_forward(x, W, b, y, **kw(P.im_linear_workspace(n, k, V, dt, G)))
        P.im_linear_backward(dy, x, W, dx, dW, db, **kw(P.im_linear_workspace(n, k, V, dt, G, backward=True, device=x.device)))
        out[tag] = [y, dx, dW.clone(), db.clone()]
        P.im_head_forward(x, W, b, target, f[0], f[1], f[2], **kw(P.im_head_workspace(n, k, V, dt, G)))
        P.im_head_backward(x, W, b, target, f[2], f[3], dh, dW, db, entropy=f[1], dentropy=f[4],
                           **kw(P.im_head_workspace(n, k, V, dt, G, backward=True, device="cuda")))
        torch.cuda.synchronize()
        out[tag] += [dh, dW, db] + [t.clone() for t in f[:3]]
    whole = torch.empty(1 << 27, dtype=torch.uint8, device="cuda")

    def exact(size):
        assert size < len(whole)
        whole[size:].fill_(77)
        sizes.append(size)
        return whole[:size]
    sizes = []
    calls("own", lambda size: None)
    calls("exact", exact)
    assert all(torch.equal(a, b) for a, b in zip(out["own"], out["exact"]))
    assert bool((whole[sizes[-1]:] == 77).all()) and max(sizes) > 0
    with pytest.raises(P.IMError) as e:
        P.im_head_backward(x, W, b, target, f[2], f[3], torch.zeros_like(x), offsets=off, workspace=whole[:sizes[-1] - 1])
    assert "workspace" in str(e.value)
