"""GPU: the operators around experts as they are used together: a policy with a layer of experts, its
rollout in 8 bits and its update with 8-bit activations; captured, on streams, again."""
import pytest

import experts_util as X
from gpu_util import need_gpu, note

pytestmark = pytest.mark.gpu
N, D, E, K, H, D2, V = 300, 40, 6, 2, 48, 32, 15


class Policy:
    """x -> router -> experts (D -> H -> D2) -> softmax head over V actions; float32 or bfloat16."""

    def __init__(self, dtype, n=N, seed=0):
        torch = need_gpu()
        self.torch, self.n = torch, n
        dt = self.dt = getattr(torch, dtype)
        g = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*s, scale=1.0, t=dt):
            return (torch.randn(*s, device="cuda", generator=g) * scale).to(t)

        def empty(*s, t=dt):
            return torch.zeros(*s, dtype=t, device="cuda")
        f, i = torch.float32, torch.int32
        S = n * K
        self.x = normal(n, D)
        self.p = dict(Wr=normal(E, D, scale=D ** -0.5), br=normal(E, t=f, scale=0.1), W1=normal(E, H, D, scale=D ** -0.5),
                      b1=normal(E, H, t=f, scale=0.1), W2=normal(E, D2, H, scale=H ** -0.5),
                      b2=normal(E, D2, t=f, scale=0.1), Wh=normal(V, D2, scale=D2 ** -0.5), bh=normal(V, t=f, scale=0.1))
        self.target = torch.randint(0, V, (n,), device="cuda", generator=g, dtype=i)
        self.dlogp = normal(n, t=f, scale=1 / max(n, 1))
        self.bias = normal(E, t=f, scale=0.02)
        self.z, self.e, self.w = empty(n, E), empty(n, K, t=i), empty(n, K, t=f)
        self.off, self.slot = empty(E + 1, t=i), empty(n, K, t=i)
        self.xs, self.h, self.ys, self.y = empty(S, D), empty(S, H), empty(S, D2), empty(n, D2)
        i8 = torch.int8
        self.xq, self.xc, self.hq, self.hc = empty(S, D, t=i8), empty(S, t=f), empty(S, H, t=i8), empty(S, t=f)
        self.logp, self.lse = empty(n, t=f), empty(n, t=f)
        self.g = {k: torch.zeros_like(v) for k, v in self.p.items()}
        self.dy, self.dys, self.dw = empty(n, D2), empty(S, D2), empty(n, K, t=f)
        self.dh, self.dxs, self.dx, self.dz, self.dxr = empty(S, H), empty(S, D), empty(n, D), empty(n, E), empty(n, D)
        self.error = torch.zeros(1, dtype=i, device="cuda")

    def forward(self, stream=None):
        import paper_2606_11440_amd as P
        p, kw = self.p, dict(error=self.error, stream=stream)
        P.im_linear_forward(self.x, p["Wr"], p["br"], self.z, **kw)
        P.im_router_forward(self.z, self.e, self.w, bias=self.bias, stream=stream)
        P.im_dispatch_plan(self.e, self.off, self.slot, **kw)
        P.im_dispatch_forward(self.x, self.slot, self.xs, **kw)
        P.im_rows_pack(self.xs, self.xq, self.xc, stream=stream)
        P.im_linear_forward(self.xs, p["W1"], p["b1"], self.h, offsets=self.off, relu=True, **kw)
        P.im_rows_pack(self.h, self.hq, self.hc, keep=True, stream=stream)
        P.im_linear_forward(self.h, p["W2"], p["b2"], self.ys, offsets=self.off, **kw)
        P.im_combine_forward(self.ys, self.slot, self.w, self.y, **kw)
        P.im_head_forward(self.y, p["Wh"], p["bh"], self.target, self.logp, lse=self.lse, **kw)

    def backward(self, stream=None):
        import paper_2606_11440_amd as P
        p, g, kw = self.p, self.g, dict(error=self.error, stream=stream)
        P.im_head_backward(self.y, p["Wh"], p["bh"], self.target, self.lse, self.dlogp, self.dy, g["Wh"], g["bh"], **kw)
        P.im_combine_backward(self.dy, self.ys, self.slot, self.w, self.dys, self.dw, **kw)
        P.im_linear_backward_packed(self.dys, self.hq, self.hc, p["W2"], self.dh, g["W2"], g["b2"], offsets=self.off,
                                    relu_in=True, **kw)
        P.im_linear_backward_packed(self.dh, self.xq, self.xc, p["W1"], self.dxs, g["W1"], g["b1"], offsets=self.off, **kw)
        P.im_dispatch_backward(self.dxs, self.slot, self.dx, **kw)
        P.im_router_backward(self.z, self.e, self.dw, self.dz, **kw)
        P.im_linear_backward(self.dz, self.x, p["Wr"], self.dxr, g["Wr"], g["br"], **kw)

    def out(self):
        return [t.clone() for t in (self.e, self.w, self.off, self.slot, self.y, self.logp, self.dx, self.dxr, self.dw,
                                    *self.g.values())]


def reference(c):
    """The update in 64 bits with the kernels' choice of experts, ReLU side and 8-bit rows."""
    torch = c.torch
    p = {k: v.double().cpu() for k, v in c.p.items()}
    x, e, slot = c.x.double().cpu(), c.e.cpu().long(), c.slot.cpu().long()
    z = x @ p["Wr"].T + p["br"]
    q = torch.softmax(z.gather(1, e), 1)
    order = slot.reshape(-1).argsort()                    # pair of each place
    row, expert = order // K, e.reshape(-1)[order]
    xs = x[row]
    h = torch.relu(torch.einsum("sd,shd->sh", xs, p["W1"][expert]) + p["b1"][expert])
    ys = torch.einsum("sh,soh->so", h, p["W2"][expert]) + p["b2"][expert]
    y = (ys[slot] * q[:, :, None]).sum(1)
    zl = y @ p["Wh"].T + p["bh"]
    lse = torch.logsumexp(zl, 1)
    t = c.target.cpu().long()
    logp = zl.gather(1, t[:, None])[:, 0] - lse
    a = c.dlogp.double().cpu()
    dzl = a[:, None] * (torch.nn.functional.one_hot(t, V) - (zl - lse[:, None]).exp())
    dy = dzl @ p["Wh"]
    dw = (ys[slot] * dy[:, None]).sum(2)
    dys = torch.zeros_like(ys)
    dys[slot.reshape(-1)] = (q[:, :, None] * dy[:, None]).reshape(-1, D2)
    hq, xq = c.hq.cpu().double() * c.hc.cpu().double()[:, None], c.xq.cpu().double() * c.xc.cpu().double()[:, None]
    dh = torch.einsum("so,soh->sh", dys, p["W2"][expert]) * (c.hq.cpu() > 0)
    dxs = torch.einsum("sh,shd->sd", dh, p["W1"][expert])
    g = dict(Wh=dzl.T @ y, bh=dzl.sum(0))
    for name, d, inner in (("2", dys, hq), ("1", dh, xq)):
        parts = [expert == k for k in range(E)]
        g["W" + name] = torch.stack([d[m].T @ inner[m] for m in parts])
        g["b" + name] = torch.stack([d[m].sum(0) for m in parts])
    dzr = torch.zeros_like(z).scatter_add_(1, e, q * (dw - (q * dw).sum(1, keepdim=True)))
    g |= dict(Wr=dzr.T @ x, br=dzr.sum(0))
    return dict(y=y, logp=logp, dx=dxs[slot].sum(1), dxr=dzr @ p["Wr"], dw=dw), g


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_update(dtype):
    """Against 64 bits. Every result is the end of eight stages at most; a stage is off by 2 (600 + 8) 2^-24
    = 7e-5 of its terms' magnitudes, in bf16 by two roundings (operand and result) of 2^-8 more. Terms outweigh
    the largest result of their tensor by 4 at most here: 8 * 4 * 7e-5 = 0.0023 and, as roundings of different
    elements do not add up in one direction, 8 * 2^-7 = 0.0625 of the largest result."""
    note(f"[experts: update] {dtype}")
    c = Policy(dtype)
    c.forward()
    c.backward()
    assert int(c.error) == 0
    assert bool((c.hq.cpu() > 0)[c.h.cpu() > 0].all())      # the ReLU's sides are those of the codes
    outs, grads = reference(c)
    share = 0.0023 if dtype == "float32" else 0.0625
    for k, want in list(outs.items()) + list(grads.items()):
        got = getattr(c, k) if k in outs else c.g[k].reshape(want.shape)
        X.same_or_close(got, want, share * want.abs().max() * c.torch.ones_like(want), k)


def test_kept_rows_are_near_enough():
    """What keeping 8-bit rows costs: dW against the gradient from the rows themselves. A code is off by half a
    scale (one where a ReLU's small values are kept), 1/127 of the row's largest value at most."""
    note("[experts: 8-bit rows]")
    import paper_2606_11440_amd as P
    c = Policy("float32")
    c.forward()
    c.backward()
    dW = c.torch.empty_like(c.p["W2"])
    P.im_linear_backward(c.dys, c.h, c.p["W2"], None, dW, None, offsets=c.off)
    size = c.torch.empty_like(dW)
    top = c.h.abs().amax(1, keepdim=True).expand_as(c.h).contiguous()
    P.im_linear_backward(c.dys.abs(), top, c.p["W2"], None, size, None, offsets=c.off)
    assert bool(((c.g["W2"] - dW).abs() <= size * (1.01 / 127) + 1e-9).all())
    P.im_rows_unpack(c.hq, c.hc, top)
    assert bool(((top - c.h).abs() <= c.hc[:, None] * 1.0001).all() and ((top > 0) == (c.h > 0)).all())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_rollout_in_8_bits(dtype):
    """Router, codes and scales sent to their experts, products in 8 bits, weighted sum."""
    note(f"[experts: rollout] {dtype}")
    import paper_2606_11440_amd as P
    c = Policy(dtype, n=1000)
    torch = c.torch
    c.forward()
    q, s = torch.empty(c.n, D, dtype=torch.int8, device="cuda"), torch.empty(c.n, 1, device="cuda")
    P.im_rows_pack(c.x, q, s[:, 0])
    S = c.n * K
    qs, ss = torch.empty(S, D, dtype=torch.int8, device="cuda"), torch.empty(S, 1, device="cuda")
    P.im_dispatch_forward(q, c.slot, qs, error=c.error)
    P.im_dispatch_forward(s, c.slot, ss, error=c.error)
    assert bool((qs == c.xq).all() and (ss[:, 0] == c.xc).all())      # packed before or after
    Wq, Ws = torch.empty(E * H, D, dtype=torch.int8, device="cuda"), torch.empty(E * H, device="cuda")
    P.im_rows_pack(c.p["W1"].reshape(E * H, D), Wq, Ws)
    Wq, Ws = Wq.reshape(E, H, D), Ws.reshape(E, H)
    h = torch.empty(S, H, dtype=c.dt, device="cuda")
    P.im_linear_forward_packed(qs, ss[:, 0].contiguous(), Wq, Ws, c.p["b1"], h, offsets=c.off, relu=True, error=c.error)
    assert int(c.error) == 0
    want, tol = X.packed_linear(qs, ss[:, 0], Wq, Ws, c.p["b1"], c.off.tolist(), True, c.dt)
    X.same_or_close(h, want, tol, "h")


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_captured(dtype):
    """Forward and backward in one graph, replayed on other inputs, with eager work between."""
    note(f"[experts: captured] {dtype}")
    c, eager = Policy(dtype), Policy(dtype)
    torch = c.torch
    c.forward()
    c.backward()      # sizes of workspaces are known, kernels loaded
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.forward()
        c.backward()
    for r in range(4):
        x = torch.randn(N, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(r)).to(c.dt)
        c.x.copy_(x)
        eager.x.copy_(x)
        for t in (c.xs, c.ys, c.dys):
            t.zero_()
        graph.replay()
        eager.forward()
        eager.backward()
        torch.cuda.synchronize()
        for a, b in zip(c.out(), eager.out()):
            assert bool((a == b).all()), r


def test_two_streams():
    """Two policies at the same time on streams of their own, each with workspaces of its own."""
    note("[experts: streams]")
    torch = need_gpu()
    n = 40000
    want = []
    for seed in (1, 2):
        c = Policy("bfloat16", n=n, seed=seed)
        c.forward()
        c.backward()
        want.append(c.out())
    both = [Policy("bfloat16", n=n, seed=seed) for seed in (1, 2)]
    streams = [torch.cuda.Stream() for _ in both]
    torch.cuda.synchronize()
    for _ in range(2):
        for c, s in zip(both, streams):     # by torch's current stream, and by handle
            with torch.cuda.stream(s):
                c.forward()
            c.backward(stream=s.cuda_stream)
    torch.cuda.synchronize()
    for c, w in zip(both, want):
        assert int(c.error) == 0
        for a, b in zip(c.out(), w):
            assert bool((a == b).all())


def test_the_same_bits_again():
    note("[experts: again]")
    c = Policy("bfloat16", n=20000, seed=5)
    c.forward()
    c.backward()
    first = c.out()
    for _ in range(2):
        c.forward()
        c.backward()
        for a, b in zip(c.out(), first):
            assert bool((a == b).all())


def test_captured_plan_and_long_sums():
    """What takes workspaces (a plan in blocks, a product in runs of k), captured and replayed on other inputs."""
    note("[experts: captured workspaces]")
    import paper_2606_11440_amd as P
    torch = need_gpu()
    n, k, e = 30000, 2, 50
    expert = torch.zeros(n, k, dtype=torch.int32, device="cuda")
    off, slot = torch.zeros(e + 1, dtype=torch.int32, device="cuda"), torch.zeros_like(expert)
    q, s = torch.zeros(20, 9000, dtype=torch.int8, device="cuda"), torch.ones(20, device="cuda")
    W, y = torch.randint(-127, 128, (33, 9000), dtype=torch.int8, device="cuda"), torch.zeros(20, 33, device="cuda")
    Ws = torch.rand(33, device="cuda")

    def run(off, slot, y):
        P.im_dispatch_plan(expert, off, slot)
        P.im_linear_forward_packed(q, s, W, Ws, None, y)
    run(off, slot, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(off, slot, y)
    for r in range(4):
        expert.copy_(torch.randint(-1, e, (n, k), dtype=torch.int32, generator=torch.Generator().manual_seed(r)))
        q.copy_(torch.randint(-127, 128, q.shape, dtype=torch.int8, generator=torch.Generator().manual_seed(r)))
        graph.replay()
        a = [torch.zeros_like(t) for t in (off, slot, y)]
        run(*a)
        torch.cuda.synchronize()
        assert all(bool((x == z).all()) for x, z in zip(a, (off, slot, y))), r
        assert bool((slot.cpu() == X.plan(expert.cpu(), e)[1]).all())


def test_no_rows_anywhere():
    """Every call without rows."""
    note("[experts: none]")
    c = Policy("float32", n=0)
    for t in list(c.g.values()):
        t.fill_(7.0)
    c.forward()
    c.backward()
    assert int(c.error) == 0 and c.off.tolist() == [0] * (E + 1)
    assert all(bool((t == 0).all()) for t in c.g.values())
