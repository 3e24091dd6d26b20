"""GPU: the operators as a training program uses them: a policy's update from a
rollout of the pool, the same update captured into a graph, calls on streams."""
import numpy as np
import pytest

import learn_util as U
import workload
from gpu_util import need_gpu, note

pytestmark = pytest.mark.gpu


class Policy:
    """Three layers, 86 -> 256 -> 256 -> 15, for G members side by side: fp32
    parameters, bf16 copies for the products, AdamW in 32 or 8 bits."""

    def __init__(self, W, b, G=1, bits=32):
        import paper_2606_11440_amd as P
        torch = need_gpu()
        self.P, self.torch, self.tensors, self.W, self.b, self.dW, self.db = P, torch, [], [], [], [], []
        for w, c in zip(W, b):
            for x, decay in ((w, True), (c, False)):
                p = torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda()
                p = p.expand(G, *p.shape).contiguous()
                t = dict(param=p, decay=decay)
                if decay:
                    t |= dict(copy=p.bfloat16(), grad=torch.zeros_like(p, dtype=torch.float32))
                else:
                    t |= dict(grad=torch.zeros_like(p))
                n = p.numel()
                if bits == 32:
                    t |= dict(m=torch.zeros_like(p), v=torch.zeros_like(p))
                else:
                    z = torch.zeros(n, dtype=torch.uint8, device="cuda")
                    t |= dict(m=z.clone().view(torch.float8_e4m3fn), v=z.view(torch.float8_e4m3fn),
                              m_scale=torch.zeros(-(-n // 256), device="cuda"), v_scale=torch.zeros(-(-n // 256), device="cuda"))
                self.tensors.append(t)
                if decay:
                    self.W.append(t["copy"])
                    self.dW.append(torch.zeros_like(t["copy"]))
                else:
                    self.b.append(p)
                    self.db.append(t["grad"])
        self.opt = P.AdamW(self.tensors, bits=bits)
        self.step = torch.zeros(1, dtype=torch.int64, device="cuda")
        self.scale = torch.ones(1, device="cuda")

    def buffers(self, n):
        e = lambda *s, t=self.torch.bfloat16: self.torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
        f = self.torch.float32
        return dict(h1=e(n, 256), h2=e(n, 256), d1=e(n, 256), d2=e(n, 256), logp=e(n, t=f), lse=e(n, t=f),
                    entropy=e(n, t=f), dlogp=e(n, t=f), dent=e(n, t=f))

    def forward(self, x, y, valid, off, o, **kw):
        P, W, b = self.P, self.W, self.b
        P.im_linear_forward(x, W[0], b[0], o["h1"], offsets=off, relu=True, **kw)
        P.im_linear_forward(o["h1"], W[1], b[1], o["h2"], offsets=off, relu=True, **kw)
        P.im_head_forward(o["h2"], W[2], b[2], y, o["logp"], entropy=o["entropy"], lse=o["lse"], valid=valid, offsets=off, **kw)

    def backward(self, x, y, valid, off, o, **kw):
        P, W, b, dW, db = self.P, self.W, self.b, self.dW, self.db
        P.im_head_backward(o["h2"], W[2], b[2], y, o["lse"], o["dlogp"], o["d2"], dW[2], db[2], valid=valid,
                           entropy=o["entropy"], dentropy=o["dent"], offsets=off, relu_in=True, **kw)
        P.im_linear_backward(o["d2"], o["h1"], W[1], o["d1"], dW[1], db[1], offsets=off, relu_in=True, **kw)
        P.im_linear_backward(o["d1"], x, W[0], None, dW[0], db[0], offsets=off, **kw)

    def update(self, **kw):
        for i in range(3):
            self.tensors[2 * i]["grad"].copy_(self.dW[i])
        self.opt.step(self.step, lr=1e-3, weight_decay=0.01, scale=self.scale, **kw)


def rollout(E=48, ticks=3, seed=5):
    """A few ticks of a c2 pool; features, masks, actions and statistics of the last."""
    torch = need_gpu()
    import paper_2606_11440_amd as P
    cfg = workload.configs.get("c2", E=E, T=ticks, lam=24.0, qcap=24)
    W, b = workload.gen.weights(cfg, seed, 0.1)
    table, _ = workload.gen.embedding(cfg, seed, rows=128)
    cap = workload.gen.capacities(cfg, seed)
    emb = torch.from_numpy(table.view(np.int16)).cuda()
    pool = P.Pool(cfg, W, b, emb, cap)
    counts = workload.gen.counts(cfg, seed)
    M, A = cfg["M"], cfg["A"]
    for t in range(ticks):
        arr = workload.gen.tick(cfg, seed, t, counts[t], 128)
        dev, n = P.device_arrivals(arr), len(arr["q_idx"])
        st = pool.state()
        act = torch.zeros(n, dtype=torch.int32, device="cuda")
        logp, ent = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
        pool.route_sample(dev, 1234 + t, act, logp, ent)
        pool.schedule(dev, act)
    env = np.repeat(np.arange(E), np.diff(arr["offsets"]))
    c = np.maximum(st["cap"], 1)
    stats = np.concatenate([st["qlen"] / cfg["qcap"], st["busy"] / c, st["ewma"] / (256 * cfg["budget_max"]),
                            st["backlog"] / (c * cfg["budget_max"])], 1).astype(np.float32)
    x = torch.cat([emb.view(torch.bfloat16)[torch.from_numpy(arr["q_idx"]).long().cuda()].float(),
                   torch.from_numpy(stats[env]).cuda(),
                   torch.from_numpy(arr["budget"].astype(np.float32) / cfg["budget_max"]).cuda()[:, None]], 1)
    ok = ((st["enabled"] != 0) & (st["cap"] > 0) & (st["qlen"] < cfg["qcap"]))[env]
    bits = (np.repeat(ok, cfg["K"], 1).astype(np.int64) << np.arange(A)).sum(1).astype(np.int32)
    pad = cfg["feat_dim"] - x.shape[1]
    x = torch.nn.functional.pad(x, (0, pad)).bfloat16().contiguous()
    assert pool.error() == 0 and M * cfg["K"] == A
    pool.close()
    return dict(W=W, b=b, x=x, valid=torch.from_numpy(bits).cuda()[:, None].contiguous(), act=act, logp=logp, ent=ent,
                env_off=arr["offsets"], E=E)


def test_update_from_a_rollout():
    """The learner's forward gives the rollout's log-probabilities and
    entropies; its gradients are those of the whole network in 64 bits; after
    the step the copies are the rounded parameters."""
    torch = need_gpu()
    r = rollout()
    n = len(r["act"])
    note(f"[update] rows={n}")
    pol = Policy(r["W"], r["b"])
    o = pol.buffers(n)
    pol.forward(r["x"], r["act"], r["valid"], None, o)
    taken = r["act"] >= 0
    assert int(taken.sum()) > 100
    # both round hidden activations to bf16, after sums in another order: a step of 2^-8 in some
    # activations moves a logit by 2^-8 of itself; logits here are below 8
    assert float((o["logp"] - r["logp"]).abs().max()) < 8 * 2 ** -8 * 2
    assert float((o["entropy"] - r["ent"]).abs().max()) < 8 * 2 ** -8 * 2
    g = torch.Generator(device="cuda").manual_seed(3)
    adv = torch.randn(n, device="cuda", generator=g)
    o["dlogp"].copy_(-adv / n)
    o["dent"].fill_(-0.1 / n)
    pol.backward(r["x"], r["act"], r["valid"], None, o)
    torch.cuda.synchronize()
    # 64 bits, on the activations the kernels made
    head = U.Head(o["h2"], pol.W[2], pol.b[2], r["valid"], r["act"], None)
    (dh, eh), (dW, eW), (db, eb) = head.grads(o["dlogp"], o["dent"], True)
    U.close(pol.dW[2], dW, eW, "dW of the head")
    U.close(o["d2"], dh, eh, "d2")
    for i, (d, x, out, relu) in enumerate(((o["d2"], o["h1"], o["d1"], True), (o["d1"], r["x"], None, False))):
        (dx, ex), (w, ew), (c, ec) = U.linear_grad(d, x, pol.W[1 - i], None, relu)
        U.close(pol.dW[1 - i], w, ew, f"dW {1 - i}")
        U.close(pol.db[1 - i], c, ec, f"db {1 - i}")
        if out is not None:
            U.close(out, dx, ex, "d1")
    before = [t["param"].clone() for t in pol.tensors]
    pol.update()
    torch.cuda.synchronize()
    assert int(pol.step) == 1
    for t, old in zip(pol.tensors, before):
        assert not torch.equal(t["param"], old)
        if "copy" in t:
            assert torch.equal(t["copy"], t["param"].bfloat16())


def case(G, bits, seed=0):
    torch = need_gpu()
    r = rollout(seed=5 + seed)
    pol = Policy(r["W"], r["b"], G=G, bits=bits)
    ends = np.linspace(0, r["E"], G + 1).astype(int)
    off = torch.from_numpy(np.asarray(r["env_off"])[ends].astype(np.int32)).cuda()
    o = pol.buffers(len(r["act"]))
    g = torch.Generator(device="cuda").manual_seed(seed)
    o["dlogp"].copy_(torch.randn(len(r["act"]), device="cuda", generator=g) / len(r["act"]))
    o["dent"].fill_(-0.1 / len(r["act"]))
    return pol, r, off, o


def train(pol, r, off, o, **kw):
    pol.forward(r["x"], r["act"], r["valid"], off, o, **kw)
    pol.backward(r["x"], r["act"], r["valid"], off, o, **kw)
    pol.update(**kw)


@pytest.mark.parametrize("G,bits", [(1, 32), (4, 8)])
def test_captured_update(G, bits):
    """A whole update in a graph, replayed with eager work between, against the
    same updates called one by one: the same bits, and the steps are counted."""
    torch = need_gpu()
    note(f"[graph] G={G} bits={bits}")
    a, b = case(G, bits), case(G, bits)
    train(*a)
    train(*b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        train(*a)
    for k in range(4):
        graph.replay()
        train(*b)
        _ = torch.randn(1000, 1000, device="cuda").sum().item()
        torch.cuda.synchronize()
        assert int(a[0].step) == int(b[0].step) == k + 2
        for s, t in zip(a[0].tensors, b[0].tensors):
            for key in s:
                if hasattr(s[key], "view"):
                    x, y = (v[key].view(torch.uint8) if v[key].dtype == torch.float8_e4m3fn else v[key] for v in (s, t))
                    assert torch.equal(x, y), (k, key)


def test_members_of_a_population_get_their_own_gradients():
    """Members side by side: each one's gradients are those of its own rows."""
    pol, r, off, o = case(3, 32)
    train(pol, r, off, o)
    cuts = off.tolist()
    assert int(pol.step) == 1
    pol, r, off, o = case(3, 32)      # the weights before the step
    pol.forward(r["x"], r["act"], r["valid"], off, o)
    pol.backward(r["x"], r["act"], r["valid"], off, o)
    head = U.Head(o["h2"], pol.W[2], pol.b[2], r["valid"], r["act"], cuts)
    U.close(o["logp"], head.logp, head.e_logp, "logp")
    _, (dW, eW), (db, eb) = head.grads(o["dlogp"], o["dent"], True)
    U.close(pol.dW[2], dW, eW, "dW of the heads")
    U.close(pol.db[2], db, eb, "db of the heads")
    for i, (d, x) in enumerate(((o["d2"], o["h1"]), (o["d1"], r["x"]))):
        _, (w, ew), (c, ec) = U.linear_grad(d, x, pol.W[1 - i], cuts, False)
        U.close(pol.dW[1 - i], w, ew, f"dW {1 - i}")
        U.close(pol.db[1 - i], c, ec, f"db {1 - i}")


def test_streams():
    """Calls on streams of their own, by handle and as the current stream, at
    the same time: each gives what it gives alone."""
    torch = need_gpu()
    note("[streams]")
    want = []
    for s in range(2):
        c = case(3, 32, seed=s)
        train(*c)
        torch.cuda.synchronize()
        want.append([t["param"].clone() for t in c[0].tensors])
    cases = [case(3, 32, seed=s) for s in range(2)]
    torch.cuda.synchronize()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    for (pol, r, off, o), stream, by_handle in zip(cases, (one, two), (True, False)):
        if by_handle:
            pol.forward(r["x"], r["act"], r["valid"], off, o, stream=stream.cuda_stream)
            pol.backward(r["x"], r["act"], r["valid"], off, o, stream=stream.cuda_stream)
            with torch.cuda.stream(stream):
                pol.update(stream=stream.cuda_stream)
        else:
            with torch.cuda.stream(stream):
                train(pol, r, off, o)
    torch.cuda.synchronize()
    for (pol, *_), w in zip(cases, want):
        assert all(torch.equal(t["param"], x) for t, x in zip(pol.tensors, w))


def test_own_workspace():
    """A workspace of the caller's own, reused by one call after the other."""
    torch = need_gpu()
    pol, r, off, o = case(2, 32)
    train(pol, r, off, o)
    want = [t["param"].clone() for t in pol.tensors]
    pol, r, off, o = case(2, 32)
    ws = torch.full((1 << 28,), 255, dtype=torch.uint8, device="cuda")
    pol.forward(r["x"], r["act"], r["valid"], off, o, workspace=ws)
    pol.backward(r["x"], r["act"], r["valid"], off, o, workspace=ws)
    pol.update()
    assert all(torch.equal(t["param"], w) for t, w in zip(pol.tensors, want))
