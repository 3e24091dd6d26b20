"""Workloads of the operators around a mixture of experts and of 8-bit rows.

  router      scores of experts (softmax or sigmoid), choice of the best few by score + bias,
              within the best sets of experts, and their weights; the gradient of the logits
  dispatch    where each chosen (row, expert) pair goes when rows are ordered by expert, the rows
              sent there; the gradient's way back
  combine     the weighted sum of what the experts return to a row; its gradient
  packed      a grouped layer in 8-bit integers: rows are packed (codes and a scale a row), then
              multiplied with packed weights
  checkpoint  gradients of a grouped layer whose input was kept as 8-bit rows

`run` computes them either in their plain form (elementary torch operations, in
32 bits and in 64 where a choice hangs on it, rounded once at the end) or, where
`own` is set, through the framework. Group sizes are ragged (some may be empty),
a few rows have no valid expert, weights are those of an untrained network.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
LARGEST = 3.4028234663852886e38
MOST_FLOPS = 2.7e11        # of the largest listed case
MOST_ELEMENTS = 1 << 27    # of the rows that the largest listed exchange moves
TYPES = dict(f32=torch.float32, bf16=torch.bfloat16)


def _router(name, kind, n, E, k, score="softmax", renorm=True, bias=False, sets=1, top_sets=1, best=1, mask=False,
            dtype="f32"):
    return dict(name=name, op="router", kind=kind, rows=n, experts=E, top_k=k, score=score, renorm=renorm, bias=bias,
                sets=sets, top_sets=top_sets, best=best, mask=mask, dtype=dtype)


def _exchange(name, op, kind, n, E, k, d, dtype="bf16", pad=0, drop=0.0):
    return dict(name=name, op=op, kind=kind, rows=n, experts=E, top_k=k, dim=d, dtype=dtype, pad=pad, drop=drop)


def _layer(name, op, G, n, k, m, dtype="bf16", relu=True, pad=0):
    return dict(name=name, op=op, groups=G, rows=n, in_dim=k, out_dim=m, dtype=dtype, relu=relu, pad=pad)


def listed():
    return [
        # a controller's few pending requests, one of 8 experts' pairs each: latency
        _router("router_few_rows", "forward", 48, 8, 2),
        # one tick of 4096 envs: 64 experts in 8 sets, balanced by a bias, scores by sigmoid
        _router("router_tick", "forward", 262144, 64, 4, score="sigmoid", bias=True, sets=8, top_sets=4, best=2),
        # gradient of a dense softmax over an odd number of experts, some masked, bf16 logits
        _router("router_backward", "backward", 100003, 193, 6, renorm=False, mask=True, dtype="bf16"),
        # the same few requests sent to 8 experts: plan and rows, latency
        _exchange("dispatch_few_rows", "dispatch", "forward", 48, 8, 2, 256, dtype="f32"),
        # rows of a wide policy's hidden layer sent to 64 experts
        _exchange("dispatch_tick", "dispatch", "forward", 65536, 64, 4, 512),
        # fp32 rows of an odd width, a tenth of the pairs dropped, out of a wider activation
        _exchange("combine_odd", "combine", "forward", 30011, 193, 3, 387, dtype="f32", pad=5, drop=0.1),
        # gradient of the weighted sum: rows to the experts, a scalar for each weight
        _exchange("combine_backward", "combine", "backward", 65536, 64, 4, 512, drop=0.02),
        # first layer of a policy on a few pending requests, in 8 bits: latency
        _layer("packed_few_rows", "packed", 1, 48, 86, 256, dtype="f32"),
        # hidden layer of 64 wide policies on one tick of 4096 envs, a rollout's product
        _layer("packed_population", "packed", 64, 262144, 512, 512),
        # eight wide experts, rows cut out of a wider activation
        _layer("packed_experts", "packed", 8, 16384, 2048, 4096, relu=False, pad=64),
        # gradients of the hidden layer of 64 wide policies from kept 8-bit rows
        _layer("checkpoint_backward", "checkpoint", 64, 262144, 512, 512),
        # of an fp32 policy's hidden layer, a ragged number of rows of 1024 envs
        _layer("checkpoint_backward_f32", "checkpoint", 1, 16001, 256, 256, dtype="f32"),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["router", "router", "dispatch", "combine", "packed", "checkpoint"])
    dtype = "f32" if rng.random() < 0.35 else "bf16"
    while True:
        n = log(1, 262144)
        if op == "router":
            sets, best = 1, 1
            E = log(4, 512)
            if rng.random() < 0.4:
                sets = rng.choice([2, 3, 4, 8, 16])
                E, best = sets * max(1, E // sets), rng.choice([1, 2])
            top_sets = rng.randint(1, sets)
            c = dict(op=op, kind=rng.choice(["forward", "backward"]), rows=n, experts=E,
                     top_k=rng.randint(1, min(16, E // sets * top_sets)), score=rng.choice(["softmax", "sigmoid"]),
                     renorm=rng.random() < 0.6, bias=rng.random() < 0.5, sets=sets, top_sets=top_sets, best=best,
                     mask=rng.random() < 0.4, dtype=dtype)
            if n * E <= 1 << 25:
                return c
        elif op in ("dispatch", "combine"):
            E = log(2, 512)
            c = dict(op=op, kind=rng.choice(["forward", "backward"]), rows=n, experts=E, top_k=rng.randint(1, min(8, E)),
                     dim=log(15, 4096), dtype=dtype, pad=rng.choice([0, 0, 1, 8, 64]), drop=rng.choice([0.0, 0.1]))
            if n * c["top_k"] * c["dim"] <= MOST_ELEMENTS:
                return c
        else:
            c = dict(op=op, groups=1 if rng.random() < 0.3 else log(2, 128), rows=n, in_dim=log(17, 4096),
                     out_dim=log(15, 4096), dtype=dtype, relu=rng.random() < 0.5, pad=rng.choice([0, 0, 1, 8, 64]))
            cap = MOST_FLOPS * (0.05 if op == "checkpoint" and dtype == "f32" else 1.0)
            wide = max(c["in_dim"], c["out_dim"])
            if work(c)["flops"] <= cap and n * wide <= MOST_ELEMENTS and c["groups"] * c["in_dim"] * c["out_dim"] <= 1 << 27:
                return c


def work(case):
    n, e = case["rows"], 4 if case["dtype"] == "f32" else 2
    back = case.get("kind") == "backward"
    if case["op"] == "router":
        E, k = case["experts"], case["top_k"]
        mask = n * 4 * ((E + 31) // 32) if case["mask"] else 0
        if back:
            return {"bytes": 2 * n * E * e + 8 * n * k + mask, "flops": 6 * n * E}
        return {"bytes": n * E * e + 8 * n * k + mask + (4 * E if case["bias"] else 0), "flops": (4 + k) * n * E}
    if case["op"] in ("dispatch", "combine"):
        E, k, d = case["experts"], case["top_k"], case["dim"]
        sent = n * k * (1 - case["drop"])    # rows that move
        pairs = 4 * n * k
        if case["op"] == "dispatch":
            return {"bytes": int(e * d * (n + sent)) + pairs + (0 if back else pairs + 4 * (E + 1)), "flops": int(sent * d)}
        if back:
            return {"bytes": int(e * d * (n + 2 * sent)) + 3 * pairs, "flops": int(3 * sent * d)}
        return {"bytes": int(e * d * (n + sent)) + 2 * pairs, "flops": int(2 * sent * d)}
    G, k, m = case["groups"], case["in_dim"], case["out_dim"]
    if case["op"] == "packed":
        return {"bytes": e * n * (k + m) + G * k * m + 8 * G * m, "flops": 2 * n * k * m}
    return {"bytes": e * n * (k + m) + n * (k + 4) + 2 * e * G * k * m + 4 * G * m, "flops": 4 * n * k * m}


# ---- inputs -----------------------------------------------------------------

def _sizes(n, G, r):
    """Ragged group sizes that sum to n."""
    share = r.gamma(2.0, 1.0, G) * (r.random(G) > 0.05)
    if not share.sum():
        share[:] = 1.0
    return r.multinomial(n, share / share.sum()) if G > 1 else np.array([n])


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    n, dt = case["rows"], TYPES[case["dtype"]]

    def normal(*shape, scale=1.0, dtype=torch.float32):
        return (torch.randn(*shape, device=DEV, generator=gen) * scale).to(dtype)

    def uniform(*shape):
        return torch.rand(*shape, device=DEV, generator=gen)

    def rows(count, width, **kw):   # rows of a wider activation where the case pads
        return normal(count, width + case["pad"], **kw)[:, :width]

    s = dict(case=case)
    if case["op"] == "router":
        E, k = case["experts"], case["top_k"]
        s |= dict(z=normal(n, E, scale=1.5, dtype=dt), bias=normal(E, scale=0.05) if case["bias"] else None, valid=None,
                  expert=torch.empty(n, k, dtype=torch.int32, device=DEV), weight=torch.empty(n, k, device=DEV))
        if case["mask"]:   # three experts in four valid; one row in a hundred has none
            bits = torch.randint(-2 ** 31, 2 ** 31, (2, n, (E + 31) // 32), device=DEV, generator=gen, dtype=torch.int64)
            bits = (bits[0] | bits[1]) & 0xffffffff
            bits[uniform(n) < 0.01] = 0
            s["valid"] = torch.where(bits >= 2 ** 31, bits - 2 ** 32, bits).to(torch.int32)
        if case["kind"] == "backward":
            s["expert"] = _plain_router(s)["expert"]     # of the forward pass
            s |= dict(dweight=normal(n, k, scale=1.0 / n), dz=torch.empty(n, E, dtype=dt, device=DEV))
        return s
    if case["op"] in ("dispatch", "combine"):
        E, k, d = case["experts"], case["top_k"], case["dim"]
        # experts are liked unequally; each row's are different ones
        like = normal(E, scale=0.7) - (-uniform(n, E).log()).log()
        expert = like.sort(dim=1, descending=True, stable=True).indices[:, :k].to(torch.int32).contiguous()
        expert[uniform(n, k) < case["drop"]] = -1
        s |= dict(expert=expert, offsets=torch.zeros(E + 1, dtype=torch.int32, device=DEV),
                  slot=torch.zeros(n, k, dtype=torch.int32, device=DEV))
        if case["op"] == "dispatch" and case["kind"] == "forward":
            return s | dict(x=rows(n, d, dtype=dt), xs=torch.zeros(n * k, d, dtype=dt, device=DEV))
        s["slot"] = _plain_plan(s)["slot"]
        if case["op"] == "dispatch":
            return s | dict(dxs=rows(n * k, d, scale=1.0 / n, dtype=dt), dx=torch.empty(n, d, dtype=dt, device=DEV))
        weight = uniform(n, k) + 0.05
        s |= dict(ys=rows(n * k, d, dtype=dt), weight=weight / weight.sum(1, keepdim=True))
        if case["kind"] == "forward":
            return s | dict(y=torch.empty(n, d, dtype=dt, device=DEV))
        return s | dict(dy=rows(n, d, scale=1.0 / n, dtype=dt), dys=torch.zeros(n * k, d, dtype=dt, device=DEV),
                        dweight=torch.empty(n, k, device=DEV))

    r = np.random.default_rng(int(seed))
    G, k, m = case["groups"], case["in_dim"], case["out_dim"]
    sizes = _sizes(n, G, r)
    s |= dict(most=int(sizes.max()),
              offsets=torch.from_numpy(np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)).to(DEV))
    W = normal(G, m, k, scale=1 / math.sqrt(k), dtype=dt)
    if case["op"] == "packed":
        codes, scale = _pack(W.reshape(G * m, k))
        return s | dict(x=rows(n, k, dtype=dt), W=codes.reshape(G, m, k), W_scale=scale.reshape(G, m),
                        b=normal(G, m, scale=0.1), codes=torch.empty(n, k, dtype=torch.int8, device=DEV),
                        scale=torch.empty(n, device=DEV), y=torch.empty(n, m, dtype=dt, device=DEV))
    x = normal(n, k, dtype=dt)
    if case["relu"]:
        x.relu_()
    codes, scale = _pack(x, keep=case["relu"])     # of the forward pass
    return s | dict(dy=rows(n, m, scale=1.0 / n, dtype=dt), x=codes, x_scale=scale, W=W,
                    dx=torch.empty(n, k, dtype=dt, device=DEV), dW=torch.empty(G, m, k, dtype=dt, device=DEV),
                    db=torch.empty(G, m, device=DEV))


# ---- plain forms --------------------------------------------------------------

def _valid(s, z):
    ok = z > -math.inf     # neither -infinity nor NaN
    if s["valid"] is not None:
        j = torch.arange(z.shape[1], device=DEV)
        ok &= ((s["valid"][:, j // 32] >> (j % 32)) & 1) != 0
    return ok


def _log_sigmoid(z):
    return z.clamp_max(0) - torch.log1p((-z.abs()).exp())


def _plain_router(s):
    c = s["case"]
    z = s["z"].double().clamp_max(LARGEST)
    ok = _valid(s, z)
    z = torch.where(ok, z, torch.full_like(z, -math.inf))
    # the choice is made in 64 bits: scores lie close to one another
    if c["score"] == "sigmoid":
        score = 1 / (1 + (-z).exp())
    else:
        top = z.amax(1, keepdim=True).clamp_min(-LARGEST)
        e = (z - top).exp()
        score = e / e.sum(1, keepdim=True)
    key = z if s["bias"] is None else score + s["bias"].double()
    key = torch.where(ok, key, torch.full_like(key, -math.inf))
    if c["sets"] > 1:
        n, E = key.shape
        v = key if c["best"] == 1 or s["bias"] is not None else torch.where(ok, score, key)
        v = v.reshape(n, c["sets"], -1).sort(dim=2, descending=True).values[:, :, :c["best"]]
        v = torch.where(v[:, :, :1] > -math.inf, torch.where(v > -math.inf, v, torch.zeros_like(v)).sum(2, keepdim=True), v[:, :, :1])
        order = v[:, :, 0].sort(dim=1, descending=True, stable=True).indices[:, :c["top_sets"]]
        chosen = torch.zeros(n, c["sets"], dtype=torch.bool, device=DEV).scatter_(1, order, True)
        key = torch.where(chosen.repeat_interleave(E // c["sets"], dim=1), key, torch.full_like(key, -math.inf))
    best = key.sort(dim=1, descending=True, stable=True)
    expert, some = best.indices[:, :c["top_k"]], best.values[:, :c["top_k"]] > -math.inf
    zf = s["z"].float().clamp_max(LARGEST)
    zc = torch.where(some, zf.gather(1, expert), torch.full_like(zf[:, :1], -math.inf))
    if c["renorm"]:
        v = _log_sigmoid(zc) if c["score"] == "sigmoid" else zc
        e = torch.where(some, (v - v.amax(1, keepdim=True)).exp(), torch.zeros_like(v))
        w = e / e.sum(1, keepdim=True)
    elif c["score"] == "sigmoid":
        w = 1 / (1 + (-zc).exp())
    else:
        zf = torch.where(ok, zf, torch.full_like(zf, -math.inf))
        top = zf.amax(1, keepdim=True)
        w = (zc - top).exp() / (zf - top).exp().sum(1, keepdim=True)
    w = torch.where(some, w, torch.zeros_like(w))
    return dict(expert=torch.where(some, expert, torch.full_like(expert, -1)).to(torch.int32), weight=w)


def _plain_router_backward(s):
    c = s["case"]
    z = s["z"].float().clamp_max(LARGEST)
    some = s["expert"] >= 0
    at = s["expert"].long().clamp_min(0)
    zero = torch.zeros_like(s["dweight"])
    dw = torch.where(some, s["dweight"], zero)
    zc = torch.where(some, z.gather(1, at), torch.full_like(zero, -math.inf))
    dz = torch.zeros_like(z)
    if c["renorm"]:
        v = _log_sigmoid(zc) if c["score"] == "sigmoid" else zc
        e = torch.where(some, (v - v.amax(1, keepdim=True)).exp(), zero)
        q = torch.where(some, e / e.sum(1, keepdim=True), zero)
        d = q * (dw - (q * dw).sum(1, keepdim=True))
        if c["score"] == "sigmoid":
            d = torch.where(some, d / (1 + zc.exp()), zero)
    elif c["score"] == "sigmoid":
        p = 1 / (1 + (-zc).exp())
        d = torch.where(some, dw * p / (1 + zc.exp()), zero)
    else:
        ok = _valid(s, z)
        z = torch.where(ok, z, torch.full_like(z, -math.inf))
        e = torch.where(ok, (z - z.amax(1, keepdim=True)).exp(), torch.zeros_like(z))
        p = torch.where(ok, e / e.sum(1, keepdim=True), torch.zeros_like(z))
        pc = torch.where(some, p.gather(1, at), zero)
        dz = -p * (pc * dw).sum(1, keepdim=True)
        d = pc * dw
    dz.scatter_add_(1, at, d)
    return dict(dz=dz.to(s["z"].dtype))


def _plain_plan(s):
    E = s["case"]["experts"]
    pair = s["expert"].reshape(-1).long()
    pair = torch.where(pair < 0, torch.full_like(pair, E), pair)
    order = pair.sort(stable=True).indices
    slot = torch.empty_like(pair)
    slot[order] = torch.arange(pair.numel(), device=DEV)
    slot[pair == E] = -1
    offsets = torch.searchsorted(pair[order], torch.arange(E + 1, device=DEV))
    return dict(offsets=offsets.to(torch.int32), slot=slot.to(torch.int32).reshape(s["expert"].shape))


def _taken(rows, slot):
    """Rows at the slots [n, k, dim], zero where there is none."""
    return torch.where(slot[:, :, None] >= 0, rows[slot.long().clamp_min(0)].float(), torch.zeros((), device=DEV))


def _plain_exchange(s):
    c = s["case"]
    if c["op"] == "dispatch" and c["kind"] == "forward":
        out = _plain_plan(s)
        i, j = torch.nonzero(out["slot"] >= 0, as_tuple=True)
        s["xs"][out["slot"][i, j].long()] = s["x"][i]
        return out | dict(xs=s["xs"])
    if c["op"] == "dispatch":
        return dict(dx=_taken(s["dxs"], s["slot"]).sum(1).to(s["dx"].dtype))
    if c["kind"] == "forward":
        return dict(y=(_taken(s["ys"], s["slot"]) * s["weight"][:, :, None]).sum(1).to(s["y"].dtype))
    i, j = torch.nonzero(s["slot"] >= 0, as_tuple=True)
    s["dys"][s["slot"][i, j].long()] = (s["dy"][i].float() * s["weight"][i, j][:, None]).to(s["dys"].dtype)
    return dict(dys=s["dys"], dweight=(_taken(s["ys"], s["slot"]) * s["dy"].float()[:, None, :]).sum(2))


def _pack(x, keep=False):
    """Codes in [-127, 127] and a scale for each row; `keep`: only zeros get the code 0."""
    x = x.float()
    scale = (x.abs().amax(1) / 127).clamp_min(2.0 ** -126)
    q = (x * (1 / scale)[:, None]).round().clamp(-127, 127)
    if keep:
        q = torch.where(q == 0, x.sign(), q)
    return q.to(torch.int8), scale


def _places(s, n):
    """Group of each row and its place in the group."""
    rows = torch.arange(n, device=DEV)
    g = torch.searchsorted(s["offsets"][1:].long().contiguous(), rows, right=True)
    return g, rows - s["offsets"].long()[g]


def _padded(x, g, at, s):
    out = torch.zeros(s["case"]["groups"], s["most"], x.shape[1], device=DEV)
    out[g, at] = x.float()
    return out


def _plain_layer(s):
    c = s["case"]
    g, at = _places(s, c["rows"])
    W = s["W"].float()
    if c["op"] == "packed":
        q, scale = _pack(s["x"])
        # sums of whole numbers: past 2^24 they need 64 bits
        x, W = _padded(q, g, at, s), W.transpose(1, 2).contiguous()
        step = 1024
        y = sum(torch.bmm(x[:, :, i:i + step].contiguous(), W[:, i:i + step].contiguous()).double()
                for i in range(0, W.shape[1], step))[g, at].float()
        y = y * scale[:, None] * s["W_scale"][g] + s["b"][g]
        return dict(y=(y.clamp_min(0) if c["relu"] else y).to(s["y"].dtype))
    x, dy = _padded(s["x"].float() * s["x_scale"][:, None], g, at, s), _padded(s["dy"], g, at, s)
    dx = torch.bmm(dy, W)[g, at]
    if c["relu"]:
        dx = dx * (s["x"] > 0)
    dW = torch.bmm(dy.transpose(1, 2).contiguous(), x)
    return dict(dx=dx.to(s["dx"].dtype), dW=dW.to(s["dW"].dtype), db=dy.sum(1))


# ---- one pass -------------------------------------------------------------------

def _own(s):
    import paper_2606_11440_amd as im
    c = s["case"]
    if c["op"] == "router":
        if c["kind"] == "backward":
            im.im_router_backward(s["z"], s["expert"], s["dweight"], s["dz"], valid=s["valid"], score=c["score"],
                                  renorm=c["renorm"])
            return dict(dz=s["dz"])
        im.im_router_forward(s["z"], s["expert"], s["weight"], bias=s["bias"], valid=s["valid"], score=c["score"],
                             renorm=c["renorm"], n_sets=c["sets"], top_sets=c["top_sets"], set_best=c["best"])
        return dict(expert=s["expert"], weight=s["weight"])
    if c["op"] == "dispatch":
        if c["kind"] == "backward":
            im.im_dispatch_backward(s["dxs"], s["slot"], s["dx"])
            return dict(dx=s["dx"])
        im.im_dispatch_plan(s["expert"], s["offsets"], s["slot"])
        im.im_dispatch_forward(s["x"], s["slot"], s["xs"])
        return dict(offsets=s["offsets"], slot=s["slot"], xs=s["xs"])
    if c["op"] == "combine":
        if c["kind"] == "backward":
            im.im_combine_backward(s["dy"], s["ys"], s["slot"], s["weight"], s["dys"], s["dweight"])
            return dict(dys=s["dys"], dweight=s["dweight"])
        im.im_combine_forward(s["ys"], s["slot"], s["weight"], s["y"])
        return dict(y=s["y"])
    if c["op"] == "packed":
        im.im_rows_pack(s["x"], s["codes"], s["scale"])
        im.im_linear_forward_packed(s["codes"], s["scale"], s["W"], s["W_scale"], s["b"], s["y"], offsets=s["offsets"],
                                    relu=c["relu"])
        return dict(y=s["y"])
    im.im_linear_backward_packed(s["dy"], s["x"], s["x_scale"], s["W"], s["dx"], s["dW"], s["db"], offsets=s["offsets"],
                                 relu_in=c["relu"])
    return dict(dx=s["dx"], dW=s["dW"], db=s["db"])


def run(state):
    if own:
        return _own(state)
    c = state["case"]
    if c["op"] == "router":
        return _plain_router(state) if c["kind"] == "forward" else _plain_router_backward(state)
    return _plain_exchange(state) if c["op"] in ("dispatch", "combine") else _plain_layer(state)


# ---- 64 bits ----------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "router":
        return _exact_router(s)
    if case["op"] in ("dispatch", "combine"):
        return _exact_exchange(s)
    off = s["offsets"].tolist()
    parts = [slice(a, b) for a, b in zip(off, off[1:])]
    if case["op"] == "packed":
        q, scale = _codes(s["x"])
        W = s["W"].double()
        y = torch.cat([(q[r] @ W[g].T) * scale[r, None] * s["W_scale"][g].double() + s["b"][g].double()
                       for g, r in enumerate(parts)])
        return dict(y=torch.relu(y) if case["relu"] else y)
    x, dy, W = s["x"].double() * s["x_scale"].double()[:, None], s["dy"].double(), s["W"].double()
    dx = torch.cat([dy[r] @ W[g] for g, r in enumerate(parts)])
    if case["relu"]:
        dx[s["x"] <= 0] = 0
    return dict(dx=dx, dW=torch.stack([dy[r].T @ x[r] for r in parts]), db=torch.stack([dy[r].sum(0) for r in parts]))


def _codes(x):
    """Codes and scales as they are defined: by operations in 32 bits, each rounded once."""
    codes, scales = [], []
    for part in x.split(1 << 15):
        a = part.float().cpu().numpy()
        scale = np.maximum(np.abs(a).max(1) / np.float32(127), np.float32(2.0 ** -126))
        a = np.rint(a * (np.float32(1) / scale)[:, None])
        codes.append(torch.from_numpy(np.clip(a, -127, 127)).to(DEV).double())
        scales.append(torch.from_numpy(scale).to(DEV).double())
    return torch.cat(codes), torch.cat(scales)


def _exact_router(s):
    c = s["case"]
    z = s["z"].double()
    n, E = z.shape
    if s["valid"] is not None:
        words = s["valid"].cpu().numpy().view(np.uint8)
        ok = np.unpackbits(words.reshape(n, -1), axis=1, bitorder="little")[:, :E]
        z[torch.from_numpy(ok == 0).to(DEV)] = -math.inf
    ok = z > -math.inf
    none = torch.full_like(z, -math.inf)
    if c["score"] == "sigmoid":
        score = torch.sigmoid(z)
    else:
        score = torch.softmax(torch.where(ok.any(1, keepdim=True), z, torch.zeros_like(z)), 1) * ok
    rows = torch.arange(n, device=DEV)
    if c["kind"] == "forward":
        key = torch.where(ok, z if s["bias"] is None else score + s["bias"].double(), none)
        if c["sets"] > 1:
            each = E // c["sets"]
            by = key if s["bias"] is not None or c["best"] == 1 else torch.where(ok, score, none)
            value = torch.empty(n, c["sets"], dtype=torch.float64, device=DEV)
            for g in range(c["sets"]):
                part = by[:, g * each:(g + 1) * each].clone()
                value[:, g], at = part.max(1)
                if c["best"] == 2 and each > 1:
                    part[rows, at] = -math.inf
                    second = part.max(1).values
                    value[:, g] += torch.where(second > -math.inf, second, torch.zeros_like(second))
            kept = torch.zeros(n, c["sets"], dtype=torch.bool, device=DEV)
            for _ in range(c["top_sets"]):
                kept[rows, _first_best(value)] = True
                value[kept] = -math.inf
            key = torch.where(kept[:, torch.arange(E, device=DEV) // each], key, none)
        expert = torch.empty(n, c["top_k"], dtype=torch.int64, device=DEV)
        for j in range(c["top_k"]):
            at = _first_best(key)
            expert[:, j] = torch.where(key[rows, at] > -math.inf, at, torch.full_like(at, -1))
            key[rows, at] = -math.inf
    else:
        expert = s["expert"].long()
    some = expert >= 0
    w = score.gather(1, expert.clamp_min(0)) * some
    total = w.sum(1, keepdim=True)
    total = torch.where(total > 0, total, torch.ones_like(total)) if c["renorm"] else torch.ones_like(total)
    if c["kind"] == "forward":
        return dict(expert=expert.to(torch.int32), weight=w / total)
    dw = s["dweight"].double() * some
    ds = dw / total
    if c["renorm"]:
        ds = ds - (w / total * dw).sum(1, keepdim=True) / total
    full = torch.zeros_like(z)
    for j in range(expert.shape[1]):
        full[rows, expert[:, j].clamp_min(0)] += ds[:, j] * some[:, j]
    if c["score"] == "sigmoid":
        return dict(dz=full * score * (1 - score))
    return dict(dz=score * (full - (score * full).sum(1, keepdim=True)))


def _first_best(v):
    """The lowest index of each row's largest value."""
    at = torch.arange(v.shape[1], device=DEV).expand_as(v)
    return torch.where(v == v.amax(1, keepdim=True), at, torch.full_like(at, v.shape[1] - 1)).amin(1)


def _exact_exchange(s):
    c = s["case"]
    if c["op"] == "dispatch" and c["kind"] == "forward":
        pair = s["expert"].reshape(-1).cpu().numpy()
        places = [np.flatnonzero(pair == e) for e in range(c["experts"])]
        offsets = np.concatenate([[0], np.cumsum([len(p) for p in places])]).astype(np.int32)
        order = np.concatenate(places)
        slot = np.full(pair.size, -1, np.int32)
        slot[order] = np.arange(order.size, dtype=np.int32)
        xs = torch.zeros(s["xs"].shape, dtype=torch.float64, device=DEV)
        xs[:order.size] = s["x"].double()[torch.from_numpy(order // c["top_k"]).to(DEV)]
        return dict(offsets=torch.from_numpy(offsets).to(DEV), slot=torch.from_numpy(slot.reshape(s["expert"].shape)).to(DEV),
                    xs=xs)
    n, k = s["slot"].shape
    if c["op"] == "dispatch" or c["kind"] == "forward":
        rows, out = (s["dxs"], "dx") if c["op"] == "dispatch" else (s["ys"], "y")
        total = torch.zeros(n, c["dim"], dtype=torch.float64, device=DEV)
        for j in range(k):
            i = torch.nonzero(s["slot"][:, j] >= 0)[:, 0]
            w = 1.0 if c["op"] == "dispatch" else s["weight"][i, j].double()[:, None]
            total[i] += rows[s["slot"][i, j].long()].double() * w
        return {out: total}
    dy, dys = s["dy"].double(), torch.zeros(s["dys"].shape, dtype=torch.float64, device=DEV)
    dweight = torch.zeros(n, k, dtype=torch.float64, device=DEV)
    for j in range(k):
        i = torch.nonzero(s["slot"][:, j] >= 0)[:, 0]
        at = s["slot"][i, j].long()
        dys[at] = dy[i] * s["weight"][i, j].double()[:, None]
        dweight[i, j] = (dy[i] * s["ys"][at].double()).sum(1)
    return dict(dys=dys, dweight=dweight)
