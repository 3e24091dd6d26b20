"""The learner's operators in 64 bits, written from their formulas with plain
torch operations, and bounds on how far a kernel may be from them.

Bounds count roundings. A sum of K products in fp32 is off by at most
2 (K + 8) 2^-24 sum |a b| (twice the bound of a sum in any order, since the
matrix cores' inner additions are not specified to round to nearest); a result
in bf16 by 2^-8 of itself more."""
import math

import torch

U = 2.0 ** -24
ROUND = {torch.float32: U, torch.bfloat16: 2.0 ** -8}


def gamma(k):
    return 2 * (k + 8) * U


def spans(offsets, n):
    """Row ranges of the groups (offsets a list, or None: one group)."""
    off = [0, n] if offsets is None else list(offsets)
    return [slice(a, b) for a, b in zip(off, off[1:])]


def close(got, want, tol, what):
    got, want, tol = got.double().cpu(), want.double().cpu(), tol.double().cpu()
    assert got.shape == want.shape, what
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    over = (got - want).abs() - tol
    over[same] = 0
    bad = ~(over <= 0)
    assert not bad.any(), (what, int(bad.sum()), got[bad][:4].tolist(), want[bad][:4].tolist(), tol[bad][:4].tolist())


def linear(x, W, b, offsets, relu):
    """y and its bound, rows of no group zero."""
    n, (G, m, k) = x.shape[0], W.shape
    X, Wd = x.double(), W.double()
    y = torch.zeros(n, m, dtype=torch.float64, device=x.device)
    size = torch.zeros_like(y)
    for g, r in enumerate(spans(offsets, n)):
        y[r] = X[r] @ Wd[g].T + (0 if b is None else b[g].double())
        size[r] = X[r].abs() @ Wd[g].abs().T + (0 if b is None else b[g].double().abs())
    tol = gamma(k) * size + ROUND[x.dtype] * y.abs()
    return (y.clamp_min(0) if relu else y), tol


def linear_grad(dy, x, W, offsets, relu_in):
    n, (G, m, k) = x.shape[0], W.shape
    X, Y, Wd = x.double(), dy.double(), W.double()
    dx, ex = torch.zeros_like(X), torch.zeros_like(X)
    dW, eW = torch.zeros_like(Wd), torch.zeros_like(Wd)
    db = torch.zeros(G, m, dtype=torch.float64, device=x.device)
    eb = torch.zeros_like(db)
    for g, r in enumerate(spans(offsets, n)):
        dx[r], ex[r] = Y[r] @ Wd[g], gamma(m) * (Y[r].abs() @ Wd[g].abs())
        dW[g], eW[g] = Y[r].T @ X[r], gamma(r.stop - r.start) * (Y[r].T.abs() @ X[r].abs())
        db[g], eb[g] = Y[r].sum(0), gamma(r.stop - r.start) * Y[r].abs().sum(0)
    if relu_in:
        dx = torch.where(X > 0, dx, torch.zeros_like(dx))
        ex = torch.where(X > 0, ex, torch.zeros_like(ex))
    R = ROUND[x.dtype]
    return (dx, ex + R * dx.abs()), (dW, eW + R * dW.abs()), (db, eb + U * db.abs())


def unpack(valid, n, V):
    if valid is None:
        return torch.ones(n, V, dtype=torch.bool)
    j = torch.arange(V)
    return ((valid.cpu().long()[:, j // 32] >> (j % 32)) & 1).bool()


class Head:
    """64-bit head: logits, statistics and gradients with their bounds.

    A logit is off by ez = gamma(dim) sum |h w| + |b| rounding. exp(z - top) is
    then off by a share of 2 ez + (|z - top| + 4) 2^-22 (the argument's product
    with log2 e is rounded once, the exponential to 1 unit), and so are p, ln p
    (absolutely) and the sums over the classes."""

    def __init__(self, h, W, b, valid, target, offsets):
        n, (G, V, d) = h.shape[0], W.shape
        self.h, self.W, self.n, self.G, self.V, self.d = h.double().cpu(), W.double().cpu(), n, G, V, d
        self.spans, self.dtype = spans(offsets, n), h.dtype
        z = torch.full((n, V), -math.inf, dtype=torch.float64)
        ez = torch.zeros(n, V, dtype=torch.float64)
        for g, r in enumerate(self.spans):
            z[r] = self.h[r] @ self.W[g].T + (0 if b is None else b[g].double().cpu())
            ez[r] = gamma(d) * (self.h[r].abs() @ self.W[g].abs().T) + (0 if b is None else U * b[g].double().cpu().abs())
        ok = unpack(valid, n, V)
        z[~ok] = -math.inf
        ok &= z != -math.inf
        self.ok, self.y = ok, target.cpu().long()
        self.lse = torch.logsumexp(z, 1)
        base = torch.where(self.lse == -math.inf, torch.zeros_like(self.lse), self.lse)
        self.lnp = torch.where(ok, z - base[:, None], torch.zeros_like(z))
        self.p = torch.where(ok, self.lnp.exp(), torch.zeros_like(z))
        self.H = -(self.p * self.lnp).sum(1)
        far = torch.where(ok, self.lnp.abs(), torch.zeros_like(z)).amax(1) + math.log(V + 1)
        e = torch.where(ok, ez, torch.zeros_like(ez)).nan_to_num(0, 0, 0).amax(1)
        self.share = 2 * e + (far + 4) * 2.0 ** -22 + 4 * U * base.abs()
        self.logp = torch.zeros(n, dtype=torch.float64)
        rows = torch.nonzero((self.y >= 0))[:, 0]
        rows = rows[self.lse[rows] != -math.inf]
        self.logp[rows] = torch.where(ok[rows, self.y[rows]], self.lnp[rows, self.y[rows]],
                                      torch.full((len(rows),), -math.inf, dtype=torch.float64))
        self.e_logp = 2 * self.share + 2 * U * self.logp.nan_to_num(0, 0, 0).abs()
        self.e_H = 2 * self.share * (self.H.abs() + 2) + 2.0 ** -21 * (1 + math.log(V + 1))

    def grads(self, dlogp, dent, relu_in):
        a = torch.where(self.y >= 0, dlogp.double().cpu(), torch.zeros(self.n, dtype=torch.float64))
        c = torch.zeros_like(a) if dent is None else dent.double().cpu()
        live = ((a != 0) | (c != 0)) & (self.lse != -math.inf)
        hit = torch.zeros_like(self.p)
        hit[torch.arange(self.n), self.y.clamp_min(0)] = 1.0
        dz = a[:, None] * (hit - self.p) - c[:, None] * self.p * (self.lnp + self.H[:, None])
        err = (a.abs()[:, None] * (self.p * 2 * self.share[:, None] + 2 * U) +
               c.abs()[:, None] * self.p * (4 * self.share[:, None] * (self.lnp.abs() + self.H[:, None] + 2)))
        off = ~(self.ok & live[:, None])
        dz[off] = 0
        err[off] = 0
        h = torch.where(live[:, None], self.h, torch.zeros_like(self.h))
        erd = err + ROUND[self.dtype] * dz.abs()     # as it enters the products
        dh, eh = torch.zeros_like(self.h), torch.zeros_like(self.h)
        dW, eW = torch.zeros_like(self.W), torch.zeros_like(self.W)
        db = torch.zeros(self.G, self.V, dtype=torch.float64)
        eb = torch.zeros_like(db)
        for g, r in enumerate(self.spans):
            k = r.stop - r.start
            dh[r] = dz[r] @ self.W[g]
            eh[r] = (erd[r] + gamma(self.V) * dz[r].abs()) @ self.W[g].abs()
            dW[g] = dz[r].T @ h[r]
            eW[g] = (erd[r] + gamma(k) * dz[r].abs()).T @ h[r].abs()
            db[g] = dz[r].sum(0)
            eb[g] = (err[r] + gamma(k) * dz[r].abs()).sum(0)
        R = ROUND[self.dtype]
        eh += R * dh.abs()
        if relu_in:
            dh[~(self.h > 0)] = 0
            eh[~(self.h > 0)] = 0
        self.dz = dz
        return (dh, eh), (dW, eW + R * dW.abs()), (db, eb + U * db.abs())
