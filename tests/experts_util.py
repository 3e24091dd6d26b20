"""The operators around experts and of rows in 8 bits, in 64 bits from their
formulas, on the CPU, and bounds on how far a kernel may be from them.

Bounds count roundings. An exponential of d <= 0 is taken of a difference that is
rounded (|d| 2^-24) and off by 2 units more: (|d| + 4) 2^-23 of itself at most, and
2^-120 where it leaves the range of normal numbers. Sums of K positive terms add
K 2^-24, a division or product 2^-24."""

import numpy as np
import torch

U = 2.0 ** -24
ROUND = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float64: 0.0}
BIG = 3.4028234663852886e38


def words(ok):
    """Mask words int32 [n, ceil(E / 32)] of a bool array [n, E]."""
    n, E = ok.shape
    pad = np.zeros((n, (E + 31) // 32 * 32), dtype=bool)
    pad[:, :E] = ok
    return torch.from_numpy(np.packbits(pad, axis=1, bitorder="little").view(np.int32).reshape(n, -1).copy())


class Router:
    """64-bit router of logits z (a CPU tensor) and a bool mask (or None)."""

    def __init__(self, z, score, ok=None):
        with np.errstate(all="ignore"):
            self.dtype = z.dtype
            z = z.double().numpy().copy()
            self.n, self.E = z.shape
            self.ok = np.ones(z.shape, bool) if ok is None else ok.copy()
            self.ok &= z > -np.inf
            z = np.minimum(z, BIG)
            z[~self.ok] = -np.inf
            self.z, self.score = z, score
            if score == "sigmoid":
                self.s = np.where(z >= 0, 1 / (1 + np.exp(-np.abs(z))), np.exp(-np.abs(z)) / (1 + np.exp(-np.abs(z))))
            else:
                top = z.max(1, keepdims=True)
                top[np.isneginf(top)] = 0
                e = np.exp(z - top)
                total = e.sum(1, keepdims=True)
                self.s = e / np.where(total > 0, total, 1)
            self.s[~self.ok] = 0

    def choose(self, k, bias=None, sets=1, top_sets=1, best=1):
        with np.errstate(all="ignore"):
            key = self.z.copy() if bias is None else self.s + bias.double().numpy()[None]
            key[~self.ok | ~(key > -np.inf)] = -np.inf
            if sets > 1:
                by = key if bias is not None or best == 1 else np.where(self.ok, self.s, -np.inf)
                v = -np.sort(-by.reshape(self.n, sets, -1), axis=2)
                value = v[:, :, 0].copy()
                if best == 2 and v.shape[2] > 1:
                    value += np.where(v[:, :, 1] > -np.inf, v[:, :, 1], 0)
                order = np.argsort(-value, axis=1, kind="stable")[:, :top_sets]
                keep = np.zeros((self.n, sets), bool)
                np.put_along_axis(keep, order, True, 1)
                key[~np.repeat(keep, self.E // sets, axis=1)] = -np.inf
            order = np.argsort(-key, axis=1, kind="stable")[:, :k]
            return np.where(np.take_along_axis(key, order, 1) > -np.inf, order, -1)

    def _shares(self, expert, renorm):
        """Scores of the chosen, their shares q of the sum (or the scores), and the distances that their
        exponentials were taken of."""
        some = expert >= 0
        at = np.where(some, expert, 0)
        with np.errstate(all="ignore"):
            zc = np.where(some, np.take_along_axis(self.z, at, 1), -np.inf)
            s = np.where(some, np.take_along_axis(self.s, at, 1), 0)
            if renorm:   # in logarithms: shares of scores too small for a float
                v = np.minimum(zc, 0) - np.log1p(np.exp(-np.abs(zc))) if self.score == "sigmoid" else zc
                m = v.max(1, keepdims=True)
                m[np.isneginf(m)] = 0
                e = np.where(some, np.exp(v - m), 0)
                total = e.sum(1, keepdims=True)
                q = e / np.where(total > 0, total, 1)
                top = zc.max(1, keepdims=True)
            else:
                q = s
                top = self.z.max(1, keepdims=True)
            d = np.where(some, np.abs(zc - np.where(np.isneginf(top), 0, top)), 0)
            if self.score == "sigmoid":
                d = np.maximum(d, np.where(some, np.abs(zc), 0))
        return some, zc, q, np.minimum(d, 110)

    def weights(self, expert, renorm, scale=1.0):
        some, _, q, d = self._shares(expert, renorm)
        tol = abs(scale) * (q * (d + 2 * expert.shape[1] + 48) * 2.0 ** -23 + 2.0 ** -120)
        return torch.from_numpy(scale * q), torch.from_numpy(tol)

    def grad(self, expert, dw, renorm, scale=1.0):
        some, zc, q, d = self._shares(expert, renorm)
        k = expert.shape[1]
        dw = np.where(some, dw.double().numpy(), 0)
        dz, tol = np.zeros_like(self.z), np.zeros_like(self.z)
        far = (d + 2 * k + 64) * 2.0 ** -22
        dot, size = (q * dw).sum(1, keepdims=True), (q * np.abs(dw)).sum(1, keepdims=True)
        with np.errstate(all="ignore"):
            if renorm:
                g, t = q * (dw - dot), q * (np.abs(dw) + size) * far
            elif self.score == "softmax":
                g, t = q * dw, q * np.abs(dw) * far
                dz = -self.s * dot
                dist = np.minimum(np.abs(self.z - self.z.max(1, keepdims=True)), 110)
                tol = np.where(self.ok, self.s * size * (dist + 2 * k + 64) * 2.0 ** -22 + size * 2.0 ** -120, 0)
            else:
                g, t = q * dw, q * np.abs(dw) * far
            if self.score == "sigmoid":
                e = np.exp(-np.abs(zc))
                rest = np.where(zc < 0, 1 / (1 + e), e / (1 + e))
                g, t = g * rest, t * rest
            t = t + np.where(some, (np.abs(dw) + size) * 2.0 ** -120, 0)
        for c in range(k):
            rows = np.nonzero(some[:, c])[0]
            dz[rows, expert[rows, c]] += g[rows, c]
            tol[rows, expert[rows, c]] += t[rows, c]
        dz, tol = scale * dz, abs(scale) * tol
        return torch.from_numpy(dz), torch.from_numpy(tol + ROUND[self.dtype] * np.abs(dz) + 2.0 ** -130)


def plan(expert, E):
    """offsets and slot of a CPU tensor of experts."""
    pair = expert.reshape(-1).numpy()
    places = [np.flatnonzero(pair == e) for e in range(E)]
    offsets = np.concatenate([[0], np.cumsum([len(p) for p in places])]).astype(np.int32)
    order = np.concatenate(places)
    slot = np.full(pair.size, -1, np.int32)
    slot[order] = np.arange(order.size, dtype=np.int32)
    return torch.from_numpy(offsets), torch.from_numpy(slot.reshape(expert.shape))


def pack(x, keep=False):
    """Codes and scales, as they are defined: operations in 32 bits, each rounded once."""
    a = x.float().cpu().numpy()
    with np.errstate(all="ignore"):
        top = np.abs(a).max(1)
        scale = np.maximum(top / np.float32(127), np.float32(2.0 ** -126)).astype(np.float32)
        q = np.rint(a * (np.float32(1) / scale)[:, None])
        if keep:
            q = np.where((q == 0) & (a != 0), np.sign(a), q)
        bad = ~np.isfinite(a).all(1)
        q[bad] = 0
        scale[bad] = np.nan
    return torch.from_numpy(q.astype(np.int8)), torch.from_numpy(scale)


def packed_linear(q, sx, W, sw, b, offsets, relu, dtype):
    """y and its bound: the sum is exact, its conversion and two products are rounded."""
    n, (G, m, k) = q.shape[0], W.shape
    off = [0, n] if offsets is None else list(offsets)
    y = torch.zeros(n, m, dtype=torch.float64)
    size = torch.zeros_like(y)
    Q, Wd = q.cpu().double(), W.cpu().double()
    for g in range(G):
        r = slice(off[g], off[g + 1])
        p = (Q[r] @ Wd[g].T) * sx.cpu().double()[r, None] * sw.cpu().double()[g]
        c = 0 if b is None else b[g].cpu().double()
        y[r], size[r] = p + c, p.abs() + (0 if b is None else c.abs())
    tol = 4 * U * size + ROUND[dtype] * y.abs() + 2.0 ** -140
    return (torch.where(y < 0, torch.zeros_like(y), y) if relu else y), tol


def same_or_close(got, want, tol, what):
    got, want, tol = got.double().cpu(), want.double().cpu(), tol.double().cpu()
    assert got.shape == want.shape, what
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    over = (got - want).abs() - tol
    over[same] = 0
    bad = ~(over <= 0)
    assert not bad.any(), (what, int(bad.sum()), torch.nonzero(bad)[:4].tolist(), got[bad][:4].tolist(),
                           want[bad][:4].tolist(), tol[bad][:4].tolist())
