"""GPU: the softmax head on biases of any magnitude, as users mask classes with.

Bounds are learn_util's with one difference: what a row's bound takes from its
classes it takes from those with a share of 2^-60 or more. A class below that
adds less than V 2^-60 (|ln p| + 1) |ln p| <= 2^-30 to no statistic, whatever
the rounding of its own logit, so that a bias of -1e38 loosens nothing but the
log-probability of its own class."""
import math

import pytest

import learn_util as U
from gpu_util import need_gpu, note
from test_gpu_learn_head import make, run_backward, run_forward

pytestmark = pytest.mark.gpu
F32, BF16 = "float32", "bfloat16"
LEAST_SHARE = 2.0 ** -60
LARGEST = 3.4028234e38      # rounds to the largest fp32


class Head(U.Head):
    def __init__(self, h, W, b, valid, target, offsets, top=None):
        """top: a class whose share is 1 and whose logit is its bias, since its
        products vanish in the sum's rounding: nothing of that rounding enters."""
        import torch
        super().__init__(h, W, b, valid, target, offsets)
        ez = torch.zeros_like(self.p)
        for g, r in enumerate(self.spans):
            ez[r] = U.gamma(self.d) * (self.h[r].abs() @ self.W[g].abs().T) + U.U * b[g].double().cpu().abs()
        seen = self.p >= LEAST_SHARE
        zero = torch.zeros_like(self.p)
        far = torch.where(seen, self.lnp.abs(), zero).amax(1) + math.log(self.V + 1)
        base = torch.where(self.lse == -math.inf, torch.zeros_like(self.lse), self.lse)
        self.share = (far + 4) * 2.0 ** -22
        own = ez[torch.arange(self.n), self.y.clamp_min(0)]
        if top is None:
            self.share += 2 * torch.where(seen, ez, zero).amax(1) + 4 * U.U * base.abs()
        else:   # another class's log-probability keeps the two logits' roundings
            own = torch.where(self.y == top, 0, own + ez[:, top])
        self.e_logp = 2 * self.share + 2 * own + 4 * U.U * self.logp.nan_to_num(0, 0, 0).abs()
        self.e_lse = 2 * self.share + 4 * U.U * base.abs()
        self.e_H = 2 * self.share * (self.H.abs() + 2) + 2.0 ** -21 * (1 + math.log(self.V + 1))


def check(c, ent=True, top=None):
    torch = c["torch"]
    o = run_forward(c)
    assert o["error"] == 0
    r = Head(c["h"], c["W"], c["b"], c["valid"], c["target"], c["off"], top)
    assert float(torch.cat([r.share, r.e_lse - 4 * U.U * r.lse.abs(), r.e_H]).max()) < 0.1   # they bound something
    U.close(o["logp"], r.logp, r.e_logp, "logp")
    U.close(o["lse"], r.lse, r.e_lse, "lse")
    U.close(o["entropy"], r.H, r.e_H, "entropy")
    q = run_backward(c, o, relu_in=True, ent=ent)
    for k, (want, tol) in zip(("dh", "dW", "db"), r.grads(c["dlogp"], c["dent"] if ent else None, True)):
        U.close(q[k], want, tol, k)


# the last: tiles of 256 classes, of which some see masked classes only
HEADS = [(15, 32, BF16), (15, 32, F32), (64, 96, BF16), (130, 40, BF16), (1000, 32, BF16), (1000, 32, F32), (4100, 24, BF16)]
# what a lane's four classes, a lane's run of joined ones, a wave's columns and a tile of classes see
MASKED = {"four": lambda V: slice(4, 8), "most": lambda V: slice(1, V), "half": lambda V: slice(0, V // 2),
          "tile": lambda V: slice(V // 256 // 2 * 256, V // 256 // 2 * 256 + min(256, V - 5)), "odd": lambda V: slice(1, V, 2)}


@pytest.mark.parametrize("far", [1e20, 1e30, 1e35, 1e36, 1e37, 1e38, 2e38, LARGEST])
@pytest.mark.parametrize("which", list(MASKED))
@pytest.mark.parametrize("V,d,dtype", HEADS)
def test_classes_far_below_the_others(V, d, dtype, which, far):
    note(f"[far below] V={V} d={d} {dtype} {which} {far}")
    c = make(150, d, V, None, dtype, seed=V, mask=False)
    masked = c["torch"].zeros(V, dtype=c["torch"].bool, device="cuda")
    masked[MASKED[which](V)] = True
    c["b"][0, masked] = -far
    free = c["torch"].nonzero(~masked)[:, 0].int()
    y = c["target"]
    c["target"] = c["torch"].where(y >= 0, free[y.clamp_min(0).long() % len(free)], y)
    check(c)


@pytest.mark.parametrize("far", [1e8, 1e20, 1e37, 1e38, 2e38, LARGEST])
@pytest.mark.parametrize("V,d,dtype", HEADS)
def test_a_class_far_above_the_others(V, d, dtype, far):
    """Its share is 1 in every row, and what it takes from the others is exactly dlogp."""
    note(f"[far above] V={V} d={d} {dtype} {far}")
    c = make(100, d, V, None, dtype, seed=V + 1, mask=False)
    c["b"][0, 9] = far
    c["W"][0, 9] *= 0.25
    c["target"][:40] = 9
    product = c["h"].double() @ c["W"][0, 9].double()
    assert float(product.abs().max()) < 2 and float(product.abs().min()) > 0   # the spacing of floats at 1e8 is 8
    check(c, top=9)


@pytest.mark.parametrize("far", [1e35, 1e38, 2.3e38, 2.5e38, LARGEST])
@pytest.mark.parametrize("V,d,dtype", HEADS)
def test_targets_far_below(V, d, dtype, far):
    """A class that its bias masks is valid as long as its logit is finite: its
    log-probability is about -far, and dlogp goes through it whole."""
    note(f"[targets far below] V={V} d={d} {dtype} {far}")
    c = make(120, d, V, None, dtype, seed=V + 2, mask=False)
    c["b"][0, 2::3] = -far
    c["target"][::2] = 5
    check(c)


@pytest.mark.parametrize("far", [2e30, 1e38, 2.3e38, 2.5e38, LARGEST])
@pytest.mark.parametrize("V,d,dtype", HEADS)
def test_rows_with_masked_classes_only(V, d, dtype, far):
    """Rows whose valid classes all have the bias -far: with no products they are
    equally likely. lse cannot hold that, so those rows have no gradient."""
    note(f"[masked rows] V={V} d={d} {dtype} {far}")
    c = make(120, d, V, None, dtype, seed=V + 3, mask=False)
    torch = c["torch"]
    masked = torch.zeros(V, dtype=torch.bool, device="cuda")
    masked[2::3] = True
    c["b"][0, masked] = -far
    y = c["target"]
    c["target"] = torch.where((y >= 0) & masked[y.clamp_min(0).long()], 0, y)
    rows = torch.zeros(120, dtype=torch.bool, device="cuda")
    rows[::4] = True
    c["h"][rows] = 0
    c["target"][rows] = 5
    bits = torch.ones(120, (V + 31) // 32 * 32, dtype=torch.bool, device="cuda")
    bits[:, :V][rows] = masked
    w = (bits.view(120, -1, 32).long() << torch.arange(32, device="cuda")).sum(2)
    c["valid"] = torch.where(w >= 2 ** 31, w - 2 ** 32, w).to(torch.int32)
    o, k = run_forward(c), int(masked.sum())
    assert o["error"] == 0
    fit = 2.0 ** -21 * (1 + math.log(k))
    assert float((o["logp"][rows].double() + math.log(k)).abs().max()) <= fit
    assert float((o["entropy"][rows].double() - math.log(k)).abs().max()) <= fit
    assert float((o["lse"][rows].double() + far).abs().max()) <= 2 * U.U * far
    # the others are as they are without those rows
    some = dict(c, **{key: c[key][~rows] for key in ("h", "target", "valid", "dlogp", "dent")})
    check(some)
    a = run_backward(c, o, relu_in=False)
    assert bool((a["dh"][rows] == 0).all())
    want = Head(some["h"], some["W"], some["b"], some["valid"], some["target"], None)
    for key, (ref, tol) in zip(("dh", "dW", "db"), want.grads(some["dlogp"], some["dent"], False)):
        U.close(a[key][~rows] if key == "dh" else a[key], ref, tol, key)


@pytest.mark.parametrize("V,d,dtype", HEADS)
def test_biases_from_end_to_end(V, d, dtype):
    """The largest and the lowest float in one row: their difference is no float."""
    note(f"[end to end] V={V} d={d} {dtype}")
    c = make(100, d, V, None, dtype, seed=V + 4, mask=False)
    c["b"][0, 3] = LARGEST
    c["b"][0, 4:11] = -LARGEST
    c["target"][:50] = 3
    c["target"][50:] = 6
    o = run_forward(c)
    q = run_backward(c, o, relu_in=False)
    assert bool((o["logp"][:50] == 0).all()) and bool(o["logp"][50:].isneginf().all()) and bool((o["entropy"] == 0).all())
    # dz of rows 50..: dlogp at class 6, -dlogp at class 3
    want = c["dlogp"][50:].double().sum()
    tol = 2 * U.gamma(100) * float(c["dlogp"].double().abs().sum())
    assert abs(float(q["db"][0, 6] - want)) <= tol and abs(float(q["db"][0, 3] + want)) <= tol
    assert not bool(q["dh"].isnan().any()) and not bool(q["dW"].isnan().any())
