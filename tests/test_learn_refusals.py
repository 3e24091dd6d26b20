"""The learner's C ABI on a machine without a GPU: exports, and every refusal
that is decided before a device is touched."""
import ctypes
import os
import re

import pytest

import paper_2606_11440_amd as P
from paper_2606_11440_amd import learn

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL = P._lib.IM_EINVAL
A = ctypes.c_void_p(4096)   # an aligned address that is never dereferenced


def L():
    return learn.load_learn()


def test_library_exports_every_declared_symbol():
    with open(os.path.join(ROOT, "include", "inframind_learn.h")) as f:
        names = set(re.findall(r"\b(im_[a-z_]+)\s*\(", f.read()))
    lib = ctypes.CDLL(learn.LEARN_PATH)
    assert not [n for n in names if not hasattr(lib, n)]
    assert names == set(P.LEARN_EXPORTED)


def linear_desc(**kw):
    d = learn.ImLinearDesc(1, 8, 16, 24, 1, 0, 0, 0, 16, 24, 16)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def head_desc(**kw):
    d = learn.ImHeadDesc(1, 8, 16, 24, 1, 0, 0, 0, 16, 16)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


BAD_LINEAR = [dict(n_groups=0), dict(n_groups=1025), dict(n_rows=-1), dict(n_rows=(1 << 30) + 1), dict(in_dim=0), dict(in_dim=65537),
              dict(out_dim=0), dict(out_dim=65537), dict(dtype=2), dict(relu=2), dict(relu_in=-1)]
BAD_HEAD = [dict(n_groups=0), dict(n_groups=1025), dict(n_rows=-1), dict(n_rows=(1 << 30) + 1), dict(dim=0), dict(dim=65537), dict(n_classes=0),
            dict(n_classes=(1 << 22) + 1), dict(dtype=-1), dict(relu_in=2)]


@pytest.mark.parametrize("over", BAD_LINEAR)
def test_bad_layers(over):
    d, out = linear_desc(**over), ctypes.c_int64(7)
    assert L().im_linear_workspace(ctypes.byref(d), 0, ctypes.byref(out)) == EINVAL and out.value == 7
    assert L().im_linear_forward(ctypes.byref(d), A, A, A, A, A, None, 0, None, None) == EINVAL
    assert L().im_linear_backward(ctypes.byref(d), A, A, A, A, A, A, A, A, 1 << 40, None, None) == EINVAL
    assert P.im_learn_last_error() != "no error"


@pytest.mark.parametrize("over", BAD_HEAD)
def test_bad_heads(over):
    d, out = head_desc(**over), ctypes.c_int64(7)
    assert L().im_head_workspace(ctypes.byref(d), 1, ctypes.byref(out)) == EINVAL and out.value == 7
    assert L().im_head_forward(ctypes.byref(d), A, A, A, A, None, A, A, A, A, A, 1 << 40, None, None) == EINVAL
    assert L().im_head_backward(ctypes.byref(d), A, A, A, A, None, A, A, A, A, A, A, A, A, A, 1 << 40, None,
                                None) == EINVAL


def test_layer_arguments():
    f = L().im_linear_forward
    d = linear_desc()
    R = ctypes.byref
    odd = ctypes.c_void_p(4097)
    for args in [(None, A, A, A, A, A, None, 0, None, None),
                 (R(d), None, None, A, A, A, None, 0, None, None), (R(d), None, A, None, A, A, None, 0, None, None),
                 (R(d), None, A, A, A, None, None, 0, None, None), (R(d), None, odd, A, A, A, None, 0, None, None),
                 (R(d), None, A, A, odd, A, None, 0, None, None), (R(d), odd, A, A, A, A, None, 0, None, None),
                 (R(linear_desc(n_groups=2)), None, A, A, A, A, None, 0, None, None),
                 (R(linear_desc(ld_x=15)), None, A, A, A, A, None, 0, None, None),
                 (R(linear_desc(ld_y=23)), None, A, A, A, A, None, 0, None, None),
                 (R(linear_desc(ld_x=(1 << 22) + 1)), None, A, A, A, A, None, 0, None, None)]:
        assert f(*args) == EINVAL
    b = L().im_linear_backward
    d = linear_desc(n_groups=3, n_rows=5000)
    need = ctypes.c_int64(0)
    assert L().im_linear_workspace(R(d), 1, R(need)) == 0 and need.value > 0
    assert L().im_linear_workspace(R(d), 2, R(need)) == EINVAL
    assert L().im_linear_workspace(R(d), 1, None) == EINVAL
    for args in [(R(d), A, A, A, A, A, A, A, None, 1 << 40, None, None),
                 (R(d), A, A, A, A, A, A, A, A, need.value - 1, None, None),
                 (R(d), A, A, A, A, A, A, A, ctypes.c_void_p(4096 + 128), 1 << 40, None, None),
                 (R(d), A, None, A, A, A, A, A, A, 1 << 40, None, None),
                 (R(d), A, A, None, A, A, A, A, A, 1 << 40, None, None),
                 (R(d), A, A, A, None, A, A, A, A, 1 << 40, None, None),
                 (R(linear_desc(n_groups=3, n_rows=5000, ld_dx=3)), A, A, A, A, A, A, A, A, 1 << 40, None, None)]:
        assert b(*args) == EINVAL
    # tiles beyond what a launch counts
    big = linear_desc(n_rows=2 ** 30, in_dim=65536, out_dim=65536, ld_x=65536, ld_y=65536)
    assert f(R(big), None, A, A, A, A, None, 0, None, None) == P._lib.IM_EUNSUPPORTED


@pytest.mark.parametrize("G,n,k,m", [(8, 16384, 4096, 16384), (2, 4096, 16384, 16384), (64, 64, 2048, 4096)])
def test_gradients_that_no_run_cuts_need_no_pieces(G, n, k, m):
    """As many tiles as fill the card: every group's sum is one block's, and the
    workspace is the groups' records (16 bytes each) alone."""
    need = ctypes.c_int64(0)
    d = linear_desc(n_groups=G, n_rows=n, in_dim=k, out_dim=m, ld_x=k, ld_y=m, ld_dx=k)
    assert L().im_linear_workspace(ctypes.byref(d), 1, ctypes.byref(need)) == 0
    assert 0 < need.value <= (16 * G + 255) // 256 * 256


def test_head_arguments():
    R = ctypes.byref
    d = head_desc()
    f = L().im_head_forward
    for args in [(R(d), None, None, A, A, None, A, A, A, A, A, 1 << 40, None, None),
                 (R(d), None, A, None, A, None, A, A, A, A, A, 1 << 40, None, None),
                 (R(d), None, A, A, A, None, None, A, A, A, A, 1 << 40, None, None),
                 (R(d), None, A, A, A, None, A, None, A, A, A, 1 << 40, None, None),
                 (R(head_desc(ld_h=15)), None, A, A, A, None, A, A, A, A, A, 1 << 40, None, None),
                 (R(head_desc(n_groups=2)), None, A, A, A, None, A, A, A, A, A, 1 << 40, None, None),
                 (R(head_desc(n_classes=5000)), None, A, A, A, None, A, A, A, A, None, 0, None, None)]:
        assert f(*args) == EINVAL
    b = L().im_head_backward
    need = ctypes.c_int64(0)
    assert L().im_head_workspace(R(d), 1, R(need)) == 0 and need.value > 0
    ok = [R(d), None, A, A, A, None, A, A, A, A, A, A, A, A, A, 1 << 40, None, None]
    for i in (2, 3, 6, 7, 9):                      # h, W, target, lse, dlogp
        assert b(*(ok[:i] + [None] + ok[i + 1:])) == EINVAL, i
    assert b(*(ok[:8] + [None] + ok[9:])) == EINVAL           # dentropy without entropy
    assert b(*(ok[:14] + [None] + ok[15:])) == EINVAL         # workspace
    assert b(*(ok[:15] + [need.value - 1] + ok[16:])) == EINVAL
    assert b(R(head_desc(ld_dh=2)), *ok[1:]) == EINVAL


def at(p):
    return None if p is None else ctypes.c_void_p(p)


FAR = 1 << 30     # between buffers that do not overlap


def test_matrices_overlap_only_where_they_share_a_byte():
    """Views of one buffer, against a count of their elements. Calls that are not
    refused for an overlap are for their missing workspace: nothing runs."""
    import random
    rng, seen = random.Random(3), [0, 0]

    def cells(first, rows, cols, ld):
        return {first + r * ld + c for r in range(rows) for c in range(cols)}
    for _ in range(4000):
        n, k, m = rng.randint(1, 7), rng.randint(1, 5), rng.randint(1, 5)
        lds = [rng.randint(w, 14) for w in (m, k, k)]
        if rng.random() < 0.6:
            lds = [max(lds)] * 3
        place = [rng.randint(0, 70) for _ in range(3)]
        dy, x, dx = (cells(a, n, w, ld) for a, w, ld in zip(place, (m, k, k), lds))
        d = linear_desc(n_groups=2, n_rows=n, in_dim=k, out_dim=m, dtype=P._lib.IM_F32, relu_in=1, ld_y=lds[0], ld_x=lds[1],
                        ld_dx=lds[2])
        pdy, px, pdx = (at((1 << 20) + 4 * a) for a in place)
        status = L().im_linear_backward(ctypes.byref(d), at(FAR), pdy, px, at(2 * FAR), pdx, None, None, None, 0, None, None)
        assert status == EINVAL
        msg, want = P.im_learn_last_error(), bool(dx & (dy | x))
        assert ("overlaps" if want else "workspace") in msg, (n, k, m, lds, place, msg)
        seen[want] += 1
    assert min(seen) > 1000


def test_outputs_do_not_overlap_anything():
    """Each output, the workspace and the error word on each other buffer of the call;
    buffers that a call does not read may lie anywhere."""
    R, n, k, m, G = ctypes.byref, 40, 16, 24, 2

    def refused(f, desc, names, outputs, unused=(), more=()):
        base = {name: (i + 1) * FAR for i, name in enumerate(names)}
        def call(over, ws=0):    # noqa: E306
            p = {k: at(v) for k, v in (base | over).items()}
            return f(R(desc), *[p[name] for name in names[:-1]], ws, p["error"], None)
        # nothing overlaps: the call ends at its workspace's size
        assert call({}) == EINVAL and "workspace of" in P.im_learn_last_error()
        for a in outputs:
            for b in names:
                if a == b or base[b] is None:
                    continue
                status = call({a: base[b]}, 1 << 40)
                assert status == EINVAL and "overlaps" in P.im_learn_last_error(), (a, b, P.im_learn_last_error())
        for a, b in unused:
            assert call({a: base[b]} | dict(more)) == EINVAL and "workspace of" in P.im_learn_last_error(), (a, b)

    layer = linear_desc(n_groups=G, n_rows=n, in_dim=4096, out_dim=m, ld_x=4096)       # in runs of k: a workspace
    refused(L().im_linear_forward, layer, ["offsets", "x", "W", "b", "y", "workspace", "error"], ["y", "workspace", "error"])
    back = linear_desc(n_groups=G, n_rows=n, relu_in=1)
    names = ["offsets", "dy", "x", "W", "dx", "dW", "db", "workspace", "error"]
    refused(L().im_linear_backward, back, names, ["dx", "dW", "db", "workspace", "error"])
    refused(L().im_linear_backward, back, names, [], unused=[("db", "W"), ("db", "x")], more=[("dx", None), ("dW", None)])
    names = ["offsets", "h", "W", "b", "valid", "target", "logp", "entropy", "lse", "workspace", "error"]
    refused(L().im_head_forward, head_desc(n_groups=G, n_rows=n, n_classes=1000), names,
            ["logp", "entropy", "lse", "workspace", "error"])
    names = ["offsets", "h", "W", "b", "valid", "target", "lse", "entropy", "dlogp", "dentropy", "dh", "dW", "db", "workspace",
             "error"]
    for V in (24, 100):     # in one pass, and in pieces of the classes
        refused(L().im_head_backward, head_desc(n_groups=G, n_rows=n, n_classes=V), names, ["dh", "dW", "db", "workspace", "error"],
                unused=[("dh", "entropy")], more=[("dentropy", None)])


def tensor(**kw):
    t = learn.ImAdamwTensor(4096, 4096, 4096, 4096, None, None, None, 10, 1, 0)
    for k, v in kw.items():
        setattr(t, k, v)
    return t


def test_adamw_arguments():
    R = ctypes.byref
    out = ctypes.c_void_p()

    def create(t, bits=32, gd=0, n=1, o=R(out)):
        return L().im_adamw_create(None if t is None else R(t), n, bits, gd, None, o)
    for t in (tensor(param=None), tensor(grad=None), tensor(m=None), tensor(v=None), tensor(n=-1), tensor(decay=2),
              tensor(param=4098), tensor(m=4098), tensor(copy=4097), tensor(m_scale=4096, v_scale=4096)):
        assert create(t) == EINVAL
    assert create(tensor(), bits=8) == EINVAL and create(tensor(m_scale=4096), bits=8) == EINVAL
    assert create(tensor(), bits=16) == EINVAL and create(tensor(), gd=2) == EINVAL
    assert create(tensor(), n=-1) == EINVAL and create(None) == EINVAL and create(tensor(), o=None) == EINVAL
    assert create(tensor(), n=65537) == EINVAL
    assert not out.value
    step = L().im_adamw_step
    assert step(None, 1e-3, 0.9, 0.99, 1e-8, 0.0, A, None, None) == EINVAL
    L().im_adamw_destroy(None)


def test_adamw_buffers_do_not_overlap():
    """A step's blocks run side by side: what one writes no other may touch."""
    out = ctypes.c_void_p()

    def at(first, n=300, **kw):        # five buffers of their own
        step = 4096
        t = dict(zip(("param", "grad", "m", "v", "copy"), range(first, first + 5 * step, step)), n=n)
        return tensor(**(t | kw))

    def create(*ts, bits=32):
        return L().im_adamw_create((learn.ImAdamwTensor * len(ts))(*ts), len(ts), bits, 0, None, ctypes.byref(out))
    base, far = 1 << 20, 1 << 24
    for ts in ((at(base), at(base)),                                     # one tensor twice
               (at(base), at(far, param=base + 299 * 4)), (at(base), at(far, v=base)), (at(base), at(far, copy=base)),
               (at(base), at(far, grad=base)), (at(base, grad=base),), (at(base, m=base + 3 * 4096),),
               (at(base, n=2000),)):
        assert create(*ts) == EINVAL and "overlap" in P.im_learn_last_error(), ts
    scales = dict(m_scale=far, v_scale=far + 4)
    assert create(at(base, **scales), bits=8) == EINVAL and "overlap" in P.im_learn_last_error()
    assert create(at(base, n=1 << 38)) == EINVAL and "elements" in P.im_learn_last_error()
    assert create(at(base, n=1 << 36), at(far, n=(1 << 36) + 1)) == EINVAL and "elements" in P.im_learn_last_error()
    assert not out.value


def test_tensors_are_checked():
    """The binding refuses what the library cannot see: types, devices, shapes."""
    import torch
    x = torch.zeros(4, 8)
    with pytest.raises(P.IMError) as e:
        P.im_linear_forward(x, torch.zeros(2, 8), None, torch.zeros(4, 2))
    assert e.value.status == EINVAL and "GPU" in str(e.value)
    with pytest.raises(P.IMError):
        P.im_head_forward(x, torch.zeros(2, 8), None, torch.zeros(4, dtype=torch.int32), torch.zeros(4))
    with pytest.raises(P.IMError):
        P.AdamW([dict(param=x, grad=x, m=x, v=x)])
    with pytest.raises(P.IMError):
        P.AdamW([], bits=4)


def test_dropped_plans_wait_for_the_next(monkeypatch):
    """The garbage collector frees no plan: that synchronises, and would spoil a capture."""
    freed = []

    class Library:
        @staticmethod
        def im_adamw_destroy(h):
            freed.append(h.value)
    monkeypatch.setattr(learn, "_learn", Library)
    monkeypatch.setattr(learn, "_dropped", [])
    for h in (16, 32, 48):
        opt = P.AdamW.__new__(P.AdamW)
        opt.h = ctypes.c_void_p(h)
        if h == 32:
            opt.close()
        del opt
    assert freed == [32]
    learn._free_dropped()
    assert sorted(freed) == [16, 32, 48] and not learn._dropped


def test_workspace_sizes():
    import torch
    out = ctypes.c_int64(0)
    for G, n, dt in ((1, 16, torch.bfloat16), (3, 5000, torch.float32), (64, 20000, torch.bfloat16)):
        for back in (0, 1):
            d = linear_desc(n_groups=G, n_rows=n, in_dim=4096, out_dim=256, dtype=int(dt is torch.bfloat16), ld_x=4096, ld_y=256)
            assert L().im_linear_workspace(ctypes.byref(d), back, ctypes.byref(out)) == 0
            assert P.im_linear_workspace(n, 4096, 256, dt, G, backward=bool(back)) == out.value
            d = head_desc(n_groups=G, n_rows=n, dim=96, n_classes=5000, dtype=int(dt is torch.bfloat16), ld_h=96, ld_dh=96)
            assert L().im_head_workspace(ctypes.byref(d), back, ctypes.byref(out)) == 0
            assert P.im_head_workspace(n, 96, 5000, dt, G, backward=bool(back)) == out.value > 0
    for call in (lambda: P.im_linear_workspace(-1, 8, 8, torch.float32), lambda: P.im_linear_workspace(1, 8, 8, torch.float16),
                 lambda: P.im_head_workspace(1, 8, 0, torch.float32), lambda: P.im_head_workspace(1, 8, 8, torch.float32, device="cpu")):
        with pytest.raises(P.IMError) as e:
            call()
        assert e.value.status == EINVAL
