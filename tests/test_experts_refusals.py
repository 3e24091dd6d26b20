"""The C ABI of the operators around experts and of rows in 8 bits on a machine without a GPU: every
refusal that is decided before a device is touched."""
import ctypes

import pytest

import paper_2606_11440_amd as P
from paper_2606_11440_amd import learn

EINVAL = P._lib.IM_EINVAL
R = ctypes.byref
BIG = 1 << 40


def at(k):
    """An aligned address of a range of its own, never dereferenced."""
    return ctypes.c_void_p((k + 1) << 44)


def L():
    return learn.load_learn()


def router_desc(**kw):
    d = learn.ImRouterDesc(8, 24, 4, 1, 1, 1, 0, 0, 1, 1.0, 24, 24)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def dispatch_desc(**kw):
    d = learn.ImDispatchDesc(8, 2, 4, 16, 24, 0, 24, 24, 24)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def rows_desc(**kw):
    d = learn.ImRowsDesc(8, 24, 1, 0, 24, 24)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def linear_desc(**kw):
    d = learn.ImLinearDesc(1, 8, 16, 24, 1, 0, 0, 0, 16, 24, 16)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def refused(call, good, changes):
    """Each change (place, argument) of a good call is refused."""
    for i, v in changes:
        args = list(good)
        args[i] = v
        assert call(*args) == EINVAL, (i, v)
    assert P.im_learn_last_error() != "no error"


@pytest.mark.parametrize("over", [dict(n_rows=-1), dict(n_rows=(1 << 30) + 1), dict(n_experts=0), dict(n_experts=1025),
                                  dict(top_k=0), dict(top_k=25), dict(dtype=2), dict(score=2), dict(renorm=2),
                                  dict(scale=float("nan")), dict(scale=float("inf")), dict(ld_z=23), dict(ld_z=(1 << 22) + 1)])
def test_bad_routers(over):
    d = router_desc(**over)
    assert L().im_router_forward(R(d), at(0), at(1), at(2), at(3), at(4), None) == EINVAL
    assert L().im_router_backward(R(d), at(0), at(1), at(2), at(3), at(4), at(5), None) == EINVAL


def test_router_arguments():
    f, b = L().im_router_forward, L().im_router_backward
    d = router_desc()
    good = [R(d), at(0), at(1), at(2), at(3), at(4), None]
    odd = ctypes.c_void_p((1 << 44) + 2)
    refused(f, good, [(0, None), (1, None), (4, None), (5, None), (1, odd), (2, odd), (3, odd), (4, odd), (5, odd),
                      (4, at(0)), (5, at(3)), (5, at(1)), (4, at(2))] +
            [(0, R(router_desc(**kw))) for kw in (dict(n_sets=0), dict(n_sets=5), dict(n_sets=48), dict(n_sets=4, top_sets=5),
                                                  dict(top_sets=0), dict(set_best=0), dict(set_best=3),
                                                  dict(n_sets=12, top_sets=1))])
    assert f(R(router_desc(n_experts=64, ld_z=64, top_k=33)), *good[1:]) == EINVAL
    good = [R(d), at(0), at(1), at(2), at(3), at(4), at(5), None]
    refused(b, good, [(0, None), (1, None), (3, None), (4, None), (5, None), (1, odd), (2, odd), (3, odd), (4, odd), (5, odd),
                      (6, odd), (5, at(0)), (5, at(3)), (6, at(2)), (0, R(router_desc(ld_dz=23)))])
    # without rows nothing is needed
    assert f(R(router_desc(n_rows=0)), None, None, None, None, None, None) == 0
    assert b(R(router_desc(n_rows=0)), None, None, None, None, None, None, None) == 0


def test_plan_arguments():
    f, need = L().im_dispatch_plan, ctypes.c_int64(7)
    for kw in (dict(n_rows=-1), dict(n_rows=(1 << 29) + 1), dict(top_k=0), dict(top_k=33), dict(n_experts=0),
               dict(n_experts=1025)):
        d = dispatch_desc(**kw)
        assert L().im_dispatch_workspace(R(d), R(need)) == EINVAL and need.value == 7
        assert f(R(d), at(0), at(1), at(2), at(3), BIG, at(4), None) == EINVAL
    d = dispatch_desc(n_rows=100000)
    assert L().im_dispatch_workspace(R(d), None) == EINVAL
    assert L().im_dispatch_workspace(R(d), R(need)) == 0 and need.value > 0
    odd = ctypes.c_void_p((1 << 44) + 2)
    good = [R(d), at(0), at(1), at(2), at(3), BIG, at(4), None]
    refused(f, good, [(0, None), (1, None), (2, None), (3, None), (4, None), (5, need.value - 1), (1, odd), (2, odd), (3, odd),
                      (6, odd), (4, ctypes.c_void_p((4 << 44) + 128)), (3, at(0)), (2, at(0)), (3, at(3)), (6, at(2)),
                      (2, at(2))])


@pytest.mark.parametrize("over", [dict(n_rows=-1), dict(n_rows=(1 << 30) + 1), dict(n_rows=(1 << 29) + 1), dict(top_k=0),
                                  dict(top_k=33), dict(n_slots=-1), dict(n_slots=(1 << 30) + 1), dict(dim=0),
                                  dict(dim=65537), dict(dtype=3), dict(ld_row=23), dict(ld_slot=23),
                                  dict(ld_row=(1 << 22) + 1)])
def test_bad_exchanges(over):
    d = dispatch_desc(**over)
    assert L().im_dispatch_forward(R(d), at(0), at(1), at(2), at(3), None) == EINVAL
    assert L().im_dispatch_backward(R(d), at(0), at(1), at(2), at(3), None) == EINVAL
    assert L().im_combine_forward(R(d), at(0), at(1), at(2), at(3), at(4), None) == EINVAL
    assert L().im_combine_backward(R(d), at(0), at(1), at(2), at(3), at(4), at(5), at(6), None) == EINVAL


def test_exchange_arguments():
    d, codes = dispatch_desc(), dispatch_desc(dtype=2)
    odd = ctypes.c_void_p((1 << 44) + 2)
    refused(L().im_dispatch_forward, [R(d), at(0), at(1), at(2), at(3), None],
            [(0, None), (1, None), (2, None), (3, None), (1, odd), (2, odd), (3, odd), (4, odd), (3, at(0)), (3, at(1)), (4, at(2))])
    refused(L().im_dispatch_backward, [R(d), at(0), at(1), at(2), at(3), None],
            [(0, None), (0, R(codes)), (1, None), (2, None), (3, None), (1, odd), (2, odd), (3, odd), (4, odd), (3, at(0)),
             (3, at(1)), (4, at(2))])
    refused(L().im_combine_forward, [R(d), at(0), at(1), at(2), at(3), at(4), None],
            [(0, None), (0, R(codes)), (1, None), (2, None), (3, None), (4, None), (3, odd), (4, at(0)), (4, at(2)), (5, at(3))])
    refused(L().im_combine_backward, [R(d), at(0), at(1), at(2), at(3), at(4), at(5), at(6), None],
            [(0, None), (0, R(codes)), (1, None), (2, None), (3, None), (4, None), (1, odd), (5, odd), (6, odd), (5, at(0)),
             (5, at(1)), (6, at(3)), (6, at(4)), (7, at(5)), (0, R(dispatch_desc(ld_dslot=23)))])


@pytest.mark.parametrize("over", [dict(n_rows=-1), dict(n_rows=(1 << 30) + 1), dict(dim=0), dict(dim=65537), dict(dtype=2),
                                  dict(keep=2), dict(ld_x=23), dict(ld_codes=23), dict(ld_codes=(1 << 22) + 1)])
def test_bad_rows(over):
    d = rows_desc(**over)
    assert L().im_rows_pack(R(d), at(0), at(1), at(2), None) == EINVAL
    assert L().im_rows_unpack(R(d), at(0), at(1), at(2), None) == EINVAL


def test_rows_arguments():
    odd = ctypes.c_void_p((1 << 44) + 1)
    refused(L().im_rows_pack, [R(rows_desc()), at(0), at(1), at(2), None],
            [(0, None), (1, None), (2, None), (3, None), (1, odd), (3, odd), (2, at(0)), (3, at(0)), (3, at(1))])
    refused(L().im_rows_unpack, [R(rows_desc()), at(0), at(1), at(2), None],
            [(0, None), (1, None), (2, None), (3, None), (2, odd), (3, odd), (3, at(0)), (3, at(1))])


BAD_LINEAR = [dict(n_groups=0), dict(n_groups=1025), dict(n_rows=-1), dict(n_rows=(1 << 30) + 1), dict(in_dim=0),
              dict(in_dim=65537), dict(out_dim=0), dict(out_dim=65537), dict(dtype=2), dict(relu=2), dict(relu_in=-1)]


@pytest.mark.parametrize("over", BAD_LINEAR)
def test_bad_layers(over):
    d, out = linear_desc(**over), ctypes.c_int64(7)
    assert L().im_linear_workspace_packed(R(d), 0, R(out)) == EINVAL and out.value == 7
    assert L().im_linear_forward_packed(R(d), at(0), at(1), at(2), at(3), at(4), at(5), at(6), at(7), BIG, None, None) == EINVAL
    assert L().im_linear_backward_packed(R(d), at(0), at(1), at(2), at(3), at(4), at(5), at(6), at(7), at(8), BIG, None,
                                         None) == EINVAL


def test_layer_arguments():
    need = ctypes.c_int64(0)
    odd = ctypes.c_void_p((1 << 44) + 1)
    d = linear_desc(n_rows=4, in_dim=8192, ld_x=8192)
    assert L().im_linear_workspace_packed(R(d), 0, R(need)) == 0 and need.value > 0
    assert L().im_linear_workspace_packed(R(d), 2, R(need)) == EINVAL
    assert L().im_linear_workspace_packed(R(d), 0, None) == EINVAL
    good = [R(d), None, at(0), at(1), at(2), at(3), at(4), at(5), at(6), BIG, at(7), None]
    refused(L().im_linear_forward_packed, good,
            [(0, None), (2, None), (3, None), (4, None), (5, None), (7, None), (8, None), (9, need.value - 1),
             (8, ctypes.c_void_p((7 << 44) + 128)), (1, odd), (3, odd), (5, odd), (6, odd), (7, odd), (10, odd), (7, at(0)),
             (7, at(1)), (7, at(3)), (8, at(5)), (10, at(4)), (0, R(linear_desc(n_groups=2))), (0, R(linear_desc(ld_x=15))),
             (0, R(linear_desc(ld_y=23)))])
    d = linear_desc(n_groups=3, n_rows=5000)
    assert L().im_linear_workspace_packed(R(d), 1, R(need)) == 0 and need.value > 0
    good = [R(d), at(0), at(1), at(2), at(3), at(4), at(5), at(6), at(7), at(8), BIG, at(9), None]
    refused(L().im_linear_backward_packed, good,
            [(0, None), (1, None), (2, None), (3, None), (4, None), (5, None), (9, None), (10, need.value - 1), (2, odd), (4, odd),
             (5, odd), (6, odd), (7, odd), (8, odd), (11, odd), (6, at(1)), (6, at(4)), (7, at(2)), (7, at(3)), (8, at(6)),
             (9, at(7)), (0, R(linear_desc(n_groups=3, n_rows=5000, ld_dx=3)))])
    big = linear_desc(n_rows=2 ** 30, in_dim=65536, out_dim=65536, ld_x=65536, ld_y=65536)
    assert L().im_linear_forward_packed(R(big), None, at(0), at(1), at(2), at(3), None, ctypes.c_void_p(6 << 50), None, 0, None,
                                        None) == P._lib.IM_EUNSUPPORTED


def test_python_refuses_before_the_library():
    import torch
    z = torch.zeros(4, 8)
    e, w = torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    for call in (lambda: P.im_router_forward(z, e, w), lambda: P.im_router_backward(z, e, w, z),
                 lambda: P.im_dispatch_plan(e, torch.zeros(9, dtype=torch.int32), e),
                 lambda: P.im_dispatch_forward(z, e, z), lambda: P.im_dispatch_backward(z, e, z),
                 lambda: P.im_combine_forward(z, e, w, z), lambda: P.im_combine_backward(z, z, e, w, z, w),
                 lambda: P.im_rows_pack(z, z.to(torch.int8), w[:, 0]), lambda: P.im_rows_unpack(z.to(torch.int8), w[:, 0], z),
                 lambda: P.im_linear_forward_packed(z.to(torch.int8), w, z.to(torch.int8), w, None, z),
                 lambda: P.im_linear_backward_packed(z, z.to(torch.int8), w, z),
                 lambda: P.im_linear_workspace_packed(4, 4, 4, torch.float16)):
        with pytest.raises(P.IMError):
            call()
    assert P.im_dispatch_workspace(10, 2, 8) == 0 and P.im_dispatch_workspace(100000, 2, 8) > 0


def test_descriptions_lie_as_the_structures_do():
    for form, cls in ((learn._LINEAR, learn.ImLinearDesc), (learn._ROUTER, learn.ImRouterDesc),
                      (learn._DISPATCH, learn.ImDispatchDesc), (learn._ROWS, learn.ImRowsDesc)):
        values = [i + 1 for i in range(len(cls._fields_))]
        assert form.size == ctypes.sizeof(cls)
        d = cls.from_buffer_copy(form.pack(*values))
        assert [getattr(d, name) for name, _ in cls._fields_] == values
        values[0] = 1 << 31
        with pytest.raises(P.IMError):
            learn._desc(form, *values)
