"""ctypes binding of libinframind_learn (include/inframind_learn.h): the
learner's operators. Argument checks and marshalling only; the work is done by
the library's HIP kernels, on torch tensors that the caller owns.

A call runs on its tensors' device and, unless `stream` (a raw HIP stream
handle) is given, on torch's current stream of that device; tensors used on
another stream than their own have to be kept until that work is done. `workspace` is
taken from torch's allocator where it is not given; calls that may run at the
same time need one each. `error` is a device int32 tensor [1] that collects
IM_ERR_* bits. Invalid arguments raise IMError with status IM_EINVAL and change
nothing; outputs that overlap an input or one another are such (columns side by
side in one buffer are not).

The functions keep the C names (im_linear_forward, im_linear_backward,
im_head_forward, im_head_backward, and im_linear_workspace and im_head_workspace
for the size of a workspace that a program keeps); AdamW holds an im_adamw plan.
Around experts: im_router_forward, im_router_backward, im_dispatch_plan,
im_dispatch_forward, im_dispatch_backward, im_combine_forward, im_combine_backward.
Rows in 8 bits: im_rows_pack, im_rows_unpack, im_linear_forward_packed,
im_linear_backward_packed (their codes are int8 tensors, the scales float32)."""
from __future__ import annotations

import ctypes
import os
import struct

from . import _lib
from ._lib import HERE, IM_BF16, IM_EINVAL, IM_F32, IM_OK, IMError, _stream

LEARN_PATH = os.path.join(HERE, "libinframind_learn.so")
LEARN_EXPORTED = ("im_linear_workspace", "im_linear_forward", "im_linear_backward", "im_head_workspace",
                  "im_head_forward", "im_head_backward", "im_adamw_create", "im_adamw_step", "im_adamw_destroy",
                  "im_learn_last_error", "im_router_forward", "im_router_backward", "im_dispatch_workspace",
                  "im_dispatch_plan", "im_dispatch_forward", "im_dispatch_backward", "im_combine_forward",
                  "im_combine_backward", "im_rows_pack", "im_rows_unpack", "im_linear_workspace_packed",
                  "im_linear_forward_packed", "im_linear_backward_packed")
IM_CODES = 2
SCORES = {"softmax": 0, "sigmoid": 1}
IM_MAX_GROUPS, IM_MAX_DIM, IM_MAX_CLASSES, IM_STATE_BLOCK = 1024, 65536, 1 << 22, 256

_P, _I32, _I64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64


class ImLinearDesc(ctypes.Structure):
    _fields_ = [("n_groups", _I32), ("n_rows", _I32), ("in_dim", _I32), ("out_dim", _I32), ("dtype", _I32),
                ("relu", _I32), ("relu_in", _I32), ("reserved", _I32), ("ld_x", _I64), ("ld_y", _I64), ("ld_dx", _I64)]


class ImHeadDesc(ctypes.Structure):
    _fields_ = [("n_groups", _I32), ("n_rows", _I32), ("dim", _I32), ("n_classes", _I32), ("dtype", _I32),
                ("relu_in", _I32), ("reserved0", _I32), ("reserved1", _I32), ("ld_h", _I64), ("ld_dh", _I64)]


class ImRouterDesc(ctypes.Structure):
    _fields_ = [("n_rows", _I32), ("n_experts", _I32), ("top_k", _I32), ("n_sets", _I32), ("top_sets", _I32),
                ("set_best", _I32), ("dtype", _I32), ("score", _I32), ("renorm", _I32), ("scale", ctypes.c_float),
                ("ld_z", _I64), ("ld_dz", _I64)]


class ImDispatchDesc(ctypes.Structure):
    _fields_ = [("n_rows", _I32), ("top_k", _I32), ("n_experts", _I32), ("n_slots", _I32), ("dim", _I32),
                ("dtype", _I32), ("ld_row", _I64), ("ld_slot", _I64), ("ld_dslot", _I64)]


class ImRowsDesc(ctypes.Structure):
    _fields_ = [("n_rows", _I32), ("dim", _I32), ("dtype", _I32), ("keep", _I32), ("ld_x", _I64), ("ld_codes", _I64)]


class ImAdamwTensor(ctypes.Structure):
    _fields_ = [("param", _P), ("grad", _P), ("m", _P), ("v", _P), ("m_scale", _P), ("v_scale", _P), ("copy", _P),
                ("n", _I64), ("decay", _I32), ("reserved", _I32)]


_learn = None


def load_learn() -> ctypes.CDLL:
    """Load the in-tree libinframind_learn.so; fails loudly when it is missing."""
    global _learn
    if _learn is not None:
        return _learn
    if not os.path.exists(LEARN_PATH):
        raise RuntimeError(f"{LEARN_PATH} is missing: build it with __graft_entry__.build() "
                           "(hipcc, gfx950); there is no fallback path")
    L = ctypes.CDLL(LEARN_PATH)
    D = ctypes.c_double
    L.im_linear_workspace.argtypes = [_P, _I32, _P]
    L.im_linear_forward.argtypes = [_P] * 7 + [_I64, _P, _P]
    L.im_linear_backward.argtypes = [_P] * 9 + [_I64, _P, _P]
    L.im_head_workspace.argtypes = [_P, _I32, _P]
    L.im_head_forward.argtypes = [_P] * 11 + [_I64, _P, _P]
    L.im_head_backward.argtypes = [_P] * 15 + [_I64, _P, _P]
    L.im_adamw_create.argtypes = [_P, _I32, _I32, _I32, _P, _P]
    L.im_adamw_step.argtypes = [_P, D, D, D, D, D, _P, _P, _P]
    L.im_adamw_destroy.argtypes = [_P]
    L.im_adamw_destroy.restype = None
    L.im_learn_last_error.restype = ctypes.c_char_p
    L.im_router_forward.argtypes = [_P] * 7
    L.im_router_backward.argtypes = [_P] * 8
    L.im_dispatch_workspace.argtypes = [_P, _P]
    L.im_dispatch_plan.argtypes = [_P] * 5 + [_I64, _P, _P]
    L.im_dispatch_forward.argtypes = [_P] * 6
    L.im_dispatch_backward.argtypes = [_P] * 6
    L.im_combine_forward.argtypes = [_P] * 7
    L.im_combine_backward.argtypes = [_P] * 9
    L.im_rows_pack.argtypes = [_P] * 5
    L.im_rows_unpack.argtypes = [_P] * 5
    L.im_linear_workspace_packed.argtypes = [_P, _I32, _P]
    L.im_linear_forward_packed.argtypes = [_P] * 9 + [_I64, _P, _P]
    L.im_linear_backward_packed.argtypes = [_P] * 10 + [_I64, _P, _P]
    _learn = L
    return L


def im_learn_last_error() -> str:
    return load_learn().im_learn_last_error().decode()


def _bad(msg):
    raise IMError(IM_EINVAL, msg)


def _done(status):
    if status != IM_OK:
        raise IMError(status, im_learn_last_error())


class _On:
    """The tensors' device as torch's current one for the length of a call."""
    __slots__ = ("index", "was")

    def __init__(self, index):
        self.index = index

    def __enter__(self):
        import torch
        self.was = torch.cuda.current_device()
        if self.was != self.index:
            torch.cuda.set_device(self.index)

    def __exit__(self, *exc):
        if self.was != self.index:
            import torch
            torch.cuda.set_device(self.was)


_device = _raw = None   # torch's accessors of the current device's number and of its current stream's handle


def _run(index, stream, call, *args):
    """A call of the library on device `index` and on `stream`, or torch's current stream of that device."""
    global _device, _raw
    if _device is None:
        _stream(None)
        _raw, _device = _lib._current
    if _device() == index:
        status = call(*args, _raw(index) if stream is None else int(stream))
    else:
        with _On(index):
            status = call(*args, _stream(stream))
    if status != IM_OK:
        raise IMError(status, im_learn_last_error())


def _matrix(t, name, dtype, device, rows, cols):
    """Row stride of a [rows, cols] tensor whose columns are contiguous."""
    if t.dtype is not dtype or t.device != device:
        _bad(f"{name} is {t.dtype} on {t.device}, {dtype} on {device} expected")
    if t.shape != (rows, cols):
        _bad(f"{name} has shape {tuple(t.shape)}, ({rows}, {cols}) expected")
    ld, inner = t.stride()
    if inner != 1 and cols > 1:
        _bad(f"the columns of {name} are not contiguous")
    if rows > 1:
        if ld < cols:
            _bad(f"the rows of {name} overlap")
        return ld
    return cols


def _flat(t, name, dtype, device, count):
    """Pointer of a contiguous tensor of `count` elements, or None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.device != device:
        _bad(f"{name} is {t.dtype} on {t.device}, {dtype} on {device} expected")
    if t.numel() != count or not t.is_contiguous():
        _bad(f"{name} has shape {tuple(t.shape)} and strides {t.stride()}: {count} contiguous elements expected")
    return t.data_ptr()


_KINDS = {}


def _kinds():
    import torch
    _KINDS.update({torch.float32: IM_F32, torch.bfloat16: IM_BF16, "f32": torch.float32, "i32": torch.int32,
                   "i64": torch.int64, "u8": torch.uint8, "i8": torch.int8, "fp8": torch.float8_e4m3fn})


def _kind(t, name):
    """im_dtype of a tensor on a GPU."""
    if not _KINDS:
        _kinds()
    if t.device.type != "cuda":
        _bad(f"{name} is on {t.device}, a GPU is expected")
    k = _KINDS.get(t.dtype)
    if k is None:
        _bad(f"{name} is {t.dtype}: float32 or bfloat16 expected")
    return k


def _weights(W, dtype, device, cols):
    """Groups and rows of contiguous weights [groups, rows, cols] or [rows, cols]."""
    if W.dtype is not dtype or W.device != device:
        _bad(f"W is {W.dtype} on {W.device}, {dtype} on {device} expected")
    if W.dim() not in (2, 3) or W.shape[-1] != cols or not W.is_contiguous():
        _bad(f"W has shape {tuple(W.shape)} and strides {W.stride()}: contiguous [groups, out, {cols}] expected")
    return (1 if W.dim() == 2 else W.shape[0]), W.shape[-2]


def _offsets(offsets, G, device):
    if offsets is None:
        if G != 1:
            _bad("offsets are needed for more than one group")
        return None
    return _flat(offsets, "offsets", _KINDS["i32"], device, G + 1)


_SIZES = {}


def _workspace(query, desc, key, backward, workspace, device, stream):
    """(tensor to keep, pointer, bytes) of a call's workspace."""
    need = _SIZES.get(key)
    if need is None:
        out = _I64(0)
        with _On(device.index):
            _done(query(ctypes.byref(desc), backward, ctypes.byref(out)))
        if len(_SIZES) >= 4096:
            _SIZES.clear()
        need = _SIZES[key] = out.value
    if need == 0:
        return None, None, 0
    import torch
    if workspace is not None:
        if workspace.device != device or not workspace.is_contiguous():
            _bad(f"workspace is on {workspace.device} or not contiguous")
        size = workspace.numel() * workspace.element_size()
        return workspace, workspace.data_ptr(), size
    if stream is None or int(stream) == torch.cuda.current_stream(device).cuda_stream:
        t = torch.empty(need, dtype=torch.uint8, device=device)
    else:   # memory that torch hands out again in the order of the stream that uses it
        with torch.cuda.stream(torch.cuda.ExternalStream(int(stream), device=device)):
            t = torch.empty(need, dtype=torch.uint8, device=device)
    return t, t.data_ptr(), need


def _size_of(query, desc, backward, device):
    out = _I64(0)
    if device is None:
        _done(query(ctypes.byref(desc), 1 if backward else 0, ctypes.byref(out)))
    else:
        import torch
        device = torch.device(device)
        if device.type != "cuda":
            _bad(f"device is {device}, a GPU is expected")
        with _On(torch.cuda.current_device() if device.index is None else device.index):
            _done(query(ctypes.byref(desc), 1 if backward else 0, ctypes.byref(out)))
    return out.value


def _kind_of(dtype):
    import torch
    if dtype not in (torch.float32, torch.bfloat16):
        _bad(f"dtype is {dtype}: float32 or bfloat16 expected")
    return IM_F32 if dtype is torch.float32 else IM_BF16


def im_linear_workspace(n_rows, in_dim, out_dim, dtype, n_groups=1, backward=False, device=None):
    """Bytes of workspace of im_linear_forward, or im_linear_backward, on `device`
    (None: the current one). A buffer for several calls takes the largest of
    theirs: fewer rows may need more."""
    d = ImLinearDesc(n_groups, n_rows, in_dim, out_dim, _kind_of(dtype), 0, 0, 0, in_dim, out_dim, in_dim)
    return _size_of((_learn or load_learn()).im_linear_workspace, d, backward, device)


def im_head_workspace(n_rows, dim, n_classes, dtype, n_groups=1, backward=False, device=None):
    """Bytes of workspace of im_head_forward, or im_head_backward; as im_linear_workspace."""
    d = ImHeadDesc(n_groups, n_rows, dim, n_classes, _kind_of(dtype), 0, 0, 0, dim, dim)
    return _size_of((_learn or load_learn()).im_head_workspace, d, backward, device)


def im_linear_forward(x, W, b, y, offsets=None, relu=False, workspace=None, error=None, stream=None):
    """y = act(x W_g^T + b_g) for the rows of each group: x [n, in], W [groups,
    out, in] (or [out, in]), b float32 [groups, out] or None, y [n, out] out.
    Rows of x and y may be strided."""
    kind, dev, dt = _kind(x, "x"), x.device, x.dtype
    n, k = x.shape if x.dim() == 2 else _bad("x is not a matrix")
    ld_x = _matrix(x, "x", dt, dev, n, k)
    G, m = _weights(W, dt, dev, k)
    ld_y = _matrix(y, "y", dt, dev, n, m)
    f32, i32 = _KINDS["f32"], _KINDS["i32"]
    L = _learn or load_learn()
    d = ImLinearDesc(G, n, k, m, kind, 1 if relu else 0, 0, 0, ld_x, ld_y, 0)
    with _On(dev.index):
        ws, at, size = _workspace(L.im_linear_workspace, d, (0, dev.index, G, n, k, m, kind), 0, workspace, dev, stream)
        _done(L.im_linear_forward(ctypes.byref(d), _offsets(offsets, G, dev), x.data_ptr(), W.data_ptr(),
                                  _flat(b, "b", f32, dev, G * m), y.data_ptr(), at, size,
                                  _flat(error, "error", i32, dev, 1), _stream(stream)))


def im_linear_backward(dy, x, W, dx=None, dW=None, db=None, offsets=None, relu_in=False, workspace=None, error=None,
                       stream=None):
    """Gradients of a layer from dy (the gradient of x W_g^T + b_g): dx [n, in],
    dW like W, db float32 [groups, out]; None skips one. relu_in: x is a ReLU
    output and dx the gradient before that ReLU."""
    kind, dev, dt = _kind(dy, "dy"), dy.device, dy.dtype
    n, m = dy.shape if dy.dim() == 2 else _bad("dy is not a matrix")
    if x.dim() != 2:
        _bad("x is not a matrix")
    k = x.shape[1]
    ld_y = _matrix(dy, "dy", dt, dev, n, m)
    ld_x = _matrix(x, "x", dt, dev, n, k)
    G, rows = _weights(W, dt, dev, k)
    if rows != m:
        _bad(f"W has {rows} outputs, dy {m}")
    ld_dx = k if dx is None else _matrix(dx, "dx", dt, dev, n, k)
    f32, i32 = _KINDS["f32"], _KINDS["i32"]
    L = _learn or load_learn()
    d = ImLinearDesc(G, n, k, m, kind, 0, 1 if relu_in else 0, 0, ld_x, ld_y, ld_dx)
    with _On(dev.index):
        ws, at, size = _workspace(L.im_linear_workspace, d, (1, dev.index, G, n, k, m, kind), 1, workspace, dev, stream)
        _done(L.im_linear_backward(ctypes.byref(d), _offsets(offsets, G, dev), dy.data_ptr(), x.data_ptr(),
                                   W.data_ptr(), None if dx is None else dx.data_ptr(),
                                   _flat(dW, "dW", dt, dev, G * m * k), _flat(db, "db", f32, dev, G * m), at, size,
                                   _flat(error, "error", i32, dev, 1), _stream(stream)))


def _head(h, W, b, target, valid):
    kind, dev, dt = _kind(h, "h"), h.device, h.dtype
    n, k = h.shape if h.dim() == 2 else _bad("h is not a matrix")
    ld = _matrix(h, "h", dt, dev, n, k)
    G, V = _weights(W, dt, dev, k)
    f32, i32 = _KINDS["f32"], _KINDS["i32"]
    if valid is not None and valid.dtype is not i32 and str(valid.dtype) != "torch.uint32":
        _bad(f"valid is {valid.dtype}: int32 (or uint32) words expected")
    return (kind, dev, dt, n, k, ld, G, V, _flat(b, "b", f32, dev, G * V), _flat(target, "target", i32, dev, n),
            None if valid is None else _flat(valid, "valid", valid.dtype, dev, n * ((V + 31) // 32)))


def im_head_forward(h, W, b, target, logp, entropy=None, lse=None, valid=None, offsets=None, workspace=None,
                    error=None, stream=None):
    """Log-probability of `target` (int32 [n], -1: none) under the softmax of
    h W_g^T + b_g over the valid classes, its entropy and its log-sum-exp:
    float32 [n] outputs. valid: int32 words [n, ceil(classes / 32)], bit j % 32 of
    word j / 32 set where class j is valid; None: all are."""
    kind, dev, dt, n, k, ld, G, V, pb, pt, pv = _head(h, W, b, target, valid)
    if target is None or logp is None:
        _bad("target and logp are needed")
    f32, i32 = _KINDS["f32"], _KINDS["i32"]
    L = _learn or load_learn()
    d = ImHeadDesc(G, n, k, V, kind, 0, 0, 0, ld, 0)
    with _On(dev.index):
        ws, at, size = _workspace(L.im_head_workspace, d, (2, dev.index, G, n, k, V, kind), 0, workspace, dev, stream)
        _done(L.im_head_forward(ctypes.byref(d), _offsets(offsets, G, dev), h.data_ptr(), W.data_ptr(), pb, pv, pt,
                                _flat(logp, "logp", f32, dev, n), _flat(entropy, "entropy", f32, dev, n),
                                _flat(lse, "lse", f32, dev, n), at, size, _flat(error, "error", i32, dev, 1),
                                _stream(stream)))


def im_head_backward(h, W, b, target, lse, dlogp, dh=None, dW=None, db=None, valid=None, entropy=None, dentropy=None,
                     offsets=None, relu_in=False, workspace=None, error=None, stream=None):
    """Gradients of sum(dlogp logp + dentropy entropy): dh [n, dim], dW like W, db
    float32 [groups, classes]; None skips one. lse and entropy are the forward
    call's; dentropy None: no entropy term. relu_in: h is a ReLU output and dh
    the gradient before that ReLU."""
    kind, dev, dt, n, k, ld, G, V, pb, pt, pv = _head(h, W, b, target, valid)
    if target is None or lse is None or dlogp is None:
        _bad("target, lse and dlogp are needed")
    ld_dh = k if dh is None else _matrix(dh, "dh", dt, dev, n, k)
    f32, i32 = _KINDS["f32"], _KINDS["i32"]
    L = _learn or load_learn()
    d = ImHeadDesc(G, n, k, V, kind, 1 if relu_in else 0, 0, 0, ld, ld_dh)
    with _On(dev.index):
        ws, at, size = _workspace(L.im_head_workspace, d, (3, dev.index, G, n, k, V, kind), 1, workspace, dev, stream)
        _done(L.im_head_backward(ctypes.byref(d), _offsets(offsets, G, dev), h.data_ptr(), W.data_ptr(), pb, pv, pt,
                                 _flat(lse, "lse", f32, dev, n), _flat(entropy, "entropy", f32, dev, n),
                                 _flat(dlogp, "dlogp", f32, dev, n), _flat(dentropy, "dentropy", f32, dev, n),
                                 None if dh is None else dh.data_ptr(), _flat(dW, "dW", dt, dev, G * V * k),
                                 _flat(db, "db", f32, dev, G * V), at, size, _flat(error, "error", i32, dev, 1),
                                 _stream(stream)))


# The calls below check a tensor in the order that passes soonest; what does not pass is looked at again by
# _flat and _matrix, which say why. Descriptions are packed as the C structures lie.
_LINEAR, _ROUTER, _DISPATCH, _ROWS = (struct.Struct(f) for f in ("=8i3q", "=9if2q", "=6i3q", "=4i2q"))


def _desc(form, *values):
    try:
        return form.pack(*values)
    except (struct.error, OverflowError) as e:
        _bad(f"an argument is out of range: {e}")


def _cuda(index):
    import torch
    return torch.device("cuda", index)


def _first(t, name):
    """im_dtype and device number of a tensor on a GPU."""
    if not _KINDS:
        _kinds()
    kind = _KINDS.get(t.dtype) if t.is_cuda else None
    return (_kind(t, name) if kind is None else kind), t.get_device()


def _at(t, name, dtype, index, count):
    """Pointer of a contiguous tensor of `count` elements, or None."""
    if t is None:
        return None
    if t.dtype is dtype and t.get_device() == index and t.numel() == count and t.is_contiguous():
        return t.data_ptr()
    return _flat(t, name, dtype, _cuda(index), count)


def _ld(t, name, dtype, index, rows, cols):
    """Row stride of a [rows, cols] tensor whose columns are contiguous."""
    if rows > 1 and t.dtype is dtype and t.get_device() == index and t.shape == (rows, cols):
        ld, inner = t.stride()
        if inner == 1 and ld >= cols:
            return ld
    return _matrix(t, name, dtype, _cuda(index), rows, cols)


def _mask(valid, n, classes, index):
    """Pointer of the words of a mask [n, ceil(classes / 32)], or None."""
    if valid is None:
        return None
    if valid.dtype is not _KINDS["i32"] and str(valid.dtype) != "torch.uint32":
        _bad(f"valid is {valid.dtype}: int32 (or uint32) words expected")
    return _at(valid, "valid", valid.dtype, index, n * ((classes + 31) // 32))


def _matrix_of(t, name):
    """Rows and columns of a tensor that must be a matrix."""
    return t.shape if t.dim() == 2 else _bad(f"{name} is not a matrix")


def _score(score):
    at = SCORES.get(score)
    return _bad(f"score is {score!r}: 'softmax' or 'sigmoid' expected") if at is None else at


def im_router_forward(z, expert, weight, bias=None, valid=None, score="softmax", renorm=True, scale=1.0, n_sets=1,
                      top_sets=None, set_best=1, stream=None):
    """Choice of experts [n, top_k] (int32; -1: none left) and their weights (float32)
    from logits z [n, experts], whose rows may be strided. score: "softmax" or "sigmoid";
    the choice goes by score + bias (float32 [experts]) within the top_sets best of
    n_sets equal sets, valued by their set_best (1 or 2) best; weights are scale times the
    scores, divided by their sum with renorm. valid: as for im_head_forward."""
    kind, on = _first(z, "z")
    n, E = _matrix_of(z, "z")
    k = _matrix_of(expert, "expert")[1]
    f32 = _KINDS["f32"]
    d = _desc(_ROUTER, n, E, k, n_sets, n_sets if top_sets is None else top_sets, set_best, kind, _score(score),
              1 if renorm else 0, scale, _ld(z, "z", z.dtype, on, n, E), 0)
    _run(on, stream, (_learn or load_learn()).im_router_forward, d, z.data_ptr(), _at(bias, "bias", f32, on, E),
         _mask(valid, n, E, on), _at(expert, "expert", _KINDS["i32"], on, n * k), _at(weight, "weight", f32, on, n * k))


def im_router_backward(z, expert, dweight, dz, valid=None, score="softmax", renorm=True, scale=1.0, error=None,
                       stream=None):
    """Gradient dz [n, experts] of the logits from dweight (float32 [n, top_k]), for the
    experts that im_router_forward chose. Rows of z and dz may be strided."""
    kind, on = _first(z, "z")
    n, E = _matrix_of(z, "z")
    k, dt, i32 = _matrix_of(expert, "expert")[1], z.dtype, _KINDS["i32"]
    d = _desc(_ROUTER, n, E, k, 1, 1, 1, kind, _score(score), 1 if renorm else 0, scale, _ld(z, "z", dt, on, n, E),
              _ld(dz, "dz", dt, on, n, E))
    _run(on, stream, (_learn or load_learn()).im_router_backward, d, z.data_ptr(), _mask(valid, n, E, on),
         _at(expert, "expert", i32, on, n * k), _at(dweight, "dweight", _KINDS["f32"], on, n * k), dz.data_ptr(),
         _at(error, "error", i32, on, 1))


def _dispatch_size(desc, backward, out):
    return (_learn or load_learn()).im_dispatch_workspace(desc, out)


def im_dispatch_workspace(n_rows, top_k, n_experts, device=None):
    """Bytes of workspace of im_dispatch_plan; as im_linear_workspace."""
    d = ImDispatchDesc(n_rows, top_k, n_experts, 0, 1, 0, 1, 1, 1)
    return _size_of(_dispatch_size, d, False, device)


def im_dispatch_plan(expert, offsets, slot, workspace=None, error=None, stream=None):
    """Places of the pairs of expert (int32 [n, top_k], -1: none) ordered by expert: slot
    like expert, and offsets int32 [experts + 1], the groups of the layers that follow."""
    if not expert.is_cuda:
        _bad(f"expert is on {expert.device}, a GPU is expected")
    if not _KINDS:
        _kinds()
    on, i32 = expert.get_device(), _KINDS["i32"]
    n, k = _matrix_of(expert, "expert")
    E = offsets.numel() - 1
    d, key = _desc(_DISPATCH, n, k, E, 0, 1, 0, 1, 1, 1), (4, on, n, k, E)
    ws, at, size = None, None, 0
    if _SIZES.get(key) != 0:
        ws, at, size = _workspace(_dispatch_size, ImDispatchDesc.from_buffer_copy(d), key, 0, workspace, expert.device,
                                  stream)
    _run(on, stream, (_learn or load_learn()).im_dispatch_plan, d, _at(expert, "expert", i32, on, n * k),
         _at(offsets, "offsets", i32, on, E + 1), _at(slot, "slot", i32, on, n * k), at, size,
         _at(error, "error", i32, on, 1))


def _exchange(rows, rows_name, slots, slots_name, slot, dslots=None, codes=False):
    """Description of an exchange between rows [n, dim] and slots' rows [n_slots, dim], the device's
    number and the slots' pointer."""
    dt = rows.dtype
    if not _KINDS:
        _kinds()
    if codes and dt is _KINDS["i8"] and rows.is_cuda:
        kind, on = IM_CODES, rows.get_device()
    else:
        kind, on = _first(rows, rows_name)
    n, dim = _matrix_of(rows, rows_name)
    k = _matrix_of(slot, "slot")[1]
    if slots is None:
        slots, slots_name = dslots, "dys"
    m, ld_slot, ld_dslot = 0, dim, dim
    if slots is not None:
        m = _matrix_of(slots, slots_name)[0]
        ld_slot = _ld(slots, slots_name, dt, on, m, dim)
    if dslots is not None:
        ld_dslot = _ld(dslots, "dys", dt, on, m, dim)
    d = _desc(_DISPATCH, n, k, 1, m, dim, kind, _ld(rows, rows_name, dt, on, n, dim), ld_slot, ld_dslot)
    return d, on, _at(slot, "slot", _KINDS["i32"], on, n * k)


def im_dispatch_forward(x, slot, xs, error=None, stream=None):
    """xs[slot[i, c]] = x[i]: rows to their places (float32, bfloat16, or the int8 codes of
    packed rows; rows of xs that no slot names stay as they are). Rows may be strided."""
    d, on, ps = _exchange(x, "x", xs, "xs", slot, codes=True)
    _run(on, stream, (_learn or load_learn()).im_dispatch_forward, d, x.data_ptr(), ps, xs.data_ptr(),
         _at(error, "error", _KINDS["i32"], on, 1))


def im_dispatch_backward(dxs, slot, dx, error=None, stream=None):
    """dx[i] = sum of dxs[slot[i, c]] over c."""
    d, on, ps = _exchange(dx, "dx", dxs, "dxs", slot)
    _run(on, stream, (_learn or load_learn()).im_dispatch_backward, d, dxs.data_ptr(), ps, dx.data_ptr(),
         _at(error, "error", _KINDS["i32"], on, 1))


def im_combine_forward(ys, slot, weight, y, error=None, stream=None):
    """y[i] = sum of weight[i, c] ys[slot[i, c]] over c (weight float32 like slot)."""
    d, on, ps = _exchange(y, "y", ys, "ys", slot)
    _run(on, stream, (_learn or load_learn()).im_combine_forward, d, ys.data_ptr(), ps,
         _at(weight, "weight", _KINDS["f32"], on, slot.numel()), y.data_ptr(), _at(error, "error", _KINDS["i32"], on, 1))


def im_combine_backward(dy, ys, slot, weight, dys=None, dweight=None, error=None, stream=None):
    """Gradients of im_combine_forward: dys[slot[i, c]] = weight[i, c] dy[i] and dweight
    (float32 like slot); None skips one."""
    if dweight is not None and ys is None:
        _bad("dweight needs ys")
    d, on, ps = _exchange(dy, "dy", ys, "ys", slot, dys)
    f32, pairs = _KINDS["f32"], slot.numel()
    _run(on, stream, (_learn or load_learn()).im_combine_backward, d, dy.data_ptr(),
         None if ys is None else ys.data_ptr(), ps, _at(weight, "weight", f32, on, pairs),
         None if dys is None else dys.data_ptr(), _at(dweight, "dweight", f32, on, pairs),
         _at(error, "error", _KINDS["i32"], on, 1))


def _rows(x, codes, scale, keep):
    kind, on = _first(x, "x")
    n, dim = _matrix_of(x, "x")
    d = _desc(_ROWS, n, dim, kind, 1 if keep else 0, _ld(x, "x", x.dtype, on, n, dim),
              _ld(codes, "codes", _KINDS["i8"], on, n, dim))
    return d, on, _at(scale, "scale", _KINDS["f32"], on, n)


def im_rows_pack(x, codes, scale, keep=False, stream=None):
    """Rows in 8 bits: codes int8 [n, dim] and scale float32 [n] of x [n, dim] (float32 or
    bfloat16), x = scale code up to half a scale. keep: what is not zero gets a code
    that is not. Rows of x and codes may be strided."""
    d, on, ps = _rows(x, codes, scale, keep)
    _run(on, stream, (_learn or load_learn()).im_rows_pack, d, x.data_ptr(), codes.data_ptr(), ps)


def im_rows_unpack(codes, scale, x, stream=None):
    """x = scale code in float32, rounded to its type."""
    d, on, ps = _rows(x, codes, scale, False)
    _run(on, stream, (_learn or load_learn()).im_rows_unpack, d, codes.data_ptr(), ps, x.data_ptr())


def im_linear_workspace_packed(n_rows, in_dim, out_dim, dtype, n_groups=1, backward=False, device=None):
    """Bytes of workspace of im_linear_forward_packed, or im_linear_backward_packed; as im_linear_workspace."""
    d = ImLinearDesc(n_groups, n_rows, in_dim, out_dim, _kind_of(dtype), 0, 0, 0, in_dim, out_dim, in_dim)
    return _size_of((_learn or load_learn()).im_linear_workspace_packed, d, backward, device)


def _groups_of(W, dtype, index, cols):
    """Groups and rows of contiguous weights [groups, rows, cols] or [rows, cols]."""
    if W.dtype is dtype and W.get_device() == index and W.is_contiguous():
        shape = W.shape
        if len(shape) == 3 and shape[2] == cols:
            return shape[0], shape[1]
    return _weights(W, dtype, _cuda(index), cols)


def _offsets_at(offsets, G, index):
    if offsets is None and G != 1:
        _bad("offsets are needed for more than one group")
    return _at(offsets, "offsets", _KINDS["i32"], index, G + 1)


def im_linear_forward_packed(x, x_scale, W, W_scale, b, y, offsets=None, relu=False, workspace=None, error=None,
                             stream=None):
    """y = act(x_scale W_scale (x W_g^T) + b_g) from packed rows x (int8 [n, in], x_scale
    float32 [n]) and packed weights W (int8 [groups, out, in] or [out, in], W_scale float32
    [groups, out]); y float32 or bfloat16 [n, out]. Rows of x and y may be strided."""
    kind, on = _first(y, "y")
    f32, i8 = _KINDS["f32"], _KINDS["i8"]
    n, k = _matrix_of(x, "x")
    G, m = _groups_of(W, i8, on, k)
    d = _desc(_LINEAR, G, n, k, m, kind, 1 if relu else 0, 0, 0, _ld(x, "x", i8, on, n, k),
              _ld(y, "y", y.dtype, on, n, m), 0)
    L, key = _learn or load_learn(), (5, on, G, n, k, m, kind)
    ws, at, size = None, None, 0
    if _SIZES.get(key) != 0:
        ws, at, size = _workspace(L.im_linear_workspace_packed, ImLinearDesc.from_buffer_copy(d), key, 0, workspace,
                                  y.device, stream)
    _run(on, stream, L.im_linear_forward_packed, d, _offsets_at(offsets, G, on), x.data_ptr(),
         _at(x_scale, "x_scale", f32, on, n), W.data_ptr(), _at(W_scale, "W_scale", f32, on, G * m),
         _at(b, "b", f32, on, G * m), y.data_ptr(), at, size, _at(error, "error", _KINDS["i32"], on, 1))


def im_linear_backward_packed(dy, x, x_scale, W, dx=None, dW=None, db=None, offsets=None, relu_in=False,
                              workspace=None, error=None, stream=None):
    """Gradients of a layer as im_linear_backward's, with its input x kept as packed rows
    (int8 [n, in], x_scale float32 [n]). relu_in: dx is zero where x's code is not above 0."""
    kind, on = _first(dy, "dy")
    dt, f32 = dy.dtype, _KINDS["f32"]
    n, m = _matrix_of(dy, "dy")
    k = _matrix_of(x, "x")[1]
    G, rows = _groups_of(W, dt, on, k)
    if rows != m:
        _bad(f"W has {rows} outputs, dy {m}")
    d = _desc(_LINEAR, G, n, k, m, kind, 0, 1 if relu_in else 0, 0, _ld(x, "x", _KINDS["i8"], on, n, k),
              _ld(dy, "dy", dt, on, n, m), k if dx is None else _ld(dx, "dx", dt, on, n, k))
    L, key = _learn or load_learn(), (6, on, G, n, k, m, kind)
    ws, at, size = None, None, 0
    if _SIZES.get(key) != 0:
        ws, at, size = _workspace(L.im_linear_workspace_packed, ImLinearDesc.from_buffer_copy(d), key, 1, workspace,
                                  dy.device, stream)
    _run(on, stream, L.im_linear_backward_packed, d, _offsets_at(offsets, G, on), dy.data_ptr(), x.data_ptr(),
         _at(x_scale, "x_scale", f32, on, n), W.data_ptr(), None if dx is None else dx.data_ptr(),
         _at(dW, "dW", dt, on, G * m * k), _at(db, "db", f32, on, G * m), at, size,
         _at(error, "error", _KINDS["i32"], on, 1))


# Plans whose AdamW was dropped. To free one synchronises the device, which would spoil a graph
# capture wherever the garbage collector happens to run: the next plan's creation, which
# synchronises itself, frees them.
_dropped = []


def _free_dropped():
    while _dropped:
        load_learn().im_adamw_destroy(_dropped.pop())


class AdamW:
    """AdamW over a list of tensors, one launch a step.

    tensors: dicts of contiguous device tensors of the same size
      param   float32 parameters
      grad    float32 or bfloat16 gradients (one type for the whole list)
      m, v    states: float32 (bits = 32), or float8_e4m3fn codes of m and
              sqrt(v) (bits = 8)
      m_scale, v_scale   bits = 8: float32 [ceil(n / 256)]
      copy    optional bfloat16 tensor that receives the rounded parameters
      decay   whether weight decay applies (default True)
    They are kept alive by this object and keep their places. States that are all
    zero start a run. Creating a plan and close() synchronise (not while a graph is
    captured); a graph with a step in it needs the plan for its replays."""

    def __init__(self, tensors, bits=32, stream=None):
        self.h = None
        if bits not in (32, 8):
            _bad("bits is 32 or 8")
        L = load_learn()
        tensors = [dict(t) for t in tensors]
        kind, dev = IM_F32, None
        table = (ImAdamwTensor * max(1, len(tensors)))()
        for i, t in enumerate(tensors):
            p, g = t["param"], t["grad"]
            _kind(p, f"param {i}")
            k = _kind(g, f"grad {i}")
            if i and (k != kind or p.device != dev):
                _bad(f"tensor {i}: another gradient type or device than the first tensor's")
            kind, dev = k, p.device
            n, f32 = p.numel(), _KINDS["f32"]
            st, blocks = (f32 if bits == 32 else _KINDS["fp8"]), -(-n // IM_STATE_BLOCK)
            if bits == 8 and (t.get("m_scale") is None or t.get("v_scale") is None):
                _bad(f"tensor {i}: 8-bit states need m_scale and v_scale")
            copy = t.get("copy")
            table[i] = ImAdamwTensor(_flat(p, f"param {i}", f32, dev, n), _flat(g, f"grad {i}", g.dtype, dev, n),
                                     _flat(t["m"], f"m {i}", st, dev, n), _flat(t["v"], f"v {i}", st, dev, n),
                                     _flat(t.get("m_scale"), f"m_scale {i}", f32, dev, blocks),
                                     _flat(t.get("v_scale"), f"v_scale {i}", f32, dev, blocks),
                                     None if copy is None else _flat(copy, f"copy {i}", _bf16(), dev, n), n,
                                     1 if t.get("decay", True) else 0, 0)
        self.tensors, self.device, self.bits = tensors, dev, bits
        out = _P()
        _free_dropped()
        with _On(_index(dev)):
            _done(L.im_adamw_create(table, len(tensors), bits, kind, _stream(stream), ctypes.byref(out)))
        self.h = out

    def step(self, step, lr, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, scale=None, stream=None):
        """One step. step: int64 [1] on the device, the steps done, counted up by
        the call; scale: float32 [1] on the device that multiplies the gradients."""
        if not self.h:
            _bad("the plan is closed")
        dev = step.device if self.device is None else self.device
        _kind_checked(dev)
        with _On(dev.index):
            _done(_learn.im_adamw_step(self.h, float(lr), float(betas[0]), float(betas[1]), float(eps),
                                       float(weight_decay), _flat(step, "step", _KINDS["i64"], dev, 1),
                                       _flat(scale, "scale", _KINDS["f32"], dev, 1), _stream(stream)))

    def close(self):
        if self.h:
            load_learn().im_adamw_destroy(self.h)
            self.h = None

    def __del__(self):
        if getattr(self, "h", None) and _dropped is not None:   # None: the interpreter ends
            _dropped.append(self.h)
            self.h = None


def _bf16():
    import torch
    return torch.bfloat16


def _index(dev):
    import torch
    return torch.cuda.current_device() if dev is None else dev.index


def _kind_checked(dev):
    if dev.type != "cuda":
        _bad(f"step is on {dev}, a GPU is expected")
