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
for the size of a workspace that a program keeps); AdamW holds an im_adamw plan."""
from __future__ import annotations

import ctypes
import os

from ._lib import HERE, IM_BF16, IM_EINVAL, IM_F32, IM_OK, IMError, _stream

LEARN_PATH = os.path.join(HERE, "libinframind_learn.so")
LEARN_EXPORTED = ("im_linear_workspace", "im_linear_forward", "im_linear_backward", "im_head_workspace",
                  "im_head_forward", "im_head_backward", "im_adamw_create", "im_adamw_step", "im_adamw_destroy",
                  "im_learn_last_error")
IM_MAX_GROUPS, IM_MAX_DIM, IM_MAX_CLASSES, IM_STATE_BLOCK = 1024, 65536, 1 << 22, 256

_P, _I32, _I64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64


class ImLinearDesc(ctypes.Structure):
    _fields_ = [("n_groups", _I32), ("n_rows", _I32), ("in_dim", _I32), ("out_dim", _I32), ("dtype", _I32),
                ("relu", _I32), ("relu_in", _I32), ("reserved", _I32), ("ld_x", _I64), ("ld_y", _I64), ("ld_dx", _I64)]


class ImHeadDesc(ctypes.Structure):
    _fields_ = [("n_groups", _I32), ("n_rows", _I32), ("dim", _I32), ("n_classes", _I32), ("dtype", _I32),
                ("relu_in", _I32), ("reserved0", _I32), ("reserved1", _I32), ("ld_h", _I64), ("ld_dh", _I64)]


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


def _matrix(t, name, dtype, device, rows, cols):
    """Row stride of a [rows, cols] tensor whose columns are contiguous."""
    if t.dtype is not dtype or t.device != device:
        _bad(f"{name} is {t.dtype} on {t.device}, {dtype} on {device} expected")
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != cols:
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


def _kind(t, name):
    """im_dtype of a tensor on a GPU."""
    if not _KINDS:
        import torch
        _KINDS.update({torch.float32: IM_F32, torch.bfloat16: IM_BF16, "f32": torch.float32, "i32": torch.int32,
                       "i64": torch.int64, "u8": torch.uint8, "fp8": torch.float8_e4m3fn})
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
