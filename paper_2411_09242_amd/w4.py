"""Products with matrices held in 4 bits, for the few rows of a decode step
(ctypes binding of include/fluid_w4.h).

    w4_pack(m, group)                a matrix [rows, cols] into 4 bits: a W4
    w4_read(w, out)                  its values as an ordinary tensor
    w4_matmul(x, w, gate, add, out)  x W^T, with a gate's SiLU and a residual

Matrices are torch tensors in fp32 or bf16 on the GPU with contiguous channels.
Calls enqueue a kernel on torch's current stream, or on ``stream``, and return
without waiting; streams, errors and tensors that want gradients are as in
``attention``.
"""
from __future__ import annotations

import ctypes as C

from . import fluid
from .attention import (_addr, _calls, _check_grad, _device_of, _as_stream, _form, _keep, _launch, _raw_stream, _record,
                        _refuse, _stream, _torch, _workspace)

_VP, _I32, _U64 = C.c_void_p, C.c_int32, C.c_uint64


class W4Desc(C.Structure):
    _fields_ = [("rows", _I32), ("cols", _I32), ("group", _I32)]


class Matrix(C.Structure):
    _fields_ = [("dtype", _I32), ("rows", _I32), ("cols", _I32), ("stride", C.c_int64)]


_PROTOS = {
    "fluid_w4_bytes": [_VP] * 2,
    "fluid_w4_pack": [_VP] * 5,
    "fluid_w4_read": [_VP] * 5,
    "fluid_w4_matmul_workspace": [_VP, _VP, _I32, _VP],
    "fluid_w4_matmul": [_VP] * 10 + [_U64, _VP],
}
SYMBOLS = tuple(_PROTOS)

_bound = None


def _lib():
    """The library that ``fluid.load`` chose, with this header's prototypes."""
    global _bound
    lib = fluid._L()
    if _bound is not lib:
        for name, args in _PROTOS.items():
            f = getattr(lib, name)
            f.restype = C.c_int
            f.argtypes = args
        _bound = lib
    return lib


def _desc(rows, cols, group):
    for name, v in (("rows", rows), ("cols", cols), ("group", group)):
        if not 0 <= v < 1 << 31:
            _refuse(f"{name}: {v} is out of range")
    return W4Desc(rows, cols, group)


def w4_bytes(rows, cols, group):
    """Bytes that a matrix takes."""
    n = _U64()
    fluid._check(_lib().fluid_w4_bytes(_addr(_desc(rows, cols, group)), C.byref(n)))
    return n.value


class W4:
    """A matrix [rows, cols] held in 4 bits: its bytes, in the format of
    include/fluid_w4.h, and its sizes."""

    def __init__(self, packed, rows, cols, group):
        n = w4_bytes(rows, cols, group)
        if packed.dtype != _torch().uint8 or packed.dim() != 1 or packed.numel() != n or not packed.is_contiguous():
            _refuse(f"packed: {n} contiguous bytes are needed for [{rows}, {cols}] in groups of {group}")
        self.packed, self.rows, self.cols, self.group = packed, rows, cols, group
        self.desc = _desc(rows, cols, group)


def _matrix(t, name, device):
    """fluid_matrix of a tensor whose leading dimensions are rows at one
    distance, or a refusal."""
    torch = _torch()
    if t.dim() < 2:
        _refuse(f"{name}: a tensor [.., channels] of two dimensions or more is needed, got {t.dim()}")
    if t.get_device() != device:
        _refuse(f"{name}: on {t.device}, not on GPU {device}")
    if t.dtype not in (torch.float32, torch.bfloat16):
        _refuse(f"{name}: dtype must be float32 or bfloat16, got {t.dtype}")
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        _refuse(f"{name}: channels must be contiguous")
    rows, stride = 1, 0
    for n, s in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if n == 1:
            continue
        if rows > 1 and s != rows * stride:
            _refuse(f"{name}: rows must lie at one distance")
        if rows == 1:
            stride = s
        rows *= n
    if rows >= 1 << 31 or t.shape[-1] >= 1 << 31:
        _refuse(f"{name}: too large")
    return Matrix(fluid.F32 if t.dtype == torch.float32 else fluid.BF16, rows, t.shape[-1], stride)


def _check_w4(w, name, device):
    if not isinstance(w, W4):
        _refuse(f"{name}: a W4 is needed")
    if w.packed.get_device() != device:
        _refuse(f"{name}: on {w.packed.device}, not on GPU {device}")


def _w4_form(w):
    return (w.rows, w.cols, w.group, w.packed.get_device()) if isinstance(w, W4) else False


def _on(stream, device, make):
    """make() with what it allocates and fills on the call's stream."""
    if stream is None:
        return make()
    with _torch().cuda.stream(_as_stream(stream, device)):
        return make()


def w4_pack(m, group=128, stream=None):
    """The matrix m [rows, cols] in 4 bits, in groups of 32, 64 or 128 channels
    of a row."""
    _check_grad(m)
    dev = _device_of(m, "m")
    if m.dim() != 2:
        _refuse(f"m: a tensor [rows, cols] is needed, got {m.dim()} dimensions")
    md = _matrix(m, "m", dev)
    n = w4_bytes(m.shape[0], m.shape[1], group)
    packed = _on(stream, dev, lambda: _torch().empty(n, dtype=_torch().uint8, device=m.device))
    w = W4(packed, m.shape[0], m.shape[1], group)
    _launch(_lib().fluid_w4_pack, dev, _addr(w.desc), _addr(md), m.data_ptr(), packed.data_ptr(),
            _raw_stream(dev) if stream is None else _stream(stream, dev))
    if stream is not None:
        _record(stream, dev, m, packed)
    return w


def w4_read(w, out=None, dtype=None, stream=None):
    """w's values as a tensor [rows, cols] (of fp32, or ``dtype``), or into
    ``out``.  Returns it."""
    if not isinstance(w, W4):
        _refuse("w: a W4 is needed")
    dev = _device_of(w.packed, "w")
    if out is None:
        dtype = _torch().float32 if dtype is None else dtype
        out = _on(stream, dev, lambda: _torch().empty(w.rows, w.cols, dtype=dtype, device=w.packed.device))
    _check_grad(out)
    if out.dim() != 2:
        _refuse(f"out: a tensor [rows, cols] is needed, got {out.dim()} dimensions")
    od = _matrix(out, "out", dev)
    _launch(_lib().fluid_w4_read, dev, _addr(w.desc), w.packed.data_ptr(), _addr(od), out.data_ptr(),
            _raw_stream(dev) if stream is None else _stream(stream, dev))
    if stream is not None:
        _record(stream, dev, w.packed, out)
    return out


def _matmul_call(x, w, gate, add, out):
    dev = _device_of(x, "x")
    _check_w4(w, "w", dev)
    if gate is not None:
        _check_w4(gate, "gate", dev)
        if (gate.rows, gate.cols, gate.group) != (w.rows, w.cols, w.group):
            _refuse("gate: must have w's sizes and group")
    xd, od = _matrix(x, "x", dev), _matrix(out, "out", dev)
    shape = tuple(x.shape[:-1]) + (w.rows,)
    ad = None
    if add is not None:
        ad = _matrix(add, "add", dev)
        if tuple(add.shape) != shape:
            _refuse(f"add: {shape} is needed, got {tuple(add.shape)}")
    if tuple(out.shape) != shape:
        _refuse(f"out: {shape} is needed, got {tuple(out.shape)}")
    need = _need(w, xd, gate is not None)
    return (_lib(), dev, _addr(xd), None if ad is None else _addr(ad), _addr(od), need, (xd, ad, od))


def _need(w, xd, gated):
    n = _U64()
    fluid._check(_lib().fluid_w4_matmul_workspace(_addr(w.desc), _addr(xd), 1 if gated else 0, C.byref(n)))
    return n.value


def w4_matmul_workspace(x, w, gated=False):
    """Bytes of workspace that ``w4_matmul`` needs for these arguments."""
    dev = _device_of(x, "x")
    _check_w4(w, "w", dev)
    return _need(w, _matrix(x, "x", dev), gated)


def w4_matmul(x, w, gate=None, add=None, out=None, workspace=None, stream=None):
    """x W^T for x [.., cols] and the 4-bit matrix w [rows, cols]; with ``gate``, a
    matrix of w's sizes, SiLU(x gate^T) * (x W^T); plus ``add`` [.., rows] if there
    is one.  out may be ``add``; it is allocated by default.  Made for few rows.
    Returns out."""
    if out is None and isinstance(w, W4):
        dtype, shape = x.dtype, tuple(x.shape[:-1]) + (w.rows,)
        out = _on(stream if x.is_cuda else None, x.get_device(), lambda: _torch().empty(shape, dtype=dtype, device=x.device))
    if x.requires_grad or (out is not None and out.requires_grad) or (add is not None and add.requires_grad):
        _check_grad(x, *(t for t in (add, out) if t is not None))
    key = (fluid._lib, x.dtype, x.shape, x.stride(), x.get_device(), None if add is None else _form(add),
           None if out is None else _form(out), _w4_form(w), None if gate is None else _w4_form(gate), "w4")
    made = _calls.get(key)
    if made is None:
        made = _keep(key, _matmul_call(x, w, gate, add, out))
    lib, dev, xd, ad, od, need, _ = made
    keep, ws, ws_bytes = _workspace(need, workspace, dev, stream) if need else (None, None, 0)
    _launch(lib.fluid_w4_matmul, dev, C.addressof(w.desc), w.packed.data_ptr(),
            None if gate is None else gate.packed.data_ptr(), xd, x.data_ptr(), ad, None if add is None else add.data_ptr(),
            od, out.data_ptr(), ws, ws_bytes, _raw_stream(dev) if stream is None else _stream(stream, dev))
    if stream is not None:
        _record(stream, dev, x, add, out, w.packed, None if gate is None else gate.packed, workspace)
    del keep
    return out
