"""Microscaled (MX) tensors: weights in 4 bits and activation checkpoints in 8, as they cross the encrypted
link, quantised, multiplied and differentiated by the library's HIP kernels. Argument marshalling only.

The format, the rounding and the sums are documented in include/fastrack.h. A float operand is a CUDA tensor
in bfloat16, float16 or float32 whose last axis is dense; the axes before it are taken together as its rows, which
may be any equal distance apart (a slice of a wider tensor, or one row expanded). Work is enqueued on the current
stream or on `stream`, which waits for nothing on the current one: order it after what it reads, and whoever reads the
results after it. New results may be used on either. A float tensor's NaN and infinity go where the formulas put
them; in a quantised block they make the whole block NaN.

Nothing here is recorded by autograd: a result needs no gradient, whatever its operands do, and a `backward()` ends at it.
Training calls the gradients by name (mx4_linear_grad_input, mx8_weight_grad, mx8_act_grad), in the backward of a
torch.autograd.Function of its own or, as examples/offloaded_layer.py does, in order.
"""
import ctypes as _ct

import torch as _torch

from . import EINVAL, _call, _check, _fresh, _raw_stream, lib

_Tensor, _uint8, _int8 = _torch.Tensor, _torch.uint8, _torch.int8
_TYPES = {_torch.bfloat16: 0, _torch.float16: 1, _torch.float32: 2}
_ACTS = {"silu": 0, "gelu": 1}
_LINEAR, _GRAD_INPUT, _WEIGHT_GRAD, _LINEAR_MX = range(4)


def _bind(L):
    vp, u64, u32 = _ct.c_void_p, _ct.c_uint64, _ct.c_uint32
    L.fastrack_mx_code_bytes.argtypes = [u32, u64, u64]
    L.fastrack_mx_code_bytes.restype = u64
    L.fastrack_mx_scale_bytes.argtypes = [u64, u64]
    L.fastrack_mx_scale_bytes.restype = u64
    L.fastrack_mx_work_bytes.argtypes = [u32, u32, vp, u64, u64, u64, u64]
    L.fastrack_mx_work_bytes.restype = u64
    L.fastrack_mx_quantize.argtypes = [u32, u32, vp, u64, u64, u64, vp, vp, vp]
    L.fastrack_mx_dequantize.argtypes = [u32, vp, vp, u64, u64, u32, vp, u64, vp]
    L.fastrack_mx_act.argtypes = [u32, u32, vp, u64, vp, u64, u64, u64, vp, u64, vp, vp, vp, vp, vp]
    L.fastrack_mx_act_grad.argtypes = [u32, u32, vp, u64, vp, vp, vp, vp, u64, u64, vp, u64, vp, u64, vp]
    product = [u32, vp, u64, vp, vp, u64, u64, u64, u32, vp, u64, vp, u64, vp]
    L.fastrack_mx_linear.argtypes = product
    L.fastrack_mx_linear_grad_input.argtypes = product
    L.fastrack_mx_weight_grad.argtypes = product[:11] + [u32] + product[11:]
    L.fastrack_mx_linear_mx.argtypes = [vp, vp, vp, vp, u64, u64, u64, u32, vp, u64, vp, u64, vp]
    for fn in (L.fastrack_mx_quantize, L.fastrack_mx_dequantize, L.fastrack_mx_act, L.fastrack_mx_act_grad,
               L.fastrack_mx_linear, L.fastrack_mx_linear_grad_input, L.fastrack_mx_weight_grad, L.fastrack_mx_linear_mx):
        fn.restype = _ct.c_int


class _MX:
    """rows x cols values in blocks of 32 along a row: `codes` (rows, blocks * block_bytes) and `scales`
    (rows, blocks), contiguous. The codes past `cols` in a row's last block must be 0."""
    __slots__ = ("codes", "scales", "rows", "cols")

    def __init__(self, codes, scales, cols):
        name = type(self).__name__
        cols = int(cols)
        blocks = -(-cols // 32)
        for t, what, dtype, width in ((codes, "codes", self.code_type, blocks * self.block_bytes),
                                      (scales, "scales", _uint8, blocks)):
            if not isinstance(t, _Tensor):
                raise ValueError("%s %s must be a torch tensor" % (name, what))
            if t.dtype != dtype:
                raise ValueError("%s %s must be %s, got %s" % (name, what, dtype, t.dtype))
            if t.dim() != 2 or t.shape[1] != width or t.shape[0] != codes.shape[0]:
                raise ValueError("%s %s of %d columns must have shape (rows, %d), got %s"
                                 % (name, what, cols, width, tuple(t.shape)))
            if not t.is_contiguous():
                raise ValueError("%s %s must be contiguous" % (name, what))
        if cols < 0:
            raise ValueError("cols must not be negative")
        if codes.device != scales.device:
            raise ValueError("%s codes are on %s, scales on %s" % (name, codes.device, scales.device))
        self.codes, self.scales, self.rows, self.cols = codes, scales, codes.shape[0], cols

    @classmethod
    def nbytes(cls, rows, cols):
        """Bytes of a rows x cols tensor in one buffer (see view)."""
        return rows * -(-cols // 32) * (cls.block_bytes + 1)

    @classmethod
    def view(cls, buf, rows, cols):
        """The tensor held in one contiguous uint8 buffer, its codes first and then its scales: what is encrypted and
        sent as one message, and used in place once decrypted."""
        if not isinstance(buf, _Tensor) or buf.dtype != _uint8 or not buf.is_contiguous():
            raise ValueError("buf must be a contiguous uint8 tensor")
        rows, cols = int(rows), int(cols)
        if rows < 0 or cols < 0 or buf.numel() != cls.nbytes(rows, cols):
            raise ValueError("a %d x %d %s takes %d bytes, buf holds %d"
                             % (rows, cols, cls.__name__, cls.nbytes(rows, cols), buf.numel()))
        blocks = -(-cols // 32)
        flat, cut = buf.view(-1), rows * blocks * cls.block_bytes
        return cls(flat[:cut].view(cls.code_type).view(rows, blocks * cls.block_bytes), flat[cut:].view(rows, blocks), cols)

    @classmethod
    def empty(cls, rows, cols, device=None):
        """An uninitialised rows x cols tensor in one buffer."""
        device = _torch.device("cuda", _torch.cuda.current_device()) if device is None else device
        return cls.view(_torch.empty(cls.nbytes(rows, cols), dtype=_uint8, device=device), rows, cols)

    @classmethod
    def _new(cls, rows, cols, device, stream):
        """What a call returns: codes and scales of their own (a call's shapes need no check, and two allocations cost
        a third of cutting one buffer into views: 2.3 and 6.4 us)."""
        q, blocks = object.__new__(cls), -(-cols // 32)
        q.codes = _fresh((rows, blocks * cls.block_bytes), device, stream, cls.code_type)
        q.scales = _fresh((rows, blocks), device, stream)
        q.rows, q.cols = rows, cols
        return q

    def __repr__(self):
        return "%s(%d x %d, %s)" % (type(self).__name__, self.rows, self.cols, self.codes.device)


class MX4(_MX):
    """A matrix in 4-bit microscaled form (E2M1 codes, two to a byte, and a scale byte per 32): codes uint8."""
    __slots__ = ()
    format, block_bytes, code_type = 4, 16, _uint8


class MX8(_MX):
    """A matrix in 8-bit microscaled form (int8 codes and a scale byte per 32): codes int8."""
    __slots__ = ()
    format, block_bytes, code_type = 8, 32, _int8


def _float(t, what, idx=None):
    """(address, row stride, rows, columns, type) of a float operand."""
    if not isinstance(t, _Tensor):
        raise ValueError("%s must be a torch tensor" % what)
    code = _TYPES.get(t.dtype)
    if code is None:
        raise ValueError("%s must be bfloat16, float16 or float32, got %s" % (what, t.dtype))
    at = t.get_device()
    if at < 0:
        raise ValueError("%s must be a CUDA tensor" % what)
    if idx is not None and at != idx:
        raise ValueError("%s is on %s, the other operands on cuda:%d" % (what, t.device, idx))
    shape = t.shape
    if len(shape) == 2:
        rows, cols = shape
        ld, step = t.stride()
    elif len(shape) == 0:
        raise ValueError("%s must have at least one axis" % what)
    else:
        cols, step = shape[-1], t.stride(-1)
        if cols > 1 and step != 1:
            raise ValueError("%s must be dense along its last axis" % what)
        rows = 1
        for s in shape[:-1]:
            rows *= s
        ld = cols
        if rows > 1:   # the leading axes as one: all rows the same distance apart
            lead = [(n, s) for n, s in zip(shape[:-1], t.stride()[:-1]) if n != 1]
            ld = lead[-1][1]
            for (_, outer), (n, inner) in zip(lead, lead[1:]):
                if outer != n * inner:
                    raise ValueError("%s: its leading axes do not form rows of one stride" % what)
    if cols > 1 and step != 1:
        raise ValueError("%s must be dense along its last axis" % what)
    return t.data_ptr(), (ld if rows > 1 else cols), rows, cols, code


def _out(t, what, shape, dtype, device, idx, stream):
    """The caller's output, checked, or a new one; (tensor, address, row stride)."""
    if t is None:
        t = _fresh(shape, device, stream, dtype)
        return t, t.data_ptr(), shape[-1]
    p, ld, _, _, _ = _float(t, what, idx)
    if t.shape != _torch.Size(shape):
        raise ValueError("%s must have shape %s, got %s" % (what, tuple(shape), tuple(t.shape)))
    if dtype is not None and t.dtype != dtype:
        raise ValueError("%s must be %s, got %s" % (what, dtype, t.dtype))
    return t, p, ld


def _mx(q, what, cls, idx=None, rows=None, cols=None):
    if type(q) is not cls:
        raise ValueError("%s must be an %s" % (what, cls.__name__))
    at = q.codes.get_device()
    if at >= 0 and idx is None and rows is None and cols is None:
        return q
    if at < 0:
        raise ValueError("%s must be a CUDA tensor" % what)
    if idx is not None and at != idx:
        raise ValueError("%s is on %s, the other operands on cuda:%d" % (what, q.codes.device, idx))
    if (rows is not None and q.rows != rows) or (cols is not None and q.cols != cols):
        raise ValueError("%s is %d x %d, the call needs %s x %s"
                         % (what, q.rows, q.cols, "any" if rows is None else rows, "any" if cols is None else cols))
    return q


def _dtype(dtype, out, default):
    """The type that a call's result is to have: asked for, or that of the output given, or the call's own."""
    if dtype is None:
        dtype = out.dtype if isinstance(out, _Tensor) else default
    if dtype not in _TYPES:
        raise ValueError("dtype must be bfloat16, float16 or float32, got %s" % dtype)
    return dtype


def _act(act):
    if act not in _ACTS:
        raise ValueError("act must be one of %s, got %r" % (", ".join(sorted(_ACTS)), act))
    return _ACTS[act]


def _new_mx(q, what, cls, rows, cols, device, idx, stream):
    if q is None:
        return cls._new(rows, cols, device, stream)
    return _mx(q, what, cls, idx, rows, cols)


def _quantize(cls, x, out, stream):
    p, ld, rows, cols, code = _float(x, "x")
    idx = x.get_device()
    out = _new_mx(out, "out", cls, rows, cols, x.device, idx, stream)
    _call(lib().fastrack_mx_quantize, idx, cls.format, code, p, ld, rows, cols, out.codes.data_ptr(), out.scales.data_ptr(),
          _raw_stream(stream, idx))
    return out


def _dequantize(cls, q, dtype, out, stream):
    _mx(q, "q", cls)
    device, idx = q.codes.device, q.codes.get_device()
    dtype = _dtype(dtype, out, _torch.bfloat16)
    out, p, ld = _out(out, "out", (q.rows, q.cols), dtype, device, idx, stream)
    _call(lib().fastrack_mx_dequantize, idx, cls.format, q.codes.data_ptr(), q.scales.data_ptr(), q.rows, q.cols, _TYPES[dtype],
          p, ld, _raw_stream(stream, idx))
    return out


def mx4_quantize(x, out=None, stream=None):
    """x (..., cols) as an MX4 of its rows: nearest code, ties to the even one, saturated at 6 times the scale.
    To send the result as one message give out=MX4.view(buf, rows, cols) of the message's buffer."""
    return _quantize(MX4, x, out, stream)


def mx8_quantize(x, out=None, stream=None):
    """x (..., cols) as an MX8 of its rows: the checkpoint of an activation in 8 bits."""
    return _quantize(MX8, x, out, stream)


def mx4_dequantize(q, dtype=None, out=None, stream=None):
    """The values (rows, cols) of an MX4, bfloat16 unless told otherwise (exact; float16 rounds and can overflow)."""
    return _dequantize(MX4, q, dtype, out, stream)


def mx8_dequantize(q, dtype=None, out=None, stream=None):
    """The values (rows, cols) of an MX8, bfloat16 unless told otherwise (exact; float16 rounds and can overflow)."""
    return _dequantize(MX8, q, dtype, out, stream)


def _product(fn, op, a, work, device, idx, stream, head, tail):
    """Run a product's C entry: its arguments are head, the sizes and tail, the workspace and the stream. a is (type, address,
    stride, m, n, k) of what its workspace depends on. Most small products need none, so the call is made without one
    first; where it is refused for that, nothing was enqueued, and it is made again with one."""
    raw = _raw_stream(stream, idx)
    if work is not None:
        if not isinstance(work, _Tensor) or work.dtype != _uint8 or not work.is_contiguous() or work.get_device() != idx:
            raise ValueError("work must be a contiguous uint8 tensor on the operands' device")
        _call(fn, idx, *head, *a[3:], *tail, work.data_ptr(), work.numel(), raw)
        return
    if _torch._C._cuda_getDevice() != idx:
        with _torch.cuda.device(idx):
            return _product(fn, op, a, work, device, idx, stream, head, tail)
    rc = fn(*head, *a[3:], *tail, None, 0, raw)
    if rc == EINVAL:
        need = lib().fastrack_mx_work_bytes(op, *a)
        if need:
            work = _fresh(need, device, stream)
            rc = fn(*head, *a[3:], *tail, work.data_ptr(), need, raw)
    if rc:
        _check(rc)


def mx4_linear(x, w, dtype=None, out=None, work=None, stream=None):
    """y = x W^T for a layer's weights w, an MX4 of (outputs, inputs): x (..., inputs) -> (..., outputs), in x's type
    unless `dtype` says otherwise. x may be an MX4 (tokens, inputs) too; y is then bfloat16 by default.
    `work` is a uint8 buffer to use as workspace; without it the call allocates what it needs."""
    w = _mx(w, "w", MX4)
    if isinstance(x, _MX):
        _mx(x, "x", MX4, w.codes.get_device(), cols=w.cols)
        device, idx, m = w.codes.device, w.codes.get_device(), x.rows
        dtype = _dtype(dtype, out, _torch.bfloat16)
        out, p, ld = _out(out, "out", (m, w.rows), dtype, device, idx, stream)
        _product(lib().fastrack_mx_linear_mx, _LINEAR_MX, (0, None, 0, m, w.rows, w.cols), work, device, idx, stream,
                 (x.codes.data_ptr(), x.scales.data_ptr(), w.codes.data_ptr(), w.scales.data_ptr()), (_TYPES[dtype], p, ld))
    else:
        device, idx = w.codes.device, w.codes.get_device()
        xp, xld, m, k, code = _float(x, "x", idx)
        if k != w.cols:
            raise ValueError("x has %d columns, the weights %d" % (k, w.cols))
        dtype = _dtype(dtype, out, x.dtype)
        out, p, ld = _out(out, "out", x.shape[:-1] + (w.rows,), dtype, device, idx, stream)
        _product(lib().fastrack_mx_linear, _LINEAR, (code, xp, xld, m, w.rows, k), work, device, idx, stream,
                 (code, xp, xld, w.codes.data_ptr(), w.scales.data_ptr()), (_TYPES[dtype], p, ld))
    return out


def mx4_linear_grad_input(dy, w, dtype=None, out=None, work=None, stream=None):
    """dx = dy W, the gradient of mx4_linear with respect to x: dy (..., outputs) -> (..., inputs), in dy's type
    unless `dtype` says otherwise."""
    w = _mx(w, "w", MX4)
    device, idx = w.codes.device, w.codes.get_device()
    yp, yld, m, n, code = _float(dy, "dy", idx)
    if n != w.rows:
        raise ValueError("dy has %d columns, the weights %d rows" % (n, w.rows))
    dtype = _dtype(dtype, out, dy.dtype)
    out, p, ld = _out(out, "out", dy.shape[:-1] + (w.cols,), dtype, device, idx, stream)
    _product(lib().fastrack_mx_linear_grad_input, _GRAD_INPUT, (code, yp, yld, m, n, w.cols), work, device, idx, stream,
             (code, yp, yld, w.codes.data_ptr(), w.scales.data_ptr()), (_TYPES[dtype], p, ld))
    return out


def mx8_weight_grad(dy, saved, dtype=None, out=None, accumulate=False, work=None, stream=None):
    """dW = dy^T x^ for a linear layer's kept input `saved`, an MX8 of (tokens, inputs): dy (..., outputs) ->
    (outputs, inputs), float32 unless `dtype` says otherwise. accumulate=True adds to `out` (float32)."""
    saved = _mx(saved, "saved", MX8)
    device, idx = saved.codes.device, saved.codes.get_device()
    yp, yld, m, n, code = _float(dy, "dy", idx)
    if m != saved.rows:
        raise ValueError("dy has %d rows, the kept input %d" % (m, saved.rows))
    dtype = _dtype(dtype, out, _torch.float32)
    if accumulate and (out is None or dtype != _torch.float32):
        raise ValueError("accumulate=True needs a float32 out to add to")
    out, p, ld = _out(out, "out", (n, saved.cols), dtype, device, idx, stream)
    _product(lib().fastrack_mx_weight_grad, _WEIGHT_GRAD, (code, yp, yld, m, n, saved.cols), work, device, idx, stream,
             (code, yp, yld, saved.codes.data_ptr(), saved.scales.data_ptr()),
             (_TYPES[dtype], p, ld, 1 if accumulate else 0))
    return out


def mx8_act(x, gate=None, act="silu", out=None, saved=None, saved_gate=None, stream=None):
    """y = f(x), or f(x) * gate, and what the gradient needs kept in 8 bits: returns (y, MX8 of x, MX8 of gate or None).
    act is "silu" or "gelu" (with the error function). x and gate may be halves of one wider tensor."""
    a = _act(act)
    p, ld, rows, cols, code = _float(x, "x")
    device, idx = x.device, x.get_device()
    gp, gld = None, 0
    if gate is not None:
        gp, gld, _, _, gcode = _float(gate, "gate", idx)
        if gate.shape != x.shape or gcode != code:
            raise ValueError("gate must have the shape and type of x: %s %s, got %s %s"
                             % (tuple(x.shape), x.dtype, tuple(gate.shape), gate.dtype))
    elif saved_gate is not None:
        raise ValueError("saved_gate without a gate")
    out, yp, yld = _out(out, "out", x.shape, x.dtype, device, idx, stream)
    saved = _new_mx(saved, "saved", MX8, rows, cols, device, idx, stream)
    if gate is not None:
        saved_gate = _new_mx(saved_gate, "saved_gate", MX8, rows, cols, device, idx, stream)
    if rows and cols:
        _call(lib().fastrack_mx_act, idx, a, code, p, ld, gp, gld, rows, cols, yp, yld, saved.codes.data_ptr(),
              saved.scales.data_ptr(), None if gate is None else saved_gate.codes.data_ptr(),
              None if gate is None else saved_gate.scales.data_ptr(), _raw_stream(stream, idx))
    return out, saved, saved_gate


def mx8_act_grad(dy, saved, saved_gate=None, act="silu", out=None, out_gate=None, stream=None):
    """(dx, dgate) of mx8_act from what it kept; dgate is None where there was no gate. Both in dy's type."""
    a = _act(act)
    saved = _mx(saved, "saved", MX8)
    device, idx = saved.codes.device, saved.codes.get_device()
    p, ld, rows, cols, code = _float(dy, "dy", idx)
    if rows != saved.rows or cols != saved.cols:
        raise ValueError("dy is %d x %d, the kept x %d x %d" % (rows, cols, saved.rows, saved.cols))
    out, xp, xld = _out(out, "out", dy.shape, dy.dtype, device, idx, stream)
    qg = gp = None
    gld = 0
    if saved_gate is not None:
        qg = _mx(saved_gate, "saved_gate", MX8, idx, rows, cols)
        out_gate, gp, gld = _out(out_gate, "out_gate", dy.shape, dy.dtype, device, idx, stream)
    elif out_gate is not None:
        raise ValueError("out_gate without a saved gate")
    if rows and cols:
        _call(lib().fastrack_mx_act_grad, idx, a, code, p, ld, saved.codes.data_ptr(), saved.scales.data_ptr(),
              None if qg is None else qg.codes.data_ptr(), None if qg is None else qg.scales.data_ptr(), rows, cols, xp, xld,
              gp, gld, _raw_stream(stream, idx))
    return out, out_gate
