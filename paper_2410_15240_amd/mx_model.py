"""What stands around a model's layers, on microscaled (MX) tensors: the lookup of its first activations in a 4-bit
table, the norm between two blocks with its 8-bit checkpoint, and the loss over a 4-bit head without its logits, each
with its gradient. Argument marshalling only.

The formulas and the roundings are documented in include/fastrack.h; operands, streams and autograd are as in mx.py. The
table and the head may be one MX4: mx4_cross_entropy_grad gives the gradient of the head, and mx4_embedding_grad with
accumulate=True adds that of the lookup to it. `work` is a uint8 buffer to use as workspace; without it a call allocates
what it needs.
"""
import ctypes as _ct

import torch as _torch

from . import _call, _fresh, _raw_stream, lib
from .mx import _TYPES, MX4, MX8, _dtype, _float, _mx, _new_mx, _out, _Tensor, _uint8

_INDEX = {_torch.int32: 0, _torch.int64: 1}
_float32 = _torch.float32


def _bind(L):
    vp, u64, u32, f32 = _ct.c_void_p, _ct.c_uint64, _ct.c_uint32, _ct.c_float
    L.fastrack_mx_norm.argtypes = [u32, vp, u64, vp, u64, vp, u64, u64, u64, u32, vp, vp, f32, f32, vp, u64, vp, u64, vp, vp, vp,
                                   vp, vp, vp, vp, vp, vp]
    L.fastrack_mx_norm_grad_work_bytes.argtypes = [u64, u64, u32]
    L.fastrack_mx_norm_grad.argtypes = [u32, vp, u64, vp, u64, u64, u64, u32, vp, vp, f32, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                        u64, vp, u64, vp, u64, vp, vp, vp, u64, vp]
    L.fastrack_mx_embedding.argtypes = [u32, vp, u64, vp, vp, u64, u64, f32, u32, vp, u64, vp]
    L.fastrack_mx_embedding_grad_work_bytes.argtypes = [u64, u64, u64]
    L.fastrack_mx_embedding_grad.argtypes = [u32, vp, u32, vp, u64, u64, u64, u64, f32, u32, vp, u64, u32, vp, u64, vp]
    L.fastrack_mx_loss_work_bytes.argtypes = [u32, vp, u64, u64, u64, u64]
    L.fastrack_mx_loss.argtypes = [u32, vp, u64, vp, vp, u32, vp, u64, u64, u64, f32, vp, vp, vp, u64, vp]
    L.fastrack_mx_loss_grad_work_bytes.argtypes = [u32, vp, u64, u64, u64, u64, u32, u32, u32, u32]
    L.fastrack_mx_loss_grad.argtypes = [u32, vp, u64, vp, vp, vp, vp, u32, vp, vp, u64, vp, u64, u64, u64, f32, u32, vp, u64, u32,
                                        vp, u64, u32, vp, u64, vp]
    for fn in (L.fastrack_mx_norm, L.fastrack_mx_norm_grad, L.fastrack_mx_embedding, L.fastrack_mx_embedding_grad,
               L.fastrack_mx_loss, L.fastrack_mx_loss_grad):
        fn.restype = _ct.c_int
    for fn in (L.fastrack_mx_norm_grad_work_bytes, L.fastrack_mx_embedding_grad_work_bytes, L.fastrack_mx_loss_work_bytes,
               L.fastrack_mx_loss_grad_work_bytes):
        fn.restype = u64


class NormSaved:
    """What mx8_norm keeps for its gradient, of (rows, cols): `normed`, h / rms(h) as an MX8; `inverse`, 1 / rms(h),
    float32 (rows,); with a post_weight `block`, x / rms(x) as an MX8, and `block_inverse`; with a gate and no
    post_weight `block`, x itself; with a gate `gate`, an MX8. What there was none of is None."""
    __slots__ = ("normed", "inverse", "block", "block_inverse", "gate")

    def __init__(self, normed, inverse, block=None, block_inverse=None, gate=None):
        idx = _mx(normed, "normed", MX8).codes.get_device()
        rows, cols = normed.rows, normed.cols
        for q, what in ((block, "block"), (gate, "gate")):
            if q is not None:
                _mx(q, what, MX8, idx, rows, cols)
        for t, what in ((inverse, "inverse"), (block_inverse, "block_inverse")):
            if t is not None or what == "inverse":
                _vector(t, what, rows, idx)
        if block is None and (block_inverse is not None or gate is not None):
            raise ValueError("block_inverse and gate need the block that they go with")
        self.normed, self.inverse, self.block, self.block_inverse, self.gate = normed, inverse, block, block_inverse, gate


def _vector(t, what, n, idx, dtype=_float32, step=False):
    """Address (and with `step` the stride) of n values of one type, contiguous or, with `step`, any distance apart."""
    if not isinstance(t, _Tensor):
        raise ValueError("%s must be a torch tensor" % what)
    if t.dtype != dtype:
        raise ValueError("%s must be %s, got %s" % (what, dtype, t.dtype))
    at = t.get_device()
    if at < 0:
        raise ValueError("%s must be a CUDA tensor" % what)
    if idx is not None and at != idx:
        raise ValueError("%s is on %s, the other operands on cuda:%d" % (what, t.device, idx))
    if t.dim() != 1 or t.shape[0] != n:
        raise ValueError("%s must have shape (%d,), got %s" % (what, n, tuple(t.shape)))
    by = t.stride(0) if n > 1 else 1
    if by != 1 and not step:
        raise ValueError("%s must be contiguous" % what)
    return (t.data_ptr(), by) if step else t.data_ptr()


def _ids(t, what, idx=None):
    """(address, number, type) of the ids of rows."""
    if not isinstance(t, _Tensor):
        raise ValueError("%s must be a torch tensor" % what)
    code = _INDEX.get(t.dtype)
    if code is None:
        raise ValueError("%s must be int32 or int64, got %s" % (what, t.dtype))
    at = t.get_device()
    if at < 0:
        raise ValueError("%s must be a CUDA tensor" % what)
    if idx is not None and at != idx:
        raise ValueError("%s is on %s, the other operands on cuda:%d" % (what, t.device, idx))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % what)
    return t.data_ptr(), t.numel(), code


def _work(work, need, device, idx, stream):
    """(workspace, its address, its bytes): the caller's, or a new one."""
    if work is None:
        work = _fresh(need, device, stream) if need else None
        return work, work.data_ptr() if need else None, need
    if not isinstance(work, _Tensor) or work.dtype != _uint8 or not work.is_contiguous() or work.get_device() != idx:
        raise ValueError("work must be a contiguous uint8 tensor on the operands' device")
    return work, work.data_ptr(), work.numel()


def _on(idx, fn, *args):
    """fn(*args), which asks about the current device, with device idx current."""
    if _torch._C._cuda_getDevice() == idx:
        return fn(*args)
    with _torch.cuda.device(idx):
        return fn(*args)


def mx4_embedding(ids, table, scale=1.0, dtype=None, out=None, stream=None):
    """scale times the rows of `table`, an MX4 of (vocabulary, cols), that `ids` (int32 or int64, of any shape) name:
    (..., cols), bfloat16 unless told otherwise. A negative id is padding, a row of zeros; one past the table gives
    a row of NaN."""
    table = _mx(table, "table", MX4)
    device, idx = table.codes.device, table.codes.get_device()
    ip, m, icode = _ids(ids, "ids", idx)
    dtype = _dtype(dtype, out, _torch.bfloat16)
    out, p, ld = _out(out, "out", ids.shape + (table.cols,), dtype, device, idx, stream)
    _call(lib().fastrack_mx_embedding, idx, icode, ip, m, table.codes.data_ptr(), table.scales.data_ptr(), table.rows, table.cols,
          scale, _TYPES[dtype], p, ld, _raw_stream(stream, idx))
    return out


def mx4_embedding_grad(dy, ids, rows, scale=1.0, dtype=None, out=None, accumulate=False, work=None, stream=None):
    """The gradient of a table of `rows` rows from that of mx4_embedding's result: scale times the sum of the rows of
    dy (..., cols) with the same id, (rows, cols), float32 unless `dtype` says otherwise; the same every time.
    accumulate=True adds to `out` (float32) and leaves the rows that no id names as they are. Ids that name no row
    count for nothing."""
    p, ld, m, cols, code = _float(dy, "dy")
    device, idx = dy.device, dy.get_device()
    ip, n, icode = _ids(ids, "ids", idx)
    if ids.shape != dy.shape[:-1]:
        raise ValueError("dy has rows of shape %s, the ids %s" % (tuple(dy.shape[:-1]), tuple(ids.shape)))
    rows = int(rows)
    if rows < 0:
        raise ValueError("rows must not be negative")
    dtype = _dtype(dtype, out, _float32)
    if accumulate and (out is None or dtype != _float32):
        raise ValueError("accumulate=True needs a float32 out to add to")
    out, op, old = _out(out, "out", (rows, cols), dtype, device, idx, stream)
    L = lib()
    work, wp, wn = _work(work, L.fastrack_mx_embedding_grad_work_bytes(m, rows, cols), device, idx, stream)
    _call(L.fastrack_mx_embedding_grad, idx, icode, ip, code, p, ld, m, rows, cols, scale, _TYPES[dtype], op, old,
          1 if accumulate else 0, wp, wn, _raw_stream(stream, idx))
    return out


def _like(t, what, x, idx, code):
    """(address, row stride) of a tensor of x's shape and type, (None, 0) for none."""
    if t is None:
        return None, 0
    p, ld, _, _, c = _float(t, what, idx)
    if t.shape != x.shape or c != code:
        raise ValueError("%s must have the shape and type of %s %s, got %s %s" % (what, tuple(x.shape), x.dtype, tuple(t.shape), t.dtype))
    return p, ld


def _norm_weights(weight, post_weight, cols, idx, dtype):
    """(type, address of weight, of post_weight or None)."""
    wtype = weight.dtype if isinstance(weight, _Tensor) and weight.dtype in (dtype, _float32) else dtype
    wp = _vector(weight, "weight", cols, idx, wtype)
    return _TYPES[wtype], wp, None if post_weight is None else _vector(post_weight, "post_weight", cols, idx, wtype)


def _codes(q):
    return (None, None) if q is None else (q.codes.data_ptr(), q.scales.data_ptr())


def mx8_norm(x, weight, residual=None, post_weight=None, gate=None, scale=1.0, eps=1e-6, out=None, hidden=None, saved=None,
             stream=None):
    """The norm between two blocks with what stands before it, in one pass: from a block's result x (..., cols)
        b = x / rms(x) * post_weight    (or b = x)
        h = residual + scale * gate * b    (residual and gate where there are any)
        y = h / rms(h) * weight
    Returns (y, h, NormSaved): the next block's input, the residual stream, and what the gradient needs, in 8 bits. Without
    residual, post_weight, gate and scale h is x and returned as None. weight and post_weight are (cols,), both of
    x's type or both float32. `saved` is a NormSaved to write into."""
    p, ld, rows, cols, code = _float(x, "x")
    device, idx = x.device, x.get_device()
    rp, rld = _like(residual, "residual", x, idx, code)
    gp, gld = _like(gate, "gate", x, idx, code)
    wtype, wp, pp = _norm_weights(weight, post_weight, cols, idx, x.dtype)
    post, gated = post_weight is not None, gate is not None
    plain = residual is None and not post and not gated and scale == 1.0
    out, yp, yld = _out(out, "out", x.shape, x.dtype, device, idx, stream)
    hp, hld = None, 0
    if hidden is not None or not plain:
        hidden, hp, hld = _out(hidden, "hidden", x.shape, x.dtype, device, idx, stream)
    if saved is None:
        saved = object.__new__(NormSaved)
        saved.normed = MX8._new(rows, cols, device, stream)
        saved.inverse = _fresh((rows,), device, stream, _float32)
        saved.block = MX8._new(rows, cols, device, stream) if post or gated else None
        saved.block_inverse = _fresh((rows,), device, stream, _float32) if post else None
        saved.gate = MX8._new(rows, cols, device, stream) if gated else None
    else:
        _saved(saved, rows, cols, idx, post, gated)
    if rows and cols:
        _call(lib().fastrack_mx_norm, idx, code, p, ld, rp, rld, gp, gld, rows, cols, wtype, wp, pp, scale, eps, yp, yld, hp, hld,
              *_codes(saved.normed), saved.inverse.data_ptr(), *_codes(saved.block), saved.block_inverse.data_ptr() if post else None,
              *_codes(saved.gate), _raw_stream(stream, idx))
    return out, hidden, saved


def _saved(saved, rows, cols, idx, post, gated):
    """A NormSaved of the caller's holds what a norm with or without a post_weight and a gate keeps."""
    if type(saved) is not NormSaved:
        raise ValueError("saved must be a NormSaved")
    _mx(saved.normed, "saved.normed", MX8, idx, rows, cols)
    for q, what, there in ((saved.block, "block", post or gated), (saved.gate, "gate", gated), (saved.block_inverse, "block_inverse", post)):
        if (q is not None) != there:
            raise ValueError("saved.%s %s" % (what, "is missing" if there else "without what it is kept for"))
    return saved


def mx8_norm_grad(dy, weight, saved, dhidden=None, post_weight=None, scale=1.0, residual=True, out=None, out_residual=None,
                  out_gate=None, work=None, stream=None):
    """The gradients of mx8_norm at what it kept, for dy of y and dhidden of h (both (..., cols)): (dx, dresidual, dgate,
    dweight, dpost_weight), None in the place of what there was none of (residual=False: of the residual). The
    weights' gradients are float32 (cols,), the others of dy's type."""
    p, ld, rows, cols, code = _float(dy, "dy")
    device, idx = dy.device, dy.get_device()
    if type(saved) is not NormSaved:
        raise ValueError("saved must be a NormSaved")
    post, gated = post_weight is not None, saved.gate is not None
    _saved(saved, rows, cols, idx, post, gated)
    hp, hld = _like(dhidden, "dhidden", dy, idx, code)
    wtype, wp, pp = _norm_weights(weight, post_weight, cols, idx, dy.dtype)
    out, xp, xld = _out(out, "out", dy.shape, dy.dtype, device, idx, stream)
    sp, sld, gp, gld = None, 0, None, 0
    if residual:
        out_residual, sp, sld = _out(out_residual, "out_residual", dy.shape, dy.dtype, device, idx, stream)
    elif out_residual is not None:
        raise ValueError("out_residual without a residual")
    if gated:
        out_gate, gp, gld = _out(out_gate, "out_gate", dy.shape, dy.dtype, device, idx, stream)
    elif out_gate is not None:
        raise ValueError("out_gate without a kept gate")
    dweight = _fresh((cols,), device, stream, _float32)
    dpost = _fresh((cols,), device, stream, _float32) if post else None
    L = lib()
    work, kp, kn = _work(work, _on(idx, L.fastrack_mx_norm_grad_work_bytes, rows, cols, 1 if post else 0), device, idx, stream)
    _call(L.fastrack_mx_norm_grad, idx, code, p, ld, hp, hld, rows, cols, wtype, wp, pp, scale, *_codes(saved.normed),
          saved.inverse.data_ptr(), *_codes(saved.block), saved.block_inverse.data_ptr() if post else None, *_codes(saved.gate),
          xp, xld, sp, sld, gp, gld, dweight.data_ptr(), dpost.data_ptr() if post else None, kp, kn, _raw_stream(stream, idx))
    return out, out_residual, out_gate, dweight, dpost


def _loss_operands(x, w, targets):
    w = _mx(w, "w", MX4)
    device, idx = w.codes.device, w.codes.get_device()
    xp, xld, m, k, code = _float(x, "x", idx)
    if k != w.cols:
        raise ValueError("x has %d columns, the weights %d" % (k, w.cols))
    tp, _, icode = _ids(targets, "targets", idx)
    if targets.shape != x.shape[:-1]:
        raise ValueError("x has rows of shape %s, the targets %s" % (tuple(x.shape[:-1]), tuple(targets.shape)))
    return device, idx, (code, xp, xld), m, k, (icode, tp)


def mx4_cross_entropy(x, w, targets, scale=1.0, work=None, stream=None):
    """(loss, lse), both float32 of targets' shape: with z = scale * x W^T for a head w, an MX4 of (classes, inputs), and x
    (..., inputs), lse = log sum exp z and loss = lse - z[target]. The logits are not kept. A negative target leaves
    its token out: loss 0, no gradient; one past the classes makes the loss NaN."""
    device, idx, (code, xp, xld), m, k, (icode, tp) = _loss_operands(x, w, targets)
    loss, lse = (_fresh(targets.shape, device, stream, _float32) for _ in range(2))
    L = lib()
    need = 0 if work is not None else _on(idx, L.fastrack_mx_loss_work_bytes, code, xp, xld, m, w.rows, k)
    work, wp, wn = _work(work, need, device, idx, stream)
    _call(L.fastrack_mx_loss, idx, code, xp, xld, *_codes(w), icode, tp, m, w.rows, k, scale, loss.data_ptr(), lse.data_ptr(), wp, wn,
          _raw_stream(stream, idx))
    return loss, lse


def mx4_cross_entropy_grad(dloss, x, w, targets, lse, saved=None, scale=1.0, grad_input=True, dtype=None, weight_dtype=None,
                           out=None, out_weight=None, accumulate=False, work=None, stream=None):
    """(dx, dw) of mx4_cross_entropy for the gradient dloss of each token's loss (float32 of targets' shape, expanded or
    not), from the same operands and the lse that they gave. dx (..., inputs) is of x's type unless `dtype` says otherwise,
    and None with grad_input=False. dw (classes, inputs) = dz^T x^ is taken with the kept x, an MX8 of (tokens, inputs), and is
    None without `saved`; float32 unless weight_dtype says otherwise; accumulate=True adds to out_weight (float32)."""
    device, idx, (code, xp, xld), m, k, (icode, tp) = _loss_operands(x, w, targets)
    for t, what in ((dloss, "dloss"), (lse, "lse")):
        if not isinstance(t, _Tensor) or t.shape != targets.shape:
            raise ValueError("%s must be a tensor of shape %s" % (what, tuple(targets.shape)))
    if not lse.is_contiguous():
        raise ValueError("lse must be contiguous")
    dp, step = _vector(dloss if dloss.dim() == 1 else _flat(dloss, "dloss"), "dloss", m, idx, step=True)
    lp = _vector(lse.view(-1), "lse", m, idx)
    dtype = _dtype(dtype, out, x.dtype)
    weight_dtype = _dtype(weight_dtype, out_weight, _float32)
    op = gp = None
    old = gld = 0
    if grad_input:
        out, op, old = _out(out, "out", x.shape, dtype, device, idx, stream)
    elif out is not None:
        raise ValueError("out without grad_input")
    if accumulate and (out_weight is None or weight_dtype != _float32):
        raise ValueError("accumulate=True needs a float32 out_weight to add to")
    if saved is not None:
        _mx(saved, "saved", MX8, idx, m, k)
        out_weight, gp, gld = _out(out_weight, "out_weight", (w.rows, k), weight_dtype, device, idx, stream)
    elif out_weight is not None:
        raise ValueError("out_weight without the kept x that it comes from")
    L = lib()
    need = 0 if work is not None else _on(idx, L.fastrack_mx_loss_grad_work_bytes, code, xp, xld, m, w.rows, k, 1 if grad_input else 0,
                                          _TYPES[dtype], 1 if saved is not None else 0, _TYPES[weight_dtype])
    work, wp, wn = _work(work, need, device, idx, stream)
    _call(L.fastrack_mx_loss_grad, idx, code, xp, xld, *_codes(w), *_codes(saved), icode, tp, dp, step, lp, m, w.rows, k, scale,
          _TYPES[dtype], op, old, _TYPES[weight_dtype], gp, gld, 1 if accumulate else 0, wp, wn, _raw_stream(stream, idx))
    return out, out_weight


def _flat(t, what):
    """t with its axes as one, without a copy: contiguous, or one value expanded."""
    if not any(s for n, s in zip(t.shape, t.stride()) if n != 1):
        return t.as_strided((t.numel(),), (0,))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous, or one value expanded" % what)
    return t.view(-1)
