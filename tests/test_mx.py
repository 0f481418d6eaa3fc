"""The microscaled operators without a GPU: the oracle against hand-worked blocks, sizes, the tensors' own checks
and what the C entries and the binding refuse."""
import ctypes

import numpy as np
import pytest
import torch

import mx_oracle as O
import paper_2410_15240_amd as F

A, B, C, D = 0x10000, 0x9000000, 0x12000000, 0x18000000   # aligned "device" addresses, never dereferenced here


@pytest.fixture(scope="module")
def L():
    import os
    if not os.path.exists(F.library_path()):
        from paper_2410_15240_amd import build
        build.build()
    return F.lib()


def test_oracle_on_worked_blocks():
    x = np.zeros((2, 32))
    # top 4 -> scale 1: the grid itself, ties (0.25 0.75 1.25 1.75 2.5 3.5 5) to the even code, then saturation
    x[0, :16] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -0.25, -0.75, 0.26, 0.74, 4.99, 5.01, 6.0, 7.9]
    x[1, 0] = np.inf
    codes, scales = O.quantize(x, 4)
    assert scales.tolist() == [[127], [255]]
    got = O.values(codes, scales, 32)
    assert got[0, :16].tolist() == [0, 1, 1, 2, 2, 4, 4, 6, 0, -1, 0.5, 0.5, 4, 6, 6, 6]
    assert np.isnan(got[1]).all() and not codes[1].any()
    x[0, 15] = 0.0
    c8, s8 = O.quantize(x[:1], 8)
    assert s8[0, 0] == 127 + 2 and c8[0, 7] == 112 and c8[0, 0] == 4   # 7 = 4 * 1.75, 0.25 = 4 / 64 * 4
    z4, z8 = O.quantize(np.zeros((1, 5)), 4), O.quantize(np.full((1, 5), 1.9999), 8)
    assert z4[1][0, 0] == 0 and not z4[0].any() and z8[0][0, 0] == 127   # rounds to 128, held to 127


def test_sizes(L):
    assert L.fastrack_mx_code_bytes(4, 3, 33) == 3 * 2 * 16
    assert L.fastrack_mx_code_bytes(8, 3, 33) == 3 * 2 * 32
    assert L.fastrack_mx_scale_bytes(3, 33) == 6
    assert L.fastrack_mx_code_bytes(5, 3, 33) == 0 and L.fastrack_mx_code_bytes(4, 1 << 31, 1) == 0
    assert L.fastrack_mx_code_bytes(4, 0, 33) == 0 and L.fastrack_mx_code_bytes(4, 3, 0) == 0
    assert F.MX4.nbytes(3, 33) == 6 * 17 and F.MX8.nbytes(3, 33) == 6 * 33
    assert F.MX4.nbytes(1 << 20, 1 << 20) == (1 << 35) * 17   # past 32 bits


def test_tensors_in_one_buffer():
    for cls, codes in ((F.MX4, torch.uint8), (F.MX8, torch.int8)):
        buf = torch.arange(cls.nbytes(5, 40), dtype=torch.int64).to(torch.uint8)
        t = cls.view(buf, 5, 40)
        assert (t.rows, t.cols) == (5, 40) and t.codes.dtype == codes
        assert tuple(t.codes.shape) == (5, 2 * cls.block_bytes) and tuple(t.scales.shape) == (5, 2)
        assert t.codes.data_ptr() == buf.data_ptr()
        assert t.scales.data_ptr() == buf.data_ptr() + 10 * cls.block_bytes
        with pytest.raises(ValueError, match="takes"):
            cls.view(buf[:-1], 5, 40)
        with pytest.raises(ValueError, match="uint8"):
            cls.view(buf.to(torch.int32), 5, 40)


@pytest.mark.parametrize("codes,scales,cols,match", [
    (torch.zeros(2, 16, dtype=torch.int32), torch.zeros(2, 1, dtype=torch.uint8), 20, "uint8"),
    (torch.zeros(2, 16, dtype=torch.uint8), torch.zeros(2, 2, dtype=torch.uint8), 20, "shape"),
    (torch.zeros(2, 15, dtype=torch.uint8), torch.zeros(2, 1, dtype=torch.uint8), 20, "shape"),
    (torch.zeros(2, 16, dtype=torch.uint8), torch.zeros(3, 1, dtype=torch.uint8), 20, "shape"),
    (torch.zeros(2, 32, dtype=torch.uint8)[:, ::2], torch.zeros(2, 1, dtype=torch.uint8), 20, "contiguous"),
    (np.zeros((2, 16), np.uint8), torch.zeros(2, 1, dtype=torch.uint8), 20, "torch tensor"),
])
def test_mx4_checks_its_parts(codes, scales, cols, match):
    with pytest.raises(ValueError, match=match):
        F.MX4(codes, scales, cols)


def host4(rows=4, cols=64):
    return F.MX4.view(torch.zeros(F.MX4.nbytes(rows, cols), dtype=torch.uint8), rows, cols)


@pytest.mark.parametrize("call,match", [
    (lambda: F.mx4_quantize(torch.zeros(4, 64)), "CUDA tensor"),
    (lambda: F.mx8_quantize(torch.zeros(4, 64, dtype=torch.float64)), "bfloat16, float16 or float32"),
    (lambda: F.mx8_quantize(np.zeros((4, 64))), "torch tensor"),
    (lambda: F.mx4_dequantize(host4()), "CUDA tensor"),
    (lambda: F.mx8_dequantize(host4()), "must be an MX8"),
    (lambda: F.mx4_linear(torch.zeros(4, 64), host4()), "CUDA tensor"),
    (lambda: F.mx4_linear(torch.zeros(4, 64), torch.zeros(4, 64)), "must be an MX4"),
    (lambda: F.mx4_linear_grad_input(torch.zeros(4, 64), host4()), "CUDA tensor"),
    (lambda: F.mx8_weight_grad(torch.zeros(4, 64), host4()), "must be an MX8"),
    (lambda: F.mx8_act(torch.zeros(4, 64)), "CUDA tensor"),
    (lambda: F.mx8_act(torch.zeros(4, 64), act="tanh"), "gelu, silu"),
    (lambda: F.mx8_act_grad(torch.zeros(4, 64), host4()), "must be an MX8"),
])
def test_binding_refuses(call, match):
    with pytest.raises(ValueError, match=match):
        call()


def quant(L, fmt=4, type=0, x=A, ld=64, rows=4, cols=64, codes=B, scales=C):
    return L.fastrack_mx_quantize(fmt, type, x, ld, rows, cols, codes, scales, None)


def dequant(L, fmt=8, type=0, out=A, ld=64, rows=4, cols=64, codes=B, scales=C):
    return L.fastrack_mx_dequantize(fmt, codes, scales, rows, cols, type, out, ld, None)


@pytest.mark.parametrize("kw", [dict(fmt=6), dict(type=3), dict(x=None), dict(x=A + 1), dict(codes=None), dict(codes=B + 8),
                                dict(scales=None), dict(rows=1 << 31), dict(cols=1 << 31), dict(codes=A + 64),
                                dict(scales=A + 511), dict(scales=B + 127), dict(ld=1 << 41), dict(type=2, x=A + 2)])
def test_quantize_rejects_bad_arguments(L, kw):
    assert quant(L, **kw) == -1 and L.fastrack_last_error()


@pytest.mark.parametrize("kw", [dict(fmt=0), dict(type=9), dict(out=None), dict(out=A + 1), dict(codes=B + 4), dict(ld=63),
                                dict(out=B + 16), dict(scales=None)])
def test_dequantize_rejects_bad_arguments(L, kw):
    assert dequant(L, **kw) == -1 and L.fastrack_last_error()


def act(L, kind=0, type=0, x=A, gate=None, y=B, xc=C, xs=D, gc=None, gs=None, rows=4, cols=64, ldy=64):
    return L.fastrack_mx_act(kind, type, x, 64, gate, 64, rows, cols, y, ldy, xc, xs, gc, gs, None)


@pytest.mark.parametrize("kw", [dict(kind=2), dict(type=3), dict(x=None), dict(y=None), dict(y=A), dict(xc=None), dict(xc=C + 8),
                                dict(gate=A + 0x1000), dict(gate=A + 0x1000, gc=D + 0x1000, gs=None), dict(xs=C + 5),
                                dict(ldy=60)])
def test_act_rejects_bad_arguments(L, kw):
    assert act(L, **kw) == -1 and L.fastrack_last_error()


def act_grad(L, kind=0, type=0, dy=A, xc=B, xs=C, gc=None, gs=None, dx=D, dg=None, rows=4, cols=64):
    return L.fastrack_mx_act_grad(kind, type, dy, 64, xc, xs, gc, gs, rows, cols, dx, 64, dg, 64, None)


@pytest.mark.parametrize("kw", [dict(kind=7), dict(dy=None), dict(dx=None), dict(dx=A + 2), dict(xc=None), dict(xs=None),
                                dict(gc=B + 0x1000, gs=C + 0x1000), dict(gc=B + 0x1000, gs=C + 0x1000, dg=D + 16)])
def test_act_grad_rejects_bad_arguments(L, kw):
    assert act_grad(L, **kw) == -1 and L.fastrack_last_error()


def linear(L, fn="fastrack_mx_linear", type=0, x=A, ld=64, codes=B, scales=C, m=4, n=64, k=64, out_type=0, y=D, ldy=64,
           work=None, nwork=0):
    return getattr(L, fn)(type, x, ld, codes, scales, m, n, k, out_type, y, ldy, work, nwork, None)


@pytest.mark.parametrize("fn", ["fastrack_mx_linear", "fastrack_mx_linear_grad_input"])
@pytest.mark.parametrize("kw", [dict(type=3), dict(out_type=3), dict(x=None), dict(x=A + 1), dict(codes=None), dict(codes=B + 8),
                                dict(scales=None), dict(y=None), dict(y=A), dict(y=B), dict(ldy=63), dict(m=1 << 31),
                                # many outputs: the terms of a float operand need a workspace
                                dict(type=2, m=4096, n=4096, k=4096, ld=4096, ldy=4096),
                                dict(type=2, m=4096, n=4096, k=4096, ld=4096, ldy=4096, work=A + 0x100000, nwork=64),
                                dict(type=2, m=4096, n=4096, k=4096, ld=4096, ldy=4096, work=A + 0x100008, nwork=1 << 30),
                                dict(m=1 << 30, n=1 << 20, k=1 << 20)])
def test_products_reject_bad_arguments(L, fn, kw):
    assert linear(L, fn, **kw) == -1 and L.fastrack_last_error()


@pytest.mark.parametrize("kw", [dict(out_type=0, acc=1), dict(out_type=2, acc=2), dict(dw=A), dict(dy=None), dict(codes=B + 1)])
def test_weight_grad_rejects_bad_arguments(L, kw):
    a = dict(dy=A, codes=B, out_type=2, dw=D, acc=0)
    a.update(kw)
    assert L.fastrack_mx_weight_grad(0, a["dy"], 64, a["codes"], C, 4, 64, 64, a["out_type"], a["dw"], 64, a["acc"], None, 0,
                                     None) == -1


@pytest.mark.parametrize("kw", [dict(x=None), dict(x=A + 8), dict(xs=None), dict(y=B), dict(y=None), dict(t=5)])
def test_linear_mx_rejects_bad_arguments(L, kw):
    a = dict(x=A, xs=A + 0x1000, y=D, t=0)
    a.update(kw)
    assert L.fastrack_mx_linear_mx(a["x"], a["xs"], B, C, 4, 64, 64, a["t"], a["y"], 64, None, 0, None) == -1


def test_rows_side_by_side_in_a_wider_tensor_do_not_overlap(L):
    """Outputs that share rows of one stride are refused only where their columns meet (the call stops at the next
    argument, a missing buffer, before any HIP call)."""
    def grads(dg):   # dx of 64 columns at D, in rows of 128
        rc = L.fastrack_mx_act_grad(0, 0, A, 64, B, C, B + 0x1000, C + 0x1000, 4, 64, D, 128, dg, 128, None)
        return rc, L.fastrack_last_error()
    for dg in (D, D + 2, D + 126, D - 2, D + 130):
        assert grads(dg) == (-1, b"d_dgate overlaps d_dx")


def test_empty_calls_are_no_ops(L):
    assert quant(L, rows=0, x=None, codes=None, scales=None) == 0
    assert dequant(L, cols=0, out=None, codes=None, scales=None) == 0
    assert act(L, rows=0, x=None, y=None, xc=None, xs=None) == 0
    assert linear(L, m=0, x=None, y=None) == 0 and linear(L, n=0, codes=None, scales=None, y=None) == 0


def test_workspace_of_a_product(L):
    work = L.fastrack_mx_work_bytes
    for op in range(4):   # a size of 0 anywhere plans nothing
        for m, n, k in ((0, 5, 5), (5, 0, 5), (5, 5, 0), (0, 0, 0)):
            assert work(op, 2, A, 8, m, n, k) == 0
    assert work(0, 0, A, 64, 4096, 8192, 8192) == 0           # read in place, a whole sum to a tile
    assert work(0, 2, A, 8192, 4096, 8192, 8192) >= 3 * 2 * 4096 * 8192   # three terms of every value
    assert work(0, 0, A, 8191, 4096, 8192, 8192) >= 2 * 4096 * 8192       # rows that are not 16-byte aligned
    assert work(4, 0, A, 64, 4, 4, 4) == 0 and work(0, 3, A, 64, 4, 4, 4) == 0 and work(0, 0, A, 64, 1 << 31, 4, 4) == 0
