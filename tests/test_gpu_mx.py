"""The microscaled operators on the GPU against their definition in 64 bits (mx_oracle).

Codes, scales and dequantised values are compared bit for bit. Products are compared exactly on inputs whose sums
32 bits hold exactly (small whole numbers), over the shapes where tiles, blocks and parts of a sum end; and on
normal inputs within the error of a 32-bit sum: `terms` products a value, each added with a relative error of at most
2^-23 of the sum of magnitudes; rounding to the output's type keeps order, so the result lies between the
rounded ends of that interval."""
import numpy as np
import pytest
import torch

import mx_oracle as O
import paper_2410_15240_amd as F

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
TERMS = {"bf16": 1, "fp16": 2, "fp32": 3}
CLS = {4: F.MX4, 8: F.MX8}
QUANT = {4: F.mx4_quantize, 8: F.mx8_quantize}
DEQUANT = {4: F.mx4_dequantize, 8: F.mx8_dequantize}


def gpu(x, dtype, pad=0):
    """x on the GPU, as a slice that starts pad // 2 elements into rows of x.shape[1] + pad."""
    t = torch.from_numpy(np.ascontiguousarray(x)).to(dtype)
    wide = torch.full((x.shape[0], x.shape[1] + pad), float("nan"), dtype=dtype)
    wide[:, pad // 2:pad // 2 + x.shape[1]] = t
    return wide.cuda()[:, pad // 2:pad // 2 + x.shape[1]]


def f64(t):
    return t.detach().cpu().double().numpy()


def check_between(got, want, bound):
    """got is some value of [want - bound, want + bound] rounded to got's type."""
    lo, hi = (f64(torch.from_numpy(want + s * bound).to(got.dtype)) for s in (-1, 1))
    g = f64(got)
    assert ((g >= lo) & (g <= hi)).all(), np.abs((g - want) / bound).max()


def to_mx(codes, scales, cols, bits):
    return CLS[bits](torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), cols)


def random_mx(rng, rows, cols, bits, whole=False):
    """(MX tensor, its values): random codes; scales near 1, or all 1 (bits 4) and 2^6 (bits 8) for whole numbers."""
    nb = O.blocks(cols)
    if bits == 4:
        codes = rng.integers(0, 256, (rows, nb * 16)).astype(np.uint8)
    else:
        codes = rng.integers(-16 if whole else -127, 17 if whole else 128, (rows, nb * 32)).astype(np.int8)
    base = 128 if bits == 4 else 133            # E2M1 has halves: twice its values are whole
    scales = (np.full((rows, nb), base) if whole else rng.integers(118, 132, (rows, nb))).astype(np.uint8)
    flat = codes.reshape(rows, nb, -1)
    keep = np.arange(nb * 32).reshape(nb, 32) < cols
    if bits == 4:
        flat &= (keep[:, 0::2] * 0x0F + keep[:, 1::2] * 0xF0).astype(np.uint8)
    else:
        flat *= keep.astype(np.int8)
    return to_mx(codes, scales, cols, bits), O.values(codes, scales, cols)


def check_mx(q, codes, scales):
    assert torch.equal(q.scales.cpu(), torch.from_numpy(scales))
    got = q.codes.cpu().numpy()
    if not np.array_equal(got, codes):
        r, c = np.argwhere(got != codes)[0]
        raise AssertionError("codes differ first at row %d byte %d: %d, want %d" % (r, c, got[r, c], codes[r, c]))


# ---- quantisation ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (3, 31, 0), (2, 32, 0), (5, 33, 0), (7, 100, 5), (4, 256, 8), (300, 136, 0),
                                           (33, 1111, 1)])
def test_quantize_is_the_definition(bits, name, rows, cols, pad):
    rng = np.random.default_rng(rows * 1000 + cols)
    x = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-12, 12, (rows, cols)))
    t = gpu(x, TYPES[name], pad)
    q = QUANT[bits](t)
    check_mx(q, *O.quantize(f64(t), bits))
    for out in TYPES.values():
        got = DEQUANT[bits](q, dtype=out)
        want = torch.from_numpy(O.values(q.codes.cpu().numpy(), q.scales.cpu().numpy(), cols)).to(out)
        assert torch.equal(got.cpu(), want)
    wide = torch.full((rows, cols + 6), 7.0, dtype=TYPES[name], device="cuda")
    got = DEQUANT[bits](q, out=wide[:, 3:3 + cols])
    assert torch.equal(got, DEQUANT[bits](q, dtype=TYPES[name])) and (wide[:, :3] == 7).all() and (wide[:, 3 + cols:] == 7).all()


@pytest.mark.parametrize("bits", [4, 8])
def test_quantize_ties_and_saturation_at_every_exponent(bits):
    """Every half step of the code's grid, at each power of two that a float32 block can have, subnormal ones too."""
    step = np.arange(-63, 64) / 16.0 if bits == 4 else np.arange(-255, 256) / 128.0
    top = 4.0 if bits == 4 else 1.0
    n = -(-step.size // 31)
    body = np.zeros((n, 31))
    body.flat[:step.size] = step
    block = np.concatenate((np.full((n, 1), top), body), axis=1)   # a 4 (or 1) in each block fixes its exponent
    block = np.where(np.abs(block) < 2 * top, block, 0.0).reshape(1, -1)
    exps = np.arange(-149, 126)
    x = (block * np.ldexp(1.0, exps)[:, None]).astype(np.float32).astype(np.float64)
    q = QUANT[bits](gpu(x, torch.float32))
    codes, scales = O.quantize(x, bits)
    check_mx(q, codes, scales)
    assert scales.min() <= 1 and scales.max() >= 252


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("name", list(TYPES))
def test_quantize_special_values(bits, name):
    big = float(torch.finfo(TYPES[name]).max)
    tiny = float(torch.finfo(TYPES[name]).smallest_normal)
    x = np.zeros((8, 70))
    x[1, 3], x[2, 40], x[3, 69] = np.inf, -np.inf, np.nan
    x[4], x[5] = big, -big
    x[6, ::2], x[6, 1::2] = tiny, -tiny
    x[7] = -0.0
    t = gpu(x, TYPES[name])
    q = QUANT[bits](t)
    codes, scales = O.quantize(f64(t), bits)
    check_mx(q, codes, scales)
    got = f64(DEQUANT[bits](q, dtype=torch.float32))
    assert np.isnan(got[1, :32]).all() and not np.isnan(got[1, 32:]).any()
    assert np.isnan(got[2, 32:64]).all() and np.isnan(got[3, 64:]).all() and (got[0] == 0).all()
    assert np.isfinite(got[4:]).all()


@pytest.mark.parametrize("bits", [4, 8])
def test_dequantize_every_scale_and_code(bits):
    scales = np.arange(256, dtype=np.uint8).reshape(-1, 1).repeat(8, axis=1)
    codes = np.tile(np.arange(256, dtype=np.uint8) if bits == 8 else np.arange(128, dtype=np.uint8), (256, 1))
    codes = codes.view(np.int8) if bits == 8 else codes
    cols = 256
    q = to_mx(np.ascontiguousarray(codes), np.ascontiguousarray(scales), cols, bits)
    want = O.values(codes, scales, cols)
    for out in TYPES.values():
        got = DEQUANT[bits](q, dtype=out).cpu()
        assert torch.equal(torch.nan_to_num(got, nan=123.0), torch.nan_to_num(torch.from_numpy(want).to(out), nan=123.0))


@pytest.mark.parametrize("bits", [4, 8])
def test_quantize_of_one_row_expanded_past_32_bit_offsets(bits):
    """4.6e9 values from one row (stride 0); the last rows' codes lie past 2^32 (or 2^31) bytes."""
    rng = np.random.default_rng(5)
    x = torch.from_numpy(rng.standard_normal((1, 65536))).to(torch.bfloat16).cuda()
    q = QUANT[bits](x.expand(70001, 65536))
    first = QUANT[bits](x)
    for r in (0, 1, 32768, 65536, 70000):
        assert torch.equal(q.codes[r], first.codes[0]) and torch.equal(q.scales[r], first.scales[0])
    assert torch.equal(q.scales, first.scales.expand_as(q.scales))


def test_rows_of_more_than_two_axes_and_empty_ones():
    x = torch.randn(3, 4, 50, device="cuda")
    assert torch.equal(F.mx8_quantize(x).codes, F.mx8_quantize(x.view(12, 50)).codes)
    assert torch.equal(F.mx8_quantize(x[:, :, 3:40]).codes, F.mx8_quantize(x[:, :, 3:40].reshape(12, 37)).codes)
    assert torch.equal(F.mx8_quantize(x[1, 2]).codes, F.mx8_quantize(x[1, 2].view(1, 50)).codes)
    with pytest.raises(ValueError, match="rows of one stride"):
        F.mx8_quantize(x[:, :2])
    with pytest.raises(ValueError, match="dense along"):
        F.mx8_quantize(x.transpose(1, 2))
    for rows, cols in ((0, 64), (5, 0)):
        q = F.mx4_quantize(torch.zeros(rows, cols, device="cuda"))
        assert (q.rows, q.cols) == (rows, cols) and F.mx4_dequantize(q).shape == (rows, cols)


# ---- products --------------------------------------------------------------------------------------------------

SHAPES = [(1, 1, 1), (1, 64, 64), (1, 5, 1000), (2, 130, 31), (3, 33, 64), (7, 64, 100), (16, 48, 256), (17, 129, 257),
          (31, 256, 96), (64, 64, 2048), (100, 72, 513), (129, 128, 65), (130, 257, 200), (257, 300, 130), (1, 3, 5000),
          (33, 1000, 40), (5, 7, 4096), (600, 16, 96), (512, 520, 264)]


def whole(rng, rows, cols, low=-8, high=9):
    return rng.integers(low, high, (rows, cols)).astype(np.float64)


def product(op, a, q, **kw):
    fn = dict(linear=F.mx4_linear, grad=F.mx4_linear_grad_input, weight=F.mx8_weight_grad)[op]
    return fn(a, q, **kw)


def layer(rng, op, m, n, k, make):
    """(float operand, MX operand, its values, the product in 64 bits as a function of the operand's values)."""
    if op == "linear":
        q, v = random_mx(rng, n, k, 4, make == "whole")
        a, f = (m, k), lambda x: x @ v.T
    elif op == "grad":
        q, v = random_mx(rng, n, k, 4, make == "whole")
        a, f = (m, n), lambda x: x @ v
    else:
        q, v = random_mx(rng, m, k, 8, make == "whole")
        a, f = (m, n), lambda x: x.T @ v
    x = whole(rng, *a) if make == "whole" else rng.standard_normal(a)
    return x, q, v, f


@pytest.mark.parametrize("op", ["linear", "grad", "weight"])
@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_products_are_exact_on_whole_numbers(op, name, m, n, k):
    """|a| <= 8, |q| <= 16 and at most 5000 terms: every partial sum is a whole number below 2^24."""
    rng = np.random.default_rng(m * 7 + n * 3 + k)
    x, q, _, f = layer(rng, op, m, n, k, "whole")
    want = f(x)
    for pad in (0, 8, 3):
        got = product(op, gpu(x, TYPES[name], pad), q, dtype=torch.float32)
        assert np.array_equal(f64(got), want), (pad, np.argwhere(f64(got) != want)[:4])
    got = product(op, gpu(x, TYPES[name]), q, dtype=torch.bfloat16)
    assert torch.equal(got.cpu(), torch.from_numpy(want).to(torch.bfloat16))


@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("m", [1, 2, 3])
@pytest.mark.parametrize("n,k", [(1, 512), (7, 600), (100, 2048), (33, 2049), (5, 4103), (130, 4096), (9, 4991)])
def test_a_few_tokens_are_exact_on_whole_numbers(name, m, n, k):
    """Each input's place on its own, and all of them at once; infinities in one token only."""
    rng = np.random.default_rng(m + n + k)
    q, v = random_mx(rng, n, k, 4, True)
    for pad in (0, 8, 3):
        x = whole(rng, m, k)
        assert np.array_equal(f64(F.mx4_linear(gpu(x, TYPES[name], pad), q, dtype=torch.float32)), x @ v.T)
    for at in rng.integers(0, k, 40):
        x = np.zeros((m, k))
        x[m - 1, at] = 1.0
        assert np.array_equal(f64(F.mx4_linear(gpu(x, TYPES[name]), q, dtype=torch.float32)), x @ v.T), at
    x = whole(rng, m, k)
    x[0, k - 1] = np.inf
    with np.errstate(invalid="ignore"):
        want = x @ v.T
    got = f64(F.mx4_linear(gpu(x, TYPES[name]), q, dtype=torch.float32))
    assert np.array_equal(np.nan_to_num(got, nan=1e9, posinf=2e9, neginf=3e9), np.nan_to_num(want, nan=1e9, posinf=2e9, neginf=3e9))


@pytest.mark.parametrize("op", ["linear", "grad", "weight"])
@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("rows,cols,sums", [(3001, 2888, 136), (2900, 3009, 700), (4096, 2304, 64), (2823, 2817, 5),
                                            (260, 32008, 320)])
def test_products_with_many_outputs_are_exact_on_whole_numbers(op, name, rows, cols, sums):
    """Enough output tiles for every CU: the largest tiles, with edges, whole stages of the sum and short ones."""
    m, n, k = dict(linear=(rows, cols, sums), grad=(rows, sums, cols), weight=(sums, rows, cols))[op]
    rng = np.random.default_rng(rows + cols + sums)
    x, q, _, f = layer(rng, op, m, n, k, "whole")
    want = torch.from_numpy(f(x)).float()
    for pad in (0, 3):
        got = product(op, gpu(x, TYPES[name], pad), q, dtype=torch.float32).cpu()
        assert torch.equal(got, want), (pad, torch.nonzero(got != want)[:4].tolist())


@pytest.mark.parametrize("op", ["linear", "grad", "weight"])
@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("m,n,k", [(6001, 500, 1111), (1000, 1001, 2000), (40, 8200, 4000), (77, 4100, 8192), (300, 3000, 3001)])
def test_products_of_middling_sizes_are_exact_on_whole_numbers(op, name, m, n, k):
    """Between small tiles and large ones: tiles of 64 and 128, sums cut into parts of uneven length."""
    rng = np.random.default_rng(m + n + k)
    x, q, _, f = layer(rng, op, m, n, k, "whole")
    x = np.clip(x, -4, 4)   # |x q| <= 64: 8200 of them stay below 2^24
    want = torch.from_numpy(f(x)).float()
    for pad in (0, 3):
        got = product(op, gpu(x, TYPES[name], pad), q, dtype=torch.float32).cpu()
        assert torch.equal(got, want), (pad, torch.nonzero(got != want)[:4].tolist())


@pytest.mark.parametrize("op", ["linear", "grad", "weight"])
@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("rows,cols,sums", [(2048, 4093, 333), (2049, 4096, 333), (1021, 4001, 1000), (3000, 1003, 200),
                                            (64, 8190, 6001), (130, 900, 9000)])
def test_products_about_one_round_of_tiles_are_exact_on_whole_numbers(op, name, rows, cols, sums):
    """The largest tiles for just up to half the CUs and for one more row, tiles of 128 for most of
    them, and so few that the sum is cut."""
    m, n, k = dict(linear=(rows, cols, sums), grad=(rows, sums, cols), weight=(sums, rows, cols))[op]
    rng = np.random.default_rng(rows + cols + sums)
    x, q, _, f = layer(rng, op, m, n, k, "whole")
    x = np.clip(x, -4, 4)   # |x q| <= 64: 9000 of them stay below 2^24
    want = torch.from_numpy(f(x)).float()
    for pad in (0, 3):
        got = product(op, gpu(x, TYPES[name], pad), q, dtype=torch.float32).cpu()
        assert torch.equal(got, want), (pad, torch.nonzero(got != want)[:4].tolist())


@pytest.mark.parametrize("m,n,k", [(2048, 4093, 700), (2049, 4096, 700), (515, 4100, 1300), (65, 8190, 5000), (130, 900, 4999)])
def test_product_of_two_mx4_about_one_round_of_tiles(m, n, k):
    rng = np.random.default_rng(m + n + k)
    qx, vx = random_mx(rng, m, k, 4, True)
    qw, vw = random_mx(rng, n, k, 4, True)
    want = torch.from_numpy(vx @ vw.T).float()
    got = F.mx4_linear(qx, qw, dtype=torch.float32).cpu()
    assert torch.equal(got, want), torch.nonzero(got != want)[:4].tolist()


@pytest.mark.parametrize("op", ["linear", "grad", "weight"])
@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("out", list(TYPES))
@pytest.mark.parametrize("m,n,k", [(1, 96, 700), (29, 200, 333), (150, 140, 260), (300, 30, 70)])
def test_products_of_normal_inputs(op, name, out, m, n, k):
    rng = np.random.default_rng(m + n + k)
    x, q, v, f = layer(rng, op, m, n, k, "normal")
    t = gpu(x, TYPES[name], 4)
    x = f64(t)
    want = f(x)
    if op == "linear":
        mag, terms = np.abs(x) @ np.abs(v).T, k
    elif op == "grad":
        mag, terms = np.abs(x) @ np.abs(v), n
    else:
        mag, terms = np.abs(x).T @ np.abs(v), m
    check_between(product(op, t, q, dtype=TYPES[out]), want, (TERMS[name] * terms + 8) * 2.0 ** -23 * mag)


@pytest.mark.parametrize("m,n,k", SHAPES + [(256, 512, 1024)])
def test_product_of_two_mx4_is_exact_on_whole_numbers(m, n, k):
    """Codes are multiples of 1 at scale 2, at most 12: sums of 5000 products stay below 2^24."""
    rng = np.random.default_rng(m + 5 * n + k)
    qx, vx = random_mx(rng, m, k, 4, True)
    qw, vw = random_mx(rng, n, k, 4, True)
    want = vx @ vw.T
    assert np.array_equal(f64(F.mx4_linear(qx, qw, dtype=torch.float32)), want)
    for dt in (torch.bfloat16, torch.float16):
        assert torch.equal(F.mx4_linear(qx, qw, dtype=dt).cpu(), torch.from_numpy(want).to(dt))


@pytest.mark.parametrize("m,n,k", [(3001, 2888, 136), (2900, 3009, 2000), (4096, 2304, 256), (2823, 2817, 5), (260, 32008, 1300),
                                   (16, 16, 5000), (300, 200, 4992)])
def test_product_of_two_mx4_with_many_outputs_or_a_long_sum(m, n, k):
    rng = np.random.default_rng(m + n + k)
    qx, vx = random_mx(rng, m, k, 4, True)
    qw, vw = random_mx(rng, n, k, 4, True)
    want = torch.from_numpy(vx @ vw.T).float()
    got = F.mx4_linear(qx, qw, dtype=torch.float32).cpu()
    assert torch.equal(got, want), torch.nonzero(got != want)[:4].tolist()


@pytest.mark.parametrize("m,n,k", [(1, 64, 500), (40, 200, 321), (200, 130, 1000), (2600, 2700, 900)])
def test_product_of_two_mx4_with_any_scales(m, n, k):
    rng = np.random.default_rng(m + n + k)
    qx, vx = random_mx(rng, m, k, 4)
    qw, vw = random_mx(rng, n, k, 4)
    got, want, mag = f64(F.mx4_linear(qx, qw, dtype=torch.float32)), vx @ vw.T, np.abs(vx) @ np.abs(vw).T
    assert (np.abs(got - want) <= (k + 8) * 2.0 ** -23 * mag).all()


@pytest.mark.parametrize("name", ["fp16", "fp32"])
def test_terms_keep_all_of_a_float(name):
    """One product a sum, so that nothing is added: y is x times a power of two, to the last bit."""
    rng = np.random.default_rng(3)
    x = np.zeros((64, 64))
    np.fill_diagonal(x, rng.standard_normal(64) * np.exp2(rng.integers(-14, 15, 64)))
    codes, scales = O.quantize(np.full((96, 64), 0.5), 4)
    t = gpu(x, TYPES[name])
    got = F.mx4_linear(t, to_mx(codes, scales, 64, 4), dtype=torch.float32)
    assert np.array_equal(f64(got), f64(t).sum(axis=1, keepdims=True).repeat(96, axis=1) * 0.5)
    got = F.mx4_linear_grad_input(t, to_mx(*O.quantize(np.full((64, 96), 0.5), 4), 96, 4), dtype=torch.float32)
    assert np.array_equal(f64(got), f64(t).sum(axis=1, keepdims=True).repeat(96, axis=1) * 0.5)


@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("op", ["linear", "grad", "weight"])
@pytest.mark.parametrize("m", [2, 40, 200])
def test_infinities_and_nans_reach_the_rows_they_belong_to(op, name, m):
    rng = np.random.default_rng(11)
    n, k = 96, 160
    x, q, v, f = layer(rng, op, m, n, k, "whole")
    x[0, 5], x[1, 7] = np.inf, np.nan
    with np.errstate(invalid="ignore"):
        want = f(x)
    got = f64(product(op, gpu(x, TYPES[name], 3), q, dtype=torch.float32))
    assert np.array_equal(np.nan_to_num(got, nan=1e9, posinf=2e9, neginf=3e9), np.nan_to_num(want, nan=1e9, posinf=2e9, neginf=3e9))
    # a block whose scale says NaN
    x, q, v, f = layer(rng, op, m, n, k, "whole")
    scales = q.scales.clone()
    scales[1, 2] = 255
    q = type(q)(q.codes, scales, k)
    v[1, 64:96] = np.nan
    want = f(x)
    got = f64(product(op, gpu(x, TYPES[name]), q, dtype=torch.float32))
    assert np.array_equal(np.nan_to_num(got, nan=1e9), np.nan_to_num(want, nan=1e9)) and np.isnan(got).any()


@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("op", ["linear", "grad", "weight"])
def test_infinities_and_nans_among_many_outputs(op, name):
    rng = np.random.default_rng(13)
    rows, cols, sums = 2900, 3000, 330
    m, n, k = dict(linear=(rows, cols, sums), grad=(rows, sums, cols), weight=(sums, rows, cols))[op]
    x, q, v, f = layer(rng, op, m, n, k, "whole")
    x[0, 5], x[300, 7], x[m - 1, x.shape[1] - 1] = np.inf, np.nan, -np.inf
    scales = q.scales.clone()
    scales[q.rows - 1, 2] = 255
    v[q.rows - 1, 64:96] = np.nan
    with np.errstate(invalid="ignore"):
        want = f(x)
    for pad in (0, 3):
        got = f64(product(op, gpu(x, TYPES[name], pad), type(q)(q.codes, scales, k), dtype=torch.float32))
        assert np.array_equal(np.nan_to_num(got, nan=1e9, posinf=2e9, neginf=3e9),
                              np.nan_to_num(want, nan=1e9, posinf=2e9, neginf=3e9))


def test_product_of_two_mx4_with_a_nan_block():
    rng = np.random.default_rng(12)
    qx, vx = random_mx(rng, 40, 160, 4, True)
    qw, vw = random_mx(rng, 70, 160, 4, True)
    sx, sw = qx.scales.clone(), qw.scales.clone()
    sx[3, 1], sw[5, 4] = 255, 255
    vx[3, 32:64], vw[5, 128:] = np.nan, np.nan
    got = f64(F.mx4_linear(F.MX4(qx.codes, sx, 160), F.MX4(qw.codes, sw, 160), dtype=torch.float32))
    assert np.array_equal(np.nan_to_num(got, nan=1e9), np.nan_to_num(vx @ vw.T, nan=1e9))


@pytest.mark.parametrize("e", [0, 3, 250])
def test_scales_at_the_ends_of_their_range(e):
    """Subnormal and huge weights, with inputs that bring the products back near 1."""
    rng = np.random.default_rng(e)
    q, _ = random_mx(rng, 70, 96, 4, True)
    scales = torch.full_like(q.scales, e)
    v = O.values(q.codes.cpu().numpy(), scales.cpu().numpy(), 96)
    q = F.MX4(q.codes, scales, 96)
    up = 2.0 ** (100 if e < 100 else -100)
    for dt in (torch.bfloat16, torch.float32):
        for m in (1, 20, 150):
            x = whole(rng, m, 96) * up
            assert np.array_equal(f64(F.mx4_linear(gpu(x, dt), q, dtype=torch.float32)), x @ v.T)
            x = whole(rng, m, 70) * up
            assert np.array_equal(f64(F.mx4_linear_grad_input(gpu(x, dt), q, dtype=torch.float32)), x @ v)
    q8, _ = random_mx(rng, 70, 96, 8, True)
    s8 = torch.full_like(q8.scales, e)
    v = O.values(q8.codes.cpu().numpy(), s8.cpu().numpy(), 96)
    x = whole(rng, 70, 40) * up
    assert np.array_equal(f64(F.mx8_weight_grad(gpu(x, torch.bfloat16), F.MX8(q8.codes, s8, 96))), x.T @ v)


def test_sums_over_nothing():
    z = lambda *s: torch.zeros(*s, device="cuda")
    assert F.mx4_linear(z(3, 0), F.mx4_quantize(z(5, 0))).tolist() == [[0.0] * 5] * 3
    assert F.mx4_linear(F.mx4_quantize(z(3, 0)), F.mx4_quantize(z(5, 0))).float().tolist() == [[0.0] * 5] * 3
    assert F.mx4_linear_grad_input(z(3, 0), F.mx4_quantize(z(0, 40))).abs().sum() == 0
    assert F.mx8_weight_grad(z(0, 7), F.mx8_quantize(z(0, 40))).tolist() == [[0.0] * 40] * 7
    acc = torch.full((7, 40), 2.0, device="cuda")
    assert (F.mx8_weight_grad(z(0, 7), F.mx8_quantize(z(0, 40)), out=acc, accumulate=True) == 2).all()
    assert F.mx4_linear(z(0, 64), F.mx4_quantize(z(5, 64))).shape == (0, 5)
    assert F.mx4_linear(z(2, 64), F.mx4_quantize(z(0, 64))).shape == (2, 0)


@pytest.mark.parametrize("m,n,k", [(40, 70, 100), (2000, 64, 96), (3, 300, 300)])
def test_weight_grad_accumulates(m, n, k):
    rng = np.random.default_rng(m)
    x, q, _, f = layer(rng, "weight", m, n, k, "whole")
    wide = torch.full((n, k + 5), 3.0, device="cuda")
    F.mx8_weight_grad(gpu(x, torch.bfloat16), q, out=wide[:, 2:2 + k], accumulate=True)
    assert np.array_equal(f64(wide[:, 2:2 + k]), f(x) + 3) and (wide[:, :2] == 3).all() and (wide[:, 2 + k:] == 3).all()
    F.mx8_weight_grad(gpu(x, torch.bfloat16), q, out=wide[:, 2:2 + k])
    assert np.array_equal(f64(wide[:, 2:2 + k]), f(x))
    with pytest.raises(ValueError, match="float32"):
        F.mx8_weight_grad(gpu(x, torch.bfloat16), q, dtype=torch.bfloat16, accumulate=True)


def test_outputs_are_the_same_every_time():
    """Long sums of few outputs are cut into parts; their joining does not depend on which part ends first."""
    rng = np.random.default_rng(21)
    for op, m, n, k in (("linear", 3, 130, 8000), ("grad", 3, 8000, 130), ("weight", 8000, 70, 130)):
        x, q, _, _ = layer(rng, op, m, n, k, "normal")
        t = gpu(x, torch.float32)
        first = product(op, t, q)
        assert all(torch.equal(first, product(op, t, q)) for _ in range(5))


def test_weights_past_32_bit_offsets():
    """140,000 x 65,536 weights, 4.6 GB of codes: the last rows use the same codes as the first."""
    rng = np.random.default_rng(8)
    q, v = random_mx(rng, 500, 65536, 4, True)
    w = F.MX4(q.codes.repeat(280, 1), q.scales.repeat(280, 1), 65536)
    x = gpu(whole(rng, 2, 65536, -1, 2), torch.bfloat16)
    got = f64(F.mx4_linear(x, w, dtype=torch.float32)).reshape(2, 280, 500)
    assert np.array_equal(got, np.repeat((f64(x) @ v.T)[:, None], 280, axis=1))
    dy = torch.zeros(2, 140000, dtype=torch.bfloat16, device="cuda")
    dy[0, 139999], dy[1, 3], dy[1, 131075] = 2.0, 1.0, 3.0
    got = f64(F.mx4_linear_grad_input(dy, w, dtype=torch.float32))
    assert np.array_equal(got[0], 2 * v[499]) and np.array_equal(got[1], v[3] + 3 * v[131075 % 500])


def test_gradients_are_the_products_differences():
    """y is linear in x and in W, so its differences are exact: <dy, y(x + d) - y(x)> = <dx, d>, and the same for
    W with x as it was kept."""
    rng = np.random.default_rng(31)
    m, n, k = 37, 65, 120
    qw, w = random_mx(rng, n, k, 4, True)
    qx, xk = random_mx(rng, m, k, 8, True)
    x, d, dy = whole(rng, m, k), whole(rng, m, k, -2, 3), whole(rng, m, n, -2, 3)
    y = lambda v: f64(F.mx4_linear(gpu(v, torch.float32), qw))
    dx = f64(F.mx4_linear_grad_input(gpu(dy, torch.float32), qw))
    assert (dy * (y(x + d) - y(x))).sum() == (dx * d).sum()
    dw = f64(F.mx8_weight_grad(gpu(dy, torch.float32), qx))
    delta = whole(rng, n, k, -2, 3)
    assert (dy * (xk @ (w + delta).T - xk @ w.T)).sum() == (dw * delta).sum()


def test_products_refuse_what_does_not_fit():
    x = torch.zeros(4, 64, device="cuda")
    w, k8 = F.mx4_quantize(torch.zeros(10, 64, device="cuda")), F.mx8_quantize(x)
    for call, match in [
        (lambda: F.mx4_linear(x[:, :63], w), "63 columns"),
        (lambda: F.mx4_linear(x, k8), "must be an MX4"),
        (lambda: F.mx4_linear(k8, w), "must be an MX4"),
        (lambda: F.mx4_linear(F.mx4_quantize(x[:, :32]), w), "any x 64"),
        (lambda: F.mx4_linear(x, w, out=torch.zeros(4, 11, device="cuda")), "shape"),
        (lambda: F.mx4_linear(x, w, dtype=torch.bfloat16, out=torch.zeros(4, 10, device="cuda")), "bfloat16"),
        (lambda: F.mx4_linear(x, w, dtype=torch.float64), "dtype must be"),
        (lambda: F.mx4_linear(x, w, work=torch.zeros(4, device="cuda")), "uint8"),
        (lambda: F.mx4_linear_grad_input(x, w), "10 rows"),
        (lambda: F.mx8_weight_grad(x[:3], k8), "3 rows"),
        (lambda: F.mx8_act(x, x[:, :32]), "shape and type"),
        (lambda: F.mx8_act(x, saved_gate=k8), "without a gate"),
        (lambda: F.mx8_act_grad(x[:2], k8), "kept x 4 x 64"),
        (lambda: F.mx8_act_grad(x, k8, out_gate=x), "without a saved gate"),
    ]:
        with pytest.raises(ValueError, match=match):
            call()
    with pytest.raises(F.FastrackError, match="workspace"):
        big = torch.zeros(4096, 63, device="cuda", dtype=torch.float16)
        F.mx4_linear(big, F.mx4_quantize(big), work=torch.zeros(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(F.FastrackError, match="overlaps"):
        F.mx4_linear(x, F.mx4_quantize(torch.zeros(64, 64, device="cuda")), out=x)


# ---- the activation ----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (3, 33, 0), (5, 64, 8), (20, 200, 3), (64, 1000, 0)])
def test_activation_and_its_gradient(kind, gated, name, rows, cols, pad):
    """f and f' to a few units of the 32-bit arithmetic (16-bit types: the hardware's exponential, 2^-19 of a term
    of magnitude 1 + |x|), then rounded to the output's type."""
    rng = np.random.default_rng(rows + cols)
    dt = TYPES[name]
    x = gpu(rng.standard_normal((rows, cols)) * 4, dt, pad)
    g = gpu(rng.standard_normal((rows, cols)), dt, pad) if gated else None
    dy = gpu(rng.standard_normal((rows, cols)), dt, pad)
    y, sx, sg = F.mx8_act(x, g, act=kind)
    check_mx(sx, *O.quantize(f64(x), 8))
    gv = 1.0
    if gated:
        check_mx(sg, *O.quantize(f64(g), 8))
        gv = f64(g)
    rel = 2.0 ** -20 if name == "fp32" else 2.0 ** -18
    xv = f64(x)
    near = lambda got, want, size: check_between(got, want, rel * size)
    near(y, O.act(xv, kind)[0] * gv, (1 + np.abs(xv)) * np.abs(gv))
    dx, dg = F.mx8_act_grad(dy, sx, sg, act=kind)
    kx = O.values(sx.codes.cpu().numpy(), sx.scales.cpu().numpy(), cols)
    kg = O.values(sg.codes.cpu().numpy(), sg.scales.cpu().numpy(), cols) if gated else 1.0
    f, df = O.act(kx, kind)
    d = f64(dy)
    near(dx, d * kg * df, (1 + np.abs(kx)) * np.abs(d * kg))
    if gated:
        near(dg, d * f, (1 + np.abs(kx)) * np.abs(d))
    else:
        assert dg is None
    # against differences of the activation itself: error h^2 / 6 times a third derivative below 1
    h = 1e-4
    diff = (O.act(kx + h, kind)[0] - O.act(kx - h, kind)[0]) / (2 * h)
    check_between(dx, d * kg * diff, np.abs(d * kg) * (1e-7 + (1 + np.abs(kx)) * rel))


def test_activation_into_given_buffers_and_special_values():
    x = torch.randn(6, 100, device="cuda").to(torch.bfloat16)
    both = torch.randn(6, 200, device="cuda").to(torch.bfloat16)
    y, sx, sg = F.mx8_act(both[:, :100], both[:, 100:])
    out, k1, k2 = torch.empty_like(y), F.MX8.empty(6, 100), F.MX8.empty(6, 100)
    r = F.mx8_act(both[:, :100], both[:, 100:], out=out, saved=k1, saved_gate=k2)
    assert r[0] is out and r[1] is k1 and r[2] is k2 and torch.equal(out, y)
    assert torch.equal(k1.codes, sx.codes) and torch.equal(k2.codes, sg.codes) and torch.equal(k2.scales, sg.scales)
    grads = torch.empty_like(both)
    dx, dg = F.mx8_act_grad(x, sx, sg, out=grads[:, :100], out_gate=grads[:, 100:])
    want = F.mx8_act_grad(x, sx, sg)
    assert torch.equal(grads[:, :100], want[0]) and torch.equal(grads[:, 100:], want[1])
    z = torch.zeros(2, 64, device="cuda")
    z[0, 3], z[1, 40] = float("inf"), float("nan")
    y, s, _ = F.mx8_act(z, act="gelu")
    assert y[0, 3] == float("inf") and y[1, 40].isnan() and y.isnan().sum() == 1
    dx, _ = F.mx8_act_grad(torch.ones_like(z), s, act="gelu")
    assert dx[0, :32].isnan().all() and dx[1, 32:].isnan().all() and (dx[0, 32:] == 0.5).all()
    big = torch.tensor([[-3e38, -200.0, -90.0, 0.0, 90.0, 200.0, 3e38]], device="cuda")
    for kind in ("silu", "gelu"):
        y, s, _ = F.mx8_act(big, act=kind)
        assert torch.equal(y[0, 3:], big[0, 3:]) and (y[0, :3].abs() < 1e-30).all()
    for rows, cols in ((0, 32), (4, 0)):
        e = torch.zeros(rows, cols, device="cuda")
        y, s, g = F.mx8_act(e, e)
        assert y.shape == e.shape and F.mx8_act_grad(e, s, g)[1].shape == e.shape


# ---- streams and graphs --------------------------------------------------------------------------------------------

def test_calls_on_another_stream():
    rng = np.random.default_rng(41)
    s = torch.cuda.Stream()
    x, q, _, f = layer(rng, "linear", 5, 300, 4000, "whole")
    t = gpu(x, torch.float32)
    ready = torch.cuda.Event()
    for _ in range(3):
        ready.record()
        s.wait_event(ready)
        y = F.mx4_linear(t, q, stream=s)
        del_me = torch.empty(1 << 20, device="cuda")   # may take what the call freed
        del_me.fill_(float("nan"))
        s.synchronize()
        assert np.array_equal(f64(y), f(x))
    with torch.cuda.stream(s):
        y2 = F.mx4_linear(t, q)
    s.synchronize()
    assert np.array_equal(f64(y2), f(x))


def test_captured_calls_replay():
    """A layer's step in a graph, replayed on new inputs between eager work, against the eager results."""
    rng = np.random.default_rng(42)
    m, n, k = 24, 200, 3000
    qw, _ = random_mx(rng, n, k, 4)
    x = torch.zeros(m, k, device="cuda", dtype=torch.bfloat16)
    dy = torch.zeros(m, n, device="cuda", dtype=torch.float16)

    def step():
        kept = F.mx8_quantize(x)
        y, s, _ = F.mx8_act(F.mx4_linear(x, qw, dtype=torch.float16), act="gelu")
        d, _ = F.mx8_act_grad(dy, s, act="gelu")
        return y, F.mx4_linear_grad_input(d, qw), F.mx8_weight_grad(d, kept), F.mx4_linear(F.mx4_quantize(x), qw)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for r in range(4):
        x.copy_(torch.randn(m, k, device="cuda"))
        dy.copy_(torch.randn(m, n, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(outs, step()):
            assert torch.equal(got, want), r
        torch.cuda.synchronize()
