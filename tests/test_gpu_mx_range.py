"""Products of 32-bit operands at the bottom of their range. Their terms in bf16 end at 2^-133 (include/fastrack.h):
bits of a value from there up come through whatever the call's size, so values from 2^-110 up come through whole; of
smaller ones the bits below may be dropped, never more."""
import numpy as np
import pytest
import torch

import mx_oracle as O
import paper_2410_15240_amd as F

pytestmark = pytest.mark.gpu

# Tokens, outputs and inputs: one and two tokens, small tiles (cut and not), tiles of 128 (cut and not), of 256, and
# of 256 with the kept input decoded before.
SIZES = [(1, 96, 600), (2, 96, 600), (3, 96, 600), (40, 96, 160), (37, 130, 3000), (300, 900, 2000), (2000, 1000, 1500),
         (2900, 3009, 700), (700, 2900, 3009)]
UP = 113


def product(op, a, m, n, k, ones):
    """The product of `a` with an MX matrix of 2^UP (ones) or of 2^UP times a random sign and 1 or 2, and its values."""
    rng = np.random.default_rng(m + n + k)
    rows, cols, bits = (m, k, 8) if op == "weight" else (n, k, 4)
    v = np.ones((rows, cols)) if ones else rng.choice([1.0, 2.0], (rows, cols)) * rng.choice([1.0, -1.0], (rows, cols))
    codes, scales = O.quantize(v * 2.0 ** UP, bits)
    q = {4: F.MX4, 8: F.MX8}[bits](torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), cols)
    t = torch.from_numpy(a.astype(np.float32)).cuda()
    fn = dict(linear=F.mx4_linear, grad=F.mx4_linear_grad_input, weight=F.mx8_weight_grad)[op]
    got = fn(t, q).cpu().double().numpy()
    return got, v * 2.0 ** UP, dict(linear=lambda w: a @ w.T, grad=lambda w: a @ w, weight=lambda w: a.T @ w)[op]


@pytest.mark.parametrize("op", ["linear", "grad", "weight"])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_single_values_down_to_the_smallest(op, m, n, k):
    rng = np.random.default_rng(m * 3 + n + k)
    rows, cols = (m, k) if op == "linear" else (m, n)
    a = np.zeros((rows, cols))
    lines = cols if op == "weight" else rows       # one value to each sum
    at = np.arange(lines)
    value = rng.uniform(1, 2, lines) * 2.0 ** rng.integers(-150, -99, lines) * rng.choice([1.0, -1.0], lines)
    value = value.astype(np.float32).astype(np.float64)
    where = (rng.integers(0, rows, lines), at) if op == "weight" else (at, rng.integers(0, cols, lines))
    a[where] = value
    got, _, _ = product(op, a, m, n, k, ones=True)
    cut = np.trunc(value * 2.0 ** 133) * 2.0 ** -133
    assert (cut == value)[np.abs(value) >= 2.0 ** -110].all() and (lines < 40 or (cut != value).any())
    whole = got == (value * 2.0 ** UP)[:, None]
    assert (whole | (got == (cut * 2.0 ** UP)[:, None])).all()


@pytest.mark.parametrize("op", ["linear", "grad", "weight"])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_sums_of_small_values_are_exact(op, m, n, k):
    """Up to 3009 terms of at most 2^10 units of 2^(UP - 133): every partial sum is below 2^23 of them."""
    rng = np.random.default_rng(m + n * 3 + k)
    a = rng.integers(-512, 513, (m, k) if op == "linear" else (m, n)) * 2.0 ** -133
    got, w, f = product(op, a, m, n, k, ones=False)
    assert np.array_equal(got, f(w))


@pytest.mark.parametrize("m,n,k", SIZES)
def test_the_largest_beside_the_smallest(m, n, k):
    """The largest finite value comes out as it is, whichever way its terms are taken, and an infinity stays one."""
    a = np.zeros((m, k))
    big = float(np.finfo(np.float32).max)
    a[0, 5], a[0, 70] = big, 2.0 ** -149
    if m > 1:
        a[1, 3], a[1, 64] = np.inf, 2.0 ** -140
    w = np.zeros((n, k))
    w[:, 5], w[:, 70], w[:, 3] = 1.0, 2.0 ** -20, 1.0
    codes, scales = O.quantize(w, 4)
    assert np.array_equal(O.values(codes, scales, k), w)
    q = F.MX4(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), k)
    got = F.mx4_linear(torch.from_numpy(a.astype(np.float32)).cuda(), q).cpu().double().numpy()
    assert (got[0] == big).all() and (m == 1 or (got[1] == np.inf).all())


@pytest.mark.parametrize("e", [252, 253, 254])
@pytest.mark.parametrize("m", [1, 3, 200])
def test_weights_at_the_top_of_the_scales(m, e):
    """Every code at the largest scales, against inputs of 2^-60 everywhere: values of 2^128 and more are infinite, but
    in the product of two MX4 matrices."""
    n, k = 16, 512
    codes = np.arange(n, dtype=np.uint8)[:, None] * np.full((1, k // 2), 17, np.uint8)
    scales = np.full((n, k // 32), e, np.uint8)
    v = O.values(codes, scales, k)
    w = F.MX4(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), k)
    x = torch.full((m, k), 2.0 ** -60, device="cuda")
    want, past = (v * 2.0 ** -60).sum(axis=1), np.abs(v[:, 0]) >= 2.0 ** 128
    assert past.any() == (e > 252)
    for row in F.mx4_linear(F.mx4_quantize(x), w, dtype=torch.float32).cpu().double().numpy():
        assert np.array_equal(row, want)
    for dt in (torch.bfloat16, torch.float16, torch.float32):
        x = torch.full((m, k), 2.0 ** -24, device="cuda", dtype=dt)
        for row in F.mx4_linear(x, w, dtype=torch.float32).cpu().double().numpy():
            assert np.array_equal(row[~past], want[~past] * 2.0 ** 36) and not np.isfinite(row[past]).any()
    got = F.mx4_dequantize(w, dtype=torch.float32).cpu().double().numpy()
    assert np.array_equal(got[~past], v[~past]) and np.array_equal(got[past], np.copysign(np.inf, v[past]))
