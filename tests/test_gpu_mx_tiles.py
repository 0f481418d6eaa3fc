"""Products by large tiles on operands that tell every block and every term apart: scales that differ from block to
block, floats whose second and third bf16 terms are not 0, outputs of every type into slices of wider tensors.

Compared bit for bit: all values are whole numbers, and each sum has so few float values that are not 0 that every
partial sum stays below 2^24. Operands lie at an odd stride, so that they are laid out in the workspace, whose size
tells that the product runs by large tiles, and in how many parts its sums are cut."""
import numpy as np
import pytest
import torch

import mx_oracle as O
import paper_2410_15240_amd as F

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
CODE = {"bf16": 0, "fp16": 1, "fp32": 2}
TERMS = {"bf16": 1, "fp16": 2, "fp32": 3}
# Largest float (8, 11 and 17 significant bits: as many terms) and how many of them a sum has; an MX value is at
# most 64.
LARGEST = {"bf16": 255, "fp16": 2047, "fp32": 131071}
COUNT = {"bf16": 900, "fp16": 120, "fp32": 2}
OPS = {"linear": 0, "grad": 1, "weight": 2}


def varied_mx(rng, rows, cols, bits):
    """Whole numbers up to 48 (64) in blocks of three scales."""
    nb = O.blocks(cols)
    if bits == 4:
        codes = rng.integers(0, 256, (rows, nb * 16)).astype(np.uint8)
    else:
        codes = rng.integers(-16, 17, (rows, nb * 32)).astype(np.int8)
    scales = ((128 if bits == 4 else 133) + rng.integers(0, 3, (rows, nb))).astype(np.uint8)
    inside = np.arange(nb * 32).reshape(nb, 32) < cols
    blocks = codes.reshape(rows, nb, -1)
    blocks &= (inside[:, 0::2] * 0x0F + inside[:, 1::2] * 0xF0).astype(np.uint8) if bits == 4 else -inside.astype(np.int8)
    q = {4: F.MX4, 8: F.MX8}[bits](torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), cols)
    return q, torch.from_numpy(O.values(codes, scales, cols))


def sparse(rng, rows, cols, name, along_rows):
    """COUNT values (odd numbers, so that no bit of theirs is spare) in every row, or in every column."""
    lines, length = (rows, cols) if along_rows else (cols, rows)
    x = np.zeros((lines, length))
    n = min(COUNT[name], length)
    at = rng.integers(0, length, (lines, n))
    low = LARGEST[name] // 2
    x[np.arange(lines)[:, None], at] = (rng.integers(low // 2, low, (lines, n)) * 2 + 1) * rng.choice([-1, 1], (lines, n))
    return torch.from_numpy(x if along_rows else np.ascontiguousarray(x.T))


def case(op, name, m, n, k):
    rng = np.random.default_rng(m + 3 * n + 7 * k + len(op) + TERMS[name])
    q, v = varied_mx(rng, m if op == "weight" else n, k, 8 if op == "weight" else 4)
    x = sparse(rng, m, k if op == "linear" else n, name, op != "weight")
    want = dict(linear=lambda: x @ v.T, grad=lambda: x @ v, weight=lambda: x.T @ v)[op]()
    wide = torch.full((x.shape[0], x.shape[1] + 4 - x.shape[1] % 2 - 1), float("nan"), dtype=TYPES[name])
    wide[:, 1:1 + x.shape[1]] = x.to(TYPES[name])
    return wide.cuda()[:, 1:1 + x.shape[1]], q, want.float()


def run(op, *a, **kw):
    return dict(linear=F.mx4_linear, grad=F.mx4_linear_grad_input, weight=F.mx8_weight_grad)[op](*a, **kw)


def check_way(op, name, t, m, n, k, parts, decoded):
    rows, cols = t.shape
    need = F.lib().fastrack_mx_work_bytes(OPS[op], CODE[name], t.data_ptr(), t.stride(0), m, n, k)
    laid = -(-TERMS[name] * rows * -(-cols // 8) * 16 // 256) * 256
    out = {"linear": m * n, "grad": m * k, "weight": n * k}[op]
    assert need == laid + (m * O.blocks(k) * 64 if decoded else 0) + (parts * out * 4 if parts > 1 else 0)


# op, m, n, k, parts by type, whether the kept input is decoded beforehand by type
SHAPES = [
    ("linear", 2900, 3009, 700, (1, 1, 1), (0, 0, 0)), ("grad", 2900, 700, 3009, (1, 1, 1), (0, 0, 0)),   # tiles of 256
    ("weight", 700, 2900, 3009, (1, 1, 1), (0, 1, 1)), ("weight", 330, 4200, 4096, (1, 1, 1), (1, 1, 1)),
    ("linear", 1021, 4001, 1000, (1, 1, 1), (0, 0, 0)), ("grad", 1021, 1000, 4001, (1, 1, 1), (0, 0, 0)),  # of 128
    ("weight", 1000, 1021, 4001, (1, 1, 1), (0, 0, 0)),
    ("linear", 300, 5000, 5000, (2, 2, 2), (0, 0, 0)), ("grad", 300, 5000, 5000, (2, 2, 2), (0, 0, 0)),    # of 128, cut
    ("weight", 6001, 500, 1111, (7, 7, 7), (0, 0, 0)),
]


@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("op,m,n,k,parts,decoded", SHAPES)
def test_scales_terms_and_outputs_of_large_tiles(op, m, n, k, parts, decoded, name):
    t, q, want = case(op, name, m, n, k)
    check_way(op, name, t, m, n, k, parts[CODE[name]], decoded[CODE[name]])
    rows, cols = want.shape
    for out in TYPES.values():
        wide = torch.full((rows, cols + 5), 7.0, dtype=out, device="cuda")
        run(op, t, q, out=wide[:, 2:2 + cols])
        got = wide[:, 2:2 + cols].cpu()
        assert torch.equal(got, want.to(out)), (out, torch.nonzero(got != want.to(out))[:4].tolist())
        assert (wide[:, :2] == 7).all() and (wide[:, 2 + cols:] == 7).all()


@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("m,n,k", [s[1:4] for s in SHAPES if s[0] == "weight"])
def test_weight_grad_accumulates_in_large_tiles(m, n, k, name):
    t, q, want = case("weight", name, m, n, k)
    wide = torch.full((n, k + 5), 3.0, device="cuda")
    for times in (1, -1):
        F.mx8_weight_grad(t * times, q, out=wide[:, 2:2 + k], accumulate=True)
        assert torch.equal(wide[:, 2:2 + k].cpu(), want + 3 if times == 1 else torch.full_like(want, 3.0))
        assert (wide[:, :2] == 3).all() and (wide[:, 2 + k:] == 3).all()


@pytest.mark.parametrize("m,n,k", [(2900, 3009, 1300), (2304, 4096, 1280), (600, 2000, 3000), (70, 2000, 5000)])
def test_product_of_two_mx4_of_varied_scales(m, n, k):
    """Values up to 48 on both sides: sums of 5000 products stay below 2^24. Tiles of 256 with five whole stages, with and
    without a short one; of 128, uncut and cut."""
    rng = np.random.default_rng(m + n + k)
    (qx, vx), (qw, vw) = varied_mx(rng, m, k, 4), varied_mx(rng, n, k, 4)
    want = (vx @ vw.T).float()
    for out in TYPES.values():
        wide = torch.full((m, n + 3), 7.0, dtype=out, device="cuda")
        F.mx4_linear(qx, qw, out=wide[:, 1:1 + n])
        got = wide[:, 1:1 + n].cpu()
        assert torch.equal(got, want.to(out)), (out, torch.nonzero(got != want.to(out))[:4].tolist())
        assert (wide[:, :1] == 7).all() and (wide[:, 1 + n:] == 7).all()
