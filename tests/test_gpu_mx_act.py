"""The activations' far ends, where the value is small: it has to be right relative to itself, not to 1.

Bounds. GELU in 32 bits: the fit of the tail (2^-28), its evaluation (3 roundings of t, 10 of the polynomial, whose terms
are at most 14 times their sum: its leading ones, where t is small, about the sum itself), the exponential and three
products, together below 16 units of 2^-24. In 16-bit types the exponential's argument, x^2 / 2, is rounded twice (its
constant is off by a quarter of a unit, for which 2^-18 leaves room), and the fit is 2^-20. SiLU in 16-bit types: the
argument is -x, times a rounded constant: 2 units of |x|, and the exponential's and the reciprocal's own unit or two.
In 32 bits: an exponential, a sum, a division and a product, 1 unit each or 2; and where s is small the gradient's
rest, 1 - s, is right to a unit of 1, times x.
"""
import numpy as np
import pytest
import torch

import mx_oracle as O
import paper_2410_15240_amd as F

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def f64(t):
    return t.detach().cpu().double().numpy()


def check_between(got, want, bound):
    """got is some value of [want - bound, want + bound] rounded to got's type."""
    lo, hi = (f64(torch.from_numpy(want + s * bound).to(got.dtype)) for s in (-1, 1))
    g = f64(got)
    worst = np.unravel_index(np.argmax(np.where((g >= lo) & (g <= hi), 0, 1)), g.shape)
    assert ((g >= lo) & (g <= hi)).all(), (g[worst], want[worst], bound[worst])


def relative(kind, name, x):
    if name == "fp32":
        return np.full(x.shape, 2.0 ** -20)
    return 2.0 ** -18 + (x * x * 2.0 ** -24 if kind == "gelu" else np.abs(x) * 2.0 ** -23)


@pytest.mark.parametrize("kind,low", [("gelu", -13.0), ("silu", -87.0)])
@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("gated", [False, True])
def test_the_negative_end_is_right_relative_to_itself(kind, low, name, gated):
    dt = TYPES[name]
    x = torch.linspace(low, -0.01, 64 * 96, dtype=torch.float64).view(64, 96).to(dt).cuda()
    gate = torch.full_like(x, 1.5) if gated else None
    y, sx, sg = F.mx8_act(x, gate, act=kind)
    by = 1.5 if gated else 1.0
    xv = f64(x)
    want = O.act(xv, kind)[0] * by
    check_between(y, want, np.abs(want) * relative(kind, name, xv))
    one = torch.ones_like(x)
    dx, dg = F.mx8_act_grad(one, sx, sg, act=kind)
    kept = O.values(sx.codes.cpu().numpy(), sx.scales.cpu().numpy(), x.shape[1])
    f, df = O.act(kept, kind)
    # f' has a zero here: its two terms are s or P and the rest
    first = f / kept
    size = np.abs(first) * (1 + np.abs(kept)) if kind == "silu" else np.abs(first) + np.abs(df - first)
    check_between(dx, df * by, size * by * 2 * relative(kind, name, kept))
    if gated:
        check_between(dg, f, np.abs(f) * relative(kind, name, kept))


@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("name", list(TYPES))
def test_the_positive_end_and_beyond(kind, name):
    """x itself far up, 0 far down, at the largest values too."""
    dt = TYPES[name]
    big = float(torch.finfo(dt).max)
    x = torch.tensor([[-big, -1e4, -300.0, -150.0, 0.0, -0.0, 25.0, 150.0, 1e4, big]], dtype=dt, device="cuda")
    y, s, _ = F.mx8_act(x, act=kind)
    assert torch.equal(y[0, 4:], x[0, 4:]) and not y[0, :4].any()
    x = torch.tensor([[20.0] * 32 + [-200.0] * 32 + [0.0] * 32], dtype=dt, device="cuda")
    dx, _ = F.mx8_act_grad(torch.ones_like(x), F.mx8_quantize(x), act=kind)
    assert (dx[0, :32] == 1).all() and not dx[0, 32:64].any() and (dx[0, 64:] == 0.5).all()
