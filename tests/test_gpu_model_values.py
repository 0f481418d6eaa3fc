"""Cross entropy on the GPU where its logits are known exactly: in 32 bits from the smallest to the largest, next to each other and
far from zero. A logit here is one product, or a sum that 24 bits hold, times the scale, rounded once: what is left to be off is the
softmax."""
import math

import pytest
import torch

import model_oracle as O
import paper_2410_15240_amd as F
from test_gpu_model import close, generator, values

pytestmark = pytest.mark.gpu

TYPES = O.TYPES
# Logits through the workspace, their statistics in one launch and in parts.
FEW = [(3, 700, 64), (40, 20000, 64), (300, 3000, 333)]
# In whole tiles of 128 and of 256.
TILES = [(600, 9000, 64), (2100, 9000, 300)]
# A sum of exponentials: 66 additions in a thread, 20 joinings of five roundings each, the exponentials' own two units and what
# their arguments' rounding makes of them (no more than the logarithm of the number of classes, 14, once and a quarter), the logarithm.
SUM = 256 * O.U32


def head(v, k, gen):
    """An MX4 head whose first column is 6 for one class, -6 for another, from -4 to 4 for the others; these two; the column."""
    w = torch.randint(-4, 5, (v, k), device="cuda", generator=gen).float()
    w[:, 1] = 6.0   # (every block's scale is 1)
    top, low = v // 3, v - 1
    w[top, 0], w[low, 0] = 6.0, -6.0
    q = F.mx4_quantize(w)
    assert torch.equal(F.mx4_dequantize(q, dtype=torch.float32)[:, :2], w[:, :2])
    return q, top, low


def targets(m, v, gen, *often):
    ids = torch.randint(0, v, (m,), device="cuda", generator=gen)
    for i, c in enumerate(often):
        ids[i + 1::len(often) + 2] = c
    return ids


def check_loss(x, w, ids, scale, z):
    """z: the logits in 64 bits."""
    loss, lse = F.mx4_cross_entropy(x, w, ids, scale=scale)
    want = torch.logsumexp(z, dim=1)
    close(lse, want, SUM, what="lse")
    want = want - z[torch.arange(len(ids), device="cuda"), ids]
    close(loss, want, SUM + O.U32 * want.abs(), what="loss")


def check_grad(x, w, ids, scale, z, t):
    m, k = x.shape
    gen = generator(m)
    lse = torch.logsumexp(z, dim=1).float()   # (the gradient is that for the lse that is given)
    x8 = F.mx8_quantize(torch.randn(m, k, device="cuda", generator=gen))
    w64, hot = F.mx4_dequantize(w, dtype=torch.float32).double(), torch.zeros_like(z)
    hot[torch.arange(m, device="cuda"), ids] = 1.0
    for dloss in (torch.rand(m, device="cuda", generator=gen) + 0.5, torch.full((m,), 0.7, device="cuda")):
        dloss = dloss / abs(scale)
        f = (dloss.double() * scale)[:, None]
        d = z - lse.double()[:, None]
        p = torch.exp(d)
        dz = f * (p - hot)
        # e^d by 2^(d / ln 2): the arguments' rounding, the exponential's units; the factor, its common part divided out and
        # multiplied in again. An exponential below 2^-126 is 0, the smallest number that the GPU's makes, and a dz has no
        # terms below 2^-133, bf16's smallest: each is less than 2^-126, of the factor and of the term.
        off_dz = f.abs() * p * O.U32 * (2 * d.abs() + 8) + 8 * O.U32 * dz.abs() + 2.0 ** -126 * (f.abs() + 1)
        for wt in ("bf16", "fp32"):
            dx, dw = F.mx4_cross_entropy_grad(dloss, x, w, ids, lse, saved=x8, scale=scale, weight_dtype=TYPES[wt])
            for got, a, o, b, n in ((dx, dz, off_dz, w64, z.shape[1]), (dw, dz.t().contiguous(), off_dz.t().contiguous(), values(x8), m)):
                if got.dtype == torch.bfloat16:
                    o = o + O.half_step(torch.bfloat16, a)
                elif got.dtype == torch.float16:
                    o = o + 2.0 ** -16 * a.abs()
                close(got, a @ b, o @ b.abs() + (3 * n + 32) * O.U32 * (a.abs() @ b.abs()), what="dx" if got is dx else "dw")


def logits_of_any_size(t, scale, m, v, k):
    """From about 1 up to 2^125, of rows whose largest is one class's and of rows where several share it."""
    gen = generator(m + v)
    w, top, low = head(v, k, gen)
    most = 13.0 if t == "fp16" else 121.0
    x = torch.zeros(m, k, device="cuda")
    size = torch.exp2(torch.linspace(0.0, most, m, device="cuda")) * (1 + 0.99 * torch.rand(m, device="cuda", generator=gen))
    x[:, 0] = (size * torch.randint(0, 2, (m,), device="cuda", generator=gen).mul(2).sub(1)).bfloat16().float()
    x = x.to(TYPES[t])
    w0 = F.mx4_dequantize(w, dtype=torch.float32)[:, 0]
    z = ((x[:, :1].float() * w0) * torch.tensor(scale, device="cuda")).double()
    assert bool(z.isfinite().all())
    return x, w, targets(m, v, gen, top, low), scale, z


KINDS = [("bf16", 1.0), ("bf16", -1.3), ("fp16", 2.0 ** 8), ("fp16", 1.3 * 2.0 ** 80), ("fp32", 0.7)]


@pytest.mark.parametrize("t,scale", KINDS)
@pytest.mark.parametrize("m,v,k", FEW + TILES)
def test_the_loss_of_logits_of_any_size(t, scale, m, v, k):
    check_loss(*logits_of_any_size(t, scale, m, v, k))


@pytest.mark.parametrize("t,scale", KINDS)
@pytest.mark.parametrize("m,v,k", FEW + TILES)
def test_the_gradient_of_logits_of_any_size(t, scale, m, v, k):
    check_grad(*logits_of_any_size(t, scale, m, v, k), t)


def logits_of_thousands(t, m, v, k):
    """Hundreds and thousands that differ by some."""
    gen = generator(m * 7 + v)
    w = torch.randint(-4, 5, (v, k), device="cuda", generator=gen).float()
    w[:, 0] = 6.0
    w[v // 2, 1] = 6.0
    w = F.mx4_quantize(w)
    w64 = F.mx4_dequantize(w, dtype=torch.float32).double()
    x = torch.zeros(m, k, device="cuda")
    x[:, 0] = torch.randint(-2047, 2048, (m,), device="cuda", generator=gen).float().bfloat16().float()
    x[:, 1] = torch.randint(1, 256, (m,), device="cuda", generator=gen).float() / 32     # 20 bits in all
    x = x.to(TYPES[t])
    z = x.double()[:, :2] @ w64[:, :2].t()
    assert torch.equal(z, z.float().double())
    return x, w, targets(m, v, gen, v // 2), 1.0, z


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("m,v,k", FEW + TILES)
def test_a_loss_that_is_small_beside_its_logits_keeps_its_digits(t, m, v, k):
    x, w, ids, scale, z = logits_of_thousands(t, m, v, k)
    check_loss(x, w, ids, scale, z)
    check_grad(x, w, ids, scale, z, t)
    loss = F.mx4_cross_entropy(x, w, z.argmax(dim=1), scale=scale)[0]
    assert bool((loss >= 0).all()) and bool((loss[x[:, 1] > 4] < math.log(v)).all())


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("t,wt", [("bf16", "bf16"), ("bf16", "fp32"), ("fp16", "fp32"), ("fp32", "fp32")])
@pytest.mark.parametrize("m,v,k", [(1, 50, 40), (29, 2777, 1003)] + FEW + TILES + [(600, 9000, 1024)])   # (the last: decoded once)
def test_tokens_left_out_count_for_nothing_whatever_they_hold(t, wt, bad, m, v, k):
    gen = generator(m + k)
    w = F.mx4_quantize(torch.randn(v, k, device="cuda", generator=gen))
    x = torch.randn(m, k, device="cuda", generator=gen).to(TYPES[t])
    ids = torch.randint(0, v, (m,), device="cuda", generator=gen)
    ids[torch.rand(m, device="cuda", generator=gen) < 0.3] = -100
    ids[-1] = -1
    out = ids < 0
    results = []
    for held in (0.0, bad):
        x = torch.where(out[:, None], held, x).to(TYPES[t])
        loss, lse = F.mx4_cross_entropy(x, w, ids)
        for dloss in (torch.where(out, held, torch.rand(m, device="cuda", generator=generator(m))), torch.ones(m, device="cuda")):
            dx, dw = F.mx4_cross_entropy_grad(dloss, x, w, ids, lse, saved=F.mx8_quantize(x), weight_dtype=TYPES[wt])
            results.append((loss, torch.where(out, 0.0, lse), dx, dw))
    for got in results[2:]:
        for a, b in zip(got, results.pop(0)):
            assert bool(a.isfinite().all()) and torch.equal(a, b)
    assert bool((dx[out] == 0).all()) and bool((loss[out] == 0).all())
