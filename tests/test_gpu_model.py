"""The operators around a model's layers on the GPU against their formulas in 64 bits, at the sizes and values where they
can go wrong. How far each may be off is derived in model_oracle.py."""
import math

import pytest
import torch

import model_oracle as O
import paper_2410_15240_amd as F

pytestmark = pytest.mark.gpu

TYPES = O.TYPES


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def rows(m, k, dtype, gen, pad=0, scale=1.0):
    wide = (torch.randn(m, k + pad, device="cuda", generator=gen) * scale).to(dtype)
    return wide[:, pad // 2:pad // 2 + k]


def close(got, want, off, dtype=None, what=""):
    """got within `off` and its own type's rounding of want."""
    assert got.shape == want.shape, what
    dtype = dtype or got.dtype
    bound = off + O.half_step(dtype, want.abs() + off)
    d = (got.double() - want).abs()
    worst = (d - bound).max().item() if d.numel() else 0.0
    assert not d.numel() or bool((d <= bound).all()), "%s: over by %.3g (largest difference %.3g)" % (what, worst, d.max().item())


# ---- embedding ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("index", [torch.int32, torch.int64])
@pytest.mark.parametrize("m,v,k", [(1, 1, 1), (1, 5, 8192), (7, 300, 33), (200, 50, 64), (333, 5003, 1111)])
def test_embedding(t, index, m, v, k):
    gen = generator(m + k)
    table = F.mx4_quantize(rows(v, k, torch.float32, gen))
    ids = torch.randint(0, v, (m,), device="cuda", generator=gen).to(index)
    ids[::5] = -1 - ids[::5] % 7
    scale = float(torch.tensor(math.sqrt(k), dtype=torch.float32))
    got = F.mx4_embedding(ids, table, scale=scale, dtype=TYPES[t])
    values = F.mx4_dequantize(table, dtype=torch.float32).double()
    want = torch.where(ids[:, None] < 0, 0.0, values[ids.clamp(min=0).long()] * scale)
    close(got, want, O.U32 * want.abs(), TYPES[t])


def test_embedding_of_ids_of_any_shape_into_a_slice_and_past_the_table():
    gen = generator(3)
    table = F.mx4_quantize(rows(10, 40, torch.float32, gen))
    ids = torch.tensor([[0, 9, 10], [-1, 1 << 40, 3]], device="cuda")
    wide = torch.full((2, 3, 50), 7.0, device="cuda", dtype=torch.bfloat16)
    out = F.mx4_embedding(ids, table, out=wide[..., 4:44])
    assert out.data_ptr() == wide[..., 4:].data_ptr()
    values = F.mx4_dequantize(table)
    assert torch.equal(out[0, 0], values[0]) and torch.equal(out[0, 1], values[9]) and torch.equal(out[1, 2], values[3])
    assert bool((out[1, 0] == 0).all()) and bool(out[0, 2].isnan().all()) and bool(out[1, 1].isnan().all())
    assert bool((wide[..., :4] == 7).all()) and bool((wide[..., 44:] == 7).all())
    assert bool(F.mx4_embedding(torch.tensor([1 << 31], device="cuda"), table).isnan().all())   # (no int32 of it is a row)


SPREADS = {"any": lambda m, v, gen: torch.randint(0, v, (m,), device="cuda", generator=gen),
           "one": lambda m, v, gen: torch.full((m,), v - 1, device="cuda"),
           "few": lambda m, v, gen: torch.randint(0, min(v, 3), (m,), device="cuda", generator=gen),
           "padded": lambda m, v, gen: torch.where(torch.rand(m, device="cuda", generator=gen) < 0.5, -100,
                                                   torch.randint(0, v + v // 4 + 1, (m,), device="cuda", generator=gen)),
           "none": lambda m, v, gen: torch.full((m,), -1, device="cuda")}


@pytest.mark.parametrize("spread", list(SPREADS))
@pytest.mark.parametrize("m,v,k,t,pad", [(1, 1, 1, "fp32", 0), (31, 7, 40, "bf16", 0), (32, 300, 33, "fp16", 5),
                                         (33, 255, 64, "fp32", 0), (1001, 5003, 111, "bf16", 3), (16384, 70000, 8, "fp32", 0),
                                         (16385, 256, 16, "bf16", 0), (40000, 3000, 24, "fp16", 0), (100, 65536, 2100, "bf16", 0),
                                         (1, 25000, 600, "fp32", 0), (777, 26000, 515, "fp16", 3), (1024, 24700, 516, "bf16", 0),
                                         (1025, 24700, 520, "fp32", 0), (2048, 3000, 70, "bf16", 0)])
def test_embedding_grad(spread, m, v, k, t, pad):
    gen = generator(m + v)
    ids, dy = SPREADS[spread](m, v, gen), rows(m, k, TYPES[t], gen, pad)
    scale = 1.5
    want, off = O.embedding_grad(dy.double(), ids, v, scale)
    got = F.mx4_embedding_grad(dy, ids.to(torch.int32) if m % 2 else ids, v, scale=scale)
    assert got.dtype == torch.float32
    close(got, want, off)
    for _ in range(2):   # the same every time
        assert torch.equal(F.mx4_embedding_grad(dy, ids, v, scale=scale), got)
    if v * k < 1 << 24:
        for dtype in (torch.bfloat16, torch.float16):
            close(F.mx4_embedding_grad(dy, ids, v, scale=scale, dtype=dtype), want, off, dtype)
        base = torch.randn(v, k + 3, device="cuda", generator=gen)
        out = base.clone()
        F.mx4_embedding_grad(dy, ids, v, scale=scale, out=out[:, :k], accumulate=True)
        named = torch.zeros(v, dtype=torch.bool, device="cuda")
        named[ids[(ids >= 0) & (ids < v)]] = True
        assert torch.equal(out[~named], base[~named]) and torch.equal(out[:, k:], base[:, k:])
        close(out[:, :k], want + base[:, :k].double(), off + O.U32 * want.abs())


def test_embedding_grad_writes_its_rows_alone():
    gen = generator(9)
    wide = torch.full((60, 50), 7.0, device="cuda", dtype=torch.float16)
    dy, ids = rows(20, 41, torch.float32, gen), torch.randint(0, 60, (20,), device="cuda", generator=gen)
    F.mx4_embedding_grad(dy, ids, 60, out=wide[:, 5:46])
    want, off = O.embedding_grad(dy.double(), ids, 60, 1.0)
    close(wide[:, 5:46], want, off)
    assert bool((wide[:, :5] == 7).all()) and bool((wide[:, 46:] == 7).all())


def test_embedding_grad_against_differences():
    """The gradient of the sum of the lookup's squares, by differences of the table."""
    gen = generator(4)
    v, k, scale = 6, 5, 1.25
    table, ids = torch.randn(v, k, dtype=torch.float64, device="cuda", generator=gen), torch.tensor([0, 3, 3, -1, 5, 0, 3], device="cuda")
    f = lambda e: torch.where(ids[:, None] < 0, 0.0, scale * e[ids.clamp(min=0)])
    y = f(table).float()
    got = F.mx4_embedding_grad(2 * y, ids, v, scale=scale)
    for i in range(v):
        for j in range(k):
            step = torch.zeros_like(table)
            step[i, j] = 1e-5
            slope = (f(table + step).square().sum() - f(table - step).square().sum()) / 2e-5
            assert abs(slope.item() - got[i, j].item()) < 1e-5 * (1 + abs(slope.item()))


# ---- norm --------------------------------------------------------------------------------------------------

NORM_SIZES = [(1, 1), (1, 8192), (3, 31), (5, 1000), (9, 1111), (300, 1024), (17, 2048), (300, 1500), (300, 4000), (270, 5000), (4, 9000), (2, 33000)]
NORM_KINDS = {"plain": (False, False, False), "residual": (True, False, False), "post": (True, True, False), "gate": (True, False, True),
              "all": (True, True, True), "alone": (False, True, True)}


def optional(there, make):
    return make() if there else None


def double(t):
    return None if t is None else t.double()


def values(q):
    return None if q is None else F.mx8_dequantize(q, dtype=torch.float32).double()


@pytest.mark.parametrize("kind", list(NORM_KINDS))
@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("m,k", NORM_SIZES)
def test_norm(kind, t, m, k):
    gen, dt = generator(m + k), TYPES[t]
    res, post, gated = NORM_KINDS[kind]
    pad = 3 if m % 2 else 0
    wt = torch.float32 if m % 3 == 0 else dt
    weight = lambda: (1 + 0.2 * torch.randn(k, device="cuda", generator=gen)).to(wt)
    x = rows(m, k, dt, gen, pad, 3.0)
    r, w2, w1, g = optional(res, lambda: rows(m, k, dt, gen, pad)), weight(), optional(post, weight), optional(gated, lambda: rows(m, k, dt, gen))
    scale, eps = 1.0 if kind == "plain" else 0.75, 1e-5
    y, h, saved = F.mx8_norm(x, w2, residual=r, post_weight=w1, gate=g, scale=scale, eps=eps)
    o = O.norm(*(double(v) for v in (x, w2, r, w1, g)), scale, eps)
    close(y, o["y"], o["off_y"], what="y")
    close(saved.inverse, o["inv2"], o["off_inv2"], what="inverse")
    if kind == "plain":
        assert h is None
    else:
        close(h, o["h"], o["off_h"], what="h")

    def kept(q, want, off, what):
        # Half a step; a whole one where the largest code holds the value (127.5 steps and more become 127), and in
        # blocks whose largest value is so near a power of two that 32 bits may put it on the other side.
        _, step = O.kept(want * (1 + 1e-5))
        _, lower = O.kept(want * (1 - 1e-5))
        held = (want.abs() + off >= 127.5 * step) | (step != lower)
        assert bool(((values(q) - want).abs() <= torch.where(held, step, step / 2) + off).all()), what
    kept(saved.normed, o["u"], o["off_u"], "normed")
    if post or gated:
        kept(saved.block, o["v"], o["off_v"], "block")
    if post:
        close(saved.block_inverse, o["inv1"], O.ROW * O.U32 * o["inv1"], what="block_inverse")
    if gated:
        q = F.mx8_quantize(g)
        assert torch.equal(saved.gate.codes, q.codes) and torch.equal(saved.gate.scales, q.scales)
    assert (saved.block is not None) == (post or gated) and (saved.gate is not None) == gated

    # the gradient, from what was kept
    dy, dh = rows(m, k, dt, gen, pad), optional(res, lambda: rows(m, k, dt, gen, pad))
    dx, dr, dg, dw2, dw1 = F.mx8_norm_grad(dy, w2, saved, dhidden=dh, post_weight=w1, scale=scale, residual=res)
    o = O.norm_grad(dy.double(), w2.double(), values(saved.normed), saved.inverse.double(), double(dh), double(w1), values(saved.block),
                    double(saved.block_inverse), values(saved.gate), scale)
    for name, got in (("dx", dx), ("dr", dr), ("dg", dg), ("dw2", dw2), ("dw1", dw1)):
        if got is None:
            assert (name, "dg" in o, "dw1" in o) in (("dr", gated, post), ("dg", False, post), ("dw1", gated, False)) and (name != "dr" or not res)
        else:
            close(got, o[name], o["off_" + name], what=name)
    assert dw2.dtype == torch.float32
    again = F.mx8_norm_grad(dy, w2, saved, dhidden=dh, post_weight=w1, scale=scale, residual=res)
    assert torch.equal(again[3], dw2) and torch.equal(again[0], dx)


def test_norm_of_nothing_and_of_zeros():
    for m, k in ((0, 64), (3, 0), (0, 0)):
        x, w = torch.zeros(m, k, device="cuda"), torch.ones(k, device="cuda")
        y, h, saved = F.mx8_norm(x, w, residual=x.clone(), post_weight=w, gate=x.clone())
        dx, dr, dg, dw, dp = F.mx8_norm_grad(x, w, saved, post_weight=w)
        assert y.shape == dx.shape == dg.shape == (m, k) and bool((dw == 0).all()) and bool((dp == 0).all())
    x, w = torch.zeros(2, 70, device="cuda"), torch.ones(70, device="cuda")
    y, _, saved = F.mx8_norm(x, w, post_weight=w, eps=1e-4)
    assert bool((y == 0).all()) and torch.allclose(saved.inverse, torch.full((2,), 100.0, device="cuda"))


def test_a_row_with_a_nan_or_an_infinity_leaves_the_others_alone():
    gen = generator(6)
    x, w = rows(6, 100, torch.bfloat16, gen), torch.ones(100, device="cuda", dtype=torch.bfloat16)
    want = F.mx8_norm(x, w, post_weight=w)[0]
    bad = x.clone()
    bad[1, 50], bad[4, 3] = math.nan, math.inf
    y, _, saved = F.mx8_norm(bad, w, post_weight=w)
    others = [0, 2, 3, 5]
    assert torch.equal(y[others], want[others]) and bool(y[1].isnan().all()) and bool(y[4].isnan().any())
    dx = F.mx8_norm_grad(x, w, saved, post_weight=w)[0]
    assert bool(dx[others].isfinite().all()) and bool(dx[1].isnan().all())


def test_norm_into_slices_and_one_row_for_all():
    gen = generator(8)
    x, one = rows(40, 300, torch.float16, gen), rows(1, 300, torch.float16, gen)
    w = torch.ones(300, device="cuda", dtype=torch.float16)
    want = F.mx8_norm(x, w, residual=one.expand(40, 300).contiguous(), gate=one.expand(40, 300).contiguous())
    wide = torch.full((40, 700), 7.0, device="cuda", dtype=torch.float16)
    y, h, _ = F.mx8_norm(x, w, residual=one.expand(40, 300), gate=one.expand(40, 300), out=wide[:, 10:310], hidden=wide[:, 350:650])
    assert torch.equal(y, want[0]) and torch.equal(h, want[1])
    for a, b in ((0, 10), (310, 350), (650, 700)):
        assert bool((wide[:, a:b] == 7).all())


# ---- cross entropy -------------------------------------------------------------------------------------------

TERMS = {"bf16": 1, "fp16": 2, "fp32": 3}


def head(m, v, k, t, seed, pad=0, ignored=0.2):
    gen = generator(seed)
    w = F.mx4_quantize(rows(v, k, torch.float32, gen, scale=2 * k ** -0.5))
    x = rows(m, k, TYPES[t], gen, pad)
    ids = torch.randint(0, v, (m,), device="cuda", generator=gen)
    ids[torch.rand(m, device="cuda", generator=gen) < ignored] = -100
    return gen, x, w, F.mx4_dequantize(w, dtype=torch.float32).double(), ids


LOSS_SIZES = [(1, 1, 1), (1, 5000, 1024), (2, 777, 600), (3, 33, 40), (29, 2777, 1003), (64, 4096, 256), (300, 3000, 333),
              (700, 9000, 128), (2100, 8200, 64), (3000, 24000, 33)]


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("m,v,k", LOSS_SIZES)
def test_cross_entropy(t, m, v, k):
    _, x, w, wv, ids = head(m, v, k, t, m + v, pad=5 if m % 2 else 0)
    loss, lse = F.mx4_cross_entropy(x, w, ids.to(torch.int32) if m % 2 else ids, scale=1.25)
    o = O.loss(x.double(), wv, ids, 1.25, TERMS[t])
    close(lse, o["lse"], o["off_lse"], what="lse")
    close(loss, o["loss"], o["off_loss"], what="loss")
    assert bool((loss[ids < 0] == 0).all())


@pytest.mark.parametrize("t,wt", [("bf16", "bf16"), ("bf16", "fp32"), ("fp16", "fp16"), ("fp16", "fp32"), ("fp32", "fp32"), ("fp32", "bf16")])
@pytest.mark.parametrize("m,v,k", LOSS_SIZES)
def test_cross_entropy_grad(t, wt, m, v, k):
    gen, x, w, wv, ids = head(m, v, k, t, m + v, pad=5 if m % 2 else 0)
    x8 = F.mx8_quantize(x)
    _, lse = F.mx4_cross_entropy(x, w, ids, scale=1.25)
    dloss = torch.rand(m, device="cuda", generator=gen) + 0.5
    dx, dw = F.mx4_cross_entropy_grad(dloss, x, w, ids, lse, saved=x8, scale=1.25, weight_dtype=TYPES[wt])
    o = O.loss_grad(x.double(), wv, ids, dloss.double(), 1.25, TERMS[t], values(x8), TYPES[t], TYPES[wt])
    close(dx, o["dx"], o["off_dx"], TYPES[t], "dx")
    close(dw, o["dw"], o["off_dw"], TYPES[wt], "dw")
    assert bool((dx[ids < 0] == 0).all())
    # one of the two alone; a gradient added to what is there; one dloss for all
    assert torch.equal(F.mx4_cross_entropy_grad(dloss, x, w, ids, lse, scale=1.25)[0], F.mx4_cross_entropy_grad(dloss, x, w, ids, lse, scale=1.25)[0])
    none, alone = F.mx4_cross_entropy_grad(dloss, x, w, ids, lse, saved=x8, scale=1.25, grad_input=False, weight_dtype=TYPES[wt])
    assert none is None
    close(alone, o["dw"], o["off_dw"], TYPES[wt], "dw alone")
    if wt == "fp32":
        base = torch.randn(v, k + 2, device="cuda", generator=gen)
        out = base.clone()
        F.mx4_cross_entropy_grad(dloss, x, w, ids, lse, saved=x8, scale=1.25, out_weight=out[:, 1:k + 1], accumulate=True)
        close(out[:, 1:k + 1], o["dw"] + base[:, 1:k + 1].double(), o["off_dw"] + O.U32 * base[:, 1:k + 1].abs())
        assert torch.equal(out[:, :1], base[:, :1]) and torch.equal(out[:, k + 1:], base[:, k + 1:])
        single = F.mx4_cross_entropy_grad(dloss[:1].expand(m), x, w, ids, lse, saved=x8, scale=1.25)
        full = F.mx4_cross_entropy_grad(dloss[:1].repeat(m), x, w, ids, lse, saved=x8, scale=1.25)
        assert torch.equal(single[0], full[0]) and torch.equal(single[1], full[1])


def test_cross_entropy_over_several_pieces():
    """More logits than one piece of the vocabulary holds, the last piece a short one."""
    m, v, k = 9000, 15001, 48
    _, x, w, wv, ids = head(m, v, k, "bf16", 5)
    x8, dloss = F.mx8_quantize(x), torch.full((m,), 1.0, device="cuda")
    loss, lse = F.mx4_cross_entropy(x, w, ids)
    o = O.loss(x.double(), wv, ids, 1.0, 1)
    close(lse, o["lse"], o["off_lse"])
    close(loss, o["loss"], o["off_loss"])
    del o
    for t, wt in ((torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32)):
        o = O.loss_grad(x.double(), wv, ids, dloss.double(), 1.0, 1, values(x8), t, wt)
        dx, dw = F.mx4_cross_entropy_grad(dloss, x, w, ids, lse, saved=x8, dtype=t, weight_dtype=wt)
        close(dx, o["dx"], o["off_dx"], t)
        close(dw, o["dw"], o["off_dw"], wt)


@pytest.mark.parametrize("m", [40, 700])
def test_a_common_dloss_does_not_round_every_target_the_same_way(m):
    """With one factor for all tokens (a mean's loss) bf16 gradients are about as near as their own rounding lets them be;
    factors of their own, ignored tokens with another one, zeros and infinities go their own way."""
    gen, x, w, wv, ids = head(m, 4000, 256, "bf16", 31, ignored=0.3)
    ids[0] = -1
    x8 = F.mx8_quantize(x)
    _, lse = F.mx4_cross_entropy(x, w, ids)
    for factor in (1.0 / 3677, 0.7 * 1.0039, 0.0):   # (1.0039 is near the middle of two bf16 values)
        dloss = torch.where(ids < 0, 5.0, factor)
        o = O.loss_grad(x.double(), wv, ids, dloss.double(), 1.0, 1, values(x8), torch.bfloat16, torch.bfloat16)
        dx, dw = F.mx4_cross_entropy_grad(dloss, x, w, ids, lse, saved=x8, weight_dtype=torch.bfloat16)
        for got, name in ((dx, "dx"), (dw, "dw")):
            close(got, o[name], o["off_" + name])
            if factor:   # the rounding of the results alone is 2^-8 / sqrt(12) of a value's power of two on average
                assert ((got.double() - o[name]).norm() / o[name].norm()).item() < 1.25 * 2.0 ** -8 / 12 ** 0.5 * 2 / 1.5
    dloss = torch.rand(m, device="cuda", generator=gen)
    o = O.loss_grad(x.double(), wv, ids, dloss.double(), 1.0, 1, values(x8), torch.bfloat16, torch.bfloat16)
    dx, dw = F.mx4_cross_entropy_grad(dloss, x, w, ids, lse, saved=x8, weight_dtype=torch.bfloat16)
    close(dx, o["dx"], o["off_dx"])
    close(dw, o["dw"], o["off_dw"])
    dx = F.mx4_cross_entropy_grad(torch.full((m,), math.inf, device="cuda"), x, w, ids, lse)[0]
    assert not bool(dx[ids >= 0].isfinite().any()) and bool((dx[ids < 0] == 0).all())
    dx = F.mx4_cross_entropy_grad(torch.ones(m, device="cuda"), x, w, torch.full_like(ids, -1), lse, saved=x8)
    assert bool((dx[0] == 0).all()) and bool((dx[1] == 0).all())


def test_cross_entropy_grad_against_differences():
    gen, x, w, wv, ids = head(4, 50, 7, "fp32", 12, ignored=0.0)
    ids[2] = -1
    dloss = torch.tensor([1.0, -2.0, 5.0, 0.5], device="cuda")
    _, lse = F.mx4_cross_entropy(x, w, ids, scale=0.7)
    dx = F.mx4_cross_entropy_grad(dloss, x, w, ids, lse, scale=0.7)[0]

    def total(xd):
        return (O.loss(xd, wv, ids, 0.7, 1)["loss"] * dloss.double()).sum()
    for i in range(4):
        for j in range(7):
            step = torch.zeros(4, 7, dtype=torch.float64, device="cuda")
            step[i, j] = 1e-5
            slope = ((total(x.double() + step) - total(x.double() - step)) / 2e-5).item()
            assert abs(slope - dx[i, j].item()) < 1e-5 * (1 + abs(slope))


@pytest.mark.parametrize("m,v,k", [(1, 600, 1024), (40, 700, 64), (600, 66000, 64)])
def test_logits_far_apart_infinite_and_nan(m, v, k):
    """Large logits neither overflow nor vanish; an infinity gives what its formula gives, in its row alone; a target
    past the classes shows."""
    _, x, w, wv, ids = head(m, v, k, "bf16", 21, ignored=0.0)
    loss, lse = F.mx4_cross_entropy(x, w, ids, scale=300.0)
    o = O.loss(x.double(), wv, ids, 300.0, 1)
    close(lse, o["lse"], o["off_lse"])
    close(loss, o["loss"], o["off_loss"])
    assert bool(loss.isfinite().all()) and loss.max() > 100
    bad = ids.clone()
    bad[0] = v
    loss, lse = F.mx4_cross_entropy(x, w, bad)
    assert bool(loss[0].isnan()) and bool(loss[1:].isfinite().all())
    dx = F.mx4_cross_entropy_grad(torch.ones(m, device="cuda"), x, w, bad, lse)[0]
    assert bool(dx[0].isnan().all()) and bool(dx[1:].isfinite().all())
    y = x.clone()
    y[0, 0] = math.nan
    loss, lse = F.mx4_cross_entropy(y, w, ids)
    assert bool(loss[0].isnan()) and bool(lse[0].isnan()) and bool(loss[1:].isfinite().all())
    y[0] = 0
    y[0, 0] = math.inf
    z = (y[:1].double() @ wv.t())[0]
    z = z[~z.isnan()]
    loss, lse = F.mx4_cross_entropy(y, w, ids)
    assert bool(loss[1:].isfinite().all()) and not bool(lse[0].isfinite())


@pytest.mark.parametrize("scale", [1.0, -1.0])
@pytest.mark.parametrize("m,v,k", [(1, 5000, 1024), (3, 700, 64), (40, 300000, 64), (700, 9000, 64)])
def test_logits_that_are_all_far_from_zero(m, v, k, scale):
    """All far below it, all far above it, and some of each row -inf: what holds no class, or none but -inf, adds nothing."""
    gen = generator(m + v)
    w = F.mx4_quantize(torch.rand(v, k, device="cuda", generator=gen) + 0.5)
    x = -(torch.rand(m, k, device="cuda", generator=gen) * 20 + 20).bfloat16()
    ids = torch.randint(0, v, (m,), device="cuda", generator=gen)
    loss, lse = F.mx4_cross_entropy(x, w, ids, scale=scale)
    o = O.loss(x.double(), F.mx4_dequantize(w, dtype=torch.float32).double(), ids, scale, 1)
    assert bool((o["z"] * scale < -500).all())
    close(lse, o["lse"], o["off_lse"])
    close(loss, o["loss"], o["off_loss"])
    w.codes[: v // 2] |= 0x88    # half of the classes the other way round
    w.scales[: v // 2] = 254     # and out of range: +-inf
    lse = F.mx4_cross_entropy(-x * scale, w, ids)[1]
    half = F.MX4(w.codes[v // 2:].contiguous(), w.scales[v // 2:].contiguous(), k)
    want = F.mx4_cross_entropy(-x * scale, half, ids.clamp(max=v - v // 2 - 1))[1]
    if scale > 0:
        assert bool(lse.isfinite().all()) and torch.allclose(lse, want, rtol=1e-6)
    else:
        assert bool((lse == math.inf).all())


@pytest.mark.parametrize("m,v,k", [(40, 700, 64), (300, 9000, 64), (1200, 33000, 64)])
def test_the_gradient_where_logits_are_all_far_from_zero(m, v, k):
    """e^(z - lse) of large z and lse: each of the two, the scale and 1 / ln 2 in it are rounded (4 times 2^-24 of |z|, 2 more for
    the sums of a logit), dz once in bf16 (2^-8), and dx."""
    gen = generator(m * v)
    w = F.mx4_quantize(torch.rand(v, k, device="cuda", generator=gen) + 0.5)
    x = -(torch.rand(m, k, device="cuda", generator=gen) + 10).bfloat16()
    ids = torch.randint(0, v, (m,), device="cuda", generator=gen)
    dloss = torch.rand(m, device="cuda", generator=gen) + 0.5
    scale = 1.3
    lse = F.mx4_cross_entropy(x, w, ids, scale=scale)[1]
    dx, _ = F.mx4_cross_entropy_grad(dloss, x, w, ids, lse, scale=scale)
    w64 = F.mx4_dequantize(w, dtype=torch.float32).double()
    z = scale * x.double() @ w64.t()
    assert bool((z < -400).all())
    p = torch.exp(z - torch.logsumexp(z, 1, keepdim=True))
    hot = torch.zeros_like(p).scatter_(1, ids[:, None], 1.0)
    f = (dloss.double() * scale)[:, None]
    off = f * ((p - hot).abs() * 2.0 ** -8 + p * z.abs() * 6 * 2.0 ** -24)
    want, bound = f * (p - hot) @ w64, off @ w64.abs()
    assert bool(((dx.double() - want).abs() <= bound * (1 + 2.0 ** -8) + want.abs() * 2.0 ** -8 + 1e-12).all())


@pytest.mark.parametrize("m,v,k", [(5, 40, 64), (300, 9000, 64)])
def test_a_gradient_with_the_largest_of_scales(m, v, k):
    """Logits of zero stay zero at a scale of 3e38, though that over ln 2 is past the type: p is 1 / v."""
    gen = generator(m + v + k)
    w = F.mx4_quantize(torch.randn(v, k, device="cuda", generator=gen))
    x = torch.zeros(m, k, device="cuda", dtype=torch.bfloat16)
    ids = torch.randint(0, v, (m,), device="cuda", generator=gen)
    loss, lse = F.mx4_cross_entropy(x, w, ids, scale=3e38)
    assert torch.allclose(loss, torch.full_like(loss, math.log(v)), rtol=1e-6)
    dx, _ = F.mx4_cross_entropy_grad(torch.full_like(loss, 1e-38), x, w, ids, lse, scale=3e38)
    w64 = F.mx4_dequantize(w, dtype=torch.float32).double()
    hot = torch.zeros(m, v, device="cuda", dtype=torch.double).scatter_(1, ids[:, None], 1.0)
    dz = 3.0 * (1.0 / v - hot)
    want, bound = dz @ w64, dz.abs() @ w64.abs()
    assert bool(((dx.double() - want).abs() <= bound * (2.0 ** -8 + 2.0 ** -20) + want.abs() * 2.0 ** -8).all())


@pytest.mark.parametrize("m", [1, 300])
def test_a_gradient_of_neither(m):
    _, x, w, _, ids = head(m, 900, 64, "bf16", 3)
    loss, lse = F.mx4_cross_entropy(x, w, ids)
    assert F.mx4_cross_entropy_grad(torch.ones_like(loss), x, w, ids, lse, grad_input=False) == (None, None)
    torch.cuda.synchronize()


def test_no_tokens():
    _, x, w, _, ids = head(4, 60, 40, "bf16", 2)
    x8 = F.mx8_quantize(x[:0])
    loss, lse = F.mx4_cross_entropy(x[:0], w, ids[:0])
    assert loss.shape == lse.shape == (0,)
    dx, dw = F.mx4_cross_entropy_grad(loss, x[:0], w, ids[:0], lse, saved=x8)
    assert dx.shape == (0, 40) and dw.shape == (60, 40) and bool((dw == 0).all())
    out = torch.ones(60, 40, device="cuda")
    F.mx4_cross_entropy_grad(loss, x[:0], w, ids[:0], lse, saved=x8, out_weight=out, accumulate=True)
    assert bool((out == 1).all())
    assert F.mx4_embedding(ids[:0], w).shape == (0, 40)
    assert bool((F.mx4_embedding_grad(x[:0], ids[:0], 60) == 0).all())
