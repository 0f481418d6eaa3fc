"""The operators around a model's layers on the GPU at the shapes that take their rarer ways."""
import pytest
import torch

import model_oracle as O
import paper_2410_15240_amd as F
import test_gpu_model as T
from test_gpu_model import close, generator, rows

pytestmark = pytest.mark.gpu

TYPES = O.TYPES


# ---- norm --------------------------------------------------------------------------------------------------

def test_the_gradients_of_weights_of_more_columns_than_one_launch_sums():
    """No rows, so that the sums are all that there is to do: zeros, for 2^28 columns and more."""
    k = (1 << 28) + 70
    used = torch.ones(2 * k, device="cuda")     # (what the gradients are written over)
    del used
    w, post = torch.ones(2, k, device="cuda", dtype=torch.bfloat16)
    x = torch.empty(0, k, device="cuda", dtype=torch.bfloat16)
    _, _, saved = F.mx8_norm(x, w, post_weight=post)
    _, _, _, dw, dpost = F.mx8_norm_grad(x, w, saved, post_weight=post)
    assert dw.shape == dpost.shape == (k,) and not bool(dw.any()) and not bool(dpost.any())
    del w, post, dw, dpost
    torch.cuda.empty_cache()


@pytest.mark.parametrize("kind", list(T.NORM_KINDS))
@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("m,k", [(2500, 40), (2501, 1000), (2500, 2000), (1101, 4000), (600, 5000), (600, 8192), (601, 9000), (600, 33000)])
def test_more_rows_than_groups_take(kind, t, m, k):
    """Groups of the gradient that take two rows and three, in each of its ways; forwards 4 units a thread (from 4097 columns)."""
    T.test_norm(kind, t, m, k)


@pytest.mark.parametrize("m,k", [(40, 300), (1500, 1000), (300, 9000), (300, 17000)])
def test_gradients_into_slices(m, k):
    gen = generator(m + k)
    x, r, g, dy, dh = (rows(m, k, torch.bfloat16, gen) for _ in range(5))
    w2, w1 = (rows(1, k, torch.bfloat16, gen)[0] for _ in range(2))
    _, _, saved = F.mx8_norm(x, w2, residual=r, post_weight=w1, gate=g)
    want = F.mx8_norm_grad(dy, w2, saved, dhidden=dh, post_weight=w1)
    wide = torch.full((m, 3 * k + 40), 7.0, device="cuda", dtype=torch.bfloat16)
    parts = [wide[:, 5 + i * (k + 11):][:, :k] for i in range(3)]
    got = F.mx8_norm_grad(dy, w2, saved, dhidden=dh, post_weight=w1, out=parts[0], out_residual=parts[1], out_gate=parts[2])
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    untouched = torch.ones_like(wide, dtype=torch.bool)
    for i in range(3):
        untouched[:, 5 + i * (k + 11):][:, :k] = False
    assert bool((wide[untouched] == 7).all())


# ---- the table's gradient ------------------------------------------------------------------------------------

def table_grad(m, v, k, out, gen, dtype=torch.float32):
    """A gradient written into `out` and the rows that its ids name, checked there."""
    ids, dy = torch.randint(-1, v, (m,), device="cuda", generator=gen), rows(m, k, dtype, gen)
    ids[:4] = torch.tensor([v - 1, 0, v - 1, v], device="cuda")
    F.mx4_embedding_grad(dy, ids, v, scale=0.75, out=out)
    if v * k < 1 << 26:
        close(out, *O.embedding_grad(dy.double(), ids, v, 0.75))
        return
    named, at = torch.unique(ids[(ids >= 0) & (ids < v)], return_inverse=True)
    good = (ids >= 0) & (ids < v)
    close(out[named], *O.embedding_grad(dy[good].double(), at, len(named), 0.75))
    out[named] = 0
    assert not any(bool(p.any()) for p in out.split(1 << 24))


# By many tokens for each row, sorted by one workgroup and by many; few tokens of a large table.
@pytest.mark.parametrize("m,v,k", [(3000, 300, 41), (20000, 777, 33), (40, 30000, 35), (900, 26000, 515), (9, 25000, 600)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("at", [0, 1, 3, 7, 8])
def test_a_tables_gradient_at_any_alignment_and_into_a_slice(m, v, k, dtype, at):
    gen = generator(m + v + at)
    flat = torch.full((v * k + 40,), 7.0, device="cuda", dtype=dtype)
    table_grad(m, v, k, flat[at:at + v * k].view(v, k), gen)
    assert bool((flat[:at] == 7).all()) and bool((flat[at + v * k:] == 7).all())
    wide = torch.full((v, k + 9 + at), 7.0, device="cuda", dtype=dtype)
    table_grad(m, v, k, wide[:, at:at + k], gen)
    assert bool((wide[:, :at] == 7).all()) and bool((wide[:, at + k:] == 7).all())


@pytest.mark.parametrize("m", [2500, 16384, 16385, 50000])
@pytest.mark.parametrize("v,k", [((1 << 18) + 5, 9), (1 << 20, 4), ((1 << 27) + 3, 1)])
def test_a_table_whose_ids_are_sorted_in_three_passes_and_four(m, v, k):
    gen = generator(m + k)
    out = torch.full((v, k), 7.0, device="cuda")
    table_grad(m, v, k, out, gen)
    ids = torch.randint(0, 50, (m,), device="cuda", generator=gen) * ((v - 1) // 49)     # many of each, over the whole range
    dy = rows(m, k, torch.bfloat16, gen)
    got = F.mx4_embedding_grad(dy, ids, v)
    named = torch.arange(50, device="cuda") * ((v - 1) // 49)
    close(got[named], *O.embedding_grad(dy.double(), ids // ((v - 1) // 49), 50, 1.0))
    assert torch.equal(F.mx4_embedding_grad(dy, ids, v), got)


# ---- cross entropy -------------------------------------------------------------------------------------------

@pytest.mark.parametrize("t,wt", [("bf16", "bf16"), ("bf16", "fp32"), ("fp16", "fp16"), ("fp32", "fp32")])
@pytest.mark.parametrize("m,v,k", [(3, 700, 64), (29, 2777, 1003), (300, 3000, 333), (600, 9000, 64), (9000, 15001, 41)])
def test_loss_gradients_into_slices_of_a_dloss_that_lies_apart_and_one_at_a_time(t, wt, m, v, k):
    gen, x, w, wv, ids = T.head(m, v, k, t, m + v)
    x8 = F.mx8_quantize(x)
    _, lse = F.mx4_cross_entropy(x, w, ids)
    apart = torch.rand(m, 5, device="cuda", generator=gen) + 0.5
    dloss = apart[:, 2]
    o = O.loss_grad(x.double(), wv, ids, dloss.double(), 1.0, T.TERMS[t], T.values(x8), TYPES[t], TYPES[wt])
    wide = torch.full((m, k + 11), 7.0, device="cuda", dtype=TYPES[t])
    head = torch.full((v, k + 7), 7.0, device="cuda", dtype=TYPES[wt])
    dx, dw = F.mx4_cross_entropy_grad(dloss, x, w, ids, lse, saved=x8, out=wide[:, 3:k + 3], out_weight=head[:, 1:k + 1])
    close(dx, o["dx"], o["off_dx"], TYPES[t], "dx")
    close(dw, o["dw"], o["off_dw"], TYPES[wt], "dw")
    for rest in (wide[:, :3], wide[:, k + 3:], head[:, :1], head[:, k + 1:]):
        assert bool((rest == 7).all())
    again = F.mx4_cross_entropy_grad(dloss.contiguous(), x, w, ids, lse, saved=x8, weight_dtype=TYPES[wt])
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)
    # The one without the other has its own terms, workspace and plan.
    alone, none = F.mx4_cross_entropy_grad(dloss, x, w, ids, lse)
    assert none is None
    close(alone, o["dx"], o["off_dx"], TYPES[t], "dx alone")


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("m,v,k", [(1, 600, 1024), (3, 20000, 64), (40, 700, 64), (600, 9000, 64), (2100, 9000, 300)])
def test_an_infinite_value_gives_what_its_formula_gives(t, m, v, k):
    """Logits of its row are infinities by their weight's sign, and NaN where that is 0; the other rows are as they were."""
    gen = generator(m + v)
    x = rows(m, k, TYPES[t], gen)
    ids = torch.randint(1, v, (m,), device="cuda", generator=gen)
    for signs in ("plus", "minus", "both", "zero"):
        w = torch.randint(1, 4, (v, k), device="cuda", generator=gen).float()
        w[:, 1] = 6.0
        if signs == "minus":
            w[:, 0].neg_()
        elif signs == "both":
            w[1::2, 0].neg_()
        elif signs == "zero":
            w[v // 2, 0] = 0.0
        w = F.mx4_quantize(w)
        want = F.mx4_cross_entropy(x, w, ids)
        y = x.clone()
        y[0] = 0.0
        y[0, 0] = float("inf")
        z = y[:1].float().double() @ F.mx4_dequantize(w, dtype=torch.float32).double().t()
        loss, lse = F.mx4_cross_entropy(y, w, ids)
        lse0 = torch.logsumexp(z, dim=1)
        assert bool(lse0.isnan().any()) == (signs == "zero") and torch.allclose(lse[:1].double(), lse0, equal_nan=True)
        assert torch.allclose(loss[:1].double(), lse0 - z[:, ids[0]], equal_nan=True)
        assert torch.equal(loss[1:], want[0][1:]) and torch.equal(lse[1:], want[1][1:])
