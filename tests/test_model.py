"""The operators around a model's layers without a GPU: the oracle against itself, workspaces, and what the C entries and the
binding refuse."""
import math

import pytest
import torch

import model_oracle as O
import paper_2410_15240_amd as F

# Aligned "device" addresses 16 MB apart, never dereferenced here.
AT = [0x1000000 * (i + 1) for i in range(24)]
BF16, FP16, FP32 = range(3)


@pytest.fixture(scope="module")
def L():
    import os
    if not os.path.exists(F.library_path()):
        from paper_2410_15240_amd import build
        build.build()
    return F.lib()


# ---- the oracle ----------------------------------------------------------------------------------------------

def test_the_oracles_gradients_are_autograds():
    gen = torch.Generator().manual_seed(1)
    draw = lambda *s: torch.randn(*s, dtype=torch.float64, generator=gen)
    m, k = 5, 37
    x, r, g = (draw(m, k).requires_grad_() for _ in range(3))
    w1, w2 = (draw(k).requires_grad_() for _ in range(2))
    dy, dh = draw(m, k), draw(m, k)
    o = O.norm(x, w2, r, w1, g, 0.7, 1e-3)
    want = torch.autograd.grad((o["y"] * dy).sum() + (o["h"] * dh).sum(), (x, r, g, w2, w1))
    d = lambda t: t.detach()
    b = O.norm_grad(dy, d(w2), d(o["u"]), d(o["inv2"]), dh, d(w1), d(o["v"]), d(o["inv1"]), d(g), 0.7)
    for name, t in zip(("dx", "dr", "dg", "dw2", "dw1"), want):
        assert torch.allclose(b[name], t, rtol=1e-10, atol=1e-10), name
    o = O.norm(x, w2, None, None, g, 0.7, 1e-3)
    want = torch.autograd.grad((o["y"] * dy).sum(), (x, g, w2))
    b = O.norm_grad(dy, d(w2), d(o["u"]), d(o["inv2"]), None, None, d(x), None, d(g), 0.7)
    for name, t in zip(("dx", "dg", "dw2"), want):
        assert torch.allclose(b[name], t, rtol=1e-10, atol=1e-10), name
    w, x = draw(20, k).requires_grad_(), draw(m, k).requires_grad_()
    ids, dloss = torch.tensor([3, -1, 19, 0, 3]), draw(m)
    f = O.loss(x, w, ids, 1.3, 1)
    nn = torch.nn.functional.cross_entropy(1.3 * x @ w.t(), ids, ignore_index=-1, reduction="none")
    assert torch.allclose(f["loss"], nn)
    want = torch.autograd.grad((nn * dloss).sum(), (x, w))
    b = O.loss_grad(d(x), d(w), ids, dloss, 1.3, 1, d(x), torch.float32, torch.float32)
    assert torch.allclose(b["dx"], want[0]) and torch.allclose(b["dw"], want[1])


def test_the_oracles_8_bits():
    import mx_oracle
    x = torch.randn(4, 70, dtype=torch.float64) * torch.exp2(torch.arange(4.0, dtype=torch.float64))[:, None]
    want = mx_oracle.values(*mx_oracle.quantize(x.numpy(), 8), 70)
    got, step = O.kept(x)
    assert (got.numpy() == want).all() and bool(((got - x).abs() <= step).all())


# ---- workspaces ------------------------------------------------------------------------------------------------

def test_workspaces(L):
    assert L.fastrack_mx_norm_grad_work_bytes(1, 100, 0) == 400 and L.fastrack_mx_norm_grad_work_bytes(1, 100, 1) == 800
    assert L.fastrack_mx_norm_grad_work_bytes(0, 100, 1) == 0
    assert L.fastrack_mx_norm_grad_work_bytes(1 << 30, 8192, 1) <= 2 * 4 * 8192 * 8192
    assert L.fastrack_mx_embedding_grad_work_bytes(0, 10, 10) == 0
    assert L.fastrack_mx_embedding_grad_work_bytes(20, 10, 10) == 0
    assert L.fastrack_mx_embedding_grad_work_bytes(3000, 10, 10) == 2 * 12000 + 188 * 2 * 16 * 4
    assert L.fastrack_mx_embedding_grad_work_bytes(1 << 31, 10, 10) == 0
    assert L.fastrack_mx_loss_work_bytes(BF16, AT[0], 4096, 0, 1000, 4096) == 0
    # The logits of a large batch are never all there.
    for m in (4096, 100000):
        whole = m * 131072 * 4
        assert L.fastrack_mx_loss_work_bytes(BF16, AT[0], 4096, m, 131072, 4096) < whole / 3
        assert L.fastrack_mx_loss_grad_work_bytes(BF16, AT[0], 4096, m, 131072, 4096, 1, BF16, 1, BF16) < whole / 3 + m * 4096 * 4
    assert (L.fastrack_mx_loss_grad_work_bytes(BF16, AT[0], 4096, 4096, 131072, 4096, 1, BF16, 0, BF16)
            <= L.fastrack_mx_loss_grad_work_bytes(BF16, AT[0], 4096, 4096, 131072, 4096, 1, BF16, 1, FP32))


# ---- the C entries -----------------------------------------------------------------------------------------------

def refused(L, rc):
    return rc == -1 and L.fastrack_last_error()


def norm(L, type=BF16, x=AT[0], ldx=64, r=AT[1], ldr=64, g=AT[2], ldg=64, rows=4, cols=64, wtype=BF16, w=AT[3], w1=AT[4], scale=1.0,
         eps=1e-6, y=AT[5], ldy=64, h=AT[6], ldh=64, uc=AT[7], us=AT[8], inv=AT[9], vc=AT[10], vs=AT[11], inv1=AT[12], gc=AT[13],
         gs=AT[14]):
    return L.fastrack_mx_norm(type, x, ldx, r, ldr, g, ldg, rows, cols, wtype, w, w1, scale, eps, y, ldy, h, ldh, uc, us, inv, vc, vs,
                              inv1, gc, gs, None)


@pytest.mark.parametrize("kw", [dict(type=3), dict(wtype=FP16), dict(wtype=7), dict(rows=1 << 31), dict(cols=1 << 31), dict(eps=-1.0),
                                dict(eps=math.nan), dict(eps=math.inf), dict(scale=math.nan), dict(x=None), dict(x=AT[0] + 1),
                                dict(r=AT[1] + 1), dict(w=None), dict(w=AT[3] + 1), dict(w1=AT[4] + 1), dict(y=None), dict(ldy=63),
                                dict(ldh=63), dict(ldx=1 << 41), dict(uc=None), dict(us=None), dict(uc=AT[7] + 8), dict(inv=None),
                                dict(inv=AT[9] + 2), dict(vc=None), dict(vs=None), dict(inv1=None), dict(gc=None), dict(gs=None),
                                dict(w1=None, vc=None), dict(y=AT[0]), dict(h=AT[1] + 16), dict(y=AT[6]), dict(uc=AT[0]), dict(inv=AT[3]),
                                dict(inv1=AT[9] + 12), dict(gc=AT[10])])
def test_norm_refuses(L, kw):
    assert refused(L, norm(L, **kw))


def norm_grad(L, type=BF16, dy=AT[0], ld=64, dh=AT[1], ldh=64, rows=4, cols=64, wtype=BF16, w=AT[2], w1=AT[3], scale=1.0, uc=AT[4],
              us=AT[5], inv=AT[6], vc=AT[7], vs=AT[8], inv1=AT[9], gc=AT[10], gs=AT[11], dx=AT[12], ldx=64, dr=AT[13], ldr=64, dg=AT[14],
              ldg=64, dw=AT[15], dw1=AT[16], work=AT[17], size=1 << 20):
    return L.fastrack_mx_norm_grad(type, dy, ld, dh, ldh, rows, cols, wtype, w, w1, scale, uc, us, inv, vc, vs, inv1, gc, gs, dx, ldx, dr,
                                   ldr, dg, ldg, dw, dw1, work, size, None)


@pytest.mark.parametrize("kw", [dict(type=3), dict(wtype=FP16), dict(rows=1 << 31), dict(scale=math.nan), dict(dy=None), dict(dy=AT[0] + 1),
                                dict(w=None), dict(w1=AT[3] + 1), dict(uc=None), dict(us=None), dict(inv=None), dict(vc=None), dict(inv1=None),
                                dict(gs=None), dict(dx=None), dict(ldx=63), dict(ldr=60), dict(dg=None), dict(ldg=3), dict(dw=None),
                                dict(dw=AT[15] + 2), dict(dw1=None), dict(work=None), dict(work=AT[17] + 8), dict(size=2047), dict(dx=AT[0]),
                                dict(dr=AT[12]), dict(dg=AT[4]), dict(dw=AT[2]), dict(dw1=AT[15] + 4), dict(work=AT[16]), dict(work=AT[6])])
def test_norm_grad_refuses(L, kw):
    assert refused(L, norm_grad(L, **kw))


def embedding(L, itype=1, ids=AT[0], m=4, codes=AT[1], scales=AT[2], rows=10, cols=64, scale=1.0, type=BF16, y=AT[3], ldy=64):
    return L.fastrack_mx_embedding(itype, ids, m, codes, scales, rows, cols, scale, type, y, ldy, None)


@pytest.mark.parametrize("kw", [dict(itype=2), dict(ids=None), dict(ids=AT[0] + 4), dict(itype=0, ids=AT[0] + 2), dict(m=1 << 31),
                                dict(rows=1 << 31), dict(cols=1 << 31), dict(codes=None), dict(codes=AT[1] + 8), dict(scales=None),
                                dict(type=3), dict(y=None), dict(y=AT[3] + 1), dict(ldy=63), dict(y=AT[0]), dict(y=AT[1] + 16), dict(y=AT[2])])
def test_embedding_refuses(L, kw):
    assert refused(L, embedding(L, **kw))


def embedding_grad(L, itype=1, ids=AT[0], type=BF16, dy=AT[1], ld=64, m=3000, rows=10, cols=64, scale=1.0, otype=FP32, dw=AT[2], ldw=64, acc=0,
                   work=AT[3], size=1 << 20):
    return L.fastrack_mx_embedding_grad(itype, ids, type, dy, ld, m, rows, cols, scale, otype, dw, ldw, acc, work, size, None)


@pytest.mark.parametrize("kw", [dict(itype=2), dict(ids=None), dict(ids=AT[0] + 4), dict(type=3), dict(otype=3), dict(dy=None),
                                dict(dy=AT[1] + 1), dict(m=1 << 31), dict(rows=1 << 31), dict(dw=None), dict(ldw=63), dict(acc=2),
                                dict(acc=1, otype=BF16), dict(work=None), dict(work=AT[3] + 8), dict(size=12031), dict(dw=AT[1]), dict(dw=AT[0]),
                                dict(work=AT[2] + 16), dict(m=(1 << 29), cols=2049, ldw=2049, ld=0, size=1 << 62)])
def test_embedding_grad_refuses(L, kw):
    assert refused(L, embedding_grad(L, **kw))


def loss(L, type=BF16, x=AT[0], ldx=64, codes=AT[1], scales=AT[2], itype=1, ids=AT[3], m=4, n=100, k=64, scale=1.0, out=AT[4], lse=AT[5],
         work=AT[6], size=1 << 20):
    return L.fastrack_mx_loss(type, x, ldx, codes, scales, itype, ids, m, n, k, scale, out, lse, work, size, None)


@pytest.mark.parametrize("kw", [dict(type=3), dict(x=None), dict(x=AT[0] + 1), dict(codes=None), dict(codes=AT[1] + 8), dict(scales=None),
                                dict(itype=2), dict(ids=None), dict(ids=AT[3] + 4), dict(m=1 << 22), dict(n=1 << 31), dict(n=0),
                                dict(out=None), dict(lse=None), dict(lse=AT[5] + 2), dict(work=None), dict(size=100), dict(work=AT[6] + 8),
                                dict(out=AT[5] + 8), dict(out=AT[0]), dict(lse=AT[3]), dict(work=AT[1]), dict(n=1 << 30, k=1 << 10)])
def test_loss_refuses(L, kw):
    assert refused(L, loss(L, **kw))


def loss_grad(L, type=BF16, x=AT[0], ldx=64, codes=AT[1], scales=AT[2], xc=AT[3], xs=AT[4], itype=1, ids=AT[5], dloss=AT[6], step=1,
              lse=AT[7], m=4, n=100, k=64, scale=1.0, xt=BF16, dx=AT[8], ldd=64, wt=FP32, dw=AT[9], ldw=64, acc=0, work=AT[10], size=1 << 24):
    return L.fastrack_mx_loss_grad(type, x, ldx, codes, scales, xc, xs, itype, ids, dloss, step, lse, m, n, k, scale, xt, dx, ldd, wt, dw,
                                   ldw, acc, work, size, None)


@pytest.mark.parametrize("kw", [dict(type=3), dict(x=None), dict(codes=None), dict(xc=None), dict(xs=None), dict(xc=AT[3] + 8), dict(itype=2),
                                dict(ids=None), dict(dloss=None), dict(dloss=AT[6] + 2), dict(step=1 << 41), dict(lse=None), dict(m=1 << 22),
                                dict(n=0), dict(xt=3), dict(wt=3), dict(ldd=63), dict(ldw=63), dict(acc=2), dict(acc=1, wt=BF16),
                                dict(work=None), dict(size=100), dict(dx=AT[0]), dict(dw=AT[8]), dict(dw=AT[1]), dict(dx=AT[7]),
                                dict(work=AT[6]), dict(dw=AT[3]), dict(dx=AT[6] + 12 * 8, step=8), dict(n=1 << 30, k=1 << 10)])
def test_loss_grad_refuses(L, kw):
    assert refused(L, loss_grad(L, **kw))


# ---- the binding ---------------------------------------------------------------------------------------------------

def host(cls, rows=4, cols=64):
    return cls.view(torch.zeros(cls.nbytes(rows, cols), dtype=torch.uint8), rows, cols)


X, IDS = torch.zeros(4, 64), torch.zeros(4, dtype=torch.int64)


@pytest.mark.parametrize("call,match", [
    (lambda: F.mx4_embedding(IDS, host(F.MX4)), "CUDA tensor"),
    (lambda: F.mx4_embedding(IDS, X), "must be an MX4"),
    (lambda: F.mx4_embedding(IDS, host(F.MX8)), "must be an MX4"),
    (lambda: F.mx4_embedding_grad(X, IDS, 10), "CUDA tensor"),
    (lambda: F.mx4_embedding_grad([1.0], IDS, 10), "torch tensor"),
    (lambda: F.mx8_norm(X, X[0]), "CUDA tensor"),
    (lambda: F.mx8_norm(X.double(), X[0]), "bfloat16, float16 or float32"),
    (lambda: F.mx8_norm_grad(X, X[0], None), "CUDA tensor"),
    (lambda: F.NormSaved(host(F.MX8), X[:, 0]), "CUDA tensor"),
    (lambda: F.NormSaved(host(F.MX4), X[:, 0]), "must be an MX8"),
    (lambda: F.mx4_cross_entropy(X, host(F.MX4), IDS), "CUDA tensor"),
    (lambda: F.mx4_cross_entropy(X, host(F.MX8), IDS), "must be an MX4"),
    (lambda: F.mx4_cross_entropy_grad(X[:, 0], X, host(F.MX4), IDS, X[:, 0]), "CUDA tensor"),
])
def test_binding_refuses(call, match):
    with pytest.raises(ValueError, match=match):
        call()
