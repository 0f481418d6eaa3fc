"""The operators around a model's layers as a program uses them: on other streams, in captured graphs, with outputs and
workspaces of the caller's, on sizes past 32 bits, and all together in a training step."""
import importlib.util
import math
import os

import pytest
import torch

import model_oracle as O
import paper_2410_15240_amd as F

pytestmark = pytest.mark.gpu

TOKENS, WIDTH, VOCABULARY = 300, 520, 4000


def tensors(result):
    for r in result if isinstance(result, (tuple, list)) else (result,):
        if isinstance(r, (F.MX4, F.MX8)):
            yield from (r.codes, r.scales)
        elif isinstance(r, F.NormSaved):
            yield from tensors([r.normed, r.inverse, r.block, r.block_inverse, r.gate])
        elif r is not None:
            yield r


def inputs(seed, dtype=torch.bfloat16):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    draw = lambda *s: torch.randn(*s, device="cuda", generator=gen).to(dtype)
    s = dict(x=draw(TOKENS, WIDTH), r=draw(TOKENS, WIDTH), g=draw(TOKENS, WIDTH), dy=draw(TOKENS, WIDTH), w1=draw(WIDTH), w2=draw(WIDTH))
    s["ids"] = torch.randint(-2, VOCABULARY, (TOKENS,), device="cuda", generator=gen)
    s["many"] = torch.randint(-2, 40, (20000,), device="cuda", generator=gen)
    s["dmany"] = draw(20000, 64)
    s["dloss"] = torch.rand(TOKENS, device="cuda", generator=gen)
    return s


def prepared(seed):
    s = inputs(seed)
    gen = torch.Generator(device="cuda").manual_seed(5)
    s["table"] = F.mx4_quantize(torch.randn(VOCABULARY, WIDTH, device="cuda", generator=gen) * WIDTH ** -0.5)
    s["x8"] = F.mx8_quantize(s["x"])
    _, _, s["saved"] = F.mx8_norm(s["x"], s["w2"], residual=s["r"], post_weight=s["w1"], gate=s["g"])
    _, s["lse"] = F.mx4_cross_entropy(s["x"], s["table"], s["ids"])
    return s


CALLS = {
    "embedding": lambda s, **kw: F.mx4_embedding(s["ids"], s["table"], **kw),
    "embedding-grad": lambda s, **kw: F.mx4_embedding_grad(s["dy"], s["ids"], VOCABULARY, **kw),
    "embedding-grad-many": lambda s, **kw: F.mx4_embedding_grad(s["dmany"], s["many"], 40, **kw),
    "embedding-grad-sorted": lambda s, **kw: F.mx4_embedding_grad(s["dmany"][:9000], s["many"][:9000], 40, **kw),
    "norm": lambda s, **kw: F.mx8_norm(s["x"], s["w2"], residual=s["r"], post_weight=s["w1"], gate=s["g"], scale=0.5, **kw),
    "norm-grad": lambda s, **kw: F.mx8_norm_grad(s["dy"], s["w2"], s["saved"], dhidden=s["r"], post_weight=s["w1"], **kw),
    "loss": lambda s, **kw: F.mx4_cross_entropy(s["x"], s["table"], s["ids"], **kw),
    "loss-fp32": lambda s, **kw: F.mx4_cross_entropy(s["x"].float(), s["table"], s["ids"], **kw),
    "loss-grad": lambda s, **kw: F.mx4_cross_entropy_grad(s["dloss"], s["x"], s["table"], s["ids"], s["lse"], saved=s["x8"], **kw),
}


@pytest.mark.parametrize("name", list(CALLS))
def test_memory_that_the_current_stream_still_reads_is_left_alone(name, monkeypatch):
    s, side = prepared(1), torch.cuda.Stream()
    if name == "loss-fp32":
        s["x"] = s["x"].float()   # (no cast on the current stream)
    call = CALLS[name]
    made, empty = [], torch.empty

    def counting(*a, **kw):
        t = empty(*a, **kw)
        made.append((t.data_ptr(), t.numel() * t.element_size()))
        return t

    with monkeypatch.context() as m:    # what the call allocates, its workspace among it
        m.setattr(torch, "empty", counting)
        want = [t.clone() for t in tensors(call(s))]
    sizes = [n for _, n in made]
    assert len(sizes) >= len(want)
    torch.cuda.synchronize()
    freed = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(2)]
    places = {t.data_ptr() for t in freed}
    torch.cuda._sleep(100_000_000)
    copies = [t.clone() for t in freed]     # queued behind the wait, reading memory that is free for this stream's next calls
    del freed
    made.clear()
    with monkeypatch.context() as m:
        m.setattr(torch, "empty", counting)
        result = call(s, stream=side)
    assert len(made) == len(sizes) and not places & {p for p, _ in made}
    side.synchronize()
    for got, t in zip(tensors(result), want):
        assert torch.equal(got, t)
    torch.cuda.synchronize()
    assert all(bool((c == 7).all()) for c in copies)


def test_captured_calls_replayed_on_new_inputs_between_eager_work():
    """All of them in one graph with a workspace that two of them share, replayed on other inputs between eager calls."""
    s = prepared(2)
    work = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")

    def everything():
        out = [CALLS[n](s) for n in ("embedding", "embedding-grad", "embedding-grad-many", "norm", "norm-grad")]
        loss, lse = F.mx4_cross_entropy(s["x"], s["table"], s["ids"], work=work)
        s["lse"].copy_(lse)
        out += [loss, F.mx4_cross_entropy_grad(s["dloss"], s["x"], s["table"], s["ids"], s["lse"], saved=s["x8"], work=work)]
        return [t for r in out for t in tensors(r)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        everything()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = everything()
    for seed in (3, 4, 5, 3):
        new = inputs(seed)
        for k, v in new.items():
            s[k].copy_(v)
        graph.replay()
        first = [t.clone() for t in got]
        want = [t.clone() for t in everything()]
        torch.cuda.synchronize()
        for a, b in zip(first, want):
            assert torch.equal(a, b)


def test_results_are_not_recorded_by_autograd():
    s = prepared(6)
    for k in ("x", "r", "g", "dy", "w1", "w2", "dloss"):
        s[k].requires_grad_()
    for call in CALLS.values():
        assert not any(t.requires_grad for t in tensors(call(s)))


def test_outputs_and_workspaces_of_the_callers():
    s = prepared(7)
    want = {n: [t.clone() for t in tensors(c(s))] for n, c in CALLS.items()}
    work = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    same = lambda n, r: all(torch.equal(a, b) for a, b in zip(tensors(r), want[n]))
    for n in ("embedding-grad-many", "norm-grad", "loss", "loss-grad"):
        assert same(n, CALLS[n](s, work=work))
        with pytest.raises(ValueError, match="work must be"):
            CALLS[n](s, work=work.to(torch.int8))
        with pytest.raises(F.FastrackError, match="workspace"):
            CALLS[n](s, work=work[:64])
    out = [torch.empty_like(s["x"]) for _ in range(3)]
    r = CALLS["norm"](s, out=out[0], hidden=out[1], saved=s["saved"])
    assert r[0] is out[0] and r[1] is out[1] and r[2] is s["saved"] and same("norm", r)
    s = prepared(7)
    r = CALLS["norm-grad"](s, out=out[0], out_residual=out[1], out_gate=out[2])
    assert all(a is b for a, b in zip(r, out)) and same("norm-grad", r)
    buf = torch.empty(F.MX8.nbytes(TOKENS, WIDTH), dtype=torch.uint8, device="cuda")   # kept in a message
    saved = F.NormSaved(F.MX8.view(buf, TOKENS, WIDTH), s["saved"].inverse, s["saved"].block, s["saved"].block_inverse, s["saved"].gate)
    assert same("norm", CALLS["norm"](s, saved=saved))


def test_shapes_of_more_axes_and_of_one():
    s = prepared(8)
    cut = lambda t: t.view((20, 15) + t.shape[1:])
    loss, lse = CALLS["loss"](s)
    many = F.mx4_cross_entropy(cut(s["x"]), s["table"], cut(s["ids"]))
    assert many[0].shape == (20, 15) and torch.equal(many[0].view(-1), loss) and torch.equal(many[1].view(-1), lse)
    dx, dw = CALLS["loss-grad"](s)
    dx3, dw3 = F.mx4_cross_entropy_grad(cut(s["dloss"]), cut(s["x"]), s["table"], cut(s["ids"]), cut(lse), saved=s["x8"])
    assert dx3.shape == (20, 15, WIDTH) and torch.equal(dx3.view(-1, WIDTH), dx) and torch.equal(dw3, dw)
    one = torch.ones((), device="cuda")
    a = F.mx4_cross_entropy_grad(one.expand(20, 15), cut(s["x"]), s["table"], cut(s["ids"]), cut(lse))[0]
    b = F.mx4_cross_entropy_grad(one.repeat(TOKENS), s["x"], s["table"], s["ids"], lse)[0]
    assert torch.equal(a.view(-1, WIDTH), b)
    y, h, _ = F.mx8_norm(cut(s["x"]), s["w2"], residual=cut(s["r"]), post_weight=s["w1"], gate=cut(s["g"]), scale=0.5)
    w = CALLS["norm"](s)
    assert y.shape == (20, 15, WIDTH) and torch.equal(y.view(-1, WIDTH), w[0]) and torch.equal(h.view(-1, WIDTH), w[1])
    token = F.mx4_cross_entropy(s["x"][3], s["table"], s["ids"][3])
    assert token[0].shape == () and F.mx4_embedding(s["ids"][3], s["table"]).shape == (WIDTH,)
    assert F.mx8_norm(s["x"][3], s["w2"])[0].shape == (WIDTH,)
    assert torch.equal(F.mx4_embedding_grad(cut(s["dy"]), cut(s["ids"]), VOCABULARY), CALLS["embedding-grad"](s))


REFUSED = [
    (lambda s: F.mx4_embedding(s["x"], s["table"]), "int32 or int64"),
    (lambda s: F.mx4_embedding(s["ids"].view(20, 15).t(), s["table"]), "contiguous"),
    (lambda s: F.mx4_embedding(s["ids"].cpu(), s["table"]), "CUDA tensor"),
    (lambda s: F.mx4_embedding(s["ids"], s["table"], out=s["x"][:, :-1]), "must have shape"),
    (lambda s: F.mx4_embedding(s["ids"], s["table"], dtype=torch.float64), "dtype must be"),
    (lambda s: F.mx4_embedding_grad(s["dy"], s["ids"][:-1], VOCABULARY), "rows of shape"),
    (lambda s: F.mx4_embedding_grad(s["dy"], s["ids"], -1), "negative"),
    (lambda s: F.mx4_embedding_grad(s["dy"], s["ids"], VOCABULARY, accumulate=True), "accumulate"),
    (lambda s: F.mx4_embedding_grad(s["dy"], s["ids"], VOCABULARY, out=s["x"].float()), "must have shape"),
    (lambda s: F.mx8_norm(s["x"], s["w2"][:-1]), "must have shape"),
    (lambda s: F.mx8_norm(s["x"], s["w2"], post_weight=s["w1"].float()), "post_weight must be"),
    (lambda s: F.mx8_norm(s["x"], s["w2"].half()), "weight must be"),
    (lambda s: F.mx8_norm(s["x"], s["w2"], residual=s["r"].float()), "shape and type"),
    (lambda s: F.mx8_norm(s["x"], s["w2"], gate=s["g"][:-1]), "shape and type"),
    (lambda s: F.mx8_norm(s["x"], s["w2"], saved=s["saved"]), "without what it is kept for"),
    (lambda s: F.mx8_norm(s["x"], s["w2"], post_weight=s["w1"], saved=F.mx8_norm(s["x"], s["w2"])[2]), "is missing"),
    (lambda s: F.mx8_norm(s["x"], s["w2"], saved=s["x8"]), "must be a NormSaved"),
    (lambda s: F.mx8_norm_grad(s["dy"], s["w2"], s["saved"]), "without what it is kept for"),
    (lambda s: F.mx8_norm_grad(s["dy"][:-1], s["w2"], s["saved"], post_weight=s["w1"]), "the call needs"),
    (lambda s: F.mx8_norm_grad(s["dy"], s["w2"], s["saved"], post_weight=s["w1"], residual=False, out_residual=s["x"]), "without a residual"),
    (lambda s: F.NormSaved(s["x8"], s["lse"][:-1]), "must have shape"),
    (lambda s: F.NormSaved(s["x8"], s["lse"].half()), "inverse must be"),
    (lambda s: F.NormSaved(s["x8"], s["lse"], gate=s["x8"]), "need the block"),
    (lambda s: F.mx4_cross_entropy(s["x"][:, :-1], s["table"], s["ids"]), "columns, the weights"),
    (lambda s: F.mx4_cross_entropy(s["x"], s["table"], s["ids"][:-1]), "rows of shape"),
    (lambda s: F.mx4_cross_entropy(s["x"], s["table"], s["ids"].float()), "int32 or int64"),
    (lambda s: F.mx4_cross_entropy(s["x"], F.mx4_quantize(s["x"][:0]), s["ids"]), "no classes"),
    (lambda s: F.mx4_cross_entropy_grad(s["dloss"][:-1], s["x"], s["table"], s["ids"], s["lse"]), "dloss must be"),
    (lambda s: F.mx4_cross_entropy_grad(s["dloss"].double(), s["x"], s["table"], s["ids"], s["lse"]), "dloss must be"),
    (lambda s: F.mx4_cross_entropy_grad(1.0, s["x"], s["table"], s["ids"], s["lse"]), "dloss must be"),
    (lambda s: F.mx4_cross_entropy_grad(s["dloss"], s["x"], s["table"], s["ids"], s["lse"].expand(2, TOKENS).t()[:, 0].half()), "lse must be"),
    (lambda s: F.mx4_cross_entropy_grad(s["dloss"], s["x"], s["table"], s["ids"], s["lse"], out_weight=s["x"]), "without the kept x"),
    (lambda s: F.mx4_cross_entropy_grad(s["dloss"], s["x"], s["table"], s["ids"], s["lse"], grad_input=False, out=s["x"]), "without grad_input"),
    (lambda s: F.mx4_cross_entropy_grad(s["dloss"], s["x"], s["table"], s["ids"], s["lse"], saved=s["table"]), "must be an MX8"),
    (lambda s: F.mx4_cross_entropy_grad(s["dloss"], s["x"], s["table"], s["ids"], s["lse"], saved=s["x8"], accumulate=True), "accumulate"),
    (lambda s: F.mx8_norm(s["x"], s["w2"], residual=s["r"], out=s["x"]), "overlaps"),
    (lambda s: F.mx8_norm(s["x"], s["w2"], residual=s["r"], hidden=s["r"]), "overlaps"),
    (lambda s: F.mx8_norm(s["x"], s["w2"], eps=-1.0), "eps"),
]


@pytest.mark.parametrize("i", range(len(REFUSED)))
def test_refused(i):
    call, match = REFUSED[i]
    s = prepared(9)
    with pytest.raises((ValueError, F.FastrackError), match=match):
        call(s)


# ---- sizes past 32 bits -------------------------------------------------------------------------------------------

def test_a_table_and_a_gradient_past_32_bits():
    """4.5 GB of codes, and a gradient of 2^32 values and more."""
    v, k = 2_200_000, 4096
    codes = torch.zeros(v, k // 2, dtype=torch.uint8, device="cuda")
    scales = torch.full((v, k // 32), 127, dtype=torch.uint8, device="cuda")
    ids = torch.tensor([v - 1, 0, v - 2, v - 1, 1_100_000, -1], device="cuda")
    for i, at in enumerate(ids[ids >= 0].tolist()):
        codes[at] = 0x22 + 0x11 * i
    table = F.MX4(codes, scales, k)
    y = F.mx4_embedding(ids, table)
    grid = [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    for i, c in enumerate((5, 3, 4, 5, 6)):   # (the last row was written twice)
        assert bool((y[i] == grid[c]).all())
    assert bool((y[5] == 0).all())
    x = torch.randn(3, k, device="cuda").bfloat16()
    loss, lse = F.mx4_cross_entropy(x, table, torch.tensor([v - 1, 5, 1_100_000], device="cuda"))
    rows = [0, v - 2, v - 1, 1_100_000]
    z = x.double() @ F.mx4_dequantize(F.MX4(codes[rows], scales[rows], k), dtype=torch.float32).double().t()
    want = torch.logsumexp(torch.cat((z, torch.full((3, 1), math.log(v - 4.0), dtype=torch.float64, device="cuda")), dim=1), dim=1)
    assert torch.allclose(lse.double(), want, rtol=1e-4) and torch.allclose(loss.double(), want - torch.stack((z[0, 2], z[1, 0] * 0, z[2, 3])), rtol=1e-3, atol=1e-3)
    del table, codes, scales, y
    torch.cuda.empty_cache()
    v = 1_100_000
    dy = torch.randn(6, k, device="cuda")
    ids = torch.tensor([v - 1, 0, v - 2, v - 1, 17, -1], device="cuda")
    dw = F.mx4_embedding_grad(dy, ids, v)
    assert torch.equal(dw[v - 1], dy[0] + dy[3]) and torch.equal(dw[v - 2], dy[2]) and torch.equal(dw[17], dy[4]) and torch.equal(dw[0], dy[1])
    named = torch.tensor([v - 1, 0, v - 2, 17], device="cuda")
    dw[named] = 0
    for part in dw.split(100_000):
        assert not bool(part.any())
    del dw
    torch.cuda.empty_cache()


def test_norms_of_rows_past_32_bits_and_of_more_than_one_launch():
    m, k = 540_000, 8192
    x = torch.randn(m // 1000, k, device="cuda").bfloat16().repeat(1000, 1)
    w = torch.ones(k, device="cuda", dtype=torch.bfloat16)
    y, h, saved = F.mx8_norm(x, w, post_weight=w, scale=0.5)
    first = F.mx8_norm(x[:m // 1000], w, post_weight=w, scale=0.5)
    for i in (0, 1, 499, 999):
        part = slice(i * (m // 1000), (i + 1) * (m // 1000))
        assert torch.equal(y[part], first[0]) and torch.equal(h[part], first[1]) and torch.equal(saved.normed.codes[part], first[2].normed.codes)
    dx = F.mx8_norm_grad(y, w, saved, post_weight=w, scale=0.5, residual=False)[0]
    want = F.mx8_norm_grad(first[0], w, first[2], post_weight=w, scale=0.5, residual=False)[0]
    assert torch.equal(dx[:m // 1000], want) and torch.equal(dx[-(m // 1000):], want)
    del x, y, h, saved, dx
    torch.cuda.empty_cache()
    m = (1 << 21) + 5
    x = torch.randn(m, 8, device="cuda")
    w = torch.ones(8, device="cuda")
    y = F.mx8_norm(x, w, eps=0.0)[0]
    want = x.double() / x.double().square().mean(dim=1, keepdim=True).sqrt()
    assert torch.allclose(y.double(), want, rtol=1e-5)


# ---- together -------------------------------------------------------------------------------------------------------

@pytest.fixture(scope="module")
def model():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "offloaded_model.py")
    spec = importlib.util.spec_from_file_location("offloaded_model", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("tokens,width,hidden,vocabulary,depth", [(9, 64, 96, 100, 1), (77, 200, 333, 1001, 2), (512, 512, 640, 5000, 2)])
def test_a_training_step_is_the_models_in_float32(model, tokens, width, hidden, vocabulary, depth):
    """Lookup, norms, layers and loss, and the way back, with weights and checkpoints over the encrypted link. Forwards a value is
    rounded to bf16 4 times a layer and twice at the ends, 2^-8 each at most. Backwards each 8-bit checkpoint takes
    3 parts in 100 of a normal tensor's norm at most (2^-7 of the largest of each 32 values): 5 a layer, 2 at the ends."""
    loss, want, errors, _ = model.run(tokens, width, hidden, vocabulary, depth)
    forwards = (4 * depth + 2) * 2.0 ** -8
    assert abs(loss - want) < forwards * abs(want)
    for name, e in errors.items():
        assert e < forwards + 0.03 * (5 * depth + 2), (name, e)
