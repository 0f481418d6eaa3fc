"""Performance cases of the operators around a model's layers: the lookup of its first activations, the norms between
its blocks and the loss at its end, with their gradients, on microscaled (MX) tensors.

MX tensors hold blocks of 32 values along a row with one power-of-two scale byte s (2^(s - 127), 255 for a block that
held a NaN or an infinity), rows padded to whole blocks. MX4 stores E2M1 codes, two to a byte (16 bytes a block,
element 2i in the low four bits of byte i); MX8 stores int8 q, worth q / 64 of the scale.

`op` names the operator:
  embed       y[t] = scale E[id_t], E [v, k] in MX4; zeros for a negative id (padding)
  embed-grad  dE[i] = scale (sum of dy[t] over the t with id_t = i), [v, k] in 32 bits
  norm        b = x / rms(x) w1 (`post`; else b = x), h = r + scale g b (`gate`: with g), y = h / rms(h) w2; and what the
              gradient needs: h / rms(h), x / rms(x) (x where there is a gate and no `post`), g in MX8, 1 / rms in 32 bits
  norm-grad   the gradients of x, r, g, w2, w1 from what was kept, for the gradients dy of y and dh of h
  loss        lse_t = log sum exp of z_t, loss_t = lse_t - z_t[id_t], z = scale x E^T, E [v, k] in MX4; 0 for a negative id
  train       the same, then its gradients dx and dE = scale dz^T x^ for that of each token's loss, x^ being x in MX8
`m` counts tokens, `v` the vocabulary, `pad` is by how many elements a row of the wider tensor that an input is a
slice of exceeds it, `wtype` is dE's type.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
EPS = 1e-6
MOST = 4096 * 4096 * 65536      # multiply-adds of the largest listed product
TABLE = 4096 * 65536            # values of the largest listed table


def listed():
    return [
        # A token that a model has just answered with: the lookup that begins its next step. Latency.
        dict(name="embed-1-token", op="embed", m=1, k=8192, v=32768, type="bf16", pad=0, ignored=0.0),
        # A batch of training tokens, and the gradient of the whole table from them.
        dict(name="embed-16384-tokens", op="embed", m=16384, k=4096, v=65536, type="bf16", pad=0, ignored=0.0),
        dict(name="embed-grad-16384-tokens", op="embed-grad", m=16384, k=4096, v=65536, type="bf16", pad=0, ignored=0.0),
        # A small padded batch over a small table, nothing a multiple of anything, a slice of a wider tensor.
        dict(name="embed-grad-odd-1001", op="embed-grad", m=1001, k=1111, v=5003, type="fp16", pad=5, ignored=0.3),
        # Between two blocks, a block's own norm, a gate: one token (latency), a batch of training tokens and its gradients.
        dict(name="norm-1-token", op="norm", m=1, k=8192, type="bf16", post=True, gate=True, pad=0),
        dict(name="norm-4096x8192", op="norm", m=4096, k=8192, type="bf16", post=True, gate=True, pad=0),
        dict(name="norm-grad-4096x8192", op="norm-grad", m=4096, k=8192, type="bf16", post=True, gate=True, pad=0),
        # The plain form of most blocks, residual and norm alone, of odd sizes in 32 bits.
        dict(name="norm-grad-odd-333x1111", op="norm-grad", m=333, k=1111, type="fp32", post=False, gate=False, pad=5),
        # How likely one token was, out of a large vocabulary: latency.
        dict(name="loss-1-token", op="loss", m=1, k=4096, v=65536, type="bf16", pad=0, ignored=0.0),
        # The score of a text of odd length under a small model, its prompt left out, in 32 bits.
        dict(name="loss-odd-777", op="loss", m=777, k=1111, v=5003, type="fp32", pad=5, ignored=0.3),
        # The end of a training step: the loss of a batch and its gradients; and of a few tokens of odd sizes.
        dict(name="train-4096-tokens", op="train", m=4096, k=4096, v=65536, type="bf16", wtype="bf16", pad=0, ignored=0.1),
        dict(name="train-29-tokens-odd", op="train", m=29, k=1003, v=2777, type="fp16", wtype="fp32", pad=0, ignored=0.3),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed", "embed-grad", "embed-grad", "norm", "norm-grad", "norm-grad", "loss", "train", "train"])
    case = dict(op=op, type=rng.choice(["bf16", "bf16", "fp16", "fp32"]), pad=rng.choice([0, 0, 0, 8, 5]))
    whole = rng.random() < 0.5   # most models' widths are whole multiples of 64
    if op in ("norm", "norm-grad"):
        k = _log(rng, 32, 16384)
        k = (k + 63) // 64 * 64 if whole else k
        case.update(m=max(1, min(_log(rng, 1, 8192), 4096 * 8192 // k)), k=k, post=rng.random() < 0.5, gate=rng.random() < 0.5)
        return case
    k, v = _log(rng, 32, 8192), _log(rng, 16, 131072)
    if whole:
        k, v = (k + 63) // 64 * 64, (v + 63) // 64 * 64
    v = min(v, TABLE // k)
    if op in ("embed", "embed-grad"):
        m = min(_log(rng, 1, 32768), 16384 * 4096 // k)
    else:
        m = min(_log(rng, 1, 8192), MOST // (k * v))
    case.update(m=max(1, m), k=k, v=v, ignored=rng.choice([0.0, 0.1, 0.3]))
    if op == "train":
        case["wtype"] = rng.choice([case["type"], "fp32"])
    return case


# ---- inputs ----------------------------------------------------------------------------------------------

def _rows(m, k, pad, scale, dtype, gen):
    wide = torch.randn((m, k + pad), dtype=torch.float32, device="cuda", generator=gen).mul_(scale).to(dtype)
    return wide[:, pad // 2:pad // 2 + k]


def _activations(m, k, pad, dtype, gen):
    # Activations of a transformer: near normal, with a few channels several times larger.
    x = torch.randn((m, k + pad), dtype=torch.float32, device="cuda", generator=gen)
    loud = torch.randint(0, k + pad, (max(1, k // 500),), device="cuda", generator=gen)
    x[:, loud] *= 8.0
    return x.to(dtype)[:, pad // 2:pad // 2 + k]


def _tokens(m, v, ignored, gen):
    # Ids as in text, the i-th most frequent 1 / i as often as the first, `ignored` of them padding.
    u = torch.rand((m,), dtype=torch.float64, device="cuda", generator=gen)
    ids = torch.exp(u * math.log(v + 1.0)).long().sub_(1).clamp_(0, v - 1)
    ids = ids * 7919 % v if v % 7919 else ids   # not the low ids alone
    return torch.where(torch.rand((m,), device="cuda", generator=gen) < ignored, -100, ids)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, m, k, v, dt, pad = case["op"], case["m"], case["k"], case.get("v", 0), TYPES[case["type"]], case["pad"]
    s = dict(case=case)
    if op in ("norm", "norm-grad"):
        s["w2"] = (1 + 0.1 * torch.randn((k,), device="cuda", generator=gen)).to(dt)
        s["w1"] = (1 + 0.1 * torch.randn((k,), device="cuda", generator=gen)).to(dt) if case["post"] else None
        s["scale"] = 0.5
    if op == "norm":
        s["x"], s["r"] = _activations(m, k, pad, dt, gen), _rows(m, k, pad, 2.0, dt, gen)
        s["g"] = _rows(m, k, pad, 1.0, dt, gen) if case["gate"] else None
    elif op == "norm-grad":
        s["dy"], s["dh"] = _rows(m, k, pad, 0.1, dt, gen), _rows(m, k, pad, 0.1, dt, gen)
        s["u"] = _quantize(_rows(m, k, 0, 1.0, torch.float32, gen), 8)
        s["inv2"] = 0.3 + torch.rand((m,), device="cuda", generator=gen)
        s["v"] = _quantize(_rows(m, k, 0, 1.0, torch.float32, gen), 8) if case["post"] or case["gate"] else None
        s["inv1"] = 0.3 + torch.rand((m,), device="cuda", generator=gen) if case["post"] else None
        s["g"] = _quantize(_rows(m, k, 0, 1.0, torch.float32, gen), 8) if case["gate"] else None
    else:
        s["ids"] = _tokens(m, v, case["ignored"], gen)
        s["scale"] = math.sqrt(k) if op in ("embed", "embed-grad") else 1.5
        if op == "embed-grad":
            s["dy"] = _rows(m, k, pad, 0.1, dt, gen)
        else:
            s["codes"], s["scales"] = _quantize(_rows(v, k, 0, k ** -0.5, torch.bfloat16, gen), 4)
        if op in ("loss", "train"):
            s["x"] = _activations(m, k, pad, dt, gen)
        if op == "train":
            s["x8"] = _quantize(s["x"], 8)
            # The mean over the tokens that count; in fp16 scaled up, as training does that would lose small gradients.
            mean = 1.0 / max(1, round(m * (1 - case["ignored"])))
            s["dloss"] = torch.full((m,), 0.125 if dt == torch.float16 else mean, device="cuda")
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        import paper_2410_15240_amd as F
        if "codes" in s:
            s["mx"] = F.MX4(s["codes"], s["scales"], case["k"])
        if "x8" in s:
            s["mx8"] = F.MX8(*s["x8"], case["k"])
        if case["op"] == "norm-grad":
            mx8 = lambda q: None if q is None else F.MX8(*q, case["k"])
            s["saved"] = F.NormSaved(mx8(s["u"]), s["inv2"], mx8(s["v"]), s["inv1"], mx8(s["g"]))
    return s


# ---- the plain form ----------------------------------------------------------------------------------------

def _quantize(x, bits):
    """(codes, scales) of the rows of x: uint8 [m, 16 nb] (4 bits) or int8 [m, 32 nb], and uint8 [m, nb]."""
    m, k = x.shape
    nb = (k + 31) // 32
    v = torch.zeros((m, nb * 32), dtype=torch.float32, device=x.device)
    v[:, :k] = x
    v = v.view(m, nb, 32)
    top = v.abs().amax(dim=2)                                    # NaN where the block holds one
    bad = ~(top < math.inf)
    e = ((top.view(torch.int32) >> 23) & 255) - 127 - (2 if bits == 4 else 0)   # floor(log2), less the code's own top
    e = e.clamp(min=-127)
    scales = torch.where(bad, 255, e + 127).to(torch.uint8)
    inv = ((127 - e) << 23).view(torch.float32)                  # 2^-e: -127 <= e <= 127 (a bad block's is not used)
    v = torch.where(bad[..., None], 0.0, v * torch.where(bad | (e == 127), 2.0 ** -127, inv)[..., None])
    if bits == 8:
        return (v * 64).round().clamp(-127, 127).to(torch.int8).view(m, nb * 32), scales
    a = v.abs()
    # E2M1: 0 0.5 1 1.5 | 2 3 | 4 6, nearest with ties to the even code
    c = torch.where(a < 2, (a * 2).round(), torch.where(a < 4, a.round() + 2, ((a / 2).round() + 4).clamp(max=7)))
    c = (c.to(torch.int32) | (v.view(torch.int32) >> 28 & 8)).view(m, nb * 16, 2)
    return (c[..., 0] | c[..., 1] << 4).to(torch.uint8), scales


def _values(codes, scales, k):
    """The values [m, k] that the codes stand for, in 32 bits."""
    m, nb = scales.shape
    e = scales.to(torch.int32)
    s = torch.where(e == 0, 2.0 ** -127, (e << 23).view(torch.float32))
    s = torch.where(e == 255, math.nan, s)
    if codes.dtype == torch.uint8:
        c = torch.stack((codes & 15, codes >> 4), dim=2).view(m, nb, 32)
        grid = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
        v = torch.tensor(grid + [-g for g in grid], dtype=torch.float32, device=codes.device)[c.to(torch.int32)]
    else:
        v = codes.view(m, nb, 32).to(torch.float32) / 64
    return (v * s[..., None]).view(m, nb * 32)[:, :k]


def _kept(x):
    return _values(*_quantize(x, 8), x.shape[1]).to(torch.bfloat16)


def _norm(s, dt):
    case, x, r = s["case"], s["x"].float(), s["r"].float()
    g = s["g"].float() if case["gate"] else None
    b, inv1 = x, None
    if case["post"]:
        inv1 = 1 / torch.sqrt((x * x).mean(dim=1) + EPS)
        x = x * inv1[:, None]
        b = x * s["w1"].float()
    h = r + s["scale"] * (b if g is None else g * b)
    inv2 = 1 / torch.sqrt((h * h).mean(dim=1) + EPS)
    u = h * inv2[:, None]
    out = [(u * s["w2"].float()).to(dt), h.to(dt), _kept(u), inv2]
    if case["post"] or case["gate"]:
        out.append(_kept(x))
    if case["post"]:
        out.append(inv1)
    if case["gate"]:
        out.append(_kept(g))
    return out


def _norm_grad(s, dt):
    case, k = s["case"], s["case"]["k"]
    dy, u = s["dy"].float(), _values(*s["u"], k)
    t = dy * s["w2"].float()
    dh = s["inv2"][:, None] * (t - u * (t * u).mean(dim=1, keepdim=True)) + s["dh"].float()
    out = [None, dh.to(dt), (dy * u).sum(dim=0)]
    db = s["scale"] * dh
    v = _values(*s["v"], k) if case["post"] or case["gate"] else None
    if case["gate"]:
        out.append((db * (v * s["w1"].float() if case["post"] else v)).to(dt))
        db = db * _values(*s["g"], k)
    if case["post"]:
        out.append((db * v).sum(dim=0))
        db = db * s["w1"].float()
        db = s["inv1"][:, None] * (db - v * (db * v).mean(dim=1, keepdim=True))
    out[0] = db.to(dt)
    return out


def _loss(s, dt):
    case, k, ids = s["case"], s["case"]["k"], s["ids"]
    w, valid, at = _values(s["codes"], s["scales"], k), ids >= 0, ids.clamp(min=0)[:, None]
    z = (s["x"].float() @ w.t()).mul_(s["scale"])
    top = z.amax(dim=1, keepdim=True)
    lse = top + torch.log(torch.exp(z - top).sum(dim=1, keepdim=True))
    loss = torch.where(valid, (lse - z.gather(1, at))[:, 0], 0.0)
    if case["op"] == "loss":
        return loss, lse[:, 0]
    dz = torch.exp_(z.sub_(lse))
    dz.scatter_(1, at, dz.gather(1, at) - 1)
    dz.mul_((torch.where(valid, s["dloss"], 0.0) * s["scale"])[:, None])
    return loss, lse[:, 0], (dz @ w).to(dt), (dz.t() @ _values(*s["x8"], k)).to(TYPES[case["wtype"]])


def _plain(s):
    case = s["case"]
    op, m, k, dt = case["op"], case["m"], case["k"], TYPES[case["type"]]
    if op == "embed":
        row = s["ids"].clamp(min=0)
        v = _values(s["codes"][row], s["scales"][row], k) * s["scale"]
        return torch.where(s["ids"][:, None] < 0, 0.0, v).to(dt)
    if op == "embed-grad":
        dw = torch.zeros((case["v"], k), dtype=torch.float32, device=s["dy"].device)
        dy = torch.where(s["ids"][:, None] < 0, 0.0, s["dy"].float() * s["scale"])
        return dw.index_add_(0, s["ids"].clamp(min=0), dy)
    if op == "norm":
        return _norm(s, dt)
    if op == "norm-grad":
        return _norm_grad(s, dt)
    return _loss(s, dt)


def run(s):
    if not own:
        return _plain(s)
    import paper_2410_15240_amd as F
    case = s["case"]
    op, dt = case["op"], TYPES[case["type"]]
    if op == "embed":
        return F.mx4_embedding(s["ids"], s["mx"], scale=s["scale"], dtype=dt)
    if op == "embed-grad":
        return F.mx4_embedding_grad(s["dy"], s["ids"], case["v"], scale=s["scale"])
    if op == "norm":
        y, h, saved = F.mx8_norm(s["x"], s["w2"], residual=s["r"], post_weight=s["w1"], gate=s["g"], scale=s["scale"], eps=EPS)
        out = [y, h, F.mx8_dequantize(saved.normed), saved.inverse]
        if saved.block is not None:
            out.append(F.mx8_dequantize(saved.block))
        if saved.block_inverse is not None:
            out.append(saved.block_inverse)
        if saved.gate is not None:
            out.append(F.mx8_dequantize(saved.gate))
        return out
    if op == "norm-grad":
        dx, dr, dg, dw2, dw1 = F.mx8_norm_grad(s["dy"], s["w2"], s["saved"], dhidden=s["dh"], post_weight=s["w1"],
                                               scale=s["scale"])
        return [t for t in (dx, dr, dw2, dg, dw1) if t is not None]
    loss, lse = F.mx4_cross_entropy(s["x"], s["mx"], s["ids"], scale=s["scale"])
    if op == "loss":
        return loss, lse
    dx, dw = F.mx4_cross_entropy_grad(s["dloss"], s["x"], s["mx"], s["ids"], lse, saved=s["mx8"], scale=s["scale"],
                                      weight_dtype=TYPES[case["wtype"]])
    return loss, lse, dx, dw


# ---- the definition in 64 bits ----------------------------------------------------------------------------

def _exact_kept(x):
    """Values of 8 bits in 64, straight from the definition: the nearest point of the block's grid."""
    m, k = x.shape
    v = torch.nn.functional.pad(x, (0, -k % 32)).view(m, (k + 31) // 32, 32)
    top = v.abs().amax(dim=2, keepdim=True)
    step = torch.exp2(torch.where(top == 0, torch.full_like(top, -127.0), torch.frexp(top)[1].double() - 1).clamp(min=-127) - 6)
    return (torch.round(v / step).clamp(-127, 127) * step).view(m, -1)[:, :k].contiguous()


def _exact_values(codes, scales, k):
    s = torch.exp2(scales.double() - 127).repeat_interleave(32, dim=1)
    if codes.dtype == torch.uint8:
        c = torch.stack((codes % 16, codes // 16), dim=2).flatten(1).long()
        mag, sign = c % 8, 1.0 - 2.0 * (c // 8).double()
        v = sign * torch.where(mag < 2, mag * 0.5, (1 + 0.5 * (mag % 2)) * torch.exp2((mag // 2 - 1).double()))
    else:
        v = codes.double() * 2.0 ** -6
    return (v * s)[:, :k].contiguous()


def _exact_norm(s):
    case, x = s["case"], s["x"].double()
    out, tail, block = [], [], x
    if case["post"]:
        rms = torch.linalg.vector_norm(x, dim=1).square().div(case["k"]).add(EPS).sqrt()
        x = x / rms[:, None]
        block = x * s["w1"].double()
    if case["post"] or case["gate"]:
        tail.append(_exact_kept(x))
    if case["post"]:
        tail.append(rms.reciprocal())
    if case["gate"]:
        block = block * s["g"].double()
        tail.append(_exact_kept(s["g"].double()))
    h = torch.add(s["r"].double(), block, alpha=s["scale"])
    rms = torch.linalg.vector_norm(h, dim=1).square().div(case["k"]).add(EPS).sqrt()
    u = h / rms[:, None]
    out = [u * s["w2"].double(), h, _exact_kept(u), rms.reciprocal()]
    return out + tail


def _exact_norm_back(d, w, normed, inv):
    """The gradient of the input of a norm with weights w, and of w, for that of its output."""
    k = d.shape[1]
    t = d * w
    along = torch.linalg.vecdot(t, normed)[:, None] / k
    return (t - along * normed) * inv.double()[:, None], (d * normed).sum(dim=0)


def _exact_norm_grad(s):
    case, k = s["case"], s["case"]["k"]
    dh, dw2 = _exact_norm_back(s["dy"].double(), s["w2"].double(), _exact_values(*s["u"], k), s["inv2"])
    dh = dh + s["dh"].double()
    db, tail = dh * s["scale"], []
    v = None if s["v"] is None else _exact_values(*s["v"], k)
    if case["gate"]:
        tail.append(db * v * (s["w1"].double() if case["post"] else 1.0))
        db = db * _exact_values(*s["g"], k)
    if case["post"]:
        db, dw1 = _exact_norm_back(db, s["w1"].double(), v, s["inv1"])
        tail.append(dw1)
    return [db, dh, dw2] + tail


def exact(case, seed):
    s = _inputs(case, seed)
    op, m, k, ids = case["op"], case["m"], case["k"], s.get("ids")
    if op == "norm":
        return _exact_norm(s)
    if op == "norm-grad":
        return _exact_norm_grad(s)
    counts = (ids >= 0).double()
    if op == "embed":
        row = ids.clamp(min=0)
        return _exact_values(s["codes"][row], s["scales"][row], k) * (counts * s["scale"])[:, None]
    if op == "embed-grad":   # sums of runs of equal ids, as differences of a running sum over them
        order = torch.argsort(ids, stable=True)
        run = (s["dy"].double() * (counts * s["scale"])[:, None])[order].cumsum(dim=0)
        run = torch.cat((torch.zeros_like(run[:1]), run))
        edge = torch.searchsorted(ids[order].contiguous(), torch.arange(case["v"] + 1, device=ids.device))
        return run[edge[1:]] - run[edge[:-1]]
    w, at = _exact_values(s["codes"], s["scales"], k), ids.clamp(min=0)
    z = torch.matmul(s["x"].double() * s["scale"], w.t().contiguous())
    lse = torch.logsumexp(z, dim=1)
    loss = (lse - z[torch.arange(m, device=z.device), at]) * counts
    if op == "loss":
        return loss, lse
    p = torch.softmax(z, dim=1)
    del z
    p[torch.arange(m, device=p.device), at] -= 1
    p *= (counts * s["dloss"].double() * s["scale"])[:, None]
    return loss, lse, torch.matmul(p, w), torch.matmul(p.t().contiguous(), _exact_values(*s["x8"], k))


def work(case):
    """Every input read once and every output written once; 2 flops to a multiply-add."""
    op, m, k, v, b = case["op"], case["m"], case["k"], case.get("v", 0), SIZE[case["type"]]
    nb = (k + 31) // 32
    if op == "embed":        # ids, the rows looked up, the values
        return {"bytes": m * (8 + nb * 17 + k * b), "flops": 0}
    if op == "embed-grad":
        return {"bytes": m * (8 + k * b) + v * k * 4, "flops": 0}
    if op == "norm":         # x, r, g in, y and h out; kept in 8 bits, and their values
        kept = 1 + (case["post"] or case["gate"]) + case["gate"]
        return {"bytes": m * k * b * (4 + case["gate"]) + m * kept * (2 * nb * 33 + k * 2), "flops": 0}
    if op == "norm-grad":    # dy, dh and what was kept in, dx, dr and dg out
        kept = 1 + (case["post"] or case["gate"]) + case["gate"]
        return {"bytes": m * k * b * (4 + case["gate"]) + m * kept * nb * 33, "flops": 0}
    if op == "loss":
        return {"bytes": v * nb * 17 + m * k * b, "flops": 2 * m * k * v}
    return {"bytes": v * nb * 17 + m * (2 * k * b + nb * 33) + v * k * SIZE[case["wtype"]], "flops": 6 * m * k * v}
