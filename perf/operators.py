"""Performance cases of the microscaled (MX) operators: quantisation, the linear layer with 4-bit weights in
both directions, and the backward pass from 8-bit activation checkpoints.

MX tensors hold blocks of 32 values along a row with one power-of-two scale byte s (2^(s - 127), 255 for a
block that held a NaN or an infinity), rows padded to whole blocks. MX4 stores E2M1 codes, two to a byte (16 bytes
a block, element 2i in the low four bits of byte i); MX8 stores int8 q, worth q / 64 of the scale.

`op` names the operator:
  quantize     x -> MX -> the values that the codes stand for, in x's type
  linear       y = x W^T, W [n, k] in MX4, x [m, k] in 16 or 32 bits
  mx-linear    the same with x in MX4 too
  grad-input   dx = dy W, W [n, k] in MX4
  act          y = f(x) * gate with x and gate kept as MX8, then their gradients from what was kept
  weight-grad  dW = dy^T x, x [m, k] kept as MX8, dW in 32 bits
`m` counts tokens, `pad` is by how many elements a row of the wider tensor that an input is a slice of exceeds it.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
MAX_WORK = 4096 * 8192 * 8192   # multiply-adds of the largest listed product


def listed():
    return [
        # The benchmark's 1 GiB of bf16 weights as one matrix: quantised before it is encrypted and sent.
        dict(name="quantize4-weights-1GiB", op="quantize", bits=4, m=16384, k=32768, type="bf16", pad=0),
        # A small activation of odd size, kept in 8 bits.
        dict(name="quantize8-odd-1001x1111", op="quantize", bits=8, m=1001, k=1111, type="fp32", pad=0),
        # One token through a layer of 2^26 weights (the benchmark's gradient buffer has as many values): latency.
        dict(name="linear-1-token", op="linear", m=1, k=8192, n=8192, type="bf16", pad=0),
        # A few tokens of several requests, sizes that divide nothing, a slice of a wider tensor.
        dict(name="linear-29-tokens-odd", op="linear", m=29, k=5003, n=2777, type="fp16", pad=5),
        # A batch of training tokens or a prompt: the largest products.
        dict(name="linear-4096-tokens", op="linear", m=4096, k=8192, n=8192, type="bf16", pad=0),
        dict(name="mx-linear-4096-tokens", op="mx-linear", m=4096, k=8192, n=8192, type="bf16", pad=0),
        # The gradient that goes back through the layer, and a small odd one in 32 bits.
        dict(name="grad-input-4096-tokens", op="grad-input", m=4096, k=8192, n=8192, type="bf16", pad=0),
        dict(name="grad-input-77-tokens-odd", op="grad-input", m=77, k=1111, n=1000, type="fp32", pad=0),
        # A gated activation between two layers, forwards and backwards; a small plain one.
        dict(name="act-silu-gated-4096x16384", op="act", m=4096, k=16384, act="silu", gate=True, type="bf16", pad=0),
        dict(name="act-gelu-odd-333x1000", op="act", m=333, k=1000, act="gelu", gate=False, type="fp32", pad=0),
        # The benchmark's 256 MiB of fp32 gradients, from a batch of training tokens; and a small odd layer over
        # many tokens, whose few outputs have a long sum.
        dict(name="weight-grad-4096-tokens", op="weight-grad", m=4096, k=8192, n=8192, type="bf16", pad=0),
        dict(name="weight-grad-6001-tokens-odd", op="weight-grad", m=6001, k=1111, n=500, type="fp16", pad=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantize", "linear", "linear", "mx-linear", "grad-input", "act", "weight-grad", "weight-grad"])
    case = dict(op=op, type=rng.choice(["bf16", "bf16", "fp16", "fp32"]), pad=rng.choice([0, 0, 0, 8, 5]))
    if op == "quantize":
        case.update(bits=rng.choice([4, 8]), m=_log(rng, 1, 16384), k=_log(rng, 32, 32768))
    elif op == "act":
        case.update(m=_log(rng, 1, 4096), k=_log(rng, 32, 16384), act=rng.choice(["silu", "gelu"]),
                    gate=rng.random() < 0.5)
    else:
        case.update(m=_log(rng, 1, 8192), k=_log(rng, 64, 8192), n=_log(rng, 64, 8192))
        if rng.random() < 0.5:   # most layers are whole multiples of 64
            case.update(k=(case["k"] + 63) // 64 * 64, n=(case["n"] + 63) // 64 * 64)
        case["m"] = max(1, min(case["m"], MAX_WORK // (case["k"] * case["n"])))
    if op == "mx-linear":
        case["pad"] = 0
    return case


# ---- inputs ----------------------------------------------------------------------------------------------

def _rows(m, k, pad, scale, dtype, gen):
    wide = torch.randn((m, k + pad), dtype=torch.float32, device="cuda", generator=gen).mul_(scale).to(dtype)
    return wide[:, pad // 2:pad // 2 + k]


def _activations(m, k, pad, dtype, gen):
    # Activations of a transformer: near normal, with a few channels tens of times larger.
    x = torch.randn((m, k + pad), dtype=torch.float32, device="cuda", generator=gen)
    loud = torch.randint(0, k + pad, (max(1, k // 500),), device="cuda", generator=gen)
    x[:, loud] *= 30.0
    return x.to(dtype)[:, pad // 2:pad // 2 + k]


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, m, k, n, dt = case["op"], case["m"], case["k"], case.get("n", 0), TYPES[case["type"]]
    pad = case["pad"]
    if op == "quantize":
        return dict(x=_rows(m, k, pad, 0.02, dt, gen) if case["bits"] == 4 else _activations(m, k, pad, dt, gen))
    if op == "act":
        s = dict(x=_rows(m, k, pad, 1.5, dt, gen), dy=_rows(m, k, pad, 0.1, dt, gen))
        s["gate"] = _rows(m, k, pad, 1.0, dt, gen) if case["gate"] else None
        return s
    if op == "weight-grad":
        s = dict(dy=_rows(m, n, pad, 0.1, dt, gen))
        s["codes"], s["scales"] = _quantize(_activations(m, k, 0, torch.bfloat16, gen), 8)
        return s
    w = _rows(n, k, 0, 0.02, torch.bfloat16, gen)
    s = {}
    s["codes"], s["scales"] = _quantize(w, 4)
    if op == "linear":
        s["x"] = _activations(m, k, pad, dt, gen)
    elif op == "mx-linear":
        s["xcodes"], s["xscales"] = _quantize(_activations(m, k, 0, dt, gen), 4)
    else:
        s["dy"] = _rows(m, n, pad, 0.1, dt, gen)
    return s


def prepare(case, seed):
    s = dict(case=case, **_inputs(case, seed))
    if own:
        import paper_2410_15240_amd as F
        kind = F.MX8 if case["op"] == "weight-grad" else F.MX4
        if "codes" in s:
            s["mx"] = kind(s["codes"], s["scales"], case["k"])
        if "xcodes" in s:
            s["mxx"] = kind(s["xcodes"], s["xscales"], case["k"])
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


def _values(codes, scales, k, dtype=torch.float32):
    """The values [m, k] that the codes stand for."""
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
    return (v * s[..., None]).view(m, nb * 32)[:, :k].to(dtype)


def _f(x, act):
    if act == "silu":
        return x / (1 + torch.exp(-x))
    return 0.5 * x * (1 + torch.erf(x * math.sqrt(0.5)))


def _df(x, act):
    if act == "silu":
        s = 1 / (1 + torch.exp(-x))
        return s * (1 + x * (1 - s))
    return 0.5 * (1 + torch.erf(x * math.sqrt(0.5))) + x * torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)


def _plain(s):
    case = s["case"]
    op, k, dt = case["op"], case["k"], TYPES[case["type"]]
    if op == "quantize":
        return _values(*_quantize(s["x"], case["bits"]), k, dt)
    if op == "linear":
        return (s["x"].float() @ _values(s["codes"], s["scales"], k).t()).to(dt)
    if op == "mx-linear":
        return (_values(s["xcodes"], s["xscales"], k) @ _values(s["codes"], s["scales"], k).t()).to(dt)
    if op == "grad-input":
        return (s["dy"].float() @ _values(s["codes"], s["scales"], k)).to(dt)
    if op == "weight-grad":
        return s["dy"].float().t() @ _values(s["codes"], s["scales"], k)
    x, dy = s["x"].float(), s["dy"].float()
    y, xq = _f(x, case["act"]), _values(*_quantize(x, 8), k)
    if s["gate"] is None:
        return y.to(dt), (dy * _df(xq, case["act"])).to(dt)
    g = s["gate"].float()
    gq = _values(*_quantize(g, 8), k)
    return ((y * g).to(dt), (dy * gq * _df(xq, case["act"])).to(dt), (dy * _f(xq, case["act"])).to(dt))


def run(s):
    if not own:
        return _plain(s)
    import paper_2410_15240_amd as F
    case = s["case"]
    op, dt = case["op"], TYPES[case["type"]]
    if op == "quantize":
        if case["bits"] == 4:
            return F.mx4_dequantize(F.mx4_quantize(s["x"]), dtype=dt)
        return F.mx8_dequantize(F.mx8_quantize(s["x"]), dtype=dt)
    if op == "linear":
        return F.mx4_linear(s["x"], s["mx"])
    if op == "mx-linear":
        return F.mx4_linear(s["mxx"], s["mx"], dtype=dt)
    if op == "grad-input":
        return F.mx4_linear_grad_input(s["dy"], s["mx"])
    if op == "weight-grad":
        return F.mx8_weight_grad(s["dy"], s["mx"])
    y, saved, saved_gate = F.mx8_act(s["x"], s["gate"], act=case["act"])
    dx, dgate = F.mx8_act_grad(s["dy"], saved, saved_gate, act=case["act"])
    return (y, dx) if s["gate"] is None else (y, dx, dgate)


# ---- the definition in 64 bits ----------------------------------------------------------------------------

def _exact_blocks(x, bits):
    """Quantised values in 64 bits, straight from the definition: the nearest point of the block's grid."""
    m, k = x.shape
    out = torch.empty((m, k), dtype=torch.float64, device=x.device)
    step = max(1, (1 << 26) // max(k, 1))
    for r in range(0, m, step):                                  # some rows at a time: 64-bit temporaries
        v = torch.nn.functional.pad(x[r:r + step].double(), (0, -k % 32)).view(-1, (k + 31) // 32, 32)
        top = v.abs().amax(dim=2, keepdim=True)
        power = torch.frexp(top)[1].double() - 1                 # floor(log2 top)
        power = torch.where(top == 0, torch.full_like(power, -127.0), power)
        if bits == 8:
            step2 = torch.exp2(power.clamp(min=-127) - 6)
            q = torch.round(v / step2).clamp(-127, 127) * step2
        else:
            unit = torch.exp2((power - 2).clamp(min=-127))
            a = (v / unit).abs()
            octave = torch.floor(torch.log2(a.clamp(min=1.0))).clamp(max=2)
            gap = torch.exp2(octave - 1)
            q = torch.sign(v) * (torch.round(a / gap) * gap).clamp(max=6) * unit
        out[r:r + step] = q.view(-1, q.shape[1] * 32)[:, :k]
    return out


def _exact_values(codes, scales, k):
    s = torch.exp2(scales.double() - 127).repeat_interleave(32, dim=1)
    if codes.dtype == torch.uint8:
        c = torch.stack((codes % 16, codes // 16), dim=2).flatten(1).long()
        mag, sign = c % 8, 1.0 - 2.0 * (c // 8).double()
        v = sign * torch.where(mag < 2, mag * 0.5, (1 + 0.5 * (mag % 2)) * torch.exp2((mag // 2 - 1).double()))
    else:
        v = codes.double() * 2.0 ** -6
    return (v * s)[:, :k]


def exact(case, seed):
    s = _inputs(case, seed)
    op, k = case["op"], case["k"]
    if op == "quantize":
        return _exact_blocks(s["x"], case["bits"])
    if op == "act":
        x, dy = s["x"].double(), s["dy"].double()
        xq = _exact_blocks(s["x"], 8)
        g = None if s["gate"] is None else s["gate"].double()
        gq = 1.0 if g is None else _exact_blocks(s["gate"], 8)

        def value_and_slope(v):
            if case["act"] == "silu":
                p = torch.sigmoid(v)
                return v * p, p + v * p * (1 - p)
            p = 0.5 * torch.erfc(-v / math.sqrt(2.0))
            return v * p, p + v * torch.exp(-v * v / 2) / math.sqrt(2.0 * math.pi)

        fq, dfq = value_and_slope(xq)
        y = value_and_slope(x)[0]
        return (y, dy * dfq) if g is None else (y * g, dy * gq * dfq, dy * fq)
    w = _exact_values(s["codes"], s["scales"], k)
    if op == "linear":
        return torch.matmul(s["x"].double(), w.t().contiguous())
    if op == "mx-linear":
        return torch.matmul(_exact_values(s["xcodes"], s["xscales"], k), w.t().contiguous())
    if op == "grad-input":
        return torch.matmul(s["dy"].double(), w)
    return torch.matmul(s["dy"].double().t().contiguous(), w)


def work(case):
    """Every input read once and every output written once; 2 flops to a multiply-add."""
    op, m, k, n, b = case["op"], case["m"], case["k"], case.get("n", 0), SIZE[case["type"]]
    nb = (k + 31) // 32
    if op == "quantize":   # x in, codes and scales out; values out
        return {"bytes": 2 * m * k * b + m * nb * (17 if case["bits"] == 4 else 33), "flops": 0}
    if op == "act":        # forwards: x, gate in, y and the kept codes out; backwards: dy, codes in, dx, dgate out
        t = 2 if case["gate"] else 1
        return {"bytes": m * k * b * (t + 1) + 2 * t * m * nb * 33 + m * k * b * (t + 1), "flops": 0}
    if op == "linear":
        return {"bytes": n * nb * 17 + (m * k + m * n) * b, "flops": 2 * m * n * k}
    if op == "mx-linear":
        return {"bytes": (n + m) * nb * 17 + m * n * b, "flops": 2 * m * n * k}
    if op == "grad-input":
        return {"bytes": n * nb * 17 + (m * k + m * n) * b, "flops": 2 * m * n * k}
    return {"bytes": m * nb * 33 + m * n * b + n * k * 4, "flops": 2 * m * n * k}
