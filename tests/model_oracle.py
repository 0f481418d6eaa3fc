"""The operators around a model's layers from their formulas, in 64 bits (torch, on any device), and how far a computation
in 32 bits may be off them: the tests' oracle.

u below is 2^-24, half a step of a 32-bit float. A sum of terms is off by at most (the number of additions that a term
goes through) u times the sum of the terms' magnitudes.
"""
import torch

U32 = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
# Additions and roundings on a value's way through the sum over a row: 8 of a unit times the units of a thread (8 at most at
# the sizes tested), 6 steps in a wave, 16 waves, and the mean, the root and the quotient after it.
ROW = 96


def half_step(t, v):
    """What rounding v to type t takes off it at most: half a step, of the smallest normal number at least."""
    f = torch.finfo(t)
    return v.abs().clamp(min=f.smallest_normal) * (f.eps / 2)


def kept(x):
    """The values of 8 bits of the rows of x (float64), and the steps between them."""
    m, k = x.shape
    v = torch.nn.functional.pad(x, (0, -k % 32)).view(m, -1, 32)
    top = v.abs().amax(dim=2, keepdim=True)
    e = torch.where(top == 0, torch.full_like(top, -127.0), torch.frexp(top)[1].double() - 1).clamp(min=-127)
    step = torch.exp2(e - 6).expand_as(v)
    q = (torch.round(v / step).clamp(-127, 127) * step)
    return q.reshape(m, -1)[:, :k], step.reshape(m, -1)[:, :k]


def rms(x, eps):
    return (x.square().mean(dim=1) + eps).sqrt()


def norm(x, w2, r, w1, g, scale, eps):
    """y, h, u, 1 / rms(h), v, 1 / rms(x) and for each but the last how far off 32 bits may be."""
    b, v, inv1, rel = x, x, None, 0.0
    if w1 is not None:
        inv1 = 1 / rms(x, eps)
        v = x * inv1[:, None]
        b, rel = v * w1, ROW * U32
    b = b * scale if g is None else b * g * scale
    h = b if r is None else r + b
    off_h = (rel + 4 * U32) * b.abs() + U32 * h.abs()
    inv2 = 1 / rms(h, eps)
    rel2 = ROW * U32 + off_h.square().mean(dim=1).sqrt() * inv2
    u = h * inv2[:, None]
    off_u = off_h * inv2[:, None] + u.abs() * (rel2 + 2 * U32)[:, None]
    return dict(y=u * w2, h=h, u=u, inv2=inv2, v=v, inv1=inv1, off_y=(off_u + 2 * U32 * u.abs()) * w2.abs(), off_h=off_h,
                off_u=off_u, off_inv2=rel2 * inv2, off_v=v.abs() * (rel + 2 * U32))


def norm_grad(dy, w2, u, inv2, dh, w1, v, inv1, g, scale):
    """dx, dr, dg, dw2, dw1 and the bounds, from kept values as they are."""
    m = dy.shape[0]
    def through(d, off, w, n, inv):
        t, off = d * w, off * w.abs() + U32 * (d * w).abs()
        along = (t * n).mean(dim=1, keepdim=True)
        off_along = (off * n.abs()).mean(dim=1, keepdim=True) + ROW * U32 * (t * n).abs().mean(dim=1, keepdim=True)
        out = inv[:, None] * (t - n * along)
        size = inv[:, None] * (t.abs() + n.abs() * along.abs())
        return out, inv[:, None] * (off + n.abs() * off_along) + 4 * U32 * size
    add = lambda t: t.sum(dim=0)
    zero = torch.zeros_like(dy)
    dw2, off_w2 = add(dy * u), (m + 24) * U32 * add((dy * u).abs())
    d, off = through(dy, zero, w2, u, inv2)
    if dh is not None:
        d = d + dh
        off = off + U32 * d.abs()
    res = dict(dr=d, off_dr=off, dw2=dw2, off_dw2=off_w2)
    d, off = d * scale, (off + 2 * U32 * d.abs()) * abs(scale)
    if g is not None:
        b = v if w1 is None else v * w1
        res.update(dg=d * b, off_dg=(off + 3 * U32 * d.abs()) * b.abs())
        d, off = d * g, (off + U32 * d.abs()) * g.abs()
    if w1 is not None:
        res.update(dw1=add(d * v), off_dw1=add(off * v.abs()) + (m + 24) * U32 * add((d * v).abs()))
        d, off = through(d, off, w1, v, inv1)
    res.update(dx=d, off_dx=off)
    return res


def embedding_grad(dy, ids, rows, scale):
    good = (ids >= 0) & (ids < rows)
    dw = torch.zeros(rows, dy.shape[1], dtype=torch.float64, device=dy.device)
    size, count = dw.clone(), torch.zeros(rows, 1, dtype=torch.float64, device=dy.device)
    dw.index_add_(0, ids[good], dy[good] * scale)
    size.index_add_(0, ids[good], dy[good].abs() * abs(scale))
    count.index_add_(0, ids[good], torch.ones_like(dy[good][:, :1]))
    return dw, (count + 4) * U32 * size


def loss(x, w, ids, scale, terms):
    """loss, lse, z and the bounds; terms: bf16 terms of a value of x."""
    m, k = x.shape
    n = w.shape[0]
    wt = w.t().contiguous()
    z = scale * (x @ wt)
    off_z = abs(scale) * (k * terms + 16) * U32 * (x.abs() @ wt.abs()) + 2 * U32 * z.abs()
    lse = torch.logsumexp(z, dim=1)
    far = (z - z.amax(dim=1, keepdim=True)).abs().amax(dim=1)
    # e^(z - top): the difference's rounding and the exponential's two units; then the joining of parts (each scales a
    # sum by an exponential) and the logarithm.
    off_lse = off_z.amax(dim=1) + U32 * (far + 64 + 2 * lse.abs())
    rows = torch.arange(m, device=x.device)
    at = ids.clamp(0, n - 1)
    good = ids >= 0
    out = torch.where(good, lse - z[rows, at], 0.0)
    off = torch.where(good, off_lse + off_z[rows, at] + U32 * out.abs(), 0.0)
    return dict(loss=out, lse=lse, z=z, off_loss=off, off_lse=off_lse, off_z=off_z)


def loss_grad(x, w, ids, dloss, scale, terms, x8, dx_type, dw_type):
    m, k = x.shape
    n = w.shape[0]
    f = loss(x, w, ids, scale, terms)
    z, lse = f["z"], f["lse"]
    p = torch.exp(z - lse[:, None])
    factor = torch.where(ids >= 0, dloss * scale, 0.0)[:, None]
    off_p = p * (f["off_z"] + f["off_lse"][:, None] + U32 * (2 * (z - lse[:, None]).abs() + 4))
    one = torch.zeros_like(p)
    rows = torch.arange(m, device=x.device)[ids >= 0]
    one[rows, ids[ids >= 0]] = 1.0
    dz = factor * (p - one)
    # (The factor's product, its common part divided out and multiplied in again, the difference's product.)
    off_dz = factor.abs() * off_p + 8 * U32 * dz.abs()
    res = {}
    for name, a, b, t, sums in (("dx", dz, w, dx_type, n), ("dw", dz.t().contiguous(), x8, dw_type, m)):
        off = off_dz if name == "dx" else off_dz.t().contiguous()
        if t == torch.bfloat16:   # dz rounded once
            off = off + half_step(torch.bfloat16, a)
        # (an fp16 gradient's two terms leave 2^-16 of a value)
        off = off + (2.0 ** -16 * a.abs() if t == torch.float16 else 0.0)
        res[name] = a @ b
        res["off_" + name] = off @ b.abs() + (3 * sums + 32) * U32 * (a.abs() @ b.abs())
    return res
