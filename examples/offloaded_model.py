"""One training step of a small language model whose tensors cross the encrypted link in few bits.

    python examples/offloaded_model.py [--tokens 4096 --width 2048 --hidden 4096 --vocabulary 32768 --layers 2]

The token table, which is the head too, and the layers' weights arrive as MX4 messages and are used as they are. What the
backward pass needs of the norms and of the layers is kept as MX8, parked in host memory, encrypted, while the rest of the
step runs, and comes back in the order in which it is needed. See offloaded_layer.py for the link and its messages.
"""
import argparse
import importlib.util
import math
import os
import sys

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, os.path.dirname(HERE))
import paper_2410_15240_amd as F  # noqa: E402

_spec = importlib.util.spec_from_file_location("offloaded_layer", os.path.join(HERE, "offloaded_layer.py"))
layer = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(layer)

BRANCH = 0.5   # the residual scale


def receive(link, sent):
    """A message of weights as the MX4 that it is."""
    message, rows, cols = sent
    return F.MX4.view(link.fetch(message), rows, cols)


class Parked:
    """8-bit checkpoints in host memory."""

    def __init__(self, link):
        self.link, self.sent = link, []

    def new(self, rows, cols):
        """An MX8 to be written, and parked by park()."""
        buf, q = layer.kept(rows, cols, torch.device("cuda"))
        self.sent.append([buf, rows, cols])
        return q

    def park(self):
        for s in self.sent:
            if isinstance(s[0], torch.Tensor):
                s[0] = self.link.park(s[0])

    def back(self):
        """The last one parked that is not back yet."""
        message, rows, cols = self.sent.pop()
        return F.MX8.view(self.link.fetch(message), rows, cols)


def forward_layer(x, up_gate, down, parked):
    """down (silu(a) * b), [a b] = up_gate x."""
    m, width = x.shape
    hidden = down.cols
    kx, ka, kb, kh = (parked.new(m, c) for c in (width, hidden, hidden, hidden))
    F.mx8_quantize(x, out=kx)
    ab = F.mx4_linear(x, up_gate)
    h, _, _ = F.mx8_act(ab[:, :hidden], ab[:, hidden:], saved=ka, saved_gate=kb)
    F.mx8_quantize(h, out=kh)
    return F.mx4_linear(h, down)


def backward_layer(dy, up_gate, down, parked):
    """(dx, gradients of up_gate and down)."""
    kh, kb, ka, kx = (parked.back() for _ in range(4))
    dab = torch.empty(dy.shape[0], 2 * down.cols, dtype=dy.dtype, device=dy.device)
    F.mx8_act_grad(F.mx4_linear_grad_input(dy, down), ka, kb, out=dab[:, :down.cols], out_gate=dab[:, down.cols:])
    return F.mx4_linear_grad_input(dab, up_gate), F.mx8_weight_grad(dab, kx), F.mx8_weight_grad(dy, kh)


def step(link, table, layers, norms, posts, ids, targets):
    """The mean loss of predicting `targets` after `ids` and all gradients: of the table, of each layer's weights, of the norms'
    (one before each layer and one before the head) and of the layers' own norms'."""
    m, dev, parked = ids.numel(), ids.device, Parked(link)
    width = table[2]
    scale = math.sqrt(width)

    def saved(post):
        normed = parked.new(m, width)
        block = parked.new(m, width) if post else None
        floats = lambda: torch.empty(m, dtype=torch.float32, device=dev)
        return F.NormSaved(normed, floats(), block, floats() if post else None)

    # forwards
    head = receive(link, table)
    h = F.mx4_embedding(ids, head, scale=scale)
    kept = [saved(False)]
    x, _, _ = F.mx8_norm(h, norms[0], saved=kept[0])
    weights = []
    for (up_gate, down), weight, post in zip(layers, norms[1:], posts):
        weights.append((receive(link, up_gate), receive(link, down)))
        y = forward_layer(x, *weights[-1], parked)
        kept.append(saved(True))
        x, h, _ = F.mx8_norm(y, weight, residual=h, post_weight=post, scale=BRANCH, saved=kept[-1])
        parked.park()
    loss, lse = F.mx4_cross_entropy(x, head, targets)
    count = (targets >= 0).sum().clamp(min=1)
    mean = loss.sum() / count
    x8 = F.mx8_quantize(x)
    # backwards
    dx, dtable = F.mx4_cross_entropy_grad((1.0 / count).expand(m), x, head, targets, lse, saved=x8)
    dh, dlayers, dnorms, dposts = None, [], [], []
    for (up_gate, down), weight, post, k in reversed(list(zip(weights, norms[1:], posts, kept[1:]))):
        block, normed = parked.back(), parked.back()
        k = F.NormSaved(normed, k.inverse, block, k.block_inverse)
        dy, dh, _, dw, dp = F.mx8_norm_grad(dx, weight, k, dhidden=dh, post_weight=post, scale=BRANCH)
        dx, dup, ddown = backward_layer(dy, up_gate, down, parked)
        dlayers.insert(0, (dup, ddown))
        dnorms.insert(0, dw)
        dposts.insert(0, dp)
    dh, _, _, dw, _ = F.mx8_norm_grad(dx, norms[0], F.NormSaved(parked.back(), kept[0].inverse), dhidden=dh, residual=False)
    F.mx4_embedding_grad(dh, ids, table[1], scale=scale, out=dtable, accumulate=True)
    return mean, dtable, dlayers, [dw] + dnorms, dposts


def reference(table, layers, norms, posts, ids, targets):
    """The same step in float32 with the weights as they were quantised."""
    leaf = lambda t: t.float().requires_grad_()
    table, norms, posts, layers = leaf(table), [leaf(w) for w in norms], [leaf(w) for w in posts], [(leaf(u), leaf(d)) for u, d in layers]
    rms = lambda x: x / (x.square().mean(dim=1, keepdim=True) + 1e-6).sqrt()
    h = torch.where(ids[:, None] < 0, 0.0, table[ids.clamp(min=0)] * math.sqrt(table.shape[1]))
    x = rms(h) * norms[0]
    for (up_gate, down), weight, post in zip(layers, norms[1:], posts):
        a, b = (x @ up_gate.t()).chunk(2, dim=1)
        h = h + BRANCH * rms((torch.nn.functional.silu(a) * b) @ down.t()) * post
        x = rms(h) * weight
    loss = torch.nn.functional.cross_entropy(x @ table.t(), torch.where(targets < 0, -1, targets), ignore_index=-1)
    flat = [t for pair in layers for t in pair]
    grads = torch.autograd.grad(loss, [table] + flat + norms + posts)
    n, k = len(layers), len(norms)
    g = grads[1:1 + 2 * n]
    return loss.detach(), grads[0], list(zip(g[::2], g[1::2])), list(grads[1 + 2 * n:1 + 2 * n + k]), list(grads[1 + 2 * n + k:])


def run(tokens, width, hidden, vocabulary, depth, seed=0):
    """(the loss, the reference's, relative errors of the gradients, bytes that crossed)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    draw = lambda *s, scale: torch.randn(*s, device="cuda", generator=gen) * scale
    near1 = lambda: (1 + draw(width, scale=0.1)).bfloat16()
    table = draw(vocabulary, width, scale=width ** -0.5)
    layers = [(draw(2 * hidden, width, scale=width ** -0.5), draw(width, hidden, scale=hidden ** -0.5)) for _ in range(depth)]
    norms, posts = [near1() for _ in range(depth + 1)], [near1() for _ in range(depth)]
    ids = torch.randint(0, vocabulary, (tokens,), device="cuda", generator=gen)
    ids[tokens - tokens // 8:] = -1   # a padded batch
    targets = torch.where(ids < 0, ids, ids.roll(-1).clamp(min=0))
    link = layer.Link(os.urandom(32))
    send = lambda w: (layer.quantised_message(link, w),) + tuple(w.shape)
    got = step(link, send(table), [(send(u), send(d)) for u, d in layers], norms, posts, ids, targets)
    whole = lambda w: F.mx4_dequantize(F.mx4_quantize(w), dtype=torch.float32)
    want = reference(whole(table), [(whole(u), whole(d)) for u, d in layers], norms, posts, ids, targets)
    far = lambda g, w: ((g.float() - w).norm() / w.norm()).item()
    errors = {"table": far(got[1], want[1])}
    for i in range(depth):
        errors["up_gate %d" % i], errors["down %d" % i] = (far(g, w) for g, w in zip(got[2][i], want[2][i]))
        errors["post %d" % i] = far(got[4][i], want[4][i])
    for i in range(depth + 1):
        errors["norm %d" % i] = far(got[3][i], want[3][i])
    return got[0].item(), want[0].item(), errors, link.bytes


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--width", type=int, default=2048)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--vocabulary", type=int, default=32768)
    ap.add_argument("--layers", type=int, default=2)
    a = ap.parse_args()
    loss, want, errors, crossed = run(a.tokens, a.width, a.hidden, a.vocabulary, a.layers)
    print("loss %.4f (float32: %.4f)" % (loss, want))
    for name, e in errors.items():
        print("gradient of %-10s differs from float32 by %.2e of its norm" % (name, e))
    print("%.1f MB crossed the link, encrypted and verified" % (crossed / 1e6))


if __name__ == "__main__":
    main()
