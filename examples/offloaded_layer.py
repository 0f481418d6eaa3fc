"""One training step of a gated feed-forward layer whose tensors cross the encrypted link in few bits.

    python examples/offloaded_layer.py [--tokens 4096 --width 4096 --hidden 8192]

The owner of the weights quantises them to MX4 and encrypts them; the GPU receives, decrypts and verifies them
chunk by chunk and multiplies with them as they arrived. Between the forward and the backward pass the layer's
inputs and activations, quantised to MX8, are encrypted on the GPU and parked in host memory. Every message has its
own number in the first four bytes of its IV (the chains of a message count in the other eight), since a key must
never meet an IV twice.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2410_15240_amd as F  # noqa: E402

CHAIN = 64 << 10


class Link:
    """Messages between this GPU and host memory that nobody on the way can read or change."""

    def __init__(self, key):
        self.key, self.sent, self.bytes = key, 0, 0
        self.copy, self.work = torch.cuda.Stream(), torch.cuda.Stream()

    def park(self, buf):
        """Encrypt a uint8 device buffer into host memory: (IV, ciphertext, tags), complete on return."""
        iv = self.sent.to_bytes(4, "big") + bytes(8)
        self.sent += 1
        self.bytes += buf.numel()
        self.work.wait_stream(torch.cuda.current_stream())
        ct, tags = F.pipeline_d2h(self.key, iv, CHAIN, buf, copy_stream=self.copy, compute_stream=self.work)
        self.copy.synchronize()
        return iv, ct, tags

    def fetch(self, message):
        """Decrypt and verify a parked message: its bytes in a device buffer, on the current stream."""
        iv, ct, tags = message
        self.bytes += ct.numel()
        buf, ok = F.pipeline_h2d(self.key, iv, CHAIN, ct, tags, copy_stream=self.copy, compute_stream=self.work)
        torch.cuda.current_stream().wait_stream(self.work)
        if not bool(ok.all()):
            raise RuntimeError("%d chains of a message failed verification" % int((ok == 0).sum()))
        return buf


def quantised_message(link, w):
    """Weights as MX4 in one message."""
    buf = torch.empty(F.MX4.nbytes(*w.shape), dtype=torch.uint8, device=w.device)
    F.mx4_quantize(w, out=F.MX4.view(buf, *w.shape))
    return link.park(buf)


def kept(rows, cols, device):
    """A buffer for one message and the MX8 that lives in it."""
    buf = torch.empty(F.MX8.nbytes(rows, cols), dtype=torch.uint8, device=device)
    return buf, F.MX8.view(buf, rows, cols)


def step(link, up_gate, down, x, dy):
    """y = down (silu(a) * b), [a b] = up_gate x, for weights that are messages ((2 hidden, width) and (width,
    hidden)); then the gradients for dy. Returns (y, dx, d_up_gate, d_down)."""
    (m, width), dev = x.shape, x.device
    hidden = up_gate["rows"] // 2
    # forwards
    wu = F.MX4.view(link.fetch(up_gate["message"]), 2 * hidden, width)
    wd = F.MX4.view(link.fetch(down["message"]), width, hidden)
    bx, kx = kept(m, width, dev)
    ba, ka = kept(m, hidden, dev)
    bb, kb = kept(m, hidden, dev)
    bh, kh = kept(m, hidden, dev)
    F.mx8_quantize(x, out=kx)
    ab = F.mx4_linear(x, wu)
    h, _, _ = F.mx8_act(ab[:, :hidden], ab[:, hidden:], saved=ka, saved_gate=kb)
    F.mx8_quantize(h, out=kh)
    y = F.mx4_linear(h, wd)
    parked = [link.park(b) for b in (bx, ba, bb, bh)]
    del bx, kx, ba, ka, bb, kb, bh, kh, ab, h
    # backwards, from what comes back
    kx, ka, kb, kh = (F.MX8.view(link.fetch(p), m, c) for p, c in zip(parked, (width, hidden, hidden, hidden)))
    d_down = F.mx8_weight_grad(dy, kh)
    dab = torch.empty(m, 2 * hidden, dtype=dy.dtype, device=dev)
    F.mx8_act_grad(F.mx4_linear_grad_input(dy, wd), ka, kb, out=dab[:, :hidden], out_gate=dab[:, hidden:])
    return y, F.mx4_linear_grad_input(dab, wu), F.mx8_weight_grad(dab, kx), d_down


def reference(wu, wd, x, dy):
    """The same layer in float32 with its weights as they were quantised."""
    wu, wd, x = wu.float().requires_grad_(), wd.float().requires_grad_(), x.float().requires_grad_()
    a, b = (x @ wu.t()).chunk(2, dim=1)
    y = (torch.nn.functional.silu(a) * b) @ wd.t()
    return (y.detach(),) + torch.autograd.grad(y, (x, wu, wd), dy.float())


def run(tokens, width, hidden, seed=0):
    """Relative errors of y, dx and both weight gradients against float32, and the bytes that crossed."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    draw = lambda *s, scale: torch.randn(*s, device="cuda", generator=gen) * scale
    wu, wd = draw(2 * hidden, width, scale=width ** -0.5), draw(width, hidden, scale=hidden ** -0.5)
    x, dy = draw(tokens, width, scale=1.0).bfloat16(), draw(tokens, width, scale=1.0).bfloat16()
    link = Link(os.urandom(32))
    messages = [dict(message=quantised_message(link, w), rows=w.shape[0]) for w in (wu, wd)]
    got = step(link, *messages, x, dy)
    exact = [F.mx4_dequantize(F.mx4_quantize(w), dtype=torch.float32) for w in (wu, wd)]
    want = reference(*exact, x, dy)
    return [((g.float() - w).norm() / w.norm()).item() for g, w in zip(got, want)], link.bytes


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--width", type=int, default=4096)
    ap.add_argument("--hidden", type=int, default=8192)
    a = ap.parse_args()
    errors, crossed = run(a.tokens, a.width, a.hidden)
    for name, e in zip(("y", "dx", "d_up_gate", "d_down"), errors):
        print("%-10s differs from float32 by %.2e of its norm" % (name, e))
    plain = 2 * 2 * (3 * a.hidden * a.width + a.tokens * (a.width + 3 * a.hidden))
    print("%.1f MB crossed the link, encrypted and verified, where bfloat16 takes %.1f" % (crossed / 1e6, plain / 1e6))


if __name__ == "__main__":
    main()
