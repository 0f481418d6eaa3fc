"""What the microscaled calls' binding does with tensors that autograd watches and with outputs that are none."""
import pytest
import torch

import paper_2410_15240_amd as F

pytestmark = pytest.mark.gpu


def test_results_are_not_recorded_by_autograd():
    x, dy = (torch.randn(40, n, device="cuda", requires_grad=True) for n in (64, 96))
    w = torch.randn(96, 64, device="cuda", requires_grad=True)
    qw, kept = F.mx4_quantize(w), F.mx8_quantize(x)
    y, s, sg = F.mx8_act(x, x)
    results = [qw.codes, kept.codes, F.mx4_dequantize(qw), F.mx4_linear(x, qw), F.mx4_linear_grad_input(dy, qw),
               F.mx8_weight_grad(dy, kept), y, s.codes, *F.mx8_act_grad(x, s, sg)]
    assert not any(r.requires_grad for r in results)
    with pytest.raises(RuntimeError, match="does not require grad"):
        F.mx4_linear(x, qw).sum().backward()


class Linear(torch.autograd.Function):
    """The layer as a user joins it: 4-bit weights, an 8-bit checkpoint of the input, a 32-bit weight gradient."""

    @staticmethod
    def forward(ctx, x, w):
        ctx.w, ctx.kept = F.mx4_quantize(w), F.mx8_quantize(x)
        return F.mx4_linear(x, ctx.w)

    @staticmethod
    def backward(ctx, dy):
        return F.mx4_linear_grad_input(dy, ctx.w), F.mx8_weight_grad(dy, ctx.kept)


def test_a_function_of_the_callers_joins_them():
    x, w = torch.randn(40, 64, device="cuda", requires_grad=True), torch.randn(96, 64, device="cuda", requires_grad=True)
    dy = torch.randn(40, 96, device="cuda")
    Linear.apply(x, w).backward(dy)
    q, k = F.mx4_quantize(w), F.mx8_quantize(x)
    assert torch.equal(x.grad, F.mx4_linear_grad_input(dy, q)) and torch.equal(w.grad, F.mx8_weight_grad(dy, k))


@pytest.mark.parametrize("out", [[1.0], "out", 3])
def test_an_output_that_is_no_tensor_is_refused(out):
    x, dy = torch.zeros(4, 64, device="cuda"), torch.zeros(4, 10, device="cuda")
    w, k = F.mx4_quantize(torch.zeros(10, 64, device="cuda")), F.mx8_quantize(x)
    for call in (lambda: F.mx4_dequantize(w, out=out), lambda: F.mx8_dequantize(k, out=out), lambda: F.mx4_linear(x, w, out=out),
                 lambda: F.mx4_linear(F.mx4_quantize(x), w, out=out), lambda: F.mx4_linear_grad_input(dy, w, out=out),
                 lambda: F.mx8_weight_grad(dy, k, out=out), lambda: F.mx8_act(x, out=out), lambda: F.mx8_act_grad(x, k, out=out)):
        with pytest.raises(ValueError, match="out must be a torch tensor"):
            call()
