"""Which float operands a microscaled product reads in place, by the workspace that it asks for (no GPU needed)."""
import pytest

import paper_2410_15240_amd as F

BF16, FP16, FP32 = range(3)
LINEAR, GRAD_INPUT, WEIGHT_GRAD = range(3)
AT = 0x10000


@pytest.fixture(scope="module")
def work():
    import os
    if not os.path.exists(F.library_path()):
        from paper_2410_15240_amd import build
        build.build()
    return F.lib().fastrack_mx_work_bytes


@pytest.mark.parametrize("op", [LINEAR, GRAD_INPUT])
@pytest.mark.parametrize("address,stride,in_place", [(0, 8192, True), (4, 8192, True), (4, 8194, True), (12, 9000, True),
                                                     (2, 8192, False), (0, 8193, False), (2, 8193, False)])
def test_bf16_is_read_in_place_at_multiples_of_4_bytes(work, op, address, stride, in_place):
    want = 0 if in_place else 2 * 4096 * 8192
    assert work(op, BF16, AT + address, stride, 4096, 8192, 8192) == want
    assert work(op, FP16, AT + address, stride, 4096, 8192, 8192) == 2 * 2 * 4096 * 8192
    assert work(op, FP32, AT + address, stride, 4096, 8192, 8192) == 3 * 2 * 4096 * 8192


def test_a_weight_gradients_operand_has_rows_of_whole_8_values_in_place(work):
    decoded = 2 * 4096 * 8192                       # (the kept input, which many tiles read)
    assert work(WEIGHT_GRAD, BF16, AT + 4, 8192, 4096, 8192, 8192) == decoded
    assert work(WEIGHT_GRAD, BF16, AT, 8192, 4096, 8185, 8192) == decoded + 2 * 4096 * 8192
    assert work(WEIGHT_GRAD, BF16, AT + 2, 8192, 4096, 8192, 8192) == decoded + 2 * 4096 * 8192


@pytest.mark.parametrize("op", [LINEAR, GRAD_INPUT, WEIGHT_GRAD])
@pytest.mark.parametrize("type", [BF16, FP16, FP32])
def test_few_outputs_need_no_workspace(work, op, type):
    for address, stride in ((0, 400), (4, 401), (12, 777)):
        assert work(op, type, AT + address, stride, 20, 300, 400) == 0
